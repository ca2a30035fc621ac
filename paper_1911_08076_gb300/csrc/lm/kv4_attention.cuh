// Attention over the paged 4-bit cache (kv4.cuh).
//
// For a query row q at position p and the tokens j it sees, with K_j = s_j c_j + m_j (codes c_j, one scale s_j and
// minimum m_j per token and head) and V_j = s'_j c'_j + m'_j:
//   t_j = scale (s_j (q . c_j) + m_j sum(q)),
//   out = sum_j p_j V_j / sum_j p_j = (sum_j (p_j s'_j) c'_j + sum_j p_j m'_j) / sum_j p_j,  p_j = exp(t_j - max t).
#pragma once
#include "kv4.cuh"

namespace ifq {

struct KvAttnArgs {
  const uint16_t* q;
  const uint8_t* cache;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* starts;   // or nullptr: one query a sequence
  uint16_t* out;
  float* lse;              // or nullptr
  long long q_stride, out_stride;
  int pages, page_size, kv_heads;
  int seqs, q_tokens, max_q, max_pages, q_heads, group;   // group: query heads per key head
  int window, sinks;
  float scale;
};

struct KvSeq {
  int first, n, len;   // first query row, queries, tokens
  bool ok;
};
__device__ __forceinline__ KvSeq kv_seq(const KvAttnArgs& a, int s) {
  KvSeq r;
  r.first = a.starts ? a.starts[s] : s;
  const int end = a.starts ? a.starts[s + 1] : s + 1;
  r.n = end - r.first;
  r.len = a.lens[s];
  r.ok = r.first >= 0 && end >= r.first && end <= a.q_tokens && r.n <= a.max_q && r.len >= 0 &&
         r.len <= (long long)a.max_pages * a.page_size;
  return r;
}
__device__ __forceinline__ bool kv_sees(const KvAttnArgs& a, int p, int j) {
  return j <= p && (a.window == 0 || j > p - a.window || j < a.sinks);
}

constexpr int kAttnWarps = 8;

// One warp a query row and head, keys one after another.
template <int D, bool BF>
__global__ void __launch_bounds__(32 * kAttnWarps) kv4_attention_kernel(const KvAttnArgs a) {
  constexpr int E = D / 32;
  grid_dep_wait();
  const long long item = (long long)blockIdx.x * kAttnWarps + (threadIdx.x >> 5);
  if (item >= (long long)a.q_tokens * a.q_heads) return;
  const int lane = threadIdx.x & 31, d0 = lane * E;
  const int t = (int)(item / a.q_heads), h = (int)(item - (long long)t * a.q_heads), hk = h / a.group;
  int s = t;
  if (a.starts) {   // the last sequence that starts at or before t
    int lo = 0, hi = a.seqs;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.starts[mid] <= t) lo = mid;
      else hi = mid;
    }
    s = lo;
  }
  const KvSeq q = kv_seq(a, s);
  if (!q.ok || t < q.first || t >= q.first + q.n) {
    if (lane == 0 && !q.ok) set_status(IFQ_ERANGE);
    return;
  }
  float x[E], o[E];
  uint32_t w[E / 2];
  load_words(w, a.q + t * a.q_stride + (long long)h * D + d0);
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const float2 f = unpack16<BF>(w[i / 2]);
    x[i] = i % 2 ? f.y : f.x;
    sum += x[i];
    o[i] = 0.0f;
  }
#pragma unroll
  for (int m = 16; m; m >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
  const int p = q.len - q.n + (t - q.first);
  float top = -INFINITY, total = 0.0f;
  for (int j = 0; j <= p; ++j) {
    if (!kv_sees(a, p, j)) continue;
    const int page = a.table[(long long)s * a.max_pages + j / a.page_size];
    if (page < 0 || page >= a.pages) {
      if (lane == 0) set_status(IFQ_ERANGE);
      continue;
    }
    const int in = j % a.page_size, row = in % kKvGroup;
    const uint8_t* g = a.cache + (((long long)page * a.kv_heads + hk) * (a.page_size / kKvGroup) + in / kKvGroup) *
                                     kv4_group_bytes(D);
    const float2 kp = __half22float2(*(const __half2*)(g + 16 * D + 4 * row));
    const float2 vp = __half22float2(*(const __half2*)(g + 16 * D + 64 + 4 * row));
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < E; i += 2) {
      const uint32_t b = g[kv4_k_byte(D, row, d0 + i)];
      dot += x[i] * (float)(b & 15u) + x[i + 1] * (float)(b >> 4);
    }
#pragma unroll
    for (int m = 16; m; m >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, m);
    const float score = a.scale * (kp.x * dot + kp.y * sum);
    const float now = fmaxf(top, score);
    const float keep = top == -INFINITY ? 0.0f : __expf(top - now), e = __expf(score - now);
    top = now;
    total = total * keep + e;
#pragma unroll
    for (int i = 0; i < E; i += 2) {
      const uint32_t b = g[kv4_v_byte(D, row, d0 + i)];
      o[i] = o[i] * keep + e * (vp.x * (float)(b & 15u) + vp.y);
      o[i + 1] = o[i + 1] * keep + e * (vp.x * (float)(b >> 4) + vp.y);
    }
  }
  const float inv = top == -INFINITY ? 0.0f : 1.0f / total;
#pragma unroll
  for (int i = 0; i < E / 2; ++i) w[i] = pack16<BF>(o[2 * i] * inv, o[2 * i + 1] * inv);
  store_words(a.out + t * a.out_stride + (long long)h * D + d0, w);
  if (a.lse && lane == 0) a.lse[(long long)t * a.q_heads + h] = top == -INFINITY ? -INFINITY : top + logf(total);
}

}  // namespace ifq
