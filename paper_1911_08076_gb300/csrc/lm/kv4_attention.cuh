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

}  // namespace ifq
