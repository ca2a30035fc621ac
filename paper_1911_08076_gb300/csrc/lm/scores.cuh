// Scores of tokens: log probabilities, log-sum-exp, entropy and the likeliest tokens of rows of logits.
//
// 97 us, 5.5 TB/s (82 % of a copy) for 2048 x 131072 in bfloat16 with 8 tokens, 88 without; one row takes 6.7 us, 13 000 cycles of steps that
// wait for each other.
//
// One pass over a row: a thread keeps its largest logit, the sum of e^(z - that) and the sum of e^(z - that) (z - that), and
// brings both sums to a new reference once for every four loads of 16 bytes.  Reading the row bounds it; a row may be
// split over a cluster of blocks, whose sums and lists the first one joins, where there are few.
//
// The likeliest tokens: if k of the block's 64 groups of threads have a logit of at least T, so have the k likeliest tokens.
// T is the k-th of the groups' maxima (some 44 of random logits reach it for k = 32); the few threads that reach it have
// their logits read again (from L2), by all threads, and what is at least T is put in a list, from which the k first are
// taken by counting.  A row with more logits at T than the list holds (many equals) is gone through once for each of the k.
#pragma once
#include <type_traits>

#include "kv4.cuh"

namespace ifq {

constexpr int kTopMax = 32;

struct ScoresArgs {
  const void* logits;
  const int64_t* tokens;
  float *logprobs, *lse, *entropy, *top_logprobs;
  int64_t* top_ids;
  long long stride;
  int rows, vocab, top;
  int parts;            // blocks (of a cluster) a row
  float scale, c;       // c = 2 scale / ln 2
};

template <int TYPE>
__device__ __forceinline__ float logit_at(const void* p, long long at) {
  if constexpr (TYPE == IFQ_F32) return ((const float*)p)[at];
  else if constexpr (TYPE == IFQ_F16) return __half2float(((const __half*)p)[at]);
  else return __bfloat162float(((const __nv_bfloat16*)p)[at]);
}

// A number that orders (logit, token) pairs as the top tokens are: larger logits first (NaN before all, -0 as 0), of
// equals the lower token.  0 is below every pair, ~0 above.
__device__ __forceinline__ uint64_t top_key(float v, int token) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  const uint32_t k = v != v ? 0xffc00000u : (int)b < 0 ? ~b : b | 0x80000000u;
  return (uint64_t)k << 32 | (uint32_t)~token;
}
__device__ __forceinline__ int key_token(uint64_t k) { return (int)~(uint32_t)k; }
__device__ __forceinline__ float key_logit(uint64_t k) {
  const uint32_t u = (uint32_t)(k >> 32);
  return __uint_as_float((int)u < 0 ? u & 0x7fffffffu : ~u);   // (a NaN's key gives a NaN)
}


constexpr int kScoreThreads = 512, kScoreList = 1024, kScoreDeep = 4;

// A row's sums are relative to its largest logit: of 2^d with d = (x - top) scale / ln 2, and of 2^d d.  The difference
// is taken before the product, so that large logits cost no digits, and of halves, x / 2 - top / 2 with one rounding, which no
// two floats take past the type's end; c = 2 scale / ln 2.
struct RowSums {
  float top;        // NaN where there is one, -infinity before any
  float sum, weighted;
};
__device__ __forceinline__ float exp2_of(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void move_to(RowSums& r, float top, float c) {
  const float d = fmaxf(fmaf(r.top, 0.5f, -0.5f * top) * c, -1000.0f), f = exp2_of(d);
  r.weighted = f * fmaf(r.sum, d, r.weighted);
  r.sum *= f;
  r.top = top;
}
// Two floats in one register pair, and operations on both.
__device__ __forceinline__ uint64_t two(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 apart(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// The larger of two logits each of a word, a NaN where there is one.
template <bool BF>
__device__ __forceinline__ uint32_t max16_nan(uint32_t a, uint32_t b) {
  uint32_t r;
  if constexpr (BF) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// 16 bytes of a row as logits.
template <int TYPE, int N>
__device__ __forceinline__ void unpack_logits(const uint32_t (&w)[4], float (&x)[N]) {
  if constexpr (TYPE == IFQ_F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = unpack16<TYPE == IFQ_BF16>(w[i]);
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
}

constexpr int kScoreGroups = 64, kScoreParts = 8;

__device__ __forceinline__ RowSums join_lanes(RowSums r, float c, int lanes) {   // over groups of `lanes`
  float top = r.top;
  for (int o = lanes / 2; o; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
  move_to(r, top, c);
  for (int o = lanes / 2; o; o >>= 1) {
    r.sum += __shfl_xor_sync(0xffffffffu, r.sum, o);
    r.weighted += __shfl_xor_sync(0xffffffffu, r.weighted, o);
  }
  return r;
}
// How many of n keys are above k.
__device__ __forceinline__ int keys_above(const uint64_t* keys, int n, uint64_t k) {
  int above = 0;
#pragma unroll 8
  for (int j = 0; j < n; ++j) above += keys[j] > k;
  return above;
}

// BLOCKS an SM: three hide each other's selections where rows are many (2048 x 131072: 115 -> 103 us), two leave more
// registers where few blocks run.
template <int TYPE, int BLOCKS>
__global__ void __launch_bounds__(kScoreThreads, BLOCKS) token_scores_kernel(const __grid_constant__ ScoresArgs a) {
  constexpr int SIZE = TYPE == IFQ_F32 ? 4 : 2, N = 16 / SIZE, U = kScoreDeep;
  __shared__ RowSums warp_sums[kScoreThreads / 32], part_sums[kScoreParts];   // (of the first block: all parts')
  // The parts' first ones, and what comes of them.  From the moment this block has started the other blocks may write to the first
  // one's part_sums[1] and part_best[top] and on: a block itself writes below those only.
  __shared__ uint64_t part_best[kScoreParts * kTopMax], best[kTopMax];
  __shared__ __align__(16) uint64_t list[kScoreList];
  __shared__ uint16_t who[kScoreThreads];
  __shared__ __align__(16) uint32_t group_top[kScoreGroups];
  __shared__ uint32_t reach;
  __shared__ int count, threads;
  const int tid = threadIdx.x, T = blockDim.x, warp = tid / 32, lane = tid % 32, warps = T / 32;
  const int parts = a.parts, rank = parts > 1 ? (int)cluster_ctarank() : 0;
  const long long row = parts == 1 ? blockIdx.x : blockIdx.x / (uint32_t)parts;
  const float c = a.c;
  if (parts > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // (this block's memory is there)
  grid_dep_wait();
  grid_dep_launch();

  // 16-byte pieces of the row, aligned, and this block's: piece i holds logits i * N - skip and on
  const uint8_t* begin = (const uint8_t*)a.logits + row * a.stride * SIZE;
  const int skip = (int)(((uintptr_t)begin & 15) / SIZE);
  const uint8_t* p = begin - skip * SIZE;
  // (32-bit divisions, and none where a row is whole: pieces are below 2^29 and parts 8 at most)
  const uint32_t pieces = ((uint32_t)a.vocab + skip + N - 1) / N;
  const int lo = parts == 1 ? 0 : pieces * rank / (uint32_t)parts, hi = parts == 1 ? pieces : pieces * (rank + 1) / (uint32_t)parts;
  const int whole_lo = skip ? 1 : 0, whole_hi = (int)(((uint32_t)a.vocab + skip) / N);   // pieces that are all logits
  auto load = [&](int i, uint32_t (&w)[4]) {
    if (i >= whole_lo && i < whole_hi) {
      load_words(w, p + 16ll * i);
      return;
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {   // a row's ends
      const long long e = (long long)i * N - skip + j;
      const bool in = i < hi && e >= 0 && e < a.vocab;
      if constexpr (SIZE == 4) w[j] = in ? ((const uint32_t*)begin)[e] : 0xff800000u;
      else {
        const uint32_t v = in ? ((const uint16_t*)begin)[e] : TYPE == IFQ_BF16 ? 0xff80u : 0xfc00u;
        w[j / 2] = j & 1 ? w[j / 2] | v << 16 : v;
      }
    }
  };

  // the given token's logit, on its way meanwhile
  long long token = -1;
  float given = 0.0f;
  if (tid == 0 && rank == 0 && a.logprobs) {
    token = a.tokens[row];
    if (token >= 0 && token < a.vocab) given = logit_at<TYPE>(begin, token);
  }
  RowSums r = {-INFINITY, 0.0f, 0.0f};
  const uint64_t c2 = two(c, c);
  auto add = [&](auto& w) {   // [pieces][4 words]
    constexpr int V = sizeof(w) / 16;
    float top = r.top;
    if constexpr (SIZE == 4) {
#pragma unroll
      for (int u = 0; u < V; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) top = max_nan(top, __uint_as_float(w[u][j]));
    } else {   // two at a time
      uint32_t m = w[0][0];
#pragma unroll
      for (int u = 0; u < V; ++u)
#pragma unroll
        for (int j = u == 0; j < 4; ++j) m = max16_nan<TYPE == IFQ_BF16>(m, w[u][j]);
      const float2 f = unpack16<TYPE == IFQ_BF16>(m);
      top = max_nan(top, max_nan(f.x, f.y));
    }
    if (top != r.top) move_to(r, top, c);
    if (top == -INFINITY) return;
    const uint64_t half = two(0.5f, 0.5f), down = two(-0.5f * top, -0.5f * top);
    uint64_t sum = two(r.sum, 0.0f), weighted = two(r.weighted, 0.0f);
#pragma unroll
    for (int u = 0; u < V; ++u) {
      float x[N];
      unpack_logits<TYPE>(w[u], x);
#pragma unroll
      for (int j = 0; j < N; j += 2) {
        // (at least -1000: a masked logit's share of 0 times its distance, -infinity, would be no number)
        float2 d = apart(mul2(fma2(two(x[j], x[j + 1]), half, down), c2));
        d.x = fmaxf(d.x, -1000.0f);
        d.y = fmaxf(d.y, -1000.0f);
        const uint64_t e = two(exp2_of(d.x), exp2_of(d.y));
        sum = add2(sum, e);
        weighted = fma2(e, two(d.x, d.y), weighted);
      }
    }
    const float2 s = apart(sum), v = apart(weighted);
    r.sum = s.x + s.y;
    r.weighted = v.x + v.y;
  };
  {
    // pieces lo + tid, lo + tid + T, ...: those that are all logits four at a time, a row's ends by themselves
    int i = lo + tid;
    const int full = min(hi, whole_hi);
    uint32_t one[1][4];
    if (i < whole_lo) {
      load(i, one[0]);
      add(one);
      i += T;
    }
    const uint8_t* q = p + 16ll * i;
    const long long ahead = 16ll * T;
    for (; i < full - (U - 1) * T; i += U * T, q += U * ahead) {
      uint32_t w[U][4];
#pragma unroll
      for (int u = 0; u < U; ++u) load_words(w[u], q + u * ahead);
      add(w);
    }
    if (i < full) {   // the last ones, under way together too
      uint32_t w[U][4];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        w[u][0] = w[u][1] = w[u][2] = w[u][3] = TYPE == IFQ_F32 ? 0xff800000u : TYPE == IFQ_BF16 ? 0xff80ff80u : 0xfc00fc00u;
        if (i + u * T < full) load_words(w[u], q + u * ahead);
      }
      add(w);
      i += (full - i + T - 1) & -T;
    }
    if (i < hi) {
      load(i, one[0]);
      add(one);
    }
  }
  const uint32_t mine = lo + tid < hi ? (uint32_t)(top_key(r.top, 0) >> 32) : 0u;   // 0: no logits
  r = join_lanes(r, c, 32);
  if (lane == 0) warp_sums[warp] = r;
  if (a.top) {
    const int per = T / kScoreGroups;   // threads a group: 1, 2, 4 or 8
    uint32_t most = mine;
    for (int o = per / 2; o; o >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
    if (tid % per == 0) group_top[tid / per] = most;
    if (tid == 0) count = threads = 0;
    if (tid < a.top) part_best[tid] = best[tid] = 0;
  }
  __syncthreads();
  if (warp == 0) {
    r = lane < warps ? warp_sums[lane] : RowSums{-INFINITY, 0.0f, 0.0f};
    r = join_lanes(r, c, 16);
    if (lane == 0) part_sums[0] = r;
  }
  if (a.top) {
    const int id = tid - (T - kScoreGroups);   // (the last two warps')
    if (id >= 0) {
      const uint32_t v = group_top[id];
      int before = 0;
#pragma unroll
      for (int j = 0; j < kScoreGroups; j += 4) {
        const uint4 q = *(const uint4*)&group_top[j];
        before += (q.x > v || (q.x == v && j < id)) + (q.y > v || (q.y == v && j + 1 < id)) +
                  (q.z > v || (q.z == v && j + 2 < id)) + (q.w > v || (q.w == v && j + 3 < id));
      }
      if (before == a.top - 1) reach = v;
    }
    __syncthreads();
    const uint32_t t = reach;   // 0 (all logits) where fewer than k groups have any
    if (mine != 0 && mine >= t) who[atomicAdd(&threads, 1)] = (uint16_t)tid;
    __syncthreads();
    // what pass() takes of piece `at` goes to the list
    auto gather = [&](int at, auto&& pass) {
      uint32_t w[4];
      load(at, w);
      float x[N];
      unpack_logits<TYPE>(w, x);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const long long e = (long long)at * N - skip + j;
        const uint64_t k = top_key(x[j], (int)e);
        if (pass((uint32_t)(k >> 32)) && e >= 0 && e < a.vocab) {
          const int to = atomicAdd(&count, 1);
          if (to < kScoreList) list[to] = k;
        }
      }
    };
    // those threads' pieces, spread over all threads
    auto gather_all = [&](auto&& pass) {
      const int each = (hi - lo + T - 1) >> (31 - __clz(T)), all = threads * each;   // (T is a power of two)
      for (int i = tid; i < all; i += T) {
        const int q = i / each, at = lo + who[q] + (i - q * each) * T;
        if (*(volatile int*)&count > kScoreList) break;   // (too many)
        if (at < hi) gather(at, pass);
      }
    };
    gather_all([&](uint32_t k) { return k >= t; });
    __syncthreads();
    if (count > kScoreList) {
      // Many equals (a mask that leaves fewer than k, a constant row): those above them, and of the equals the first that
      // are found going through the row from its start, 512 logits or fewer at a time.
      __syncthreads();
      if (tid == 0) count = threads = 0;
      __syncthreads();
      if (mine > t) who[atomicAdd(&threads, 1)] = (uint16_t)tid;
      __syncthreads();
      gather_all([&](uint32_t k) { return k > t; });
      __syncthreads();
      const int above = count;
      int now = above;
      __syncthreads();
      for (int i = lo; i < hi && now < above + a.top && now <= kScoreList - 512; i += 64) {
        if (tid < 64 && i + tid < hi) gather(i + tid, [&](uint32_t k) { return k == t; });
        __syncthreads();
        now = count;
        __syncthreads();
      }
      if (now > kScoreList - 512 && now < above + a.top && tid == 0) count = kScoreList + 1;   // (too many above them)
    }
    __syncthreads();
    const int n = count;
    if (n <= kScoreList) {
      for (int i = tid; i < n; i += T) {
        const uint64_t k = list[i];
        const int before = keys_above(list, n, k);
        if (before < a.top) part_best[before] = k;
      }
    } else {
      uint64_t last = ~0ull;
      for (int j = 0; j < a.top; ++j) {
        uint64_t k = 0;
        for (int i = lo + tid; i < hi; i += T) {
          uint32_t w[4];
          load(i, w);
          float x[N];
          unpack_logits<TYPE>(w, x);
#pragma unroll
          for (int q = 0; q < N; ++q) {
            const long long e = (long long)i * N - skip + q;
            const uint64_t v = top_key(x[q], (int)e);
            if (v < last && v > k && e >= 0 && e < a.vocab) k = v;
          }
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) k = max(k, __shfl_xor_sync(0xffffffffu, k, o));
        if (lane == 0) list[warp] = k;
        __syncthreads();
        for (int i = 0; i < warps; ++i) k = max(k, list[i]);
        if (tid == 0) part_best[j] = k;
        last = k;
        __syncthreads();
      }
    }
  }
  __syncthreads();

  // the parts' results meet in the first block
  const uint64_t* tops = part_best;
  if (parts > 1) {
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (rank) {
      if (tid < a.top)
        asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(mapa_shared(smem_u32(&part_best[rank * a.top + tid]), 0)), "l"(part_best[tid])
                     : "memory");
      if (tid < 3)
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(mapa_shared(smem_u32(&part_sums[rank]) + 4 * tid, 0)),
                     "f"(((const float*)&part_sums[0])[tid])
                     : "memory");
    }
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    if (rank) return;
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (warp == 0) {
      r = lane < parts ? part_sums[lane] : RowSums{-INFINITY, 0.0f, 0.0f};
      r = join_lanes(r, c, kScoreParts);
      __syncwarp();
      if (lane == 0) part_sums[0] = r;
    }
    for (int i = tid; i < parts * a.top; i += T) {
      const uint64_t k = part_best[i];
      const int before = keys_above(part_best, parts * a.top, k);
      if (k && before < a.top) best[before] = k;
    }
    __syncthreads();
    tops = best;
  }

  r = part_sums[0];
  const float log2_sum = log2f(r.sum), log_sum = 0.69314718055994531f * log2_sum;
  auto logprob = [&](float x) {
    return r.top == -INFINITY ? r.top : fmaf(x, 0.5f, -0.5f * r.top) * (2.0f * a.scale) - (r.top == INFINITY ? 0.0f : log_sum);
  };
  if (tid == 0) {
    if (a.lse) a.lse[row] = fabsf(r.top) == INFINITY ? r.top : fmaf(r.top, a.scale, log_sum);
    if (a.entropy)
      a.entropy[row] = r.top == -INFINITY ? 0.0f : r.top == INFINITY || r.top != r.top ? NAN
                                                     : 0.69314718055994531f * (log2_sum - __fdividef(r.weighted, r.sum));
    if (a.logprobs) {
      if (token >= a.vocab) set_status(IFQ_ERANGE);
      a.logprobs[row] = token < 0 ? 0.0f : token >= a.vocab ? NAN : logprob(given);
    }
  }
  if (tid < a.top) {
    const uint64_t k = tops[tid];
    if (a.top_ids) a.top_ids[row * a.top + tid] = key_token(k);
    if (a.top_logprobs) a.top_logprobs[row * a.top + tid] = logprob(key_logit(k));
  }
}

}  // namespace ifq
