// Scores of tokens: log probabilities, log-sum-exp, entropy and the likeliest tokens of rows of logits.
#pragma once
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
  float scale;
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

// What a row's sums come to.  most: largest z; sum: of e^(z - most); weighted: of e^(z - most) (z - most).
struct RowScores {
  float most, log_sum;
  __device__ RowScores(float m, float sum) : most(m), log_sum(logf(sum)) {}
  __device__ float lse() const { return most == -INFINITY || most == INFINITY ? most : most + log_sum; }
  __device__ float logprob(float z) const { return most == -INFINITY ? most : most == INFINITY ? z - most : z - most - log_sum; }
  __device__ float entropy(float sum, float weighted) const { return most == -INFINITY ? 0.0f : log_sum - weighted / sum; }
};

__device__ __forceinline__ float block_sum(float v, float* part) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = v;
  __syncthreads();
  v = 0.0f;
  for (int i = 0; i < (int)blockDim.x / 32; ++i) v += part[i];
  return v;
}

template <int TYPE>
__global__ void __launch_bounds__(256) token_scores_kernel(const __grid_constant__ ScoresArgs a) {
  grid_dep_wait();
  grid_dep_launch();
  __shared__ float part[8];
  __shared__ uint64_t best[8];
  const long long row = blockIdx.x, at = row * a.stride;
  float most = -INFINITY;
  for (int i = threadIdx.x; i < a.vocab; i += 256) most = max_nan(most, logit_at<TYPE>(a.logits, at + i) * a.scale);
#pragma unroll
  for (int o = 16; o; o >>= 1) most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, o));
  if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = most;
  __syncthreads();
  for (int i = 0; i < 8; ++i) most = max_nan(most, part[i]);
  const float ref = most == -INFINITY ? 0.0f : most;
  float sum = 0.0f, weighted = 0.0f;
  for (int i = threadIdx.x; i < a.vocab; i += 256) {
    const float d = logit_at<TYPE>(a.logits, at + i) * a.scale - ref, e = expf(d);
    sum += e;
    weighted += e > 0.0f ? e * d : e;
  }
  sum = block_sum(sum, part);
  weighted = block_sum(weighted, part);
  const RowScores s(most, sum);
  if (threadIdx.x == 0) {
    if (a.lse) a.lse[row] = s.lse();
    if (a.entropy) a.entropy[row] = s.entropy(sum, weighted);
    if (a.logprobs) {
      const long long t = a.tokens[row];
      if (t >= a.vocab) set_status(IFQ_ERANGE);
      a.logprobs[row] = t < 0 ? 0.0f : t >= a.vocab ? NAN : s.logprob(logit_at<TYPE>(a.logits, at + t) * a.scale);
    }
  }
  uint64_t last = ~0ull;
  for (int j = 0; j < a.top; ++j) {
    uint64_t k = 0;
    for (int i = threadIdx.x; i < a.vocab; i += 256) {
      const uint64_t u = top_key(logit_at<TYPE>(a.logits, at + i), i);
      if (u < last && u > k) k = u;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) k = max(k, __shfl_xor_sync(0xffffffffu, k, o));
    __syncthreads();
    if (threadIdx.x % 32 == 0) best[threadIdx.x / 32] = k;
    __syncthreads();
    for (int i = 0; i < 8; ++i) k = max(k, best[i]);
    last = k;
    if (threadIdx.x == 0) {
      if (a.top_ids) a.top_ids[row * a.top + j] = key_token(k);
      if (a.top_logprobs) a.top_logprobs[row * a.top + j] = s.logprob(key_logit(k) * a.scale);
    }
  }
}

}  // namespace ifq
