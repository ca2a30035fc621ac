// Products in e4m3 with a float scale for each block of 128 along k, and the quantiser of their
// activations.
#pragma once
#include <cuda_fp8.h>

#include "kv4.cuh"

namespace ifq {

constexpr int kFp8Block = 128;
constexpr int kFp8QuantWarps = 8;

struct Fp8QuantArgs {
  const uint16_t* x;
  uint8_t* codes;
  float* scales;
  long long x_stride;
  int m, k, kb;
};

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

// One warp a block of 128 values, four a lane (k is a multiple of 16, so a lane's four are all there or none).
template <bool BF>
__global__ void __launch_bounds__(32 * kFp8QuantWarps) fp8_quantize_kernel(const Fp8QuantArgs a) {
  grid_dep_wait();
  const long long item = (long long)blockIdx.x * kFp8QuantWarps + (threadIdx.x >> 5);
  if (item >= (long long)a.m * a.kb) return;
  const int r = (int)(item / a.kb), b = (int)(item - (long long)r * a.kb);
  const int lane = threadIdx.x & 31, c = b * kFp8Block + lane * 4;
  uint32_t w[2] = {0, 0};
  if (c < a.k) load_words(w, a.x + r * a.x_stride + c);
  const float2 u = unpack16<BF>(w[0]), v = unpack16<BF>(w[1]);
  float top = max_nan(max_nan(fabsf(u.x), fabsf(u.y)), max_nan(fabsf(v.x), fabsf(v.y)));
#pragma unroll
  for (int o = 16; o; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
  const float s = __fmul_rn(top, 1.0f / 448.0f);
  uint32_t out = 0;
  if (s != 0.0f)
    out = e4m3x2(__fdiv_rn(u.x, s), __fdiv_rn(u.y, s)) | e4m3x2(__fdiv_rn(v.x, s), __fdiv_rn(v.y, s)) << 16;
  if (c < a.k) *(uint32_t*)(a.codes + (long long)r * a.k + c) = out;
  if (lane == 0) a.scales[(long long)b * a.m + r] = s;
}

struct Fp8Args {
  const uint8_t *x, *w;
  const float *xs, *ws;
  void* out;
  long long out_stride;
  int m, n, k, kb, out_type;
};

__device__ __forceinline__ float e4m3_value(uint8_t b) {
  return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)b, __NV_E4M3)));
}

// 64 x 64 outputs a block of 256 threads, 4 x 4 a thread.
__global__ void __launch_bounds__(256) fp8_matmul_kernel(const Fp8Args a) {
  __shared__ float sx[32][65], sw[32][65];
  grid_dep_wait();
  const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64, ti = threadIdx.x / 16, tj = threadIdx.x % 16;
  float acc[4][4] = {}, part[4][4] = {};
  for (int k0 = 0; k0 < a.k; k0 += 32) {
    for (int e = threadIdx.x; e < 64 * 32; e += 256) {
      const int r = e / 32, c = e % 32;
      const bool in = k0 + c < a.k;
      sx[c][r] = in && i0 + r < a.m ? e4m3_value(a.x[(long long)(i0 + r) * a.k + k0 + c]) : 0.0f;
      sw[c][r] = in && j0 + r < a.n ? e4m3_value(a.w[(long long)(j0 + r) * a.k + k0 + c]) : 0.0f;
    }
    __syncthreads();
    for (int c = 0; c < 32; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) part[i][j] += sx[c][ti + 16 * i] * sw[c][tj + 16 * j];
    __syncthreads();
    if ((k0 + 32) % kFp8Block == 0 || k0 + 32 >= a.k) {
      const int b = k0 / kFp8Block;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = i0 + ti + 16 * i, c = j0 + tj + 16 * j;
          if (r < a.m && c < a.n) acc[i][j] += a.xs[(long long)b * a.m + r] * a.ws[(long long)(c / 128) * a.kb + b] * part[i][j];
          part[i][j] = 0.0f;
        }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = i0 + ti + 16 * i, c = j0 + tj + 16 * j;
      if (r >= a.m || c >= a.n) continue;
      const long long at = r * a.out_stride + c;
      if (a.out_type == IFQ_F32) ((float*)a.out)[at] = acc[i][j];
      else if (a.out_type == IFQ_F16) ((__half*)a.out)[at] = __float2half_rn(acc[i][j]);
      else ((__nv_bfloat16*)a.out)[at] = __float2bfloat16_rn(acc[i][j]);
    }
}

}  // namespace ifq
