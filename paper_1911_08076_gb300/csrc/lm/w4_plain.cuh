// Products with weights in 4 bits, a thread an output.
#pragma once
#include "w4.cuh"

namespace ifq {

template <bool BF, int G>
__global__ void __launch_bounds__(256) w4_plain_kernel(const __grid_constant__ W4Args a) {
  grid_dep_wait();
  grid_dep_launch();
  const int j = blockIdx.x * 32 + threadIdx.x % 32;
  if (j >= a.n) return;
  const bool gated = a.act != 0;
  for (long long i = blockIdx.y * 8 + threadIdx.x / 32; i < a.m; i += 8ll * gridDim.y) {
    float sum[2] = {0.0f, 0.0f};
    const int r = gated ? j % 8 : j % 16;
    const uint8_t* rb = a.w + (long long)(gated ? j / 8 : j / 16) * a.kb * w4_block_bytes(G);
    for (int c = 0; c < a.k; ++c) {
      const uint8_t* b = rb + (long long)(c / 128) * w4_block_bytes(G);
      const int cc = c % 128, u = cc / 64, s = cc % 64 / 16, e = cc % 16, t = e % 8 / 2;
      const uint32_t w = *(const uint32_t*)(b + 512 * u + 16 * (4 * (r % 8) + t) + 4 * s);
      const float x = unpack16<BF>(a.x[i * a.x_stride + c]).x;
      for (int h = 0; h < 1 + gated; ++h) {
        const int half = gated ? h : r / 8;
        const uint32_t p = *(const uint32_t*)(b + 1024 + 64 * (cc / G) + 8 * (r % 8) + 4 * half);
        const int code = (w >> (4 * (half + 2 * (e / 8)) + 16 * (e & 1))) & 15;
        sum[h] = fmaf(x, w4_value<BF>(code, (uint16_t)p, (uint16_t)(p >> 16)), sum[h]);
      }
    }
    float v = gated ? w4_act(a.act, sum[0]) * sum[1] : sum[0];
    if (a.res) v += w4_load(a.out_type, a.res, i * a.res_stride + j);
    w4_store(a.out_type, a.out, i * a.out_stride + j, v);
  }
}

}  // namespace ifq
