// Root-mean-square norm of rows, with the residual's addition before it.
#pragma once
#include "kv4.cuh"

namespace ifq {

struct NormArgs {
  const uint16_t *x, *res, *weight;
  uint16_t *sum, *out;
  long long x_stride, res_stride, sum_stride, out_stride;
  int rows, dim;
  float eps;
};

// A block a row, V times 8 values a thread, all loads under way before the first is used: the row stays in registers
// between its sum of squares and its products, so memory sees every value once.
//
// The squares' sum is single precision.  Where it leaves that range (values past 2^63 or so, or all of them so small that
// the squares vanish, which matters where eps does not cover it) it is taken again in double.
template <bool BF, int V>
__global__ void __launch_bounds__(1024) rms_norm_kernel(const __grid_constant__ NormArgs a) {
  grid_dep_wait();
  grid_dep_launch();
  __shared__ float part[32];
  __shared__ double part2[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const long long row = blockIdx.x;
  uint32_t h[V][4], w[V][4];
  {
    uint32_t r[V][4];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * blockDim.x + threadIdx.x) * 8;
#pragma unroll
      for (int i = 0; i < 4; ++i) h[v][i] = r[v][i] = w[v][i] = 0;
      if (c < a.dim) {
        load_words(h[v], a.x + row * a.x_stride + c);
        if (a.res) load_words(r[v], a.res + row * a.res_stride + c);
        load_words(w[v], a.weight + c);
      }
    }
    if (a.res)
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 p = unpack16<BF>(h[v][i]), q = unpack16<BF>(r[v][i]);
          h[v][i] = pack16<BF>(p.x + q.x, p.y + q.y);
        }
  }
  float s = 0.0f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = (v * blockDim.x + threadIdx.x) * 8;
    if (a.sum && c < a.dim) store_words(a.sum + row * a.sum_stride + c, h[v]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 p = unpack16<BF>(h[v][i]);
      s = fmaf(p.x, p.x, fmaf(p.y, p.y, s));
    }
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (warps > 1) {
    if (lane == 0) part[warp] = s;
    __syncthreads();
    s = lane < warps ? part[lane] : 0.0f;
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  }
  float scale = rsqrtf(s / (float)a.dim + a.eps);
  if (!(s < 1e37f) || (s < 1e-30f && a.eps < 1e-30f)) {   // (the whole block: s is the same in every thread)
    double d = 0.0;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 p = unpack16<BF>(h[v][i]);
        d += (double)p.x * p.x + (double)p.y * p.y;
      }
#pragma unroll
    for (int o = 16; o; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
    if (lane == 0) part2[warp] = d;
    __syncthreads();
    d = 0.0;
    for (int i = 0; i < warps; ++i) d += part2[i];
    // (applied in two steps, since its own square root may be past single precision's ends)
    const double r = 1.0 / sqrt(d / a.dim + (double)a.eps);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * blockDim.x + threadIdx.x) * 8;
      uint32_t o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 p = unpack16<BF>(h[v][i]), q = unpack16<BF>(w[v][i]);
        o[i] = pack16<BF>((float)(p.x * r) * q.x, (float)(p.y * r) * q.y);
      }
      if (c < a.dim) store_words(a.out + row * a.out_stride + c, o);
    }
    return;
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = (v * blockDim.x + threadIdx.x) * 8;
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 p = unpack16<BF>(h[v][i]), q = unpack16<BF>(w[v][i]);
      o[i] = pack16<BF>(p.x * scale * q.x, p.y * scale * q.y);
    }
    if (c < a.dim) store_words(a.out + row * a.out_stride + c, o);
  }
}

}  // namespace ifq
