// Root-mean-square norm of rows, with the residual's addition before it.
#pragma once
#include "kv4.cuh"

namespace ifq {

struct NormArgs {
  const uint16_t *x, *res, *weight;
  uint16_t *sum, *out;
  long long x_stride, res_stride, sum_stride, out_stride;
  int rows, dim;
  int threads;   // a row
  float eps;
};

// A block a row (a warp where rows are short), V times 8 values a thread: the row stays in registers between its sum of squares and its
// products, so memory sees every value once.  Up to V = 4 all loads are under way before the first is used; with 8 the residual
// comes in two halves, and the weights after the sum.  40 us, 6.7 TB/s (98 % of a copy) for 8191 x 4096 with a residual; one row
// takes 4 us, which is the call.
//
// The squares' sum is single precision.  Where it leaves that range (values past 2^63 or so, or all of them so small that
// the squares vanish, which matters where eps does not cover it) it is taken again in double.
// MOST: threads a block at most, and so the registers for a row's values.
template <bool BF, int V, int MOST>
__global__ void __launch_bounds__(MOST) rms_norm_kernel(const __grid_constant__ NormArgs a) {
  constexpr bool AHEAD = V <= 4;   // the weights too are under way with the row
  grid_dep_wait();
  grid_dep_launch();
  __shared__ float part[32];
  __shared__ double part2[32];
  // a block's warps share a row, or have one each where 32 threads are enough
  const int T = a.threads, tid = T == 32 ? threadIdx.x & 31 : threadIdx.x, lane = threadIdx.x & 31, warp = tid >> 5, warps = T >> 5;
  const long long row = T == 32 ? blockIdx.x * (long long)(blockDim.x / 32) + threadIdx.x / 32 : blockIdx.x;
  if (row >= a.rows) return;
  uint32_t h[V][4], w[AHEAD ? V : 1][4];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = (v * T + tid) * 8;
    h[v][0] = h[v][1] = h[v][2] = h[v][3] = 0;
    if (c < a.dim) load_words(h[v], a.x + row * a.x_stride + c);
    if constexpr (AHEAD) {
      w[v][0] = w[v][1] = w[v][2] = w[v][3] = 0;
      if (c < a.dim) load_words(w[v], a.weight + c);
    }
  }
  auto weights = [&](int v, uint32_t (&q)[4]) {
    const int c = (v * T + tid) * 8;
    if constexpr (AHEAD) {
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = w[v][i];
    } else {
      q[0] = q[1] = q[2] = q[3] = 0;
      if (c < a.dim) load_words(q, a.weight + c);
    }
  };
  if (a.res) {
    constexpr int N = AHEAD ? V : 4;   // loads of the residual under way
#pragma unroll
    for (int v0 = 0; v0 < V; v0 += N) {
      uint32_t r[N][4];
#pragma unroll
      for (int v = 0; v < N; ++v) {
        const int c = ((v0 + v) * T + tid) * 8;
        r[v][0] = r[v][1] = r[v][2] = r[v][3] = 0;
        if (c < a.dim) load_words(r[v], a.res + row * a.res_stride + c);
      }
#pragma unroll
      for (int v = 0; v < N; ++v)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 p = unpack16<BF>(h[v0 + v][i]), q = unpack16<BF>(r[v][i]);
          h[v0 + v][i] = pack16<BF>(p.x + q.x, p.y + q.y);
        }
    }
  }
  float s = 0.0f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = (v * T + tid) * 8;
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
  if (!(s < 1e37f) || (s < 1e-30f && a.eps < 1e-30f)) {   // (the whole row: s is the same in all its threads)
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
    if (warps > 1) {
      if (lane == 0) part2[warp] = d;
      __syncthreads();
      d = 0.0;
      for (int i = 0; i < warps; ++i) d += part2[i];
    }
    // (applied in two steps, since its own square root may be past single precision's ends)
    const double r = 1.0 / sqrt(d / a.dim + (double)a.eps);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * T + tid) * 8;
      uint32_t o[4], u[4];
      weights(v, u);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 p = unpack16<BF>(h[v][i]), q = unpack16<BF>(u[i]);
        o[i] = pack16<BF>((float)(p.x * r) * q.x, (float)(p.y * r) * q.y);
      }
      if (c < a.dim) store_words(a.out + row * a.out_stride + c, o);
    }
    return;
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = (v * T + tid) * 8;
    uint32_t o[4], u[4];
    weights(v, u);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 p = unpack16<BF>(h[v][i]), q = unpack16<BF>(u[i]);
      o[i] = pack16<BF>(p.x * scale * q.x, p.y * scale * q.y);
    }
    if (c < a.dim) store_words(a.out + row * a.out_stride + c, o);
  }
}

}  // namespace ifq
