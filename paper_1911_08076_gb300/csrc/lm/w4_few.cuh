// Products with weights in 4 bits, few rows of x: the weights are read once, and are what bounds it.
//
// mma.sync with 16 rows of w on M and 8 rows of x on N (NT such tiles): a lane's 16 bytes of codes are its operands of
// four steps of k.  A block is 16 warps, WR of them beside each other along w's rows and WK along k; the partial sums of
// a row block's WK warps meet in shared memory and are added in order.  Row blocks go round the blocks of the grid.
// A warp has four blocks of 128 columns under way, 70 KB an SM, whatever row block they belong to.
//
// The expansion is 88 of some 167 warp instructions for a block of 16 x 128, half of them on the integer pipe (59 % busy
// over all, issue slots 60 %; the rest are waits).  1 x 4096 x 4096 takes 4.2 us in a row of calls, where a call alone is 4;
// 8 x 131072 x 4096 in the second form 63 us, 4.85 TB/s (71 % of a copy).
//
// x stands in shared memory as operands: of every 32 columns, the 16 bytes of lane t of a quad are its registers of two
// steps, and rows begin 64 bytes apart modulo 128, so that eight lanes read all banks once.
#pragma once
#include <type_traits>

#include "w4.cuh"

namespace ifq {

struct W4Few {
  W4Args a;
  int wk, wr, blocks;   // warps along k and along rows; row blocks in all
};

constexpr int kW4FewWarps = 16, kW4FewDeep = 4;

__host__ __device__ constexpr long long w4_few_pitch(int kb) { return kb * 256ll + 64; }
__host__ __device__ constexpr long long w4_few_smem(int m, int kb, int nt) {   // x, and two turns of partial sums
  return m * w4_few_pitch(kb) + 2ll * kW4FewWarps * 16 * 8 * nt * 4;
}

template <bool BF>
__device__ __forceinline__ void mma_16x8x16(float (&c)[4], const uint32_t* a, uint32_t b0, uint32_t b1) {
  if constexpr (BF)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 load_once(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 load_once2(const void* p) {
  uint2 v;
  asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}

// One block of 128 columns: acc += 16 rows of w times 8 NT rows of x, whose operands stand at xs + xo.  The tensor cores
// truncate what they add: a block's sums begin at 0, and are added to the others' in single precision (8 x 131072 x 4096 to
// floats: off by 1.1e-6 of the result in one chain, 1.1e-7 so).
template <bool BF, bool FAST, int G, int NT>
__device__ __forceinline__ void w4_block(const uint4 (&w)[2], const uint2 (&p)[kW4Cols / G], const uint8_t* const (&xs)[NT], int xo,
                                         float (&acc)[NT][4]) {
  const uint32_t words[8] = {w[0].x, w[0].y, w[0].z, w[0].w, w[1].x, w[1].y, w[1].z, w[1].w};
  uint32_t s[2], m[2];
  float sum[NT][4] = {};
#pragma unroll
  for (int j = 0; j < 8; j += 2) {   // 32 columns
    if (j * 16 % G == 0) w4_params(p[j * 16 / G], s, m);
    uint32_t v[8];
    w4_expand<BF, FAST>(words[j], s, m, v);
    w4_expand<BF, FAST>(words[j + 1], s, m, v + 4);
#pragma unroll
    for (int q = 0; q < NT; ++q) {
      const uint4 b = *(const uint4*)(xs[q] + xo + j * 32);
      mma_16x8x16<BF>(sum[q], v, b.x, b.y);
      mma_16x8x16<BF>(sum[q], v + 4, b.z, b.w);
    }
  }
#pragma unroll
  for (int q = 0; q < NT; ++q)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[q][j] += sum[q][j];
}

// x into shared memory, 16 bytes at a time: four pairs of columns of one step's half, one for each lane of a quad.
__device__ __forceinline__ void w4_stage_x(const W4Args& a, uint8_t* smem, long long pitch, int id, int threads) {
  for (int c = id; c < a.kb * 16; c += threads) {
    uint8_t* to = smem + (c / 4) * 64 + (c % 4) * 4;
    for (int r0 = 0; r0 < a.m; r0 += 4) {
      uint32_t v[4][4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        v[u][0] = v[u][1] = v[u][2] = v[u][3] = 0;
        if (r0 + u < a.m && c * 8 < a.k) load_words(v[u], a.x + (r0 + u) * a.x_stride + c * 8);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (r0 + u < a.m)
#pragma unroll
          for (int j = 0; j < 4; ++j) *(uint32_t*)(to + (r0 + u) * pitch + 16 * j) = v[u][j];
    }
  }
}

// A row block's outputs from its partial sums, part[WK][8 NT tokens][16 rows], by threads id of `threads`.
template <bool GATED, int NT>
__device__ __forceinline__ void w4_few_out(const W4Args& a, const float* part, int wk, int rb, int id, int threads, float add) {
  constexpr int NO = GATED ? 8 : 16;
  for (int i = id; i < NO * a.m; i += threads) {
    const float* s = part + (i / NO) * 16 + i % NO;
    float v = 0.0f, u = 0.0f;
    for (int q = 0; q < wk; ++q) {
      v += s[q * (16 * 8 * NT)];
      if (GATED) u += s[q * (16 * 8 * NT) + 8];
    }
    const int n = rb * NO + i % NO;
    if (n >= a.n) continue;
    if (GATED) v = w4_act(a.act, v) * u;
    else if (a.res) v += i == id ? add : w4_load(a.out_type, a.res, (i / NO) * a.res_stride + n);
    w4_store(a.out_type, a.out, (i / NO) * a.out_stride + n, v);
  }
}
// The residual of output `id` of a row block, loaded before its sums are there.
template <bool GATED>
__device__ __forceinline__ float w4_few_residual(const W4Args& a, int rb, int id) {
  const int n = rb * 16 + id % 16;
  return !GATED && a.res && id < 16 * a.m && n < a.n ? w4_load(a.out_type, a.res, (id / 16) * a.res_stride + n) : 0.0f;
}
template <int NT>
__device__ __forceinline__ void w4_few_put(float* part, float (&acc)[NT][4], int g, int t) {
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      part[(8 * i + 2 * t + (j & 1)) * 16 + g + 8 * (j >> 1)] = acc[i][j];
      acc[i][j] = 0.0f;
    }
}

template <bool BF, int G, bool GATED, int NT>
__global__ void __launch_bounds__(32 * kW4FewWarps, 1) w4_few_kernel(const __grid_constant__ W4Few r) {
  constexpr int WB = w4_block_bytes(G), NP = kW4Cols / G, P = kW4FewDeep;
  const W4Args& a = r.a;
  extern __shared__ __align__(16) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane / 4, t = lane % 4;
  const int wk = warp % r.wk, wr = warp / r.wk, id = wk * 32 + lane;   // id: the thread among its row block's
  const long long pitch = w4_few_pitch(a.kb);
  float* part = (float*)(smem + a.m * pitch) + wr * r.wk * (16 * 8 * NT);   // [2][WR][WK][8 NT tokens][16 rows]
  constexpr int TURN = kW4FewWarps * 16 * 8 * NT;
  // this warp's blocks: columns k0 to k1 of row blocks first, first + step, ...
  const int k0 = wk * a.kb / r.wk, nk = (wk + 1) * a.kb / r.wk - k0;
  const int first = blockIdx.x * r.wr + wr, step = gridDim.x * r.wr;
  const int rows = first < r.blocks ? (r.blocks - first + step - 1) / step : 0;
  const int total = rows * nk;
  // While the kernel before this one ends, the first blocks come as far as L2, which has them right whoever writes them
  // (1 x 4096 x 4096 in a row of calls: 5.1 -> 4.2 us).
  if (rows && lane < (WB + 127) / 128)
    for (int u = 0; u < min(nk, P); ++u)
      asm volatile("prefetch.global.L2 [%0];" ::"l"(a.w + w4_place(first, k0 + u, a.kb) * WB + min(128 * lane, WB - 16)));
  grid_dep_wait();
  grid_dep_launch();

  const uint8_t *codes, *pars;
  int at = first;
  auto seek = [&] {
    codes = a.w + w4_place(at, k0, a.kb) * WB + 16 * lane;
    pars = codes - 16 * lane + 1024 + 8 * g;
    at += step;
  };
  seek();
  uint4 w[P][2];
  uint2 p[P][NP];
  int left = nk;
  auto load = [&](int u) {
    w[u][0] = load_once(codes);
    w[u][1] = load_once(codes + 512);
#pragma unroll
    for (int i = 0; i < NP; ++i) p[u][i] = load_once2(pars + 64 * i);
    codes += 8 * WB;
    pars += 8 * WB;
    if (--left == 0) {
      left = nk;
      seek();
    }
  };
#pragma unroll
  for (int u = 0; u < P; ++u)
    if (u < total) load(u);
  const bool large = *a.large != 0;

  w4_stage_x(a, smem, pitch, threadIdx.x, 32 * kW4FewWarps);
  __syncthreads();

  float acc[NT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0.0f;
  const uint8_t* xs[NT];   // (rows past the last read the last: their results are not stored)
#pragma unroll
  for (int i = 0; i < NT; ++i) xs[i] = smem + min(8 * i + g, a.m - 1) * pitch + k0 * 256 + 16 * t;

  int rb = first, turn = 0;
  float add = rows > 0 ? w4_few_residual<GATED>(a, rb, id) : 0.0f;
  auto flush = [&] {   // a row block's sums
    float* sums = part + turn * TURN;
    w4_few_put<NT>(sums + wk * (16 * 8 * NT), acc, g, t);
    if (r.wk == 1) __syncwarp();
    else named_bar(1 + wr, r.wk * 32);
    w4_few_out<GATED, NT>(a, sums, r.wk, rb, id, r.wk * 32, add);
    turn ^= 1;   // (the next sums go elsewhere: who writes to this place again has passed the barrier after these reads)
    rb += step;
    if (rb < r.blocks) add = w4_few_residual<GATED>(a, rb, id);
  };

  if (nk == 0) {   // fewer blocks of k than warps: zeros for the others' sums
    for (int i = 0; i < rows; ++i) flush();
    return;
  }
  // (the loop in two forms, of which a launch runs one)
  auto multiply = [&](auto fast) {
    constexpr bool FAST = decltype(fast)::value;
    int kk = nk, xo = 0;
    for (int i = total; i > 0; i -= P) {
#pragma unroll
      for (int u = 0; u < P; ++u) {
        if (u >= i) break;
        w4_block<BF, FAST, G, NT>(w[u], p[u], xs, xo, acc);
        if (u + P < i) load(u);
        xo += 256;
        if (--kk == 0) {
          kk = nk;
          xo = 0;
          flush();
        }
      }
    }
  };
  if (large) multiply(std::false_type());
  else multiply(std::true_type());
}

// The same for weights of many rows: a block takes tiles of eight row blocks, whose codes a warp of its own brings in by bulk
// copies, a block of 128 columns of the tile each, as many ahead as shared memory holds; WK warps a row block take every
// WK-th of them.  Those go through a ring of their own, `deep` stages each: copies may land in any order, and a wait for a
// phase of a barrier holds only for who has seen the one before it.
struct W4Ring {
  W4Args a;
  int tiles, deep;
};

__host__ __device__ constexpr int w4_ring_wk(int nt) { return nt == 1 ? 3 : 2; }
__host__ __device__ constexpr int w4_ring_part(int nt) { return 2 * 8 * w4_ring_wk(nt) * 16 * 8 * nt * 4; }
__host__ __device__ constexpr long long w4_ring_fixed(int m, int kb, int nt) {   // without the stages
  return m * w4_few_pitch(kb) + w4_ring_part(nt) + 1024;
}
constexpr int kW4RingMost = 32;   // stages, all rings'
// Stages of a ring where shared memory has room for `fit` in all.
__host__ __device__ constexpr int w4_ring_deep(int fit, int nt) { return (fit < kW4RingMost ? fit : kW4RingMost) / w4_ring_wk(nt); }

template <bool BF, int G, bool GATED, int NT>
__global__ void __launch_bounds__(32 * (8 * w4_ring_wk(NT) + 1), 1) w4_ring_kernel(const __grid_constant__ W4Ring r) {
  constexpr int WB = w4_block_bytes(G), NP = kW4Cols / G, WK = w4_ring_wk(NT);
  const W4Args& a = r.a;
  extern __shared__ __align__(16) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, D = r.deep, ST = D * WK;
  const long long pitch = w4_few_pitch(a.kb);
  uint8_t* ring = smem + a.m * pitch;   // (a multiple of 64 bytes)
  float* part = (float*)(ring + ST * 8 * WB);
  const uint32_t bars = smem_u32(part) + w4_ring_part(NT);
  auto full = [&](int s) { return bars + 8 * s; };
  auto empty = [&](int s) { return bars + 8 * (ST + s); };
  if (threadIdx.x == 0) {
    for (int s = 0; s < ST; ++s) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), 8);
    }
    fence_mbar_init();
  }
  const int first = blockIdx.x, step = gridDim.x;
  if (threadIdx.x == 32)   // (into L2 while the kernel before this one ends)
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(a.w + w4_place(8ll * first, 0, a.kb) * WB),
                 "r"(min(ST, a.kb) * 8 * WB)
                 : "memory");
  __syncthreads();
  grid_dep_wait();
  grid_dep_launch();
  if (warp == 8 * WK) {
    int at[WK] = {}, ph[WK];   // of each ring: the stage that is filled next, and the phase that frees it
#pragma unroll
    for (int w = 0; w < WK; ++w) ph[w] = 1;
    auto ahead = [&](int w) {
      if (++at[w] == D) at[w] = 0, ph[w] ^= 1;
    };
    bool ok = true;
    for (int t = first; t < r.tiles && ok; t += step) {
      const uint8_t* from = a.w + w4_place(8ll * t, 0, a.kb) * WB;
      for (int k = 0; k < a.kb && ok; k += WK) {
#pragma unroll
        for (int w = 0; w < WK; ++w, from += 8 * WB) {
          if (k + w >= a.kb) break;
          const int s = w * D + at[w];
          if (!__all_sync(0xffffffffu, mbar_wait(empty(s), ph[w]))) { ok = false; break; }
          if (elect_one()) {
            mbar_arrive_expect_tx(full(s), 8 * WB);
            bulk_copy_g2s(smem_u32(ring) + s * 8 * WB, from, 8 * WB, full(s));
          }
          __syncwarp();
          ahead(w);
        }
      }
    }
    // What was copied has landed, and in the end been read, before the block may exit.  (A stage's last copy completes the phase of
    // full that its release completes of empty; one that was never filled waits for nothing.)
#pragma unroll
    for (int w = 0; w < WK; ++w)
      for (int i = 0; i < D; ++i) {
        mbar_wait(ok ? empty(w * D + at[w]) : full(w * D + at[w]), ph[w]);
        ahead(w);
      }
    return;
  }
  w4_stage_x(a, smem, pitch, threadIdx.x, 32 * 8 * WK);
  const bool large = *a.large != 0;
  named_bar(10, 32 * 8 * WK);

  const int row = warp & 7, wk = warp >> 3, g = lane / 4, t4 = lane % 4, id = wk * 32 + lane;
  float acc[NT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0.0f;
  const uint8_t* xs[NT];   // (rows past the last read the last: their results are not stored)
#pragma unroll
  for (int i = 0; i < NT; ++i) xs[i] = smem + min(8 * i + g, a.m - 1) * pitch + 16 * t4;
  const uint8_t* mine = ring + row * WB;
  auto multiply = [&](auto fast) {
    constexpr bool FAST = decltype(fast)::value;
    int at = 0, ph = 0, turn = 0;   // the next stage of these warps' ring, and its phase
    bool ok = true;
    for (int t = first; t < r.tiles; t += step, turn ^= 1) {
      const int rb = 8 * t + row;
      const float add = w4_few_residual<GATED>(a, rb, id);
      for (int k = wk; k < a.kb; k += WK) {
        const int s = wk * D + at;
        ok = ok && __all_sync(0xffffffffu, mbar_wait(full(s), ph));   // (after one that ran out none waits again)
        const uint8_t* c = mine + s * 8 * WB;
        uint4 w[2] = {*(const uint4*)(c + 16 * lane), *(const uint4*)(c + 512 + 16 * lane)};
        uint2 p[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) p[i] = *(const uint2*)(c + 1024 + 64 * i + 8 * g);
        w4_block<BF, FAST, G, NT>(w, p, xs, k * 256, acc);
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(s));
        if (++at == D) at = 0, ph ^= 1;
      }
      float* sums = part + turn * (w4_ring_part(NT) / 8) + row * WK * (16 * 8 * NT);
      w4_few_put<NT>(sums + wk * (16 * 8 * NT), acc, g, t4);
      named_bar(1 + row, 32 * WK);
      w4_few_out<GATED, NT>(a, sums, WK, rb, id, 32 * WK, add);
    }
  };
  if (large) multiply(std::false_type());
  else multiply(std::true_type());
}

}  // namespace ifq
