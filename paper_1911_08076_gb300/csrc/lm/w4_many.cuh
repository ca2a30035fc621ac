// Products with weights in 4 bits, many rows of x: tcgen05 tiles whose weights are expanded into tensor memory.
//
// A tile is 128 packed rows of w (tensor-memory lanes, the MMA's A operand) x bn rows of x (columns, up to 256).  The
// weights go from 4 bits to 16 once for all of a tile's columns, in registers, and from there to tensor memory: their
// fragments need no swizzle, no shared memory, and leave its bandwidth to x.  A block of 128 columns of 16 rows is
// contiguous, so the codes of a tile's block are eight bulk copies; x comes by TMA in the 128-byte swizzle.
//
// Warps: sixteen that expand (a quadrant of 32 lanes, half of the columns of every other block of k each), two that load,
// one that issues MMAs, four that take results out.  Two accumulators take turns, so that a tile's results leave tensor
// memory beside the next tile's products.
//
// A tile's k may be split over a cluster of ks blocks: each sends its partial columns to the block that owns them through
// distributed shared memory, which adds them in the order of the ranks.
#pragma once
#include <cuda.h>

#include "tmem.cuh"
#include "w4.cuh"

namespace ifq {

struct W4Many {
  W4Args a;
  int bn, stages;              // columns a tile (a multiple of 16, up to 192); shared-memory stages of 128 columns of k
  int tiles, tiles_w, tiles_x; // items; tiles of w's rows and of x's
  int ks;                      // blocks that a tile's k is split over
};

constexpr int kW4Expand = 16, kW4Out = kW4Expand + 4, kW4ManyThreads = 32 * (kW4Out + 4);   // first warp that stores
constexpr int kW4CodeSlots = 3, kW4AStages = 2, kW4MaxCols = 192, kW4ACol = 2 * kW4MaxCols;
constexpr int kW4ManySmem = 232448;

__host__ __device__ constexpr int w4_many_codes(int group) { return kW4CodeSlots * 8 * w4_block_bytes(group); }
// a receive slot a rank: the owner's columns, 129 floats each
__host__ __device__ constexpr int w4_many_recv(int bn, int ks) { return ks > 1 ? (bn + 8) * 129 * 4 : 0; }
constexpr int w4_many_stages(int group, int bn, int ks) {
  const int n = (kW4ManySmem - 1024 - 512 - w4_many_codes(group) - w4_many_recv(bn, ks)) / (bn * 256);
  return n < 8 ? n : 8;
}

// A word's four pairs of codes to 16-bit values: rows g (s[0], m[0]) and g + 8 (s[1], m[1]).
template <bool BF>
__device__ __forceinline__ void w4_expand(uint32_t w, const uint32_t (&s)[2], const uint32_t (&m)[2], uint32_t* v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    // 128 + code as bfloat16, 1024 + code as half: exact, and so is the difference
    uint32_t c = ((w >> (4 * i)) & 0x000f000fu) | (BF ? 0x43004300u : 0x64006400u);
    if constexpr (BF) {
      asm("{.reg .b32 t; mov.b32 t, 0xc300c300; add.rn.bf16x2 %0, %0, t;}" : "+r"(c));
      asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(v[i]) : "r"(c), "r"(s[i & 1]), "r"(m[i & 1]));
    } else {
      asm("{.reg .b32 t; mov.b32 t, 0xe400e400; add.rn.f16x2 %0, %0, t;}" : "+r"(c));
      asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(v[i]) : "r"(c), "r"(s[i & 1]), "r"(m[i & 1]));
    }
  }
}
// A lane's parameters (scale, min of row g; of row g + 8) in both halves of a register each.
__device__ __forceinline__ void w4_params(uint2 p, uint32_t (&s)[2], uint32_t (&m)[2]) {
  s[0] = __byte_perm(p.x, 0, 0x1010);
  m[0] = __byte_perm(p.x, 0, 0x3232);
  s[1] = __byte_perm(p.y, 0, 0x1010);
  m[1] = __byte_perm(p.y, 0, 0x3232);
}

template <bool BF, int G, bool GATED>
__global__ void __launch_bounds__(kW4ManyThreads, 1)
    w4_many_kernel(const __grid_constant__ CUtensorMap tx, const __grid_constant__ W4Many r) {
  constexpr int WB = w4_block_bytes(G), CS = kW4CodeSlots, AS = kW4AStages;
  const W4Args& a = r.a;
  extern __shared__ uint8_t raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
  const uint32_t base = smem_u32(smem);
  const int ST = r.stages, xb = r.bn * 256;
  uint8_t* codes = smem + ST * xb;
  float* recv = (float*)(codes + CS * 8 * WB);
  const uint32_t cbase = smem_u32(codes);
  const uint32_t bars = cbase + CS * 8 * WB + w4_many_recv(r.bn, r.ks);
  // full: a block's x has landed and its weights stand in tensor memory; free: its products are done
  auto full = [&](int s) { return bars + 8 * s; };
  auto free = [&](int s) { return bars + 8 * (ST + s); };
  const uint32_t fixed = bars + 16 * ST;
  auto cfull = [&](int s) { return fixed + 8 * s; };
  auto cempty = [&](int s) { return fixed + 8 * (CS + s); };
  auto dfull = [&](int b) { return fixed + 8 * (2 * CS + b); };
  auto dempty = [&](int b) { return fixed + 8 * (2 * CS + 2 + b); };
  uint32_t* tptr = (uint32_t*)(smem + (dempty(2) - base));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int ks = r.ks, rank = ks > 1 ? (int)cluster_ctarank() : 0;
  if (threadIdx.x == 0) {
    for (int i = 0; i < ST; ++i) {
      mbar_init(full(i), 1 + kW4Expand / 2);
      mbar_init(free(i), 1);
    }
    for (int i = 0; i < CS; ++i) {
      mbar_init(cfull(i), 1);
      mbar_init(cempty(i), kW4Expand / 2);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(dfull(i), 1);
      mbar_init(dempty(i), 4);
    }
    fence_mbar_init();
    prefetch_tmap(&tx);
  }
  if (warp == 0) {
    tmem_alloc(smem_u32(tptr), 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tptr;
  if (ks > 1) cluster_sync_all();   // the partners' shared memory is there
  grid_dep_wait();
  grid_dep_launch();

  const uint32_t uks = ks;
  const int k0 = (uint32_t)(rank * a.kb) / uks, k1 = (uint32_t)((rank + 1) * a.kb) / uks;
  const int first = blockIdx.x / uks, step = gridDim.x / uks;
  // Tiles in groups of 16 tiles of w, within a group along w first.
  auto tile = [&](uint32_t t, int& iw, int& ix) {
    const uint32_t g = t / (16u * r.tiles_x), in = t - g * 16u * r.tiles_x, wide = min(16u, r.tiles_w - 16u * g);
    ix = in / wide;
    iw = 16 * g + in - ix * wide;
  };

  if (warp < kW4Expand) {
    const int q = warp & 3, h = (warp >> 2) & 1, odd = warp >> 3;
    constexpr int NP = G == 32 ? 2 : 1;   // groups in 64 columns
    const uint32_t tl = tmem + kW4ACol + ((uint32_t)(q * 32) << 16);
    // this warp's blocks are every other one of all that the CTA goes through
    const uint32_t turns = first < r.tiles ? (r.tiles - first + step - 1) / step : 0, total = turns * (k1 - k0);
    uint4 w[2];
    uint2 p[2][NP];
    bool ok = true;
    auto fetch = [&](uint32_t it) {
      const uint32_t slot = it % CS;
      if (!__all_sync(0xffffffffu, mbar_wait(cfull(slot), (it / CS) & 1))) { ok = false; return; }
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const uint8_t* c = codes + (slot * 8 + 2 * q + b) * WB;
        w[b] = *(const uint4*)(c + 512 * h + 16 * lane);
#pragma unroll
        for (int i = 0; i < NP; ++i) p[b][i] = *(const uint2*)(c + 1024 + 64 * (h * 64 / G + i) + 8 * (lane / 4));
      }
    };
    if (odd < total) fetch(odd);
    for (uint32_t it = odd; it < total && ok; it += 2) {
      uint32_t v[2][2][8];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const uint32_t words[4] = {w[b].x, w[b].y, w[b].z, w[b].w};
        uint32_t s[2], m[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (j < NP) w4_params(p[b][j], s, m);
          w4_expand<BF>(words[2 * j], s, m, v[b][j]);
          w4_expand<BF>(words[2 * j + 1], s, m, v[b][j] + 4);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(cempty(it % CS));
      if (it + 2 < total) fetch(it + 2);   // the next codes are on their way while these go to tensor memory
      // (two blocks stand in tensor memory: the products of the last but one are done)
      if (!ok || (it >= AS && !__all_sync(0xffffffffu, mbar_wait(free((it - AS) % ST), ((it - AS) / ST) & 1)))) break;
      tc_fence_after();
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int j = 0; j < 2; ++j) tmem_st_frag(tl + 64 * odd + 32 * h + ((uint32_t)(16 * b) << 16) + 16 * j, v[b][j]);
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(full(it % ST));
    }
  } else if (warp == kW4Expand) {   // x
    int it = 0;
    bool ok = true;
    for (int t = first; t < r.tiles && ok; t += step) {
      int iw, ix;
      tile(t, iw, ix);
      for (int k = k0; k < k1; ++k, ++it) {
        const int s = it % ST;
        if (it >= ST && !__all_sync(0xffffffffu, mbar_wait(free(s), (it / ST - 1) & 1))) { ok = false; break; }
        if (elect_one()) {
          mbar_arrive_expect_tx(full(s), xb);
          tma_load_2d(base + s * xb, &tx, full(s), k * 128, ix * r.bn);
          tma_load_2d(base + s * xb + xb / 2, &tx, full(s), k * 128 + 64, ix * r.bn);
        }
        __syncwarp();
      }
    }
    // what was loaded has landed, and in the end been read, before the block may exit
    for (int i = it - ST < 0 ? 0 : it - ST; i < it; ++i) mbar_wait(ok ? free(i % ST) : full(i % ST), (i / ST) & 1);
  } else if (warp == kW4Expand + 1) {   // codes and parameters
    int it = 0;
    bool ok = true;
    for (int t = first; t < r.tiles && ok; t += step) {
      int iw, ix;
      tile(t, iw, ix);
      for (int k = k0; k < k1; ++k, ++it) {
        const int s = it % CS;
        if (it >= CS && !__all_sync(0xffffffffu, mbar_wait(cempty(s), (it / CS - 1) & 1))) { ok = false; break; }
        if (lane == 0) mbar_arrive_expect_tx(cfull(s), 8 * WB);
        __syncwarp();
        if (lane < 8)
          bulk_copy_g2s(cbase + (s * 8 + lane) * WB, a.w + ((8ll * iw + lane) * a.kb + k) * WB, WB, cfull(s));
        __syncwarp();
      }
    }
    for (int i = it - CS < 0 ? 0 : it - CS; i < it; ++i) mbar_wait(ok ? cempty(i % CS) : cfull(i % CS), (i / CS) & 1);
  } else if (warp == kW4Expand + 2) {   // MMAs
    const uint32_t idesc = idesc_f16_f32(128, r.bn, BF);
    uint32_t it = 0, nt = 0, ph = 0;
    int s = 0;
    bool ok = true;
    for (int t = first; t < r.tiles && ok; t += step, ++nt) {
      const uint32_t acc = nt & 1, td = tmem + acc * kW4MaxCols;
      if (nt > 1 && !__all_sync(0xffffffffu, mbar_wait(dempty(acc), (nt / 2 - 1) & 1))) break;
      for (int k = k0; k < k1; ++k) {
        if (!__all_sync(0xffffffffu, mbar_wait(full(s), ph))) { ok = false; break; }
        tc_fence_after();
        if (elect_one()) {
          const uint64_t db = sdesc_sw128(base + s * xb);
          const uint32_t ta = tmem + kW4ACol + 64 * (it & 1);
#pragma unroll
          for (int j = 0; j < 8; ++j)   // 16 columns of k: 8 of tensor memory, two 16-byte units of the descriptor's address
            mma_f16_ts(td, ta + 8 * j, db + 2 * (j & 3) + (j >> 2) * (xb / 32), idesc, (k > k0) | (j > 0));
          mma_commit(free(s));
          if (k + 1 == k1) mma_commit(dfull(acc));
        }
        __syncwarp();
        ++it;
        if (++s == ST) s = 0, ph ^= 1;
      }
    }
  } else if (warp >= kW4Out) {   // results
    const int q = warp & 3, row = q * 32 + lane;
    uint32_t nt = 0;
    for (int t = first; t < r.tiles; t += step, ++nt) {
      int iw, ix;
      tile(t, iw, ix);
      const uint32_t acc = nt & 1, tl = tmem + acc * kW4MaxCols + ((uint32_t)(q * 32) << 16);
      if (!__all_sync(0xffffffffu, mbar_wait(dfull(acc), (nt / 2) & 1))) break;
      tc_fence_after();
      if (ks > 1) {
        const int per = (r.bn + ks - 1) / uks;
        for (int c0 = 0; c0 < r.bn; c0 += 16) {
          uint32_t v[16];
          tmem_ld<16>(tl + c0, v);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int c = c0 + i, own = ((c + 1) * uks - 1) / r.bn, lo = own * r.bn / uks;   // own bn / ks <= c
            asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(mapa_shared(smem_u32(recv + (rank * per + c - lo) * 129 + row), own)),
                         "r"(v[i])
                         : "memory");
          }
        }
        break;
      }
      const int e = (lane >> 3) & 1;
      const int n = GATED ? iw * 64 + q * 16 + (lane >> 4) * 8 + (lane & 7) : iw * 128 + row;
      float add[16], next[16];   // the residual, loaded 16 columns ahead
      auto residual = [&](int c0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int m = ix * r.bn + c0 + i;
          next[i] = c0 < r.bn && m < a.m && n < a.n ? w4_load(a.out_type, a.res, m * a.res_stride + n) : 0.0f;
        }
      };
      if (!GATED && a.res) residual(0);
      for (int c0 = 0; c0 < r.bn; c0 += 16) {
        uint32_t v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) add[i] = next[i];
        if (!GATED && a.res) residual(c0 + 16);
        tmem_ld<16>(tl + c0, v);
        if (c0 + 16 == r.bn) {   // the accumulator has been read
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(dempty(acc));
        }
        const int m0 = ix * r.bn + c0;
        if constexpr (GATED) {
          // lanes with bit 3 clear hold the gate's rows: they do the even columns, the others the odd ones
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            const float mine = __uint_as_float(e ? v[i + 1] : v[i]);
            const float other = __uint_as_float(__shfl_xor_sync(0xffffffffu, e ? v[i] : v[i + 1], 8));
            const float y = w4_act(a.act, e ? other : mine) * (e ? mine : other);
            const int m = m0 + i + e;
            if (m < a.m && n < a.n) w4_store(BF ? IFQ_BF16 : IFQ_F16, a.out, m * a.out_stride + n, y);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int m = m0 + i;
            const float y = __uint_as_float(v[i]) + (a.res ? add[i] : 0.0f);
            if (m < a.m && n < a.n) w4_store(a.out_type, a.out, m * a.out_stride + n, y);
          }
        }
      }
    }
  }
  if (ks > 1) {
    __syncwarp();
    cluster_sync_all();   // every partial sum has arrived
    int iw, ix;
    tile(first, iw, ix);
    const int lo = rank * r.bn / uks, wide = (rank + 1) * r.bn / uks - lo, per = (r.bn + ks - 1) / uks;
    const int total = (GATED ? 64 : 128) * wide;
    for (int i = threadIdx.x; i < total; i += kW4ManyThreads) {
      const int c = i / (GATED ? 64 : 128), j = i % (GATED ? 64 : 128), m = ix * r.bn + lo + c;
      const int n = iw * (GATED ? 64 : 128) + j, row = GATED ? j / 8 * 16 + j % 8 : j;
      float v = 0.0f, u = 0.0f;
      for (int p = 0; p < ks; ++p) {
        v += recv[(p * per + c) * 129 + row];
        if (GATED) u += recv[(p * per + c) * 129 + row + 8];
      }
      if (m >= a.m || n >= a.n) continue;
      if (GATED) v = w4_act(a.act, v) * u;
      else if (a.res) v += w4_load(a.out_type, a.res, m * a.res_stride + n);
      w4_store(a.out_type, a.out, m * a.out_stride + n, v);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, 512);
}

}  // namespace ifq
