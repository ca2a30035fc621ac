// Products with weights in 4 bits, many rows of x: tcgen05 tiles whose weights are expanded into tensor memory.
//
// A tile is 128 packed rows of w (tensor-memory lanes, the MMA's A operand) x bn rows of x (columns).  The weights go
// from 4 bits to 16 once for all of a tile's columns, in registers, and from there to tensor memory: their fragments need
// no swizzle, no shared memory, and leave its bandwidth to x.  The codes of a tile's 128 columns are contiguous, one bulk
// copy (eight took 800 cycles to issue); x comes by TMA in the 128-byte swizzle.
//
// CG = 2: two CTAs of a cluster share a tile of 256 rows (128 lanes each) x up to 256 columns, whose x they hold half
// each: one thread issues the MMAs of both SMs, and a value of x leaves L2 half as often.
// CG = 1, for fewer columns: up to 128, and a tile's k may be split over a cluster of ks blocks: each sends its partial
// columns to the block that owns them through distributed shared memory, which adds them in the order of the ranks.
//
// Tensor memory: columns 0 to 255 are the accumulator (two that take turns where bn <= 128, so that a tile's results
// leave beside the next tile's products), the others four blocks of expanded weights: from an MMA that frees a block to
// one that reads its successor take 700 cycles, and more between two SMs.
// The tensor cores truncate what they add, which shows in results of 32 bits (1000 x 2048 x 16384: off by 1.4e-5 of the
// result).  Those (bn <= 128) are added in tensor memory over 1024 columns of k at most; the sums of such chains meet in shared
// memory, in single precision, beside the next chain's products.
// Where bn > 128 results are of 16 bits, and leave through shared memory: the accumulator is free again after some 4000 cycles.
//
// Measured: 4096 x 4096 x 9216 in 186 to 193 us from card to card, 1.66 to 1.60 PFLOP/s, gated 2048 x 9216 x 4096 in 178 to 187, 1.74 to 1.65
// (a library product of bfloat16: 1.86 in a burst, 1.70 for long); one SM a tile took 277.  With few columns a block of 128 of k takes 600 cycles whatever bn is.
//
// Warps: sixteen that expand (a quadrant of 32 lanes, half of the columns of every other block of k each), two that load,
// one that issues MMAs, eight that take results out.
#pragma once
#include <cuda.h>

#include <type_traits>

#include "tmem.cuh"
#include "w4.cuh"

namespace ifq {

struct W4Many {
  W4Args a;
  int bn, stages, slots;       // columns a tile; stages of 128 columns of k of x, and of codes, in shared memory
  int tiles, tiles_w, tiles_x; // items; tiles of w's rows (CG times 128) and of x's
  int whole;                   // items that are whole tiles; the rest are halves (CG = 2)
  int ks;                      // blocks that a tile's k is split over
  int chain;                   // blocks of 128 columns of k that are added in tensor memory
  int turn;                    // bytes of shared memory for results on their way out, or sums of several chains
  int vec;                     // rows of out (and of the residual) can be accessed 16 bytes at a time
};

constexpr int kW4Expand = 16, kW4Out = kW4Expand + 4, kW4Outs = 8, kW4ManyThreads = 32 * (kW4Out + kW4Outs);   // kW4Out: first warp that stores
constexpr int kW4Bars = 8;         // barriers in turn: no fewer than stages of x or blocks of expanded weights
constexpr int kW4AStages = 4, kW4ACol = 256;
constexpr int kW4ManySmem = 232448;
// Slots for blocks of codes where shared memory has room for `fit`.  The two sets of expanding warps take alternate blocks, and a
// wait for a phase of a slot's barrier holds only where the block that had the slot before is known to have landed: it was the same
// set's (an even number), or it is behind the block whose products the set has waited for, kW4AStages + 2 before.
__host__ __device__ constexpr int w4_code_slots(int fit) {
  const int n = fit < 12 ? fit : 12;
  return n % 2 == 0 || n > kW4AStages + 2 ? n : n - 1;
}
static_assert(w4_code_slots(3) == 2 && w4_code_slots(5) == 4 && w4_code_slots(6) == 6 && w4_code_slots(7) == 7 && w4_code_slots(30) == 12,
              "slots that alternate blocks may share");

// a receive slot a rank: the owner's columns, 129 floats each
__host__ __device__ constexpr int w4_many_recv(int bn, int ks) { return ks > 1 ? (bn + 8) * 129 * 4 : 0; }
// results of 16 bits on their way out: a row a column of the tile (a gated pair's fragments write four at a time: apart)
__host__ __device__ constexpr int w4_out_pitch(bool gated) { return gated ? 144 : 256; }

// The instructions of two CTAs' MMAs.
template <int CG>
__device__ __forceinline__ void w4_mma(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  if constexpr (CG == 1) mma_f16_ts(d, a, b, idesc, acc);
  else
    asm volatile("{.reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;}" ::"r"(d),
                 "r"(a), "l"(b), "r"(idesc), "r"(acc)
                 : "memory");
}
template <int CG>   // arrives on the barrier of this CTA, or of both
__device__ __forceinline__ void w4_commit(uint32_t bar) {
  if constexpr (CG == 1) mma_commit(bar);
  else
    asm volatile(
        "{.reg .b16 m; mov.b16 m, 3; tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 "
        "[%0], m;}" ::"r"(bar)
        : "memory");
}
template <int CG>   // bar: a shared::cluster address where CG = 2
__device__ __forceinline__ void w4_load_x(uint32_t dst, const void* tmap, uint32_t bar, int x, int y) {
  if constexpr (CG == 1) tma_load_2d(dst, tmap, bar, x, y);
  else
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], "
        "[%2];" ::"r"(dst),
        "l"(tmap), "r"(bar), "r"(x), "r"(y)
        : "memory");
}
template <int CG>
__device__ __forceinline__ void w4_alloc(uint32_t dst) {
  if constexpr (CG == 1) {
    tmem_alloc(dst, 512);
    tmem_relinquish();
  } else {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(dst) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
}
template <int CG>
__device__ __forceinline__ void w4_dealloc(uint32_t t) {
  if constexpr (CG == 1) tmem_dealloc(t, 512);
  else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(t) : "memory");
}

template <bool BF, int G, bool GATED, int CG>
__global__ void __launch_bounds__(kW4ManyThreads, 1)
    w4_many_kernel(const __grid_constant__ CUtensorMap tx, const __grid_constant__ W4Many r) {
  constexpr int WB = w4_block_bytes(G), AS = kW4AStages, NB = kW4Bars, PITCH = w4_out_pitch(GATED), NO = GATED ? 64 : 128;
  const W4Args& a = r.a;
  extern __shared__ uint8_t raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
  const uint32_t base = smem_u32(smem);
  const int ST = r.stages, CS = r.slots, half = r.bn / CG * 128, xb = 2 * half;   // bytes of 64 and 128 columns of k
  uint8_t* codes = smem + ST * xb;
  uint8_t* turn = codes + CS * 8 * WB;
  float* recv = (float*)turn;
  const uint32_t cbase = smem_u32(codes);
  const uint32_t bars = smem_u32(turn) + w4_many_recv(r.bn, r.ks) + r.turn;
  // Block it of all that the CTA goes through: full(it % NB): its x has landed and its weights stand in tensor memory (of
  // both CTAs, on the first one's barrier); done(it % NB): its products are there.
  auto full = [&](int i) { return bars + 8 * i; };
  auto done = [&](int i) { return bars + 8 * (NB + i); };
  auto dfull = [&](int b) { return bars + 8 * (2 * NB + b); };
  auto dempty = [&](int b) { return bars + 8 * (2 * NB + 2 + b); };
  auto cfull = [&](int s) { return bars + 8 * (2 * NB + 4 + s); };
  auto cempty = [&](int s) { return bars + 8 * (2 * NB + 4 + CS + s); };
  uint32_t* tptr = (uint32_t*)(smem + (cempty(CS) - base));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = CG == 2 || r.ks > 1 ? (int)cluster_ctarank() : 0, ks = r.ks;
  if (threadIdx.x == 0) {
    for (int i = 0; i < NB; ++i) {
      mbar_init(full(i), 1 + CG * kW4Expand / 2);
      mbar_init(done(i), 1);
    }
    for (int i = 0; i < CS; ++i) {
      mbar_init(cfull(i), 1);
      mbar_init(cempty(i), kW4Expand / 2);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(dfull(i), 1);
      mbar_init(dempty(i), kW4Outs * CG);
    }
    fence_mbar_init();
    prefetch_tmap(&tx);
  }
  if (warp == 0) w4_alloc<CG>(smem_u32(tptr));
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tptr;
  const uint32_t uks = ks, uc = CG == 2 ? 2 : uks;   // CTAs of a cluster
  const int k0 = CG == 2 ? 0 : (uint32_t)(rank * a.kb) / uks, k1 = CG == 2 ? a.kb : (uint32_t)((rank + 1) * a.kb) / uks;
  const int first = blockIdx.x / uc, step = gridDim.x / uc, accs = r.bn <= 128 ? 2 : 1;
  // Item t: columns m0 to m0 + wd of the rows of w in tile iw (of this CTA).  Tiles in groups of 16 tiles of w, within a
  // group along w first.
  auto tile = [&](uint32_t t, int& iw, int& m0, int& wd) {
    wd = r.bn;
    uint32_t odd = 0;
    if (CG == 2 && t >= (uint32_t)r.whole) {
      odd = (t - r.whole) & 1;
      t = r.whole + (t - r.whole) / 2;
      wd = r.bn / 2;
    }
    const uint32_t g = t / (16u * r.tiles_x), in = t - g * 16u * r.tiles_x, wide = min(16u, r.tiles_w - 16u * g), ix = in / wide;
    iw = (16 * g + in - ix * wide) * CG + (CG == 2 ? rank : 0);
    m0 = ix * r.bn + odd * (r.bn / 2);
  };
  // Where the codes of a tile begin.  (The second of two CTAs may have no rows: it goes through the last ones' again.)
  auto source = [&](int iw) { return a.w + w4_place(8ll * min(iw, (a.n - 1) / NO), k0, a.kb) * WB; };
  // While the kernel before this one ends, the first codes come as far as L2, which has them right whoever writes them.
  if (threadIdx.x == 32) {
    int iw, m0, wd;
    tile(first, iw, m0, wd);
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(source(iw)), "r"(min(CS, k1 - k0) * 8 * WB) : "memory");
  }
  if (CG == 2 || ks > 1) cluster_sync_all();   // the partners' shared memory is there
  grid_dep_wait();
  grid_dep_launch();

  // An arrival on a barrier of the CTA that issues the MMAs.  What it tells of is tensor memory, which the tcgen05 fences
  // order; a release of the cluster's scope, for all other memory, took 1600 cycles beside the loads.
  auto tell = [&](uint32_t bar) {
    if (CG == 2) asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(mapa_shared(bar, 0)) : "memory");
    else mbar_arrive(bar);
  };

  if (warp < kW4Expand) {
    const int q = warp & 3, h = (warp >> 2) & 1, odd = warp >> 3;
    constexpr int NP = G == 32 ? 2 : 1;   // groups in 64 columns
    const uint32_t tl = tmem + kW4ACol + 32 * h + ((uint32_t)(q * 32) << 16);
    // this warp's blocks are every other one of all that the CTA goes through
    const uint32_t turns = first < r.tiles ? (r.tiles - first + step - 1) / step : 0, total = turns * (k1 - k0);
    uint4 w[2];
    uint2 p[2][NP];
    bool ok = true;
    uint32_t slot = odd % CS, ph = odd / CS & 1;
    auto fetch = [&] {
      if (!__all_sync(0xffffffffu, mbar_wait(cfull(slot), ph))) { ok = false; return; }
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const uint8_t* c = codes + (slot * 8 + 2 * q + b) * WB;
        w[b] = *(const uint4*)(c + 512 * h + 16 * lane);
#pragma unroll
        for (int i = 0; i < NP; ++i) p[b][i] = *(const uint2*)(c + 1024 + 64 * (h * 64 / G + i) + 8 * (lane / 4));
      }
    };
    uint32_t v[2][2][8];
    auto convert = [&](auto fast) {
      constexpr bool FAST = decltype(fast)::value;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const uint32_t words[4] = {w[b].x, w[b].y, w[b].z, w[b].w};
        uint32_t s[2], m[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (j < NP) w4_params(p[b][j], s, m);
          w4_expand<BF, FAST>(words[2 * j], s, m, v[b][j]);
          w4_expand<BF, FAST>(words[2 * j + 1], s, m, v[b][j] + 4);
        }
      }
    };
    const bool large = *a.large != 0;
    auto expand = [&] {
      fetch();
      if (large) convert(std::false_type());
      else convert(std::true_type());
      __syncwarp();
      if (lane == 0) mbar_arrive(cempty(slot));
      if ((slot += 2) >= CS) slot -= CS, ph ^= 1;
    };
    if (odd < total) expand();
    for (uint32_t it = odd; it < total && ok; it += 2) {
      if (it >= AS && !__all_sync(0xffffffffu, mbar_wait(done((it - AS) % NB), (it - AS) / NB & 1))) break;
      tc_fence_after();
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          tmem_st_frag(tl + 64 * (it % AS) + ((uint32_t)(16 * b) << 16) + 16 * j, v[b][j]);
      // the stores wait for their turn beside the MMAs: the next block is expanded meanwhile
      if (it + 2 < total) expand();
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) tell(full(it % NB));
    }
  } else if (warp == kW4Expand) {   // x
    int it = 0, s = 0;
    bool ok = true;
    for (int t = first; t < r.tiles && ok; t += step) {
      int iw, m0, wd;
      tile(t, iw, m0, wd);
      const int rows = wd / CG, box = r.bn / (CG == 2 ? 4 : 1);
      m0 += rank * (CG == 2 ? rows : 0);
      for (int k = k0; k < k1; ++k, ++it) {
        if (it >= ST && !__all_sync(0xffffffffu, mbar_wait(done((it - ST) % NB), (it - ST) / NB & 1))) { ok = false; break; }
        if (elect_one()) {
          const uint32_t bar = CG == 2 ? mapa_shared(full(it % NB), 0) : full(it % NB);
          if (CG == 1 || rank == 0) mbar_arrive_expect_tx(full(it % NB), wd * 256);
          for (int u = 0; u < 2; ++u)
            for (int c = 0; c < rows; c += box)
              w4_load_x<CG>(base + s * xb + u * half + c * 128, &tx, bar, k * 128 + 64 * u, m0 + c);
        }
        __syncwarp();
        if (++s == ST) s = 0;
      }
    }
    // what was loaded has landed, and in the end been read, before the block may exit
    for (int i = it - ST < 0 ? 0 : it - ST; i < it; ++i) mbar_wait(ok ? done(i % NB) : full(i % NB), i / NB & 1);
  } else if (warp == kW4Expand + 1) {   // codes and parameters
    int it = 0, s = 0, ph = 1;
    bool ok = true;
    for (int t = first; t < r.tiles && ok; t += step) {
      int iw, m0, wd;
      tile(t, iw, m0, wd);
      const uint8_t* from = source(iw);
      for (int k = k0; k < k1; ++k, ++it, from += 8 * WB) {
        if (!__all_sync(0xffffffffu, mbar_wait(cempty(s), ph))) { ok = false; break; }
        if (elect_one()) {
          mbar_arrive_expect_tx(cfull(s), 8 * WB);
          bulk_copy_g2s(cbase + s * 8 * WB, from, 8 * WB, cfull(s));
        }
        __syncwarp();
        if (++s == CS) s = 0, ph ^= 1;
      }
    }
    for (int i = it - CS < 0 ? 0 : it - CS; i < it; ++i) mbar_wait(ok ? cempty(i % CS) : cfull(i % CS), i / CS & 1);
  } else if (warp == kW4Expand + 2) {   // MMAs: one thread, of the first CTA where there are two
    if ((CG == 1 || rank == 0) && elect_one()) {
      uint32_t it = 0, nt = 0;
      int s = 0;
      bool ok = true;
      for (int t = first; t < r.tiles && ok; t += step) {
        const uint32_t idesc = idesc_f16_f32(128 * CG, CG == 2 && t >= r.whole ? r.bn / 2 : r.bn, BF);
        for (int kc = k0; kc < k1 && ok; kc += r.chain, ++nt) {   // a chain an accumulator
          const uint32_t acc = accs == 2 ? nt & 1 : 0, use = nt / accs, td = tmem + acc * 128;
          if (use && !(CG == 2 ? mbar_wait_cluster(dempty(acc), (use - 1) & 1) : mbar_wait(dempty(acc), (use - 1) & 1))) {
            ok = false;
            break;
          }
          const int end = min(kc + r.chain, k1);
          for (int k = kc; k < end; ++k, ++it) {
            const uint32_t bar = full(it % NB), ph = it / NB & 1;
            if (!(CG == 2 ? mbar_wait_cluster(bar, ph) : mbar_wait(bar, ph))) { ok = false; break; }
            tc_fence_after();
            const uint64_t db = sdesc_sw128(base + s * xb);
            const uint32_t ta = tmem + kW4ACol + 64 * (it % AS);
#pragma unroll
            for (int j = 0; j < 8; ++j)   // 16 columns of k: 8 of tensor memory, two 16-byte units of the descriptor's address
              w4_mma<CG>(td, ta + 8 * j, db + 2 * (j & 3) + (j >> 2) * (half / 16), idesc, (k > kc) | (j > 0));
            w4_commit<CG>(done(it % NB));
            if (k + 1 == end) w4_commit<CG>(dfull(acc));
            if (++s == ST) s = 0;
          }
        }
      }
    }
    __syncwarp();
  } else if (warp >= kW4Out) {   // results
    // a quadrant of 32 lanes and every other 16 columns a warp
    const int q = warp & 3, row = q * 32 + lane, e = (lane >> 3) & 1, first_col = 16 * ((warp - kW4Out) >> 2);
    // a lane's column of out in its tile; a gated pair's lanes with bit 3 clear hold the gate's rows, and do the even
    // columns, the others the odd ones
    const int nc = GATED ? q * 16 + (lane >> 4) * 8 + (lane & 7) : row;
    auto pair = [&](const uint32_t* v, int i) {
      const float mine = __uint_as_float(e ? v[i + 1] : v[i]);
      const float other = __uint_as_float(__shfl_xor_sync(0xffffffffu, e ? v[i] : v[i + 1], 8));
      return w4_act(a.act, e ? other : mine) * (e ? mine : other);
    };
    uint32_t nt = 0;
    bool ok = true;
    for (int t = first; t < r.tiles; t += step, ++nt) {
      int iw, m0, wd;
      tile(t, iw, m0, wd);
      // the sums of all chains but the last: a thread's own row, so nothing waits for others
      float* sums = (float*)(turn + (ks > 1 ? w4_many_recv(r.bn, ks) : 0)) + row;
      bool some = false;
      for (int kc = k0 + r.chain; kc < k1 && ok; kc += r.chain, ++nt, some = true) {
        const uint32_t acc = accs == 2 ? nt & 1 : 0, tl = tmem + acc * 128 + ((uint32_t)(q * 32) << 16);
        ok = __all_sync(0xffffffffu, mbar_wait(dfull(acc), (nt / accs) & 1));
        tc_fence_after();
        for (int c0 = first_col; c0 < wd; c0 += 32) {
          uint32_t v[16];
          tmem_ld<16>(tl + c0, v);
#pragma unroll
          for (int i = 0; i < 16; ++i) sums[(c0 + i) * 128] = __uint_as_float(v[i]) + (some ? sums[(c0 + i) * 128] : 0.0f);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) tell(dempty(acc));
      }
      const uint32_t acc = accs == 2 ? nt & 1 : 0, tl = tmem + acc * 128 + ((uint32_t)(q * 32) << 16);
      const int n0 = iw * NO, n = n0 + nc;
      auto release = [&] {   // the accumulator has been read
        tc_fence_before();
        __syncwarp();
        if (lane == 0) tell(dempty(acc));
      };
      if (CG == 2 && a.out_type != IFQ_F32) {
        // through shared memory: rows of out in pieces of 16 bytes, before (the residual) and after
        const int id = threadIdx.x - 32 * kW4Out, wide = min(NO, a.n - n0), tall = min(wd, a.m - m0);
        auto move = [&](bool in) {
          if (r.vec) {
            for (int i = id; i < tall * (NO / 8); i += 32 * kW4Outs) {
              const int c = i / (NO / 8), j = i % (NO / 8) * 8;
              uint4* to = (uint4*)(turn + c * PITCH + 2 * j);
              if (j < wide) {
                if (in) *to = *(const uint4*)((const uint16_t*)a.res + (m0 + c) * a.res_stride + n0 + j);
                else *(uint4*)((uint16_t*)a.out + (m0 + c) * a.out_stride + n0 + j) = *to;
              }
            }
          } else {
            for (int i = id; i < tall * NO; i += 32 * kW4Outs) {
              const int c = i / NO, j = i % NO;
              uint16_t* to = (uint16_t*)(turn + c * PITCH + 2 * j);
              if (j < wide) {
                if (in) *to = ((const uint16_t*)a.res)[(m0 + c) * a.res_stride + n0 + j];
                else ((uint16_t*)a.out)[(m0 + c) * a.out_stride + n0 + j] = *to;
              }
            }
          }
          named_bar(1, 32 * kW4Outs);
        };
        if (!GATED && a.res) move(true);
        // (a wait that ran out: the warps still meet at every named barrier)
        ok = ok && __all_sync(0xffffffffu, mbar_wait(dfull(acc), (nt / accs) & 1));
        tc_fence_after();
        if (first_col >= wd) release();
        for (int c0 = first_col; c0 < wd; c0 += 32) {
          if constexpr (GATED) {   // as fragments: rows g and g + 8, a gate's and its other's, are in one thread
            uint32_t v[2][8];
            tmem_ld_frag(tl + c0, v);
            if (c0 + 32 >= wd) release();
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const int h = j >> 3, k = (j >> 2) & 1, i = j & 1;
              if (j & 2) continue;
              const float y = w4_act(a.act, __uint_as_float(v[h][4 * k + i])) * __uint_as_float(v[h][4 * k + 2 + i]);
              w4_store(BF ? IFQ_BF16 : IFQ_F16, turn + (c0 + 8 * k + 2 * (lane & 3) + i) * PITCH, q * 16 + 8 * h + lane / 4, y);
            }
          } else {
            uint32_t v[16];
            tmem_ld<16>(tl + c0, v);
            if (c0 + 32 >= wd) release();
            uint8_t* to = turn + c0 * PITCH;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float add = a.res ? w4_load(a.out_type, to + i * PITCH, nc) : 0.0f;
              w4_store(a.out_type, to + i * PITCH, nc, __uint_as_float(v[i]) + add);
            }
          }
        }
        named_bar(1, 32 * kW4Outs);
        move(false);
        continue;
      }
      float add[16], next[16];   // the residual, loaded 16 columns ahead
      auto residual = [&](int c0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int m = m0 + c0 + i;
          next[i] = c0 < wd && m < a.m && n < a.n ? w4_load(a.out_type, a.res, m * a.res_stride + n) : 0.0f;
        }
      };
      if (!GATED && a.res && ks == 1) residual(first_col);
      if (!__all_sync(0xffffffffu, mbar_wait(dfull(acc), (nt / accs) & 1))) break;
      tc_fence_after();
      if (CG == 1 && ks > 1) {
        const int per = (r.bn + ks - 1) / uks;
        for (int c0 = first_col; c0 < r.bn; c0 += 32) {
          uint32_t v[16];
          tmem_ld<16>(tl + c0, v);
          if (some)
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + sums[(c0 + i) * 128]);
          // owner of column c: own bn / ks <= c < end
          int own = ((c0 + 1) * uks - 1) / r.bn, end = (own + 1) * r.bn / uks;
          uint32_t to = mapa_shared(smem_u32(recv + (int)(rank * per - own * r.bn / uks) * 129 + row), own);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int c = c0 + i;
            if (c == end) {
              to = mapa_shared(smem_u32(recv + (rank * per - end) * 129 + row), ++own);
              end = (own + 1) * r.bn / uks;
            }
            asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(to + c * 129 * 4), "r"(v[i]) : "memory");
          }
        }
        break;
      }
      if (first_col >= wd) release();
      for (int c0 = first_col; c0 < wd; c0 += 32) {
        uint32_t v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) add[i] = next[i];
        if (!GATED && a.res) residual(c0 + 32);
        tmem_ld<16>(tl + c0, v);
        if (c0 + 32 >= wd) release();
        if (!GATED && some)
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + sums[(c0 + i) * 128]);
        if constexpr (GATED) {
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            const float y = pair(v, i);
            const int m = m0 + c0 + i + e;
            if (m < a.m && n < a.n) w4_store(BF ? IFQ_BF16 : IFQ_F16, a.out, m * a.out_stride + n, y);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int m = m0 + c0 + i;
            const float y = __uint_as_float(v[i]) + (a.res ? add[i] : 0.0f);
            if (m < a.m && n < a.n) w4_store(a.out_type, a.out, m * a.out_stride + n, y);
          }
        }
      }
    }
  }
  if (CG == 1 && ks > 1) {
    __syncwarp();
    cluster_sync_all();   // every partial sum has arrived
    int iw, m0, wd;
    tile(first, iw, m0, wd);
    const int lo = rank * r.bn / uks, wide = (rank + 1) * r.bn / uks - lo, per = (r.bn + ks - 1) / uks;
    const int total = NO * wide;
    for (int i = threadIdx.x; i < total; i += kW4ManyThreads) {
      const int c = i / NO, j = i % NO, m = m0 + lo + c;
      const int n = iw * NO + j, row = GATED ? j / 8 * 16 + j % 8 : j;
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
  if (CG == 2) cluster_sync_all();   // neither CTA's memory is used by the other any more
  if (warp == 0) w4_dealloc<CG>(tmem);
}

}  // namespace ifq
