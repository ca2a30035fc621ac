// Products in e4m3 with a float scale for each block of 128 along k, and the quantiser of their
// activations.
#pragma once
#include <cuda.h>

#include "kv4.cuh"
#include "tmem.cuh"

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

// Eight values (16 bytes) a lane, 16 lanes a block, kFp8Pass times two blocks in a row a warp, their loads all under way
// before the first is used (k is a multiple of 16, so a lane's eight are all there or none).  blockIdx.x: eight rows,
// blockIdx.y: blocks along k.  29 us, 3.9 TB/s, for 4096 x 9216, with 70 % of the issue slots: neither memory nor the eight
// divisions bound it (quotients by an inverse were no faster), but warps that load once and end.  (A block a warp: 50.)
constexpr int kFp8Pass = 4;

template <bool BF>
__global__ void __launch_bounds__(32 * kFp8QuantWarps) fp8_quantize_kernel(const __grid_constant__ Fp8QuantArgs a) {
  grid_dep_wait();
  grid_dep_launch();
  const int r = blockIdx.x * kFp8QuantWarps + (threadIdx.x >> 5);
  if (r >= a.m) return;
  const int lane = threadIdx.x & 31, b0 = blockIdx.y * 2 * kFp8Pass + lane / 16, c0 = (lane % 16) * 8;
  const uint16_t* x = a.x + r * a.x_stride;
  uint8_t* codes = a.codes + (long long)r * a.k;
  uint32_t w[kFp8Pass][4];
#pragma unroll
  for (int u = 0; u < kFp8Pass; ++u) {
    const long long c = (long long)(b0 + 2 * u) * kFp8Block + c0;
    w[u][0] = w[u][1] = w[u][2] = w[u][3] = 0;
    if (c < a.k) load_words(w[u], x + c);
  }
#pragma unroll
  for (int u = 0; u < kFp8Pass; ++u) {
    const int b = b0 + 2 * u;
    float v[8], top = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = unpack16<BF>(w[u][i]);
      v[2 * i] = f.x;
      v[2 * i + 1] = f.y;
      top = max_nan(top, max_nan(fabsf(f.x), fabsf(f.y)));
    }
#pragma unroll
    for (int o = 8; o; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float s = __fmul_rn(top, 1.0f / 448.0f);
    uint32_t out[2] = {0, 0};
    if (s != 0.0f) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        out[i] = e4m3x2(__fdiv_rn(v[4 * i], s), __fdiv_rn(v[4 * i + 1], s)) |
                 e4m3x2(__fdiv_rn(v[4 * i + 2], s), __fdiv_rn(v[4 * i + 3], s)) << 16;
    }
    const long long c = (long long)b * kFp8Block + c0;
    if (c < a.k) store_words(codes + c, out);
    if (lane % 16 == 0 && b < a.kb) a.scales[(long long)b * a.m + r] = s;
    __syncwarp();
  }
}

// ---------------------------------------------------------------- the product
//
// One tcgen05.mma tile: 128 rows of operand A (tensor-memory lanes) x BN rows of operand B (columns).
// Where there are many rows of x, A is x and B is w; with few (SWAP) A is w, so that the weights, which
// are then what is read, fill the lanes, and the rows of x are as few columns as 16.
//
// A block of 128 along k is one pipeline stage and one tensor-memory accumulator (two or four take turns): its
// sum has scales of its own, so it leaves tensor memory for registers, where the tile's sum is kept:
//   acc += (x_scale w_scale) * block      (one fma an element; the factor is a lane's own, or with SWAP
//                                          a column's).
// Warps: eight that promote and store (32 lanes x half the columns each), one that loads (TMA, 128-byte
// swizzle), two that issue MMAs, every other block each (one alone took 650 cycles a block, whatever BN).
//
// A tile's k may be split over a cluster of ks blocks: each sends its partial columns to the block that
// owns them through distributed shared memory, which adds them in the order of the ranks.
//
// Where BN = 256 a block's 128 sums a thread and two loads from tensor memory under way take more registers than three
// warps a scheduler may have, so the warpgroups divide them anew; and where the tiles of the last turn fill half of the
// SMs or less, they are cut in two (1300 x 4096 x 4096 with both: 36.4 -> 31.5 us, 4096 x 4096 x 1024 32.2 -> 28.8).
//
// Measured with many rows: 4096 x 4096 x 9216 in 138 us, 2.2 PFLOP/s.  Without the promotion it takes 117, with a quarter of
// the MMAs as long; tiles of 256 x 256 on two SMs, with two thirds of the bytes from L2, took 141.  With few rows the
// launch, the cluster's join and a block's way through the pipeline (425 cycles) count: 1 x 4096 x 9216 in 10.8 us
// with the quantiser where the weights stand in L2, 13 us where two matrices take turns.
struct Fp8Args {
  const float *xs, *ws;
  void* out;
  long long out_stride;
  int m, n, kb, out_type, vec;   // vec: 16-byte stores are aligned
  int tiles, tiles_a, tiles_b, ks;   // items in all, tiles of A and of B; blocks a tile's k is split over
  int whole;                         // items that are whole tiles; the rest are halves (BN = 256)
};

constexpr int kFp8Promote = 8;
// Registers a thread of the promoting warpgroups and of the other one where BN = 256: 2 x 128 x 216 + 128 x 72 =
// 384 x 168, what the block is launched with.
constexpr int kFp8MoreRegs = 216, kFp8FewRegs = 72;

template <int BN, bool SWAP>
struct Fp8Shape {
  static constexpr bool wide = BN == 256;
  static constexpr int stage = 16384 + BN * 128;
  static constexpr bool split = BN < 256;
  static constexpr int threads = 32 * (kFp8Promote + (wide ? 4 : 3));   // (the last warp makes a whole warpgroup)
  // a receive slot a rank: the owner's columns, 129 floats each; or 32 x 32 results a warp on their way out
  static constexpr int recv = split ? (BN + 8) * 129 * 4 : kFp8Promote * 32 * 33 * 4;
  static constexpr int fac = SWAP ? kFp8Promote * 2 * (BN / 2) * 4 : 0;   // the columns' factors, two a warp
  static constexpr int fit = (232448 - 1024 - 1024 - recv - fac) / stage;
  static constexpr int stages = fit < 8 ? fit : 8;
  static constexpr int bytes = 1024 + stages * stage + recv + fac + 256;
  static constexpr int acc = BN <= 64 ? 4 : 2;              // accumulators
  static constexpr int cols = acc * BN;                     // tensor memory
  static_assert(bytes <= 232448 && stages >= 3, "shared memory budget");
};

// Two steps, for work beside the load; between them nothing may read v, and what does after them is volatile.
__device__ __forceinline__ void tmem_ld_begin(uint32_t t, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(t)
      : "memory");
}
__device__ __forceinline__ void tmem_ld_end() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fma2_after(uint64_t& c, uint32_t a0, uint32_t a1, float f) {
  asm volatile("{.reg .b64 a, f; mov.b64 a, {%1, %2}; mov.b64 f, {%3, %3}; fma.rn.f32x2 %0, a, f, %0;}"
               : "+l"(c)
               : "r"(a0), "r"(a1), "f"(f));
}
__device__ __forceinline__ void fma2(uint64_t& c, uint32_t a0, uint32_t a1, float f0, float f1) {
  uint64_t a, f;
  asm("mov.b64 %0, {%1, %2};" : "=l"(a) : "r"(a0), "r"(a1));
  asm("mov.b64 %0, {%1, %2};" : "=l"(f) : "f"(f0), "f"(f1));
  asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(c) : "l"(a), "l"(f));
}
__device__ __forceinline__ float2 halves2(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ void fp8_store(const Fp8Args& a, long long at, float v) {
  if (a.out_type == IFQ_F32) ((float*)a.out)[at] = v;
  else if (a.out_type == IFQ_F16) ((__half*)a.out)[at] = __float2half_rn(v);
  else ((__nv_bfloat16*)a.out)[at] = __float2bfloat16_rn(v);
}
__device__ __forceinline__ uint32_t fp8_pack(int type, float a, float b) {
  return type == IFQ_F16 ? pack16<false>(a, b) : pack16<true>(a, b);
}

template <int BN, bool SWAP>
__global__ void __launch_bounds__((Fp8Shape<BN, SWAP>::threads), 1)
    fp8_matmul_kernel(const __grid_constant__ CUtensorMap ta, const __grid_constant__ CUtensorMap tb, const __grid_constant__ Fp8Args a) {
  using C = Fp8Shape<BN, SWAP>;
  constexpr int ST = C::stages, NA = C::acc, HC = BN / 2;   // columns a thread
  constexpr bool WIDE = C::wide;
  constexpr int LD = HC < 32 ? HC : 32;                      // columns a load with SWAP
  extern __shared__ uint8_t raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
  const uint32_t base = smem_u32(smem);
  float* recv = (float*)(smem + ST * C::stage);
  float* fac = (float*)(smem + ST * C::stage + C::recv);
  const uint32_t bars = base + ST * C::stage + C::recv + C::fac;
  auto full = [&](int s) { return bars + 8 * s; };
  auto empty = [&](int s) { return bars + 8 * (ST + s); };
  auto dfull = [&](int b) { return bars + 8 * (2 * ST + b); };
  auto dempty = [&](int b) { return bars + 8 * (2 * ST + NA + b); };
  uint32_t* tptr = (uint32_t*)(smem + ST * C::stage + C::recv + C::fac + 8 * (2 * ST + 2 * NA));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int ks = a.ks, rank = ks > 1 ? (int)cluster_ctarank() : 0;
  if (threadIdx.x == 0) {
    for (int i = 0; i < ST; ++i) {
      mbar_init(full(i), 1);
      mbar_init(empty(i), 1);
    }
    for (int b = 0; b < NA; ++b) {
      mbar_init(dfull(b), 1);
      mbar_init(dempty(b), kFp8Promote);
    }
    fence_mbar_init();
    prefetch_tmap(&ta);
    prefetch_tmap(&tb);
  }
  if (warp == 0) {
    tmem_alloc(smem_u32(tptr), C::cols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tptr;
  if (ks > 1) cluster_sync_all();   // the partners' shared memory is there
  grid_dep_wait();
  grid_dep_launch();

  // (32-bit divisions: 64-bit ones took 1400 cycles before the first load)
  const uint32_t uks = ks;
  const int k0 = (uint32_t)(rank * a.kb) / uks, k1 = (uint32_t)((rank + 1) * a.kb) / uks;
  const int first = blockIdx.x / uks, step = gridDim.x / uks;
  // Item t: columns n0 to n0 + wd of the tile's rows of A, 128 ia.  Tiles in groups of 16 tiles of A, within a group along A
  // first; from tile a.whole on, halves of tiles.
  auto tile = [&](uint32_t t, int& ia, int& n0, int& wd) {
    wd = BN;
    uint32_t odd = 0;
    if (WIDE && t >= (uint32_t)a.whole) {
      odd = (t - a.whole) & 1;
      t = a.whole + (t - a.whole) / 2;
      wd = BN / 2;
    }
    const uint32_t g = t / (16u * a.tiles_b), in = t - g * 16u * a.tiles_b, wide = min(16u, a.tiles_a - 16u * g), ib = in / wide;
    ia = 16 * g + in - ib * wide;
    n0 = ib * BN + odd * (BN / 2);
  };

  if (warp >= kFp8Promote) {
    if constexpr (WIDE) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFp8FewRegs));
  if (warp == kFp8Promote) {
    int it = 0;
    bool ok = true;
    for (int t = first; t < a.tiles && ok; t += step) {
      int ia, n0, wd;
      tile(t, ia, n0, wd);
      for (int k = k0; k < k1; ++k, ++it) {
        const int s = it % ST;
        if (it >= ST && !__all_sync(0xffffffffu, mbar_wait(empty(s), (it / ST - 1) & 1))) { ok = false; break; }
        if (elect_one()) {
          mbar_arrive_expect_tx(full(s), 16384 + 128 * wd);
          tma_load_2d(base + s * C::stage, &ta, full(s), k * kFp8Block, ia * 128);
          tma_load_2d(base + s * C::stage + 16384, &tb, full(s), k * kFp8Block, n0);
          if (WIDE && wd == BN) tma_load_2d(base + s * C::stage + 32768, &tb, full(s), k * kFp8Block, n0 + 128);
        }
        __syncwarp();
      }
    }
    // what was loaded has landed, and in the end been read, before the block may exit
    for (int i = it - ST < 0 ? 0 : it - ST; i < it; ++i) mbar_wait(ok ? empty(i % ST) : full(i % ST), (i / ST) & 1);
  } else if (warp <= kFp8Promote + 2) {
    const int parity = warp - kFp8Promote - 1;
    int it = 0;
    bool ok = true;
    for (int t = first; t < a.tiles && ok; t += step) {
      const uint32_t idesc = WIDE && t >= a.whole ? idesc_e4m3_f32(128, BN / 2) : idesc_e4m3_f32(128, BN);
      for (int k = k0; k < k1; ++k, ++it) {
        if ((it & 1) != parity) continue;
        const int s = it % ST, b = it % NA;
        if (!__all_sync(0xffffffffu, mbar_wait(full(s), (it / ST) & 1)) ||
            (it >= NA && !__all_sync(0xffffffffu, mbar_wait(dempty(b), (it / NA - 1) & 1)))) { ok = false; break; }
        tc_fence_after();
        if (elect_one()) {
          const uint64_t da = sdesc_sw128(base + s * C::stage), db = sdesc_sw128(base + s * C::stage + 16384);
#pragma unroll
          for (int j = 0; j < kFp8Block / 32; ++j)   // 32 bytes along k: two 16-byte units of the descriptors' address
            mma_e4m3(tmem + b * BN, da + 2 * j, db + 2 * j, idesc, j > 0);
          mma_commit(empty(s));
          mma_commit(dfull(b));
        }
        __syncwarp();
      }
    }
  }
  } else {
    if constexpr (WIDE) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kFp8MoreRegs));
    const int quad = warp & 3, half = warp >> 2, row = quad * 32 + lane;
    const uint32_t tl = tmem + ((uint32_t)(quad * 32) << 16);
    int it = 0;
    bool ok = true;
    for (int t = first; t < a.tiles && ok; t += step) {
      int ia, n0, wd;
      tile(t, ia, n0, wd);
      const int hc = WIDE ? wd / 2 : HC, c0 = half * hc;   // this thread's columns
      uint64_t acc[HC / 2];
#pragma unroll
      for (int i = 0; i < HC / 2; ++i) acc[i] = 0;
      // the factors of block k: a thread's own row of x and its columns' 128 rows of w; with SWAP its row of w, and
      // lane c of a warp has column c0 + c's (and c0 + 32 + c's) of x
      // (past the operands' ends the last row's, for results that are not stored: no load waits for a condition)
      const int wb = min(SWAP ? ia : (n0 + c0) / 128, (a.n - 1) / 128);
      const int xr = min(SWAP ? n0 + c0 + lane : ia * 128 + row, a.m - 1);
      const float* xp = a.xs + xr;
      const float* wp = a.ws + (long long)wb * a.kb;
      // (the next block's, loaded a block ahead and multiplied only when that block is there: a product that moves up to
      // the loads waits for them)
      float xn = xp[(long long)k0 * a.m], wn = wp[k0];
      for (int k = k0; k < k1; ++k, ++it) {
        const int b = it % NA;
        if (!__all_sync(0xffffffffu, mbar_wait(dfull(b), (it / NA) & 1))) { ok = false; break; }
        tc_fence_after();
        asm volatile("" : "+f"(xn), "+f"(wn));
        const float f = xn * wn;
        const int kn = min(k + 1, k1 - 1);
        xn = xp[(long long)kn * a.m];
        wn = wp[kn];
        float* fw = fac + (warp * 2 + (it & 1)) * HC;
        if constexpr (SWAP) {
          if (lane < HC) fw[lane] = f;
          __syncwarp();
        }
        auto release = [&] {   // the accumulator has been read
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(dempty(b));
        };
        if constexpr (!SWAP) {   // the next columns are on their way while these are added
          constexpr int NC = HC / 16;
          uint32_t v[2][16];
          tmem_ld_begin(tl + b * BN + c0, v[0]);
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            tmem_ld_end();
            const bool last = c + 1 == NC || (WIDE && 16 * (c + 1) == hc);
            if (last) release();
            else tmem_ld_begin(tl + b * BN + c0 + 16 * (c + 1), v[(c + 1) & 1]);
#pragma unroll
            for (int i = 0; i < 8; ++i) fma2_after(acc[8 * c + i], v[c & 1][2 * i], v[c & 1][2 * i + 1], f);
            if (last) break;
          }
        } else {
#pragma unroll
          for (int c = 0; c < HC; c += LD) {
            uint32_t v[LD];
            tmem_ld<LD>(tl + b * BN + c0 + c, v);
            if (c + LD == HC) release();
#pragma unroll
            for (int i = 0; i < LD; i += 4) {
              const float4 g = *(const float4*)(fw + c + i);
              fma2(acc[(c + i) / 2], v[i], v[i + 1], g.x, g.y);
              fma2(acc[(c + i) / 2 + 1], v[i + 2], v[i + 3], g.z, g.w);
            }
          }
        }
      }
      if (!ok) break;
      if (C::split && ks > 1) {
        const int per = (BN + ks - 1) / uks;
        int own = ((c0 + 1) * uks - 1) / BN, end = (own + 1) * BN / uks;   // owner of column c: own BN / ks <= c < end
        auto slot = [&](int lo) { return mapa_shared(smem_u32(recv + (rank * per - lo) * 129 + row), own); };
        uint32_t to = slot(own * BN / uks);
#pragma unroll
        for (int i = 0; i < HC; ++i) {
          const int c = c0 + i;
          if (c == end) {
            to = (++own, slot(end));
            end = (own + 1) * BN / uks;
          }
          const float2 v = halves2(acc[i / 2]);
          asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + c * 129 * 4), "f"(i & 1 ? v.y : v.x) : "memory");
        }
        break;
      }
      if constexpr (SWAP) {
        const int n = ia * 128 + row;
        if (n < a.n) {
#pragma unroll
          for (int i = 0; i < HC / 2; ++i) {
            const float2 v = halves2(acc[i]);
            const int m = n0 + c0 + 2 * i;
            if (m < a.m) fp8_store(a, (long long)m * a.out_stride + n, v.x);
            if (m + 1 < a.m) fp8_store(a, (long long)(m + 1) * a.out_stride + n, v.y);
          }
        }
      } else if (!a.vec) {
        // rows that start anywhere: 32 columns at a time through shared memory, so that a warp's stores are a row's
        float* turn = recv + warp * 32 * 33;
        const int m0 = ia * 128 + quad * 32;
#pragma unroll
        for (int i = 0; i < HC; i += 32) {
          if (WIDE && i == hc) break;
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            const float2 v = halves2(acc[(i + j) / 2]);
            turn[lane * 33 + j] = v.x;
            turn[lane * 33 + j + 1] = v.y;
          }
          __syncwarp();
          const int n = n0 + c0 + i + lane;
          const int rows = min(32, a.m - m0);
          if (n < a.n)
#pragma unroll 8
            for (int r = 0; r < rows; ++r) fp8_store(a, (long long)(m0 + r) * a.out_stride + n, turn[r * 33 + lane]);
          __syncwarp();
        }
      } else {
        const int m = ia * 128 + row, n = n0 + c0;
        if (m < a.m) {
#pragma unroll
          for (int i = 0; i < HC; i += 8) {
            if (WIDE && i == hc) break;
            const long long at = (long long)m * a.out_stride + n + i;
            float2 v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = halves2(acc[i / 2 + j]);
            if (n + i + 8 <= a.n) {
              if (a.out_type == IFQ_F32) {
                *(float4*)((float*)a.out + at) = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
                *(float4*)((float*)a.out + at + 4) = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
              } else {
                *(uint4*)((uint16_t*)a.out + at) =
                    make_uint4(fp8_pack(a.out_type, v[0].x, v[0].y), fp8_pack(a.out_type, v[1].x, v[1].y),
                               fp8_pack(a.out_type, v[2].x, v[2].y), fp8_pack(a.out_type, v[3].x, v[3].y));
              }
            } else {
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                if (n + i + 2 * j < a.n) fp8_store(a, at + 2 * j, v[j].x);
                if (n + i + 2 * j + 1 < a.n) fp8_store(a, at + 2 * j + 1, v[j].y);
              }
            }
          }
        }
      }
    }
  }
  if (C::split && ks > 1) {
    __syncwarp();
    cluster_sync_all();   // every partial sum has arrived
    if (warp < kFp8Promote) {
      int ia, n0, wd;
      tile(first, ia, n0, wd);
      const int lo = rank * BN / uks, hi = (rank + 1) * BN / uks, wide = hi - lo, per = (BN + ks - 1) / uks;
      // Out rows are contiguous along w's rows: those are the lanes (SWAP) or the columns.  Eight outputs a thread at a
      // time, so that their loads are under way together.
      const int total = 128 * wide;
      for (int i0 = threadIdx.x; i0 < total; i0 += 8 * 32 * kFp8Promote) {
        float v[8];
        int r[8], c[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int i = min(i0 + j * 32 * kFp8Promote, total - 1);
          r[j] = SWAP ? i % 128 : i / (uint32_t)wide;
          c[j] = SWAP ? i / 128 : i - r[j] * wide;
          v[j] = 0.0f;
        }
        for (int p = 0; p < ks; ++p)
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] += recv[(p * per + c[j]) * 129 + r[j]];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int m = SWAP ? n0 + lo + c[j] : ia * 128 + r[j], n = SWAP ? ia * 128 + r[j] : n0 + lo + c[j];
          if (i0 + j * 32 * kFp8Promote < total && m < a.m && n < a.n) fp8_store(a, (long long)m * a.out_stride + n, v[j]);
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, C::cols);
}

}  // namespace ifq
