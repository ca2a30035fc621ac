// Attention of many query rows per sequence over the paged 4-bit cache (chunks of a prompt), on tcgen05.
//
// A block takes 128 RT rows of a key head (query tokens x the heads that share it) and their keys in tiles of 128:
//   S[row][key] = sum_d q[row][d] c[key][d]    (half x half, both operands in shared memory),
//   O[row][d]  += sum_key p[row][key] v[key][d] (p from tensor memory, over S's columns; v in shared memory).
// Bound by the tensor cores' half rate in the limit, by the chain of product, softmax and product of a tile as measured:
// 2 x 2048 queries of 32 heads of 128 on 8192 tokens each in 656 us (bfloat16; half 840), 0.73 PFLOP/s, with 36 % of the
// tensor pipe and 40 % of the issue slots.
//
// Keys: codes are expanded to halves as the subnormals c 2^-24 and 16 c 2^-24 (masks alone, as in kv4_rows.cuh; q's
// elements stand in the order that leaves the codes of a word in, with the factors 1/16 in them).  Products with them
// are exact, sums fp32; the scale and the minimum of a key are applied to the sum,
//   t = s (q . c) + (m sum(q) - reference),   two packed fma a pair of keys (scale, log2 e and powers of two in s).
// q itself is multiplied by 16 to keep small elements out of the half's subnormals; a row with an element over 2^11 is
// brought down by a power of two of its own, which its scores are then multiplied with (a branch no usual row takes).
// Values: where rows are bfloat16, v = half(s' (c' / 2) + m' / 2), one fma of halves: eight times finer than the result, as
// fine as the minimum that the cache holds (a half), and within the half's range where s' c' + m' would leave it.  Where
// rows are half the product takes c' - 8, exact, and the scale goes into the weight's exponent, w = 2^(t - m + log2 s');
// then sum p = sum w / s', and the values of code 8, m'' = m' + 8 s', are added in fp32, sum w m'' / s'.  (The rounding of
// v would be as large as that of the result.)  Both sums take w as the product has it, rounded, so that what it loses is
// 2^-11 of v.  A value far from 0 beside its scale (a constant one: s' = 0) would have a weight that vanishes as a half while
// m'' / s' is large: it takes the scale S = 2^k s' in place of s', with |m''| <= 16 S, and (c' - 8) 2^-k, still exact.
// Weights are halves of 2^(t - m), the denominator is the sum of the unrounded p.  The reference m of a row is set 10 below
// its first maximum, and again below a later one when a sum of 8 weights passes 61440, or for exact values one 2^15.5 (no
// half overflows before), in whole powers of two: weights keep their 11 bits down to 2^-23 of that maximum and vanish at
// 2^-34.  (With the reference at the maximum a first token that takes almost all left the others 10 bits fewer.  A limit of
// 2^15 for the sum, which is passed more often, took 675 us where this takes 655, on 2 x 8192 tokens.)
// A value whose parameters are not finite must reach only the rows that see it, and not their log-sum-exp: its operand is a
// number, and a block that met one looks its keys' parameters through again at the end, for the rows that see them.
//
// Warps: one or two groups of four run the softmax, in matrix fragments: a thread has four rows and two of every eight
// keys (with a thread a row, as many broadcast loads of the keys' parameters as scores took 2000 of 4500 cycles a tile);
// four expand codes (global memory to registers a tile ahead, then to swizzled shared memory); one issues MMAs.  Two S
// buffers: with RT = 2 one a row tile; else the key tiles alternate, and with two groups each has an O of its own, joined
// at the end.
// A block's keys may be split over `splits` blocks, joined by kv4_chunk_join_kernel.
#pragma once
#include "kv4_rows.cuh"
#include "tmem.cuh"

namespace ifq {

struct KvChunkArgs {
  KvAttnArgs a;
  KvDiv by_gpp, by_group;
  int blocks, splits;        // blocks of rows of a (sequence, head) at most; blocks a block's keys are split over
  float* part;               // [seqs][heads][blocks][splits][rows][D]
  float2* part_ml;           // the same without D: reference and sum
};

constexpr int kChunkKeys = 128, kChunkPar = 4;   // keys a tile; tiles whose parameters are held
constexpr float kChunkAbove = 10.0f;             // a row's reference is this far below its maximum when it is set

template <int D, int RT>
struct KvChunkShape {
  static constexpr int NG = D == 256 ? 1 : 2;               // softmax groups
  static constexpr int NB = D == 256 ? 1 : 2;               // key and value buffers
  static constexpr int threads = 32 * (4 * NG + 5);
  static constexpr int q_bytes = RT * 128 * D * 2, kv_bytes = 128 * D * 2;
  static constexpr int par_bytes = kChunkPar * kChunkKeys * 20;
  static constexpr int bytes = 1024 + q_bytes + 2 * NB * kv_bytes + par_bytes + 512;
  static_assert(RT == 1 || NG == 2, "a group a row tile");
  static_assert(bytes <= 232448, "shared memory budget");
};

__device__ __forceinline__ void mma_f16_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile("{.reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;}" ::"r"(d),
               "l"(a), "l"(b), "r"(idesc), "r"(acc)
               : "memory");
}
// 16 / 32 registers of a lane to consecutive columns of its row.
__device__ __forceinline__ void tmem_st16(uint32_t t, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(t),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
      "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
// 32 lanes x 32 columns as matrix fragments: with q = t / 4, thread t has v[h][4 k + 2 e + i] = column 8 k + 2 (t % 4) + i
// of lane 16 h + q + 8 e.
__device__ __forceinline__ void tmem_ld_frag(uint32_t t, uint32_t (&v)[2][16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%32];\n\t"
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%33];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(v[0][0]), "=r"(v[0][1]), "=r"(v[0][2]), "=r"(v[0][3]), "=r"(v[0][4]), "=r"(v[0][5]), "=r"(v[0][6]),
        "=r"(v[0][7]), "=r"(v[0][8]), "=r"(v[0][9]), "=r"(v[0][10]), "=r"(v[0][11]), "=r"(v[0][12]), "=r"(v[0][13]),
        "=r"(v[0][14]), "=r"(v[0][15]), "=r"(v[1][0]), "=r"(v[1][1]), "=r"(v[1][2]), "=r"(v[1][3]), "=r"(v[1][4]),
        "=r"(v[1][5]), "=r"(v[1][6]), "=r"(v[1][7]), "=r"(v[1][8]), "=r"(v[1][9]), "=r"(v[1][10]), "=r"(v[1][11]),
        "=r"(v[1][12]), "=r"(v[1][13]), "=r"(v[1][14]), "=r"(v[1][15])
      : "r"(t), "r"(t + (16u << 16))
      : "memory");
}
__device__ __forceinline__ uint64_t pair2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2v(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// The key tiles that a block of rows reads: those with the first tokens (sinks), then those in reach.
struct KvTiles {
  int n, sg, skip;
};
__device__ __forceinline__ KvTiles kv_tiles(const KvAttnArgs& a, int len, int p_lo, int p_hi) {
  KvTiles t;
  const int all = p_hi < 0 ? 0 : p_hi / kChunkKeys + 1;
  const int lo = a.window > 0 && p_lo >= a.window ? (p_lo - a.window + 1) / kChunkKeys : 0;
  const int sinks = min(a.sinks, len);
  t.sg = min((sinks + kChunkKeys - 1) / kChunkKeys, lo);
  t.skip = lo - t.sg;
  t.n = max(0, all - t.skip);
  return t;
}

// Parameters of an exact value: its scale (0 counts as the smallest half: its codes are 0, and the value of code 8 makes up
// for it), the value of code 8, and the k that brings that within 16 2^k scales of 0 (by their exponents).
struct KvExact {
  float sc, eight;
  int k;
  __device__ __forceinline__ explicit KvExact(uint32_t par) {
    const float2 y = unpack16<false>(par);
    sc = fmaxf(y.x, 5.9604645e-8f);
    eight = y.y + 8.0f * sc;
    k = max(0, (int)(__float_as_uint(eight) >> 23 & 255u) - (int)(__float_as_uint(sc) >> 23) - 3);
  }
};

// Whether a value's parameters are numbers: neither an infinity nor a NaN in either half.
__device__ __forceinline__ bool kv_finite(uint32_t par) {
  return (par & 0x7c00u) != 0x7c00u && (par & 0x7c000000u) != 0x7c000000u;
}

// Keeps the use of loaded registers after this point: work on them that is moved up to the loads waits for them there
// (900 of 3200 cycles a tile).
template <int N>
__device__ __forceinline__ void hold(uint32_t (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+r"(v[i]));
}

template <int D, bool BF, int RT>
__global__ void __launch_bounds__(KvChunkShape<D, RT>::threads, 1) kv4_chunk_kernel(const __grid_constant__ KvChunkArgs A) {
  using C = KvChunkShape<D, RT>;
  constexpr bool EX = !BF;   // exact values
  constexpr int NG = C::NG, NB = C::NB, DB = kv4_block(D), NBLK = D / DB, WPB = DB / 32, GB = kv4_group_bytes(D);
  extern __shared__ uint8_t raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
  uint8_t *sQ = smem, *sK = sQ + C::q_bytes, *sV = sK + NB * C::kv_bytes;
  float4* sPar = (float4*)(sV + NB * C::kv_bytes);          // [kChunkPar][64 pairs of keys]: s, s, m, m of the keys
  float4* sVal = sPar + kChunkPar * (kChunkKeys / 2);       // of values in half: 1/S, 1/S, m''/S, m''/S
  float2* sLog = (float2*)(sVal + kChunkPar * (kChunkKeys / 2));   // and log2 S, twice
  const uint32_t bars = smem_u32(sPar) + C::par_bytes;
  auto kfull = [&](int b) { return bars + 8 * b; };          // expanded keys
  auto kempty = [&](int b) { return bars + 16 + 8 * b; };
  auto vfull = [&](int b) { return bars + 32 + 8 * b; };
  auto vempty = [&](int b) { return bars + 48 + 8 * b; };
  auto sfull = [&](int b) { return bars + 64 + 8 * b; };     // a finished S, its weights, a finished O
  auto pready = [&](int b) { return bars + 80 + 8 * b; };
  auto odone = [&](int r) { return bars + 96 + 8 * r; };
  auto pfull = [&](int b) { return bars + 112 + 8 * b; };    // parameters
  const uint32_t qready = bars + 112 + 8 * kChunkPar;
  auto olast = [&](int g) { return qready + 8 + 8 * g; };    // group g's last product
  uint32_t* tptr = (uint32_t*)((uint8_t*)sPar + C::par_bytes + 112 + 8 * kChunkPar + 24);
  uint32_t* sOdd = tptr + 1;   // some value's parameters are not finite
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    *sOdd = 0;
    for (int b = 0; b < 2; ++b) {
      mbar_init(kfull(b), 4);
      mbar_init(kempty(b), 1);
      mbar_init(vfull(b), 4);
      mbar_init(vempty(b), 1);
      mbar_init(sfull(b), 1);
      mbar_init(pready(b), 4);
      mbar_init(odone(b), 1);
      mbar_init(olast(b), 1);
    }
    for (int b = 0; b < kChunkPar; ++b) mbar_init(pfull(b), 4);
    mbar_init(qready, 4 * RT);
    fence_mbar_init();
  }
  if (warp == 4 * NG + 4) {
    tmem_alloc(smem_u32(tptr), 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tptr;
  grid_dep_wait();
  grid_dep_launch();

  const KvAttnArgs& a = A.a;
  const int s = blockIdx.z / A.splits, sp = blockIdx.z - s * A.splits, head = blockIdx.y;
  const KvSeq q = kv_seq(a, s);
  const int rows = q.ok ? q.n * a.group : 0, r0 = (A.blocks - 1 - (int)blockIdx.x) * 128 * RT;   // the longest first
  if (!q.ok && threadIdx.x == 0) set_status(IFQ_ERANGE);
  const bool work = r0 < rows;
  const int p_lo = q.len - q.n + (work ? (int)kv_div(r0, A.by_group) : 0);
  const int p_hi = q.len - q.n + (work ? (int)kv_div(min(rows, r0 + 128 * RT) - 1, A.by_group) : 0);
  const KvTiles tiles = kv_tiles(a, q.len, p_lo, p_hi);
  const int t0 = work ? (int)((long long)tiles.n * sp / A.splits) : 0, t1 = work ? (int)((long long)tiles.n * (sp + 1) / A.splits) : 0;
  const int nt = t1 - t0, steps = nt * RT;   // step x: tile x / RT, S buffer x % 2, softmax group x % NG
  const int gpp = A.by_gpp.d;   // groups a page
  const long long page_bytes = (long long)a.kv_heads * gpp * GB;
  const uint8_t* heads = a.cache + (long long)head * gpp * GB;
  const int32_t* table = a.table + (long long)s * a.max_pages;
  auto first_key = [&](int i) { return (t0 + i < tiles.sg ? t0 + i : t0 + i + tiles.skip) * kChunkKeys; };

  if (warp < 4 * NG) {
    // ------------------------------------------------------------ softmax
    const int grp = warp >> 2, row = threadIdx.x & 127, rt = RT == 2 ? grp : 0, r = r0 + rt * 128 + row;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, tO = tmem + lanes + 256 + grp * D;
    const bool have = work && r < rows;
    const int qi = have ? (int)kv_div(r, A.by_group) : 0, hq = head * a.group + (have ? r - qi * a.group : 0);
    const int p = q.len - q.n + qi, p_first = a.window > 0 ? p - a.window + 1 : 0;
    float fa = 1.0f, fb = 0.0f;
    if (work) {
      // the row of q as halves; with one row tile the second group only needs the factors
      const uint16_t* src = a.q + (long long)(q.first + qi) * a.q_stride + (long long)hq * D;
      float top = 0.0f, sum = 0.0f;
#pragma unroll 4
      for (int i = 0; i < D / 8; ++i) {
        uint32_t w[4] = {0, 0, 0, 0};
        if (have) load_words(w, src + 8 * i);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 f = unpack16<BF>(w[k]);
          top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y)));
          sum += f.x + f.y;
        }
      }
      const int e = max(0, min(117, (int)(__float_as_uint(top) >> 23) - 127 - 10));   // (largest below 2^15 once it is 16 q 2^-e)
      const float down = __uint_as_float((uint32_t)(131 - e) << 23), low = down * 0.0625f;
      fa = __uint_as_float((uint32_t)(127 + e) << 23);
      fb = a.scale * 1.44269504f * sum;
      if (RT == 2 || grp == 0) {
#pragma unroll 4
        for (int i = 0; i < D / 8; ++i) {
          uint32_t w[4] = {0, 0, 0, 0};
          if (have) load_words(w, src + 8 * i);
          const float2 f0 = unpack16<BF>(w[0]), f1 = unpack16<BF>(w[1]), f2 = unpack16<BF>(w[2]), f3 = unpack16<BF>(w[3]);
          const uint4 v = make_uint4(pack16<false>(f0.x * down, f2.x * down), pack16<false>(f0.y * low, f2.y * low),
                                     pack16<false>(f1.x * down, f3.x * down), pack16<false>(f1.y * low, f3.y * low));
          *(uint4*)(sQ + rt * 128 * D * 2 + (i >> 3) * 16384 + row * 128 + (((i & 7) ^ (row & 7)) << 4)) = v;
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(qready);
      }
    }
    // From here a thread has four rows, q + 8 y of its warp's 32 (q = lane / 4), and of every 8 keys two: a key's
    // parameters then serve four rows a load.
    const int quad = lane >> 2, pos = lane & 3;
    uint64_t fb2[4], l2[4], z2[4];
    float m[4], up[4];
    int py[4], pf[4];
    uint32_t fresh = 0;
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const float v = __shfl_sync(0xffffffffu, fb, quad + 8 * y);
      up[y] = __shfl_sync(0xffffffffu, fa, quad + 8 * y);
      fb2[y] = pair2(v, v);
      l2[y] = 0;
      z2[y] = 0;
      m[y] = 0.0f;
      py[y] = __shfl_sync(0xffffffffu, p, quad + 8 * y);
      pf[y] = __shfl_sync(0xffffffffu, p_first, quad + 8 * y);
      fresh |= (uint32_t)__shfl_sync(0xffffffffu, (int)have, quad + 8 * y) << y;
    }
    const bool large = __any_sync(0xffffffffu, fa != 1.0f);   // some row's q is out of the usual range
    // of a value per own row, the one of row `lane` of the warp
    auto by_lane = [&](const float (&x)[4]) {
      float r = 0.0f;
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const float t = __shfl_sync(0xffffffffu, x[y], 4 * (lane & 7));
        r = lane >> 3 == y ? t : r;
      }
      return r;
    };
    bool ok = true;
    int mine = 0;   // steps of this group so far
    for (int x = grp; x < steps && ok; x += NG, ++mine) {
      const int i = x / RT, b = x & 1, pb = i % kChunkPar, j0 = first_key(i);
      const uint32_t tS = tmem + lanes + b * 128;
      ok = __all_sync(0xffffffffu, mbar_wait(pfull(pb), (i / kChunkPar) & 1) && mbar_wait(sfull(b), (x >> 1) & 1));
      if (!ok) break;
      tc_fence_after();
      const float4 *par = sPar + pb * (kChunkKeys / 2) + pos, *val = sVal + pb * (kChunkKeys / 2) + pos;
      const float2* slog = sLog + pb * (kChunkKeys / 2) + pos;
      const bool full = j0 + kChunkKeys - 1 <= p_lo && (a.window == 0 || j0 > p_hi - a.window || j0 + kChunkKeys <= a.sinks);
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {
        uint32_t v[2][16];
        tmem_ld_frag(tS + 32 * c, v);
        float t[4][8];   // [row][2 k + i]: key 8 k + 2 pos + i of the 32
        if (large) {
#pragma unroll
          for (int k = 0; k < 16; ++k) {
#pragma unroll
            for (int h = 0; h < 2; ++h) v[h][k] = __float_as_uint(__uint_as_float(v[h][k]) * up[2 * h + (k >> 1 & 1)]);
          }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float4 kp = par[16 * c + 4 * k];
          const uint64_t s2 = pair2(kp.x, kp.y), n2 = pair2(kp.z, kp.w);
          const float2 lg = EX ? slog[16 * c + 4 * k] : make_float2(0.0f, 0.0f);
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const uint32_t* w = &v[y >> 1][4 * k + 2 * (y & 1)];
            const uint64_t ref = pair2(EX ? lg.x - m[y] : -m[y], EX ? lg.y - m[y] : -m[y]);
            const float2 z = halves2(fma2v(pair2(__uint_as_float(w[0]), __uint_as_float(w[1])), s2, fma2v(n2, fb2[y], ref)));
            t[y][2 * k] = z.x;
            t[y][2 * k + 1] = z.y;
          }
        }
        if (!full) {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const int j = j0 + 32 * c + 8 * (k >> 1) + 2 * pos + (k & 1);
#pragma unroll
            for (int y = 0; y < 4; ++y)
              if (j > py[y] || (j < pf[y] && j >= a.sinks)) t[y][k] = -INFINITY;
          }
        }
        uint32_t w[2][8];
        uint64_t part[4];
        float most = 0.0f;
        auto weights = [&]() {
          most = 0.0f;
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            part[y] = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float u0 = exp2_fast(t[y][2 * k]), u1 = exp2_fast(t[y][2 * k + 1]);
              part[y] = k ? add2(part[y], pair2(u0, u1)) : pair2(u0, u1);
              w[y >> 1][2 * k + (y & 1)] = pack16<false>(u0, u1);
            }
            const float2 u = halves2(part[y]);
            most = fmaxf(most, u.x + u.y);
          }
        };
        if constexpr (EX) {
#pragma unroll
          for (int y = 0; y < 4; ++y)
#pragma unroll
            for (int k = 0; k < 8; k += 2) most = fmaxf(most, fmaxf(t[y][k], t[y][k + 1]));
        } else {
          weights();
        }
        if (__any_sync(0xffffffffu, most > (EX ? 15.5f : 61440.0f) || fresh)) {
          float f[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            float top = t[y][0];
#pragma unroll
            for (int k = 1; k < 8; ++k) top = fmaxf(top, t[y][k]);
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const bool begin = (fresh >> y & 1u) && top > -INFINITY;
            const float rise = begin || top > kChunkAbove ? ceilf(top) - kChunkAbove : 0.0f;
            f[y] = begin ? 1.0f : exp2_fast(-rise);
            if (begin) fresh &= ~(1u << y);
            m[y] += rise;
            l2[y] = mul2(l2[y], pair2(f[y], f[y]));
            if constexpr (EX) z2[y] = mul2(z2[y], pair2(f[y], f[y]));
#pragma unroll
            for (int k = 0; k < 8; ++k) t[y][k] -= rise;
          }
          if constexpr (!EX) weights();
          const float fl = by_lane(f);
          if (__any_sync(0xffffffffu, fl != 1.0f)) {
            // what this tile's columns and the sum already hold (the factor may be below what a half can be)
            tmem_wait_st();
            for (int d = 0; d < c; ++d) {
              uint32_t x[16];
              tmem_ld<16>(tS + 16 * d, x);
#pragma unroll
              for (int k = 0; k < 16; ++k) {
                const float2 y = unpack16<false>(x[k]);
                x[k] = pack16<false>(y.x * fl, y.y * fl);
              }
              tmem_st16(tS + 16 * d, x);
            }
            if (mine > 0) {
              // (these scores were asked for after the product before the last, so the barrier is in the phase of the
              // last one or past it)
              ok = __all_sync(0xffffffffu, mbar_wait(odone(grp), (mine - 1) & 1));
              if (!ok) break;
              tc_fence_after();
#pragma unroll 1
              for (int d = 0; d < D; d += 16) {
                uint32_t x[16];
                tmem_ld<16>(tO + d, x);
#pragma unroll
                for (int k = 0; k < 16; ++k) x[k] = __float_as_uint(__uint_as_float(x[k]) * fl);
                tmem_st16(tO + d, x);
              }
            }
          }
        }
        if constexpr (EX) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float4 q4 = val[16 * c + 4 * k];
            const uint64_t i2 = pair2(q4.x, q4.y), v2 = pair2(q4.z, q4.w);
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const float u0 = exp2_fast(t[y][2 * k]), u1 = exp2_fast(t[y][2 * k + 1]);
              const uint32_t h2 = w[y >> 1][2 * k + (y & 1)] = pack16<false>(u0, u1);
              const float2 r = unpack16<false>(h2);   // as the product has them: what is lost goes with v, not with c' - 8
              l2[y] = fma2v(pair2(u0, u1), i2, l2[y]);
              z2[y] = fma2v(pair2(r.x, r.y), v2, z2[y]);
            }
          }
        } else {
#pragma unroll
          for (int y = 0; y < 4; ++y) l2[y] = add2(l2[y], part[y]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) tmem_st_frag(tS + ((uint32_t)(16 * h) << 16) + 16 * c, w[h]);
      }
      if (!ok) break;
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(pready(b));
    }
    if (mine > 0 && ok) ok = __all_sync(0xffffffffu, mbar_wait(olast(grp), 0));
    tc_fence_after();
    float sums[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const float2 u = halves2(l2[y]);
      sums[y] = u.x + u.y;
      sums[y] += __shfl_xor_sync(0xffffffffu, sums[y], 1);
      sums[y] += __shfl_xor_sync(0xffffffffu, sums[y], 2);
      if (fresh >> y & 1u) m[y] = kNoMax;
    }
    float sum = by_lane(sums), top = by_lane(m), zl = 0.0f;   // a thread a row again
    if constexpr (EX) {
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const float2 u = halves2(z2[y]);
        sums[y] = u.x + u.y;
        sums[y] += __shfl_xor_sync(0xffffffffu, sums[y], 1);
        sums[y] += __shfl_xor_sync(0xffffffffu, sums[y], 2);
      }
      zl = by_lane(sums);
    }
    if (!have) top = kNoMax;
    float other_top = kNoMax, other_f = 0.0f, my_f = 1.0f;
    float* xo = (float*)sK;   // [128][D + 4], and the second group's references and sums
    float2* xml = (float2*)(xo + 128 * (D + 4));
    if (NG == 2 && RT == 1 && work) {
      // the other half of the keys; all products are done once both groups have passed their waits
      named_bar(1, 256);
      if (grp == 1) {
        xml[row] = make_float2(top, sum);
#pragma unroll 1
        for (int d = 0; d < D; d += 16) {
          uint32_t w[16];
          if (mine > 0) tmem_ld<16>(tO + d, w);
#pragma unroll
          for (int k = 0; k < 16; k += 4)
            *(float4*)(xo + row * (D + 4) + d + k) =
                mine > 0 ? make_float4(__uint_as_float(w[k]) + zl, __uint_as_float(w[k + 1]) + zl, __uint_as_float(w[k + 2]) + zl, __uint_as_float(w[k + 3]) + zl)
                         : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
      }
      named_bar(1, 256);
      if (grp == 0) {
        const float2 o = xml[row];
        other_top = o.x;
        const float all = fmaxf(top, other_top);
        my_f = exp2_fast(top - all);
        other_f = exp2_fast(other_top - all);
        sum = sum * my_f + o.y * other_f;
        top = all;
      }
    }
    if (work && (RT == 2 || grp == 0) && *sOdd && have && nt > 0) {
      const int last_seen = min(p, q.len - 1);
      for (int i = 0; i < nt; ++i)
        for (int j = first_key(i), end = min(j + kChunkKeys, last_seen + 1); j < end; j += kKvGroup) {
          const int group = j / kKvGroup, in_table = kv_div(group, A.by_gpp), page = table[in_table];
          if (page < 0 || page >= a.pages) continue;
          const uint32_t* par = (const uint32_t*)(heads + page * page_bytes + (group - in_table * gpp) * GB + 16 * D + 64);
          for (int k = 0; k < kKvGroup; ++k)
            if (j + k < end && (j + k >= p_first || j + k < a.sinks) && !kv_finite(par[k])) zl = __uint_as_float(0x7fc00000u);
        }
    }
    __syncwarp();
    if (work && (RT == 2 || grp == 0)) {
      const bool parts = A.splits > 1;
      const long long at = ((((long long)s * a.kv_heads + head) * A.blocks + r0 / (128 * RT)) * A.splits + sp) * (128 * RT) + rt * 128 + row;
      constexpr float kUnit = EX ? 1.0f : 2.0f;
      const float inv = parts ? kUnit : sum == 0.0f ? 0.0f : kUnit / sum;
#pragma unroll 1
      for (int d = 0; d < D; d += 16) {
        uint32_t w[16];
        if (mine > 0) tmem_ld<16>(tO + d, w);
        float o[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) o[k] = mine > 0 ? __uint_as_float(w[k]) + zl : 0.0f;
        if (NG == 2 && RT == 1) {
#pragma unroll
          for (int k = 0; k < 16; k += 4) {
            const float4 y = *(const float4*)(xo + row * (D + 4) + d + k);
            o[k] = o[k] * my_f + y.x * other_f, o[k + 1] = o[k + 1] * my_f + y.y * other_f;
            o[k + 2] = o[k + 2] * my_f + y.z * other_f, o[k + 3] = o[k + 3] * my_f + y.w * other_f;
          }
        }
        if (have && parts) {
#pragma unroll
          for (int k = 0; k < 16; k += 4)
            *(float4*)(A.part + at * D + d + k) = make_float4(o[k] * inv, o[k + 1] * inv, o[k + 2] * inv, o[k + 3] * inv);
        } else if (have) {
          uint16_t* dst = a.out + (long long)(q.first + qi) * a.out_stride + (long long)hq * D + d;
#pragma unroll
          for (int k = 0; k < 16; k += 8) {
            const uint32_t y[4] = {pack16<BF>(o[k] * inv, o[k + 1] * inv), pack16<BF>(o[k + 2] * inv, o[k + 3] * inv),
                                   pack16<BF>(o[k + 4] * inv, o[k + 5] * inv), pack16<BF>(o[k + 6] * inv, o[k + 7] * inv)};
            store_words(dst + k, y);
          }
        }
        __syncwarp();
      }
      if (have) {
        if (parts) A.part_ml[at] = make_float2(top, sum);
        else if (a.lse)
          a.lse[(long long)(q.first + qi) * a.q_heads + hq] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * 0.69314718f;
      }
    }
  } else if (warp < 4 * NG + 4) {
    // ------------------------------------------------------------ expansion: a thread a key, and 8 keys x D/8 values
    const int tid = threadIdx.x - 128 * NG, w = warp - 4 * NG;
    const int kg = tid >> 4, krow = tid & 15;                                  // the key's group of the tile, row of it
    const int c8 = lane & 7, vg = (w >> 1) * 4 + (c8 >> 1), vh = c8 & 1, slice = (lane >> 3) | (w & 1) << 2;
    uint32_t kw[NBLK * WPB * 4], vw[NBLK * WPB * 4], kpar = 0, vpar = 0, vp[EX ? 2 : 8];
    // The thread's two groups of each tile, a cursor each: place in the page table, group of the page.  A page's number
    // is read two tiles ahead, so that nothing waits for it; nor is any load made on a condition, which would be waited
    // for at once: a group past the tokens is looked up in the last page's place, and where there is no page any
    // group's bytes will do (codes are numbers, and the parameters are then left out).
    const int last_group = (q.len - 1) / kKvGroup, last_page = (int)kv_div(max(last_group, 0), A.by_gpp);
    const int step_pages = 8 / gpp, step_groups = 8 - step_pages * gpp;   // (8 groups a tile)
    struct Cursor {
      int group, page, in;   // group of the sequence; its place in the table and in its page
    };
    auto at_tile = [&](int i, int g) {
      Cursor c;
      c.group = first_key(i) / kKvGroup + g;
      c.page = kv_div(c.group, A.by_gpp);
      c.in = c.group - c.page * gpp;
      return c;
    };
    auto forward = [&](Cursor& c, int i, int g) {   // from tile i - 1 to i
      if (t0 + i == tiles.sg && tiles.skip) {
        c = at_tile(i, g);
        return;
      }
      c.group += 8;
      c.page += step_pages;
      c.in += step_groups;
      if (c.in >= gpp) c.in -= gpp, ++c.page;
    };
    auto look = [&](const Cursor& c) { return table[min(c.page, last_page)]; };
    auto place = [&](const Cursor& c, int page, bool& there) -> const uint8_t* {
      const bool tokens = c.group <= last_group, known = page >= 0 && page < a.pages;
      if (tokens && !known) set_status(IFQ_ERANGE);
      there = tokens && known;
      return heads + (known ? page : 0) * page_bytes + c.in * GB;
    };
    auto load_k = [&](const uint8_t* g) {
#pragma unroll
      for (int b = 0; b < NBLK; ++b)
#pragma unroll
        for (int k = 0; k < WPB; ++k) {
          const uint4 y = *(const uint4*)(g + b * 8 * DB + krow * (DB / 2) + 16 * k);
          const int o = (b * WPB + k) * 4;
          kw[o] = y.x, kw[o + 1] = y.y, kw[o + 2] = y.z, kw[o + 3] = y.w;
        }
      kpar = *(const uint32_t*)(g + 16 * D + 4 * krow);
      vpar = *(const uint32_t*)(g + 16 * D + 64 + 4 * krow);
    };
    auto load_v = [&](const uint8_t* g) {
#pragma unroll
      for (int b = 0; b < NBLK; ++b)
#pragma unroll
        for (int k = 0; k < WPB; ++k) {
          const uint4 y = *(const uint4*)(g + 8 * D + b * 8 * DB + vh * 4 * DB + slice * 4 * (DB / 8) + 16 * k);
          const int o = (b * WPB + k) * 4;
          vw[o] = y.x, vw[o + 1] = y.y, vw[o + 2] = y.z, vw[o + 3] = y.w;
        }
      if constexpr (EX) {   // two of the eight tokens, the others' from the three lanes that share them
        load_words(vp, g + 16 * D + 64 + 32 * vh + 8 * (lane >> 3));
      } else {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint4 y = *(const uint4*)(g + 16 * D + 64 + 32 * vh + 16 * k);
          vp[4 * k] = y.x, vp[4 * k + 1] = y.y, vp[4 * k + 2] = y.z, vp[4 * k + 3] = y.w;
        }
      }
    };
    bool ok = true;
    int page_k = 0, page_v = 0;             // of the tile after the one at hand
    bool have_k = false, have_v = false;    // whether the tile at hand has the thread's groups
    Cursor ck = {}, cv = {}, nk = {}, nv = {};   // of the tile after the one at hand, and of the one after that
    if (nt > 0) {
      ck = at_tile(0, kg);
      cv = at_tile(0, vg);
      load_k(place(ck, look(ck), have_k));
      load_v(place(cv, look(cv), have_v));
      forward(ck, 1, kg);
      forward(cv, 1, vg);
      page_k = look(ck);
      page_v = look(cv);
      nk = ck;
      nv = cv;
    }
    for (int i = 0; i < nt && ok; ++i) {
      const int b = i % NB, pb = i % kChunkPar, j0 = first_key(i);
      forward(nk, i + 2, kg);
      forward(nv, i + 2, vg);
      const int next_k = look(nk), next_v = look(nv);
      // (The buffer's last S is done.  It was asked for after the weights of the tile two before it, so the parameters
      // of tile i - 4 have been used too.)
      ok = __all_sync(0xffffffffu, i < NB || mbar_wait(kempty(b), (i / NB - 1) & 1));
      if (!ok) break;
      hold(kw);
      asm volatile("" : "+r"(kpar), "+r"(vpar));
      {
        const bool there = have_k && j0 + tid < q.len;
        const float2 f = unpack16<false>(there ? kpar : 0u);
        if (there && !kv_finite(vpar)) *sOdd = 1;
        float* dst = (float*)(sPar + pb * (kChunkKeys / 2) + tid / 2) + (tid & 1);
        dst[0] = f.x * (a.scale * 1.44269504f * 1048576.0f);   // codes are in units of 2^-24, q of 2^-4
        dst[2] = f.y;
        if constexpr (EX) {
          const KvExact y(there && kv_finite(vpar) ? vpar : 0x3c00u);   // (scale 1, minimum 0)
          const float r = __uint_as_float((uint32_t)(127 - y.k) << 23) / y.sc;
          float* dv4 = (float*)(sVal + pb * (kChunkKeys / 2) + tid / 2) + (tid & 1);
          dv4[0] = there ? r : 0.0f;
          dv4[2] = there ? y.eight * r : 0.0f;
          ((float*)(sLog + pb * (kChunkKeys / 2)))[tid] = there ? log2f(y.sc) + (float)y.k : 0.0f;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(pfull(pb));
      }
      uint8_t* dk = sK + b * C::kv_bytes + tid * 128;
#pragma unroll
      for (int k = 0; k < NBLK * WPB * 4; ++k) {
        const uint32_t u = kw[k], h = u >> 8;
        *(uint4*)(dk + (k >> 3) * 16384 + (((k & 7) ^ (tid & 7)) << 4)) =
            make_uint4(u & 0x000f000fu, u & 0x00f000f0u, h & 0x000f000fu, h & 0x00f000f0u);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(kfull(b));
      if (i + 1 < nt) load_k(place(ck, page_k, have_k));
      hold(vp);
      __half2 vs[4], vm[4];   // pairs of tokens: scales, and minima halved; of exact values 2^-k
      auto param = [&](int i, int j) { return have_v && j0 + vg * kKvGroup + 8 * vh + j < q.len && kv_finite(vp[i]) ? vp[i] : 0u; };
      bool down = false;      // some k is not 0
      if constexpr (EX) {
        const int k0 = KvExact(param(0, 2 * (lane >> 3))).k, k1 = KvExact(param(1, 2 * (lane >> 3) + 1)).k;
        down = __any_sync(0xffffffffu, k0 | k1);
        if (down) {   // (past 2^20 a step is nothing beside the value)
          const uint32_t f = pack16<false>(__uint_as_float(k0 > 20 ? 0u : (uint32_t)(127 - k0) << 23),
                                           __uint_as_float(k1 > 20 ? 0u : (uint32_t)(127 - k1) << 23));
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const uint32_t y = __shfl_sync(0xffffffffu, f, t << 3 | c8);
            vs[t] = *(const __half2*)&y;
          }
        }
      } else {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const uint32_t y0 = param(2 * t, 2 * t), y1 = param(2 * t + 1, 2 * t + 1);
          const uint32_t sc = __byte_perm(y0, y1, 0x5410), mn = __byte_perm(y0, y1, 0x7632);
          vs[t] = *(const __half2*)&sc;   // (the codes are halved: a scale may be one of the smallest halves)
          vm[t] = __hmul2(*(const __half2*)&mn, __float2half2_rn(0.5f));
        }
      }
      ok = __all_sync(0xffffffffu, i < NB || mbar_wait(vempty(b), (i / NB - 1) & 1));
      if (!ok) break;
      hold(vw);
      uint8_t* dv = sV + b * C::kv_bytes + (w >> 1) * (D * 128);
#pragma unroll
      for (int blk = 0; blk < NBLK; ++blk)
#pragma unroll
        for (int k = 0; k < WPB; ++k) {      // word k of each pair of tokens: four dimensions
          const int d0 = blk * DB + slice * (DB / 8) + 4 * k;
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            uint32_t y[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              const uint32_t u = vw[blk * WPB * 4 + t * WPB + k] >> (n & 2 ? 8 : 0);
              const uint32_t g = (u & (n & 1 ? 0x00f000f0u : 0x000f000fu)) | 0x64006400u;   // 1024 + c, 1024 + 16 c
              // c' - 8, or c' / 2
              const __half2 code = n & 1 ? __hfma2(*(const __half2*)&g, __float2half2_rn(EX ? 0.0625f : 0.03125f), __float2half2_rn(EX ? -72.0f : -32.0f))
                                   : EX  ? __hadd2(*(const __half2*)&g, __float2half2_rn(-1032.0f))
                                         : __hfma2(*(const __half2*)&g, __float2half2_rn(0.5f), __float2half2_rn(-512.0f));
              const __half2 v = EX ? code : __hfma2(code, vs[t], vm[t]);
              y[t] = *(const uint32_t*)&v;
            }
            if (EX && down) {
#pragma unroll
              for (int t = 0; t < 4; ++t) {
                const __half2 v = __hmul2(*(const __half2*)&y[t], vs[t]);
                y[t] = *(const uint32_t*)&v;
              }
            }
            const int d = d0 + n;
            *(uint4*)(dv + d * 128 + ((c8 ^ (d & 7)) << 4)) = make_uint4(y[0], y[1], y[2], y[3]);
          }
        }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(vfull(b));
      if (i + 1 < nt) load_v(place(cv, page_v, have_v));
      page_k = next_k;
      page_v = next_v;
      ck = nk;
      cv = nv;
    }
  } else {
    // ------------------------------------------------------------ MMA
    constexpr uint32_t is = idesc_f16_f32(128, kChunkKeys), io = idesc_f16_f32(128, D);
    bool ok = steps > 0 && __all_sync(0xffffffffu, mbar_wait(qready, 0));
    auto scores = [&](int x) {   // S of step x
      const int i = x / RT, b = i % NB;
      if (x % RT == 0 && !__all_sync(0xffffffffu, mbar_wait(kfull(b), (i / NB) & 1))) return false;
      tc_fence_after();
      if (elect_one()) {
        const uint32_t q0 = smem_u32(sQ) + (RT == 2 ? (x & 1) * 128 * D * 2 : 0), k0 = smem_u32(sK) + b * C::kv_bytes;
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
          mma_f16_ss(tmem + (x & 1) * 128, sdesc_sw128(q0 + (k >> 2) * 16384 + (k & 3) * 32),
                     sdesc_sw128(k0 + (k >> 2) * 16384 + (k & 3) * 32), is, k > 0);
        mma_commit(sfull(x & 1));
        if (x % RT == RT - 1) mma_commit(kempty(b));
      }
      __syncwarp();
      return true;
    };
    for (int x = 0; x < 2 && x < steps && ok; ++x) ok = scores(x);
    for (int x = 0; x < steps && ok; ++x) {
      const int i = x / RT, b = i % NB;
      ok = __all_sync(0xffffffffu, mbar_wait(pready(x & 1), (x >> 1) & 1)) &&
           (x % RT != 0 || __all_sync(0xffffffffu, mbar_wait(vfull(b), (i / NB) & 1)));
      if (!ok) break;
      tc_fence_after();
      if (elect_one()) {
        const uint32_t v0 = smem_u32(sV) + b * C::kv_bytes;
#pragma unroll
        for (int k = 0; k < kChunkKeys / 16; ++k)
          mma_f16_ts(tmem + 256 + (x % NG) * D, tmem + (x & 1) * 128 + 8 * k, sdesc_sw128(v0 + (k >> 2) * (D * 128) + (k & 3) * 32),
                     io, x >= NG || k > 0);
        mma_commit(odone(x % NG));
        if (x + NG >= steps) mma_commit(olast(x % NG));
        if (x % RT == RT - 1) mma_commit(vempty(b));
      }
      __syncwarp();
      if (x + 2 < steps) {
        // The next S overwrites the weights that this product reads, and MMAs of different shapes need not run in the
        // order they were issued in.
        ok = __all_sync(0xffffffffu, mbar_wait(odone(x % NG), x / NG & 1)) && scores(x + 2);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 4 * NG + 4) tmem_dealloc(tmem, 512);
}

// The parts of a block's split keys: a warp a row.
template <int D, bool BF>
__global__ void __launch_bounds__(256) kv4_chunk_join_kernel(const __grid_constant__ KvChunkArgs A, int block_rows) {
  grid_dep_wait();
  grid_dep_launch();
  const KvAttnArgs& a = A.a;
  const int lane = threadIdx.x & 31, s = blockIdx.z, head = blockIdx.y, r = blockIdx.x * 8 + (threadIdx.x >> 5);
  const KvSeq q = kv_seq(a, s);
  if (!q.ok || r >= q.n * a.group) return;
  const int blk = r / block_rows, in = r - blk * block_rows;
  const long long at = (((long long)s * a.kv_heads + head) * A.blocks + blk) * A.splits * block_rows + in;
  float top = kNoMax, sum = 0.0f;
  for (int i = 0; i < A.splits; ++i) top = fmaxf(top, A.part_ml[at + (long long)i * block_rows].x);
  constexpr int N = D > 128 ? 2 : 1;
  float4 v[N];
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int i = 0; i < A.splits; ++i) {
    const float2 ml = A.part_ml[at + (long long)i * block_rows];
    const float f = exp2_fast(ml.x - top);
    sum += ml.y * f;
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (lane * 4 + 128 * k < D) {
        const float4 x = *(const float4*)(A.part + (at + (long long)i * block_rows) * D + lane * 4 + 128 * k);
        v[k].x += x.x * f, v[k].y += x.y * f, v[k].z += x.z * f, v[k].w += x.w * f;
      }
  }
  const int qi = kv_div(r, A.by_group), hq = head * a.group + r - qi * a.group;
  const long long t = q.first + qi;
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (lane * 4 + 128 * k < D) {
      const uint32_t w[2] = {pack16<BF>(v[k].x * inv, v[k].y * inv), pack16<BF>(v[k].z * inv, v[k].w * inv)};
      store_words(a.out + t * a.out_stride + (long long)hq * D + lane * 4 + 128 * k, w);
    }
  if (a.lse && lane == 0) a.lse[t * a.q_heads + hq] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * 0.69314718f;
}

}  // namespace ifq
