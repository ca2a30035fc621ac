// Attention of few query rows per sequence over the paged 4-bit cache: single tokens, drafted tokens.
//
// Bound by reading the cache: (D + 8) bytes a token and head, used once for all the rows that share the head.  The
// rows of an item (a sequence, a key head, a block of R = 8 NT rows: query tokens x the heads that share the key head)
// stand on the N side of mma.sync.m16n8k16, the 16 tokens of a cache group on its M side, so eight rows fill a tile:
//   S^T[token][row] = sum_d c[token][d] q[row][d],    O^T[d][row] = sum_token c'[token][d] w[token][row].
// Codes become operands by masks alone: four bits c at the bottom of a half are the subnormal c 2^-24, one place
// higher 16 c 2^-24, which the tensor cores multiply exactly; the factors 16 go to q (halved in exponent, exact) and
// to the rows of O, 2^24 to the scales.  q is brought to half by a power of two per row (exact for both types, but for
// elements 2^-34 below the row's largest).  Sums are fp32.
//
// The weights w = p s' are halves.  p = 2^(t - m) with m a maximum that is only raised when a score passes it by 8
// (p <= 2^8; the quotient does not depend on m), and s' is scaled by a power of two that follows the largest scale
// seen, so that w < 2^15 and weights keep their 11 bits down to 2^-20 of the largest.  p in the denominator and in
// the sum with the minima stays fp32.
//
// Work: an item's groups are taken in units of U; the units of all items in a row are cut into as many equal ranges as
// there are blocks, whatever the lengths; or, where no sequence is long, a block takes an item.  In a block whose range
// lies within one item the warps take the units in turn and their sums are joined in shared memory; else the range is
// cut again, a contiguous part a warp, so that no warp waits for another at an item's end (joining at each of them took
// 8000 cycles beside 2700 a unit).  An item that several parts share leaves sums in the workspace, which
// kv4_join_kernel adds (the block itself, where its warps have all of it).  One more warp fetches for all, a lane a group
// (page lookup and one bulk copy of the group's contiguous bytes), three units ahead and across the ends of items.
//
// Measured, the join with it: one sequence of 131072 tokens, 8 key heads of 128 and 4 rows each, 36.7 us (3.9 TB/s); 48
// sequences of up to 8192, 195780 tokens in all, 54 us (4.0 TB/s); 64 windows of 1028 tokens 7.9 us from L2, 15 from
// memory; 40 rows on 16 sequences of 4096, three passes, 61 us.  Issue slots are 50 % busy, with 268 instructions a group:
// bound by the latency of 3.5 computing warps a scheduler.
#pragma once
#include "kv4_attention.cuh"

namespace ifq {

constexpr float kNoMax = -3.0e38f;   // stands for the maximum of nothing

struct KvRowsArgs {
  KvAttnArgs a;
  KvDiv by_gpp, by_group;   // groups a page, query heads a key head
  int direct;               // one block an item: blockIdx = (key head, block of rows, sequence)
  // workspace of the ranges, a part a block and warp: sums [parts][2][R][D], their (max, sum) [parts][2][R], of an item
  // begun before the part (0) and of one it leaves open (1), and which item that is [parts]
  float* part;
  float2* part_ml;
  int4* cut;                // (sequence, block of rows * key heads + head, blocks it reaches into (0: none), last warp)
};

constexpr int kKvRowsWarps = 7;   // computing warps of a block; with the fetching one, two a scheduler

template <int D>
struct KvRowsShape {
  static constexpr int W = kKvRowsWarps;
  static constexpr int U = D == 64 ? 4 : 2;         // groups a unit
  static constexpr int stages = 3;                  // units in flight a warp
  static constexpr int threads = 32 * (W + 1);
  static_assert(W * U <= 32, "a fetching lane a group");
};
// Blocks an SM: two of 128 registers a thread where those do, else one.
__host__ __device__ constexpr int kv_rows_per_sm(int D, int NT) { return D < 256 && NT == 1 ? 2 : 1; }
template <int D>
__host__ __device__ constexpr int kv_rows_smem(int R) {
  using C = KvRowsShape<D>;
  return C::W * C::stages * (C::U * kv4_group_bytes(D) + 16) + C::W * 4 * (D + 4) * 4 + 3 * C::W * R * 4 + 16 * 8;
}

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// A sequence's groups, in the order they are read: those with its first tokens (sinks), then those in reach of a
// window.
struct KvCursor {
  int s;           // sequence
  KvSeq q;
  int it, nit;     // item of the sequence (block of rows * key heads + key head), items
  int ng, sg, skip, nu;   // groups, of those at its start, groups left out after them, units
  int base;        // the unit at which the item starts, relative to the block's range
};

template <int R, int U>
__device__ __forceinline__ void kv_shape(const KvRowsArgs& A, KvCursor& c) {
  const KvAttnArgs& a = A.a;
  c.q = kv_seq(a, c.s);
  c.nit = c.q.ok ? (c.q.n * a.group + R - 1) / R * a.kv_heads : 0;
  const int all = c.q.len > 0 ? (c.q.len - 1) / kKvGroup + 1 : 1;
  int lo = c.q.len - c.q.n;   // the first query's position
  lo = a.window > 0 && lo >= a.window ? (lo - a.window + 1) / kKvGroup : 0;
  const int sinks = a.sinks < c.q.len ? a.sinks : c.q.len;
  c.sg = (sinks + kKvGroup - 1) / kKvGroup;
  c.sg = c.sg < lo ? c.sg : lo;
  c.skip = lo - c.sg;
  c.ng = all - c.skip;
  c.nu = (c.ng + U - 1) / U;
}
// Move on to the item that holds unit o of the range.
template <int R, int U>
__device__ __forceinline__ void kv_advance(const KvRowsArgs& A, KvCursor& c, int o) {
  while (o >= c.base + c.nu) {
    c.base += c.nu;
    if (++c.it >= c.nit) {
      c.it = 0;
      do {
        ++c.s;
        kv_shape<R, U>(A, c);
      } while (c.nit == 0);
    }
  }
}

// A warp's sum of parts of a row: reference, sum of the weights, and values (four dimensions a lane).
template <int D>
struct KvSum {
  static constexpr int N = D > 128 ? 2 : 1;
  float top = kNoMax, sum = 0.0f;
  float4 v[N] = {};

  __device__ __forceinline__ void raise(float now) {
    const float old = exp2_fast(top - now);
    top = now;
    sum *= old;
#pragma unroll
    for (int n = 0; n < N; ++n) v[n].x *= old, v[n].y *= old, v[n].z *= old, v[n].w *= old;
  }
  // Parts i0, i0 + step, .. (a lane each, below `parts`); at(i): where part i stands.
  template <typename F>
  __device__ __forceinline__ void add(const KvRowsArgs& A, int lane, int i0, int step, int parts, F&& at) {
    const int mine = i0 + step * lane;
    const float2 ml = mine < parts ? A.part_ml[at(mine)] : make_float2(kNoMax, 0.0f);
    float now = fmaxf(top, ml.x);
#pragma unroll
    for (int k = 16; k; k >>= 1) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, k));
    raise(now);
    // (nothing seen: no sums were written; a sum that is not a number is taken along)
    uint32_t some = __ballot_sync(0xffffffffu, !(ml.x == kNoMax && ml.y == 0.0f));
    while (some) {   // eight at a time, so that their loads are under way together
      float4 x[8][N];
      float f[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int j = some ? __ffs(some) - 1 : 0;
        const float jm = __shfl_sync(0xffffffffu, ml.x, j), jl = __shfl_sync(0xffffffffu, ml.y, j);
        f[k] = some ? exp2_fast(jm - top) : 0.0f;
        if (some) sum += jl * f[k];
#pragma unroll
        for (int n = 0; n < N; ++n) {
          x[k][n] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          if (some && lane * 4 + 128 * n < D) x[k][n] = *(const float4*)(A.part + at(i0 + step * j) * D + lane * 4 + 128 * n);
        }
        some &= some - 1;
      }
#pragma unroll
      for (int k = 0; k < 8; ++k)
#pragma unroll
        for (int n = 0; n < N; ++n) {
          v[n].x += x[k][n].x * f[k], v[n].y += x[k][n].y * f[k];
          v[n].z += x[k][n].z * f[k], v[n].w += x[k][n].w * f[k];
        }
    }
  }
  // Another warp's.
  __device__ __forceinline__ void add(float2 ml, const float* x, int lane) {
    raise(fmaxf(top, ml.x));
    const float f = exp2_fast(ml.x - top);
    sum += ml.y * f;
#pragma unroll
    for (int n = 0; n < N; ++n)
      if (lane * 4 + 128 * n < D) {
        const float4 y = *(const float4*)(x + lane * 4 + 128 * n);
        v[n].x += y.x * f, v[n].y += y.y * f, v[n].z += y.z * f, v[n].w += y.w * f;
      }
  }
  template <bool BF>
  __device__ __forceinline__ void write(const KvRowsArgs& A, const KvSeq& q, int head, int r, int lane) const {
    const KvAttnArgs& a = A.a;
    const int qi = kv_div(r, A.by_group), hq = head * a.group + r - qi * a.group;
    const long long t = q.first + qi;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int n = 0; n < N; ++n)
      if (lane * 4 + 128 * n < D) {
        const uint32_t w[2] = {pack16<BF>(v[n].x * inv, v[n].y * inv), pack16<BF>(v[n].z * inv, v[n].w * inv)};
        store_words(a.out + t * a.out_stride + (long long)hq * D + lane * 4 + 128 * n, w);
      }
    if (a.lse && lane == 0) a.lse[t * a.q_heads + hq] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * 0.69314718f;
  }
};

template <int D, bool BF, int NT>
__global__ void __launch_bounds__(KvRowsShape<D>::threads, kv_rows_per_sm(D, NT)) kv4_rows_kernel(const __grid_constant__ KvRowsArgs A) {
  using C = KvRowsShape<D>;
  constexpr int W = C::W, U = C::U, ST = C::stages, R = 8 * NT, GB = kv4_group_bytes(D);
  constexpr int DB = kv4_block(D), NB = D / DB, WPL = DB / 32;   // blocks of dimensions, words a lane and row
  constexpr int KS = D / 16, MT = D / 16;                        // steps along d of S, tiles along d of O
  static_assert(4 * U * NT <= 32, "a bit a score");
  extern __shared__ __align__(128) uint8_t smem[];
  const KvAttnArgs& a = A.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
  float* jO = (float*)(smem + W * ST * U * GB);             // [W][4][D + 4]
  float* jm = jO + W * 4 * (D + 4);                         // [W][R] each
  float *jl = jm + W * R, *jz = jl + W * R;
  uint64_t* bars = (uint64_t*)(jz + W * R);                 // full [W][ST], empty [W][ST]
  long long* scan = (long long*)(bars + 2 * W * ST);        // [W + 1]
  __shared__ KvCursor first;
  __shared__ int4 cuts[W];
  const uint32_t bar_full = smem_u32(bars), bar_empty = smem_u32(bars + W * ST);
  if (threadIdx.x == 0) {
    for (int i = 0; i < W * ST; ++i) {
      mbar_init(bar_full + 8 * i, U);
      mbar_init(bar_empty + 8 * i, 1);
    }
    fence_mbar_init();
  }
  __syncthreads();
  grid_dep_wait();
  grid_dep_launch();

  KvCursor cur;
  int n;        // units of this block
  int full_share = 0;     // of a block whose range is not the last
  long long ends = 0;     // units from this block's start to the end of all
  if (A.direct) {
    cur.s = blockIdx.z;
    kv_shape<R, U>(A, cur);
    if (!cur.q.ok && threadIdx.x == 0) set_status(IFQ_ERANGE);
    cur.it = blockIdx.y * a.kv_heads + blockIdx.x;
    cur.base = 0;
    if (cur.it >= cur.nit) return;
    n = cur.nu;
  } else {
    // the units of every sequence, summed over the block's threads' shares of the sequences
    const int per = (a.seqs + C::threads - 1) / C::threads, s0 = threadIdx.x * per, s1 = min(a.seqs, s0 + per);
    long long mine = 0;
    for (int s = s0; s < s1; ++s) {
      KvCursor t;
      t.s = s;
      kv_shape<R, U>(A, t);
      if (!t.q.ok && blockIdx.x == 0) set_status(IFQ_ERANGE);
      mine += (long long)t.nit * t.nu;
    }
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long up = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += up;
    }
    if (lane == 31) scan[warp] = incl;
    __syncthreads();
    long long before = incl - mine, total = 0;
#pragma unroll
    for (int w = 0; w <= W; ++w) {
      if (w < warp) before += scan[w];
      total += scan[w];
    }
    // (64-bit divisions only where they are needed: they take as long as the loads above)
    const bool small = total < 0x7fff0000ll;
    long long share = small ? ((uint32_t)total + gridDim.x - 1) / gridDim.x : (total + gridDim.x - 1) / gridDim.x;
    if (share < 2 * W) share = 2 * W;
    const long long start = share * blockIdx.x;
    if (start >= total) {
      if (threadIdx.x < W) A.cut[blockIdx.x * W + threadIdx.x] = make_int4(0, 0, 0, 0);
      return;
    }
    full_share = (int)min(share, (long long)0x7fffffff);
    ends = total - start;
    n = (int)min(share, total - start);
    if (start >= before && start < before + mine) {   // one thread: its sequences hold the start
      long long at = before;
      KvCursor t;
      t.s = s0;
      for (;; ++t.s) {
        kv_shape<R, U>(A, t);
        const long long c = (long long)t.nit * t.nu;
        if (start < at + c) break;
        at += c;
      }
      const long long in = start - at;
      t.it = small ? (int)((uint32_t)in / (uint32_t)t.nu) : (int)(in / t.nu);
      t.base = -(int)(in - (long long)t.it * t.nu);
      first = t;
    }
    __syncthreads();
    cur = first;
  }

  const bool one = cur.base + cur.nu >= n;   // the range lies within one item
  auto part_begin = [&](int w) { return one ? w : (int)((long long)n * w / W); };
  auto part_end = [&](int w) { return one ? n : (int)((long long)n * (w + 1) / W); };
  const int step = one ? W : 1;
  if (warp == W) {
    // fetch: lane (w, u) the u-th group of warp w's units.  No lane waits for another warp's buffers.
    const int w = lane / U, u = lane % U, last = part_end(w);
    if (w < W) {
      const uint32_t ring = smem_u32(smem + w * ST * U * GB + u * GB);
      int o = part_begin(w), k = 0, st = 0, page = 0, gi = 0;
      bool there = false;
      auto look_up = [&]() {   // the next unit's page
        if (o >= last) return;
        kv_advance<R, U>(A, cur, o);
        const int g = (o - cur.base) * U + u;
        gi = g < cur.sg ? g : g + cur.skip;
        there = g < cur.ng && gi * kKvGroup < cur.q.len;
        if (there) page = a.table[(long long)cur.s * a.max_pages + kv_div(gi, A.by_gpp)];
      };
      look_up();
      unsigned long long t0 = 0;
      uint32_t idle = 0;
      while (o < last) {
        if (k < ST || mbar_test(bar_empty + 8 * (w * ST + st), (k / ST - 1) & 1)) {
          const uint32_t bar = bar_full + 8 * (w * ST + st);
          if (there && page >= 0 && page < a.pages) {
            const int head = cur.it % a.kv_heads, in = gi - (int)kv_div(gi, A.by_gpp) * (int)A.by_gpp.d;
            const uint8_t* src = a.cache + (((long long)page * a.kv_heads + head) * A.by_gpp.d + in) * GB;
            mbar_arrive_expect_tx(bar, GB);
            bulk_copy_g2s(ring + st * U * GB, src, GB, bar);
          } else {
            if (there) {   // no such page: parameters of 0, so that the result does not depend on what was here before
              set_status(IFQ_ERANGE);
              uint4* par = (uint4*)(smem + w * ST * U * GB + st * U * GB + u * GB + 16 * D);
              for (int i = 0; i < 8; ++i) par[i] = make_uint4(0, 0, 0, 0);
              fence_proxy_async_smem();   // (the next copy to this place comes after)
            }
            mbar_arrive(bar);
          }
          o += step;
          ++k;
          st = st + 1 < ST ? st + 1 : 0;
          idle = 0;
          look_up();
        } else {
          __nanosleep(40);   // (the computing warps' issue slots)
          if ((++idle & 255u) == 0) {
            const unsigned long long now = global_ns();
            if (idle == 256) t0 = now;
            else if (now - t0 > 2 * kWaitNs) {   // a computing warp gave up
              set_status(IFQ_ETIMEOUT);
              break;
            }
          }
        }
      }
      // the block's memory is there until its last copies have landed, also where a computing warp gave up
      for (int i = max(k - ST, 0); i < k; ++i) mbar_wait_backoff(bar_full + 8 * (w * ST + i % ST), (i / ST) & 1, 100);
    }
    return;
  }

  const uint8_t* ring = smem + warp * ST * U * GB;
  const int last = part_end(warp);
  int used = 0, co = part_begin(warp);
  bool alive = true, open = false;
  for (int o0 = one ? 0 : co; o0 < last;) {
    kv_advance<R, U>(A, cur, o0);
    const int o1 = min(last, cur.base + cur.nu);
    const int rb = cur.it / a.kv_heads, head = cur.it - rb * a.kv_heads, nrows = cur.q.n * a.group;
    const int p_lo = cur.q.len - cur.q.n + (int)kv_div(rb * R, A.by_group);
    const int p_hi = cur.q.len - cur.q.n + (int)kv_div(min(nrows, rb * R + R) - 1, A.by_group);
    // the rows: operand registers, and per column of the tiles (rows 2 tig, 2 tig + 1) the affine terms
    uint32_t qf[NT][KS][2];
    float fa[NT][2], fb[NT][2], m[NT][2], l[NT][2], z[NT][2];
    int prow[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = rb * R + nt * 8 + gid;
      const bool have = r < nrows;
      const int qi = kv_div(have ? r : 0, A.by_group);
      const uint16_t* src = a.q + (long long)(cur.q.first + qi) * a.q_stride +
                            (long long)(head * a.group + (have ? r - qi * a.group : 0)) * D + tig * (DB / 4);
      uint32_t w[NB * WPL * 4];
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < WPL; ++i) {
          const uint4 v = have ? *(const uint4*)(src + b * DB + 8 * i) : make_uint4(0, 0, 0, 0);
          w[(b * WPL + i) * 4] = v.x, w[(b * WPL + i) * 4 + 1] = v.y, w[(b * WPL + i) * 4 + 2] = v.z, w[(b * WPL + i) * 4 + 3] = v.w;
        }
      float top = 0.0f, sum = 0.0f;
#pragma unroll
      for (int i = 0; i < NB * WPL * 4; ++i) {
        const float2 f = unpack16<BF>(w[i]);
        top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y)));
        sum += f.x + f.y;
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      int e = (int)(__float_as_uint(top) >> 23) - 127 - 14;
      e = max(-100, min(113, e));
      const float down = __uint_as_float((uint32_t)(127 - e) << 23), low = down * 0.0625f;
#pragma unroll
      for (int i = 0; i < NB * WPL; ++i) {   // a word of codes: eight dimensions, in pairs (0,4) (1,5) (2,6) (3,7)
        const float2 f0 = unpack16<BF>(w[4 * i]), f1 = unpack16<BF>(w[4 * i + 1]);
        const float2 f2 = unpack16<BF>(w[4 * i + 2]), f3 = unpack16<BF>(w[4 * i + 3]);
        qf[nt][2 * i][0] = pack16<false>(f0.x * down, f2.x * down);
        qf[nt][2 * i][1] = pack16<false>(f0.y * low, f2.y * low);
        qf[nt][2 * i + 1][0] = pack16<false>(f1.x * down, f3.x * down);
        qf[nt][2 * i + 1][1] = pack16<false>(f1.y * low, f3.y * low);
      }
      const float sc = a.scale * 1.44269504f;
      const float va = sc * __uint_as_float((uint32_t)(127 + e) << 23), vb = sc * sum;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        fa[nt][c] = __shfl_sync(0xffffffffu, va, 8 * tig + 4 * c);
        fb[nt][c] = __shfl_sync(0xffffffffu, vb, 8 * tig + 4 * c);
        m[nt][c] = 0.0f;
        l[nt][c] = 0.0f;
        z[nt][c] = 0.0f;
        const int rc = rb * R + nt * 8 + 2 * tig + c;
        prow[nt][c] = rc < nrows ? cur.q.len - cur.q.n + (int)kv_div(rc, A.by_group) : -1;
      }
    }
    float o[MT][NT][4];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[i][nt][c] = 0.0f;
    float ow[NT][4];   // 8 sum w, as the products have it: values are taken about code 8, so that what rounding the
                       // weights changes goes with the values' spread and not with their distance from code 0
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 4; ++c) ow[nt][c] = 0.0f;
    uint32_t fresh = 0;   // columns that have no score yet, a bit each (theirs that are no rows never count)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) fresh |= (rb * R + nt * 8 + 2 * tig + c < nrows ? 1u : 0u) << (2 * nt + c);
    float vmul = 1.0f, vtop = 0.0f;   // factor of the value scales, and the scale that raises it

    for (; co < o1; co += step) {
      const int st = used % ST;
      if (alive) alive = mbar_wait(bar_full + 8 * (warp * ST + st), (used / ST) & 1);
      ++used;
      const uint8_t* unit = ring + st * U * GB;
      float s[U][NT][4];
      float2 v[U][2];
      uint32_t hidden = 0;   // of the lane's scores, 4 a tile
      float most = -INFINITY, wide = 0.0f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint8_t* g = unit + u * GB;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 4; ++c) s[u][nt][c] = 0.0f;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          uint32_t ka[WPL], kb[WPL];
          load_words(ka, g + b * 8 * DB + gid * (DB / 2) + tig * (DB / 8));
          load_words(kb, g + b * 8 * DB + (gid + 8) * (DB / 2) + tig * (DB / 8));
#pragma unroll
          for (int i = 0; i < WPL; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t x = h ? ka[i] >> 8 : ka[i], y = h ? kb[i] >> 8 : kb[i];
              const int k = (b * WPL + i) * 2 + h;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
                mma_f16(s[u][nt], x & 0x000f000fu, y & 0x000f000fu, x & 0x00f000f0u, y & 0x00f000f0u, qf[nt][k][0],
                        qf[nt][k][1]);
            }
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {   // the exponents t - m
        const uint32_t* par = (const uint32_t*)(unit + u * GB + 16 * D);
        float2 k0 = unpack16<false>(par[gid]), k1 = unpack16<false>(par[gid + 8]);
        k0.x *= 16777216.0f;   // the codes are in units of 2^-24
        k1.x *= 16777216.0f;
        v[u][0] = unpack16<false>(par[16 + gid]), v[u][1] = unpack16<false>(par[16 + gid + 8]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            s[u][nt][c] = s[u][nt][c] * (fa[nt][c] * k0.x) + (fb[nt][c] * k0.y - m[nt][c]);
            s[u][nt][2 + c] = s[u][nt][2 + c] * (fa[nt][c] * k1.x) + (fb[nt][c] * k1.y - m[nt][c]);
          }
      }
      const int g0 = (co - cur.base) * U;
      // all the unit's groups there, in reach of every row (and none of them past a gap)
      const int i0 = g0 < cur.sg ? g0 : g0 + cur.skip, j0 = i0 * kKvGroup, jn = j0 + U * kKvGroup;
      const bool full = jn - 1 <= p_lo && (g0 + U <= cur.sg || g0 >= cur.sg) &&
                        (a.window == 0 || j0 > p_hi - a.window || jn <= a.sinks);
      if (!full) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int gu = g0 + u, ju = (gu < cur.sg ? gu : gu + cur.skip) * kKvGroup + gid;
          const bool out0 = gu >= cur.ng || ju > p_hi, out1 = gu >= cur.ng || ju + 8 > p_hi;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 4; ++c)
              if ((c < 2 ? out0 : out1) || !kv_sees(a, prow[nt][c & 1], ju + (c & 2) * 4)) {
                hidden |= 1u << ((u * NT + nt) * 4 + c);
                s[u][nt][c] = -INFINITY;
              }
          // what no row sees may hold anything
          if (out0) v[u][0] = make_float2(0.0f, 0.0f);
          if (out1) v[u][1] = make_float2(0.0f, 0.0f);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 4; ++c) most = fmaxf(most, s[u][nt][c]);
        wide = fmaxf(wide, fmaxf(v[u][0].x, v[u][1].x));
      }
      if (__any_sync(0xffffffffu, most > 8.0f || wide > vtop || fresh)) {
        if (wide > 65504.0f) {   // an infinite scale: the factor is every row's, also theirs that do not see it
          wide = 0.0f;
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) wide = fmaxf(wide, v[u][h].x <= 65504.0f ? v[u][h].x : 0.0f);
        }
#pragma unroll
        for (int k = 4; k <= 16; k <<= 1) wide = fmaxf(wide, __shfl_xor_sync(0xffffffffu, wide, k));
        float vf = 1.0f;
        if (wide > vtop) {   // the largest scale to [2^5, 2^6); it may grow to 2^7 before the next time
          const uint32_t e = __float_as_uint(wide) >> 23;
          const float now = __uint_as_float((254u + 5u - e) << 23);
          vf = vtop == 0.0f ? 1.0f : now / vmul;
          vmul = now;
          vtop = 128.0f / now;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float t = -INFINITY;
#pragma unroll
            for (int u = 0; u < U; ++u) t = fmaxf(t, fmaxf(s[u][nt][c], s[u][nt][2 + c]));
#pragma unroll
            for (int k = 4; k <= 16; k <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, k));
            const uint32_t bit = 1u << (2 * nt + c);
            const bool begin = (fresh & bit) && t > -INFINITY;
            const float rise = begin || t > 8.0f ? t : 0.0f, f = begin ? 1.0f : exp2_fast(-rise);
            if (begin) fresh &= ~bit;
            m[nt][c] += rise;
#pragma unroll
            for (int u = 0; u < U; ++u) {
              s[u][nt][c] -= rise;
              s[u][nt][2 + c] -= rise;
            }
            l[nt][c] *= f;
            z[nt][c] *= f;
            ow[nt][c] *= f * vf;
#pragma unroll
            for (int i = 0; i < MT; ++i) {
              o[i][nt][c] *= f * vf;
              o[i][nt][2 + c] *= f * vf;
            }
          }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float w0 = v[u][0].x * vmul, w1 = v[u][1].x * vmul;
        const float c0 = v[u][0].y + 8.0f * v[u][0].x, c1 = v[u][1].y + 8.0f * v[u][1].x;   // the values of code 8
        uint32_t wf[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float p[4], w[4], y[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            p[c] = exp2_fast(s[u][nt][c]);
            w[c] = p[c] * (c < 2 ? w0 : w1);
            y[c] = p[c] * (c < 2 ? c0 : c1);
          }
          if (!full) {   // (a hidden token's parameters need not be numbers)
#pragma unroll
            for (int c = 0; c < 4; ++c)
              if (hidden >> ((u * NT + nt) * 4 + c) & 1u) w[c] = y[c] = 0.0f;
          }
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            l[nt][c] += p[c] + p[2 + c];
            z[nt][c] += y[c] + y[2 + c];
          }
          wf[nt][0] = transpose8x8(pack16<false>(w[0], w[1]));
          wf[nt][1] = transpose8x8(pack16<false>(w[2], w[3]));
          mma_f16(ow[nt], 0x00080008u, 0x00080008u, 0x00080008u, 0x00080008u, wf[nt][0], wf[nt][1]);
        }
        const uint8_t* g = unit + u * GB + 8 * D;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          uint32_t x[WPL], y[WPL];
          load_words(x, g + b * 8 * DB + lane * (DB / 8));
          load_words(y, g + b * 8 * DB + 4 * DB + lane * (DB / 8));
#pragma unroll
          for (int i = 0; i < WPL; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t p = h ? x[i] >> 8 : x[i], q = h ? y[i] >> 8 : y[i];
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
                mma_f16(o[(b * WPL + i) * 2 + h][nt], p & 0x000f000fu, p & 0x00f000f0u, q & 0x000f000fu, q & 0x00f000f0u,
                        wf[nt][0], wf[nt][1]);
            }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_empty + 8 * (warp * ST + st));
    }

    const bool whole = o0 == cur.base && o1 - cur.base == cur.nu;
    open = o0 == cur.base && !whole;
    const float back = 16777216.0f / vmul;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int k = 4; k <= 16; k <<= 1) {
          l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], k);
          z[nt][c] += __shfl_xor_sync(0xffffffffu, z[nt][c], k);
        }
        if (fresh >> (2 * nt + c) & 1u) m[nt][c] = kNoMax;
      }
    if (one) {
      // join the warps' sums: of each row the maximum, then everything relative to it
      if (gid == 0) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int r = warp * R + nt * 8 + 2 * tig + c;
            jm[r] = m[nt][c];
            jl[r] = l[nt][c];
            jz[r] = z[nt][c];
          }
      }
      named_bar(1, 32 * W);
#pragma unroll
      for (int pass = 0; pass < 2 * NT; ++pass) {   // four rows: those of half the lanes
        const int nt = pass >> 1, four = pass & 1;
        if (tig >> 1 == four) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int row = nt * 8 + 2 * tig + c;
            float top = kNoMax;
#pragma unroll
            for (int w = 0; w < W; ++w) top = fmaxf(top, jm[w * R + row]);
            const float f = exp2_fast(m[nt][c] - top) * back;
            float* dst = jO + (warp * 4 + (row & 3)) * (D + 4);
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
              for (int i = 0; i < WPL; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  const float* v = o[(b * WPL + i) * 2 + h][nt];
                  *(float2*)(dst + b * DB + gid * (DB / 8) + 4 * i + 2 * h) =
                      make_float2((v[c] - ow[nt][c]) * f, (v[2 + c] * 0.0625f - ow[nt][c]) * f);
                }
          }
        }
        named_bar(1, 32 * W);
        for (int i = threadIdx.x; i < 4 * D / 4; i += 32 * W) {   // four dimensions of a row each
          const int r4 = i / (D / 4), d0 = i % (D / 4) * 4, row = 4 * four + r4, r = rb * R + nt * 8 + row;
          if (r >= nrows) break;
          float top = kNoMax, sum = 0.0f, zs = 0.0f;
          float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
          for (int w = 0; w < W; ++w) top = fmaxf(top, jm[w * R + nt * 8 + row]);
#pragma unroll
          for (int w = 0; w < W; ++w) {
            const float f = exp2_fast(jm[w * R + nt * 8 + row] - top);
            sum += jl[w * R + nt * 8 + row] * f;
            zs += jz[w * R + nt * 8 + row] * f;
            const float4 x = *(const float4*)(jO + (w * 4 + r4) * (D + 4) + d0);
            v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w;
          }
          if (whole) {
            const int qi = kv_div(r, A.by_group), hq = head * a.group + r - qi * a.group;
            const long long t = cur.q.first + qi;
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            const uint32_t w[2] = {pack16<BF>((v.x + zs) * inv, (v.y + zs) * inv), pack16<BF>((v.z + zs) * inv, (v.w + zs) * inv)};
            store_words(a.out + t * a.out_stride + (long long)hq * D + d0, w);
            if (a.lse && d0 == 0)
              a.lse[t * a.q_heads + hq] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * 0.69314718f;
          } else {
            const long long at = ((long long)blockIdx.x * W * 2 + (o0 == cur.base ? 1 : 0)) * R + nt * 8 + row;
            *(float4*)(A.part + at * D + d0) = make_float4(v.x + zs, v.y + zs, v.z + zs, v.w + zs);
            if (d0 == 0) A.part_ml[at] = make_float2(top, sum);
          }
        }
        named_bar(1, 32 * W);
      }
      if (!whole && warp > 0)   // the block's part is the first warp's
        for (int r = lane; r < R; r += 32) A.part_ml[((long long)(blockIdx.x * W + warp) * 2) * R + r] = make_float2(kNoMax, 0.0f);
    } else {
      // this warp's own
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int row = nt * 8 + 2 * tig + c, r = rb * R + row;
          if (r >= nrows) continue;
          const int qi = kv_div(r, A.by_group), hq = head * a.group + r - qi * a.group;
          const long long t = cur.q.first + qi;
          const float inv = l[nt][c] == 0.0f ? 0.0f : 1.0f / l[nt][c], f = whole ? back * inv : back, zf = whole ? z[nt][c] * inv : z[nt][c];
          const long long at = ((long long)(blockIdx.x * W + warp) * 2 + (o0 == cur.base ? 1 : 0)) * R + row;
          uint16_t* out = a.out + t * a.out_stride + (long long)hq * D;
          float* part = A.part + at * D;
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < WPL; ++i)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const float* v = o[(b * WPL + i) * 2 + h][nt];
                const int d = b * DB + gid * (DB / 8) + 4 * i + 2 * h;
                const float x = (v[c] - ow[nt][c]) * f + zf, y = (v[2 + c] * 0.0625f - ow[nt][c]) * f + zf;
                if (whole) *(uint32_t*)(out + d) = pack16<BF>(x, y);
                else *(float2*)(part + d) = make_float2(x, y);
              }
          if (gid == 0) {
            if (!whole) A.part_ml[at] = make_float2(m[nt][c], l[nt][c]);
            else if (a.lse)
              a.lse[t * a.q_heads + hq] = l[nt][c] == 0.0f ? -INFINITY : (m[nt][c] + log2f(l[nt][c])) * 0.69314718f;
          }
        }
    }
    o0 = o1;
  }
  if (!A.direct && lane == 0) {
    // the parts that the item which this one leaves open reaches into: to the block and warp of its last unit
    int blocks = 0, w = 0;
    if (open && (!one || warp == 0)) {
      const long long to = (long long)cur.base + cur.nu - 1;
      const int blk = (int)(to / full_share), in = (int)(to - (long long)blk * full_share);
      const int units = (int)min((long long)full_share, ends - (long long)blk * full_share);
      blocks = blk + 1;
      w = (int)(((long long)(in + 1) * W - 1) / units);
    }
    A.cut[blockIdx.x * W + warp] = cuts[warp] = make_int4(cur.s, cur.it, blocks, w);
  }
  if (!A.direct && !one && part_begin(warp) == last)   // nothing: an item that others share has no sums here
    for (int r = lane; r < R; r += 32) A.part_ml[((long long)(blockIdx.x * W + warp) * 2) * R + r] = make_float2(kNoMax, 0.0f);
  if (A.direct || one) return;
  // the items that several warps of this block share and no other block: a warp an item and row
  named_bar(1, 32 * W);
  for (int i = warp; i < W * R; i += W) {
    const int w0 = i / R, row = i - w0 * R;
    const int4 cut = cuts[w0];
    if (cut.z != 1) continue;
    const KvSeq q = kv_seq(a, cut.x);
    const int rb = cut.y / a.kv_heads, head = cut.y - rb * a.kv_heads, r = rb * R + row;
    if (r >= q.n * a.group) continue;
    KvSum<D> t;
    t.add(A, lane, 0, 1, cut.w - w0 + 1, [&](int k) { return ((long long)(blockIdx.x * W + w0 + k) * 2 + (k == 0 ? 1 : 0)) * R + row; });
    t.template write<BF>(A, q, head, r, lane);
  }
}

// The parts of the item that a range leaves to the next ones: a block a range and row, its four warps a quarter of the
// parts each.  Of the ranges between the item's first and last it has all, in one part each.
template <int D, bool BF, int NT>
__global__ void __launch_bounds__(128) kv4_join_kernel(const __grid_constant__ KvRowsArgs A) {
  constexpr int R = 8 * NT, W = kKvRowsWarps;
  __shared__ float sv[4][D];
  __shared__ float2 ss[4];
  grid_dep_wait();
  grid_dep_launch();
  const KvAttnArgs& a = A.a;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, blk = blockIdx.x, row = blockIdx.y;
  const int4 mine = lane < W ? A.cut[blk * W + lane] : make_int4(0, 0, 0, 0);
  const uint32_t some = __ballot_sync(0xffffffffu, mine.z > 1);
  if (!some) return;
  const int w0 = __ffs(some) - 1;
  const int4 cut = make_int4(__shfl_sync(0xffffffffu, mine.x, w0), __shfl_sync(0xffffffffu, mine.y, w0),
                             __shfl_sync(0xffffffffu, mine.z, w0), __shfl_sync(0xffffffffu, mine.w, w0));
  const KvSeq q = kv_seq(a, cut.x);
  const int rb = cut.y / a.kv_heads, head = cut.y - rb * a.kv_heads, r = rb * R + row;
  if (r >= q.n * a.group) return;
  const int own = W - w0, mid = cut.z - 2, parts = own + mid + cut.w + 1;
  auto at = [&](int i) {
    const int p = i < own ? blk * W + w0 + i : i < own + mid ? (blk + 1 + i - own) * W : (blk + cut.z - 1) * W + i - own - mid;
    return ((long long)p * 2 + (i == 0 ? 1 : 0)) * R + row;
  };
  KvSum<D> t;
  for (int i0 = warp; i0 < parts; i0 += 128) t.add(A, lane, i0, 4, parts, at);
#pragma unroll
  for (int n = 0; n < t.N; ++n)
    if (lane * 4 + 128 * n < D) *(float4*)(sv[warp] + lane * 4 + 128 * n) = t.v[n];
  if (lane == 0) ss[warp] = make_float2(t.top, t.sum);
  __syncthreads();
  if (warp > 0) return;
#pragma unroll
  for (int k = 1; k < 4; ++k) t.add(ss[k], sv[k], lane);
  t.template write<BF>(A, q, head, r, lane);
}

}  // namespace ifq
