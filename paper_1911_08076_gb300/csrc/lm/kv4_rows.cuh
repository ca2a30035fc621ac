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
// Work: the groups of all items in a row are cut into as many equal ranges as there are blocks, whatever the lengths
// (an item cut by a range's end leaves partial sums in the workspace, joined by kv4_join_kernel); or, where no
// sequence is long, one block an item.  Each warp takes every W-th group of its block's range, with a ring of its own
// filled by bulk copies (one contiguous block a group), across the ends of items; at an item's end the warps' sums
// are joined in shared memory.
#pragma once
#include "kv4_attention.cuh"

namespace ifq {

constexpr float kNoMax = -3.0e38f;   // stands for the maximum of nothing

struct KvDiv {   // n / d for 0 <= n < 2^31
  uint32_t d, mul, shift;
};
__device__ __forceinline__ uint32_t kv_div(uint32_t n, const KvDiv& f) {
  return (uint32_t)(((uint64_t)__umulhi(n, f.mul) + n) >> f.shift);
}

struct KvRowsArgs {
  KvAttnArgs a;
  KvDiv by_gpp, by_group;   // groups a page, query heads a key head
  int direct;               // one block an item: blockIdx = (key head, block of rows, sequence)
  // workspace of the ranges: parts [blocks][2][R][D], their (max, sum) [blocks][2][R], and who is cut [blocks]
  float* part;
  float2* part_ml;
  int4* cut;                // (sequence, block of rows * key heads + head, parts, 0) of the item a range leaves open
};

template <int D>
struct KvRowsShape {
  static constexpr int W = D == 256 ? 4 : 8;        // warps
  static constexpr int stages = D == 64 ? 6 : 4;    // groups in flight a warp
};
template <int D>
__host__ __device__ constexpr int kv_rows_smem(int R) {
  using C = KvRowsShape<D>;
  return C::W * C::stages * (kv4_group_bytes(D) + 8) + C::W * 8 * (D + 4) * 4 + 3 * C::W * R * 4 + 64 * 8 + 64;
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
  int ng, sg, skip;
  int base;        // where the item starts, relative to the block's range
};

template <int R>
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
}
// Move on to the item that holds offset o of the range.
template <int R>
__device__ __forceinline__ void kv_advance(const KvRowsArgs& A, KvCursor& c, int o) {
  while (o >= c.base + c.ng) {
    c.base += c.ng;
    if (++c.it >= c.nit) {
      c.it = 0;
      do {
        ++c.s;
        kv_shape<R>(A, c);
      } while (c.nit == 0);
    }
  }
}

template <int D, bool BF, int NT>
__global__ void __launch_bounds__(32 * KvRowsShape<D>::W, NT == 1 ? 2 : 1) kv4_rows_kernel(const __grid_constant__ KvRowsArgs A) {
  using C = KvRowsShape<D>;
  constexpr int W = C::W, ST = C::stages, R = 8 * NT, GB = kv4_group_bytes(D);
  constexpr int DB = kv4_block(D), NB = D / DB, WPL = DB / 32;   // blocks of dimensions, words a lane and row
  constexpr int KS = D / 16, MT = D / 16;                        // steps along d of S, tiles along d of O
  extern __shared__ __align__(128) uint8_t smem[];
  const KvAttnArgs& a = A.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
  uint8_t* ring = smem + warp * ST * GB;
  float* jO = (float*)(smem + W * ST * GB);                 // [W][8][D + 4]
  float* jm = jO + W * 8 * (D + 4);                         // [W][R] each
  float *jl = jm + W * R, *jz = jl + W * R;
  uint64_t* bars = (uint64_t*)(jz + W * R);                 // [W][ST]
  long long* scan = (long long*)(bars + W * ST);            // [W + 1]
  __shared__ int first[4];
  const uint32_t bar0 = smem_u32(bars + warp * ST);
  if (lane == 0) {
    for (int i = 0; i < ST; ++i) mbar_init(bar0 + 8 * i, 1);
    fence_mbar_init();
  }
  __syncwarp();
  grid_dep_wait();
  grid_dep_launch();

  KvCursor cur;
  int n;        // groups of this block
  if (A.direct) {
    cur.s = blockIdx.z;
    kv_shape<R>(A, cur);
    if (!cur.q.ok && threadIdx.x == 0) set_status(IFQ_ERANGE);
    cur.it = blockIdx.y * a.kv_heads + blockIdx.x;
    cur.base = 0;
    if (cur.it >= cur.nit) return;
    n = cur.ng;
  } else {
    // the groups of every sequence, summed over the block's threads' shares of the sequences
    const int per = (a.seqs + 32 * W - 1) / (32 * W), s0 = threadIdx.x * per, s1 = min(a.seqs, s0 + per);
    long long mine = 0;
    for (int s = s0; s < s1; ++s) {
      KvCursor t;
      t.s = s;
      kv_shape<R>(A, t);
      if (!t.q.ok && blockIdx.x == 0) set_status(IFQ_ERANGE);
      mine += (long long)t.nit * t.ng;
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
    for (int w = 0; w < W; ++w) {
      if (w < warp) before += scan[w];
      total += scan[w];
    }
    long long share = (total + gridDim.x - 1) / gridDim.x;
    if (share < 2 * W) share = 2 * W;
    const long long start = share * blockIdx.x;
    if (start >= total) {
      if (threadIdx.x == 0) A.cut[blockIdx.x] = make_int4(0, 0, 0, 0);
      return;
    }
    n = (int)min(share, total - start);
    if (start >= before && start < before + mine) {   // one thread: its sequences hold the start
      long long at = before;
      KvCursor t;
      t.s = s0;
      for (;; ++t.s) {
        kv_shape<R>(A, t);
        const long long c = (long long)t.nit * t.ng;
        if (start < at + c) break;
        at += c;
      }
      const long long in = start - at;
      first[0] = t.s;
      first[1] = (int)(in / t.ng);
      first[2] = (int)(in % t.ng);
    }
    __syncthreads();
    cur.s = first[0];
    kv_shape<R>(A, cur);
    cur.it = first[1];
    cur.base = -first[2];
  }

  // the producer's side: the next group to fetch, in order; its page is looked up one fetch ahead
  KvCursor pro = cur;
  int po = warp;          // its offset
  int issued = 0, page = 0, where = 0, pro_head = 0;
  bool there = false;
  auto look_up = [&]() {
    if (po < n) {
      kv_advance<R>(A, pro, po);
      const int g = po - pro.base, gi = g < pro.sg ? g : g + pro.skip;
      const int pi = kv_div(gi, A.by_gpp);
      where = gi - pi * A.by_gpp.d;
      pro_head = pro.it % a.kv_heads;
      there = gi * kKvGroup < pro.q.len;
      if (there) page = a.table[(long long)pro.s * a.max_pages + pi];
    }
  };
  auto fetch = [&]() {
    if (po < n) {
      const int st = issued % ST;
      if (lane == 0) {
        const bool good = there && page >= 0 && page < a.pages;
        if (good) {
          const uint8_t* src = a.cache + (((long long)page * a.kv_heads + pro_head) * A.by_gpp.d + where) * GB;
          mbar_arrive_expect_tx(bar0 + 8 * st, GB);
          bulk_copy_g2s(smem_u32(ring + st * GB), src, GB, bar0 + 8 * st);
        } else {
          if (there) set_status(IFQ_ERANGE);
          mbar_arrive(bar0 + 8 * st);
        }
      }
      ++issued;
      po += W;
      look_up();
    }
  };
  look_up();
#pragma unroll
  for (int i = 0; i < ST; ++i) fetch();

  int used = 0, co = warp;
  bool alive = true;
  for (int o0 = 0; o0 < n;) {
    kv_advance<R>(A, cur, o0);
    const int o1 = min(n, cur.base + cur.ng);
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
        m[nt][c] = kNoMax;
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
    float vmul = 1.0f, vtop = 0.0f;   // factor of the value scales, and the scale that raises it

    for (; co < o1; co += W) {
      const int st = used % ST;
      if (alive) alive = mbar_wait(bar0 + 8 * st, (used / ST) & 1);
      ++used;
      const uint8_t* g = ring + st * GB;
      const int gg = co - cur.base, gi = gg < cur.sg ? gg : gg + cur.skip, j0 = gi * kKvGroup;
      float s[NT][4], s2[NT][4];   // two chains of products
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 4; ++c) s[nt][c] = s2[nt][c] = 0.0f;
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
              mma_f16(h ? s2[nt] : s[nt], x & 0x000f000fu, y & 0x000f000fu, x & 0x00f000f0u, y & 0x00f000f0u, qf[nt][k][0], qf[nt][k][1]);
          }
      }
      const uint32_t* par = (const uint32_t*)(g + 16 * D);
      const float2 k0 = unpack16<false>(par[gid]), k1 = unpack16<false>(par[gid + 8]);
      float2 v0 = unpack16<false>(par[16 + gid]), v1 = unpack16<false>(par[16 + gid + 8]);
      const float ks0 = k0.x * 16777216.0f, ks1 = k1.x * 16777216.0f;
      const bool full = j0 + kKvGroup - 1 <= p_lo && (a.window == 0 || j0 > p_hi - a.window || j0 + kKvGroup <= a.sinks);
      uint32_t hidden = 0;   // of the lane's four scores a tile
      bool up = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          s[nt][c] = ((s[nt][c] + s2[nt][c]) * fa[nt][c]) * ks0 + fb[nt][c] * k0.y;
          s[nt][2 + c] = ((s[nt][2 + c] + s2[nt][2 + c]) * fa[nt][c]) * ks1 + fb[nt][c] * k1.y;
        }
      if (!full) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            if (!kv_sees(a, prow[nt][c & 1], j0 + gid + (c & 2) * 4)) {
              hidden |= 1u << (4 * nt + c);
              s[nt][c] = -INFINITY;
            }
          }
        // scales of tokens that no row sees must not raise the factor
        if (j0 + gid > p_hi) v0 = make_float2(0.0f, 0.0f);
        if (j0 + gid + 8 > p_hi) v1 = make_float2(0.0f, 0.0f);
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) up |= fmaxf(s[nt][c], s[nt][2 + c]) > m[nt][c] + 8.0f;
      up |= fmaxf(v0.x, v1.x) > vtop;
      if (__any_sync(0xffffffffu, up)) {
        float vm = fmaxf(v0.x, v1.x);
#pragma unroll
        for (int k = 4; k <= 16; k <<= 1) vm = fmaxf(vm, __shfl_xor_sync(0xffffffffu, vm, k));
        float vf = 1.0f;
        if (vm > vtop) {   // the largest scale to [2^5, 2^6); it may grow to 2^7 before the next time
          const uint32_t e = __float_as_uint(vm) >> 23;
          const float now = __uint_as_float((254u + 5u - e) << 23);
          vf = vtop == 0.0f ? 1.0f : now / vmul;
          vmul = now;
          vtop = 128.0f / now;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float t = fmaxf(s[nt][c], s[nt][2 + c]);
#pragma unroll
            for (int k = 4; k <= 16; k <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, k));
            const float now = t > m[nt][c] + 8.0f ? t : m[nt][c];
            const float f = exp2_fast(m[nt][c] - now);
            m[nt][c] = now;
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
      const float w0 = v0.x * vmul, w1 = v1.x * vmul;
      v0.y += 8.0f * v0.x;   // the value of code 8
      v1.y += 8.0f * v1.x;
      uint32_t wf[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float p[4], w[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          p[c] = exp2_fast(s[nt][c] - m[nt][c & 1]);
          w[c] = p[c] * (c < 2 ? w0 : w1);
        }
        if (!full) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (hidden >> (4 * nt + c) & 1u) w[c] = 0.0f;
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          l[nt][c] += p[c] + p[2 + c];
          const bool h0 = !full && (hidden >> (4 * nt + c) & 1u), h1 = !full && (hidden >> (4 * nt + 2 + c) & 1u);
          z[nt][c] += (h0 ? 0.0f : p[c] * v0.y) + (h1 ? 0.0f : p[2 + c] * v1.y);
        }
        wf[nt][0] = transpose8x8(pack16<false>(w[0], w[1]));
        wf[nt][1] = transpose8x8(pack16<false>(w[2], w[3]));
        mma_f16(ow[nt], 0x00080008u, 0x00080008u, 0x00080008u, 0x00080008u, wf[nt][0], wf[nt][1]);
      }
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        uint32_t x[WPL], y[WPL];
        load_words(x, g + 8 * D + b * 8 * DB + lane * (DB / 8));
        load_words(y, g + 8 * D + b * 8 * DB + 4 * DB + lane * (DB / 8));
#pragma unroll
        for (int i = 0; i < WPL; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t u = h ? x[i] >> 8 : x[i], v = h ? y[i] >> 8 : y[i];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
              mma_f16(o[(b * WPL + i) * 2 + h][nt], u & 0x000f000fu, u & 0x00f000f0u, v & 0x000f000fu, v & 0x00f000f0u,
                      wf[nt][0], wf[nt][1]);
          }
      }
      __syncwarp();
      fetch();
    }

    // join the warps' sums: of each row the maximum, then everything relative to it
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int k = 4; k <= 16; k <<= 1) {
          l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], k);
          z[nt][c] += __shfl_xor_sync(0xffffffffu, z[nt][c], k);
        }
        if (gid == 0) {
          const int r = warp * R + nt * 8 + 2 * tig + c;
          jm[r] = m[nt][c];
          jl[r] = l[nt][c];
          jz[r] = z[nt][c];
        }
      }
    __syncthreads();
    const bool whole = o0 - cur.base == 0 && o1 - cur.base == cur.ng;
    const float back = 16777216.0f / vmul;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int row = 2 * tig + c;
        float top = kNoMax;
#pragma unroll
        for (int w = 0; w < W; ++w) top = fmaxf(top, jm[w * R + nt * 8 + row]);
        const float f = exp2_fast(m[nt][c] - top) * back;
        float* dst = jO + (warp * 8 + row) * (D + 4);
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
      __syncthreads();
      constexpr int kPer = 8 * D / (32 * W);          // consecutive dimensions of a row a thread
      const int row = threadIdx.x / (D / kPer), d0 = (threadIdx.x % (D / kPer)) * kPer;
      const int r = rb * R + nt * 8 + row;
      if (r < nrows) {
        float top = kNoMax, sum = 0.0f, zs = 0.0f, v[kPer];
#pragma unroll
        for (int w = 0; w < W; ++w) top = fmaxf(top, jm[w * R + nt * 8 + row]);
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[i] = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
          const float f = exp2_fast(jm[w * R + nt * 8 + row] - top);
          sum += jl[w * R + nt * 8 + row] * f;
          zs += jz[w * R + nt * 8 + row] * f;
#pragma unroll
          for (int i = 0; i < kPer; i += 2) {
            const float2 t = *(const float2*)(jO + (w * 8 + row) * (D + 4) + d0 + i);
            v[i] += t.x;
            v[i + 1] += t.y;
          }
        }
        if (whole) {
          const int qi = kv_div(r, A.by_group), hq = head * a.group + r - qi * a.group;
          const long long t = cur.q.first + qi;
          const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
          constexpr int kW = kPer / 2 < 4 ? kPer / 2 : 4;   // words a store
#pragma unroll
          for (int i = 0; i < kPer / 2; i += kW) {
            uint32_t w[kW];
#pragma unroll
            for (int k = 0; k < kW; ++k)
              w[k] = pack16<BF>((v[2 * (i + k)] + zs) * inv, (v[2 * (i + k) + 1] + zs) * inv);
            store_words(a.out + t * a.out_stride + (long long)hq * D + d0 + 2 * i, w);
          }
          if (a.lse && d0 == 0)
            a.lse[t * a.q_heads + hq] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * 0.69314718f;
        } else {
          const int slot = o0 == cur.base ? 1 : 0;   // an item left open by the range's end, or one begun before it
          const long long at = ((long long)blockIdx.x * 2 + slot) * R + nt * 8 + row;
#pragma unroll
          for (int i = 0; i < kPer; i += 2) *(float2*)(A.part + at * D + d0 + i) = make_float2(v[i] + zs, v[i + 1] + zs);
          if (d0 == 0) A.part_ml[at] = make_float2(top, sum);
        }
      }
      __syncthreads();
    }
    if (!A.direct && o1 == n && threadIdx.x == 0) {
      const bool open = o0 == cur.base && !whole;
      // the ranges that the item's groups reach into: each has n groups, the last one or fewer
      const int rest = cur.ng - (o1 - o0);
      A.cut[blockIdx.x] = make_int4(cur.s, cur.it, open ? 1 + (rest + n - 1) / n : 0, 0);
    }
    o0 = o1;
  }
}

// The parts of an item that several ranges share: one block a range and a row; the range that begins the item does it.
template <int D, bool BF, int NT>
__global__ void __launch_bounds__(128) kv4_join_kernel(const __grid_constant__ KvRowsArgs A) {
  constexpr int R = 8 * NT, T = D / 4, P = 128 / T > 0 ? 128 / T : 1;   // threads a row's dimensions, parts at once
  __shared__ float4 sv[P][T];
  __shared__ float ss[P], st[4];
  grid_dep_wait();
  grid_dep_launch();
  const KvAttnArgs& a = A.a;
  const int4 cut = A.cut[blockIdx.x];
  const int parts = cut.z;
  if (parts == 0) return;
  KvCursor c;
  c.s = cut.x;
  kv_shape<R>(A, c);
  const int rb = cut.y / a.kv_heads, head = cut.y - rb * a.kv_heads, r = rb * R + blockIdx.y;
  if (r >= c.q.n * a.group) return;
  auto at = [&](int i) { return ((long long)(blockIdx.x + i) * 2 + (i == 0 ? 1 : 0)) * R + blockIdx.y; };
  float top = kNoMax;
  for (int i = threadIdx.x; i < parts; i += 128) top = fmaxf(top, A.part_ml[at(i)].x);
#pragma unroll
  for (int k = 16; k; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
  if (threadIdx.x % 32 == 0) st[threadIdx.x / 32] = top;
  __syncthreads();
  top = fmaxf(fmaxf(st[0], st[1]), fmaxf(st[2], st[3]));
  const int d = threadIdx.x % T, p0 = threadIdx.x / T;
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  float sum = 0.0f;
  if (p0 < P)
#pragma unroll 4
    for (int i = p0; i < parts; i += P) {
      const float2 ml = A.part_ml[at(i)];
      const float f = exp2_fast(ml.x - top);
      const float4 x = *(const float4*)(A.part + at(i) * D + 4 * d);
      v.x += x.x * f, v.y += x.y * f, v.z += x.z * f, v.w += x.w * f;
      sum += ml.y * f;
    }
  if (p0 < P) {
    sv[p0][d] = v;
    if (d == 0) ss[p0] = sum;
  }
  __syncthreads();
  if (threadIdx.x < T) {
    v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    sum = 0.0f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const float4 x = sv[p][d];
      v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w;
      sum += ss[p];
    }
    const int qi = kv_div(r, A.by_group), hq = head * a.group + r - qi * a.group;
    const long long t = c.q.first + qi;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    uint32_t w[2] = {pack16<BF>(v.x * inv, v.y * inv), pack16<BF>(v.z * inv, v.w * inv)};
    store_words(a.out + t * a.out_stride + (long long)hq * D + 4 * d, w);
    if (a.lse && d == 0) a.lse[t * a.q_heads + hq] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * 0.69314718f;
  }
}

}  // namespace ifq
