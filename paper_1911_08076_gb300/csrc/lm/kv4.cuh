// The paged 4-bit key/value cache: its layout, and the kernels that write tokens into it and read
// them back.
//
// A group holds 16 tokens of one head (ifq.h): K codes, V codes, K parameters, V parameters.  K codes
// are row by row; a 32-bit word of V codes holds the same four dimensions of two neighbouring tokens.
// In both the attention kernels take a word apart with masks alone into pairs of codes that are
// operand registers of the tensor cores (see kv4_attention.cuh).
//
// Both kernels move each value once: memory is their floor (and their launch where a call has few tokens).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

#include "../ptx.cuh"

namespace ifq {

constexpr int kKvGroup = 16;   // tokens per group

__host__ __device__ constexpr int kv4_group_bytes(int D) { return 16 * D + 128; }
__host__ __device__ constexpr int kv4_block(int D) { return D < 128 ? D : 128; }   // DB

// Byte of a group that holds the K code of (row, d) / the V code of (row, d), d even (d + 1 is its high half).
__device__ __forceinline__ int kv4_k_byte(int D, int row, int d) {
  const int DB = kv4_block(D);
  return (d / DB) * 8 * DB + row * (DB / 2) + (d % DB) / 2;
}
__device__ __forceinline__ int kv4_v_byte(int D, int row, int d) {
  const int DB = kv4_block(D), S = DB / 8, dd = d % DB;
  return 8 * D + (d / DB) * 8 * DB + (row / 8) * 4 * DB + ((dd / S) * 4 + (row % 8) / 2) * S + ((dd % S) / 4) * 4 +
         (row % 2) * 2 + (dd % 4) / 2;
}

struct KvDiv {   // n / d for 0 <= n < 2^31
  uint32_t d, mul, shift;
};
__device__ __forceinline__ uint32_t kv_div(uint32_t n, const KvDiv& f) {
  return (uint32_t)(((uint64_t)__umulhi(n, f.mul) + n) >> f.shift);
}

struct KvCacheArgs {
  uint8_t* p;
  long long slots;     // pages * page_size
  KvDiv by_page;       // tokens a page
  int kv_heads;
};
// Page of a slot and row in it (a 64-bit division only past 2^31 slots).
__device__ __forceinline__ void kv4_place(const KvCacheArgs& c, long long slot, long long& page, int& row) {
  page = c.slots <= 0x7fffffffll ? (long long)kv_div((uint32_t)slot, c.by_page) : slot / (long long)c.by_page.d;
  row = (int)(slot - page * c.by_page.d);
}
__device__ __forceinline__ uint8_t* kv4_group(const KvCacheArgs& c, int D, long long page, int row, int head) {
  return c.p + ((page * c.kv_heads + head) * (long long)(c.by_page.d / kKvGroup) + row / kKvGroup) * kv4_group_bytes(D);
}

__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// 16-bit types: two values of a 32-bit word, and back.
template <bool BF>
__device__ __forceinline__ float2 unpack16(uint32_t w) {
  if constexpr (BF) return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w));
  else return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <bool BF>
__device__ __forceinline__ uint32_t pack16(float a, float b) {
  if constexpr (BF) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
  } else {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
}

// N 32-bit words from / to memory in one access (N = 1, 2, 4).
template <int N>
__device__ __forceinline__ void load_words(uint32_t (&w)[N], const void* p) {
  if constexpr (N == 1) w[0] = *(const uint32_t*)p;
  else if constexpr (N == 2) { const uint2 v = *(const uint2*)p; w[0] = v.x; w[1] = v.y; }
  else { const uint4 v = *(const uint4*)p; w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
}
template <int N>
__device__ __forceinline__ void store_words(void* p, const uint32_t (&w)[N]) {
  if constexpr (N == 1) *(uint32_t*)p = w[0];
  else if constexpr (N == 2) *(uint2*)p = make_uint2(w[0], w[1]);
  else *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
}

struct KvAppendArgs {
  KvCacheArgs cache;
  const uint16_t *q, *k, *v;
  uint16_t* q_out;
  const float *cos, *sin;
  const int32_t* pos;
  const int64_t* slots;
  long long q_stride, k_stride, v_stride, q_out_stride;
  int tokens, q_heads;   // q_heads = 0: no q
  int rope, rot, positions, vec;   // vec: the tables are 16-byte aligned
};

// Both kernels: eight dimensions (16 bytes) a lane, so D / 8 lanes a head and 256 / D heads a warp at once, kKvPass
// times; a warp's heads are of one token and one kind (q, k or v).  blockIdx.y: the kind and its heads, blockIdx.x:
// eight tokens.  The heads' loads are all under way before the first is used, and cos and sin are read once for them
// (8191 tokens of 32 + 2 x 8 heads of 128: 57 us, 2.6 TB/s of DRAM traffic, with 60 % of the issue slots at work on the exact steps, and
// 14 us reading them back; with a head a warp and 8-byte loads 104 and 31).
constexpr int kAppendWarps = 8, kKvPass = 4;
__host__ __device__ constexpr int kv4_warp_heads(int D) { return kKvPass * 256 / D; }

// Head size D; in the pairs (i, i + rot/2) the partner of a lane's dimensions is a whole lane's (rot/2 is a multiple of 8).
template <int D, bool BF>
__global__ void __launch_bounds__(32 * kAppendWarps) kv4_append_kernel(const __grid_constant__ KvAppendArgs a) {
  constexpr int L = D / 8, HP = 32 / L, HB = kv4_warp_heads(D);   // lanes a head, heads a pass, heads a warp
  grid_dep_wait();
  grid_dep_launch();
  const int t = blockIdx.x * kAppendWarps + (threadIdx.x >> 5);
  if (t >= a.tokens) return;
  const int lane = threadIdx.x & 31, dl = lane % L, d0 = 8 * dl;
  const int qb = (a.q_heads + HB - 1) / HB, kb = (a.cache.kv_heads + HB - 1) / HB;
  const int y = blockIdx.y;
  const bool is_q = y < qb, is_v = y >= qb + kb;
  const int heads = is_q ? a.q_heads : a.cache.kv_heads, h0 = (is_q ? y : is_v ? y - qb - kb : y - qb) * HB + lane / L;
  const uint16_t* src = (is_q ? a.q + t * a.q_stride : is_v ? a.v + t * a.v_stride : a.k + t * a.k_stride) + d0;
  uint32_t w[kKvPass][4];
#pragma unroll
  for (int u = 0; u < kKvPass; ++u) {
    const int h = h0 + u * HP;
    w[u][0] = w[u][1] = w[u][2] = w[u][3] = 0;
    if (h < heads) load_words(w[u], src + (long long)h * D);
  }
  const long long slot = a.slots[t];
  const bool turn = a.rope != IFQ_ROPE_NONE;
  const int pos = turn ? a.pos[t] : 0;
  if ((turn && (pos < 0 || pos >= a.positions)) || slot >= a.cache.slots) {
    if (lane == 0) set_status(IFQ_ERANGE);
    return;
  }
  if (!is_q && slot < 0) return;

  const int half = a.rot / 2;
  const bool turned = turn && !is_v && d0 < a.rot, halves = a.rope == IFQ_ROPE_HALVES;
  const bool first = d0 < half;
  float cs[8], sn[8];
  if (turned) {   // halves: a lane's eight pairs; pairs: its four
    const int at = halves ? (first ? d0 : d0 - half) : d0 / 2;
    const float *c = a.cos + (long long)pos * half + at, *s = a.sin + (long long)pos * half + at;
#pragma unroll
    for (int i = 0; i < 8; i += 4)
      if (halves || i < 4) {
        const float4 u = a.vec ? *(const float4*)(c + i) : make_float4(c[i], c[i + 1], c[i + 2], c[i + 3]);
        const float4 v = a.vec ? *(const float4*)(s + i) : make_float4(s[i], s[i + 1], s[i + 2], s[i + 3]);
        cs[i] = u.x, cs[i + 1] = u.y, cs[i + 2] = u.z, cs[i + 3] = u.w;
        sn[i] = v.x, sn[i + 1] = v.y, sn[i + 2] = v.z, sn[i + 3] = v.w;
      }
  }
  long long page = 0;
  int row = 0;
  if (!is_q) kv4_place(a.cache, slot, page, row);

#pragma unroll
  for (int u = 0; u < kKvPass; ++u) {
    const int h = h0 + u * HP;
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = unpack16<BF>(w[u][i]);
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
    if (!is_v && turn) {
      if (halves) {
        const int from = turned ? (first ? lane + half / 8 : lane - half / 8) : lane;
        uint32_t pw[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) pw[i] = __shfl_sync(0xffffffffu, w[u][i], from);
        if (turned) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float2 f = unpack16<BF>(pw[i / 2]);
            const float m = __fmul_rn(x[i], cs[i]), n = __fmul_rn(i % 2 ? f.y : f.x, sn[i]);
            x[i] = first ? __fsub_rn(m, n) : __fadd_rn(m, n);   // a cos - b sin, b cos + a sin
          }
        }
      } else if (turned) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const float p = x[i], q = x[i + 1], c = cs[i / 2], s = sn[i / 2];
          x[i] = __fsub_rn(__fmul_rn(p, c), __fmul_rn(q, s));
          x[i + 1] = __fadd_rn(__fmul_rn(q, c), __fmul_rn(p, s));
        }
      }
    }
    if (is_q) {
      if (h < heads) {
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = pack16<BF>(x[2 * i], x[2 * i + 1]);
        store_words(a.q_out + t * a.q_out_stride + (long long)h * D + d0, o);
      }
      continue;
    }
    float lo = 65504.0f, hi = -65504.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = min_nan(max_nan(x[i], -65504.0f), 65504.0f);
      lo = min_nan(lo, x[i]);
      hi = max_nan(hi, x[i]);
    }
#pragma unroll
    for (int o = L / 2; o; o >>= 1) {
      lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
      hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    const __half hs = __float2half_rn(__fmul_rn(__fsub_rn(hi, lo), 1.0f / 15.0f)), hm = __float2half_rn(lo);
    const float sc = __half2float(hs), mn = __half2float(hm);
    uint32_t code = 0;
    if (sc > 0.0f) {   // (0 where the scale is NaN)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        code |= (uint32_t)fminf(fmaxf(rintf(__fdiv_rn(__fsub_rn(x[i], mn), sc)), 0.0f), 15.0f) << (4 * i);
    }
    if (h < heads) {
      uint8_t* g = kv4_group(a.cache, D, page, row, h);
      const int r = row % kKvGroup;
      if (is_v) {
        *(uint16_t*)(g + kv4_v_byte(D, r, d0)) = (uint16_t)code;
        *(uint16_t*)(g + kv4_v_byte(D, r, d0 + 4)) = (uint16_t)(code >> 16);
      } else {
        *(uint32_t*)(g + kv4_k_byte(D, r, d0)) = code;
      }
      if (dl == 0)
        *(uint32_t*)(g + 16 * D + (is_v ? 64 : 0) + 4 * r) = (uint32_t)__half_as_ushort(hs) | (uint32_t)__half_as_ushort(hm) << 16;
    }
    __syncwarp();
  }
}

struct KvReadArgs {
  KvCacheArgs cache;
  const int64_t* slots;
  uint16_t *k_out, *v_out;
  int tokens;
};

template <int D, bool BF>
__global__ void __launch_bounds__(32 * kAppendWarps) kv4_read_kernel(const __grid_constant__ KvReadArgs a) {
  constexpr int L = D / 8, HP = 32 / L, HB = kv4_warp_heads(D);
  grid_dep_wait();
  grid_dep_launch();
  const int t = blockIdx.x * kAppendWarps + (threadIdx.x >> 5);
  if (t >= a.tokens) return;
  const int lane = threadIdx.x & 31, dl = lane % L, d0 = 8 * dl, hk = a.cache.kv_heads, kb = (hk + HB - 1) / HB;
  const bool is_v = (int)blockIdx.y >= kb;
  uint16_t* out = is_v ? a.v_out : a.k_out;
  if (!out) return;
  const int h0 = (is_v ? blockIdx.y - kb : blockIdx.y) * HB + lane / L;
  const long long slot = a.slots[t];
  const bool there = slot >= 0 && slot < a.cache.slots;
  if (slot >= a.cache.slots && lane == 0) set_status(IFQ_ERANGE);
  uint32_t code[kKvPass], par[kKvPass];
  long long page = 0;
  int row = 0;
  if (there) kv4_place(a.cache, slot, page, row);
  const int r = row % kKvGroup;
#pragma unroll
  for (int u = 0; u < kKvPass; ++u) {
    const int h = h0 + u * HP;
    code[u] = par[u] = 0;
    if (there && h < hk) {
      const uint8_t* g = kv4_group(a.cache, D, page, row, h);
      par[u] = *(const uint32_t*)(g + 16 * D + (is_v ? 64 : 0) + 4 * r);
      if (is_v)
        code[u] = (uint32_t) * (const uint16_t*)(g + kv4_v_byte(D, r, d0)) | (uint32_t) * (const uint16_t*)(g + kv4_v_byte(D, r, d0 + 4)) << 16;
      else
        code[u] = *(const uint32_t*)(g + kv4_k_byte(D, r, d0));
    }
  }
#pragma unroll
  for (int u = 0; u < kKvPass; ++u) {
    const int h = h0 + u * HP;
    const float2 p = unpack16<false>(par[u]);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t c = code[u] >> (8 * i);
      w[i] = pack16<BF>(__fadd_rn(__fmul_rn((float)(c & 15u), p.x), p.y), __fadd_rn(__fmul_rn((float)(c >> 4 & 15u), p.x), p.y));
    }
    if (h < hk) store_words(out + ((long long)t * hk + h) * D + d0, w);
  }
}

}  // namespace ifq
