// The paged 4-bit key/value cache: its layout, and the kernels that write tokens into it and read
// them back.
//
// A group holds 16 tokens of one head (ifq.h): K codes, V codes, K parameters, V parameters.  K codes
// are row by row; a 32-bit word of V codes holds the same four dimensions of two neighbouring tokens.
// In both the attention kernels take a word apart with masks alone into pairs of codes that are
// operand registers of the tensor cores (see kv4_attention.cuh).
//
// Both kernels move each value once and do little with it: they are bound by memory (and by their
// launch where a call has few tokens).
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

struct KvCacheArgs {
  uint8_t* p;
  long long slots;     // pages * page_size
  int page_size;
  int kv_heads;
};
__device__ __forceinline__ uint8_t* kv4_group(const KvCacheArgs& c, int D, long long slot, int head) {
  const long long page = slot / c.page_size;
  const int row = (int)(slot - page * c.page_size);
  return c.p + ((page * c.kv_heads + head) * (c.page_size / kKvGroup) + row / kKvGroup) * (long long)kv4_group_bytes(D);
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
  int rope, rot, positions;
};

constexpr int kAppendWarps = 8;

// One warp a row (a head of q, k or v of a token), head size D = 32 E: lane l holds dimensions E l .. E l + E - 1.
// In the pairs (i, i + rot/2) the partner of a lane's dimensions is a whole lane's (rot/2 is a multiple of 8 >= E).
template <int D, bool BF>
__global__ void __launch_bounds__(32 * kAppendWarps) kv4_append_kernel(const KvAppendArgs a) {
  constexpr int E = D / 32;
  grid_dep_wait();
  const int rows = a.q_heads + 2 * a.cache.kv_heads;
  const long long item = (long long)blockIdx.x * kAppendWarps + (threadIdx.x >> 5);
  if (item >= (long long)a.tokens * rows) return;
  const int lane = threadIdx.x & 31, d0 = lane * E;
  const int t = (int)(item / rows), r = (int)(item - (long long)t * rows);
  const bool is_q = r < a.q_heads, is_v = r >= a.q_heads + a.cache.kv_heads;
  const int head = is_q ? r : (r - a.q_heads) % a.cache.kv_heads;
  const long long slot = a.slots[t];
  int pos = 0;
  if (a.rope != IFQ_ROPE_NONE) {
    pos = a.pos[t];
    if (pos < 0 || pos >= a.positions) {
      if (lane == 0) set_status(IFQ_ERANGE);
      return;
    }
  }
  if (slot >= a.cache.slots) {
    if (lane == 0) set_status(IFQ_ERANGE);
    return;
  }
  if (!is_q && slot < 0) return;

  const uint16_t* src = is_q   ? a.q + t * a.q_stride + head * D
                        : is_v ? a.v + t * a.v_stride + head * D
                               : a.k + t * a.k_stride + head * D;
  uint32_t w[E / 2];
  load_words(w, src + d0);
  float x[E];
#pragma unroll
  for (int i = 0; i < E / 2; ++i) {
    const float2 f = unpack16<BF>(w[i]);
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
  if (!is_v && a.rope == IFQ_ROPE_HALVES) {
    const int half = a.rot / 2, hl = half / E;
    const bool first = d0 < half, turned = d0 < a.rot;
    uint32_t pw[E / 2];
#pragma unroll
    for (int i = 0; i < E / 2; ++i) pw[i] = __shfl_sync(0xffffffffu, w[i], (turned ? (first ? lane + hl : lane - hl) : lane));
    if (turned) {
      const float* c = a.cos + (long long)pos * half + (first ? d0 : d0 - half);
      const float* s = a.sin + (long long)pos * half + (first ? d0 : d0 - half);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float2 f = unpack16<BF>(pw[i / 2]);
        const float p = i % 2 ? f.y : f.x;
        const float m = __fmul_rn(x[i], c[i]), n = __fmul_rn(p, s[i]);
        x[i] = first ? __fsub_rn(m, n) : __fadd_rn(m, n);   // a cos - b sin, b cos + a sin
      }
    }
  } else if (!is_v && a.rope == IFQ_ROPE_PAIRS && d0 < a.rot) {
    const float* c = a.cos + (long long)pos * (a.rot / 2) + d0 / 2;
    const float* s = a.sin + (long long)pos * (a.rot / 2) + d0 / 2;
#pragma unroll
    for (int i = 0; i < E; i += 2) {
      const float u = x[i], v = x[i + 1], cc = c[i / 2], ss = s[i / 2];
      x[i] = __fsub_rn(__fmul_rn(u, cc), __fmul_rn(v, ss));
      x[i + 1] = __fadd_rn(__fmul_rn(v, cc), __fmul_rn(u, ss));
    }
  }
  if (is_q) {
#pragma unroll
    for (int i = 0; i < E / 2; ++i) w[i] = pack16<BF>(x[2 * i], x[2 * i + 1]);
    store_words(a.q_out + t * a.q_out_stride + head * D + d0, w);
    return;
  }

  float lo = 65504.0f, hi = -65504.0f;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    x[i] = min_nan(max_nan(x[i], -65504.0f), 65504.0f);
    lo = min_nan(lo, x[i]);
    hi = max_nan(hi, x[i]);
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  const __half hs = __float2half_rn(__fmul_rn(__fsub_rn(hi, lo), 1.0f / 15.0f)), hm = __float2half_rn(lo);
  const float sc = __half2float(hs), mn = __half2float(hm);
  uint32_t code[E];
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const float c = rintf(__fdiv_rn(__fsub_rn(x[i], mn), sc));
    code[i] = sc > 0.0f ? (uint32_t)fminf(fmaxf(c, 0.0f), 15.0f) : 0u;   // (also 0 where the scale is NaN)
  }
  uint8_t* g = kv4_group(a.cache, D, slot, head);
  const int row = (int)(slot % a.cache.page_size) % kKvGroup;
  uint8_t b[E / 2];
#pragma unroll
  for (int i = 0; i < E / 2; ++i) b[i] = (uint8_t)(code[2 * i] | code[2 * i + 1] << 4);
  if (is_v) {
#pragma unroll
    for (int i = 0; i < E / 2; i += 2) {
      uint8_t* p = g + kv4_v_byte(D, row, d0 + 2 * i);
      if constexpr (E >= 4) *(uint16_t*)p = (uint16_t)(b[i] | b[i + 1] << 8);
      else *p = b[i];
    }
  } else {
    uint8_t* p = g + kv4_k_byte(D, row, d0);
    if constexpr (E == 2) *p = b[0];
    else if constexpr (E == 4) *(uint16_t*)p = (uint16_t)(b[0] | b[1] << 8);
    else *(uint32_t*)p = (uint32_t)b[0] | (uint32_t)b[1] << 8 | (uint32_t)b[2] << 16 | (uint32_t)b[3] << 24;
  }
  if (lane == 0)
    *(uint32_t*)(g + 16 * D + (is_v ? 64 : 0) + 4 * row) =
        (uint32_t)__half_as_ushort(hs) | (uint32_t)__half_as_ushort(hm) << 16;
}

struct KvReadArgs {
  KvCacheArgs cache;
  const int64_t* slots;
  uint16_t *k_out, *v_out;
  int tokens;
};

// One warp a head of a token's K or V.
template <int D, bool BF>
__global__ void __launch_bounds__(32 * kAppendWarps) kv4_read_kernel(const KvReadArgs a) {
  constexpr int E = D / 32;
  grid_dep_wait();
  const int hk = a.cache.kv_heads;
  const long long item = (long long)blockIdx.x * kAppendWarps + (threadIdx.x >> 5);
  if (item >= (long long)a.tokens * 2 * hk) return;
  const int lane = threadIdx.x & 31, d0 = lane * E;
  const int t = (int)(item / (2 * hk)), r = (int)(item - (long long)t * 2 * hk), head = r % hk;
  const bool is_v = r >= hk;
  uint16_t* out = is_v ? a.v_out : a.k_out;
  if (!out) return;
  const long long slot = a.slots[t];
  if (slot >= a.cache.slots && lane == 0) set_status(IFQ_ERANGE);
  uint32_t w[E / 2];
  if (slot < 0 || slot >= a.cache.slots) {
#pragma unroll
    for (int i = 0; i < E / 2; ++i) w[i] = 0;
  } else {
    const uint8_t* g = kv4_group(a.cache, D, slot, head);
    const int row = (int)(slot % a.cache.page_size) % kKvGroup;
    const float2 par = __half22float2(*(const __half2*)(g + 16 * D + (is_v ? 64 : 0) + 4 * row));
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
      const uint32_t b = g[is_v ? kv4_v_byte(D, row, d0 + 2 * i) : kv4_k_byte(D, row, d0 + 2 * i)];
      w[i] = pack16<BF>(__fadd_rn(__fmul_rn((float)(b & 15u), par.x), par.y),
                        __fadd_rn(__fmul_rn((float)(b >> 4), par.x), par.y));
    }
  }
  store_words(out + ((long long)t * hk + head) * D + d0, w);
}

}  // namespace ifq
