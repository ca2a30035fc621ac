// Products with weights in 4 bits: the packed layout, and the kernel that makes it.
//
// w = round(code * scale + min): one fma in the weights' type, so every kernel multiplies the same values.
//
// A row block is 16 packed rows: 16 rows of w, or of a gated pair the gate's rows 8 b .. 8 b + 7 and the other's after
// them, so that a lane that holds rows g and g + 8 of a block has both factors of an output.  A block of 128 columns
// of a row block is contiguous, 1024 bytes of codes and 64 of parameters a group; those of eight row blocks (a tile of 128
// rows) follow each other, and then those of the next 128 columns:
//   codes       [2 units of 64 columns][32 lanes][4 words]; the word of step j (16 columns) in lane 4 g + t holds four
//               pairs of neighbouring columns, pair i in the bits that rotating the word right by 4 i brings to
//               w4_at .. w4_at + 3 of either half: i = 0, 1: rows g, g + 8, columns 16 j + 2 t and the next; i = 2, 3: the
//               same rows, 8 columns further
//   parameters  [128 / group][8][2] pairs (scale, min): of row g, of row g + 8
// Behind the blocks stand 64 bytes whose first word says whether every scale is below 1/4 in size (0), see w4_expand: the
// scales stand there times 2^130 (bfloat16) or 2^18 (half) then.
// A pair of codes masked out of a word and made floats is thus one register of an mma.sync operand (A, 16 x 16), and a
// register of a tcgen05.st in 16-lane fragments.  Rows and columns past the matrix hold zeros up to whole tiles of 128.
#pragma once
#include "kv4.cuh"

namespace ifq {

constexpr int kW4Cols = 128, kW4Tail = 64;
__host__ __device__ constexpr int w4_at(bool bf) { return bf ? 3 : 6; }   // first bit of a code: the upper ones of a mantissa

__host__ __device__ constexpr int w4_block_bytes(int group) { return 1024 + 64 * (kW4Cols / group); }
// Where block kb of row block rb stands, in blocks.
__host__ __device__ constexpr long long w4_place(long long rb, int kb, int blocks) { return (rb / 8 * blocks + kb) * 8 + rb % 8; }

struct W4Args {
  const uint8_t* w;
  const uint32_t* large;   // a word behind the blocks: 0 if no scale is 1/4 or more
  const uint16_t* x;
  const void* res;     // NULL: none
  void* out;
  long long x_stride, res_stride, out_stride;
  int m, n, k, kb;     // kb: blocks of 128 columns
  int out_type, act;
};

// act(a) of a gated pair.  The exponentials are of -|.|, so that none overflows.
__device__ __forceinline__ float w4_sigmoid(float a) {
  const float e = __expf(-fabsf(a)), s = __fdividef(1.0f, 1.0f + e);
  return a < 0.0f ? e * s : s;
}
__device__ __forceinline__ float w4_act(int act, float a) {
  if (act == IFQ_ACT_SILU) return a * w4_sigmoid(a);
  if (act == IFQ_ACT_GELU) return 0.5f * a * erfcf(-0.70710678118654752f * a);
  return a * w4_sigmoid(1.5957691216057308f * (a + 0.044715f * a * a * a));
}

__device__ __forceinline__ float w4_load(int type, const void* p, long long at) {
  if (type == IFQ_F32) return ((const float*)p)[at];
  if (type == IFQ_F16) return __half2float(((const __half*)p)[at]);
  return __bfloat162float(((const __nv_bfloat16*)p)[at]);
}
__device__ __forceinline__ void w4_store(int type, void* p, long long at, float v) {
  if (type == IFQ_F32) ((float*)p)[at] = v;
  else if (type == IFQ_F16) ((__half*)p)[at] = __float2half_rn(v);
  else ((__nv_bfloat16*)p)[at] = __float2bfloat16_rn(v);
}

// A word's four pairs of codes to 16-bit values: rows g (s[0], m[0]) and g + 8 (s[1], m[1]), each code * scale + min with
// one rounding.
//
// FAST: the masked code is a number as it stands, a subnormal one, code * 2^-130 in bfloat16 and code * 2^-18 in half, which
// the fma takes as exactly as any other; the packed scale carries the factor that is missing, and must be below 1/4 for it
// to be finite.  Otherwise the code is made the mantissa of 16 + code, from which 16 is taken: one operation more for each pair.
template <bool BF, bool FAST>
__device__ __forceinline__ void w4_expand(uint32_t w, const uint32_t (&s)[2], const uint32_t (&m)[2], uint32_t* v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t c = __funnelshift_r(w, w, 4 * i) & (0x000f000fu << w4_at(BF));
    if (!FAST) c |= BF ? 0x41804180u : 0x4c004c00u;
    if constexpr (BF) {
      if (!FAST) asm("{.reg .b32 t; mov.b32 t, 0xc180c180; add.rn.bf16x2 %0, %0, t;}" : "+r"(c));
      asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(v[i]) : "r"(c), "r"(s[i & 1]), "r"(m[i & 1]));
    } else {
      if (!FAST) asm("{.reg .b32 t; mov.b32 t, 0xcc00cc00; add.rn.f16x2 %0, %0, t;}" : "+r"(c));
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

// ---------------------------------------------------------------- packing

struct W4PackArgs {
  const uint8_t* codes;
  const uint16_t *scales, *mins;
  uint8_t* out;
  uint32_t* large;
  int n, k, kb, groups, gated;
  int row_blocks;   // all of them, those past the matrix too
};

constexpr int kW4PackWarps = 8;

// Whether a scale is 1/4 or more, an infinity or a NaN (a.large begins at 0; all that write write the same).
template <bool BF>
__global__ void __launch_bounds__(256) w4_scan_kernel(const __grid_constant__ W4PackArgs a) {
  grid_dep_wait();
  grid_dep_launch();
  const long long total = (long long)a.n * (a.gated ? 2 : 1) * a.groups;
  bool any = false;
  for (long long i = blockIdx.x * 256ll + threadIdx.x; i < total; i += 256ll * gridDim.x)
    any |= (a.scales[i] & 0x7fffu) >= (BF ? 0x3e80u : 0x3400u);
  if (__any_sync(0xffffffffu, any) && threadIdx.x % 32 == 0) *a.large = 1;
}

// Run once a matrix (131072 x 4096 in 138 us with the scan).  A warp makes one block (16 rows x 128 columns): its codes go through shared
// memory, where a row has 17 words, so that the bytes that a lane gathers (rows g and g + 8) lie in different banks.
template <bool BF, int G>
__global__ void __launch_bounds__(32 * kW4PackWarps) w4_pack_kernel(const __grid_constant__ W4PackArgs a) {
  grid_dep_wait();
  grid_dep_launch();
  __shared__ uint32_t turn[kW4PackWarps][16 * 17];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane / 4, t = lane % 4;
  uint32_t* in = turn[warp];
  const long long blocks = (long long)a.row_blocks * a.kb, words = a.k / 8;
  const bool large = *a.large != 0;
  const auto source = [&](long long rb, int r) -> long long {   // the row of the matrix, or -1
    const long long j = a.gated ? rb * 8 + r % 8 : rb * 16 + r;
    return j >= a.n ? -1 : a.gated && r >= 8 ? j + a.n : j;
  };
  for (long long b = (long long)blockIdx.x * kW4PackWarps + warp; b < blocks; b += (long long)gridDim.x * kW4PackWarps) {
    const long long rb = b / (8ll * a.kb) * 8 + b % 8;
    const int kb = (int)(b / 8 % a.kb);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = 2 * i + lane / 16, c = lane % 16;
      const long long j = source(rb, r), at = kb * 16ll + c;
      in[r * 17 + c] = j >= 0 && at < words ? ((const uint32_t*)a.codes)[j * words + at] : 0u;
    }
    __syncwarp();
    uint8_t* out = a.out + b * w4_block_bytes(G);
    const uint8_t* bytes = (const uint8_t*)in;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        w[j] = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t v = bytes[(g + 8 * (i & 1)) * 68 + (64 * u + 16 * j + 2 * t + 8 * (i >> 1)) / 2];
          const uint32_t two = ((v & 15u) | (v >> 4) << 16) << w4_at(BF);
          w[j] |= __funnelshift_l(two, two, 4 * i);
        }
      }
      *(uint4*)(out + 512 * u + 16 * lane) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    for (int i = lane; i < 16 * (kW4Cols / G); i += 32) {
      const int q = i / 16, r = i % 16;
      const long long j = source(rb, r), at = (long long)kb * (kW4Cols / G) + q;
      uint32_t v = 0;
      if (j >= 0 && at < a.groups) {
        float scale = unpack16<BF>(a.scales[j * a.groups + at]).x;
        if (!large) scale *= BF ? 0x1p65f : 0x1p9f, scale *= BF ? 0x1p65f : 0x1p9f;   // (exact)
        v = (pack16<BF>(scale, 0.0f) & 0xffffu) | (uint32_t)a.mins[j * a.groups + at] << 16;
      }
      *(uint32_t*)(out + 1024 + 64 * q + 8 * (r % 8) + 4 * (r / 8)) = v;
    }
    __syncwarp();
  }
}

}  // namespace ifq
