// C ABI entry points of the attention block of a quantised decoder: the paged 4-bit key/value cache,
// attention over it, and products in e4m3 with block scales.
#include "lm_api.h"

#include <cmath>
#include <algorithm>
#include <type_traits>

#include "fp8.cuh"
#include "ifq.h"
#include "kv4.cuh"
#include "kv4_attention.cuh"
#include "kv4_chunk.cuh"
#include "kv4_rows.cuh"
#include "lm_host.h"

namespace {

using namespace ifq;

// The kernel instance of a head size and type: f(head size, bfloat16) with both as types.
template <int D, typename F>
int by_type(int dtype, F&& f) {
  return dtype == IFQ_BF16 ? f(std::integral_constant<int, D>(), std::true_type())
                           : f(std::integral_constant<int, D>(), std::false_type());
}
template <typename F>
int by_head(int head_dim, int dtype, F&& f) {
  switch (head_dim) {
    case 64: return by_type<64>(dtype, f);
    case 128: return by_type<128>(dtype, f);
    default: return by_type<256>(dtype, f);
  }
}

int check_cache(const ifq_kv4_cache* c, size_t* bytes) {
  if (c->pages < 1 || c->page_size < 1 || c->kv_heads < 1 || c->head_dim < 1) return IFQ_EINVAL;
  if (c->page_size % kKvGroup != 0) return IFQ_ESHAPE;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return IFQ_EUNSUPPORTED;
  // (sizes are ints: the product of three, and of the fourth, is checked against overflow)
  const double b = (double)c->pages * c->page_size * c->kv_heads * (c->head_dim + 8);
  if (b > 4e18 || (double)c->pages * c->page_size > 4e18 || c->kv_heads > 65536) return IFQ_ERANGE;
  *bytes = (size_t)c->pages * c->kv_heads * (c->page_size / kKvGroup) * kv4_group_bytes(c->head_dim);
  return IFQ_OK;
}

KvDiv make_div(uint32_t d) {
  KvDiv f;
  f.d = d;
  f.shift = 0;
  while ((1ull << f.shift) < d) ++f.shift;
  f.mul = (uint32_t)(((1ull << 32) * ((1ull << f.shift) - d)) / d + 1ull);
  return f;
}

KvCacheArgs cache_args(const ifq_kv4_cache& c, const void* p) {
  KvCacheArgs a;
  a.p = (uint8_t*)p;
  a.slots = (long long)c.pages * c.page_size;
  a.by_page = make_div(c.page_size);
  a.kv_heads = c.kv_heads;
  return a;
}

// ---------------------------------------------------------------- attention

int check_attention(const ifq_kv4_attention_desc* d, KvAttnArgs* a) {
  if (!d) return IFQ_EINVAL;
  size_t bytes;
  int rc = check_cache(&d->cache, &bytes);
  if (rc) return rc;
  if (d->seqs < 0 || d->q_tokens < 0 || d->max_q < 0 || d->max_pages < 0 || d->max_len < 0 || d->q_heads < 1 ||
      d->window < 0 || d->sinks < 0 || !is16(d->dtype) || !std::isfinite(d->scale))
    return IFQ_EINVAL;
  if (d->q_heads % d->cache.kv_heads != 0) return IFQ_ESHAPE;
  if (d->q_heads > 65536 || (long long)d->max_pages * d->cache.page_size > kMaxSize ||
      (long long)d->max_q * d->q_heads > kMaxSize || d->seqs > kMaxSize || d->q_tokens > kMaxSize)
    return IFQ_ERANGE;
  const long long width = (long long)d->q_heads * d->cache.head_dim;
  if ((rc = stride_of(d->q_stride, width, &a->q_stride))) return rc;
  if ((rc = stride_of(d->out_stride, width, &a->out_stride))) return rc;
  a->pages = d->cache.pages;
  a->page_size = d->cache.page_size;
  a->kv_heads = d->cache.kv_heads;
  a->seqs = d->seqs;
  a->q_tokens = d->q_tokens;
  a->max_q = d->max_q;
  a->max_pages = d->max_pages;
  a->q_heads = d->q_heads;
  a->group = d->q_heads / d->cache.kv_heads;
  a->window = d->window;
  a->sinks = d->sinks;
  a->scale = d->scale;
  return IFQ_OK;
}

// Rows of a key head from which the kernel for many may be taken.
constexpr int kChunkRows = 32;

// Whether it is.  The kernel for few reads the cache once for every 8 or 16 rows, the one for many once for 128 or 256,
// but expands it to halves first and takes longer to begin.  In picoseconds a token and key head, measured with 5 to 40
// queries on up to 4096 tokens (16 x 5 queries of 8 heads a key head, 40 rows: 53 against 66 us; 2 x 40 of 4, 160 rows:
// 12.6 against 24; 16 x 12 of 8 with heads of 64, 96 rows: 30 against 18).
bool take_chunk(int D, long long rows, int nt, long long tokens) {
  const double pass = D == 64 ? 80 : 64, block = D == 64 ? 94 : D == 128 ? 160 : 460;
  const double few = pass * ((rows + 8 * nt - 1) / (8 * nt));
  const double many = rows <= 128 ? block : D < 256 ? 1.25 * block * ((rows + 255) / 256) : block * ((rows + 127) / 128);
  return rows > kChunkRows && few * tokens > many * tokens + 24e6;
}

struct AttnPlan {
  int chunk;       // the kernel for many rows (kv4_chunk.cuh): row tiles of 128 a block; 0: that for few
  int splits;      // chunk: blocks that a block's keys are split over
  int nt;          // few rows: row tiles of an item
  int direct;      // a block an item
  int blocks;      // of a sequence's rows (chunk, direct), or ranges
  size_t ws;
};

int plan_attention(const ifq_kv4_attention_desc* d, const KvAttnArgs& a, AttnPlan* p) {
  const int D = d->cache.head_dim;
  const long long rows = (long long)d->max_q * a.group;
  long long reach = (long long)d->max_pages * d->cache.page_size;   // tokens that a sequence's queries read at most
  if (d->max_len > 0) reach = std::min<long long>(reach, d->max_len);
  if (d->window > 0) reach = std::min<long long>(reach, (long long)d->window + d->sinks + d->max_q + 2 * kKvGroup);
  p->nt = rows > 8 && D < 256 ? 2 : 1;   // (two tiles of size 256 do not fit the registers)
  if (d->seqs <= 65535 && a.kv_heads <= 65535 && take_chunk(D, rows, p->nt, reach * d->seqs * a.kv_heads)) {
    p->chunk = rows > 128 && D < 256 ? 2 : 1;
    const int R = 128 * p->chunk;
    p->blocks = (int)((rows + R - 1) / R);
    const long long all = (long long)d->seqs * a.kv_heads * p->blocks, tiles = (reach + kChunkKeys - 1) / kChunkKeys;
    p->splits = (int)std::max<long long>(1, std::min({sm_count() / std::max<long long>(all, 1), tiles / 2, 65535ll / std::max(d->seqs, 1)}));
    p->ws = p->splits > 1 ? round_up((size_t)all * p->splits * R * (D * 4 + 8), 256) : 0;
    return IFQ_OK;
  }
  p->chunk = 0;
  const int R = 8 * p->nt;
  const long long blocks = std::max<long long>(1, (rows + R - 1) / R);   // (the device checks max_q = 0 too)
  // A block an item, or ranges: the longer of an item's units in seven warps and of what all items leave to an SM,
  // against three quarters of all units evenly spread and a longer start and a second kernel.  (Microseconds as measured:
  // 64 windows of 1028 tokens, two heads of 64: 7.8 against 16 to 18; 6 sequences of up to 1233, four heads of 64: in
  // ranges 11.3.)
  const int per_sm = kv_rows_per_sm(D, p->nt), unit = kKvGroup * (D == 64 ? 4 : 2), sms = sm_count();
  const double items = (double)blocks * a.kv_heads * d->seqs, units = (double)((reach + unit - 1) / unit);
  const double us = D == 64 ? 1.6 : D == 128 ? 1.45 : 2.2, lanes = (double)kKvRowsWarps * per_sm * sms;
  const double alone = 4.5 + us * std::ceil(units / kKvRowsWarps) * std::max(1.0, items / (per_sm * sms));
  const double spread = 9.5 + us * std::ceil(0.75 * items * units / lanes);
  p->direct = alone < spread && blocks <= 65535 && d->seqs <= 65535;
  p->blocks = p->direct ? (int)blocks : sms * per_sm;
  p->ws = p->direct ? 0 : round_up((size_t)p->blocks * kKvRowsWarps * (2 * R * (D * 4 + 8) + 16), 256);
  return IFQ_OK;
}

template <int D, bool BF, int RT>
int run_chunk(const KvAttnArgs& a, const AttnPlan& p, void* ws, cudaStream_t st) {
  using C = KvChunkShape<D, RT>;
  static bool set[kMaxDevices];
  const int rc = allow_smem(kv4_chunk_kernel<D, BF, RT>, C::bytes, set);
  if (rc) return rc;
  KvChunkArgs r = {};
  r.a = a;
  r.by_gpp = make_div(a.page_size / kKvGroup);
  r.by_group = make_div(a.group);
  r.blocks = p.blocks;
  r.splits = p.splits;
  if (p.splits > 1) {
    r.part = (float*)ws;
    r.part_ml = (float2*)(r.part + (size_t)a.seqs * a.kv_heads * p.blocks * p.splits * 128 * RT * D);
  }
  const cudaError_t e = launch_k(kv4_chunk_kernel<D, BF, RT>, dim3(p.blocks, a.kv_heads, a.seqs * p.splits), dim3(C::threads),
                                 C::bytes, st, r);
  if (e != cudaSuccess || p.splits == 1) return done(e);
  const int rows = a.max_q * a.group;
  return done(launch_k(kv4_chunk_join_kernel<D, BF>, dim3(ceil_div(rows, 8), a.kv_heads, a.seqs), dim3(256), 0, st, r, 128 * RT));
}

template <int D, bool BF, int NT>
int run_rows(const KvAttnArgs& a, const AttnPlan& p, void* ws, cudaStream_t st) {
  constexpr int R = 8 * NT, smem = kv_rows_smem<D>(R);
  static_assert(smem <= 232448, "shared memory budget");
  static bool set[kMaxDevices];
  const int rc = allow_smem(kv4_rows_kernel<D, BF, NT>, smem, set);
  if (rc) return rc;
  KvRowsArgs r = {};
  r.a = a;
  r.by_gpp = make_div(a.page_size / kKvGroup);
  r.by_group = make_div(a.group);
  r.direct = p.direct;
  if (!p.direct) {
    r.cut = (int4*)ws;
    r.part_ml = (float2*)(r.cut + p.blocks * kKvRowsWarps);
    r.part = (float*)(r.part_ml + (size_t)p.blocks * kKvRowsWarps * 2 * R);
  }
  const dim3 grid = p.direct ? dim3(a.kv_heads, p.blocks, a.seqs) : dim3(p.blocks);
  const cudaError_t e = launch_k(kv4_rows_kernel<D, BF, NT>, grid, dim3(KvRowsShape<D>::threads), smem, st, r);
  if (e != cudaSuccess || p.direct) return done(e);
  return done(launch_k(kv4_join_kernel<D, BF, NT>, dim3(p.blocks, R), dim3(128), 0, st, r));
}

// ---------------------------------------------------------------- products in e4m3

struct Fp8Operands {
  const void* x;
  const float* xs;
  const void* w;
  const float* ws;
  void* out;
  cudaStream_t st;
};

// TMA descriptor of an e4m3 operand: [rows][k] bytes, boxes of `box` rows x 128 bytes in the 128-byte swizzle; rows and
// columns past the end read as zeros.
bool encode_e4m3(const void* p, int rows, int k, int box, CUtensorMap* tm) {
  const cuuint64_t gdim[2] = {(cuuint64_t)k, (cuuint64_t)rows}, gstride[1] = {(cuuint64_t)k};
  const cuuint32_t bdim[2] = {(cuuint32_t)kFp8Block, (cuuint32_t)box}, estr[2] = {1, 1};
  return g_encode(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(p), gdim, gstride, bdim, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr int kFp8MaxSplit = 8;

// One-time setup of an instance on the current device: its shared memory, and how many clusters of each size run at
// once (in `slots`; a plain launch is size 1).
template <int BN, bool SWAP>
int fp8_setup(const int** slots) {
  static int known[kMaxDevices][kFp8MaxSplit + 1];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return IFQ_ECUDA;
  const int sms = sm_count();
  std::lock_guard<std::mutex> lk(g_lm_mu);
  int* s = known[dev];
  if (!s[1]) {
    using C = Fp8Shape<BN, SWAP>;
    auto kern = fp8_matmul_kernel<BN, SWAP>;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::bytes) != cudaSuccess) return IFQ_ECUDA;
    for (int ks = 2; C::split && ks <= kFp8MaxSplit; ++ks) {
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3((unsigned)(sms / ks * ks));
      cfg.blockDim = dim3(C::threads);
      cfg.dynamicSmemBytes = C::bytes;
      cudaLaunchAttribute at[1];
      at[0].id = cudaLaunchAttributeClusterDimension;
      at[0].val.clusterDim.x = (unsigned)ks;
      at[0].val.clusterDim.y = 1;
      at[0].val.clusterDim.z = 1;
      cfg.attrs = at;
      cfg.numAttrs = 1;
      int n = 0;
      s[ks] = cudaOccupancyMaxActiveClusters(&n, kern, &cfg) == cudaSuccess ? n : 0;
    }
    cudaGetLastError();   // (a cluster size that does not fit is no error of this call)
    s[1] = sms;
  }
  *slots = s;
  return IFQ_OK;
}

template <int BN, bool SWAP>
int run_fp8(const ifq_fp8_desc* d, const Fp8Operands& o) {
  using C = Fp8Shape<BN, SWAP>;
  const int* slots;
  const int rc = fp8_setup<BN, SWAP>(&slots);
  if (rc) return rc;
  Fp8Args a;
  a.xs = o.xs;
  a.ws = o.ws;
  a.out = o.out;
  a.out_stride = d->out_stride ? d->out_stride : d->n;
  a.m = d->m;
  a.n = d->n;
  a.kb = ceil_div(d->k, kFp8Block);
  a.out_type = d->out_dtype;
  a.vec = a.out_stride * (d->out_dtype == IFQ_F32 ? 4 : 2) % 16 == 0;
  a.tiles_a = ceil_div(SWAP ? d->n : d->m, 128);
  a.tiles_b = ceil_div(SWAP ? d->m : d->n, BN);
  const long long tiles = (long long)a.tiles_a * a.tiles_b;
  if (tiles > INT_MAX / kFp8MaxSplit) return IFQ_ERANGE;
  a.tiles = (int)tiles;
  // The tiles of a last turn that fills half of the SMs or less are cut in two.
  a.whole = a.tiles;
  const int rest = a.tiles % slots[1];
  if (C::wide && 2 * rest <= slots[1]) {
    a.whole -= rest;
    a.tiles += rest;
  }
  // the split of k with the fewest blocks of k in a row, each launch or cluster also costing as much as a few blocks
  a.ks = 1;
  double best = (double)ceil_div(a.tiles, slots[1]) * (a.kb + 6);
  for (int ks = 2; C::split && ks <= kFp8MaxSplit && ks <= a.kb; ++ks) {
    if (slots[ks] < 1) continue;
    const double c = (double)ceil_div(a.tiles, slots[ks]) * (ceil_div(a.kb, ks) + 6) + 4;
    if (c < best) best = c, a.ks = ks;
  }
  CUtensorMap tx, tw;
  const int box = std::min(BN, 128);
  if (!encode_e4m3(o.x, d->m, d->k, SWAP ? box : 128, &tx) || !encode_e4m3(o.w, d->n, d->k, SWAP ? 128 : box, &tw)) return IFQ_ECUDA;
  const CUtensorMap &ta = SWAP ? tw : tx, &tb = SWAP ? tx : tw;
  if (a.ks > 1)
    return done(launch_k_cluster(fp8_matmul_kernel<BN, SWAP>, a.ks, dim3((unsigned)(a.tiles * a.ks)), dim3(C::threads), C::bytes,
                                 o.st, ta, tb, a));
  return done(launch_k(fp8_matmul_kernel<BN, SWAP>, dim3((unsigned)std::min(a.tiles, slots[1])), dim3(C::threads), C::bytes, o.st,
                       ta, tb, a));
}

}  // namespace

namespace ifq {

int lm_take_status(int* status) {
  int v = 0, zero = 0;
  if (cudaMemcpyFromSymbol(&v, g_status, sizeof(int)) != cudaSuccess) return IFQ_ECUDA;
  if (v != 0 && cudaMemcpyToSymbol(g_status, &zero, sizeof(int)) != cudaSuccess) return IFQ_ECUDA;
  *status = v;
  return IFQ_OK;
}

}  // namespace ifq

extern "C" {

int ifq_kv4_cache_bytes(const ifq_kv4_cache* c, size_t* bytes) {
  if (!c || !bytes) return IFQ_EINVAL;
  return check_cache(c, bytes);
}

int ifq_kv4_append(const ifq_kv4_append_desc* d, const void* q, const void* k, const void* v, const float* cos,
                   const float* sin, const int32_t* positions, const int64_t* slots, void* q_out, void* cache,
                   void* stream) {
  if (!d) return IFQ_EINVAL;
  size_t bytes;
  int rc = check_cache(&d->cache, &bytes);
  if (rc) return rc;
  const int D = d->cache.head_dim;
  if (d->tokens < 0 || d->q_heads < 0 || !is16(d->dtype)) return IFQ_EINVAL;
  if (d->q_heads > 65536 || d->tokens > kMaxSize) return IFQ_ERANGE;
  if (d->rope != IFQ_ROPE_NONE && d->rope != IFQ_ROPE_HALVES && d->rope != IFQ_ROPE_PAIRS) return IFQ_EINVAL;
  if (d->rope != IFQ_ROPE_NONE && (d->rot_dim < 16 || d->rot_dim > D || d->rot_dim % 16 != 0)) return IFQ_ESHAPE;
  if (d->rope != IFQ_ROPE_NONE && d->positions < 1) return IFQ_EINVAL;
  KvAppendArgs a = {};
  if (q && (rc = stride_of(d->q_stride, (long long)d->q_heads * D, &a.q_stride))) return rc;
  if (q && (rc = stride_of(d->q_out_stride, (long long)d->q_heads * D, &a.q_out_stride))) return rc;
  if ((rc = stride_of(d->k_stride, (long long)d->cache.kv_heads * D, &a.k_stride))) return rc;
  if ((rc = stride_of(d->v_stride, (long long)d->cache.kv_heads * D, &a.v_stride))) return rc;
  if (!d->tokens) return IFQ_OK;   // (before the pointers: those of empty tensors may be NULL)
  if (!k || !v || !slots || !cache || (q && (!q_out || d->q_heads < 1))) return IFQ_EINVAL;
  if (d->rope != IFQ_ROPE_NONE && (!cos || !sin || !positions)) return IFQ_EINVAL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q ? q_out : nullptr) || !aligned16(cache) ||
      !aligned(slots, 8) || !aligned(cos, 4) || !aligned(sin, 4) || !aligned(positions, 4))
    return IFQ_EALIGN;
  a.cache = cache_args(d->cache, cache);
  a.q = (const uint16_t*)q;
  a.k = (const uint16_t*)k;
  a.v = (const uint16_t*)v;
  a.q_out = (uint16_t*)q_out;
  a.cos = cos;
  a.sin = sin;
  a.pos = positions;
  a.slots = slots;
  a.tokens = d->tokens;
  a.q_heads = q ? d->q_heads : 0;
  a.rope = d->rope;
  a.rot = d->rot_dim;
  a.positions = d->positions;
  a.vec = aligned16(cos) && aligned16(sin);
  const int HB = kv4_warp_heads(D);
  const dim3 grid(ceil_div(d->tokens, kAppendWarps), ceil_div(a.q_heads, HB) + 2 * ceil_div(d->cache.kv_heads, HB));
  if (grid.y > 65535) return IFQ_ERANGE;
  return by_head(D, d->dtype, [&](auto dim, auto bf) {
    return done(launch_k(kv4_append_kernel<decltype(dim)::value, decltype(bf)::value>, grid, dim3(32 * kAppendWarps), 0,
                         S(stream), a));
  });
}

int ifq_kv4_read(const ifq_kv4_append_desc* d, const void* cache, const int64_t* slots, void* k_out, void* v_out,
                 void* stream) {
  if (!d) return IFQ_EINVAL;
  size_t bytes;
  int rc = check_cache(&d->cache, &bytes);
  if (rc) return rc;
  if (d->tokens < 0 || !is16(d->dtype)) return IFQ_EINVAL;
  if (d->tokens > kMaxSize) return IFQ_ERANGE;
  if (!d->tokens) return IFQ_OK;
  if (!cache || !slots) return IFQ_EINVAL;
  if (!aligned16(cache) || !aligned16(k_out) || !aligned16(v_out) || !aligned(slots, 8)) return IFQ_EALIGN;
  if (!k_out && !v_out) return IFQ_OK;
  const dim3 grid(ceil_div(d->tokens, kAppendWarps), 2 * ceil_div(d->cache.kv_heads, kv4_warp_heads(d->cache.head_dim)));
  if (grid.y > 65535) return IFQ_ERANGE;
  KvReadArgs a;
  a.cache = cache_args(d->cache, cache);
  a.slots = slots;
  a.k_out = (uint16_t*)k_out;
  a.v_out = (uint16_t*)v_out;
  a.tokens = d->tokens;
  return by_head(d->cache.head_dim, d->dtype, [&](auto dim, auto bf) {
    return done(launch_k(kv4_read_kernel<decltype(dim)::value, decltype(bf)::value>, grid, dim3(32 * kAppendWarps), 0,
                         S(stream), a));
  });
}

int ifq_kv4_attention_workspace_bytes(const ifq_kv4_attention_desc* d, size_t* bytes) {
  if (!bytes) return IFQ_EINVAL;
  KvAttnArgs a = {};
  AttnPlan p;
  int rc = check_attention(d, &a);
  if (rc || (rc = plan_attention(d, a, &p))) return rc;
  *bytes = p.ws;
  return IFQ_OK;
}

int ifq_kv4_attention(const ifq_kv4_attention_desc* d, const void* q, const void* cache, const int32_t* page_table,
                      const int32_t* lens, const int32_t* q_starts, void* out, float* lse, void* ws, size_t ws_bytes,
                      void* stream) {
  KvAttnArgs a = {};
  AttnPlan p;
  int rc = check_attention(d, &a);
  if (rc) return rc;
  const bool some = d->q_tokens && d->seqs;
  if (some && (!q || !cache || !lens || !out || (!page_table && d->max_pages > 0))) return IFQ_EINVAL;
  if (!q_starts && (d->q_tokens != d->seqs)) return IFQ_ESHAPE;
  if (!some) return IFQ_OK;
  if (!aligned16(q) || !aligned16(cache) || !aligned16(out) || !aligned(page_table, 4) || !aligned(lens, 4) ||
      !aligned(q_starts, 4) || !aligned(lse, 4) || !aligned16(ws))
    return IFQ_EALIGN;
  if ((rc = plan_attention(d, a, &p))) return rc;
  if (p.ws && (!ws || ws_bytes < p.ws)) return IFQ_EWORKSPACE;
  a.q = (const uint16_t*)q;
  a.cache = (const uint8_t*)cache;
  a.table = page_table;
  a.lens = lens;
  a.starts = q_starts;
  a.out = (uint16_t*)out;
  a.lse = lse;
  return by_head(d->cache.head_dim, d->dtype, [&](auto dim, auto bf) {
    constexpr int D = decltype(dim)::value;
    constexpr bool BF = decltype(bf)::value;
    if constexpr (D < 256)
      if (p.chunk == 2) return run_chunk<D, BF, 2>(a, p, ws, S(stream));
    if (p.chunk) return run_chunk<D, BF, 1>(a, p, ws, S(stream));
    if constexpr (D < 256)
      if (p.nt == 2) return run_rows<D, BF, 2>(a, p, ws, S(stream));
    return run_rows<D, BF, 1>(a, p, ws, S(stream));
  });
}

static int check_fp8(const ifq_fp8_desc* d) {
  if (!d) return IFQ_EINVAL;
  if (d->m < 0 || d->n < 1 || d->k < 1) return IFQ_EINVAL;
  if (d->k % 16 != 0) return IFQ_ESHAPE;
  if (d->m > kMaxSize || d->n > kMaxSize || d->k > kMaxSize) return IFQ_ERANGE;
  return IFQ_OK;
}

int ifq_fp8_quantize(const ifq_fp8_desc* d, const void* x, void* codes, float* scales, void* stream) {
  int rc = check_fp8(d);
  if (rc) return rc;
  Fp8QuantArgs a;
  if (!is16(d->dtype)) return IFQ_EINVAL;
  if ((rc = stride_of(d->x_stride, d->k, &a.x_stride))) return rc;
  if (!d->m) return IFQ_OK;
  if (!x || !codes || !scales) return IFQ_EINVAL;
  if (!aligned16(x) || !aligned16(codes) || !aligned(scales, 4)) return IFQ_EALIGN;
  a.x = (const uint16_t*)x;
  a.codes = (uint8_t*)codes;
  a.scales = scales;
  a.m = d->m;
  a.k = d->k;
  a.kb = ceil_div(d->k, kFp8Block);
  const dim3 grid(ceil_div(a.m, kFp8QuantWarps), ceil_div(a.kb, 2 * kFp8Pass));
  if (grid.y > 65535) return IFQ_ERANGE;
  return done(d->dtype == IFQ_BF16 ? launch_k(fp8_quantize_kernel<true>, grid, dim3(32 * kFp8QuantWarps), 0, S(stream), a)
                                   : launch_k(fp8_quantize_kernel<false>, grid, dim3(32 * kFp8QuantWarps), 0, S(stream), a));
}

int ifq_fp8_workspace_bytes(const ifq_fp8_desc* d, size_t* bytes) {
  if (!bytes) return IFQ_EINVAL;
  const int rc = check_fp8(d);
  if (rc) return rc;
  *bytes = 0;
  return IFQ_OK;
}

int ifq_fp8_matmul(const ifq_fp8_desc* d, const void* x, const float* x_scale, const void* w, const float* w_scale,
                   void* out, void* ws, size_t ws_bytes, void* stream) {
  const int rc = check_fp8(d);
  if (rc) return rc;
  if (!is16(d->out_dtype) && d->out_dtype != IFQ_F32) return IFQ_EINVAL;
  if (d->out_stride < 0 || (d->out_stride != 0 && d->out_stride < d->n)) return IFQ_EINVAL;
  if (!d->m) return IFQ_OK;
  if (!x || !x_scale || !w || !w_scale || !out) return IFQ_EINVAL;
  if (!aligned16(x) || !aligned16(w) || !aligned16(out) || !aligned16(ws) || !aligned(x_scale, 4) || !aligned(w_scale, 4))
    return IFQ_EALIGN;
  (void)ws_bytes;
  if (!get_encode()) return IFQ_ECUDA;
  const Fp8Operands o = {x, x_scale, w, w_scale, out, S(stream)};
  if (d->m <= 16) return run_fp8<16, true>(d, o);
  if (d->m <= 32) return run_fp8<32, true>(d, o);
  if (d->m <= 64) return run_fp8<64, true>(d, o);
  // wide tiles where they fill the SMs
  if ((long long)ceil_div(d->m, 128) * ceil_div(d->n, 256) >= sm_count()) return run_fp8<256, false>(d, o);
  return run_fp8<128, false>(d, o);
}

}  // extern "C"
