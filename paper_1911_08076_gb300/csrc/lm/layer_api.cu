// C ABI entry points of the rest of a quantised decoder layer and of its answers: products with weights in 4 bits,
// the norm between the blocks, scores of tokens.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ifq.h"
#include "lm_api.h"
#include "lm_host.h"
#include "norm.cuh"
#include "scores.cuh"
#include "w4.cuh"
#include "w4_many.cuh"

namespace {

using namespace ifq;

// ---------------------------------------------------------------- products with weights in 4 bits

int check_w4(const ifq_w4_weights* w, size_t* bytes) {
  if (w->n < 1 || w->k < 1 || !is16(w->dtype) || (w->gated != 0 && w->gated != 1)) return IFQ_EINVAL;
  if (w->group != 32 && w->group != 64 && w->group != 128) return IFQ_EUNSUPPORTED;
  if (w->k % 8 != 0) return IFQ_ESHAPE;
  if (w->n > (w->gated ? kMaxSize / 2 : kMaxSize) || w->k > kMaxSize) return IFQ_ERANGE;
  const size_t rows = (size_t)w->n * (w->gated ? 2 : 1);
  // (a gated pair's blocks hold 8 rows of each matrix)
  const size_t blocks = round_up(w->gated ? (size_t)(w->n + 7) / 8 : (rows + 15) / 16, 8);
  *bytes = blocks * (size_t)ceil_div(w->k, kW4Cols) * w4_block_bytes(w->group);
  return IFQ_OK;
}

// The instance of a type and group: f(bfloat16, group) with both as types.
template <typename F>
int by_weights(const ifq_w4_weights& w, F&& f) {
  const auto grouped = [&](auto bf) {
    switch (w.group) {
      case 32: return f(bf, std::integral_constant<int, 32>());
      case 64: return f(bf, std::integral_constant<int, 64>());
      default: return f(bf, std::integral_constant<int, 128>());
    }
  };
  return w.dtype == IFQ_BF16 ? grouped(std::true_type()) : grouped(std::false_type());
}

// A row stride of any number of elements (0: dense).
int any_stride(int64_t given, long long width, long long* out) {
  if (given < 0 || (given != 0 && given < width)) return IFQ_EINVAL;
  *out = given ? given : width;
  return IFQ_OK;
}

int check_w4_desc(const ifq_w4_desc* d, int gated, W4Args* a) {
  if (!d) return IFQ_EINVAL;
  size_t bytes;
  int rc = check_w4(&d->weights, &bytes);
  if (rc) return rc;
  const ifq_w4_weights& w = d->weights;
  if (w.gated != gated || d->m < 0 || (!is16(d->out_dtype) && d->out_dtype != IFQ_F32)) return IFQ_EINVAL;
  if (gated && (d->out_dtype != w.dtype || d->act < IFQ_ACT_SILU || d->act > IFQ_ACT_GELU_TANH)) return IFQ_EINVAL;
  if (d->m > kMaxSize) return IFQ_ERANGE;
  if ((rc = stride_of(d->x_stride, w.k, &a->x_stride))) return rc;
  if ((rc = any_stride(d->out_stride, w.n, &a->out_stride))) return rc;
  a->m = d->m;
  a->n = w.n;
  a->k = w.k;
  a->kb = ceil_div(w.k, kW4Cols);
  a->out_type = d->out_dtype;
  a->act = gated ? d->act : 0;
  return IFQ_OK;
}

// TMA descriptor of x: [m][k] 16-bit values, boxes of `box` rows x 64 in the 128-byte swizzle; what is past the ends reads
// as zeros.
bool encode_x(const W4Args& a, int box, CUtensorMap* tm) {
  const cuuint64_t gdim[2] = {(cuuint64_t)a.k, (cuuint64_t)a.m}, gstride[1] = {(cuuint64_t)a.x_stride * 2};
  const cuuint32_t bdim[2] = {64, (cuuint32_t)box}, estr[2] = {1, 1};
  return g_encode(tm, CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<uint16_t*>(a.x), gdim, gstride, bdim, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr int kW4MaxSplit = 8, kW4SplitCols = 128;

// One-time setup of an instance on the current device: its shared memory, and how many clusters of each size run at once
// (in `slots`; a plain launch is size 1).
template <typename K>
int w4_many_setup(K kern, int (&known)[kMaxDevices][kW4MaxSplit + 1], const int** slots) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return IFQ_ECUDA;
  const int sms = sm_count();
  std::lock_guard<std::mutex> lk(g_lm_mu);
  int* s = known[dev];
  if (!s[1]) {
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kW4ManySmem) != cudaSuccess) return IFQ_ECUDA;
    for (int ks = 2; ks <= kW4MaxSplit; ++ks) {
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3((unsigned)(sms / ks * ks));
      cfg.blockDim = dim3(kW4ManyThreads);
      cfg.dynamicSmemBytes = kW4ManySmem;
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

template <bool BF, int G, bool GATED>
int run_w4_many(const W4Args& a, cudaStream_t st) {
  static int known[kMaxDevices][kW4MaxSplit + 1];
  const auto kern = w4_many_kernel<BF, G, GATED>;
  const int* slots;
  const int rc = w4_many_setup(kern, known, &slots);
  if (rc) return rc;
  W4Many r;
  r.a = a;
  r.tiles_w = ceil_div(a.n, GATED ? 64 : 128);
  // The columns of a tile and the split of k with the least time: blocks of k in a row, each 256 cycles of expansion or
  // 4 a column of MMAs, and what a tile and a cluster's join cost besides.
  double best = 1e300;
  for (int tx = ceil_div(a.m, kW4MaxCols), n = 0; n < 3; ++n, ++tx) {
    const int bn = (int)round_up(ceil_div(a.m, tx), 16);
    const long long tiles = (long long)r.tiles_w * ceil_div(a.m, bn);
    if (tiles > INT_MAX / kW4MaxSplit) return IFQ_ERANGE;
    const double block = std::max(350.0, 4.0 * bn);
    for (int ks = 1; ks <= kW4MaxSplit && ks <= a.kb; ++ks) {
      if (slots[ks] < 1 || (ks > 1 && bn > kW4SplitCols)) continue;
      const double turns = (double)((tiles + slots[ks] - 1) / slots[ks]);
      const double c = turns * (ceil_div(a.kb, ks) * block + 1500 + 4 * bn) + (ks > 1 ? 2500 : 0);
      if (c < best) best = c, r.bn = bn, r.ks = ks, r.tiles = (int)tiles;
    }
  }
  r.tiles_x = ceil_div(a.m, r.bn);
  r.stages = w4_many_stages(G, r.bn, r.ks);
  CUtensorMap tx;
  if (!encode_x(a, r.bn, &tx)) return IFQ_ECUDA;
  if (r.ks > 1)
    return done(launch_k_cluster(kern, r.ks, dim3((unsigned)(r.tiles * r.ks)), dim3(kW4ManyThreads), kW4ManySmem, st, tx, r));
  return done(launch_k(kern, dim3((unsigned)std::min(r.tiles, slots[1])), dim3(kW4ManyThreads), kW4ManySmem, st, tx, r));
}

int run_w4(const ifq_w4_desc* d, W4Args& a, const void* x, const void* packed, void* out, const void* res, cudaStream_t st) {
  if (!d->m) return IFQ_OK;
  if (!x || !packed || !out) return IFQ_EINVAL;
  if (!aligned16(x) || !aligned16(packed) || !aligned16(out) || !aligned16(res)) return IFQ_EALIGN;
  a.x = (const uint16_t*)x;
  a.w = (const uint8_t*)packed;
  a.out = out;
  a.res = res;
  if (!get_encode()) return IFQ_ECUDA;
  return by_weights(d->weights, [&](auto bf, auto group) {
    constexpr bool BF = decltype(bf)::value;
    constexpr int G = decltype(group)::value;
    return d->weights.gated ? run_w4_many<BF, G, true>(a, st) : run_w4_many<BF, G, false>(a, st);
  });
}

// ---------------------------------------------------------------- rows

template <bool BF>
int run_norm(const NormArgs& a, cudaStream_t st) {
  const int vecs = a.dim / 8;
  // few rows: as many threads as there are; many: four times 16 bytes a thread, so that blocks are small
  const int v = vecs > 4096 ? 8 : a.rows >= 2 * sm_count() || vecs > 2048 ? 4 : vecs > 1024 ? 2 : 1;
  const dim3 grid(a.rows), block(round_up(ceil_div(vecs, v), 32));
  switch (v) {
    case 1: return done(launch_k(rms_norm_kernel<BF, 1>, grid, block, 0, st, a));
    case 2: return done(launch_k(rms_norm_kernel<BF, 2>, grid, block, 0, st, a));
    case 4: return done(launch_k(rms_norm_kernel<BF, 4>, grid, block, 0, st, a));
    default: return done(launch_k(rms_norm_kernel<BF, 8>, grid, block, 0, st, a));
  }
}

template <int TYPE>
int run_scores(const ScoresArgs& a, cudaStream_t st) {
  return done(launch_k(token_scores_kernel<TYPE>, dim3(a.rows), dim3(256), 0, st, a));
}

}  // namespace

namespace ifq {

int layer_take_status(int* status) {
  int v = 0, zero = 0;
  if (cudaMemcpyFromSymbol(&v, g_status, sizeof(int)) != cudaSuccess) return IFQ_ECUDA;
  if (v != 0 && cudaMemcpyToSymbol(g_status, &zero, sizeof(int)) != cudaSuccess) return IFQ_ECUDA;
  *status = v;
  return IFQ_OK;
}

}  // namespace ifq

extern "C" {

int ifq_w4_bytes(const ifq_w4_weights* w, size_t* bytes) {
  if (!w || !bytes) return IFQ_EINVAL;
  return check_w4(w, bytes);
}

int ifq_w4_pack(const ifq_w4_weights* w, const void* codes, const void* scales, const void* mins, void* packed,
                void* stream) {
  if (!w) return IFQ_EINVAL;
  size_t bytes;
  const int rc = check_w4(w, &bytes);
  if (rc) return rc;
  if (!codes || !scales || !mins || !packed) return IFQ_EINVAL;
  if (!aligned(codes, 4) || !aligned(scales, 2) || !aligned(mins, 2) || !aligned16(packed)) return IFQ_EALIGN;
  W4PackArgs a;
  a.codes = (const uint8_t*)codes;
  a.scales = (const uint16_t*)scales;
  a.mins = (const uint16_t*)mins;
  a.out = (uint8_t*)packed;
  a.n = w->n;
  a.k = w->k;
  a.kb = ceil_div(w->k, kW4Cols);
  a.groups = ceil_div(w->k, w->group);
  a.gated = w->gated;
  const size_t blocks = bytes / w4_block_bytes(w->group);
  a.row_blocks = (int)(blocks / a.kb);
  const dim3 grid((unsigned)std::min<size_t>((blocks + kW4PackWarps - 1) / kW4PackWarps, 16 * 1024));
  return by_weights(*w, [&](auto, auto group) {
    return done(launch_k(w4_pack_kernel<decltype(group)::value>, grid, dim3(32 * kW4PackWarps), 0, S(stream), a));
  });
}

int ifq_w4_matmul(const ifq_w4_desc* d, const void* x, const void* packed, void* out, const void* residual,
                  void* stream) {
  W4Args a = {};
  int rc = check_w4_desc(d, 0, &a);
  if (rc) return rc;
  if (residual && (rc = any_stride(d->residual_stride, d->weights.n, &a.res_stride))) return rc;
  if (residual && residual == out && a.res_stride != a.out_stride) return IFQ_EINVAL;
  return run_w4(d, a, x, packed, out, residual, S(stream));
}

int ifq_w4_gated(const ifq_w4_desc* d, const void* x, const void* packed, void* out, void* stream) {
  W4Args a = {};
  const int rc = check_w4_desc(d, 1, &a);
  if (rc) return rc;
  return run_w4(d, a, x, packed, out, nullptr, S(stream));
}

int ifq_rms_norm(const ifq_norm_desc* d, const void* x, const void* residual, const void* weight, void* sum, void* out,
                 void* stream) {
  if (!d || d->rows < 0 || d->dim < 1 || !is16(d->dtype) || !std::isfinite(d->eps) || d->eps < 0.0f) return IFQ_EINVAL;
  if (d->dim % 8 != 0) return IFQ_ESHAPE;
  if (d->dim > 65536) return IFQ_EUNSUPPORTED;
  if (d->rows > kMaxSize) return IFQ_ERANGE;
  NormArgs a = {};
  int rc;
  if ((rc = stride_of(d->x_stride, d->dim, &a.x_stride))) return rc;
  if ((rc = stride_of(d->out_stride, d->dim, &a.out_stride))) return rc;
  if (residual && (rc = stride_of(d->residual_stride, d->dim, &a.res_stride))) return rc;
  if (sum && (rc = stride_of(d->sum_stride, d->dim, &a.sum_stride))) return rc;
  if (!d->rows) return IFQ_OK;
  if (!x || !weight || !out || (sum && (!residual || sum == out))) return IFQ_EINVAL;
  if ((out == x && a.out_stride != a.x_stride) || (residual && out == residual && a.out_stride != a.res_stride) ||
      (sum && ((sum == x && a.sum_stride != a.x_stride) || (sum == residual && a.sum_stride != a.res_stride))))
    return IFQ_EINVAL;
  if (!aligned16(x) || !aligned16(residual) || !aligned16(weight) || !aligned16(sum) || !aligned16(out)) return IFQ_EALIGN;
  a.x = (const uint16_t*)x;
  a.res = (const uint16_t*)residual;
  a.weight = (const uint16_t*)weight;
  a.sum = (uint16_t*)sum;
  a.out = (uint16_t*)out;
  a.rows = d->rows;
  a.dim = d->dim;
  a.eps = d->eps;
  return d->dtype == IFQ_BF16 ? run_norm<true>(a, S(stream)) : run_norm<false>(a, S(stream));
}

int ifq_token_scores(const ifq_scores_desc* d, const void* logits, const int64_t* tokens, float* logprobs, float* lse,
                     float* entropy, int64_t* top_ids, float* top_logprobs, void* stream) {
  if (!d || d->rows < 0 || d->vocab < 1 || (!is16(d->dtype) && d->dtype != IFQ_F32) || d->top < 0 ||
      !std::isfinite(d->scale) || d->scale <= 0.0f)
    return IFQ_EINVAL;
  if (d->top > kTopMax) return IFQ_EUNSUPPORTED;
  if (d->top > d->vocab) return IFQ_ESHAPE;
  if (d->rows > kMaxSize || d->vocab > kMaxSize) return IFQ_ERANGE;
  ScoresArgs a = {};
  const int rc = any_stride(d->stride, d->vocab, &a.stride);
  if (rc) return rc;
  if (!d->rows) return IFQ_OK;
  if (!logits || (logprobs && !tokens)) return IFQ_EINVAL;
  if (!aligned(logits, d->dtype == IFQ_F32 ? 4 : 2) || !aligned(tokens, 8) || !aligned(logprobs, 4) || !aligned(lse, 4) ||
      !aligned(entropy, 4) || !aligned(top_ids, 8) || !aligned(top_logprobs, 4))
    return IFQ_EALIGN;
  a.logits = logits;
  a.tokens = tokens;
  a.logprobs = logprobs;
  a.lse = lse;
  a.entropy = entropy;
  a.top_ids = top_ids;
  a.top_logprobs = top_logprobs;
  a.rows = d->rows;
  a.vocab = d->vocab;
  a.top = top_ids || top_logprobs ? d->top : 0;
  a.scale = d->scale;
  switch (d->dtype) {
    case IFQ_F16: return run_scores<IFQ_F16>(a, S(stream));
    case IFQ_BF16: return run_scores<IFQ_BF16>(a, S(stream));
    default: return run_scores<IFQ_F32>(a, S(stream));
  }
}

}  // extern "C"
