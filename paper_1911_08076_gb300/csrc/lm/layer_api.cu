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
#include "w4_few.cuh"
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
  *bytes = blocks * (size_t)ceil_div(w->k, kW4Cols) * w4_block_bytes(w->group) + kW4Tail;
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

int check_w4_desc(const ifq_w4_desc* d, int gated, W4Args* a, size_t* bytes) {
  if (!d) return IFQ_EINVAL;
  int rc = check_w4(&d->weights, bytes);
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

constexpr int kW4MaxSplit = 8;

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

constexpr int kW4Chain = 8;

// How a product runs: columns of a tile, a pair of CTAs a tile or one, the split of k.
struct W4Plan {
  int cg, bn, ks, halves;
  double cycles;
};

// An estimate of the cycles of `turns` tiles in a row: blocks of k at 650 cycles of expansion and waits (as measured) or 4 a
// column of MMAs, and a tile's start and end.  (With 450 tiles came out too narrow: 1000 x 4096 x 9216 60 us instead of 46,
// gated 448 x 9216 x 4096 53 instead of 44.)
double w4_cycles(double turns, int blocks, int bn) { return turns * (blocks * std::max(650.0, 4.0 * bn) + 1200); }

W4Plan plan_w4_one(const W4Args& a, bool gated, const int* slots) {
  W4Plan best = {1, 16, 1, 0, 1e300};
  const long long tw = ceil_div(a.n, gated ? 64 : 128);
  for (int tx = ceil_div(a.m, 128), n = 0; n < 3; ++n, ++tx) {
    const int bn = (int)round_up(ceil_div(a.m, tx), 16);
    const long long tiles = tw * ceil_div(a.m, bn);
    for (int ks = 1; ks <= kW4MaxSplit && ks <= a.kb; ++ks) {
      if (slots[ks] < 1) continue;
      const double turns = (double)((tiles + slots[ks] - 1) / slots[ks]);
      // (a cluster does one tile and ends)
      const double c = w4_cycles(turns, ceil_div(a.kb, ks), bn) + (ks > 1 ? 2500 + 5000 * (turns - 1) : 0);
      if (c < best.cycles) best = {1, bn, ks, 0, c};
    }
  }
  return best;
}
W4Plan plan_w4_two(const W4Args& a, bool gated, const int* slots) {
  W4Plan best = {2, 0, 1, 0, 1e300};
  if (slots[2] < 1) return best;
  const int most = a.out_type == IFQ_F32 ? 128 : 256;
  const long long tw = ceil_div(a.n, gated ? 128 : 256);
  for (int tx = ceil_div(a.m, most), n = 0; n < 3; ++n, ++tx) {
    const int bn = (int)round_up(ceil_div(a.m, tx), 64);
    const long long tiles = tw * ceil_div(a.m, bn);
    const int rest = (int)(tiles % slots[2]);
    // the tiles of a last turn that fills half of the SMs or less are cut in two
    const int halves = rest && 2 * rest <= slots[2];
    const double c = w4_cycles((double)(tiles / slots[2]), a.kb, bn) + (rest ? w4_cycles(1, a.kb, halves ? bn / 2 : bn) : 0);
    if (c < best.cycles) best = {2, bn, 1, halves, c};
  }
  return best;
}

template <bool BF, int G, bool GATED, int CG>
int run_w4_many(const W4Args& a, const W4Plan& p, const int* slots, cudaStream_t st) {
  const auto kern = w4_many_kernel<BF, G, GATED, CG>;
  W4Many r;
  r.a = a;
  r.bn = p.bn;
  r.ks = p.ks;
  r.tiles_w = ceil_div(a.n, (GATED ? 64 : 128) * CG);
  r.tiles_x = ceil_div(a.m, p.bn);
  const long long tiles = (long long)r.tiles_w * r.tiles_x;
  if (tiles > INT_MAX / (2 * kW4MaxSplit)) return IFQ_ERANGE;
  r.tiles = r.whole = (int)tiles;
  if (p.halves) {
    const int rest = r.tiles % slots[2];
    r.whole -= rest;
    r.tiles += rest;
  }
  const auto wide = [&](const void* q, long long stride) { return aligned16(q) && stride % 8 == 0; };
  r.chain = a.out_type == IFQ_F32 ? kW4Chain : a.kb;
  r.vec = a.n % 8 == 0 && wide(a.out, a.out_stride) && (!a.res || wide(a.res, a.res_stride));
  if (a.out_type == IFQ_F32) r.turn = ceil_div(a.kb, p.ks) > r.chain ? p.bn * 512 : 0;
  else r.turn = CG == 2 ? p.bn * w4_out_pitch(GATED) : 0;
  // shared memory: three blocks of x (two where they do not fit beside two of codes), then codes, then what is left for x
  const int xb = p.bn / CG * 256, cb = 8 * w4_block_bytes(G);
  int room = kW4ManySmem - 1024 - 512 - w4_many_recv(p.bn, p.ks) - r.turn;
  r.stages = 3 * xb + 2 * cb <= room ? 3 : 2;
  room -= r.stages * xb;
  r.slots = w4_code_slots(room / cb);
  room -= r.slots * cb;
  r.stages += std::min(kW4Bars - r.stages, room / xb);
  if (r.slots < 2) return IFQ_EUNSUPPORTED;   // (128 columns in floats over a cluster: two of each)
  CUtensorMap tx;
  if (!encode_x(a, CG == 2 ? p.bn / 4 : p.bn, &tx)) return IFQ_ECUDA;
  const int cluster = CG == 2 ? 2 : p.ks, most = CG == 2 ? slots[2] : p.ks > 1 ? r.tiles : slots[1];
  const dim3 grid((unsigned)(std::min(r.tiles, most) * cluster));
  if (cluster > 1) return done(launch_k_cluster(kern, cluster, grid, dim3(kW4ManyThreads), kW4ManySmem, st, tx, r));
  return done(launch_k(kern, grid, dim3(kW4ManyThreads), kW4ManySmem, st, tx, r));
}

template <bool BF, int G, bool GATED>
int run_w4_tiles(const W4Args& a, cudaStream_t st) {
  static int known[2][kMaxDevices][kW4MaxSplit + 1];
  const int *one, *two;
  int rc;
  if ((rc = w4_many_setup(w4_many_kernel<BF, G, GATED, 1>, known[0], &one))) return rc;
  if ((rc = w4_many_setup(w4_many_kernel<BF, G, GATED, 2>, known[1], &two))) return rc;
  const W4Plan p1 = plan_w4_one(a, GATED, one), p2 = plan_w4_two(a, GATED, two);
  if (a.m > 128 && p2.cycles < p1.cycles) return run_w4_many<BF, G, GATED, 2>(a, p2, two, st);
  return run_w4_many<BF, G, GATED, 1>(a, p1, one, st);
}

constexpr int kW4FewRows = 16;

template <bool BF, int G, bool GATED, int NT>
int run_w4_few(const W4Args& a, cudaStream_t st) {
  const int sms = sm_count(), tiles = ceil_div(a.n, GATED ? 64 : 128);
  const long long room = kW4ManySmem - w4_ring_fixed(a.m, a.kb, NT);
  const int deep = w4_ring_deep((int)(room / (8 * w4_block_bytes(G))), NT);
  // The ring takes whole tiles of 128 rows, a block an SM, so it waits for turns that are full, or nearly, and for more than four rows
  // of x (131072 x 4096, ring against none: 1 row 61.6 against 60.2 us, 4 rows 61.4 and 60.6, 8 rows 61.8 and 62.6, 12 rows
  // 71.4 and 75.5; 16 x 131072 x 1024 23.2 and 26.7; 3.4 turns, 12 x 65536 x 6144: 68.6 and 59.1).  Less than two stages a ring
  // is no ring: 8 x 65536 x 10240 118 and 79.
  const int turns = ceil_div(tiles, sms);
  if (a.m > 4 && tiles >= 2 * sms && 10ll * tiles >= 9ll * turns * sms && deep >= 2) {
    static bool set[kMaxDevices];
    const auto kern = w4_ring_kernel<BF, G, GATED, NT>;
    const int rc = allow_smem(kern, kW4ManySmem, set);
    if (rc) return rc;
    const W4Ring r = {a, tiles, deep};
    const size_t smem = (size_t)w4_ring_fixed(a.m, a.kb, NT) + (size_t)deep * w4_ring_wk(NT) * 8 * w4_block_bytes(G);
    return done(launch_k(kern, dim3((unsigned)std::min(tiles, sms)), dim3(32 * (8 * w4_ring_wk(NT) + 1)), smem, st, r));
  }
  static bool set[kMaxDevices];
  const auto kern = w4_few_kernel<BF, G, GATED, NT>;
  const int rc = allow_smem(kern, kW4ManySmem, set);
  if (rc) return rc;
  W4Few r;
  r.a = a;
  r.blocks = ceil_div(a.n, GATED ? 8 : 16);
  // Warps along k: a warp's blocks in a row, and a row block's sums at the cost of one more.
  long long best = LLONG_MAX;
  for (int wk = 1; wk <= kW4FewWarps; wk *= 2) {
    const int wr = kW4FewWarps / wk;
    const long long c = ((r.blocks + (long long)wr * sms - 1) / ((long long)wr * sms)) * (ceil_div(a.kb, wk) + 1);
    if (c < best) best = c, r.wk = wk, r.wr = wr;
  }
  const dim3 grid((unsigned)std::min(ceil_div(r.blocks, r.wr), sms));
  return done(launch_k(kern, grid, dim3(32 * kW4FewWarps), (size_t)w4_few_smem(a.m, a.kb, NT), st, r));
}

int run_w4(const ifq_w4_desc* d, W4Args& a, size_t bytes, const void* x, const void* packed, void* out, const void* res, cudaStream_t st) {
  if (!d->m) return IFQ_OK;
  if (!x || !packed || !out) return IFQ_EINVAL;
  if (!aligned16(x) || !aligned16(packed) || !aligned16(out) || !aligned16(res)) return IFQ_EALIGN;
  a.x = (const uint16_t*)x;
  a.w = (const uint8_t*)packed;
  a.large = (const uint32_t*)(a.w + bytes - kW4Tail);
  a.out = out;
  a.res = res;
  if (!get_encode()) return IFQ_ECUDA;
  return by_weights(d->weights, [&](auto bf, auto group) {
    constexpr bool BF = decltype(bf)::value;
    constexpr int G = decltype(group)::value;
    const auto run = [&](auto pair) {
      constexpr bool GATED = decltype(pair)::value;
      // Few rows, whose x fits shared memory.  (16 against 17 rows, the first of the tiles: 4096 x 4096 7.4 and 9.5 us,
      // 6144 x 4096 10.3 and 12.0, gated 9216 x 4096 15.7 and 15.4; four tiles of 8 rows would take 20 there.  On either side of
      // what fits, 4096 rows of w: 16 rows of x with k = 6144 10.9 us, with 6272 10.8; 8 rows with 13312 14.6, with 13568 15.8; 3 rows
      // with 32768 24.2, with 36864 31.8.)
      if (a.m <= 8 && w4_few_smem(a.m, a.kb, 1) <= kW4ManySmem) return run_w4_few<BF, G, GATED, 1>(a, st);
      if (a.m <= kW4FewRows && w4_few_smem(a.m, a.kb, 2) <= kW4ManySmem) return run_w4_few<BF, G, GATED, 2>(a, st);
      return run_w4_tiles<BF, G, GATED>(a, st);
    };
    return d->weights.gated ? run(std::true_type()) : run(std::false_type());
  });
}

// ---------------------------------------------------------------- rows

template <bool BF>
int run_norm(NormArgs& a, cudaStream_t st) {
  const int vecs = a.dim / 8;
  // Few rows: as many threads as there are, so that one load is waited for; many: four times 16 bytes a thread, and many
  // small blocks an SM (8191 x 4096 in 40 us, 98 % of a copy; eight times 16 bytes where a row is longer).
  const int v = vecs > 2048 ? 8 : a.rows >= 2 * sm_count() ? 4 : vecs > 1024 ? 2 : 1;
  a.threads = (int)round_up(ceil_div(vecs, v), 32);
  const int rows = a.threads == 32 ? 8 : 1;   // a block
  const dim3 grid(ceil_div(a.rows, rows)), block(a.threads * rows);
  switch (v) {
    case 1: return done(launch_k(rms_norm_kernel<BF, 1, 1024>, grid, block, 0, st, a));
    case 2: return done(launch_k(rms_norm_kernel<BF, 2, 1024>, grid, block, 0, st, a));
    case 4: return done(launch_k(rms_norm_kernel<BF, 4, 512>, grid, block, 0, st, a));
    default:
      if (a.threads <= 512) return done(launch_k(rms_norm_kernel<BF, 8, 512>, grid, block, 0, st, a));
      return done(launch_k(rms_norm_kernel<BF, 8, 1024>, grid, block, 0, st, a));
  }
}

template <int TYPE>
int run_scores(ScoresArgs& a, cudaStream_t st) {
  // Threads: four loads each, in earnest sizes 512.  A row is split where rows are few, while a thread has a load.
  const long long pieces = (long long)a.vocab * (TYPE == IFQ_F32 ? 4 : 2) / 16 + 2;
  int threads = 64;
  while (threads < kScoreThreads && threads * 4 < pieces) threads *= 2;
  // The part of a row that the fullest SM reads, and a little for each block whose results are joined.
  int parts = 1;
  double best = 1e300;
  for (int n = 1; n <= kScoreParts && (n == 1 || ((long long)a.rows * n <= 2 * sm_count() && pieces >= n * threads)); ++n) {
    const double c = (double)(((long long)a.rows * n + sm_count() - 1) / sm_count()) / n + 0.01 * n;
    if (c < best) best = c, parts = n;
  }
  if ((long long)a.rows * parts > INT_MAX) return IFQ_ERANGE;
  a.parts = parts;
  const dim3 grid(a.rows * parts), block(threads);
  if (parts > 1) return done(launch_k_cluster(token_scores_kernel<TYPE, 2>, parts, grid, block, 0, st, a));
  if (a.rows <= 2 * sm_count()) return done(launch_k(token_scores_kernel<TYPE, 2>, grid, block, 0, st, a));
  return done(launch_k(token_scores_kernel<TYPE, 3>, grid, block, 0, st, a));
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
  const size_t blocks = (bytes - kW4Tail) / w4_block_bytes(w->group);
  a.row_blocks = (int)(blocks / a.kb);
  a.large = (uint32_t*)(a.out + bytes - kW4Tail);
  if (cudaMemsetAsync(a.large, 0, kW4Tail, S(stream)) != cudaSuccess) return IFQ_ECUDA;
  const long long count = (long long)w->n * (w->gated ? 2 : 1) * a.groups;
  const dim3 scan((unsigned)std::min<long long>((count + 2047) / 2048, 4 * sm_count()));
  const cudaError_t e = w->dtype == IFQ_BF16 ? launch_k(w4_scan_kernel<true>, scan, dim3(256), 0, S(stream), a)
                                             : launch_k(w4_scan_kernel<false>, scan, dim3(256), 0, S(stream), a);
  if (e != cudaSuccess) return IFQ_ECUDA;
  const dim3 grid((unsigned)std::min<size_t>((blocks + kW4PackWarps - 1) / kW4PackWarps, 16 * 1024));
  return by_weights(*w, [&](auto bf, auto group) {
    return done(launch_k(w4_pack_kernel<decltype(bf)::value, decltype(group)::value>, grid, dim3(32 * kW4PackWarps), 0, S(stream), a));
  });
}

int ifq_w4_matmul(const ifq_w4_desc* d, const void* x, const void* packed, void* out, const void* residual,
                  void* stream) {
  W4Args a = {};
  size_t bytes;
  int rc = check_w4_desc(d, 0, &a, &bytes);
  if (rc) return rc;
  if (residual && (rc = any_stride(d->residual_stride, d->weights.n, &a.res_stride))) return rc;
  if (residual && residual == out && a.res_stride != a.out_stride) return IFQ_EINVAL;
  return run_w4(d, a, bytes, x, packed, out, residual, S(stream));
}

int ifq_w4_gated(const ifq_w4_desc* d, const void* x, const void* packed, void* out, void* stream) {
  W4Args a = {};
  size_t bytes;
  const int rc = check_w4_desc(d, 1, &a, &bytes);
  if (rc) return rc;
  return run_w4(d, a, bytes, x, packed, out, nullptr, S(stream));
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
  if (d->rows > kMaxSize || d->vocab > kMaxSize || d->scale > 0x1p100f) return IFQ_ERANGE;
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
  a.c = (float)(d->scale * 2.8853900817779268);
  switch (d->dtype) {
    case IFQ_F16: return run_scores<IFQ_F16>(a, S(stream));
    case IFQ_BF16: return run_scores<IFQ_BF16>(a, S(stream));
    default: return run_scores<IFQ_F32>(a, S(stream));
  }
}

}  // extern "C"
