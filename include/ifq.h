/*
 * ifq.h -- C ABI of the GB300 library for the quantized substructure of
 * IFQ-Net (Gao et al., "IFQ-Net: Integrated Fixed-point Quantization Networks
 * for Embedded Vision", arXiv:1911.08076).
 *
 * The library computes, on one GPU, the quantized convolution of Eq. (1) with
 * +-1 filters W_b and unsigned k-bit input codes X_q (k = 2, 3 or 4), and
 * applies the integrated fixed-point conversion of Sec. 3.2 as its epilogue:
 * the integer accumulator W_b (x) X_q is compared with per-channel integer
 * thresholds (Eq. (7) after the floor; Eq. (8) for k bits), which emits the
 * next layer's k-bit codes.
 *
 * Conventions shared by every call:
 *   - Return value: an ifq_status.  Argument, shape, alignment and range
 *     errors are returned synchronously, before anything is launched.
 *   - Pointers marked (device) are CUDA device pointers; (host) are host
 *     pointers.  The caller owns every buffer; nothing is retained after the
 *     call returns, and the library allocates no device memory in any call
 *     named here except ifq_graph_create (which owns the captured graph).
 *   - `stream` is a cudaStream_t passed as void* (NULL = legacy default
 *     stream).  Device work is enqueued on it and the call returns without
 *     waiting, except where stated.
 *   - Device-side failures (a bounded wait that ran out, a failed bounds
 *     check) never trap: they set a device status word that
 *     ifq_device_status reads.
 *   - A batch of n = 0 images is valid everywhere: arguments are checked as
 *     usual and nothing is launched.
 *
 * Data formats:
 *   - Codes: NHWC, packed along C in fields of f bits: f = 2 for k = 2 (four
 *     codes per byte), f = 4 for k = 3 and k = 4 (two codes per byte, a 3-bit
 *     code in the low bits of its field).  Channel c of a pixel is bits
 *     f*(c%(8/f)) .. f*(c%(8/f))+f-1 of byte c/(8/f) of that pixel.  C must be
 *     a multiple of 4, so a pixel is C*f/8 bytes.  Buffers are at least
 *     16-byte aligned (cudaMalloc / torch allocations are).
 *   - Filter signs: one row per output channel over K = kh*kw*cin in
 *     (dy, dx, c) order (c fastest); bit k%32 of 32-bit word k/32 is 1 for +1
 *     and 0 for -1; a row is ceil(K/32) words.
 *   - Thresholds: int32 [cout][2^k - 1], ascending (not necessarily strictly),
 *     and int8 sign [cout] in {+1, -1}; the code of accumulator A in channel n
 *     is the number of i with sign[n]*A > T[n][i].
 *   - Accumulators: int32 NHWC [n][ho][wo][cout].
 *   - Convolution geometry: cross-correlation, symmetric zero padding `pad`
 *     (a padded cell is code 0), ho = (h + 2*pad - kh)/stride + 1.
 *   - Pooling geometry: k x k windows starting at (oy*stride, ox*stride),
 *     `pad` extra empty cells at the bottom and right that are skipped,
 *     ho = (h + pad - k)/stride + 1.
 */
#ifndef IFQ_H
#define IFQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  IFQ_OK = 0,
  IFQ_EINVAL = 1,        /* null pointer or invalid parameter value */
  IFQ_ESHAPE = 2,        /* inconsistent or unsupported shape */
  IFQ_EALIGN = 3,        /* pointer not aligned as required */
  IFQ_ERANGE = 4,        /* a size exceeds what the library supports */
  IFQ_ECUDA = 5,         /* a CUDA runtime call failed */
  IFQ_ETIMEOUT = 6,      /* (device status) a bounded wait in a kernel ran out */
  IFQ_EUNSUPPORTED = 7,  /* valid request that the library does not implement */
  IFQ_EWORKSPACE = 8     /* workspace missing or too small */
} ifq_status;

/* Output selection of a convolution. */
enum { IFQ_OUT_CODES = 1, IFQ_OUT_ACC = 2, IFQ_OUT_BOTH = 3 };

/* Kernel path of a convolution (ifq_conv_desc.path). */
enum {
  IFQ_PATH_AUTO = 0,
  IFQ_PATH_TC = 1,
  IFQ_PATH_BITSERIAL = 2,
  IFQ_PATH_DIRECT = 3,
  IFQ_PATH_WIN = 4,
  IFQ_PATH_WARP = 5
};

/* Layer kinds of ifq_forward. */
enum { IFQ_LAYER_CONV = 1, IFQ_LAYER_POOL = 2, IFQ_LAYER_FIXED = 3 };

/* Text for a status code (static storage; never NULL). */
const char* ifq_status_str(int status);

/* Library ABI version: 100*major + minor. */
int ifq_version(void);

/*
 * Environment switches, read on every call that uses them (for experiments; the defaults are the
 * measured best):
 *   IFQ_FORCE_PATH   = 1 / 2 / 3 / 4 / 5: request IFQ_PATH_TC / IFQ_PATH_BITSERIAL / IFQ_PATH_DIRECT /
 *                      IFQ_PATH_WIN / IFQ_PATH_WARP where a descriptor says IFQ_PATH_AUTO
 *                      (ifq_conv_plan reports the result).
 *   IFQ_WIN          = 0: never take the window path (IFQ_PATH_WIN requests take the tensor-core path).
 *   IFQ_WARP         = 0: never take the warp-MMA path (IFQ_PATH_WARP requests take the tensor-core
 *                      path).
 *   IFQ_BAND         = 0: the tensor-core path always runs its im2col kernel; 2 .. 7: its band kernel in
 *                      that launch shape where the layer and the shape fit (by default the faster of
 *                      the two, estimated).  The next three ask for the im2col kernel.
 *   IFQ_TC_BN        = 32 / 64 / 128: the tensor-core kernel's output-channel tile width.
 *   IFQ_TC_KS        = 1 / 2: forbid / force splitting K over clusters of two CTAs (by default only
 *                      layers that would leave more than half of the SMs idle are split).
 *   IFQ_TC_BX        = 1 / 2: the split tensor-core kernel expands its filter tiles in shared memory
 *                      from the sign bits (1 bit per weight read instead of 8) for layers with at most
 *                      two 128-row tiles / wherever it runs (off by default: not faster where measured).
 *   IFQ_PDL          = 0: launch without programmatic dependent launch.
 *   IFQ_GRAPH_BRANCH = 0: capture stacks as one chain, without side branches.
 *   IFQ_STACK        = 1: run qualifying stacks as one persistent launch (ifq_forward).
 * None changes a result; all change only how it is computed.
 */

/*
 * ifq_fold_layer -- integrated fixed-point conversion of one quantized
 * substructure (Sec. 3.2, Eq. (6)-(7), floor of the composed thresholds).
 * Host only, pure, thread-safe; nothing is launched.
 *
 * For output channel n the float substructure is
 *   y = alpha[n]*delta_in*A + bias[n]                        (Eq. (1))
 *   z = gamma[n]*(y - mean[n])/sqrt(var[n] + eps) + beta[n]   (Eq. (2), affine BN)
 *   code = #{ i in 1..L : z > q_base*i + q_offset }           (Eq. (3), L = 2^kbits - 1)
 * and the fold returns T[n][i-1] and sign[n] such that
 *   code = #{ i : sign[n]*A > T[n][i-1] }
 * for every integer A with |A| <= L*K:
 *   tau_i = ((thr_i - beta)*sqrt(var + eps)/gamma + mean - bias)/(alpha*delta_in)
 *   gamma > 0: sign = +1, T = floor(tau_i);  gamma < 0: sign = -1, T = floor(-tau_i)
 *   gamma = 0: sign = +1, T = -L*K-1 if beta > thr_i else L*K
 * T is clamped to [-L*K-1, L*K].  The arithmetic is IEEE double in the order
 * written above.
 *
 * Arguments (host): alpha, gamma, beta, mean, var: [cout] float; bias: [cout]
 * or NULL (zero); thr_out: [cout][L] int32; sign_out: [cout] int8.
 * Requires cout >= 1, K >= 1, 1 <= kbits <= 8, delta_in > 0, q_base > 0,
 * alpha[n] > 0, var[n] + eps > 0, all values finite (else IFQ_EINVAL).
 */
int ifq_fold_layer(int cout, int K, int kbits, const float* alpha, float delta_in, const float* bias,
                   const float* gamma, const float* beta, const float* mean, const float* var, float eps,
                   float q_base, float q_offset, int32_t* thr_out, int8_t* sign_out);

/*
 * ifq_fold_layer_separated -- the same thresholds for the SEPARATED fixed-point
 * conversion of Sec. 2.2 (Fig. 3a), the baseline the paper compares against:
 * with Q = 2^m each float is floored at its own scale, a = floor(alpha*Q),
 * d = floor(delta_in*Q), bq = floor(bias*Q^2), theta = floor(mean*Q),
 * sigma = floor(sqrt(var + eps)/gamma * Q) (the affine BN's divisor),
 * be = floor(beta*Q), t_i = floor(thr_i*Q), and the substructure computes
 *   Y^conv = (a*d*A + bq)/Q^2,  Y^BN = (Y^conv - theta/Q)/(sigma/Q) + be/Q,
 *   code = #{ i : Y^BN > t_i/Q }.
 * That is monotone in A, so it too is code = #{ i : sign*A > T_i }; this
 * returns those exact integer thresholds (64-bit integer arithmetic, no
 * rounding), to run the separated conversion on the same kernels.
 * Same arguments as ifq_fold_layer plus m (1..20); IFQ_EINVAL also when some
 * channel's sigma floors to 0 (no fixed-point divisor).
 */
int ifq_fold_layer_separated(int cout, int K, int kbits, int m, const float* alpha, float delta_in,
                             const float* bias, const float* gamma, const float* beta, const float* mean,
                             const float* var, float eps, float q_base, float q_offset, int32_t* thr_out,
                             int8_t* sign_out);

/*
 * Size in bits/8 (rounded up) of an n x h x w x c map of densely packed
 * kbits-bit codes, 1 <= kbits <= 32 (host, pure): the memory count of the
 * paper's comparison of feature-map sizes.  The library's own buffers use the
 * field format above; ifq_codes_storage_bytes gives their size.
 */
int ifq_codes_bytes(int n, int h, int w, int c, int kbits, size_t* bytes);

/*
 * Bytes of a packed code buffer in the library's format (host, pure):
 * n*h*w*c*f/8 with f = 2 (kbits 0 or 2) or 4 (kbits 3, 4); c % 4 == 0
 * (IFQ_ESHAPE otherwise); other kbits: IFQ_EUNSUPPORTED (negative: IFQ_EINVAL).
 */
int ifq_codes_storage_bytes(int n, int h, int w, int c, int kbits, size_t* bytes);

/*
 * Convolution descriptor.  Input codes NHWC [n][h][w][cin] (cin % 4 == 0),
 * filters [cout][kh][kw][cin], output [n][ho][wo][cout].  out_mode is one of
 * IFQ_OUT_*; codes output needs cout % 4 == 0.  path selects a kernel path
 * (IFQ_PATH_AUTO lets the library choose).  Limits: n >= 0, all other sizes >= 1,
 * K = kh*kw*cin <= 65536, cout <= 65536, n*ho*wo < 2^31.
 * kbits: the code width k of the input codes and of the output codes (0
 * means 2; 2, 3 or 4, else IFQ_EUNSUPPORTED); the thresholds are then
 * [cout][2^k - 1] (Eq. (8)).
 * in_bits: 0 (or kbits) for k-bit input codes; 8 for unsigned 8-bit input
 * values, one byte each (a first layer on image pixels, whose substructure
 * the integrated conversion covers as well: binary filters, integer inputs).
 * An 8-bit input needs cin % 4 == 0 (pad RGB with a zero channel), the
 * tensor-core path and 255*K <= 196608 (IFQ_EUNSUPPORTED otherwise); its
 * layer can only read the stack input in ifq_forward, and its fold takes
 * K_fold = ceil(255*K / (2^k - 1)) so that the clamp covers |A| <= 255*K.
 * pool: 0 or 1 for none; p = 2 or 4 max-pools the convolution output over
 * p x p windows with stride p before the thresholds (Sec. 2.1: the pool acts
 * on Y^conv, before BN and the quantizer), so that the codes are those of the
 * window maximum of A and the output is [n][ho/p][wo/p][cout].  Needs
 * ho % p == 0, wo % p == 0, out_mode IFQ_OUT_CODES and the tensor-core path
 * (IFQ_EUNSUPPORTED otherwise).
 */
typedef struct {
  int n, h, w, cin;
  int cout;
  int kh, kw, stride, pad;
  int out_mode;
  int path;
  int pool;
  int kbits;
  int in_bits;
} ifq_conv_desc;

/* Output spatial size of a conv descriptor (host, pure). */
int ifq_conv_out_shape(const ifq_conv_desc* d, int* ho, int* wo);   /* after the pool, if any */

/*
 * Size of the prepared-filter buffer that ifq_pack_weights fills for `d`
 * (host, pure).  The prepared layout is private to the library and may change
 * with ifq_version.  Layout and size depend on cin, cout, kh, kw and the
 * stored field width (in_bits 8, or 2- or 4-bit fields) alone: filters
 * prepared for one descriptor serve every descriptor that agrees in these,
 * whatever its map, stride, padding, pool, outputs or path.  With more than
 * 32 output channels, kh, kw <= 15 and at most 49 taps (and, in 4-bit fields,
 * cin % 8 == 0 and 7*K <= 196608) codes are served by two tensor-core kernels,
 * and the buffer holds the operands of both: per weight 1 byte and two sign
 * bits, and 1/2 byte (2-bit fields) or 1 byte (4-bit fields) more for the band
 * kernel, also where a layer with these filters runs on another path.
 */
int ifq_weights_prep_bytes(const ifq_conv_desc* d, size_t* bytes);

/*
 * ifq_pack_weights -- expand the filter sign bits of Eq. (1)'s W_b into the
 * library's prepared form (tensor-core operand rows and a sign-bit copy).
 * w_bits (device): [cout][ceil(K/32)] uint32 sign words as in the header;
 * w_prep (device): ifq_weights_prep_bytes bytes, 16-byte aligned.
 * Run once per layer; the result is reused by every ifq_conv2bit call.
 */
int ifq_pack_weights(const ifq_conv_desc* d, const uint32_t* w_bits, void* w_prep, void* stream);

/*
 * The kernel path ifq_conv2bit takes for `d` (host; reads IFQ_FORCE_PATH as
 * ifq_conv2bit does): IFQ_PATH_TC, IFQ_PATH_BITSERIAL, IFQ_PATH_DIRECT,
 * IFQ_PATH_WIN or IFQ_PATH_WARP.  The warp-MMA path (mma.sync tiles of 16 pixels x 8
 * channels, e4m3 or, with 8 channels of codes and a fused pool, f16; accumulators and the
 * fused pool in registers)
 * serves 3 x 3 stride-1 layers with padding 1 on 2-bit codes with cin 8 or 16
 * or on 8-bit values with cin 4, with 2-bit codes or accumulators out,
 * cout 8, 16 or 32, and no pool or a 2 x 2 pool on even sizes; it is the
 * default (where it was measured faster) for such layers on codes with cin 8
 * and for such layers on 8-bit values without a pool, and a request for it
 * elsewhere takes the tensor-core path.  The window path serves stride-1 k x k layers with "same"
 * padding (k odd, <= 7) on 2-bit codes with cin 16 or a multiple of 32, cout
 * 32, 64 or a multiple of 128, no pool or a 2 x 2 pool on even sizes, input
 * rows of whole 16-byte units, output rows of at most 256 pixels, and a
 * filter bank that stays resident in one CTA's shared memory; it is the
 * default for such layers with a fused 2 x 2 pool and cin <= 64 (where it was
 * measured faster), and a request for it elsewhere takes the tensor-core
 * path.  The
 * tensor-core path needs (2^k - 1)*K <= 196608 (the accumulator range checked
 * exact on the fp8 and fp4 tensor cores; 255*K for 8-bit inputs), kh, kw <= 15, and
 * for k = 3, 4 cin % 8 == 0; it runs an im2col kernel or, for unpooled layers on
 * codes with stride 1 or a 1 x 1 filter and more than 32 channels where that is estimated faster,
 * a band kernel; a request for it outside that range takes the
 * bit-serial path.  The direct CUDA-core path serves layers on 8-bit inputs
 * with cout <= 32 and K <= 257 (the default for them; 3 x 3 layers with cin 4, cout <= 16,
 * 2-bit codes out and a fused 2 x 2 pool run on f16 mma.sync instead); a request for it
 * elsewhere takes the tensor-core path.  IFQ_EUNSUPPORTED for a fused pool
 * or an 8-bit input that would land on the bit-serial path.
 */
int ifq_conv_plan(const ifq_conv_desc* d, int* path);

/*
 * The kernel that ifq_conv2bit launches for `d` on the current device (a full
 * GB300's launch shape, without K split, where there is none), as text (host;
 * reads the switches as ifq_conv2bit does): its name, for the tensor-core
 * path's kernels with the channels per tile and then key=value pairs of the
 * launch shape, e.g. "conv_band_kernel<128, 2> subtiles=1 channel_tiles=2
 * resident=1 ctas=152 ...": ctas: the grid; units: accumulators (128 pixels x
 * a channel tile) that a CTA computes at most; cycles: the planner's estimate.
 * For reports and tests; the keys may change with ifq_version.  Writes at most
 * `size` bytes (192 are enough) with the terminating zero.
 */
int ifq_conv_kernel(const ifq_conv_desc* d, char* text, size_t size);

/* Device workspace that ifq_conv2bit needs for `d` (host, pure); may be 0. */
int ifq_conv_workspace_bytes(const ifq_conv_desc* d, size_t* bytes);

/*
 * ifq_conv2bit -- one quantized substructure (Eq. (1) integer core followed
 * by the thresholds of Eq. (7), or of Eq. (8) for k bits; the name keeps the
 * paper's k = 2 case).  For every output pixel and channel n:
 *   A = sum over (dy, dx, c) of w[n][dy][dx][c] * x[b][oy*s+dy-pad][ox*s+dx-pad][c]
 *   y_codes = #{ i : sign[n]*A > thr[n][i] }  (k-bit codes, packed)
 *   y_acc   = A                                (int32), per out_mode
 * x (device): packed codes; w_prep (device): from ifq_pack_weights for the
 * same filters (see ifq_weights_prep_bytes); thr (device): int32 [cout][2^k - 1], ascending per channel;
 * sign (device): int8 [cout];
 * y_codes (device, out_mode & CODES): packed [n][ho][wo][cout*f/8] bytes;
 * y_acc (device, out_mode & ACC): int32 [n][ho][wo][cout];
 * ws (device): ifq_conv_workspace_bytes bytes (may be NULL if that is 0).
 * The results are exact integers; x must not alias the outputs.
 */
int ifq_conv2bit(const ifq_conv_desc* d, const void* x, const void* w_prep, const int32_t* thr,
                 const int8_t* sign, void* y_codes, int32_t* y_acc, void* ws, size_t ws_bytes, void* stream);

/* Pooling descriptor (geometry in the header comment); c % 4 == 0; kbits is the code width as in
 * ifq_conv_desc (0 means 2). */
typedef struct {
  int n, h, w, c;
  int k, stride, pad;
  int kbits;
} ifq_pool_desc;

int ifq_pool_out_shape(const ifq_pool_desc* d, int* ho, int* wo);

/*
 * ifq_maxpool2bit -- max pooling placed between conv and BN (Sec. 2.1),
 * computed on the codes.  With sign (device, int8 [c]) given, channel c takes
 * the max of its codes where sign = +1 and the min where sign = -1; since the
 * composed conv/BN/quantizer map is monotone in the accumulator (increasing
 * for +1, decreasing for -1), this equals quantizing the max of Y^conv.  With
 * sign NULL it is the plain max of the codes (pooling after the quantizer).
 * x, y (device): packed codes of width d->kbits.  Limit: the output's packed
 * bytes n*ho*wo*c*f/8 < 2^31 (IFQ_ERANGE).
 */
int ifq_maxpool2bit(const ifq_pool_desc* d, const void* x, const int8_t* sign, void* y, void* stream);

/*
 * ifq_fold_output_separated -- the separated fixed-point conversion (Sec. 2.2)
 * of a NON-quantized substructure's output (the linear detection conv of a
 * YOLO head; AlexNet's last substructure): with Q = 2^m,
 *   mul[n] = floor(alpha[n]*Q) * floor(delta_in*Q),  add[n] = floor(bias[n]*Q^2)
 * so that Y^conv = (mul*A + add) / Q^2 is Eq. (1) with every float floored at
 * its own scale.  Host, pure.  alpha: [cout] > 0, finite; bias: [cout] or NULL;
 * delta_in > 0; m in 1..24; mul_out, add_out: [cout] int64 (IFQ_EINVAL otherwise).
 */
int ifq_fold_output_separated(int cout, int m, const float* alpha, float delta_in, const float* bias,
                              int64_t* mul_out, int64_t* add_out);

/*
 * ifq_fixed_output -- the fixed-point value of that output at scale Q = 2^m:
 *   y[r][n] = floor((mul[n]*A[r][n] + add[n]) / 2^m)   (exact 64-bit integer
 * arithmetic), saturated to the int32 range, i.e. y/Q is Y^conv with m
 * fractional bits.  acc (device): int32 [rows][cout]; mul, add (device): int64
 * [cout] from ifq_fold_output_separated; y (device): int32 [rows][cout];
 * m in 1..24, rows >= 0, cout >= 1; pointers 8-byte aligned (mul, add) and
 * 4-byte aligned (acc, y).
 */
int ifq_fixed_output(const int32_t* acc, int rows, int cout, const int64_t* mul, const int64_t* add, int m,
                     int32_t* y, void* stream);

/* Fixed-point output layer of ifq_forward (kind IFQ_LAYER_FIXED). */
typedef struct {
  int m;
} ifq_fixed_desc;

/*
 * One layer of a stack for ifq_forward.  src is the index of the layer whose
 * output codes are this layer's input (-1: the stack input x).  For a conv,
 * `conv`, w_prep, thr and sign describe it and y_codes / y_acc receive its
 * outputs per conv.out_mode; for a pool, `pool` describes it, sign is the
 * pooled layer's channel signs (or NULL for a plain max) and y_codes receives
 * the pooled codes.  For a fixed-point output (IFQ_LAYER_FIXED), src is a
 * conv layer that writes int32 accumulators, `fixed`, fx_mul and fx_add
 * describe the conversion (ifq_fixed_output) and y_acc receives the int32
 * fixed-point values [rows][cout] of the source conv's shape.  All pointers
 * are device pointers owned by the caller.
 */
typedef struct {
  int kind;
  int src;
  ifq_conv_desc conv;
  ifq_pool_desc pool;
  const void* w_prep;
  const int32_t* thr;
  const int8_t* sign;
  void* y_codes;
  int32_t* y_acc;
  ifq_fixed_desc fixed;
  const int64_t* fx_mul;
  const int64_t* fx_add;
} ifq_layer;

/*
 * Workspace that lets ifq_forward run `layers` as one persistent launch (host;
 * reads the environment variable IFQ_STACK): 4 bytes per 128-output-row block
 * of every layer, rounded up to 256; 0 when the persistent launch is not
 * selected (IFQ_STACK is not "1") or the stack does not qualify (it then runs
 * one launch per layer and needs no workspace).
 */
int ifq_forward_workspace_bytes(const ifq_layer* layers, int nlayers, size_t* bytes);

/*
 * ifq_forward -- run a layer stack in order on one stream (Sec. 3.1: a
 * quantized network is a chain of substructures; the codes of one are the
 * input of the next, and the output scale of one is the input step of the
 * next).  Shapes are checked along the chain before any launch.
 * x (device): the stack input codes; ws (device): workspace, or NULL.
 * By default one launch per layer in stream order (consecutive launches
 * overlap their prologues through programmatic dependent launch).  With
 * IFQ_STACK=1 in the environment and a workspace of
 * ifq_forward_workspace_bytes bytes, a stack of conv layers that all take the
 * tensor-core path, whose written buffers overlap no other buffer of the
 * stack, runs instead as one cooperative persistent launch: its completion
 * counters (in ws, zeroed on `stream` by every call) let each output tile
 * start as soon as the rows it reads exist.  Calls in flight at the same time
 * must not share a workspace.  Results are identical either way.
 */
int ifq_forward(const ifq_layer* layers, int nlayers, const void* x, void* ws, size_t ws_bytes, void* stream);

/*
 * ifq_forward_noalloc -- ifq_forward for callers that cannot hand the library
 * device scratch: a plain C host that owns no device allocator, or a serving
 * loop that must not call cudaMalloc (which can synchronize the whole device).
 * The paper has no counterpart; this is a deployment convenience.  It
 * allocates nothing.  A stack that qualifies for the persistent launch (see
 * ifq_forward; IFQ_STACK is not consulted) keeps that launch's completion
 * counters in a file-scope device array of 256 KiB: 65536 counters, one per
 * 128-output-row block of every layer.  A stack that needs more counters is
 * rejected with IFQ_EWORKSPACE before anything is launched.  The counters
 * must be zero when the kernel starts: every call zeroes the part it uses, on
 * `stream`, before the launch.  Other stacks run one launch per layer, which
 * needs no scratch.  The first call on each device looks up the array's device
 * address (cudaGetSymbolAddress with that device current, no allocation) and
 * should come before any stream capture.  All calls on one device share the
 * array, so calls whose executions overlap in time (on other streams or from
 * other host threads) race on it and must be serialised by the caller.
 * The looked-up address is kept for the life of the process: after
 * cudaDeviceReset (or anything else that destroys the device's primary
 * context) it is stale, so a process that resets a device must not call this
 * entry point on that device again.  Results are identical to ifq_forward's.
 */
int ifq_forward_noalloc(const ifq_layer* layers, int nlayers, const void* x, void* stream);

/*
 * ifq_last_forward_mode -- how the calling host thread's last successful
 * ifq_forward or ifq_forward_noalloc call ran its stack: IFQ_FORWARD_LAYERS
 * (one launch per layer) or IFQ_FORWARD_PERSISTENT (the whole stack as one
 * persistent launch).  The paper has no counterpart; this is a diagnostic for
 * callers and tests that need to know which launch served a request (results
 * are identical either way).  Host only, thread-local; IFQ_EINVAL if `mode` is
 * NULL or the thread has made no successful forward call.
 */
enum { IFQ_FORWARD_LAYERS = 1, IFQ_FORWARD_PERSISTENT = 2 };
int ifq_last_forward_mode(int* mode);

/*
 * CUDA-graph form of ifq_forward: ifq_graph_create captures the launches of
 * ifq_forward(layers, nlayers, x, ws, ws_bytes) on `stream` into a graph that
 * ifq_graph_launch replays on any stream with the same buffers.  The graph is
 * owned by the returned handle; ifq_graph_destroy frees it.  In the graph a
 * layer whose output no later layer reads (other than the last layer) hangs
 * off its source layer as a side branch joined at the end, so it overlaps the
 * layers after it (IFQ_GRAPH_BRANCH=0 keeps one chain); results are identical.
 */
typedef struct ifq_graph ifq_graph;
int ifq_graph_create(const ifq_layer* layers, int nlayers, const void* x, void* ws, size_t ws_bytes, void* stream,
                     ifq_graph** out);
int ifq_graph_launch(ifq_graph* g, void* stream);
int ifq_graph_destroy(ifq_graph* g);

/*
 * ifq_graph_create_io -- ifq_graph_create whose graph also moves the stack's
 * input in and its results out, so that one ifq_graph_launch serves a request
 * end to end.  The paper has no counterpart; this is a serving convenience.
 *   x_src, x_bytes: when x_src is not NULL, the graph first copies x_bytes from
 *     x_src to x.  x_bytes must equal the bytes of packed input that the layers
 *     with src = -1 read (n * h * w * c * field bits / 8; IFQ_ESHAPE otherwise).
 *   y_codes_dst, y_acc_dst: NULL, or arrays of nlayers destinations.  When entry
 *     i is not NULL, the graph copies layer i's y_codes (y_acc) buffer, all of
 *     it, to that address right after layer i, on layer i's branch of the graph.
 *     The results of a side branch are then copied while the main chain runs.
 *     A destination for a buffer that layer i does not have is IFQ_EINVAL.
 * The addresses are part of the graph: every launch copies from and to the same
 * buffers.  A copy between buffers the device addresses directly (device
 * memory, or pinned host memory under unified addressing), 16-byte aligned and
 * a multiple of 16 bytes, runs on the SMs as in ifq_copy_bytes; any other is a
 * cudaMemcpyAsync node.  Argument errors are returned before anything is
 * captured.
 */
int ifq_graph_create_io(const ifq_layer* layers, int nlayers, const void* x, void* ws, size_t ws_bytes,
                        const void* x_src, size_t x_bytes, void* const* y_codes_dst, void* const* y_acc_dst,
                        void* stream, ifq_graph** out);

/*
 * Codes <-> packed format helpers (device buffers; n % 4 == 0 codes, one code
 * per byte on the unpacked side).  The _kbits forms take the code width
 * (0, 2, 3, 4; a code keeps its low f bits); the plain forms are kbits = 2.
 */
int ifq_pack_codes(const uint8_t* codes, void* packed, size_t n, void* stream);
int ifq_unpack_codes(const void* packed, uint8_t* codes, size_t n, void* stream);
int ifq_pack_codes_kbits(const uint8_t* codes, void* packed, size_t n, int kbits, void* stream);
int ifq_unpack_codes_kbits(const void* packed, uint8_t* codes, size_t n, int kbits, void* stream);
/* +-1 int8 filters [rows][K] (device) -> sign words [rows][ceil(K/32)] (device). */
int ifq_pack_signs(const int8_t* w, uint32_t* bits, int rows, int K, void* stream);

/*
 * ifq_copy_bytes -- copy n bytes on `stream` (either side may be device memory
 * or pinned host memory that the device addresses directly under unified
 * addressing).  With both pointers 16-byte aligned, n % 16 == 0 and both
 * addressable by the device at the same address (device memory, or host memory
 * from cudaHostAlloc / cudaHostRegister), the SMs do the copy with 16-byte loads
 * and stores (on a GB300 over NVLink-C2C for host memory); otherwise it is
 * cudaMemcpyAsync.  For staging a stack's inputs and results.
 */
int ifq_copy_bytes(void* dst, const void* src, size_t n, void* stream);

/*
 * ifq_wait_selftest -- exercise the failure path of the bounded device waits:
 * one warp waits on an mbarrier phase that nothing completes for limit_us
 * microseconds (1..1000000), then records IFQ_ETIMEOUT in the device status
 * word and returns normally, as every kernel's waits do after 2 s.  Read it
 * with ifq_device_status; the context stays usable.
 */
int ifq_wait_selftest(int limit_us, void* stream);

/*
 * ifq_device_status -- synchronize `stream`, then read and clear the device
 * status word of the current device: IFQ_OK, or the first device-side error
 * recorded (IFQ_ETIMEOUT, IFQ_ERANGE) since the last read.
 */
int ifq_device_status(void* stream, int* status);

/*
 * ---------------------------------------------------------------------------
 * The attention block of a quantised decoder.
 *
 * The same conventions hold for these calls (status, ownership, streams, no
 * allocation).  Rows, columns, tokens, and the tokens of a row of the page
 * table are at most 2^31 - 1024 (IFQ_ERANGE otherwise).  Types of 16- and
 * 32-bit tensors:
 */
enum { IFQ_F16 = 1, IFQ_BF16 = 2, IFQ_F32 = 3 };

/*
 * A paged key/value cache whose entries are held in 4 bits.  A page holds
 * page_size tokens (a multiple of 16) of every key/value head; the buffer is
 *   [pages][kv_heads][page_size / 16] groups of 16 tokens,
 * and a group of head size D (64, 128 or 256) has 16 * D + 128 bytes:
 *   K codes (8 * D bytes), V codes (8 * D bytes),
 *   K parameters, V parameters: 16 pairs (scale, min) of IEEE half each.
 * The value of a code is code * scale + min, with one pair per token and head.
 * Codes are 4-bit fields as everywhere in the library, the lower-numbered of
 * two in the low half of their byte.  With DB = min(D, 128), K codes are
 * [D / DB][16 tokens][DB]; V codes are [D / DB][2][8][4][DB / 32][2][4] with
 * token = 8 * (2nd axis) + 2 * (4th) + (6th) and dimension = DB / 8 * (3rd) +
 * 4 * (5th) + (7th) of its block, so that a 32-bit word holds the same four
 * dimensions of two neighbouring tokens.
 * The caller owns the buffer (16-byte aligned); a page is contiguous, so pages
 * can be copied or moved as bytes.  A slot is page * page_size + offset.
 */
typedef struct {
  int pages;
  int page_size;
  int kv_heads;
  int head_dim;
} ifq_kv4_cache;

/* Bytes of the cache's buffer (host, pure). */
int ifq_kv4_cache_bytes(const ifq_kv4_cache* c, size_t* bytes);

/* Rotation of the positions: none, pairs (i, i + rot_dim/2), or pairs (2i, 2i + 1). */
enum { IFQ_ROPE_NONE = 0, IFQ_ROPE_HALVES = 1, IFQ_ROPE_PAIRS = 2 };

/*
 * New tokens of ifq_kv4_append and ifq_kv4_read.  Rows of q, k, v and q_out
 * are tokens; within a row the heads are contiguous, [heads][head_dim]; the
 * strides count elements from row to row (0: rows are dense), so that q, k and
 * v may be parts of one projection's rows.  dtype is IFQ_F16 or IFQ_BF16.
 * rot_dim: the rotated dimensions of a head, the first ones, a multiple of 16
 * (<= head_dim; ignored for IFQ_ROPE_NONE); positions: rows of the cos and sin
 * tables.  tokens may be 0 (pointers are not looked at then).  Strides are
 * multiples of 8 elements and at least a row's width (IFQ_EINVAL otherwise).
 */
typedef struct {
  ifq_kv4_cache cache;
  int tokens;
  int q_heads;
  int dtype;
  int rope;
  int rot_dim;
  int positions;
  int64_t q_stride, k_stride, v_stride, q_out_stride;
} ifq_kv4_append_desc;

/*
 * ifq_kv4_append -- rotate q and k by their positions, quantise k and v to 4
 * bits and write them into the cache.  For a token at position p with table
 * rows cos[p], sin[p] (float [positions][rot_dim/2]), each rotated pair (a, b)
 * becomes (a*cos - b*sin, b*cos + a*sin); q is rounded to dtype and written to
 * q_out (which may be q).  Each head's row of k (rotated) and of v is
 * quantised by itself: with the row clamped to +-65504,
 *   min = half(smallest), scale = half((largest - smallest) * single(1/15)),
 *   code = clamp(rint((x - min) / scale), 0, 15), or 0 where scale is 0.
 * All of it in IEEE single, rounded operation by operation in the order
 * written (no fused multiply-add), so the codes are those of any program that
 * does the same.  A NaN in a row makes both its parameters NaN.
 * q (device): may be NULL, then q_out is not written.  positions (device):
 * int32 [tokens] (not read for IFQ_ROPE_NONE).  slots (device): int64
 * [tokens]; a negative slot leaves the cache as it is (padding tokens).  No
 * two tokens of a call may have the same slot.
 * Device-side checks: a slot past the cache or a position outside the tables
 * sets IFQ_ERANGE (ifq_device_status) and that token is skipped.
 * Pointers are 16-byte aligned (positions and tables 4, slots 8).
 */
int ifq_kv4_append(const ifq_kv4_append_desc* d, const void* q, const void* k, const void* v, const float* cos,
                   const float* sin, const int32_t* positions, const int64_t* slots, void* q_out, void* cache,
                   void* stream);

/*
 * ifq_kv4_read -- the values that the cache holds at `slots` (device, int64
 * [tokens]): code * scale + min in IEEE single, rounded to dtype, into k_out
 * and v_out (device, dense rows [tokens][kv_heads][head_dim]; either may be
 * NULL).  Uses cache, tokens and dtype of the descriptor.  A negative slot
 * reads as zeros; one past the cache too, and sets IFQ_ERANGE.
 */
int ifq_kv4_read(const ifq_kv4_append_desc* d, const void* cache, const int64_t* slots, void* k_out, void* v_out,
                 void* stream);

/*
 * Attention of new tokens' queries over the cache.  seqs sequences; sequence s
 * has lens[s] tokens in the cache (its new ones included), token j of it in
 * page page_table[s][j / page_size], row j % page_size.  Its queries are rows
 * q_starts[s] .. q_starts[s+1]-1 of q (n_s of them; q_starts NULL: row s
 * alone) and sit at its last n_s positions.  Query head h reads key/value head
 * h / (q_heads / kv_heads).  A query at position p sees the tokens j <= p, or
 * with window > 0 those with j > p - window or j < sinks.
 * q_tokens: rows of q; max_q: no sequence has more queries than this;
 * max_pages: entries of a row of page_table; max_len: no sequence is longer
 * (0: max_pages * page_size).  max_q and max_len choose the kernel and its
 * launch shape.  Strides of q and out as in ifq_kv4_append_desc.  seqs and
 * q_tokens may be 0 (pointers other than q_starts are not looked at then).
 */
typedef struct {
  ifq_kv4_cache cache;
  int seqs;
  int q_tokens;
  int max_q;
  int max_pages;
  int max_len;
  int q_heads;
  int dtype;
  float scale;
  int window;
  int sinks;
  int64_t q_stride, out_stride;
} ifq_kv4_attention_desc;

/* Device workspace of ifq_kv4_attention for `d` (host; the current device's, or a full GB300's where there is none). */
int ifq_kv4_attention_workspace_bytes(const ifq_kv4_attention_desc* d, size_t* bytes);

/*
 * ifq_kv4_attention -- out = softmax(scale * q K^T) V over the visible tokens,
 * with K and V the values the cache holds.  Codes enter the products as exact
 * numbers; scales, minima, sums and the softmax are in IEEE single, the weights
 * of V in half: eleven bits down to 2^-20 of the largest product of a weight and
 * a value's scale.  Where a key head has more than 32 rows
 * (max_q * q_heads / kv_heads) and dtype is bfloat16, the values of V are
 * rounded to half as well.  A token whose value parameters are not finite makes
 * the results of the queries that see it not finite and leaves their lse; one
 * whose key parameters are NaN makes both NaN.
 * out (device): [q_tokens] rows of [q_heads][head_dim], dtype.  lse (device,
 * may be NULL): float [q_tokens][q_heads], the log of the softmax's sum.  A
 * query that sees nothing gives zeros and -infinity.
 * page_table (device): int32 [seqs][max_pages]; lens (device): int32 [seqs];
 * q_starts (device): int32 [seqs + 1], ascending, or NULL.  Entries of
 * page_table past a sequence's length are not read, nor are tokens past it.
 * Device-side checks: a length that is negative or past the table's row,
 * q_starts out of order or past q_tokens, or more queries than max_q set
 * IFQ_ERANGE and leave that sequence's rows unwritten; a page past the cache
 * sets IFQ_ERANGE and its values are undefined (but the same in every call).
 * ws (device): ifq_kv4_attention_workspace_bytes bytes, 16-byte aligned; calls
 * in flight at the same time must not share it.  Results do not depend on
 * what it holds, nor on timing.
 */
int ifq_kv4_attention(const ifq_kv4_attention_desc* d, const void* q, const void* cache, const int32_t* page_table,
                      const int32_t* lens, const int32_t* q_starts, void* out, float* lse, void* ws, size_t ws_bytes,
                      void* stream);

/*
 * Product with operands in e4m3 and a float scale for each block of 128:
 *   out[i][j] = sum over blocks b of  x_scale[b][i] * w_scale[j / 128][b] *
 *               sum over k in block b of x[i][k] * w[j][k]
 * x: [m][k] e4m3, w: [n][k] e4m3 (dense rows), x_scale: float [ceil(k/128)][m],
 * w_scale: float [ceil(n/128)][ceil(k/128)].  The last block may hold fewer
 * than 128.  k is a multiple of 16 (IFQ_ESHAPE otherwise); m may be 0 (pointers
 * are not looked at then).
 * dtype: type of the activations that ifq_fp8_quantize reads (IFQ_F16 or
 * IFQ_BF16), with x_stride elements from row to row (0: dense; a multiple of
 * 8).  out_dtype: IFQ_F16, IFQ_BF16 or IFQ_F32, with out_stride elements from
 * row to row (0: dense).
 */
typedef struct {
  int m, n, k;
  int dtype;
  int out_dtype;
  int64_t x_stride, out_stride;
} ifq_fp8_desc;

/*
 * ifq_fp8_quantize -- activations to e4m3 with a scale per row and block of
 * 128 along k: scale = largest |x| of the block * single(1/448), code =
 * e4m3(x / scale) (nearest even), 0 where scale is 0, in IEEE single.  x (device): [m][k]
 * dtype; codes (device): [m][k] bytes; scales (device): float
 * [ceil(k/128)][m].  A NaN or an infinity in a block makes its scale NaN or
 * infinite, and with it the products of that row's block.
 */
int ifq_fp8_quantize(const ifq_fp8_desc* d, const void* x, void* codes, float* scales, void* stream);

/* Device workspace of ifq_fp8_matmul for `d` (host); may be 0. */
int ifq_fp8_workspace_bytes(const ifq_fp8_desc* d, size_t* bytes);

/*
 * ifq_fp8_matmul -- the product above.  Products are exact, their sums within a
 * block the tensor cores' in single precision (which may truncate), the scaled
 * blocks are added in IEEE single, and the sum is rounded once to out_dtype.
 * All pointers are device pointers, 16-byte aligned (scales 4; out 16, and out
 * rows start on a multiple of their element).
 */
int ifq_fp8_matmul(const ifq_fp8_desc* d, const void* x, const float* x_scale, const void* w, const float* w_scale,
                   void* out, void* ws, size_t ws_bytes, void* stream);

/*
 * ---------------------------------------------------------------------------
 * The rest of a quantised decoder layer, and its answers: products with weights
 * in 4 bits, the norm between the blocks, and scores of tokens.  Sizes as for
 * the attention block: at most 2^31 - 1024 (IFQ_ERANGE otherwise).
 */

/*
 * Weights held in 4 bits: w[j][c] = code * scale + min, rounded once to dtype
 * (IFQ_F16 or IFQ_BF16), with a scale and a minimum of that type for each row j
 * and group of 32, 64 or 128 along k (IFQ_EUNSUPPORTED otherwise; the last group
 * may hold fewer).  k is a multiple of 8 (IFQ_ESHAPE otherwise).  gated = 0: n
 * rows.  gated = 1: a pair of matrices of n rows each, 2n rows in all, the
 * gate's first.
 */
typedef struct {
  int n, k, group;
  int dtype;
  int gated;
} ifq_w4_weights;

/* Bytes of the packed weights (host, pure). */
int ifq_w4_bytes(const ifq_w4_weights* w, size_t* bytes);

/*
 * ifq_w4_pack -- the layout that the products read, made once per matrix.
 * codes (device): bytes [rows][k / 2], the even column in the low half of a
 * byte; scales, mins (device): dtype [rows][ceil(k / group)].  packed (device):
 * ifq_w4_bytes bytes, all of them written.  codes are 4-byte aligned, scales and
 * mins 2, packed 16.  The layout is the library's own; packed weights may be
 * copied as bytes.
 */
int ifq_w4_pack(const ifq_w4_weights* w, const void* codes, const void* scales, const void* mins, void* packed,
                void* stream);

/* What the gate's products go through before they meet the others'. */
enum { IFQ_ACT_SILU = 1, IFQ_ACT_GELU = 2, IFQ_ACT_GELU_TANH = 3 };

/*
 * A product of m rows.  Strides count elements from row to row (0: dense); x's
 * is a multiple of 8.  out_dtype: IFQ_F16, IFQ_BF16 or IFQ_F32, the type of out
 * and residual.  act: of ifq_w4_gated (ignored by ifq_w4_matmul).  m may be 0
 * (pointers are not looked at then).  All device pointers are 16-byte aligned.
 */
typedef struct {
  ifq_w4_weights weights;
  int m;
  int out_dtype;
  int act;
  int64_t x_stride, out_stride, residual_stride;
} ifq_w4_desc;

/*
 * ifq_w4_matmul -- out[i][j] = sum over c of x[i][c] * w[j][c] (+ residual[i][j]).
 * x (device): [m][k] of the weights' dtype; residual (device): [m][n], may be
 * NULL, and may be out where the strides agree; out overlaps nothing else.
 * Products are exact, sums in single precision (which the tensor cores may
 * truncate), rounded once to out_dtype.  Results do not depend on timing; they
 * may on m, which chooses the kernel and so the order of the sums.  What is not
 * finite in a row of x or of the weights stays in that row of out, or column.
 * weights.gated is 0.
 */
int ifq_w4_matmul(const ifq_w4_desc* d, const void* x, const void* packed, void* out, const void* residual,
                  void* stream);

/*
 * ifq_w4_gated -- out[i][j] = act(sum x[i][c] * w[j][c]) * sum x[i][c] * w[n+j][c]:
 * both projections of a gated feed-forward block, the activation and the product
 * in one launch, with sums as above, act in single precision (what is below
 * 2^-126 there may be 0), and one rounding.
 *   IFQ_ACT_SILU: a / (1 + e^-a);  IFQ_ACT_GELU: a * (1 + erf(a / sqrt 2)) / 2;
 *   IFQ_ACT_GELU_TANH: a * (1 + tanh(sqrt(2 / pi) (a + 0.044715 a^3))) / 2.
 * weights.gated is 1, out_dtype the weights' dtype.  residual_stride is not read.
 */
int ifq_w4_gated(const ifq_w4_desc* d, const void* x, const void* packed, void* out, void* stream);

/*
 * Rows of dim values of dtype (IFQ_F16 or IFQ_BF16).  dim is a multiple of 8
 * (IFQ_ESHAPE) and at most 65536 (IFQ_EUNSUPPORTED); eps is finite and >= 0.
 * Strides count elements from row to row (0: dense), multiples of 8.
 */
typedef struct {
  int rows, dim;
  int dtype;
  float eps;
  int64_t x_stride, residual_stride, sum_stride, out_stride;
} ifq_norm_desc;

/*
 * ifq_rms_norm -- out = h * weight / sqrt(mean(h * h) + eps), with h = x, or with
 * a residual h = x + residual, added in single precision and rounded to dtype,
 * which is written to sum (may be NULL).  Squares and their sum in single
 * precision (in double where they leave its range), h / sqrt(...) and its product
 * with weight in single precision too (where the first is below 2^-126 it has
 * fewer digits), out rounded to dtype.  weight (device): dtype [dim].  sum and out may
 * each be x or residual, where the strides agree, but not the same buffer.
 * Without a residual sum is NULL.
 * rows may be 0.  Pointers are 16-byte aligned.
 */
int ifq_rms_norm(const ifq_norm_desc* d, const void* x, const void* residual, const void* weight, void* sum, void* out,
                 void* stream);

/*
 * Rows of vocab logits of dtype (IFQ_F16, IFQ_BF16 or IFQ_F32), stride elements
 * from row to row (0: dense; any number of them).  top: how many of the
 * likeliest tokens are wanted, 0 to 32 (IFQ_EUNSUPPORTED) and at most vocab
 * (IFQ_ESHAPE).  scale: one over a temperature, > 0 and at most 2^100
 * (IFQ_ERANGE).
 */
typedef struct {
  int rows, vocab;
  int dtype;
  int top;
  float scale;
  int64_t stride;
} ifq_scores_desc;

/*
 * ifq_token_scores -- with z = scale * logits of a row and p = softmax(z):
 *   lse = log sum exp z, logprobs = z[token] - lse, entropy = -sum p log p,
 *   top_ids: the tokens of the top largest logits, in descending order, of equals
 *   the lowest first; top_logprobs: z - lse of those.
 * tokens (device): int64 [rows]; a negative one (padding) gives 0; one past the
 * vocabulary sets IFQ_ERANGE (ifq_device_status) and gives NaN.  logprobs, lse,
 * entropy (device): float [rows]; top_ids: int64 [rows][top]; top_logprobs:
 * float [rows][top].  Each output may be NULL (tokens too, with logprobs).
 * A token of -infinity has no share in lse and entropy; where all are, lse and
 * all log probabilities are -infinity and the entropy is 0.  A logit of
 * +infinity makes lse +infinity and the entropy NaN, a NaN all of the row's
 * numbers; NaN comes before every number among top_ids.  Computed in single
 * precision; results do not depend on timing.  logits are aligned to their
 * type, tokens and top_ids to 8 bytes.
 * rows may be 0 (pointers are not looked at then).
 */
int ifq_token_scores(const ifq_scores_desc* d, const void* logits, const int64_t* tokens, float* logprobs, float* lse,
                     float* entropy, int64_t* top_ids, float* top_logprobs, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* IFQ_H */
