/*
 * int8t.h -- C ABI of the MI355X (gfx950) INT8 training-convolution library.
 *
 * The calls are the per-layer steps of "Towards Unified INT8 Training for
 * Convolutional Neural Network":
 *
 *   int8t_quantize         Eq.1 (symmetric uniform quantizer, s = c/127) with
 *                          round-to-nearest for activations / weights and the
 *                          stochastic rounding of Eq.3 for output gradients;
 *                          optionally reports the direction deviation of Eq.6.
 *   int8t_dsgc_clip        Direction Sensitive Gradient Clipping (Sec.3.4): picks
 *                          the clip value of the output gradient that minimises
 *                          the cosine deviation d_c of Eq.6, as a search over
 *                          caller-supplied candidates; also returns d_c, the
 *                          scalar Eq.7 consumes.
 *   int8t_conv_fwd         z  = q_a (*) q_W          int8 x int8 -> int32, then Eq.2
 *   int8t_conv_bwd_data    g_a = q_gz (*)^T q_W      (Sec.3.4; Suppl. "INT8 Convolution")
 *   int8t_conv_bwd_weight  g_W = q_gz^T q_a          (Sec.3.4)
 *   int8t_dclr_scale       Eq.7, phi(d_c) = max(exp(-alpha d_c), beta)   (host)
 *
 * General conventions
 *   - Every pointer named *_dev is DEVICE memory owned by the caller.  The library
 *     never allocates, frees or keeps device memory between calls.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  All
 *     work is enqueued asynchronously on it; no call synchronises with the host.
 *   - Scalars that flow between calls (clip, scale, deviation) stay in device
 *     memory, so the calls of one layer step chain without a host round trip.
 *   - fp32 tensors are dense, in PyTorch's logical order: activations and
 *     gradients N,C,H,W; weights K,C/groups,R,S.  They must be 16-byte aligned.
 *   - Errors are return codes.  Argument errors are detected before anything is
 *     launched; in that case no output is touched.
 *   - `ws_dev` is scratch the caller provides; ask int8t_workspace_bytes() how
 *     much a call needs.  Its contents need no initialisation and are
 *     unspecified afterwards.  Two calls that run concurrently (different
 *     streams) must not share scratch.
 *   - Inputs must be finite.  NaN quantizes to code 0; results derived from
 *     non-finite inputs are otherwise unspecified (but memory safe).
 *
 * Layout of int8 code tensors (the library's own; Suppl. "INT8 Convolution"
 * packs the reduction dimension innermost for the dot-product instruction, and
 * so do we, in granules of 16 bytes for the int8 MFMA):
 *   INT8T_ACT         dims {N,C,H,W}: codes[((n*H + h)*W + w)*Cp + c], Cp = C rounded up
 *                     to a multiple of 16, bytes c >= C are zero.  N*H*W*Cp bytes.
 *   INT8T_ACT_PLANAR  dims {N,C,H,W}: codes in logical N,C,H,W order (depthwise layers).
 *   INT8T_WGT         dims {K,Cg,R,S} (Cg = C/groups, groups == 1): two copies,
 *                       [0, K*R*S*Cp):             codes[((k*R + r)*S + s)*Cp + c]
 *                       [align256(K*R*S*Cp), ...): codes[((c*R + r)*S + s)*Kp + k]
 *                     (the second serves backward-data), Cp/Kp rounded up to 16, pad zero.
 *   INT8T_WGT_PLANAR  dims {K,Cg,R,S}: codes in logical order (depthwise layers).
 * int8t_code_bytes() returns the size of each.
 *
 * The stochastic draw of element i is a function of (seed, i) only, where i is
 * the element's linear index in LOGICAL order, so codes do not depend on the
 * code layout, the launch geometry or the clip search.
 */
#ifndef INT8T_H
#define INT8T_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    INT8T_OK = 0,
    INT8T_ERR_NULL = 1,       /* a required pointer is NULL */
    INT8T_ERR_SHAPE = 2,      /* non-positive or unsupported dimensions */
    INT8T_ERR_ARG = 3,        /* bad enum value, misaligned pointer, too many candidates */
    INT8T_ERR_WORKSPACE = 4,  /* ws_bytes smaller than int8t_workspace_bytes() */
    INT8T_ERR_RUNTIME = 5,    /* a HIP launch failed */
    INT8T_ERR_LIMIT = 6,      /* size beyond what an allocation-free variant (int8t_dsgc_clip_static) takes */
    INT8T_STATUS_MAX_ENUM = 0x7fffffff
} int8t_status;

/* (The *_MAX_ENUM enumerators only make every non-negative int a representable value of its enum, so
 * that a caller's out-of-range argument reaches the argument checks as a value, not as undefined
 * behaviour in the C++ implementation.  They are never returned and never valid as arguments.) */
typedef enum { INT8T_ROUND_NEAREST_EVEN = 0, INT8T_ROUND_STOCHASTIC = 1, INT8T_ROUND_MAX_ENUM = 0x7fffffff } int8t_round;

typedef enum {
    INT8T_ACT = 0,
    INT8T_WGT = 1,
    INT8T_ACT_PLANAR = 2,
    INT8T_WGT_PLANAR = 3,
    INT8T_KIND_MAX_ENUM = 0x7fffffff
} int8t_kind;

typedef enum {
    INT8T_OP_QUANTIZE = 0,
    INT8T_OP_DSGC = 1,
    INT8T_OP_CONV_FWD = 2,
    INT8T_OP_CONV_BWD_DATA = 3,
    INT8T_OP_CONV_BWD_WEIGHT = 4,
    INT8T_OP_MAX_ENUM = 0x7fffffff
} int8t_op;

/* Convolution geometry, PyTorch conventions: cross-correlation, zero padding,
 * P = floor((H + 2 pad_h - R)/stride_h) + 1, dilation 1.  groups must be 1
 * (dense; code layouts INT8T_ACT / INT8T_WGT) or C == K == groups (depthwise;
 * INT8T_ACT_PLANAR / INT8T_WGT_PLANAR). */
typedef struct {
    int N, C, H, W, K, R, S, stride_h, stride_w, pad_h, pad_w, groups;
} int8t_conv_desc;

#define INT8T_MAX_CANDIDATES 64

const char *int8t_status_string(int8t_status s);

/* Bytes of the int8 code tensor of `kind` for logical dims; 0 on bad input. */
size_t int8t_code_bytes(const int dims[4], int8t_kind kind);

/*
 * Checking aid (HOST memory on both sides, plain loops, no GPU work): rewrites a code tensor from the
 * library's layout (see "Layout of int8 code tensors" above; Suppl. "INT8 Convolution" for why the
 * reduction dimension is packed innermost) into logical order, so that a caller can compare codes
 * with Eq.1 / Eq.3 evaluated element by element without knowing the layout.
 *   codes_host    int8t_code_bytes(dims, kind) bytes copied back from the device
 *   copy          INT8T_WGT only: 0 = the forward copy [K][R][S][Cp], 1 = the backward-data copy
 *                 [C][R][S][Kp]; must be 0 for the other kinds
 *   out_host      out: dims[0]*dims[1]*dims[2]*dims[3] codes in logical order (N,C,H,W or K,Cg,R,S)
 *   pad_nonzero   NULL, or out: number of padding bytes (channel positions >= C resp. >= K) of the
 *                 unpacked copy that are not zero -- the convolutions rely on their being zero
 * Returns INT8T_ERR_NULL / INT8T_ERR_SHAPE / INT8T_ERR_ARG on bad input and touches nothing then.
 */
int8t_status int8t_unpack_codes(const int8_t *codes_host, const int dims[4], int8t_kind kind, int copy,
                                int8_t *out_host, size_t *pad_nonzero);

/* Scratch a call needs.  DSGC: n = element count, n_cand = number of candidates, desc ignored.
 * CONV_*: desc required, n / n_cand ignored.  QUANTIZE: use int8t_quantize_workspace_bytes()
 * (this function returns 0 for it).  0 also means "bad arguments" for the CONV ops whose
 * descriptor is invalid; the call itself then reports the error.
 * CONV_BWD_WEIGHT and DSGC require their scratch.  CONV_FWD / CONV_BWD_DATA only use it as a
 * performance aid (layers with few output tiles and a long reduction split the reduction over
 * several workgroups and keep int32 partial sums there; the forward pass of a stride-2 layer with
 * at most 4 input channels -- the stem of an image network -- runs on a space-to-depth copy of its
 * codes kept there, four times the channels per 16-byte pixel and a quarter of the taps; integer
 * sums of the same products either way, so the result is the same bit for bit): ws_dev may be NULL
 * or smaller, the call then runs without them.  CONV_BWD_WEIGHT of such a layer holds the same
 * copy of the input codes in its (required) scratch. */
size_t int8t_workspace_bytes(int8t_op op, const int8t_conv_desc *desc, size_t n, int n_cand);

/* Scratch of int8t_quantize for a tensor of logical dims and code layout `kind`; covers both the
 * absmax pass (clip_dev == NULL) and the deviation output.  0 on bad input. */
size_t int8t_quantize_workspace_bytes(const int dims[4], int8t_kind kind);

/*
 * Eq.1 / Eq.3.  Per element (fp32, each operation rounded once, no fused multiply-add):
 *     inv = 127 / c
 *     nearest:    q = rint(min(max(x * inv, -127), 127))                 (ties to even)
 *     stochastic: m = min(127, floor((|x| * (inv * 2^24) + u) / 2^24)) in exact arithmetic,
 *                 q = sign(x) * m,  u = 24 uniform bits drawn from (seed, logical index)
 *                 ==> |q| = floor(|x|/s) + 1 with probability frac(|x|/s), resolved to 2^-24:
 *                 the distribution of Eq.3 (rounding the magnitude and restoring the sign keeps
 *                 the probabilities of floor and floor + 1 also for negative values).
 *   x_dev          fp32 tensor, logical order, dims[0]*dims[1]*dims[2]*dims[3] elements
 *   clip_dev       clip value c (1 float), or NULL: c = max|x| is computed first
 *   q_dev          out: int8 codes in the layout of `kind`, int8t_code_bytes() bytes
 *   scale_dev      out: 1 float, s = c / 127 (0 when c == 0, and then all codes are 0)
 *   deviation_dev  NULL, or out: 1 double, d_c of Eq.6 between x and q*s
 *                  (0 when x is all zero; 1 when every code is 0 but x is not)
 */
int8t_status int8t_quantize(const float *x_dev, const int dims[4], int8t_kind kind,
                            const float *clip_dev, int8t_round mode, uint64_t seed,
                            int8_t *q_dev, float *scale_dev, double *deviation_dev,
                            void *ws_dev, size_t ws_bytes, void *stream);

/*
 * Eq.1 / Eq.3 for several tensors at once (no deviation output): the result of each item is exactly
 * what int8t_quantize(..., mode, seed, ...) writes for it, but all absmax passes share one launch
 * and all quantize passes another.  Meant for the activations and the weights of a layer -- and, in
 * an iteration that keeps the clip value of an earlier search (Periodic Update, Sec.3.4), its
 * output gradient too -- or the weights of many layers: a small tensor no longer costs two kernel
 * launches of its own.
 *   items    host array of `count` (1 .. INT8T_MAX_BATCH) items, read before the call returns;
 *            fields as the arguments of the same names of int8t_quantize
 *   ws_dev   int8t_quantize_batch_workspace_bytes() bytes, 16-byte aligned; may be NULL when every
 *            item brings its clip value
 */
#define INT8T_MAX_BATCH 8
typedef struct int8t_quantize_item {
    const float *x_dev;
    int dims[4];
    int8t_kind kind;
    const float *clip_dev;
    int8_t *q_dev;
    float *scale_dev;
    int8t_round mode;
    uint64_t seed;             /* used by INT8T_ROUND_STOCHASTIC only */
} int8t_quantize_item;
size_t int8t_quantize_batch_workspace_bytes(int count, const int8t_quantize_item *items);
int8t_status int8t_quantize_batch(int count, const int8t_quantize_item *items,
                                  void *ws_dev, size_t ws_bytes, void *stream);

/*
 * Clip search of Sec.3.4.  Candidates c_j = fl32(max|g| * ratios[j]), j < n_cand
 * (1 <= n_cand <= INT8T_MAX_CANDIDATES).  For each, the tensor is quantized exactly
 * as int8t_quantize(mode, seed) would, and d_j = 1 - cos(g, q*s) (Eq.6) is evaluated;
 * the smallest d_j wins, ties go to the smallest j.
 *   g_dev              fp32 tensor, n elements (n < 2^31), logical order
 *   ratios_dev         n_cand floats in (0, 1]
 *   clip_dev           out: 1 float, the winning c_j
 *   deviation_dev      out: 1 double, its d_j
 *   deviation_all_dev  NULL, or out: n_cand doubles, every d_j
 */
int8t_status int8t_dsgc_clip(const float *g_dev, size_t n, const float *ratios_dev, int n_cand,
                             int8t_round mode, uint64_t seed,
                             float *clip_dev, double *deviation_dev, double *deviation_all_dev,
                             void *ws_dev, size_t ws_bytes, void *stream);

/*
 * The same search in its two phases, for callers that want to put something between them (an event
 * for a second stream, say): int8t_dsgc_prepare is the pass over g that finds max|g| and the sum of
 * squares of Eq.6 and clears the accumulators in the scratch; int8t_dsgc_search is the sweep over
 * the candidates, which needs the scratch exactly as the preceding int8t_dsgc_prepare on the same g,
 * n and ws_dev left it.  int8t_dsgc_clip is the two calls in a row; arguments as there.
 */
int8t_status int8t_dsgc_prepare(const float *g_dev, size_t n, void *ws_dev, size_t ws_bytes, void *stream);
/*
 * int8t_quantize_batch and int8t_dsgc_prepare in one call: the pass over g shares the launch of the items'
 * absmax passes (a step on one stream then has one launch fewer; Sec.3.4: max|.| of a, W and g_z are
 * independent of each other).  Writes what the two calls write, bit for bit; int8t_dsgc_search follows it
 * as it follows int8t_dsgc_prepare.
 *   count, items, ws_dev, ws_bytes   as for int8t_quantize_batch
 *   g_dev, n                         as for int8t_dsgc_prepare (required)
 *   dsgc_ws_dev, dsgc_ws_bytes       the search's scratch: int8t_workspace_bytes(INT8T_OP_DSGC, NULL, n, n_cand) bytes,
 *                                    16-byte aligned, not overlapping ws_dev
 * Errors as for the two calls; nothing is launched then.
 */
int8t_status int8t_quantize_batch_prepare(int count, const int8t_quantize_item *items, void *ws_dev, size_t ws_bytes,
                                          const float *g_dev, size_t n, void *dsgc_ws_dev, size_t dsgc_ws_bytes,
                                          void *stream);
int8t_status int8t_dsgc_search(const float *g_dev, size_t n, const float *ratios_dev, int n_cand,
                               int8t_round mode, uint64_t seed,
                               float *clip_dev, double *deviation_dev, double *deviation_all_dev,
                               void *ws_dev, size_t ws_bytes, void *stream);

/*
 * int8t_dsgc_clip for callers that cannot provide scratch because they cannot allocate: code under
 * HIP graph capture, tight serving / training loops, harnesses that forbid hipMalloc.  Same search,
 * same results bit for bit, same arguments minus ws_dev / ws_bytes: the scratch (absmax partials,
 * accumulator sets and ticket, sum-of-squares partials; INT8T_DSGC_STATIC_SCRATCH_BYTES = 61 696 bytes,
 * whatever n is) is an array inside the library's device image, one copy per GPU, held until the
 * process ends.  The call allocates and frees nothing -- no hipMalloc, no hipFree, no allocating
 * library routine -- and clears what must start at zero with a kernel's own stores, not a memset node.
 *   Limits: n <= INT8T_DSGC_STATIC_MAX_ELEMS and n_cand <= INT8T_MAX_CANDIDATES, else
 *   INT8T_ERR_LIMIT and nothing is launched (n == 0 is INT8T_ERR_SHAPE, n_cand < 1 INT8T_ERR_ARG).
 *   All calls on one GPU share that GPU's array, which keeps the previous call's contents: calls on
 *   the same stream are ordered and safe; calls that OVERLAP on one GPU (different streams, or
 *   several host threads on several streams) race on it and give wrong results.  Use
 *   int8t_dsgc_clip with separate scratch for concurrent searches.
 *   The first call on a GPU looks the array's device address up (hipGetSymbolAddress, with that GPU
 *   current); make that call outside stream capture.
 */
#define INT8T_DSGC_STATIC_SCRATCH_BYTES 61696
#define INT8T_DSGC_STATIC_MAX_ELEMS 0x7FFFFFFFull
int8t_status int8t_dsgc_clip_static(const float *g_dev, size_t n, const float *ratios_dev, int n_cand,
                                    int8t_round mode, uint64_t seed,
                                    float *clip_dev, double *deviation_dev, double *deviation_all_dev,
                                    void *stream);

/*
 * Forward convolution on codes: acc[n,k,p,q] = sum_{c,r,s} xq[n,c,p*sh+r-ph,q*sw+s-pw] * wq[k,c,r,s]
 * in int32 (two's-complement wrap), then Eq.2: y = (float)acc * (sx * sw).
 *   xq_dev   INT8T_ACT codes of dims {N,C,H,W}   (INT8T_ACT_PLANAR when depthwise)
 *   wq_dev   INT8T_WGT codes of dims {K,C/g,R,S} (INT8T_WGT_PLANAR when depthwise)
 *   sx_dev, sw_dev   1 float each (the scales int8t_quantize wrote)
 *   y_dev    out: fp32 N,K,P,Q
 *   acc_dev  NULL, or out: int32 N,K,P,Q, the raw accumulators
 *   ws_dev   NULL, or int8t_workspace_bytes(INT8T_OP_CONV_FWD, ...) bytes of scratch, 16-byte aligned
 *            (optional, see there; the same holds for int8t_conv_bwd_data)
 */
int8t_status int8t_conv_fwd(const int8t_conv_desc *desc,
                            const int8_t *xq_dev, const float *sx_dev,
                            const int8_t *wq_dev, const float *sw_dev,
                            float *y_dev, int32_t *acc_dev,
                            void *ws_dev, size_t ws_bytes, void *stream);

/*
 * The quantization-convolution fused kernel of the paper's Suppl. "INT8 Convolution" ("avoids one
 * extra global memory read and write"), for the layers where it saves traffic here: a 1 x 1 filter at
 * stride 1 without padding (dense).  int8t_quantize(a) + int8t_conv_fwd in one call: the forward pass
 * reads the fp32 activations, applies Eq.1 (round to nearest) in its load path with c = *clip_dev or
 * max|a| (found by a first pass when clip_dev is NULL), and multiplies the codes without their making
 * the round trip through memory.  Results are bit for bit those of the two separate calls.
 *   x_dev    fp32 N,C,H,W;  wq_dev / sw_dev as in int8t_conv_fwd
 *   xq_dev   NULL, or out: the INT8T_ACT codes of a, for the backward-weight pass (a forward-only
 *            caller leaves it out and saves their write as well)
 *   sx_dev   out: 1 float, the scale of a
 *   ws_dev   1024 floats of scratch when clip_dev is NULL, else unused
 * INT8T_ERR_SHAPE for any other filter, stride, padding or a depthwise layer.  A layer with more
 * than 128 filters reads (and quantizes) its activations once per 128 filters: the separate calls are
 * the better choice there.
 */
int8t_status int8t_conv_fwd_fused(const int8t_conv_desc *desc, const float *x_dev, const float *clip_dev,
                                  const int8_t *wq_dev, const float *sw_dev,
                                  float *y_dev, int32_t *acc_dev, int8_t *xq_dev, float *sx_dev,
                                  void *ws_dev, size_t ws_bytes, void *stream);

/*
 * Backward-data: acc[n,c,h,w] = sum over (k,r,s,p,q) with p*sh+r-ph = h, q*sw+s-pw = w of
 * dyq[n,k,p,q] * wq[k,c,r,s];  dx = (float)acc * (sdy * sw).
 *   dyq_dev  INT8T_ACT codes of dims {N,K,P,Q} (planar when depthwise);  wq_dev as in forward
 *   dx_dev   out: fp32 N,C,H,W;   acc_dev NULL or int32 N,C,H,W
 */
int8t_status int8t_conv_bwd_data(const int8t_conv_desc *desc,
                                 const int8_t *dyq_dev, const float *sdy_dev,
                                 const int8_t *wq_dev, const float *sw_dev,
                                 float *dx_dev, int32_t *acc_dev,
                                 void *ws_dev, size_t ws_bytes, void *stream);

/*
 * Backward-weight: acc[k,c,r,s] = sum_{n,p,q} dyq[n,k,p,q] * xq[n,c,p*sh+r-ph,q*sw+s-pw];
 * dw = (float)acc * (sdy * sx).  The forward's codes of x are re-used.
 *   dw_dev   out: fp32 K,C/g,R,S;   acc_dev NULL or int32 K,C/g,R,S
 */
int8t_status int8t_conv_bwd_weight(const int8t_conv_desc *desc,
                                   const int8_t *xq_dev, const float *sx_dev,
                                   const int8_t *dyq_dev, const float *sdy_dev,
                                   float *dw_dev, int32_t *acc_dev,
                                   void *ws_dev, size_t ws_bytes, void *stream);

/*
 * The same with the scratch that an int8t_conv_fwd on this layer and these codes xq was given, its contents unchanged since (and that
 * call ordered before this one): where both passes of a layer rewrite the codes of a first (stride 2 on at most 4 channels),
 * the forward pass's are used.  fwd_ws_bytes is what that call was given.  fwd_ws_dev NULL, of too few bytes for the rewritten codes
 * (the forward pass then did without), or within ws_dev, which this call writes: as int8t_conv_bwd_weight.
 */
int8t_status int8t_conv_bwd_weight_fwd(const int8t_conv_desc *desc,
                                       const int8_t *xq_dev, const float *sx_dev,
                                       const int8_t *dyq_dev, const float *sdy_dev,
                                       float *dw_dev, int32_t *acc_dev,
                                       void *ws_dev, size_t ws_bytes,
                                       const void *fwd_ws_dev, size_t fwd_ws_bytes, void *stream);

/*
 * The calls of one layer's training step (Sec.3.4) in one: what int8t_quantize_batch_prepare, int8t_dsgc_search,
 * int8t_quantize of g_z and the three convolutions write, bit for bit, in fewer launches -- calls that do not depend on
 * one another share a launch, and a step of a small layer is a chain of launches before it is anything else.
 *   parts   which of the calls run, an OR of the values below; each needs the results of the ones named with it from this
 *           or an earlier call.  A caller with two streams deals the parts to them; everything else passes INT8T_STEP_ALL
 *           (search and input gradient left out where they are not wanted).
 *   b       device pointers as in the calls of the same argument names; y_acc, dx_acc, dw_acc, dev_all and dev_final
 *           may be NULL (dev_final: d_c of Eq.6 of the codes of g_z, as int8t_quantize reports it), those that no part of
 *           this call uses as well.  Read before the call returns.
 *   ws_quant     3 x int8t_quantize_batch_workspace_bytes(1, ..) bytes: the absmax partials of a and W, kept between
 *                INT8T_STEP_ABSMAX and INT8T_STEP_QUANT_XW
 *   ws_dy        max(int8t_workspace_bytes(INT8T_OP_DSGC, ..), int8t_quantize_workspace_bytes(dims of g_z)) bytes; between
 *                INT8T_STEP_ABSMAX and INT8T_STEP_QUANT_XW a search may not run in memory that overlaps ws_quant
 *                (INT8T_ERR_ARG within one call)
 *   ws_fwd, ws_bwd_data    as for int8t_conv_fwd / int8t_conv_bwd_data (optional);  ws_bwd_weight: required by that part
 * Errors as for the calls; arguments are checked before anything is launched.
 */
typedef enum {
    INT8T_STEP_ABSMAX = 1,       /* max|a|, max|W|; with INT8T_STEP_PREPARE also the first pass of the clip search, same launch */
    INT8T_STEP_PREPARE = 2,
    INT8T_STEP_SEARCH = 4,       /* the sweep over the candidates (after PREPARE) */
    INT8T_STEP_QUANT_XW = 8,     /* codes of a and W (after ABSMAX) */
    INT8T_STEP_QUANT_G = 16,     /* codes of g_z, stochastic rounding, with the clip value at `clip` */
    INT8T_STEP_FWD = 32,         /* (after QUANT_XW) */
    INT8T_STEP_BWD_DATA = 64,    /* (after QUANT_XW, QUANT_G) */
    INT8T_STEP_BWD_WEIGHT = 128, /* (after QUANT_XW, QUANT_G) */
    INT8T_STEP_ALL = 255,
    INT8T_STEP_MAX_ENUM = 0x7fffffff
} int8t_step_part;
typedef struct int8t_layer_buffers {
    const float *x, *w, *dy;
    int8_t *xq, *wq, *dyq;
    float *sx, *sw, *sdy;
    const float *ratios;
    float *clip;
    double *dev_search, *dev_all, *dev_final;
    float *y, *dx, *dw;
    int32_t *y_acc, *dx_acc, *dw_acc;
    void *ws_quant, *ws_dy, *ws_fwd, *ws_bwd_data, *ws_bwd_weight;
    size_t ws_quant_bytes, ws_dy_bytes, ws_fwd_bytes, ws_bwd_data_bytes, ws_bwd_weight_bytes;
    int n_cand;
} int8t_layer_buffers;
int8t_status int8t_layer_step(const int8t_conv_desc *desc, const int8t_layer_buffers *b, int parts, uint64_t seed,
                              void *stream);

/*
 * The launch that passes of a step share: what int8t_layer_step does with these parts where no two buffers overlap, the scratch is as
 * int8t_workspace_bytes() says and dev_final is NULL.  (INT8T_FORM_APART also for arguments that it refuses.)
 */
typedef enum {
    INT8T_FORM_APART = 0,                /* a launch per pass */
    INT8T_FORM_128X128 = 1,              /* dense, stride 1: the passes on tiles of 128 rows x 128 columns, */
    INT8T_FORM_128X64 = 2,               /* 128 x 64, */
    INT8T_FORM_64X128 = 3,               /* 64 x 128 (all have at most 64 rows), */
    INT8T_FORM_64X128_AND_128X128 = 4,   /* or by their rows */
    INT8T_FORM_STRIDED = 5,              /* dense, strided: backward-data pixel by pixel, */
    INT8T_FORM_STRIDED_CLASSES = 6,      /* a class of pixels per tile, */
    INT8T_FORM_STRIDED_CELL = 7,         /* cells of pixels of which one has taps, */
    INT8T_FORM_STRIDED_CELLS = 8,        /* the classes of a cell one after the other */
    INT8T_FORM_DW_PASSES = 9,            /* depthwise: the passes, */
    INT8T_FORM_DW_CODES = 10,            /* and the codes as well */
    INT8T_FORM_BANDS = 11,               /* dense, stride 1: bands of rows, the filter bank on chip; the forward pass ahead where its form is another */
    INT8T_FORM_MAX_ENUM = 0x7fffffff
} int8t_form;
int8t_form int8t_layer_step_form(const int8t_conv_desc *desc, int parts);

/*
 * The backward half of a step in one call, for callers whose forward pass ran earlier (a layer inside a network): as
 * int8t_layer_step with any of INT8T_STEP_PREPARE together with INT8T_STEP_SEARCH (here without INT8T_STEP_ABSMAX),
 * INT8T_STEP_QUANT_G, INT8T_STEP_BWD_DATA and INT8T_STEP_BWD_WEIGHT; other parts: INT8T_ERR_ARG.
 *   db_dev   NULL, or K floats: out, the sum of dy over the batch (the gradient of a bias; summed in fp64), for layers with one
 *            output pixel (P = Q = 1; INT8T_ERR_ARG for others).  It may not overlap what the call reads or writes otherwise.
 *            64 columns are one block, which walks all rows of the batch: meant for up to a thousand rows or two.
 */
int8t_status int8t_layer_backward(const int8t_conv_desc *desc, const int8t_layer_buffers *b, int parts, uint64_t seed,
                                  float *db_dev, void *stream);

/*
 * The forward pass of a layer nobody wants the codes of (a network in use): y as int8t_layer_step with INT8T_STEP_ABSMAX,
 * INT8T_STEP_QUANT_XW and INT8T_STEP_FWD writes it, bit for bit; the same buffers are required.  xq, wq, sx and sw then either
 * hold what those parts write or are as they were (a 1x1 layer with few filters quantizes inside the convolution): codes of W that an
 * earlier call left there are still those of the same W.
 */
int8t_status int8t_layer_infer(const int8t_conv_desc *desc, const int8t_layer_buffers *b, void *stream);

/*
 * Choice of the kernel per layer by measurement "before training" (Suppl. "INT8 Convolution", last
 * paragraph: the paper picks between its two convolution algorithms per layer; here the choice is
 * among this library's kernels for a pass).  Every variant computes the same integer sums, so the
 * results are identical bit for bit; a caller times the variants int8t_conv_variant_ok() admits on
 * the layer's own buffers and selects the fastest.  The selection is kept in a process-wide table
 * keyed by (pass, descriptor) until it is changed; INT8T_VARIANT_AUTO (the default for every layer)
 * restores the library's own rules.  Thread-safe; not device-specific.
 *   forward / backward-data:  BAND, TILE, TILE_SPLIT, WIDE128, WIDE256, WIDE_SQ128, WIDE_SQ128_DEEP, WIDE_128X64;
 *   backward-data only:       WIDE_CELLS
 *   backward-weight:          WGRAD_IMAGES, WGRAD_LINES (the two kernels), WGRAD_FEWER, WGRAD_MORE (half / twice the
 *                             reduction shares of the cost model's choice); query int8t_workspace_bytes() again
 *                             after selecting any of them
 * Depthwise layers are served by the library's own choice among their kernels only.  A variant that needs scratch (TILE_SPLIT) and is not
 * given enough falls back to TILE.  A pass with a selected variant does not share a launch with others in int8t_layer_step,
 * nor do they then with it: time the step's passes together before keeping a selection.
 */
typedef enum {
    INT8T_VARIANT_AUTO = 0,
    INT8T_VARIANT_BAND = 1,          /* filter bank resident on chip, output rows streamed (small banks, stride 1) */
    INT8T_VARIANT_TILE = 2,          /* 64/128 x 128 implicit-GEMM tiles staged through registers */
    INT8T_VARIANT_TILE_SPLIT = 3,    /* ... with the reduction split over several blocks per tile */
    INT8T_VARIANT_WIDE128 = 4,       /* 128 x 256 tiles, operands loaded straight into a 3-stage LDS ring */
    INT8T_VARIANT_WIDE256 = 5,       /* 256 x 256 tiles, 2 stages of 128 reduction bytes */
    INT8T_VARIANT_WGRAD_FEWER = 6,
    INT8T_VARIANT_WGRAD_MORE = 7,
    INT8T_VARIANT_WGRAD_IMAGES = 8,  /* backward-weight: operands of 16 images per pixel, transposed in registers */
    INT8T_VARIANT_WGRAD_LINES = 9,   /* backward-weight, stride 1 with 1, 3, 5 or 7 taps along an axis, 1x1 at any stride without
                                        padding, or 3x3 at stride 2 x 2: operands of 32 image lines per position through
                                        transposing LDS reads, gradient operands in a sliding window */
    INT8T_VARIANT_WIDE_SQ128 = 10,   /* forward / backward-data: 128 x 128 tiles from a 3-stage LDS ring, three blocks per
                                        compute unit: layers that have too few of the larger tiles to go round */
    INT8T_VARIANT_WIDE_SQ128_DEEP = 11,  /* ... with 2 stages of 128 reduction bytes: long reductions */
    INT8T_VARIANT_WIDE_128X64 = 12,      /* ... 128 x 64 tiles with 128-byte stages: few columns (7 x 7 images) */
    INT8T_VARIANT_WIDE_CELLS = 13,       /* backward-data of a layer with stride 2 x 2 and a filter of at least 2 x 2: tiles of 128
                                            rows x 64 cells of 2 x 2 pixels; a block runs the four pixel classes in turn and
                                            writes whole cells */
    INT8T_VARIANT_MAX_ENUM = 0x7fffffff
} int8t_variant;
#define INT8T_VARIANT_COUNT 14
/* 1 when `variant` can run pass `op` (INT8T_OP_CONV_*) of the layer, else 0 (also on a bad descriptor). */
int int8t_conv_variant_ok(int8t_op op, const int8t_conv_desc *desc, int8t_variant variant);
/* INT8T_ERR_ARG when the variant cannot run that pass of that layer; then nothing changes. */
int8t_status int8t_conv_select_variant(int8t_op op, const int8t_conv_desc *desc, int8t_variant variant);
int8t_variant int8t_conv_selected_variant(int8t_op op, const int8t_conv_desc *desc);

/*
 * Kernel timing (measurement aid, not part of the method).  Between int8t_profile_start and
 * int8t_profile_stop every launch of the selected kernel carries a pair of HIP events that take
 * the dispatch's own start and end time stamps on the launch stream.  A timed dispatch costs a few
 * microseconds of idle time before and after it; int8t_profile_start_sampled(kernel, every) times
 * only every `every`-th launch (every >= 1) of each selected kernel, so that a measured loop is
 * disturbed correspondingly less.
 *   kernel   host string: the kernel's name ("dsgc_sweep_kernel", "absmax_kernel",
 *            "absmax_batch_kernel", "quantize_batch_kernel", "quantize_act_kernel", "quantize_planar_kernel", "quantize_wgt_kernel",
 *            "deviation_finish_kernel", "igemm_kernel", "igemm_dma_kernel", "igemm_fused_kernel", "igemm_reduce_kernel",
 *            "band_kernel", "band_reg_kernel", "wgrad_kernel", "wgrad_lines_kernel", "wgrad_reduce_kernel", "s2d_repack_kernel",
 *            "conv_trio_kernel", "quantize_rows_kernel", "quantize_cols_kernel" (both passes), "transpose_codes_kernel", "product_kernel",
 *            "product_reduce_kernel", "few_tokens_kernel", "cache_write_kernel", "cache_read_kernel", "attend_kernel", "attend_join_kernel", "mx4_quantize_kernel" (all passes), "mx4_product_kernel",
 *            "mx4_reduce_kernel", "mx4_few_kernel", "mx4_cache_write_kernel", "mx4_cache_read_kernel", "mx4_attend_kernel", "rotate_kernel", "pages_kernel", "dw_conv_kernel" (every depthwise forward / backward-data variant),
 *            "dw_wgrad_kernel" (every depthwise backward-weight variant), "dw_wgrad_reduce_kernel", "dw_trio_kernel", "infer_1x1_kernel");
 *            "conv_trio_kernel" and "dw_trio_kernel" are all the launches that several passes share: strided layers' and the one that
 *            quantizes depthwise tensors too;
 *            NULL or "" selects every kernel.
 *            An unknown name returns INT8T_ERR_ARG and leaves timing off.
 * int8t_profile_stop waits for the recorded events, writes one entry per kernel that was
 * launched (name: static string owned by the library; launches; summed duration in ms) into
 * out[0..capacity), stores the number of kernels seen in *count (which may exceed capacity) and
 * switches timing off.  Host pointers throughout.  Not thread-safe; event objects are created
 * while timing is on, so keep it off under stream capture.
 */
typedef struct int8t_kernel_time {
    const char *name;
    int launches;
    double total_ms;
} int8t_kernel_time;
int8t_status int8t_profile_start(const char *kernel);
int8t_status int8t_profile_start_sampled(const char *kernel, int every);
int8t_status int8t_profile_stop(int8t_kernel_time *out, int capacity, int *count);

/*
 * Measurement aid: what the int8 matrix cores of the current GPU sustain.  Runs, on every compute
 * unit, eight waves of independent 32x32x32 int8 MFMAs (the wave tile of the wide convolution kernels)
 * for `iters` iterations of 16 MFMAs per wave, with operand bytes all zero (random_operands == 0) or
 * pseudo-random, held in registers (lds_reads == 0) or re-read from LDS before every eight MFMAs as
 * an implicit GEMM does.  Synchronises with the host.
 *   tops_out   host, out: int8 operations per second / 1e12 over the kernel's duration
 *   ghz_out    host, out: the shader clock the loop ran at (shader-clock counter against the constant
 *              100 MHz counter, both read inside the kernel)
 *   ws_dev     64 bytes of device scratch, 8-byte aligned
 * The published peak (5.0 POP/s at 2.4 GHz) is what zero operands reach; with random operands the
 * power limit lowers the clock, and that figure is the ceiling a convolution on real codes has.
 */
int8t_status int8t_profile_mfma_ceiling(int random_operands, int lds_reads, int iters,
                                        double *tops_out, double *ghz_out, void *ws_dev, void *stream);

/* Eq.7 on the host: max(exp(-alpha * d_c), beta).  The paper uses alpha = 20, beta = 0.1. */
double int8t_dclr_scale(double d_c, double alpha, double beta);

/*
 * ---- Tokens: scales per token and output channel, a paged cache, attention over it ---------------------------------------
 * The quantizer of Eq.1 / Eq.3 with c the maximum of a ROW (a token, an output channel) or a COLUMN in place of the tensor's: for the
 * linear layers and the attention of transformers, whose tokens differ in size.  Floating tensors are of an int8t_dtype; a result is
 * formed in fp32 and rounded once.  `pitch` arguments are in elements; rows themselves are contiguous.  Any alignment of an element is
 * served; rows that start on 16 bytes are faster.  fp32 vectors (scales, factors, biases) and codes lie on 16 bytes.
 * A row or column (token, channel, head of a cached token) that holds NaN or an infinity gets codes of 0 and that as its scale, so what is computed from it is NaN:
 * a training program sees the overflow of a gradient in fp16.
 * Codes of `rows` x `cols`: INT8T_ACT codes of dims {rows, cols, 1, 1}, i.e. [rows][cols rounded up to 16], zero beyond cols.
 * Sums of products are exact: at most INT8T_MAX_REDUCTION products (16129 each at most) go into one int32.
 */
typedef enum { INT8T_F32 = 0, INT8T_BF16 = 1, INT8T_F16 = 2, INT8T_DTYPE_MAX_ENUM = 0x7fffffff } int8t_dtype;
#define INT8T_MAX_REDUCTION 131072

/*
 * Codes with a scale for each row: v = x (times factor[col], rounded, where factor_dev is given), c = max|v| of the row,
 * codes as int8t_quantize makes them of v with that c; the draw of an element goes by row * cols + col.
 *   x_dev       rows x cols elements of `type`, rows `pitch` elements apart (pitch >= cols); rows * (cols rounded up to 16) < 2^31,
 *               cols at most 2^31 - 2^15, rows at most 2^26 - 4 (so do linear layers' tokens and weights)
 *   factor_dev  NULL, or cols floats
 *   q_dev       out: codes of rows x cols;   scale_dev  out: rows floats, c / 127
 */
int8t_status int8t_quantize_rows(const void *x_dev, int8t_dtype type, int rows, int cols, size_t pitch, const float *factor_dev,
                                 int8t_round mode, uint64_t seed, int8_t *q_dev, float *scale_dev, void *stream);

/*
 * The same with a scale for each column, the codes transposed: for a reduction over the rows.
 *   factor_dev  NULL, or rows floats
 *   q_dev       out: codes of cols x rows;   scale_dev  out: cols floats
 *   sum_dev     NULL, or out: cols floats, the columns' sums of x (without the factor)
 *   ws_dev      int8t_quantize_cols_workspace_bytes(rows, cols) bytes, 16-byte aligned
 */
size_t int8t_quantize_cols_workspace_bytes(int rows, int cols);
int8t_status int8t_quantize_cols(const void *x_dev, int8t_dtype type, int rows, int cols, size_t pitch, const float *factor_dev,
                                 int8t_round mode, uint64_t seed, int8_t *q_dev, float *scale_dev, float *sum_dev,
                                 void *ws_dev, size_t ws_bytes, void *stream);

/* Codes of rows x cols to codes of cols x rows (both dimensions at most what a reduction may be, or the other way round). */
int8t_status int8t_transpose_codes(const int8_t *q_dev, int rows, int cols, int8_t *qt_dev, void *stream);

/*
 * y[m][n] = (float)(sum_k a[m][k] b[n][k]) * (sa[m] * sb[n]) + bias[n]
 *   a_dev, b_dev   codes of M x K and N x K, zero beyond K
 *   sb_dev, bias_dev   NULL (ones; none), or N floats;   sa_dev  M floats
 *   y_dev          out: M x N of `type`, rows `pitch` apart
 *   ws_dev         NULL, or int8t_product_workspace_bytes(M, N, K) bytes, 16-byte aligned: products with few results split their
 *                  reduction with it (the sums are integers: the result is the same)
 */
size_t int8t_product_workspace_bytes(int M, int N, int K);
int8t_status int8t_product(const int8_t *a_dev, const float *sa_dev, const int8_t *b_dev, const float *sb_dev, int M, int N, int K,
                           const float *bias_dev, void *y_dev, int8t_dtype type, size_t pitch, void *ws_dev, size_t ws_bytes,
                           void *stream);

/*
 * A linear layer of M tokens, y = x W^T + b, with a scale for each token and each output channel.
 *   forward   codes of x and W by rows, nearest;  y as int8t_product
 *   backward  dx[m][k] = sg[m] sum_n gq[m][n] wq[n][k],   gq, sg = stochastic codes by rows of dy[m][n] * sw[n], draws of `seed`
 *             dw[n][k] = sh[n] sum_m hq[m][n] xq[m][k],   hq, sh = stochastic codes by columns of dy[m][n] * sx[m], draws of
 *                                                          `seed` with its highest bit flipped
 *             db[n] = sum_m dy[m][n]
 *             (the scale that changes along the summed axis is in the values before their codes are made)
 * int8t_linear_fwd: w NULL takes the codes at wq, sw (laid out before) as they are; xq NULL keeps no codes of x (nobody's backward
 * pass comes for them).  M may be 0 there.  int8t_linear_bwd: dx, dw, db NULL: not wanted (one of them at least); reads xq, sx
 * (for dw), wq, sw (for dx) of the forward pass.  ws: int8t_linear_workspace_bytes() bytes, 16-byte aligned; may be NULL where that is 0.
 */
typedef struct int8t_linear_desc {
    int M, K, N;
    int8t_dtype type, wtype;       /* of x, y, dy, dx; of w, dw */
} int8t_linear_desc;
typedef struct int8t_linear_buffers {
    const void *x, *w, *dy;
    size_t x_pitch, w_pitch, y_pitch, dy_pitch;
    int8_t *xq, *wq;
    float *sx, *sw;
    const float *bias;
    void *y, *dx, *dw;             /* dx, dw: rows of K elements, dense */
    float *db;
    void *ws;
    size_t ws_bytes;
} int8t_linear_buffers;
/* direction: 0 forward, 1 backward, 2 forward that keeps no codes of x and takes those of W as they are */
size_t int8t_linear_workspace_bytes(const int8t_linear_desc *desc, int direction);
int8t_status int8t_linear_fwd(const int8t_linear_desc *desc, const int8t_linear_buffers *b, void *stream);
int8t_status int8t_linear_bwd(const int8t_linear_desc *desc, const int8t_linear_buffers *b, uint64_t seed, void *stream);

/*
 * A paged cache of keys and values in 8 bits, a scale for each token and head.  Place `slot` is row slot % page_size of page
 * slot / page_size.  dim: a multiple of 16, at most 256; pages * page_size < 2^31 (the cache itself may pass 4 GiB).
 */
typedef struct int8t_cache {
    int8_t *kq, *vq;               /* [pages][heads][page_size][dim] */
    float *ks, *vs;                /* [pages][heads][page_size] */
    int pages, page_size, heads, dim;
} int8t_cache;

/*
 * Writes `tokens` rows of every head to their slots, as Eq.1 codes with the row's own maximum (nearest).  A slot below 0 or beyond the
 * last place: the token is left out.  No two tokens of a call share a slot.
 *   k_dev, v_dev   element (t, h, d) at t * token_pitch + h * head_pitch + d
 *   slots_dev      `tokens` 64-bit integers
 */
int8t_status int8t_cache_write(const int8t_cache *cache, const void *k_dev, const void *v_dev, int8t_dtype type, int tokens,
                               size_t k_token_pitch, size_t k_head_pitch, size_t v_token_pitch, size_t v_head_pitch,
                               const int64_t *slots_dev, void *stream);
/* Reads back: [tokens][heads][dim] of `type`, code times scale; zeros for a slot outside the cache. */
int8t_status int8t_cache_read(const int8t_cache *cache, const int64_t *slots_dev, int tokens, void *k_dev, void *v_dev,
                              int8t_dtype type, void *stream);

/*
 * Attention of new tokens over the cache: token i of request b (of n = starts[b+1] - starts[b] tokens) sees the keys j < lengths[b],
 * causal: j <= lengths[b] - n + i (its own key is in the cache already, and those of the tokens after it may be).  Query head
 * h * group + g goes with head h of the cache.
 *   out = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale * q . k_j), sums in fp32;  zeros where a token sees nothing (its lse: -infinity)
 *   q_dev        element (t, head, d) at t * q_token_pitch + head * q_head_pitch + d
 *   starts_dev   requests + 1 ints, ascending, at most `tokens`; tokens before the first or behind the last are no request's: nothing of theirs is written
 *   lengths_dev  `requests` ints
 *   table_dev    pages of a request in order: [requests][table_width], rows table_pitch apart; entries behind the last page that a length
 *                needs are not used; keys on a page that is not in the cache are not seen; table_width * page_size < 2^31 - 4096
 *   longest      no length is larger (a guide for the division of the work, by which sums are ordered; keys behind it are seen all the same); 0: unknown
 *   out_dev      out: [tokens][heads * group][dim] of `type`, 16-byte aligned
 *   lse_dev      NULL, or out: [tokens][heads * group] floats, the natural logarithm of sum_j p_j
 *   NaN in a query, or in a scale of a key that a token sees, makes that row NaN and no other; places that no row sees, or not yet, may hold anything
 *   ws_dev       int8t_cache_attend_workspace_bytes(cache, desc) bytes, 16-byte aligned; may be NULL where that is 0
 * Products run on fp16 with sums in fp32: codes are exact, each q is scaled by a power of two, and p_j times the value scale is rounded to 11 bits for bf16
 * and fp16 tensors (one fp16) and 22 bits for fp32 ones (two pieces, as q's), with steps of 2^-38 of the row's largest at least: of its own, keys that a row does
 * not see do not matter.  (Value scales below 2^-95 and above 2^103 lose bits.)
 */
typedef struct int8t_attend_desc {
    int tokens, requests, group, table_width, longest;
    int8t_dtype type;
    int causal;
    float scale;
    size_t q_token_pitch, q_head_pitch, table_pitch;
} int8t_attend_desc;
size_t int8t_cache_attend_workspace_bytes(const int8t_cache *cache, const int8t_attend_desc *desc);
int8t_status int8t_cache_attend(const int8t_cache *cache, const int8t_attend_desc *desc, const void *q_dev, const int *starts_dev,
                                const int *lengths_dev, const int *table_dev, void *out_dev, float *lse_dev, void *ws_dev,
                                size_t ws_bytes, void *stream);

/*
 * How a call of these sizes is divided (on the host, nothing is launched): rows of a block -- of its results' columns too, in products --, its waves, stages of
 * operands that it holds in LDS (products), and into how many shares the reduction (the keys) goes.  ws_bytes: as the call will have it.
 */
typedef struct int8t_division {
    int rows, waves, stages, shares;
} int8t_division;
int8t_status int8t_product_division(int M, int N, int K, size_t ws_bytes, int8t_division *out);
int8t_status int8t_cache_attend_division(const int8t_cache *cache, const int8t_attend_desc *desc, int8t_division *out);

/*
 * ---- Microscaled 4-bit tokens ---------------------------------------------------------------------------------------------
 * Codes of four bits: a sign (the highest bit) over 0, .5, 1, 1.5, 2, 3, 4, 6.  A block of 32 values along the axis that a product sums over shares a power of
 * two 2^e, held as the byte e + 127; e is the least integer of [-127, 127] for which the block's largest magnitude is at most 6 * 2^e, so that no value is
 * clipped.  Nearest: ties to the even code.  Stochastic: with a = |v| 2^-e, F = floor(a 2^23) for a < 1 and (the bits of a) - (the bits of 0.5) above counts 2^-22 of
 * a step, and the magnitude's code is (F + u) >> 22 with u the upper 22 of the 24 bits drawn for (seed, row * cols + col): unbiased.
 * A block that holds NaN or an infinity has the byte 255 (NaN) and codes of 0.
 *   codes    [rows][16 * blocks] bytes, blocks = cols / 32 rounded up: value c is the low (c even) or high half of byte c / 2; zero beyond cols
 *   scales   [panels][rows][8] bytes, panels = blocks / 8 rounded up: block b of row r is at ((b / 8) * rows + r) * 8 + b % 8; zero beyond the last block
 * Sums of products are in fp32.  Pointers to codes and scales lie on 16 bytes.
 */

/*
 * Codes of rows x cols values with blocks along the columns (q, s) and, transposed, of cols x rows with blocks along the rows (qt, st), of one matrix.
 *   x_dev         rows x cols elements of `type`, rows `pitch` apart;  rows, cols at most INT8T_MAX_REDUCTION where they are the blocks' axis (the 8-bit
 *                 operators' bound, kept for sizes to be alike: sums here are in fp32 and set none)
 *   q_dev, s_dev  NULL, or out: codes and scales of rows x cols;   draws of `seed`
 *   qt_dev, st_dev   NULL, or out: codes and scales of cols x rows;   draws of `seed` with its highest bit flipped, of the same index
 *   sum_dev       NULL, or out: cols floats, the columns' sums
 *   ws_dev        with sum_dev: int8t_mx4_quantize_workspace_bytes(rows, cols) bytes, 16-byte aligned; else unused
 */
size_t int8t_mx4_quantize_workspace_bytes(int rows, int cols);
int8t_status int8t_mx4_quantize(const void *x_dev, int8t_dtype type, int rows, int cols, size_t pitch, int8t_round mode, uint64_t seed,
                                uint8_t *q_dev, uint8_t *s_dev, uint8_t *qt_dev, uint8_t *st_dev, float *sum_dev, void *ws_dev,
                                size_t ws_bytes, void *stream);

/*
 * y[m][n] = sum_k a[m][k] b[n][k] + bias[n] of what codes and scales of M x K and N x K stand for
 *   bias_dev   NULL, or N floats;   y_dev  out: M x N of `type`, rows `pitch` apart
 *   ws_dev     NULL, or int8t_mx4_product_workspace_bytes(M, N, K) bytes, 16-byte aligned: products with few results split their reduction with it (the order of
 *              the sums goes by M, N, K and whether it is there, nothing else)
 */
size_t int8t_mx4_product_workspace_bytes(int M, int N, int K);
int8t_status int8t_mx4_product(const uint8_t *a_dev, const uint8_t *sa_dev, const uint8_t *b_dev, const uint8_t *sb_dev, int M, int N, int K,
                               const float *bias_dev, void *y_dev, int8t_dtype type, size_t pitch, void *ws_dev, size_t ws_bytes,
                               void *stream);

/*
 * A linear layer of M tokens, y = x W^T + b: every product's operands have their blocks along its summed axis.
 *   forward   y  = Q(x) Q(W)^T + b           blocks along K, nearest
 *   backward  dx = S(dy) Q'(W)               blocks along N;  S: stochastic, draws of `seed`
 *             dw = S'(dy)^T Q'(x)            blocks along M;  S': draws of `seed` with its highest bit flipped
 *             db = sum_m dy[m]
 * int8t_mx4_linear_fwd: w NULL takes wq, sw (codes of N x K, laid out before).  With w: they are written where given (else in scratch), and so are wt, swt (codes
 * of K x N, for dx).  xt, sxt: codes of K x M of x, for dw; NULL: not kept.  M may be 0.
 * int8t_mx4_linear_bwd: dx, dw, db NULL: not wanted (one of them at least); dx reads wt, swt, dw reads xt, sxt of the forward pass.
 * ws: int8t_mx4_linear_workspace_bytes() bytes, 16-byte aligned; may be NULL where that is 0.
 */
typedef struct int8t_mx4_linear_buffers {
    const void *x, *w, *dy;
    size_t x_pitch, w_pitch, y_pitch, dy_pitch;
    uint8_t *wq, *sw, *wt, *swt, *xt, *sxt;
    const float *bias;
    void *y, *dx, *dw;             /* dx, dw: rows of K elements, dense */
    float *db;
    void *ws;
    size_t ws_bytes;
} int8t_mx4_linear_buffers;
/* direction: 0 forward, 1 backward, 2 forward with w and xt NULL */
size_t int8t_mx4_linear_workspace_bytes(const int8t_linear_desc *desc, int direction);
int8t_status int8t_mx4_linear_fwd(const int8t_linear_desc *desc, const int8t_mx4_linear_buffers *b, void *stream);
int8t_status int8t_mx4_linear_bwd(const int8t_linear_desc *desc, const int8t_mx4_linear_buffers *b, uint64_t seed, void *stream);

/*
 * A paged cache of keys and values in these codes, blocks along a head's dims: places, slots and limits as int8t_cache.  dim: a multiple of 16, at most 256.
 * int8t_mx4_cache_write, _read, _attend: as int8t_cache_write, _read, _attend with k, v what codes and scales stand for.
 * attend: blocks with the byte 0 (below 2^-124) may count as zeros;  q . k_j exact products in fp32 sums (blocks of 16 rows; larger ones as the 8-bit cache's, with fp16 codes
 * relative to the largest scale of a key's row: blocks 2^36 below it lose bits, but keys of bf16 tensors, whose products stay exact); p_j is rounded to 16 bits for bf16 and fp16
 * tensors and 24 for fp32 ones, and held down to 2^-126 of the row's largest (value scales beyond 2^96 shorten that by up to as much); in larger blocks to 11 and 22, with
 * steps as the 8-bit cache's (value scales below 2^-82 and above 2^116 lose bits).  A key or value with a block of scale 255 (values, in blocks of 16 rows: 253 and more, whose products pass
 * fp32) makes the rows that see it, with a p_j above zero in fp32, NaN, all of their dims, and no others.
 */
typedef struct int8t_mx4_cache {
    uint8_t *kq, *vq;              /* [pages][heads][page_size][16 * blocks], blocks = dim / 32 rounded up */
    uint8_t *ks, *vs;              /* [pages][heads][page_size][blocks] */
    int pages, page_size, heads, dim;
} int8t_mx4_cache;
int8t_status int8t_mx4_cache_write(const int8t_mx4_cache *cache, const void *k_dev, const void *v_dev, int8t_dtype type, int tokens,
                                   size_t k_token_pitch, size_t k_head_pitch, size_t v_token_pitch, size_t v_head_pitch,
                                   const int64_t *slots_dev, void *stream);
int8t_status int8t_mx4_cache_read(const int8t_mx4_cache *cache, const int64_t *slots_dev, int tokens, void *k_dev, void *v_dev,
                                  int8t_dtype type, void *stream);
size_t int8t_mx4_cache_attend_workspace_bytes(const int8t_mx4_cache *cache, const int8t_attend_desc *desc);
int8t_status int8t_mx4_cache_attend(const int8t_mx4_cache *cache, const int8t_attend_desc *desc, const void *q_dev, const int *starts_dev,
                                    const int *lengths_dev, const int *table_dev, void *out_dev, float *lse_dev, void *ws_dev,
                                    size_t ws_bytes, void *stream);

int8t_status int8t_mx4_product_division(int M, int N, int K, size_t ws_bytes, int8t_division *out);
int8t_status int8t_mx4_cache_attend_division(const int8t_mx4_cache *cache, const int8t_attend_desc *desc, int8t_division *out);

/*
 * ---- Positions -------------------------------------------------------------------------------------------------------------
 * Rotary positions: pair i of a head's first `rot` values, (a, b), of a token at position p becomes
 *   amplitude * (a cos t - b sin t, a sin t + b cos t),   t = 2 pi p turns[i],
 * and with back = 1 the same with -t (the gradient: of the result's gradient the argument's).  Pairs are values (i, i + rot / 2), or (2 i, 2 i + 1) with interleaved = 1.
 * Values from `rot` on are copied.  p turns[i] is formed in 64 bits; results in fp32, rounded once.
 *   x, y            element (token, head, d) at token * token_pitch + head * head_pitch + d;  y may be x (the same pitches then), and overlaps it in no other way
 *   second          heads of a second tensor of the same tokens (keys beside queries), 0: none
 *   positions_dev   tokens ints;   turns_dev  rot / 2 doubles
 */
typedef struct int8t_rotate_tensor {
    const void *x;
    void *y;
    size_t x_token_pitch, x_head_pitch, y_token_pitch, y_head_pitch;
    int heads;
} int8t_rotate_tensor;
typedef struct int8t_rotate_desc {
    int tokens, dim, rot;
    int8t_dtype type;
    int interleaved, back;
    float amplitude;
} int8t_rotate_desc;
int8t_status int8t_rotate(const int8t_rotate_desc *desc, const int8t_rotate_tensor *first, const int8t_rotate_tensor *second,
                          const int *positions_dev, const double *turns_dev, void *stream);

/*
 * Pages of the new tokens of a batch, found on the GPU: what int8t_cache_write (slots), int8t_rotate (positions) and int8t_cache_attend (starts, lengths, table) take.
 * Request b has have[b] tokens on the first have[b] / page_size (rounded up) pages of table[b], and add[b] new ones (below 0: none).  Free pages are a stack,
 * free[0 .. available - 1], taken from its end in the order of the requests and of their pages.  A request gets no pages where its tokens end behind `tokens`, where its
 * row of the table is too short, or where the pages that it and all before it need are more than there are: its new tokens have no slots, its length stays.
 *   table_dev      [requests][width], rows table_pitch apart; entries of new pages are written
 *   lengths_dev    out: requests ints, have + add, or have where there were no pages
 *   left_dev       out: 1 int, pages that are still free
 *   starts_dev     out: requests + 1 ints, sums of the new tokens
 *   slots_dev      out: `tokens` 64-bit integers, page * page_size + row; -1: no place, or behind the last request's tokens
 *   positions_dev  out: `tokens` ints, 0 without a place
 *   without_dev    out: 1 int, requests that got none (without a new token too, where its length is beyond its table's row)
 * No output is an input (but table).  width * page_size < 2^31.  `pages`: the length of free.
 */
typedef struct int8t_pages_desc {
    int requests, width, page_size, pages, tokens;
    size_t table_pitch;
} int8t_pages_desc;
int8t_status int8t_pages_extend(const int8t_pages_desc *desc, const int *have_dev, const int *add_dev, int *table_dev, const int *free_dev,
                                const int *available_dev, int *lengths_dev, int *left_dev, int *starts_dev, int64_t *slots_dev,
                                int *positions_dev, int *without_dev, void *stream);
/*
 * Only the first stay[b] tokens of each request stay (0: it has ended; more than it has: all): lengths_dev, in and out; pages behind them go back onto the stack free_dev,
 * in the order of the requests, and available_dev, in and out, counts them.  `tokens` of the descriptor is not used.
 */
int8t_status int8t_pages_shrink(const int8t_pages_desc *desc, const int *stay_dev, int *lengths_dev, const int *table_dev, int *free_dev,
                                int *available_dev, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* INT8T_H */
