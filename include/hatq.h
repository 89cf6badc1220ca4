/*
 * hatq.h -- C ABI of the MI355X (gfx950) Hadamard-domain INT8 linear operator.
 *
 * The operator is the inference-time layer of HaTQ ("Hadamard-Domain Model
 * Quantization for Learned Image Coding"): a convolution or fully connected
 * layer Y = X W^T + b (Eq. supp_linear_operator) evaluated with INT8 operands in
 * a Hadamard domain, in one of two per-layer forms (Sec. IV-B):
 *
 *   DH (double-Hadamard, Eq. double_hadamard_quantization): activations and
 *      weights are both transformed along the contracted input channels,
 *      Y = Q(X T_in) Q(W T_in)^T.
 *   WH (weight-only Hadamard, Eq. weight_only_hadamard_quantization): weights
 *      are transformed along output channels, activations are quantized in the
 *      original domain, and the accumulator is mapped back,
 *      Y = [Q(X) Q(T_out^T W)^T + b~] T_out^T   (Eq. supp_padded_wh).
 *
 * Transforms are block diagonal, B_C = I_{C/b} (x) H~_b, with H~_b the
 * unnormalized Sylvester matrix of order b (Eq. supp_sylvester, natural order).
 * The normalization 1/sqrt(b) of each side is folded into the dequantization
 * scale as one exact factor 1/b (Supplementary, "Deployment Realization").
 *
 * Quantization is symmetric INT8 with codes in [-127, 127] (Eq. symmetric_q):
 * per-sample dynamic activation scale s_x = ||S||_inf / 127 (Eq. current_scale)
 * and per-output-channel weight scale; rounding is round-half-to-even and x/s is
 * an IEEE fp32 division.  The INT8 x INT8 products accumulate in INT32
 * (Eq. integer_accumulation); the accumulator of channel c has scale
 * s_x * s_w,c (Eq. accumulator_scale).
 *
 * Conventions for every entry point:
 *  - Tensors are NHWC, row-major, densely packed.  All tensor pointers are
 *    DEVICE pointers owned by the caller (hatq_export_weights also takes host
 *    destinations); the library never allocates, frees or synchronizes, and
 *    keeps no global state.  Calls are reentrant; calls on one stream execute
 *    in order.
 *  - `stream` is a hipStream_t (NULL = the default stream).  Some launch
 *    shapes (the persistent convolution grids) follow the CU count of the
 *    current device; results do not depend on them.
 *  - Arguments are validated on the host before any launch.  On error nothing
 *    is launched and outputs are untouched.  A launch failure is reported as
 *    HATQ_EHIP; faults inside kernels surface at the caller's next
 *    synchronization.  Nothing is printed and no C++ exception crosses the ABI.
 *  - Unless noted, no entry point reads device memory on the host.
 */
#ifndef HATQ_H
#define HATQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    HATQ_OK = 0,
    HATQ_EINVAL = 1,        /* bad argument: null pointer, bad size, form mismatch */
    HATQ_EUNSUPPORTED = 2,  /* valid operator outside the kernels' supported geometry */
    HATQ_EWORKSPACE = 3,    /* caller-provided buffer too small */
    HATQ_EHIP = 4           /* a HIP launch or runtime call failed */
} hatq_status;

typedef enum { HATQ_DH = 0, HATQ_WH = 1 } hatq_form;

typedef enum {
    HATQ_OUT_I32 = 0,       /* raw INT32 accumulators [n][ho][wo][cout_pad], no bias;
                               WH accumulators stay in the output Hadamard basis */
    HATQ_OUT_F32 = 1,       /* dequantized fp32 output [n][ho][wo][cout], original basis */
    HATQ_OUT_I8 = 2         /* the next operand's INT8 codes [n][ho][wo][cout] (requantization,
                               Eq. integer_requantization) */
} hatq_out_mode;

/* Flags of the convolution entry points (bitwise or; 0 = none).
 *   HATQ_PAIRED: a WH layer whose next operand uses the same transform blocks
 *     (next_hblock == hblock > 1) with nothing applied between the layers
 *     (identity nonlinearity) may take the next operand through the cancellation
 *     of Table I: B_next y = B_next (B_Cout z) / b = z, z the dequantized
 *     accumulators before the output restore (Sylvester blocks square to b I).
 *     Neither butterfly then runs: the next operand's absmax is max|z|, its
 *     codes are those of z, and the integer transition uses B_next B_Cout = b I.
 *     Without the flag both transforms run explicitly (the general Table I
 *     transition, which a nonlinearity between the layers needs).  Ignored for
 *     every other layer and output. */
/*   HATQ_XQ_C64: the input codes xq are in the chunk-major layout
 *     [n][cin_pad/64][h][w][64] (64-channel planes) instead of [n][h][w][cin_pad],
 *     as hatq_fwht_quant_act_c64 and HATQ_YQ_C64 write them.  Same codes, same
 *     results; the window refills of the 5x5 stride-2 kernel then read whole
 *     128-byte lines (Eq. linear_operator: the contraction is unchanged, only
 *     where each code sits).  Supported for regular (not transposed) 5x5 stride-2
 *     layers with cin_pad % 64 == 0 and cout_pad 192 or 320, except a call
 *     whose epilogue transforms by the order 320 (a WH restore of order 320 or
 *     next_hblock 320 with a float or code output); HATQ_EUNSUPPORTED
 *     otherwise.
 *   HATQ_YQ_C64: code outputs (HATQ_OUT_I8, hatq_conv_int8_requant,
 *     hatq_conv_int8_int_transition) go out chunk-major,
 *     [n][cout/64][ho][wo][64]; needs cout % 64 == 0 (HATQ_EUNSUPPORTED
 *     otherwise), HATQ_EINVAL for F32 and I32 outputs. */
typedef enum { HATQ_PAIRED = 1, HATQ_XQ_C64 = 2, HATQ_YQ_C64 = 4 } hatq_conv_flags;

/* One layer's geometry.  Square kernels only.
 *   conv:        ho = (h + 2*pad - k)/stride + 1
 *   transposed:  ho = (h - 1)*stride - 2*pad + k + out_pad
 * hblock: block order b of the transform B = I (x) H_b; it acts on cin for DH
 * and on cout for WH.  b = 1 means no transform.  A power of two in [1, 128]
 * (Sylvester H~_b), or one of the orders m(C) of Eq. hadamard_order that the
 * Sylvester family lacks, built as Kronecker products with a Paley-I factor
 * (supplementary, Hadamard construction): 192 = P_12 (x) H~_16 and
 * 320 = P_20 (x) H~_16, index a*16 + l (Paley index a, Sylvester index l).
 * Those two are supported for DH layers in hatq_fwht_quant_act,
 * hatq_prepare_weights, hatq_conv_int8 and hatq_layer_forward (the DH
 * dequantization factor is fl(s_x s_w / b)), and by the activation-side
 * profiling and affine entry points (hatq_range_expansion,
 * hatq_fwht_quant_act_affine) for whole blocks (c % b == 0); the entry points
 * below that say so take them also for the convolution epilogues (192 with
 * cout_pad 192, 320 with cout_pad 320 and cin_pad % 64 == 0). */
typedef struct {
    int32_t cin, cout;
    int32_t k;
    int32_t stride, pad, out_pad;
    int32_t transposed;     /* 0: convolution, 1: transposed convolution */
    int32_t hblock;
} hatq_conv_desc;

/* Prepared weights: a plain view into the caller's device buffer, filled by
 * hatq_prepare_weights.  Layout of wq: [cout_pad][k_stride] int8, row co holds
 * the contraction index d = (kh*k + kw)*cin_pad + ci (the Kronecker order
 * I_{KhKw} (x) H of Eq. input_hadamard_transform); bytes d >= k_total are 0.
 * For a transposed convolution (kh, kw) index the kernel as stored in PyTorch
 * (weight[ci][co][kh][kw]).  w_scale and bias are fp32 [cout_pad]; for WH the
 * bias is the transformed b~ = B_Cout [b; 0] (Eq. supp_padded_wh_parameters).
 * wpack holds the same codes again in the order the convolution kernels stream
 * them (K-blocked: [pack_stride/64][cout_pad][64], contiguous per 64-deep
 * contraction step); it is library-internal and callers must not depend on
 * its order.  hatq_prepare_weights fills both copies. */
typedef struct {
    hatq_conv_desc d;
    int32_t form;           /* hatq_form, fixed for the layer's lifetime (Sec. IV-C) */
    int32_t cin_pad;        /* cin (DH: rounded up to hblock) */
    int32_t cout_pad;       /* cout (WH: rounded up to hblock) */
    int32_t k_total;        /* k*k*cin_pad */
    int32_t k_stride;       /* k_total rounded up to 64 */
    int8_t *wq;
    float *w_scale;
    float *bias;
    int8_t *wpack;          /* kernel-order copy of wq (see above) */
    int32_t pack_stride;    /* contraction bytes per output channel in wpack */
} hatq_weights;

/* Static description of a status code.  Never NULL. */
const char *hatq_status_string(int32_t status);

/* Output spatial size of `d` for an input of h x w.  HATQ_EINVAL if the result
 * would be empty. Host only. */
int32_t hatq_conv_out_hw(const hatq_conv_desc *d, int32_t h, int32_t w, int32_t *ho, int32_t *wo);

/* Bytes of device memory hatq_prepare_weights needs for `d` in form `form`
 * (0 for an invalid descriptor). */
size_t hatq_weights_bytes(const hatq_conv_desc *d, int32_t form);

/* Offline weight preparation (Eq. hadamard_linear_equivalence and
 * Eq. weight_only_hadamard_equivalence with the padded forms of the
 * supplementary; per-channel symmetric quantization, Eq. symmetric_q).
 *   w:    device fp32 weights in PyTorch layout, OIHW [cout][cin][k][k] for a
 *         convolution, IOHW [cin][cout][k][k] for a transposed convolution.
 *   bias: device fp32 [cout], or NULL for no bias.
 *   dst:  device buffer of at least hatq_weights_bytes(d, form) bytes; it holds
 *         wq, w_scale and bias afterwards.  `out` (host struct) receives the
 *         view into it.
 * The transform is evaluated in fp64 and rounded once to fp32; then
 * s_w,c = fl32(max|W'_c| / 127) (1 for an all-zero row) and
 * wq = clamp(rne(fl32(W'/s_w,c)), -127, 127).  Runs on `stream`.
 * Supported: DH needs cin % hblock == 0, WH needs cout % hblock == 0. */
int32_t hatq_prepare_weights(const hatq_conv_desc *d, int32_t form, const float *w,
                             const float *bias, void *dst, size_t dst_bytes,
                             hatq_weights *out, void *stream);

/* Copy prepared weights out in their documented layout (Eq. hadamard_linear_equivalence
 * and Eq. weight_only_hadamard_equivalence: the transformed, quantized operator):
 *   wq:      int8 [cout_pad][k][k][cin_pad], the codes of W' (row co holds
 *            d = (kh*k + kw)*cin_pad + ci, as W->wq without its zero K padding);
 *   w_scale: fp32 [cout_pad], s_w,c;  bias: fp32 [cout_pad] (WH: b~ = B_Cout [b; 0]).
 * Destinations may be host or device memory (any of them NULL to skip it); the
 * copies are enqueued on `stream` and host destinations hold the data once the
 * caller has synchronized the stream (with pageable host memory the HIP runtime
 * may complete the copy before returning). */
int32_t hatq_export_weights(const hatq_weights *W, int8_t *wq, float *w_scale, float *bias, void *stream);

/* Rebuild W->wpack from the codes in W->wq, for callers that write codes into
 * wq themselves (codes quantized elsewhere, e.g. loaded from a deployment
 * checkpoint, with w_scale and bias filled to match).  W must be a view returned
 * by hatq_prepare_weights (same geometry); wq bytes past k_total must be 0.
 * Runs on `stream`. */
int32_t hatq_pack_weights(const hatq_weights *W, void *stream);

/* Workspace bytes hatq_fwht_quant_act needs for a batch of n samples. */
size_t hatq_fwht_quant_ws_bytes(int32_t n);

/* Activation transform and quantization, steps a2-a4 of one layer
 * (Eq. input_hadamard_transform, Eq. symmetric_q, Eq. current_scale):
 *   S[p] = B_c x[p] along channels (hblock = 1: S = x),
 *   s_x[i] = fl32(max |S over sample i| / 127)  (1 if that max is 0),
 *   xq = clamp(rne(fl32(S / s_x[i])), -127, 127).
 *   x:        device fp32 [n][h][w][c].
 *   absmax:   NULL, or device fp32 [n] holding max |S| per sample already (as
 *             produced by hatq_conv_int8's next_absmax); then the input is read
 *             once instead of twice.
 *   xq:       device int8 [n][h][w][c].
 *   act_scale: device fp32 [n], receives s_x (unnormalized-domain scale).
 *   ws:       device workspace of hatq_fwht_quant_ws_bytes(n) bytes (unused
 *             when absmax is given).
 * Supported: c % hblock == 0, and c % 4 == 0 or hblock == 1; for the Kronecker
 * orders 192 and 320, h*w*c % 4 == 0. */
int32_t hatq_fwht_quant_act(const float *x, int32_t n, int32_t h, int32_t w, int32_t c,
                            int32_t hblock, const float *absmax, int8_t *xq, float *act_scale,
                            void *ws, size_t ws_bytes, void *stream);

/* hatq_fwht_quant_act with the codes in the chunk-major layout of HATQ_XQ_C64:
 *   xq: device int8 [n][c/64][h][w][64], 16-byte aligned; the code of channel
 *       64m + j of pixel p at ((i*(c/64) + m)*h*w + p)*64 + j for sample i.
 * Same codes and scales as hatq_fwht_quant_act.  Supported: c % 64 == 0 and
 * hblock a power of two at most 64 (HATQ_EUNSUPPORTED otherwise). */
int32_t hatq_fwht_quant_act_c64(const float *x, int32_t n, int32_t h, int32_t w, int32_t c,
                                int32_t hblock, const float *absmax, int8_t *xq, float *act_scale,
                                void *ws, size_t ws_bytes, void *stream);

/* hatq_fwht_quant_act without a workspace, for callers that cannot allocate
 * device memory (code under HIP graph capture, tight serving loops, harnesses
 * that forbid allocation): the two-pass form (absmax, then codes) keeps the
 * per-sample absmax in a static array inside the library, one copy per GPU,
 * of HATQ_NOALLOC_MAX_SAMPLES x 32 floats (512 KB: the per-block maxima of a
 * sample spread over 32 slots), held until the process ends.
 * Arguments, results and support as hatq_fwht_quant_act with absmax = NULL;
 * n > HATQ_NOALLOC_MAX_SAMPLES returns HATQ_EUNSUPPORTED.  Allocates nothing.
 * Every call on one GPU shares that GPU's array (it is cleared by the call
 * itself on the stream), so calls that overlap on one GPU (on different
 * streams, or from several threads) race and must not be issued. */
#define HATQ_NOALLOC_MAX_SAMPLES 4096
int32_t hatq_fwht_quant_act_noalloc(const float *x, int32_t n, int32_t h, int32_t w, int32_t c, int32_t hblock,
                                    int8_t *xq, float *act_scale, void *stream);

/* INT8 convolution with INT32 accumulation and the fused epilogue, steps a5-a6
 * (Eq. integer_accumulation, Eq. accumulator_scale, Table I).
 *   xq:        device int8 [n][h][w][cin_pad] (codes from hatq_fwht_quant_act).
 *   act_scale: device fp32 [n].
 *   mode HATQ_OUT_I32: y is int32 [n][ho][wo][cout_pad], raw accumulators.
 *   mode HATQ_OUT_F32: y is fp32 [n][ho][wo][cout]:
 *     DH: y = fma(float(acc), fl(s_x*s_w,c) * (1/b), bias_c);
 *     WH: z_c = fma(float(acc), fl(s_x*s_w,c), b~_c) (scale before the basis
 *         change, Supplementary "General Nonlinearities"), y = (B_Cout z)/b,
 *         truncated to cout.
 *   mode HATQ_OUT_I8: y is int8 [n][ho][wo][cout], the next layer's codes
 *     clamp(rne(fl32(y' / s))), y' = B_next y with blocks of next_hblock (1: y'
 *     = y) and s = out_scale[n], a static per-sample scale (Eq.
 *     integer_requantization); exactly hatq_conv_int8_requant with that static
 *     scale.  y (fp32) itself is never written.
 *   out_scale: device fp32 [n], required in I8 mode, NULL otherwise.
 *   next_hblock / next_absmax (F32 mode only): if next_absmax is non-NULL it
 *     receives, per sample, max |B_{next} y| with block size next_hblock (1: max
 *     |y|), the exact value hatq_fwht_quant_act would compute from y; the next
 *     layer can then quantize y reading it once.  It is overwritten, not
 *     accumulated.  y may be NULL in F32 mode when next_absmax is given: the
 *     call then only produces next_absmax (the first pass of
 *     hatq_conv_int8_requant's dynamic scale).  With HATQ_PAIRED (see above)
 *     a WH layer whose block equals next_hblock takes max |z| instead.
 *   next_hblock (I8 mode): the next operand's transform block.
 *   flags:     HATQ_PAIRED, HATQ_XQ_C64, HATQ_YQ_C64 (I8 mode only), or 0.
 * Supported: cin_pad % 64 == 0 with k <= 8, or cin_pad <= 4 with k*k*cin_pad <= 128;
 * cout_pad % 64 == 0; WH block and next_hblock a power of two at most 64, or
 * a Kronecker order equal to cout_pad: 192 (P_12 (x) H~_16), or 320
 * (P_20 (x) H~_16) when cin_pad % 64 == 0 (applied as H~_16 then the Paley
 * factor; the WH restore multiplies by B^T), or 128 with cout_pad 128 or 256
 * (with cin_pad <= 4 only for the row-run geometry: k <= 8, stride <= 2,
 * k*cin_pad <= 16, not transposed) (I8: as hatq_conv_int8_requant).  Transposed: stride 2.  xq and y (F32, I32) must be
 * 16-byte aligned, y in I8 mode 4-byte aligned. */
int32_t hatq_conv_int8(const hatq_weights *W, const int8_t *xq, const float *act_scale,
                       int32_t n, int32_t h, int32_t w, int32_t out_mode, const float *out_scale, void *y,
                       int32_t next_hblock, float *next_absmax, int32_t flags, void *stream);

/* INT8 convolution with the requantizing epilogue (step a6, I8 output; Eq.
 * integer_requantization with the dynamic per-tensor scale of Eq. symmetric_q):
 * the layer's fp32 output y (as hatq_conv_int8 computes it in F32 mode) is
 * transformed for the next layer, y' = B_next y with blocks of next_hblock (1:
 * y' = y, the WH input case), and quantized in registers,
 *   yq = clamp(rne(fl(y' / s)), -127, 127),
 * exactly as hatq_fwht_quant_act(y, ..., next_hblock, absmax = next_absmax)
 * would from y (the same fp32 butterflies in the same order, the same
 * rounding); y itself is never written.  With HATQ_PAIRED a WH layer whose
 * block equals next_hblock quantizes z instead (B_next y = z in exact
 * arithmetic, Table I): the codes are those of z, and can differ from the
 * explicit path's by the rounding of its two fp32 butterflies.
 *   next_absmax: device fp32 [n] with max |B_next y| per sample (from an
 *     earlier hatq_conv_int8 call with y = NULL, or an upper bound of it); the
 *     scale is then s = fl32(next_absmax / 127) (1 if it is 0) and is written to
 *     next_scale.  NULL: next_scale [n] is an input, a static scale.
 *   next_scale: device fp32 [n], the next layer's act_scale.
 *   yq:        device int8 [n][ho][wo][cout], the next layer's xq (with
 *              HATQ_YQ_C64: [n][cout/64][ho][wo][64]).
 *   flags:     HATQ_PAIRED, HATQ_XQ_C64, HATQ_YQ_C64, or 0.
 * Supported: as hatq_conv_int8, with cout % 4 == 0 and cout % next_hblock == 0. */
int32_t hatq_conv_int8_requant(const hatq_weights *W, const int8_t *xq, const float *act_scale,
                               int32_t n, int32_t h, int32_t w, int32_t next_hblock,
                               const float *next_absmax, float *next_scale, int8_t *yq,
                               int32_t flags, void *stream);

/* Affine activation quantization (Eq. affine_q, Eq. uniform_q), the dynamic
 * per-sample form of the paper's PTQ setting, on the signed grid [-128, 127]
 * (the paper's unsigned grid shifted by -128: the same dequantized values, codes
 * that the signed INT8 product takes).  For S = the activation transform of
 * each sample (as hatq_fwht_quant_act): with lo = max(-min S, 0), hi = max(max
 * S, 0), r = fl32(hi + lo):
 *   s = fl32(r / 255), z = clamp(rne(fl32(lo / s)) - 128, -128, 127); r = 0 gives
 *   s = 1, z = 0;  xq = clamp(rne(fl32(S / s)) + z, -128, 127).
 *   act_scale, act_zero: device fp32 / int32 [n], written.
 *   ws: device workspace of hatq_fwht_quant_affine_ws_bytes(n) bytes.
 * hblock: a power of two <= 128 or a Kronecker order (192, 320).
 * Supported: c % hblock == 0, h*w*c % 4 == 0, n <= 65535. */
size_t hatq_fwht_quant_affine_ws_bytes(int32_t n);
int32_t hatq_fwht_quant_act_affine(const float *x, int32_t n, int32_t h, int32_t w, int32_t c, int32_t hblock,
                                   int8_t *xq, float *act_scale, int32_t *act_zero, void *ws, size_t ws_bytes,
                                   void *stream);

/* Weight sums for the zero-point correction: tapsum[t][c] = sum over ci of the
 * code W_q[c][t][ci] for each tap t < k*k, then tapsum[k*k][c] = their total.
 * hatq_tapsum_len gives the int32 entries ((k*k + 1) * cout_pad, 0 for invalid
 * weights); tapsum is device memory, 16-byte aligned, written on the stream. */
size_t hatq_tapsum_len(const hatq_weights *W);
int32_t hatq_weight_tapsums(const hatq_weights *W, int32_t *tapsum, void *stream);

/* INT8 convolution of affine codes (Eq. integer_accumulation with zero points
 * z_x per sample and z_w = 0): the accumulator is the sum of (x - z_x) w over
 * the input pixels inside the image (padding is the value zero), formed as the
 * sum of x w minus z_x times the weight sum of the pixel's inside taps; then
 * the same output modes as hatq_conv_int8 (HATQ_OUT_I32: these centered
 * accumulators; HATQ_OUT_F32: the same epilogue with s_x = act_scale).
 *   act_zero: device int32 [n] (from hatq_fwht_quant_act_affine).
 *   tapsum:   from hatq_weight_tapsums for W.
 * Supported: as hatq_conv_int8 (no next-operand absmax; not a WH layer of
 * block 128). */
int32_t hatq_conv_int8_affine(const hatq_weights *W, const int8_t *xq, const float *act_scale,
                              const int32_t *act_zero, const int32_t *tapsum, int32_t n, int32_t h, int32_t w,
                              int32_t out_mode, void *y, void *stream);

/* Integer-only transition (Eq. integer_accumulation, Eq.
 * integer_fixed_point_scale, Eq. integer_hadamard_transition, the integer
 * column of Table I) with static per-tensor scales: the layer's INT32
 * accumulators become the next layer's INT8 codes with no floating point.
 *
 * hatq_int_table_len: int32 entries of the parameter table of W (2*cout_pad + 1),
 * 0 for invalid weights.
 *
 * hatq_int_transition_params: calibration step, fills the table on the device.
 *   s_x:   the static scale of W's input codes (unnormalized domain).
 *   s_y:   the static scale of the next operand's codes.
 *   next_hblock: the next operand's transform block (1: none), a power of two
 *          <= 64, 192 or 320 (not 128, and W not a WH layer of block 128:
 *          HATQ_EUNSUPPORTED); the overflow bound depends on it, so the table serves
 *          only calls with this next_hblock.
 *   table: device int32 [2*cout_pad + 1], 16-byte aligned, written as
 *     M[c]         = rne(2^n rho_c), rho_c = u_c / (beta_out s_y),
 *     b_int[c]     = rne(b_c / u_c),  u_c = s_x s_w,c / beta_in,
 *     table[2*cout_pad] = n,
 *   with (beta_in, beta_out) = (hblock, 1) for DH and (1, hblock) for WH (one
 *   accumulator step is worth u_c; the WH output transform divides by its
 *   block), b the prepared bias (WH: in the output basis) and n the largest
 *   shift in [0, 62] with every M_c <= floor(2^62 / (A_max G)) and < 2^31,
 *   A_max = k*k*cin_pad*127^2 + max|b_int|, G = (WH: hblock) * next_hblock:
 *   every int64 sum of the transition is then exact.  fp64 arithmetic with
 *   correctly rounded division.
 *   Enqueued on `stream` like every other call (it does not wait): when no
 *   shift fits (or |b_int| >= 2^30) the table holds n = -1 and every M_c = 0,
 *   which the caller reads back after its own synchronization; a transition
 *   with such a table writes all-zero codes.
 *
 * hatq_conv_int8_int_transition: convolution plus the integer epilogue,
 *   p = M (.) (acc + b_int) in int64, v = B_Cout^T p (WH; truncated to cout),
 *   w = B_next v (blocks of next_hblock), yq = clamp(rne(w / 2^n), -127, 127)
 *   with rne rounding exact halves to even; no act_scale (it is inside M).
 *   table: as written by hatq_int_transition_params for W and next_hblock.
 *   yq:    device int8 [n][ho][wo][cout], the next layer's codes.
 *   flags: HATQ_PAIRED (a WH layer whose block equals next_hblock then uses
 *          B_next B_Cout = b I: bit-identical codes, no butterflies),
 *          HATQ_XQ_C64, HATQ_YQ_C64, or 0.
 *   Supported: as hatq_conv_int8_requant. */
size_t hatq_int_table_len(const hatq_weights *W);
int32_t hatq_int_transition_params(const hatq_weights *W, float s_x, float s_y, int32_t next_hblock,
                                   int32_t *table, void *stream);
int32_t hatq_conv_int8_int_transition(const hatq_weights *W, const int8_t *xq, int32_t n, int32_t h,
                                      int32_t w, int32_t next_hblock, const int32_t *table,
                                      int8_t *yq, int32_t flags, void *stream);

/* Range-expansion profiling (Eq. hadamard_sensitivity): for each sample k of
 * a layer's input x, whether the layer's input-side transform enlarges the
 * range, ||H x_k||_inf > ||x_k||_inf with H = B_C / sqrt(hblock) orthonormal
 * (B_C the block-diagonal Sylvester transform, channels zero-padded to a
 * multiple of hblock).  Decided exactly as max|S|^2 > hblock * max|x|^2 in
 * fp64, S the fp32 butterfly transform hatq_fwht_quant_act applies.
 *   x:      device fp32 [n][h][w][c], 16-byte aligned; n <= 65535.
 *   hblock: a supported order (1: no transform, never an expansion); the
 *           Kronecker orders 192 and 320 need c % hblock == 0 and h*w*c % 4 == 0.
 *   amax:   device fp32 [2n], written: max|x_k| at [k], max|S_k| at [n + k].
 *   flags:  NULL, or device int32 [n] receiving 1 (expands) or 0.
 *   count:  NULL, or device int32 [1] to which the number of expanding samples
 *           is added (not overwritten: calls over the batches of a profiling
 *           set accumulate).
 * The probability p_l is *count / images over the profiling set. */
int32_t hatq_range_expansion(const float *x, int32_t n, int32_t h, int32_t w, int32_t c, int32_t hblock,
                             float *amax, int32_t *flags, int32_t *count, void *stream);

/* Form rule (Eq. layerwise_hadamard_selection): *form = HATQ_WH if
 * p = expansions / images (correctly rounded fp64) exceeds tau, else HATQ_DH.
 * HATQ_EINVAL for images <= 0, expansions outside [0, images] or a non-finite
 * tau.  Host only. */
int32_t hatq_select_form(int64_t expansions, int64_t images, double tau, int32_t *form);

/* Transform order rule (Eq. hadamard_order with the supplementary Hadamard
 * construction): m(c) = the smallest order m >= 4 ceil(c/4) for which a
 * Hadamard matrix is built, the orders being 1 and 2, q + 1 (Paley-I, q an odd
 * prime power, q = 3 mod 4), 2(q + 1) (Paley-II, q = 1 mod 4), and every
 * product of two of them (Kronecker products); m(192) = 192 and m(320) = 320.
 * Returns m(c), or 0 for c < 1 or c > 4096.  Whether the kernels take the
 * order is a separate question: hblock documents that (the powers of two up to
 * 128, 192 and 320).  Host only. */
int32_t hatq_hadamard_order(int32_t c);

/* Workspace bytes of hatq_layer_forward for an input of n x h x w. */
size_t hatq_layer_ws_bytes(const hatq_weights *W, int32_t n, int32_t h, int32_t w);

/* One whole layer (step a7): hatq_fwht_quant_act then hatq_conv_int8 in F32
 * mode, with the transform of the layer's own form (DH: hblock on cin; WH: none
 * on the activations).
 *   form:      must equal W->form (the per-layer form flag), else HATQ_EINVAL.
 *   x:         device fp32 [n][h][w][cin].
 *   x_absmax:  NULL, or per-sample max |T_in x| already known (see above).
 *   y:         device fp32 [n][ho][wo][cout].
 *   act_scale: NULL, or device fp32 [n] receiving s_x.
 *   next_hblock, next_absmax: as in hatq_conv_int8.
 *   ws:        at least hatq_layer_ws_bytes(W, n, h, w) bytes of device memory. */
int32_t hatq_layer_forward(const hatq_weights *W, int32_t form, const float *x, int32_t n,
                           int32_t h, int32_t w, const float *x_absmax, float *y,
                           float *act_scale, int32_t next_hblock, float *next_absmax,
                           void *ws, size_t ws_bytes, void *stream);

/* ---- Linear layers over tokens -------------------------------------------------
 *
 * The fully connected layer Y = X W^T + b of rows of tokens, in the DH form
 * (Eq. double_hadamard_quantization) with a scale for each token instead of one
 * for each sample, one layer or several experts.  For token t, channel c, block
 * b = hblock:
 *   S[t]   = B_cin x[t]                      fp32 butterflies, ascending stages
 *   s[t]   = fl32(max|S[t]| / 127)           1 where that is 0
 *   q[t,d] = clamp(rne(fl32(S[t,d] / s[t])), -127, 127)
 *   z[t,c] = fma(float(sum_d q[t,d] wq[c,d]), fl((s[t] / b) w_scale[c]), bias[c])
 *            (s[t] / b is exact unless it is below 2^-126)
 *   y[t,c] = z[t,c], or for a gated layer, which holds 2 cout channels, gates
 *            first: g / (1 + exp(-g)) u with g = z[t,c], u = z[t,cout+c], each
 *            operation in fp32 (0 where exp(-g) overflows: g < -88.7).
 * The sums are exact in INT32.  y is rounded once, to y_type.  A token that
 * holds a NaN or an infinity, or whose transform overflows fp32, has the scale
 * NaN and codes 0: its outputs are NaN, every other token's are unaffected.
 *
 * Here rows have strides, in elements; the elements of a row are adjacent.  A
 * call with no rows is HATQ_OK and launches nothing (but hatq_expert_order, which
 * writes its ends), one of more than 2^24 rows HATQ_EUNSUPPORTED.  x and y may have
 * any alignment of their type; codes and prepared weights are 16-byte aligned.
 * Outputs and the workspace do not overlap the inputs.  No kernel's result depends
 * on the order in which blocks run. */
typedef enum { HATQ_F32 = 0, HATQ_BF16 = 1, HATQ_F16 = 2 } hatq_dtype;

/* Prepared linear weights: a plain view into the caller's device buffer.
 * experts >= 1 layers of the same shape.  k_stride = cin rounded up to 64 is the
 * row stride of the layer's input codes; cout_pad the channels held, a gated
 * layer's gates and values taken 32 by 32 in turn, rounded up to 32 each.
 * wpack holds the codes in the kernels' order (library-internal): per expert,
 * per 16 channels, per 64-deep contraction step, 1 KB as [4][16 channels][16].
 * w_scale and bias are fp32 [experts][cout_pad] in wpack's channel order, 0 in
 * the padding. */
typedef struct {
    int32_t experts, cin, cout;
    int32_t gated;          /* 1: holds 2 cout channels, gives cout */
    int32_t hblock;         /* transform block on cin, a power of two in [1, 128] */
    int32_t k_stride, cout_pad;
    int8_t *wpack;
    float *w_scale;
    float *bias;
} hatq_linear_weights;

/* Bytes of device memory for such weights; 0 for sizes that are not supported
 * (cin % hblock != 0, cin or held channels over 65536, experts over 1024). */
size_t hatq_linear_weights_bytes(int32_t experts, int32_t cin, int32_t cout, int32_t gated, int32_t hblock);

/* Weights from floats: w device [experts][held][cin] of w_type (held = cout, or
 * 2 cout for a gated layer: gates, then values), bias device fp32
 * [experts][held] or NULL.  As hatq_prepare_weights: the transform in fp64,
 * rounded once to fp32, w_scale = fl32(max|W'| / 127) (1 where that is 0), codes
 * clamp(rne(fl32(W' / w_scale)), -127, 127).  A channel with a NaN or an infinity
 * among its W' has the scale NaN and codes 0: its outputs are NaN.
 *   dst: device buffer of at least hatq_linear_weights_bytes, 256-byte aligned;
 *   *out receives the view into it.  Runs on `stream`. */
int32_t hatq_prepare_linear(int32_t experts, int32_t cin, int32_t cout, int32_t gated, int32_t hblock, const void *w,
                            int32_t w_type, const float *bias, void *dst, size_t dst_bytes,
                            hatq_linear_weights *out, void *stream);

/* The same from codes quantized elsewhere (a deployment checkpoint): codes
 * device int8 [experts][held][cin] of the transformed weights, w_scale device
 * fp32 [experts][held], bias fp32 [experts][held] or NULL. */
int32_t hatq_pack_linear(int32_t experts, int32_t cin, int32_t cout, int32_t gated, int32_t hblock,
                         const int8_t *codes, const float *w_scale, const float *bias, void *dst, size_t dst_bytes,
                         hatq_linear_weights *out, void *stream);

/* Codes and scales of tokens.
 *   x:  device [rows][cin] of x_type, row stride x_stride >= cin elements.
 *   xq: device int8 [rows][k_stride], k_stride = cin rounded up to 64, the bytes
 *       past cin written 0; act_scale: device fp32 [rows].
 * cin % hblock == 0, cin <= 65536, hblock a power of two in [1, 128]
 * (HATQ_EUNSUPPORTED for the orders 192 and 320). */
int32_t hatq_token_quant(const void *x, int32_t x_type, int32_t rows, int32_t cin, int64_t x_stride, int32_t hblock,
                         int8_t *xq, float *act_scale, void *stream);

/* The product of token codes with one layer's weights (W->experts == 1) and its
 * epilogue.
 *   xq, act_scale: as hatq_token_quant writes them (any bytes past cin).
 *   y: device [rows][cout] of y_type, row stride y_stride >= cout elements. */
int32_t hatq_linear_int8(const hatq_linear_weights *W, const int8_t *xq, const float *act_scale, int32_t rows,
                         void *y, int32_t y_type, int64_t y_stride, void *stream);

/* The whole layer, floats in: hatq_token_quant into the workspace, then
 * hatq_linear_int8, or for a few tokens (rows <= HATQ_TOKEN_ROWS and rows
 * k_stride <= HATQ_TOKEN_CODES) and for small layers one kernel that does both,
 * with the same result.
 * ws: device memory, 256-byte aligned, of at least hatq_linear_ws_bytes(W, rows)
 * bytes; for a few tokens it is not used and may be NULL. */
#define HATQ_TOKEN_ROWS 16
#define HATQ_TOKEN_CODES 16384
size_t hatq_linear_ws_bytes(const hatq_linear_weights *W, int32_t rows);
int32_t hatq_linear_forward(const hatq_linear_weights *W, const void *x, int32_t x_type, int32_t rows,
                            int64_t x_stride, void *y, int32_t y_type, int64_t y_stride, void *ws, size_t ws_bytes,
                            void *stream);

/* Products grouped by expert: output row i belongs to the first expert e with
 * i < ends[e] and takes the codes of token src[i].
 *   ends: device int32 [experts], the experts' row ends, ascending; values are
 *         taken into [the end before, rows], so no contents make a call unsafe.
 *         Rows past the last end are written 0.
 *   src:  device int32 [rows], or NULL (then x_rows >= rows, token i).  A value
 *         outside [0, x_rows) stands for an empty token: y is the layer's output
 *         for x = 0, its bias (gated: of its biases).
 *   x_rows: tokens in xq and act_scale (at least 1 where rows is). */
int32_t hatq_experts_int8(const hatq_linear_weights *W, const int8_t *xq, const float *act_scale, int32_t x_rows,
                          const int32_t *ends, const int32_t *src, int32_t rows, void *y, int32_t y_type,
                          int64_t y_stride, void *stream);

/* The same, floats in: hatq_token_quant of the x_rows tokens into the workspace, then
 * hatq_experts_int8, or for few rows and small products one kernel that quantizes
 * each output row's token, with the same result.  ws: at least
 * hatq_linear_ws_bytes(W, x_rows) bytes, 256-byte aligned. */
int32_t hatq_experts_forward(const hatq_linear_weights *W, const void *x, int32_t x_type, int32_t x_rows,
                             int64_t x_stride, const int32_t *ends, const int32_t *src, int32_t rows, void *y,
                             int32_t y_type, int64_t y_stride, void *ws, size_t ws_bytes, void *stream);

/* The rows of hatq_experts_* from each token's chosen experts: a stable counting
 * sort of the pairs p = t topk + j by ids[p].
 *   ids:  device int32 [tokens][topk]; a pair whose id is outside [0, experts)
 *         is masked: it has no row.
 *   ends: device int32 [experts], written.
 *   src:  device int32 [tokens topk], written: the token of each row, -1 past the
 *         last end.
 *   pos:  device int32 [tokens topk], written: the row of each pair, -1 for a
 *         masked one.
 *   ws:   device memory, 256-byte aligned, of at least hatq_expert_order_ws_bytes
 *         bytes (0 for sizes that are not supported: tokens topk over 2^24,
 *         experts over 1024). */
size_t hatq_expert_order_ws_bytes(int32_t tokens, int32_t topk, int32_t experts);
int32_t hatq_expert_order(const int32_t *ids, int32_t tokens, int32_t topk, int32_t experts, int32_t *ends,
                          int32_t *src, int32_t *pos, void *ws, size_t ws_bytes, void *stream);

/* The weighted sum of each token's rows, y[t] = sum_j weights[t,j] h[pos[t,j]],
 * fp32 fma in ascending j, rounded once to y_type.
 *   h: device fp32 [h_rows][cols], row stride h_stride elements, cols <= 2^30.
 *   pos: device int32 [tokens][topk]; a value outside [0, h_rows) adds nothing
 *   (a token with none gives 0).  weights: device fp32 [tokens][topk]. */
int32_t hatq_expert_combine(const float *h, int32_t h_rows, int32_t cols, int64_t h_stride, const int32_t *pos,
                            const float *weights, int32_t tokens, int32_t topk, void *y, int32_t y_type,
                            int64_t y_stride, void *stream);

/* A feed-forward block of gated experts, the calls above in one: hatq_expert_order
 * of ids; hatq_experts_forward of x through the gated W_in into fp32 hidden rows;
 * of those through W_out into fp32 rows; hatq_expert_combine with the weights.
 *   W_in, W_out: as many experts, W_in gated, W_out plain, W_in->cout == W_out->cin.
 *   x: device [tokens][W_in->cin] of x_type; ids int32, weights fp32, device
 *   [tokens][topk]; y: device [tokens][W_out->cout] of y_type.
 *   ws: device memory, 256-byte aligned, of at least hatq_expert_mlp_ws_bytes bytes
 *       (0 for weights that do not fit together, or sizes that are not supported). */
size_t hatq_expert_mlp_ws_bytes(const hatq_linear_weights *W_in, const hatq_linear_weights *W_out, int32_t tokens,
                                int32_t topk);
int32_t hatq_expert_mlp(const hatq_linear_weights *W_in, const hatq_linear_weights *W_out, const void *x,
                        int32_t x_type, int32_t tokens, int64_t x_stride, const int32_t *ids, const float *weights,
                        int32_t topk, void *y, int32_t y_type, int64_t y_stride, void *ws, size_t ws_bytes,
                        void *stream);

/* ---- Linear layers of 4-bit weights ---------------------------------------------
 *
 * hatq_linear_forward's layer with 15 (or 16) levels of weights and a scale for each
 * channel and group of `group` adjacent input channels, for the bytes that a few tokens
 * have to read: tokens as there (S, s and q of each token t, its codes INT8), and
 *   z[t,c] = (s[t] / b) sum_g w_scale[c,g] float(sum_{d in g} q[t,d] wq[c,d]) + bias[c]
 * with exact sums in each group and fp32 sums over the groups; y from z as there, gated or
 * not.  A NaN among a channel's scales makes its outputs NaN, a token that is not finite
 * its own.
 * Any number of rows is taken; the kernels are made for up to about 128.  Outputs and the
 * workspace do not overlap the inputs. */
typedef struct {
    int32_t cin, cout;
    int32_t gated;          /* 1: holds 2 cout channels, gives cout */
    int32_t hblock;         /* transform block on cin, a power of two in [1, 128] */
    int32_t group;          /* 64 or 128 input channels */
    int32_t k_stride;       /* cin rounded up to 128 */
    int32_t cout_pad;       /* the channels held: cout rounded up to 16, twice if gated */
    uint8_t *wpack;         /* library-internal order, as w_scale and bias */
    uint16_t *w_scale;      /* bf16 [cout_pad][k_stride / group] */
    float *bias;
} hatq_linear4_weights;

/* Bytes of device memory for such weights; 0 for sizes that are not supported (cin %
 * hblock != 0, cin or held channels over 65536). */
size_t hatq_linear4_weights_bytes(int32_t cin, int32_t cout, int32_t gated, int32_t hblock, int32_t group);

/* Weights from floats: w device [held][cin] of w_type (held = cout, or 2 cout for a gated
 * layer: gates, then values), bias device fp32 [held] or NULL.  W' = B w in fp64, rounded
 * once to fp32; for each group w_scale = bf16(fl32(max|W'| / 7)), at least 2^-100, and codes
 * clamp(rne(fl32(W' / w_scale)), -7, 7).  A group with a NaN or an infinity among its W'
 * has the scale NaN and codes 0.
 *   dst: device buffer of at least hatq_linear4_weights_bytes, 256-byte aligned; *out
 *   receives the view into it.  Runs on `stream`. */
int32_t hatq_prepare_linear4(int32_t cin, int32_t cout, int32_t gated, int32_t hblock, int32_t group, const void *w,
                             int32_t w_type, const float *bias, void *dst, size_t dst_bytes,
                             hatq_linear4_weights *out, void *stream);

/* The same from codes quantized elsewhere (a deployment checkpoint): codes device int8
 * [held][cin] of the transformed weights, taken into [-8, 7]; w_scale device bf16
 * [held][groups], groups = cin / group rounded up. */
int32_t hatq_pack_linear4(int32_t cin, int32_t cout, int32_t gated, int32_t hblock, int32_t group,
                          const int8_t *codes, const uint16_t *w_scale, const float *bias, void *dst,
                          size_t dst_bytes, hatq_linear4_weights *out, void *stream);

/* The whole layer, floats in.
 *   x: device [rows][cin] of x_type, row stride x_stride >= cin elements;
 *   y: device [rows][cout] of y_type, row stride y_stride >= cout elements.
 *   ws: device memory, 256-byte aligned, of at least hatq_linear4_ws_bytes(W, rows) bytes;
 *       may be NULL where that is 0 (a few tokens, small layers of a short contraction).  Calls
 *       that may overlap need workspaces of their own. */
size_t hatq_linear4_ws_bytes(const hatq_linear4_weights *W, int32_t rows);
int32_t hatq_linear4_forward(const hatq_linear4_weights *W, const void *x, int32_t x_type, int32_t rows,
                             int64_t x_stride, void *y, int32_t y_type, int64_t y_stride, void *ws, size_t ws_bytes,
                             void *stream);

/* ---- A cache of keys and values in 4 bits, and attention over it ------------------
 *
 * The symmetric quantizer of Eq. symmetric_q with 15 levels in the Hadamard domain, for
 * heads of `dim` channels.  For a key or value x of one position and head, block b =
 * hblock, and each group g of 64 adjacent channels (the last one may be shorter):
 *   S    = B_dim x                           fp32 butterflies, ascending stages
 *   s[g] = bf16(fl32(max_{d in g}|S[d]| / 7))  rounded half to even, at least 2^-100
 *   c[d] = clamp(rne(fl32(S[d] / s[g])), -7, 7)
 * and what they stand for is x' = B_dim (s c) / b.  A head with a NaN, an infinity or a
 * magnitude of 2^102 (5e30) and more among its S has all its scales NaN and codes 0: it
 * stands for NaN.
 *
 * The cache is made of pages of page_size positions of all heads.  Sequence i's position
 * p is in page table[i][p / page_size]; a page of which the cache has none (negative, or
 * >= pages) is absent.  Pages may be shared between sequences as long as no call writes
 * one of them twice.  The library keeps no table, lengths or free pages of its own.
 *
 * The calls below take rows of new tokens, sequence by sequence: sequence i has the rows
 * [ends[i - 1], ends[i]), n of them, which are its positions lens[i] - n .. lens[i] - 1, so
 * lens counts the new tokens too.  ends NULL: rows / batch each.
 *   table: device int32 [batch][width];  lens: device int32 [batch];
 *   ends:  device int32 [batch], ascending, or NULL (then rows % batch == 0).
 * Any contents of the three are safe.  Positions below 0, past the table's width or in an
 * absent page are left out: not written, read as 0, not attended to (a length past the
 * table counts all the same: its rows come after the table's positions).  Values of ends that
 * do not ascend within [0, rows] give rows to some sequence or to none.  Rows past the
 * last end stay as they are.
 *
 * Tensors [rows][heads][dim] have a stride in elements between rows and between heads,
 * and adjacent channels; outputs' rows and heads do not overlap, nor do outputs and the workspace
 * overlap each other, the cache or inputs, unless said below.  Any alignment of the type.
 * rows <= 2^24; no rows: HATQ_OK, nothing launched.  A sequence has at most 2^30 positions
 * (width page_size, else HATQ_EUNSUPPORTED). */
typedef struct {
    int32_t pages;
    int32_t page_size;      /* positions, a power of two in [16, 65536] */
    int32_t heads, dim;     /* of the keys and values */
    int32_t hblock;         /* transform block on dim, a power of two in [1, 128] */
    void *buf;              /* library-internal layout: a position's key and value 68 bytes for each 64
                               channels of a head, the last ones whole */
} hatq_cache4;

typedef struct {
    int32_t type;           /* hatq_dtype */
    int64_t row_stride, head_stride;
    void *p;
} hatq_heads;

/* Bytes of such a cache; 0 for sizes that are not supported (dim % hblock != 0, dim over
 * 256, heads over 1024, pages page_size over 2^31 - 1).  hatq_cache4_init, host only,
 * makes the view of a device buffer of at least as many bytes, 256-byte aligned.  The
 * contents need no clearing: positions are written before a length reaches them. */
size_t hatq_cache4_bytes(int32_t pages, int32_t page_size, int32_t heads, int32_t dim, int32_t hblock);
int32_t hatq_cache4_init(int32_t pages, int32_t page_size, int32_t heads, int32_t dim, int32_t hblock, void *buf,
                         size_t bytes, hatq_cache4 *out);

/* New tokens' keys and values into the cache.  k, v: device [rows][heads][dim]. */
int32_t hatq_cache4_append(const hatq_cache4 *C, const hatq_heads *k, const hatq_heads *v, int32_t rows,
                           const int32_t *table, int32_t width, const int32_t *lens, const int32_t *ends,
                           int32_t batch, void *stream);

/* The values that the cache holds for such rows, written to k and v (each its own type):
 * the sequences' last positions. */
int32_t hatq_cache4_read(const hatq_cache4 *C, const hatq_heads *k, const hatq_heads *v, int32_t rows,
                         const int32_t *table, int32_t width, const int32_t *lens, const int32_t *ends,
                         int32_t batch, void *stream);

/* Attention of query rows over the cache: for query head h, which reads the cached head
 * h / (q_heads / heads), and a row of sequence i at position p,
 *   y = sum_j w_j v'_j,  w = softmax over j of scale q . k'_j,
 * j over [0, lens[i]), or causal: over [0, p], and with a window over (p - window, p] of
 * those.  A row that sees no position gives 0.
 *   q, y: device [rows][q_heads][dim], each its own type; q_heads % C->heads == 0.
 *   scale: a finite number, mostly dim^-1/2.
 *   causal: 0 or 1;  window: 0 for none, else at least 1, and causal.
 *   max_len: 0, or what the lengths will not exceed, for the choice of the launch alone
 *       (0: width page_size): any value gives the same sums, in another order.
 *   ws: device memory, 256-byte aligned, of at least hatq_attention4_ws_bytes bytes for
 *       the same sizes (ragged: ends is given); may be NULL where that is 0.  Calls that may
 *       overlap need workspaces of their own.
 * y may be q, with the same strides and type.  Scores, weights and sums are fp32.  Products:
 * the transformed query in two fp16 halves, 22 bits (many rows of bf16: one, 11 bits; which
 * rows are many goes by all of a call's), against the codes; the weights times the values'
 * scales in fp16, off by 2^-11 of each (if q or y is not bf16, in two halves, 2^-21 of each) or
 * by 2^-37 of the head's largest, that of all its groups of 64 channels.  So a group whose
 * scales are 2^-r of another's in the same positions has an error of up to 2^(r-37) of its own
 * largest, and from 2^-38 on it can be lost.  The values of a query's transform are off by up to
 * 2^-38 of its head's largest alike.  Scores up to 2^120 in magnitude give numbers: where float32
 * no longer resolves their softmax, a mean of the values at the top.  No result depends on the
 * order in which blocks run. */
size_t hatq_attention4_ws_bytes(const hatq_cache4 *C, int32_t rows, int32_t q_heads, int32_t width, int32_t batch,
                                int32_t ragged, int32_t window, int32_t max_len);
int32_t hatq_attention4(const hatq_cache4 *C, const hatq_heads *q, const hatq_heads *y, int32_t rows, int32_t q_heads,
                        const int32_t *table, int32_t width, const int32_t *lens, const int32_t *ends, int32_t batch,
                        float scale, int32_t causal, int32_t window, int32_t max_len, void *ws, size_t ws_bytes,
                        void *stream);

#ifdef __cplusplus
}
#endif
#endif /* HATQ_H */
