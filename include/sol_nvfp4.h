/*
 * sol_nvfp4.h -- C ABI of the B200 (sm_100a) NVFP4 linear-layer library.
 *
 * The library computes the W4A4 linear layers of a diffusion-transformer rollout:
 *     Y = Q(X) . Q(W)^T + bias
 * where Q is the NVFP4 quantizer of the paper's Section 2 ("FP4 Quantization and
 * Hardware Acceleration"):  x~ = S * Pi_FP4(x / S), FP4 = E2M1 (1 sign, 2 exponent,
 * 1 mantissa bit), one E4M3 scale per 16 contiguous elements along K.  S is split in two
 * levels: the E4M3 block scale and one FP32 scale T per tensor.  A BF16 linear of the
 * same shape is the full-precision reference the paper's second stage runs in.
 *
 * General rules
 *   - Every pointer is a DEVICE pointer unless its comment says host.  The caller owns
 *     every buffer; the library allocates no device memory (it keeps a small host-side
 *     cache of TMA descriptors and reads device properties once).
 *   - `stream` is a cudaStream_t passed as void* (NULL = the legacy default stream).
 *     All work is asynchronous on it; no call synchronises or reads device scalars on the
 *     host.  T flows from kernel to kernel through device memory.
 *   - Every function returns a sol_status_t; nothing throws.  Arguments are validated on
 *     the host before anything is launched: on an error status no kernel was launched.
 *   - Matrices are row-major with the K dimension contiguous: X is [M, K], W is [N, K]
 *     (the nn.Linear convention), Y is [M, N].  ld* are row pitches in ELEMENTS.
 *   - Requirements: M, N, K > 0; K % 32 == 0; N % 8 == 0; pointers 16-byte aligned; BF16
 *     row pitches multiples of 8 elements.  Inputs must be finite.
 *   - Only sm_100 devices are supported (SOL_ERR_UNSUPPORTED_ARCH otherwise); there is
 *     no CPU path.
 *   - A launch the CUDA runtime rejects returns SOL_ERR_CUDA; with the environment variable
 *     SOL_NVFP4_VERBOSE set, the runtime's error string is also printed to stderr.
 *
 * NVFP4 storage
 *   data   : uint8 [rows, K/2]; byte j of a row holds element 2j in its low nibble and
 *            element 2j+1 in its high nibble; nibble = s e e m.
 *   scales : uint8 E4M3 (unsigned use).  SOL_SF_ROW_MAJOR: [rows, K/16].
 *            SOL_SF_SWIZZLED_128x4: 512-byte chunks of 128 rows x 4 blocks, chunk order
 *            [ceil(rows/128)][ceil(K/64)]; inside a chunk the scale of (row r, block b) is at
 *            (r%32)*16 + ((r%128)/32)*4 + b%4.  Padding bytes are written as 0.  This is
 *            the layout the tensor core's scale-factor copy consumes; the GEMM entries
 *            require it.
 *   T      : one float; dequantized value = E2M1(nibble) * E4M3(scale) * T.
 */
#ifndef SOL_NVFP4_H_
#define SOL_NVFP4_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    SOL_OK = 0,
    SOL_ERR_NULL_POINTER = 1,
    SOL_ERR_BAD_SHAPE = 2,
    SOL_ERR_ALIGNMENT = 3,
    SOL_ERR_WORKSPACE_TOO_SMALL = 4,
    SOL_ERR_UNSUPPORTED_ARCH = 5,
    SOL_ERR_CUDA = 6,
    SOL_ERR_TIMEOUT = 7,
    SOL_ERR_BAD_LAYOUT = 8
} sol_status_t;

typedef enum { SOL_SF_ROW_MAJOR = 0, SOL_SF_SWIZZLED_128x4 = 1 } sol_sf_layout_t;
typedef enum { SOL_ACT_NONE = 0, SOL_ACT_GELU_TANH = 1, SOL_ACT_SILU = 2 } sol_activation_t;

/* Static, human-readable name of a status (host pointer, never NULL). */
const char *sol_status_string(sol_status_t status);

/* Bytes of packed FP4 data for a [rows, K] tensor: rows * K / 2.  0 on bad arguments. */
size_t sol_nvfp4_data_bytes(int64_t rows, int64_t K);

/* Bytes of the scale buffer in the given layout (swizzled: ceil(rows/128) * ceil(K/64) * 512).
 * 0 on bad arguments. */
size_t sol_nvfp4_scale_bytes(int64_t rows, int64_t K, sol_sf_layout_t layout);

/* Bytes of workspace nvfp4_quantize_linear needs for an [M, K] activation: packed data,
 * swizzled scales and one float, each region 256-byte aligned.  0 on bad arguments. */
size_t sol_nvfp4_linear_workspace_bytes(int64_t M, int64_t N, int64_t K);

/*
 * Per-tensor scale (second scaling level; the paper's single S is split so that block
 * scales span E4M3's range):  T = max|x| / (6 * 448), or 1 for an all-zero tensor.
 *   x                [rows, K] BF16, pitch ld
 *   tensor_scale_out one float (device), overwritten
 * The max is exact (order-independent), so the result is deterministic.
 */
sol_status_t sol_amax_bf16(const void *x, int64_t rows, int64_t K, int64_t ld,
                           float *tensor_scale_out, void *stream);

/*
 * Activation quantizer, Section 2's Q(x) with S = block scale * T.  Per row and per block
 * of 16 elements along K, in IEEE binary32 (round-to-nearest-even, no contraction):
 *     a = max|x|;  sb = E4M3_rne_sat(a / (6*T));  rcp = 1 / (float(sb) * T)  (0 if sb == 0)
 *     nibble_k = E2M1_rne_sat(x_k * rcp)   (ties to the even code, sign bit of x kept)
 *   x_bf16       [M, K] BF16, pitch ldx
 *   tensor_scale one float (device), read by the kernel; > 0
 *   q_out        sol_nvfp4_data_bytes(M, K) bytes
 *   sf_out       sol_nvfp4_scale_bytes(M, K, layout) bytes; every byte is written
 */
sol_status_t nvfp4_quantize(const void *x_bf16, int64_t M, int64_t K, int64_t ldx,
                            const float *tensor_scale, void *q_out, void *sf_out,
                            sol_sf_layout_t layout, void *stream);

/*
 * Weight quantizer: the same mapping applied to W [N, K] along K, preceded by the
 * per-tensor scale of W (the paper re-quantizes the policy weights after each update,
 * Section 3.4 / Appendix B.2).
 *   tensor_scale_out one float (device), written by the first kernel, read by the second
 */
sol_status_t nvfp4_quantize_weight(const void *w_bf16, int64_t N, int64_t K, int64_t ldw,
                                   void *q_out, void *sf_out, float *tensor_scale_out,
                                   sol_sf_layout_t layout, void *stream);

/*
 * Weight refresh: merge rank-r adapters into the base weights and quantize the result, the step
 * that follows every policy update (Section 3.4, Appendix B.2; Section 4.1: r = 32, alpha = 64,
 * so scaling = alpha / r = 2).  The paper does not spell the merge out; this is the usual
 *     W'[n][k] = bf16_rne( fma(scaling, acc, W[n][k]) ),
 *     acc = 0;  acc = fma(B[n][j], A[j][k], acc)  for j = 0 .. r-1 in this order   (IEEE binary32)
 * followed by nvfp4_quantize_weight's mapping applied to W'.
 *   w_bf16      [N, K] BF16, pitch ldw; not modified (training keeps base and adapters apart)
 *   lora_a      [r, K] BF16, pitch lda ("down" projection)
 *   lora_b      [N, r] BF16, pitch ldb ("up" projection); 1 <= r <= 64
 *   merged_bf16 [N, K] BF16, dense; receives W' (also the scratch the quantizer reads back)
 *   q_out, sf_out, layout: as for nvfp4_quantize_weight
 *   tensor_scale_out  TWO floats (device): [0] receives T of W'; [1] is scratch (it is left holding
 *                     max|W'|, the value T was derived from)
 * Three launches on the stream: clear the scratch word, the merge kernel, the quantizer.
 */
sol_status_t nvfp4_requantize_lora(const void *w_bf16, int64_t ldw, const void *lora_a, int64_t lda,
                                   const void *lora_b, int64_t ldb, int64_t N, int64_t K, int64_t r,
                                   float scaling, void *merged_bf16, void *q_out, void *sf_out,
                                   float *tensor_scale_out, sol_sf_layout_t layout, void *stream);

/*
 * The same for `count` matrices of one shape (all targeted projections of a model after a policy
 * update), in one call.  One matrix is ~20 us of GPU work, so launches are shared: matrices are
 * processed in groups of up to min(merged_matrices, 8), three launches per group.  The six lists
 * are HOST arrays of `count` DEVICE pointers; matrix i uses w_list[i] [N, K], a_list[i] [r, K],
 * b_list[i] [N, r] (all dense) and writes q_list[i], sf_list[i], ts_list[i] (two floats each).
 *   merged_bf16      device scratch for `merged_matrices` (>= 1) dense [N, K] BF16 matrices, reused
 *                    group after group in stream order (contents undefined afterwards); a scratch
 *                    that fits L2 keeps the merged weights out of HBM
 * Everything is validated before the first launch.
 */
sol_status_t nvfp4_requantize_lora_batch(int64_t count, const void *const *w_list, const void *const *a_list,
                                         const void *const *b_list, void *const *q_list, void *const *sf_list,
                                         float *const *ts_list, int64_t N, int64_t K, int64_t r, float scaling,
                                         void *merged_bf16, int64_t merged_matrices, sol_sf_layout_t layout,
                                         void *stream);

/*
 * Low-rank adapters of many requests at once beside a shared projection whose output is y (in any precision): request i is the
 * rows [offsets[i], offsets[i+1]) and has the adapter a = ids[i], or none (an index outside [0, adapters)):
 *     t = x A_a^T;     y = bf16_rne( y + scaling[a] t B_a^T )                       (in place)
 *   x_bf16   [M, K], pitch ldx;   y_bf16  [M, N], pitch ldy
 *   lora_a   [adapters, r, K] BF16, dense;   lora_b  [adapters, N, r] BF16, dense;   scaling  [adapters] FP32
 *   offsets  [requests + 1] int32, ascending, held to [0, M];   ids  [requests] int32   (device, as everything here).  Rows in
 *            front of the first offset and behind the last stay as they are, requests without rows are fine
 *   t_out    [M, 2 r] BF16 or NULL: t in two parts (columns [0, r): rounded; [r, 2 r): what that left), for the gradients;
 *            rows without an adapter are not written
 *   K, N multiples of 8 up to 1048576;  r a multiple of 8, 8 <= r <= 64;  adapters, requests <= 1024
 *   workspace  sol_lora_workspace_bytes(M, K, N, r, adapters, requests, 0) bytes of device scratch, 256-byte aligned; two calls
 *              that may overlap need one each
 * Sums are FP32 in a fixed order; t enters the second product with 16 bits.  Two launches.  A wait that runs out
 * (sol_last_device_status) leaves y incomplete or NaN.  Where a value of t is infinite its row of y is NaN, also where the formula has
 * an infinity: the part that its rounding leaves is a difference of infinities.  No other request's rows see it.
 */
size_t sol_lora_workspace_bytes(int64_t M, int64_t K, int64_t N, int64_t r, int64_t adapters, int64_t requests, int backward);
sol_status_t sol_lora_apply(const void *x_bf16, int64_t ldx, const void *lora_a, const void *lora_b, const float *scaling,
                            const int32_t *offsets, const int32_t *ids, int64_t requests, int64_t adapters, void *y_bf16, int64_t ldy,
                            void *t_out, int64_t M, int64_t K, int64_t N, int64_t r, void *workspace, size_t workspace_bytes,
                            void *stream);

/*
 * Gradients of sol_lora_apply from dy = d loss / d y; with dt = scaling[a] dy B_a:
 *     dx = bf16_rne( dx + dt A_a ),   dlora_a = sum over the adapter's rows of dt^T x,   dlora_b = scaling[a] sum of dy^T t
 *   t        [M, 2 r] as sol_lora_apply left it;  dx_bf16  [M, K], pitch ld_dx, in place: the gradient that x has from the shared
 *            projection, or NULL
 *   dlora_a, dlora_b  FP32, shaped as the factors, 16-byte aligned, overwritten (zeros for an adapter without rows)
 *   workspace  sol_lora_workspace_bytes(..., 1) bytes.  Everything else as there (dt in t's place).  Three or four launches.
 * dt enters dlora_a with 24 bits and dx, which is BF16, with 16.
 */
sol_status_t sol_lora_backward(const void *dy_bf16, int64_t ld_dy, const void *x_bf16, int64_t ldx, const void *t, const void *lora_a,
                               const void *lora_b, const float *scaling, const int32_t *offsets, const int32_t *ids, int64_t requests,
                               int64_t adapters, void *dx_bf16, int64_t ld_dx, float *dlora_a, float *dlora_b, int64_t M, int64_t K,
                               int64_t N, int64_t r, void *workspace, size_t workspace_bytes, void *stream);

/*
 * One AdamW step over many tensors (the policy update in front of that refresh), in place.  Per element, FP32, with t the step:
 *     g = grad * grad_scale;  m = beta1 m + (1 - beta1) g;   v = beta2 v + (1 - beta2) g^2       (every operation rounded)
 *     param = param (1 - lr weight_decay) - lr / (1 - beta1^t) m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
 * Root and quotient are the hardware's approximate ones, products and sums of the second line are fused: param is off by at most 2^-24
 * (2 |param| + 16 |update|) before it is rounded to its type.
 *   tensors     HOST array of `count` descriptions (read during the call only) of device tensors of n >= 0 dense elements, 16-byte
 *               aligned, no two of them overlapping:  param FP32 or BF16;  copy BF16 or NULL, receives bf16_rne(param) beside an FP32
 *               param;  grad FP32 or BF16, of the same types for all;  m, v the states
 *   state_bits  32: m and v are FP32 [n], the scales NULL.   8: blocks of 32 elements under a power of two, one byte 2^(b-127)
 *               each in m_scale and v_scale [ceil(n/32)], m as E4M3 and v as E5M2 codes [n] (all zero at the start); the
 *               power of two takes a block's largest finite |m| to [2^7, 2^8), its largest v to [2^14, 2^15) (b >= 1)
 *   stochastic  8-bit states and BF16 params are rounded up or down by chance, in proportion, from a hash of seed, t, the tensor's
 *               place in the list and the element's in the tensor; 0: to nearest, ties to even
 *   step_state  two 64-bit words (device, 8-byte aligned): [0] steps done so far, read and advanced by this call (t is one more),
 *               [1] scratch, 0 between calls.  The same for all tensors of a call
 *   lr_scale, grad_scale  one float each (device) or NULL (1): factors that change between the replays of a captured call
 * lr and weight_decay >= 0, 0 <= beta < 1, eps >= 0.  An element whose g is not finite becomes NaN; its 8-bit states too, its FP32 ones
 * are what the formulas give (infinite, or NaN).  Where g is finite and its square is not (|g| above 1.8e19) v is infinite, and the element
 * keeps its value but for the decay; an 8-bit v is NaN then, and the element is NaN from the next step on.  The other elements
 * of a block are not affected.  One launch for up to 448 tensors.
 */
typedef struct {
    void *param, *copy;
    const void *grad;
    void *m, *v, *m_scale, *v_scale;
    int64_t n;
} sol_adamw_tensor_t;
typedef struct {
    double lr, beta1, beta2, eps, weight_decay;
    const float *lr_scale, *grad_scale;
    uint64_t seed;
    int32_t stochastic, param_bf16, grad_bf16, state_bits;
} sol_adamw_options_t;
sol_status_t sol_adamw_step(const sol_adamw_tensor_t *tensors, int64_t count, const sol_adamw_options_t *options, int64_t *step_state,
                            void *stream);

/*
 * Block-scaled FP4 GEMM with BF16 output (the NVFP4 linear the rollout runs, Section 3.4):
 *     acc[m,n] = sum_b sx[m,b] * sw[n,b] * sum_{k in b} qx[m,k] * qw[n,k]      (FP32 accumulate)
 *     Y[m,n]   = bf16_rne( fma(acc, Tx*Tw, bias[n]) )
 *   xq, wq     packed data [M, K/2], [N, K/2] (dense pitch K/2 bytes)
 *   xsf, wsf   scales in SOL_SF_SWIZZLED_128x4 layout
 *   x_tscale, w_tscale   one float each (device)
 *   bias_bf16  [N] BF16 or NULL
 *   y_bf16     [M, N] BF16, pitch ldy
 */
sol_status_t nvfp4_linear(const void *xq, const void *xsf, const float *x_tscale,
                          const void *wq, const void *wsf, const float *w_tscale,
                          const void *bias_bf16, void *y_bf16, int64_t M, int64_t N, int64_t K,
                          int64_t ldy, void *stream);

/*
 * The NVFP4 linear with its output already quantized for the NEXT NVFP4 linear: between two
 * rollout linears (Section 3.4) the activations never exist in BF16 in memory, which removes the
 * 2 B/element store, the amax pass and the 2.56 B/element quantizer pass of the next layer.
 *     y[m,n] = fma(acc[m,n], Tx*Tw, bias[n])                     (as nvfp4_linear, FP32)
 *     h[m,n] = bf16_rne( act(y[m,n]) )       act = identity or GELU (tanh form), FP32
 *     (hq, hsf) = the activation quantizer of nvfp4_quantize applied to h along N with T = *out_tscale
 * The two-level scale needs T before the first output exists, so T is the caller's: a calibrated
 * value or the one derived from the previous step's amax_out (a value too small only saturates
 * more blocks at 6*448*T).
 *   out_tscale  one float (device), > 0
 *   hq_out      packed nibbles [M, N/2];  hsf_out  scales, SOL_SF_SWIZZLED_128x4 layout of an [M, N]
 *               tensor, sol_nvfp4_scale_bytes(M, N, ...) bytes, padding rows written as 0
 *   amax_out    nullable; one device word holding max|h| as an FP32 value, updated with an atomic
 *               max (a running maximum: the caller zeroes it to start a new window)
 *   N % 64 == 0.  GELU is evaluated in FP32 with the hardware tanh (absolute error of tanh about
 *   2^-11): far below the BF16 rounding and the FP4 grid that follow, but h can differ from an exactly
 *   evaluated GELU in its last BF16 place more often than the GEMM's accumulation order alone causes.
 */
sol_status_t nvfp4_linear_quantized_out(const void *xq, const void *xsf, const float *x_tscale, const void *wq,
                                        const void *wsf, const float *w_tscale, const void *bias_bf16,
                                        sol_activation_t activation, const float *out_tscale, void *hq_out,
                                        void *hsf_out, float *amax_out, int64_t M, int64_t N, int64_t K,
                                        void *stream);

/*
 * The same for a linear whose outputs feed two consumers, as the first linear of a single-stream
 * DiT block does (3072 -> 9216 + 12288 in the FLUX-shaped config): columns [0, n_split) leave as BF16
 * (q, k, v for attention); columns [n_split, N) pass through the activation and leave quantized
 * into columns [dest_col0, dest_col0 + N - n_split) of a WIDER quantized tensor [M, dest_K] -- the
 * concatenated input of the next linear, whose other columns nvfp4_quantize_into fills.
 *   y_bf16      [M, n_split] BF16, pitch ldy
 *   hq_dest     packed nibbles [M, dest_K/2];  hsf_dest  chunked scales of an [M, dest_K] tensor
 *   out_tscale  the tensor scale of the whole destination tensor (one T for all its parts)
 *   n_split % 256 == 0, (N - n_split) % 64 == 0, dest_K % 64 == 0, dest_col0 % 64 == 0.
 * Everything else as nvfp4_linear_quantized_out.
 */
sol_status_t nvfp4_linear_split_out(const void *xq, const void *xsf, const float *x_tscale, const void *wq,
                                    const void *wsf, const float *w_tscale, const void *bias_bf16, void *y_bf16,
                                    int64_t ldy, int64_t n_split, sol_activation_t activation,
                                    const float *out_tscale, void *hq_dest, void *hsf_dest, int64_t dest_K,
                                    int64_t dest_col0, float *amax_out, int64_t M, int64_t N, int64_t K,
                                    void *stream);

/*
 * nvfp4_quantize writing into columns [dest_col0, dest_col0 + K) of a wider quantized tensor
 * [M, dest_K] (chunked scale layout): the part of a concatenated activation that arrives in BF16.
 * K, dest_K and dest_col0 are multiples of 64; bytes outside the column range are not touched, so
 * the rows past M of the destination's last 128-row scale chunk must have been zeroed once.
 */
sol_status_t nvfp4_quantize_into(const void *x_bf16, int64_t M, int64_t K, int64_t ldx, const float *tensor_scale,
                                 void *q_dest, void *sf_dest, int64_t dest_K, int64_t dest_col0, void *stream);

/*
 * The quantizer fused into the other producer of a DiT linear's input: an adaptive layer norm.
 *     mu, var = mean and population variance of row m;  xhat = (x - mu) / sqrt(var + eps)   (FP32)
 *     h[m,k]  = bf16_rne( xhat[k] * (1 + scale[s,k]) + shift[s,k] ),   s = m / rows_per_sample
 *     (q, sf) = nvfp4_quantize's mapping applied to h with T = *tensor_scale (caller supplied)
 * One pass over x: 2 B read and 0.56 B written per element instead of a norm pass, an amax pass
 * and a quantizer pass.
 *   x_bf16       [M, K] BF16, pitch ldx;  K % 64 == 0, K <= 4096
 *   scale, shift [ceil(M / rows_per_sample), K] BF16, dense (the per-sample modulation)
 *   q_out        [M, K/2];  sf_out  SOL_SF_SWIZZLED_128x4 scales of an [M, K] tensor, every byte written
 *   amax_out     nullable running max|h| (atomic max on the FP32 value), as in nvfp4_linear_quantized_out
 */
sol_status_t nvfp4_layernorm_quantize(const void *x_bf16, int64_t M, int64_t K, int64_t ldx, const void *scale_bf16,
                                      const void *shift_bf16, int64_t rows_per_sample, float eps,
                                      const float *tensor_scale, void *q_out, void *sf_out, float *amax_out,
                                      void *stream);

/*
 * The training pass's form of that norm: BF16 out, the row statistics kept for the gradients.  Arithmetic in FP32:
 *     xhat = (x - mean) rstd,  rstd = 1 / sqrt(var + eps);   y[m,k] = bf16_rne( xhat (scale_offset + scale[s,k]) + shift[s,k] )
 *     s = m / rows_per_sample:  scale_offset = 1 is the modulation above, 0 a plain weight (one sample: rows_per_sample >= M)
 *   x_bf16       [M, K] BF16, pitch ldx;  K % 8 == 0, K <= 16384;  y_bf16  [M, K], pitch ldy; may be x with the same pitch
 *   scale, shift [ceil(M / rows_per_sample), K] BF16, pitch ld_mod (slices of one modulation vector per sample will do); either may
 *                be NULL (gain 1, shift 0)
 *   stats_out    [M, 2] FP32 (mean, rstd), 8-byte aligned, or NULL;  eps >= 0 (with eps = 0 a constant row gives NaN)
 */
sol_status_t sol_layernorm(const void *x_bf16, int64_t M, int64_t K, int64_t ldx, const void *scale_bf16, const void *shift_bf16,
                           int64_t ld_mod, int64_t rows_per_sample, float scale_offset, float eps, void *y_bf16, int64_t ldy, float *stats_out,
                           void *stream);

/*
 * Gradients of sol_layernorm from dy = d loss / d y, with w = dy (scale_offset + scale):
 *     dx = rstd (w - mean(w) - xhat mean(w xhat)),   dscale[s] = sum over the sample's rows of dy xhat,   dshift[s] = sum of dy
 *   dy, x, dx      [M, K] BF16 with pitches; x and stats [M, 2] are the forward call's; dx may be dy or x, with the same pitch
 *   scale          the forward call's, pitch ld_scale, or NULL
 *   dscale, dshift [ceil(M / rows_per_sample), K] FP32, dense, 16-byte aligned, overwritten; either may be NULL
 *   workspace      sol_layernorm_backward_workspace_bytes(...) bytes of device scratch, 256-byte aligned (the size may be 0:
 *                  NULL will do).  Two calls that may overlap need one each.
 * The sums over rows are taken in a fixed order (equal inputs give equal bits): per GPU thread in FP32, over the blocks in FP64.
 */
size_t sol_layernorm_backward_workspace_bytes(int64_t M, int64_t K, int64_t rows_per_sample);
sol_status_t sol_layernorm_backward(const void *dy_bf16, int64_t ld_dy, const void *x_bf16, int64_t ldx, const float *stats,
                                    const void *scale_bf16, int64_t ld_scale, int64_t M, int64_t K, int64_t rows_per_sample,
                                    float scale_offset, void *dx_bf16, int64_t ld_dx, float *dscale, float *dshift, void *workspace,
                                    size_t workspace_bytes, void *stream);

/*
 * Scaled-dot-product attention of a DiT block in BF16 (the rollout models of Section 4.1 are
 * diffusion transformers; the method quantizes their linear layers, Section 3, and leaves attention
 * in BF16 in the FP4 and in the BF16 path alike):
 *     out[b, s, h, :] = sum_t softmax_t( q[b,s,h,:] . k[b,t,h,:] / sqrt(head_dim) ) v[b,t,h,:]
 * No mask, no dropout; head_dim is 128 (FLUX.1) or 64 (SD3.5).  Scores and sums in FP32, probabilities rounded to BF16
 * before the product with V, output rounded to BF16.
 *   q, out   [batch, seq_q, heads, head_dim] BF16: element (b, s, h, d) at ((b * seq_q + s) * ld + h * head_dim + d),
 *            ld_q / ld_out elements between consecutive tokens (>= heads * head_dim, multiple of 8), so q, k
 *            and v may be column slices of one fused projection output
 *   k, v     [batch, seq_kv, heads, head_dim] BF16, the same way with ld_k / ld_v
 * All pointers are device pointers, 16-byte aligned, owned by the caller; out must not alias an input.
 * Errors: SOL_ERR_NULL_POINTER, SOL_ERR_BAD_SHAPE (a non-positive extent, another head_dim, ld < heads * head_dim,
 * heads or batch above 65535), SOL_ERR_ALIGNMENT, SOL_ERR_UNSUPPORTED_ARCH, SOL_ERR_CUDA; nothing is launched on an error.
 */
sol_status_t sol_attention_bf16(const void *q, const void *k, const void *v, void *out, int64_t batch, int64_t seq_q,
                                int64_t seq_kv, int64_t heads, int64_t head_dim, int64_t ld_q, int64_t ld_k, int64_t ld_v,
                                int64_t ld_out, void *stream);

/*
 * sol_attention_bf16 whose output leaves as the quantized activations of the linear that follows it in
 * a DiT block (the output projection; in a single-stream block the concatenated input it shares
 * with the MLP branch): h = bf16(attention output), then nvfp4_quantize's mapping with
 * T = *out_tscale, written into columns [dest_col0, dest_col0 + heads * head_dim) of the NVFP4 tensor
 * [batch * seq_q, dest_K] (rows of all samples stacked; chunked scale layout).  Bit for bit what
 * sol_attention_bf16 followed by nvfp4_quantize_into produces, without the BF16 round trip through HBM.
 *   out_tscale   caller supplied (a delayed scale); amax_out: nullable running max|h| as in
 *                nvfp4_linear_quantized_out
 *   dest_K % 64 == 0, dest_col0 % 64 == 0, dest_col0 + heads * head_dim <= dest_K
 * Bytes outside the column range are not touched, so the rows past batch * seq_q of the destination's
 * last 128-row scale chunk must have been zeroed once.  Everything else as sol_attention_bf16.
 */
sol_status_t sol_attention_nvfp4_out(const void *q, const void *k, const void *v, int64_t batch, int64_t seq_q,
                                     int64_t seq_kv, int64_t heads, int64_t head_dim, int64_t ld_q, int64_t ld_k, int64_t ld_v,
                                     const float *out_tscale, void *q_dest, void *sf_dest, int64_t dest_K,
                                     int64_t dest_col0, float *amax_out, void *stream);

/*
 * The same attention over two token streams that are projected separately and attend jointly, as in
 * the double-stream blocks of the FLUX.1 model of Section 4.1 (text tokens and image tokens): the
 * joint sequence is the first stream's tokens followed by the second's; queries, keys and values
 * are read from, and outputs written to, each stream's own tensors -- no concatenated copy exists.
 *   first, second   host pointers to the two descriptions below (read during the call only);
 *                   q, k, v, out: device pointers laid out as in sol_attention_bf16, `seq` tokens each
 *   first->seq % 256 == 0 (the first stream fills whole query-tile pairs); second->seq is free
 * Errors as for sol_attention_bf16, plus SOL_ERR_BAD_SHAPE for a first stream that is not a multiple
 * of 256 tokens.
 */
typedef struct {
    const void *q, *k, *v;
    void *out;
    int64_t seq, ld_q, ld_k, ld_v, ld_out;
} sol_attention_stream_t;
sol_status_t sol_attention_bf16_joint(const sol_attention_stream_t *first, const sol_attention_stream_t *second,
                                      int64_t batch, int64_t heads, int64_t head_dim, void *stream);

/*
 * Block-sparse attention for the explore phase (no counterpart in the paper, whose attention is dense): each block of
 * 256 queries of each head attends to a list of key blocks of 128 tokens.
 *
 * sol_select_blocks chooses the lists by a cheap score, per batch element and head:
 *     score[i][j] = mean(query rows of block i) . mean(key rows of block j)           (FP64)
 *     list[i] = the `count` key blocks of highest score, ascending; the first keep_first blocks are kept whatever their
 *     score (text tokens in front); among equal scores the lower index
 *   q  [batch, seq_q, heads, head_dim] BF16, token pitch ld_q as in sol_attention_bf16;  k  the same with heads_kv heads;
 *      query head h reads key head h / (heads / heads_kv)
 *   kv_lens      [batch] int32 (device) or NULL: keys of a batch element that exist (held to [0, seq_kv]); means are taken over
 *                them and blocks without any are not chosen
 *   block_lists  [batch, heads, ceil(seq_q / 256), count] int32, -1 behind the last;  counts the lists' lengths
 *   scores       same shape as block_lists, FP32 scores of the chosen blocks (-inf behind the last), or NULL
 *   workspace    sol_select_blocks_workspace_bytes(...) bytes of device scratch, 256-byte aligned (one per call that may overlap)
 *   head_dim 64 or 128, seq_kv <= 1048576, 1 <= count <= 8192, keep_first <= count.  Inputs must be finite.
 *
 * sol_attention_blocks computes softmax(q k^T / sqrt(head_dim)) v over the keys of the listed blocks (rounding as
 * sol_attention_bf16).  Any lists will do: entries outside [0, ceil(keys / 128)) are skipped, the order is free, a block
 * listed twice counts twice, a row of queries whose list names no existing key gets zeros.  A count is held to [0, max_blocks].
 * Keys and values behind a batch element's kv_lens may hold anything, NaN included; before it they must be finite.
 *   block_lists [batch, heads, ceil(seq_q / 256), max_blocks];  out as in sol_attention_bf16, no alias of an input
 */
size_t sol_select_blocks_workspace_bytes(int64_t batch, int64_t seq_q, int64_t seq_kv, int64_t heads, int64_t heads_kv,
                                         int64_t head_dim);
sol_status_t sol_select_blocks(const void *q, const void *k, int64_t batch, int64_t seq_q, int64_t seq_kv, int64_t heads,
                               int64_t heads_kv, int64_t head_dim, int64_t ld_q, int64_t ld_k, int64_t count, int64_t keep_first,
                               const int32_t *kv_lens, int32_t *block_lists, int32_t *counts, float *scores, void *workspace,
                               size_t workspace_bytes, void *stream);
sol_status_t sol_attention_blocks(const void *q, const void *k, const void *v, void *out, int64_t batch, int64_t seq_q,
                                  int64_t seq_kv, int64_t heads, int64_t heads_kv, int64_t head_dim, int64_t ld_q,
                                  int64_t ld_k, int64_t ld_v, int64_t ld_out, const int32_t *block_lists,
                                  const int32_t *counts, int64_t max_blocks, const int32_t *kv_lens, void *stream);

/*
 * Linear of a few BF16 rows against a weight in NVFP4 or MXFP4, x kept in 16 bits (weight-only: the rollout models'
 * modulation and embedding linears, whose rows are samples; the paper quantizes both operands of the token linears):
 *     y[m,n] = bf16_rne( T * sum_k act(x[m,k]) * code[n,k] * scale[n, block of k] + bias[n] )      (MXFP4: T = 1)
 *   x_bf16      [M, K] BF16, pitch ldx;  wq, wsf  as written by nvfp4_quantize_weight / mxfp4_quantize with
 *               SOL_SF_SWIZZLED_128x4;  w_tscale one float (device);  bias_bf16 [N] or NULL;  y_bf16 [M, N], pitch ldy
 *   activation  applied to x: SOL_ACT_NONE or SOL_ACT_SILU (x / (1 + exp(-x)), FP32), SOL_ERR_BAD_LAYOUT otherwise
 *   workspace   device scratch of at least sol_matvec_workspace_bytes(M, K) bytes, 256-byte aligned; holds x in the
 *               products' layout; contents undefined after.  Two calls that may overlap need one each.  The size is 0, and
 *               NULL will do, for up to four rows of up to 3072 columns, which every block prepares for itself
 *   M >= 1 (the weight is read once per 64 rows), N % 8 == 0, K % 32 == 0;  y shares no element with an input
 * Two launches, one where no workspace is needed.  Sums are FP32 and in a fixed order.  Before the product act(x) is
 * scaled by a power of two per row (and slice of K) and held in FP16: BF16 values down to 2^-29 of the row's largest are kept
 * exactly where that is at least 2^-100 (an activation's result to 11 bits).  The operands' scales may lie anywhere: only a sum
 * over a slice of K that FP32 does not hold is lost.
 */
size_t sol_matvec_workspace_bytes(int64_t M, int64_t K);
sol_status_t nvfp4_matvec(const void *x_bf16, int64_t ldx, const void *wq, const void *wsf, const float *w_tscale,
                          const void *bias_bf16, sol_activation_t activation, void *y_bf16, int64_t ldy, int64_t M,
                          int64_t N, int64_t K, void *workspace, size_t workspace_bytes, void *stream);
sol_status_t mxfp4_matvec(const void *x_bf16, int64_t ldx, const void *wq, const void *wsf, const void *bias_bf16,
                          sol_activation_t activation, void *y_bf16, int64_t ldy, int64_t M, int64_t N, int64_t K,
                          void *workspace, size_t workspace_bytes, void *stream);

/*
 * What stands between the fused q/k/v projection and the attention of a DiT block: RMS norm of every query and key
 * head, and rotary positions (the paper names the models of Section 4.1 and leaves both to them).  Per (token, head)
 * row x of head_dim values, all arithmetic in FP32:
 *     n = weight * x / sqrt(mean(x^2) + eps)          (no weight: n = x)
 *     each pair (a, b) of the first R = sum(axis_dims) columns becomes (s (a cos t - b sin t), s (b cos t + a sin t)),
 *     t = positions[token, axis of the pair] * freqs[pair]  (formed and reduced in FP64);  the other columns keep n
 * rounded once to BF16.
 *   q, k      host pointers to the descriptions below (read during the call only); k may be NULL
 *   x, out    [rows, heads, head_dim] BF16: element (m, h, d) at m * ld + h * head_dim + d; ld a multiple of 8,
 *             >= heads * head_dim.  out may be x itself with the same pitch (in place); otherwise they do not overlap
 *   weight    [head_dim] BF16, 8-byte aligned, or NULL for no norm
 *   rotary    host pointer, NULL: norm only (a weight is then needed).  A token m (0 <= m < rows) takes the positions
 *             of row m % position_rows, so samples of one geometry share a table.
 *             Pairs are neighbours (2i, 2i+1) or halves (i, i + R/2); pair i takes freqs[i]; the first axis_dims[0] / 2
 *             pairs belong to axis 0 and so on.  axis_dims are positive and even, 1 <= axes <= 4, R % 8 == 0, R <= head_dim
 *   head_dim  32, 64, 128 or 256;  eps >= 0 (with eps = 0 a head of zeros has no norm: NaN, in its gradients as well)
 * The mean of squares is FP32 too: values beyond 2^60, or with eps = 0 a head all below 2^-60, may leave its range.
 */
typedef enum { SOL_ROTARY_INTERLEAVED = 0, SOL_ROTARY_HALF = 1 } sol_rotary_layout_t;
typedef enum {
    SOL_ROTARY_SCALE_NONE = 0, SOL_ROTARY_SCALE_LINEAR = 1, SOL_ROTARY_SCALE_NTK = 2, SOL_ROTARY_SCALE_YARN = 3
} sol_rotary_scaling_t;
typedef struct {
    const int64_t *positions; /* device, [position_rows, axes] */
    const double *freqs;      /* device, [R / 2] radians per position */
    int64_t position_rows, axes, axis_dims[4];
    sol_rotary_layout_t layout;
    float scale;              /* s: 1, or the factor that a long-context scaling puts on cosine and sine */
} sol_rotary_t;
typedef struct {
    const void *x;
    void *out;
    const void *weight;
    int64_t heads, ld_in, ld_out;
} sol_head_tensor_t;
sol_status_t sol_qk_rotary(const sol_head_tensor_t *q, const sol_head_tensor_t *k, int64_t rows, int64_t head_dim,
                           const sol_rotary_t *rotary, float eps, void *stream);

/*
 * Gradients of sol_qk_rotary: from dy = d loss / d out,
 *     dn = the inverse turn of dy (times s);  without a weight dx = dn, with one, xhat = x / sqrt(mean(x^2) + eps):
 *     dx = (weight dn - xhat mean(weight dn xhat)) / sqrt(mean(x^2) + eps),   dweight = sum over tokens and heads of dn xhat
 *   dy, x, dx  laid out as x above; x is the forward call's input, read only when there is a weight (else it may be NULL);
 *              dx may be dy itself or x itself, with the same pitch
 *   dweight    [head_dim] FP32, overwritten; needed when there is a weight (NULL without one)
 *   workspace  device scratch of sol_qk_rotary_backward_workspace_bytes(head_dim) bytes, 256-byte aligned; needed when
 *              there is a weight.  Two calls that may overlap need one each.
 * The weight gradients are summed in a fixed order: equal inputs give equal bits.  The terms that one GPU thread meets on its
 * walk over the tokens are added in FP32, the sums of different warps in FP64.
 */
typedef struct {
    const void *dy, *x;
    void *dx;
    const void *weight;
    float *dweight;
    int64_t heads, ld_dy, ld_x, ld_dx;
} sol_head_grad_t;
size_t sol_qk_rotary_backward_workspace_bytes(int64_t head_dim);
sol_status_t sol_qk_rotary_backward(const sol_head_grad_t *q, const sol_head_grad_t *k, int64_t rows, int64_t head_dim,
                                    const sol_rotary_t *rotary, float eps, void *workspace, size_t workspace_bytes,
                                    void *stream);

/*
 * Frequencies of one position axis of `dim` rotated columns, computed on the host:
 *     freqs_out[i] = theta^(-2 i / dim), i < dim / 2        (HOST array of doubles), and *scale_out = 1, scaled for
 * contexts `factor` times longer than the model was trained on:
 *   LINEAR  freqs / factor;   NTK  theta replaced by theta * factor^(dim / (dim - 2))  (dim > 2)
 *   YARN    freqs / factor where a pair turns less than beta_slow times over original_length positions, freqs where it
 *           turns more than beta_fast times, a linear ramp over the pair index between; *scale_out = 0.1 ln(factor) + 1
 * dim even and positive, theta > 0, factor >= 1; YARN: theta > 1, original_length > 0, beta_fast >= beta_slow > 0.
 * A caller with several axes calls it once per axis and lays the results side by side.
 */
sol_status_t sol_rotary_frequencies(int64_t dim, double theta, sol_rotary_scaling_t scaling, double factor,
                                    double original_length, double beta_fast, double beta_slow, double *freqs_out,
                                    double *scale_out);

/*
 * BF16 linear, the full-precision stage-2 reference (Section 3.4):
 *     Y[m,n] = bf16_rne( sum_k x[m,k] * w[n,k] + bias[n] ),  FP32 accumulate.
 */
sol_status_t bf16_linear(const void *x_bf16, const void *w_bf16, const void *bias_bf16,
                         void *y_bf16, int64_t M, int64_t N, int64_t K, int64_t ldx,
                         int64_t ldw, int64_t ldy, void *stream);

/*
 * Fused entry: dynamic per-tensor scale of X, quantize X, NVFP4 GEMM against
 * pre-quantized weights, in one call on one stream.
 *   workspace  device scratch of at least sol_nvfp4_linear_workspace_bytes(M, N, K) bytes,
 *              256-byte aligned; holds Q(X) between the kernels; contents undefined after.
 */
sol_status_t nvfp4_quantize_linear(const void *x_bf16, int64_t ldx, const void *wq,
                                   const void *wsf, const float *w_tscale,
                                   const void *bias_bf16, void *y_bf16, int64_t M, int64_t N,
                                   int64_t K, int64_t ldy, void *workspace,
                                   size_t workspace_bytes, void *stream);

/*
 * The fused entry without the amax pass ("delayed" tensor scale): X is quantized with the T the
 * caller carries over from an earlier call on the same activation stream, and the amax of THIS X
 * is collected by the quantizer as a by-product (it computes every block maximum anyway), so the
 * second HBM read of X disappears.  A T that has become too small only saturates more block scales.
 *   scale_state  two floats (device, 8-byte aligned): [0] = T used by this call (> 0; read only),
 *                [1] = running max|x| as an FP32 value, raised by this call with an atomic max
 *   sol_roll_tensor_scale(state): [0] <- max|x| / 2688 (1 if it is 0), [1] <- 0 -- one tiny kernel,
 *                called between denoising steps (or whenever the caller wants T refreshed)
 * Given the same T the result is bit-identical to nvfp4_quantize + nvfp4_linear.
 */
sol_status_t nvfp4_quantize_linear_delayed(const void *x_bf16, int64_t ldx, const void *wq, const void *wsf,
                                           const float *w_tscale, const void *bias_bf16, void *y_bf16, int64_t M,
                                           int64_t N, int64_t K, int64_t ldy, float *scale_state, void *workspace,
                                           size_t workspace_bytes, void *stream);
sol_status_t sol_roll_tensor_scale(float *scale_state, void *stream);

/*
 * The fused entry for HOST activations and outputs (the end-to-end path a caller with data in host
 * memory takes): copies X host -> x_dev, runs nvfp4_quantize_linear, copies y_dev -> Y host, all
 * queued on `stream` (truly asynchronous only if the host buffers are pinned).
 *   x_host, y_host  HOST pointers, BF16 [M, K] / [M, N], pitches ldx / ldy in elements
 *   x_dev, y_dev    device staging buffers, dense [M, K] / [M, N] BF16, 16-byte aligned
 *   weights, bias, workspace: device, as for nvfp4_quantize_linear
 */
sol_status_t nvfp4_quantize_linear_host(const void *x_host, int64_t ldx, const void *wq,
                                        const void *wsf, const float *w_tscale,
                                        const void *bias_bf16, void *y_host, int64_t M, int64_t N,
                                        int64_t K, int64_t ldy, void *x_dev, void *y_dev,
                                        void *workspace, size_t workspace_bytes, void *stream);

/*
 * MXFP4, the OCP format Section 2 sets beside NVFP4: 32 contiguous elements along K under one E8M0
 * scale (a bare exponent: byte b = 2^(b-127)), no tensor-level scale.
 *     scale = 2^(floor(log2 max|x|) - 2), exponent clamped to [-127, 127]; byte 0 for an all-zero block
 *     nibble_k = E2M1_rne_sat(x_k / scale)    (the division is an exact power-of-two scaling)
 * Storage: nibbles as for NVFP4; scales row-major [rows, K/32], or SOL_SF_SWIZZLED_128x4: the same
 * 512-byte chunks of 128 rows x 4 scales (a chunk now spans 128 elements of K), chunk order
 * [ceil(rows/128)][ceil(K/128)], padding 0.  sol_mxfp4_scale_bytes gives the buffer size.
 */
size_t sol_mxfp4_scale_bytes(int64_t rows, int64_t K, sol_sf_layout_t layout);
sol_status_t mxfp4_quantize(const void *x_bf16, int64_t rows, int64_t K, int64_t ldx, void *q_out, void *sf_out,
                            sol_sf_layout_t layout, void *stream);

/*
 * MXFP4 linear: Y[m,n] = bf16_rne( sum_b 2^(ex[m,b] + ew[n,b]) sum_{k in b} qx[m,k] qw[n,k] + bias[n] ),
 * FP32 accumulation in the tensor core (kind::mxf4, two scales per row per K = 64 instruction).
 * Operands as written by mxfp4_quantize with the chunked scale layout; otherwise as nvfp4_linear.
 */
sol_status_t mxfp4_linear(const void *xq, const void *xsf, const void *wq, const void *wsf, const void *bias_bf16,
                          void *y_bf16, int64_t M, int64_t N, int64_t K, int64_t ldy, void *stream);

/*
 * mxfp4_linear whose output leaves as the MXFP4 activations of the next linear (the MXFP4 form of
 * nvfp4_linear_quantized_out): h = bf16_rne(act(Y)), then mxfp4_quantize's mapping along N.
 *   hq_out   [M, N/2] nibbles;  hsf_out  SOL_SF_SWIZZLED_128x4 MXFP4 scales of an [M, N] tensor, every byte written
 *   amax_out nullable running max|h| (FP32 bits, atomic max); N % 128 == 0
 * No tensor scales anywhere: the format has none.  Errors as nvfp4_linear_quantized_out.
 */
sol_status_t mxfp4_linear_quantized_out(const void *xq, const void *xsf, const void *wq, const void *wsf,
                                        const void *bias_bf16, sol_activation_t activation, void *hq_out, void *hsf_out,
                                        float *amax_out, int64_t M, int64_t N, int64_t K, void *stream);

/*
 * The MXFP4 forms of nvfp4_linear_split_out and nvfp4_quantize_into (Section 2 names MXFP4 beside NVFP4;
 * the concatenated input of a single-stream block's second linear, as there): columns [0, n_split) of the
 * linear leave as BF16, columns [n_split, N) pass through the activation and leave as MXFP4 into columns
 * [dest_col0, dest_col0 + N - n_split) of a wider MXFP4 tensor [M, dest_K]; mxfp4_quantize_into quantizes a
 * BF16 tensor [M, K] into columns [dest_col0, dest_col0 + K) of such a tensor and touches no other column.
 *   hq_dest / q_dest  packed nibbles [M, dest_K/2];  hsf_dest / sf_dest  chunked MXFP4 scales of an [M, dest_K] tensor
 *   n_split % 256 == 0;  N - n_split, K, dest_K and dest_col0 multiples of 128 (a scale chunk spans 128 columns).
 * No tensor scale: the format has none.  Errors as the NVFP4 forms.
 */
sol_status_t mxfp4_linear_split_out(const void *xq, const void *xsf, const void *wq, const void *wsf,
                                    const void *bias_bf16, void *y_bf16, int64_t ldy, int64_t n_split,
                                    sol_activation_t activation, void *hq_dest, void *hsf_dest, int64_t dest_K,
                                    int64_t dest_col0, float *amax_out, int64_t M, int64_t N, int64_t K, void *stream);
sol_status_t mxfp4_quantize_into(const void *x_bf16, int64_t M, int64_t K, int64_t ldx, void *q_dest, void *sf_dest,
                                 int64_t dest_K, int64_t dest_col0, void *stream);

/*
 * Stage-1 selection (Section 3.4; Section 4.1 "Rollout Generation": N = 96 candidates per prompt,
 * the 12 best and 12 worst kept, their initial noises preserved) and the group-standardised
 * advantages of the GRPO equation in Section 2, A_i = (R_i - mean) / population std.
 *   rewards        [P, N] FP32 proxy rewards, finite; N <= 4096
 *   seeds          [P, N] 64-bit noise seeds (nullable when seeds_out is null)
 *   idx_out        [P, K] int32: K/2 best candidates in descending order of reward, then the K/2
 *                  worst starting from the lowest; among equal rewards the lower index ranks higher
 *   seeds_out      [P, K] the selected candidates' seeds (nullable)
 *   advantages_out [P, N] FP32 (nullable); statistics in FP64; all zeros when the std is 0
 *   K even, 0 < K <= N.  One block per prompt; indices and seeds are exact.
 */
sol_status_t solrl_select_contrastive(const float *rewards, const uint64_t *seeds, int64_t P, int64_t N, int64_t K,
                                      int32_t *idx_out, uint64_t *seeds_out, float *advantages_out, void *stream);

/*
 * Rank consistency between reference and proxy rewards (appendix "Group-Relative Ranking
 * Consistency"): per prompt
 *   counts_out  [P, 4] int64: concordant minus discordant pairs (ties count 0), sum of squared
 *               rank differences (ordinal ranks, ties to the lower index), candidates in both top-k
 *               sets, candidates in both bottom-k sets -- all exact
 *   metrics_out [P, 4] FP32 (nullable): Kendall tau-a = count / (N(N-1)/2), Spearman rho =
 *               1 - 6 sum d^2 / (N(N^2-1)), top-k and bottom-k match rates
 *   2 <= N <= 2048, 0 < k <= N.
 */
sol_status_t solrl_rank_consistency(const float *rewards_ref, const float *rewards_proxy, int64_t P, int64_t N,
                                    int64_t k, int64_t *counts_out, float *metrics_out, void *stream);

/*
 * (No counterpart in the paper: an addition for callers that cannot allocate device memory.)
 *
 * Same computation and result as nvfp4_quantize_linear, but without a workspace argument: the
 * scratch for the quantized activations lives in a fixed 64 MiB device array that is part of the
 * library image, so the call performs no device allocation of any kind.  It is meant for callers
 * that are handed input and output buffers only, or that run after their memory pool has been
 * frozen (serving loops, plugins, frameworks that forbid allocation once set up).
 *   - Problems whose scratch (sol_nvfp4_linear_workspace_bytes(M, N, K)) exceeds
 *     sol_nvfp4_static_scratch_bytes() are rejected with SOL_ERR_WORKSPACE_TOO_SMALL; nothing is launched.
 *   - The first call on each device looks up the array's device address (with that device current);
 *     make that first call outside any stream capture.
 *   - All calls on a device share the one array, which keeps the previous call's contents.  Calls
 *     that may overlap on the GPU (different streams, or several host threads) race on it and give
 *     undefined results; serialise them.  Every GPU that loads the library holds the array until
 *     the process exits.
 */
size_t sol_nvfp4_static_scratch_bytes(void);
sol_status_t nvfp4_quantize_linear_static(const void *x_bf16, int64_t ldx, const void *wq,
                                          const void *wsf, const float *w_tscale,
                                          const void *bias_bf16, void *y_bf16, int64_t M, int64_t N,
                                          int64_t K, int64_t ldy, void *stream);

/*
 * Device-side waits in the GEMM kernels are bounded; a wait that runs out records a code
 * in a device status word and the kernel returns.  This call synchronises `stream`, reads
 * that word, clears it, and returns SOL_ERR_TIMEOUT if it was set, SOL_ERR_CUDA if the
 * stream reported an error, SOL_OK otherwise.  `detail_out` (host, nullable) receives the
 * raw word.
 */
sol_status_t sol_last_device_status(void *stream, uint32_t *detail_out);

/*
 * (No counterpart in the paper: failure detection of the kernels themselves.)
 *
 * Sets, for the current device, the limit of every bounded device-side wait in SM clock cycles
 * (default 4e9, about two seconds; `cycles` <= 0 restores the default).  Synchronous: it copies
 * eight bytes to the device and affects kernels launched afterwards.  A wait that exceeds the limit
 * makes its kernel leave through the normal teardown (outputs incomplete) and is reported by
 * sol_last_device_status as SOL_ERR_TIMEOUT; the context stays usable.
 */
sol_status_t sol_set_wait_limit_cycles(int64_t cycles);

/*
 * Test hook for that path (no counterpart in the paper).  While `on` is non-zero on the current
 * device, the load-issuing warps of the CTA-pair GEMM kernels (M > 128: nvfp4_linear, mxfp4_linear,
 * bf16_linear and the entries built on them) and of sol_attention_blocks issue no loads, so every consumer wait of such a launch
 * runs into the wait limit: nothing traps, faults or spins without bound, the kernel returns with Y
 * unwritten (queries with empty lists aside) and the status word set.  The few-row linears (nvfp4_matvec, mxfp4_matvec) then load their first codes, but x is
 * never handed to the products, with the same outcome.  Use it with a short limit (about 1e6 cycles) and switch it off
 * again; it is not meant for anything but exercising the time-out path.
 */
sol_status_t sol_test_hold_loads(int on);

#ifdef __cplusplus
}
#endif
#endif /* SOL_NVFP4_H_ */
