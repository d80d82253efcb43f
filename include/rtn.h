/*
 * rtn.h -- C ABI of librtn_b200: the forward ternary-by-ternary contraction of the
 * Reparameterized Ternary Network (RTN, arXiv 1912.02057) on NVIDIA B200 (sm_100a).
 *
 * Path: ternarize + pack (Eq. 1-3, Table 1)  ->  packed ternary GEMM / implicit-GEMM conv2d
 * (Eq. 9)  ->  affine scale/offset epilogue (Eq. 10, generalised to a weight offset).
 *
 * Conventions
 *   - Every data pointer is a DEVICE pointer unless its comment says "host".  The caller owns
 *     every input and output buffer.  The library keeps no state besides one device status word (see
 *     rtn_last_device_status) and, per device, the fixed scratch array of rtn_ternary_conv2d_noalloc.
 *     Convolutions that take the two-kernel path (rtn_conv_kernel_launches / rtn_conv_next_kernel_launches
 *     say which) borrow a scratch buffer from the stream-ordered allocator for the duration of the call
 *     (cudaMallocAsync / cudaFreeAsync on `stream`), and so does the tensor-core GEMM for its expanded
 *     operands (rtn_gemm_kernel_launches); nothing else is allocated.
 *   - `stream` is a cudaStream_t passed as void* (NULL = the default stream).  Calls only
 *     enqueue work and return without synchronising, except rtn_pack_weights and
 *     rtn_last_device_status, which synchronise the stream.
 *   - Errors are return codes; argument errors are found on the host before any launch and
 *     leave every buffer untouched.  Nothing throws, aborts or traps.
 *   - Codes: x (activation) and w (weight) in {-1, 0, +1}.  S_xw = sum_k x*w, S_x = sum_k x,
 *     S_w = sum_k w (exact int32; |S| <= K <= 2^24).
 *
 * Packed operand format (Table 1 and the bit-plane vectors W1, W2, A1, A2 of Eq. 9)
 *   A row of K codes occupies ceil(K/128) blocks of 32 bytes (2 bits per code):
 *     block j, bytes  0..15 : plane 1 ("non-zero" bit) of codes 128j .. 128j+127
 *     block j, bytes 16..31 : plane 2 ("sign" bit, 1 = positive) of the same codes
 *   Code 128j+i sits in bit (i mod 8) of byte (i div 8) of its plane (little-endian words:
 *   bit (i mod 32) of 32-bit word (i div 32)).  Table 1: 00 -> 0, 01 -> 0, 10 -> -1, 11 -> +1.
 *   The packers emit the canonical zero 00 and zero-fill positions past K; every consumer also
 *   accepts 01 as zero.  Rows are contiguous: row stride = rtn_packed_row_bytes(K).  Packed
 *   buffers must be 16-byte aligned.
 *   Convolution filters [N][C][kh][kw] are packed as rows of length rtn_conv_packed_k(C,kh,kw)
 *   = kh*kw*Cw, Cw = C rounded up to 32, in (kh, kw, c) order with zero codes in the channel
 *   padding (the im2col patch of the paper's "Methodology" section, channel innermost).
 */
#ifndef RTN_H_
#define RTN_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    RTN_OK = 0,
    RTN_ERR_NULL = 1,           /* a required pointer is NULL                                  */
    RTN_ERR_SHAPE = 2,          /* a size is <= 0, too large, or inconsistent                  */
    RTN_ERR_ALIGN = 3,          /* a buffer misses its alignment                               */
    RTN_ERR_VALUE = 4,          /* a weight code outside {-1,0,+1}, or a bad enum value        */
    RTN_ERR_UNSUPPORTED = 5,    /* the requested variant cannot run this shape                 */
    RTN_ERR_CUDA = 6,           /* a CUDA runtime call failed (launch, attribute, copy)        */
    RTN_ERR_DEVICE_TIMEOUT = 7, /* a bounded device-side wait gave up (see last_device_status) */
    RTN_ERR_DEVICE_INDEX = 8    /* an index read on the device was out of range (see last_device_status) */
} rtn_status;

/* Treatment of filter taps that fall outside the image.  The paper never mentions padding; the
 * constant term C of Eq. 10 can be stored ahead of time, as the paper has it, only under
 * RTN_PAD_CODE_ZERO: an outside tap has CODE 0, i.e. real value a_offset, and S_w and K cover
 * all C*kh*kw taps.  RTN_PAD_VALUE_ZERO makes an outside tap contribute nothing (what a
 * floating-point conv2d on the de-quantised tensor does): S_w and K then cover inside taps only. */
typedef enum { RTN_PAD_CODE_ZERO = 0, RTN_PAD_VALUE_ZERO = 1 } rtn_pad_mode;

/* Kernel family.  POPC: Eq. 9 evaluated with AND/XOR/popcount on the packed planes.
 * I8: planes expanded to int8 in shared memory and contracted on the tensor cores
 * (tcgen05 kind::i8).  AUTO picks per shape.  Both give identical integers. */
typedef enum { RTN_VARIANT_AUTO = 0, RTN_VARIANT_POPC = 1, RTN_VARIANT_I8 = 2 } rtn_variant;

/* Bytes of one packed row of K codes: ceil(K/128)*32.  0 if K <= 0. */
size_t rtn_packed_row_bytes(int64_t K);
/* Bytes of a packed operand of `rows` rows. */
size_t rtn_packed_bytes(int64_t rows, int64_t K);
/* Length of a packed convolution filter row: kh*kw*roundup(C,32).  0 on bad arguments. */
int64_t rtn_conv_packed_k(int64_t C, int64_t kh, int64_t kw);
/* Output extent of a convolution: (in + 2*pad - k)/stride + 1 (0 if not positive). */
int64_t rtn_conv_out_dim(int64_t in, int64_t k, int64_t stride, int64_t pad);

/* Weight ternary codes -> packed planes and code sums (Table 1; W1, W2 of Eq. 9; the
 * pre-stored 1 (x) W^t of Eq. 10).  Offline step.
 *   w_codes  int8 [N][C][kh][kw] in {-1,0,+1} (a GEMM weight [N][K] is C=K, kh=kw=1)
 *   w_packed out, N rows of rtn_conv_packed_k(C,kh,kw) codes, 16-byte aligned
 *   w_sum    out, int32 [1 + kh*kw][N]: row 0 = S_w over all taps and channels, row 1+t = sum
 *            over the channels of tap t = i*kw + j (used by RTN_PAD_VALUE_ZERO at borders)
 * Synchronises `stream`.  Returns RTN_ERR_VALUE if any code is outside {-1,0,+1} (outputs are
 * then unspecified). */
rtn_status rtn_pack_weights(const int8_t* w_codes, int64_t N, int64_t C, int64_t kh, int64_t kw,
                            void* w_packed, int32_t* w_sum, void* stream);

/* fp32 activations -> ternary codes (Eq. 3) -> packed planes (Table 1), plus S_x per row.
 *   a        fp32 [M][K] row-major
 *   t_lo,t_hi  n_thr thresholds (n_thr == 1: per layer; n_thr == K: per input feature k).
 *            code = +1 if a > t_hi, else -1 if a < t_lo, else 0; comparisons are strict and
 *            done in fp32, so a value equal to a threshold, and a NaN, code to 0.  With the BN
 *            transform k*a+b of Eq. 2 (k > 0): t_hi = (0.5-b)/k, t_lo = -(0.5+b)/k.
 *   a_packed out, M packed rows of K codes, 16-byte aligned
 *   a_sum    out, int32 [M] = S_x (may be NULL) */
rtn_status rtn_ternarize_pack_act(const float* a, int64_t M, int64_t K,
                                  const float* t_lo, const float* t_hi, int64_t n_thr,
                                  void* a_packed, int32_t* a_sum, void* stream);

/* Packed ternary GEMM with the affine epilogue (Eq. 9 then Eq. 10 with a weight offset):
 *   out[m][n] = a_s*w_s*S_xw + a_s*w_o*S_x[m] + a_o*w_s*S_w[n] + K*a_o*w_o
 *             = sum_k (a_s*x[m][k] + a_o) * (w_s*w[n][k] + w_o)
 *   a_packed M rows, w_packed N rows of K codes (w_packed from rtn_pack_weights with C=K)
 *   a_sum    int32 [M] (S_x), w_sum int32 [N] (row 0 of rtn_pack_weights' w_sum)
 *   a_scale,a_offset  n_aparam floats: 1 (per layer: gamma, beta of Eq. 4) or M (per row)
 *   w_scale,w_offset  n_wparam floats: 1 or N (per output channel: alpha of Eq. 5; the paper
 *                     has w_offset = 0)
 *   out      fp32 [M][N] row-major
 *   dbg_acc  NULL, or int32 [M][N] that receives the raw S_xw */
rtn_status rtn_ternary_gemm(const void* a_packed, const int32_t* a_sum,
                            const void* w_packed, const int32_t* w_sum,
                            int64_t M, int64_t N, int64_t K,
                            const float* a_scale, const float* a_offset, int64_t n_aparam,
                            const float* w_scale, const float* w_offset, int64_t n_wparam,
                            float* out, int32_t* dbg_acc, rtn_variant variant, void* stream);

/* Ternary conv2d as an implicit GEMM (im2col never materialised), input ternarized in-kernel:
 *   x        fp32 [B][C][H][W]; code per Eq. 3 with thresholds per layer (n_thr == 1) or per
 *            input channel (n_thr == C)
 *   w_packed,w_sum  from rtn_pack_weights(w_codes, N, C, kh, kw)
 *   a_scale,a_offset  per-layer gamma, beta (by value); w_scale,w_offset as in the GEMM
 *   out      fp32 [B][N][Ho][Wo], Ho = rtn_conv_out_dim(H,kh,stride,pad), same for Wo
 *   dbg_acc  NULL, or int32 of out's shape that receives the raw S_xw
 * out[b][n][ho][wo] = sum over taps of (a_s*x + a_o)*(w_s*w + w_o) under pad_mode's rule.
 * Stream order: x, out and dbg_acc are ordered after all earlier work of the stream, as usual.  The
 * tensor-core kernels start their set-up while the stream's previous kernel is still draining
 * (programmatic dependent launch), and that set-up reads the layer's parameters: t_lo, t_hi,
 * w_packed, w_sum, w_scale, w_offset must therefore not be buffers that an earlier
 * rtn_ternary_conv2d call of the same stream writes (its out or dbg_acc), unless the stream was
 * synchronized or ran another kernel in between (they are constants of the layer in every intended
 * use). */
rtn_status rtn_ternary_conv2d(const float* x, int64_t B, int64_t C, int64_t H, int64_t W,
                              const float* t_lo, const float* t_hi, int64_t n_thr,
                              const void* w_packed, const int32_t* w_sum,
                              int64_t N, int64_t kh, int64_t kw, int64_t stride, int64_t pad,
                              rtn_pad_mode pad_mode, float a_scale, float a_offset,
                              const float* w_scale, const float* w_offset, int64_t n_wparam,
                              float* out, int32_t* dbg_acc, rtn_variant variant, void* stream);

/* Variant of rtn_ternary_conv2d that allocates nothing (the paper has no counterpart; it is for
 * callers that must not touch an allocator on the hot path).  It always takes the two-kernel
 * tensor-core path (int8 codes of the input in a scratch buffer, filter bank split over CTAs),
 * the path rtn_ternary_conv2d chooses for strided 3x3 layers and, by its cost estimate, for some 1x1
 * stride-2 layers and wide layers at large batch, and gives the same bits.  The scratch is one array of 16 MiB per device, part of the library's image; the
 * call performs no cudaMalloc, cudaMallocAsync, cudaFree or other allocating routine.
 *   - RTN_ERR_UNSUPPORTED: a shape the path does not take (e.g. 3x3 with stride 3), or a layer whose codes
 *     (about B*(H+2pad)*(W+2pad)*(C rounded up to 32) bytes) exceed the array.
 *   - The array is shared by every caller on the device: two calls whose kernels may overlap in
 *     time (different streams, or different host threads on different streams) race on it.
 *     Issue them on one stream, or order them with events.
 *   - The first call on a device does set-up (address of the array, kernel attributes) and must come
 *     before any stream capture; later calls can be captured.
 * Arguments, layouts and the stream-order rule are those of rtn_ternary_conv2d. */
rtn_status rtn_ternary_conv2d_noalloc(const float* x, int64_t B, int64_t C, int64_t H, int64_t W,
                              const float* t_lo, const float* t_hi, int64_t n_thr,
                              const void* w_packed, const int32_t* w_sum,
                              int64_t N, int64_t kh, int64_t kw, int64_t stride, int64_t pad,
                              rtn_pad_mode pad_mode, float a_scale, float a_offset,
                              const float* w_scale, const float* w_offset, int64_t n_wparam,
                              float* out, int32_t* dbg_acc, void* stream);

/* Ternary conv2d that hands its result to the next layer from its epilogue (Eq. 10 with its phi;
 * section "Activation Ternarization": BN sits after the ReLU, so the next layer's BN folds into
 * that layer's threshold pair of Eq. 3).  Per output value:
 *     y    = phi(affine form of rtn_ternary_conv2d) + skip      phi = ReLU if relu == 1, else identity
 *     out        <- y (fp32)                                    if out != NULL
 *     out_packed <- +1 if y > next_t_hi, -1 if y < next_t_lo, else 0, as a packed pixel row
 *                                                               if out_packed != NULL
 * so a layer whose only consumer is the next ternary layer writes 2 bits per value instead of 32.
 *   x ... n_wparam   as in rtn_ternary_conv2d
 *   skip        NULL, or fp32 [B][N][Ho][Wo] (the residual block's skip connection), added after phi
 *   out         NULL, or fp32 [B][N][Ho][Wo]
 *   next_t_lo, next_t_hi   thresholds of the NEXT layer's ternarizer: n_next_thr = 1 (per layer) or N
 *               (per channel of this layer's output); strict fp32 comparisons on the fp32 y, +1 first;
 *               required when out_packed != NULL
 *   out_packed  NULL, or B*Ho*Wo packed rows of N codes each (rtn_packed_bytes(B*Ho*Wo, N) bytes,
 *               16-byte aligned): pixel (b, ho, wo) is row (b*Ho + ho)*Wo + wo, channel n is code n of
 *               the row; canonical zeros, zero fill past N.  This is the x_packed of
 *               rtn_ternary_conv2d_packed.
 *   dbg_acc     NULL, or int32 [B][N][Ho][Wo] raw S_xw
 * At least one of out, out_packed must be given.  Runs on the tensor cores only: the one-kernel variant with
 * the filters resident in shared memory where they fit (stride 1), else the streamed-filter variant or the
 * two-kernel variant with int8 codes in a scratch buffer from the stream-ordered allocator
 * (rtn_conv_next_kernel_launches says how many launches a shape takes); RTN_ERR_UNSUPPORTED for shapes none of
 * the three takes (e.g. 3x3 with stride 3).  Stream-order rule as for rtn_ternary_conv2d; the next-layer
 * thresholds count as parameters of the layer. */
rtn_status rtn_ternary_conv2d_fused(const float* x, int64_t B, int64_t C, int64_t H, int64_t W,
                                    const float* t_lo, const float* t_hi, int64_t n_thr,
                                    const void* w_packed, const int32_t* w_sum,
                                    int64_t N, int64_t kh, int64_t kw, int64_t stride, int64_t pad,
                                    rtn_pad_mode pad_mode, float a_scale, float a_offset,
                                    const float* w_scale, const float* w_offset, int64_t n_wparam,
                                    int relu, const float* skip, float* out,
                                    const float* next_t_lo, const float* next_t_hi, int64_t n_next_thr,
                                    void* out_packed, int32_t* dbg_acc, void* stream);

/* The same layer on an input that is already ternary: packed pixel rows (Table 1 planes; A1, A2 of
 * Eq. 9 with the channel as the fast index), as written by the out_packed of the layer before or by
 * rtn_ternarize_pack_act on an fp32 [B*H*W][C] (NHWC) matrix.
 *   x_packed    B*H*W packed rows of C codes: pixel (b, h, w) is row (b*H + h)*W + w; 16-byte aligned
 * Everything else as in rtn_ternary_conv2d_fused (there are no thresholds for the input: it is codes). */
rtn_status rtn_ternary_conv2d_packed(const void* x_packed, int64_t B, int64_t C, int64_t H, int64_t W,
                                     const void* w_packed, const int32_t* w_sum,
                                     int64_t N, int64_t kh, int64_t kw, int64_t stride, int64_t pad,
                                     rtn_pad_mode pad_mode, float a_scale, float a_offset,
                                     const float* w_scale, const float* w_offset, int64_t n_wparam,
                                     int relu, const float* skip, float* out,
                                     const float* next_t_lo, const float* next_t_hi, int64_t n_next_thr,
                                     void* out_packed, int32_t* dbg_acc, void* stream);

/* The paper's comparison workload (section "Efficient Computation Pattern", Table 1's last column and the
 * DoReFa-Net pattern it cites): 2-bit quaternary values q = 2*b1 + b2 in {0,1,2,3}, dot products by AND
 * between each bit plane of the two inputs, popcount, power-of-two shifts and four partial sums:
 *     x.w = 4 bC(X1&W1) + 2 bC(X1&W2) + 2 bC(X2&W1) + bC(X2&W2).
 * Same packed operand format, with plane 1 = first bit (weight 2) and plane 2 = second bit (weight 1).
 *
 * rtn_pack_quaternary: q_values uint8 [rows][K] in {0..3} -> packed rows (16-byte aligned).  Synchronises
 *   `stream`; RTN_ERR_VALUE if a value is above 3 (output then unspecified).
 * rtn_quaternary_gemm: out[m][n] = sum_k x[m][k] * w[n][k], exact int32 ([M][N] row-major; <= 9 K). */
rtn_status rtn_pack_quaternary(const uint8_t* q_values, int64_t rows, int64_t K, void* packed, void* stream);
rtn_status rtn_quaternary_gemm(const void* a_packed, const void* w_packed, int64_t M, int64_t N, int64_t K,
                               int32_t* out, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Operators of a ternary language-model layer around the packed products (the paper has no counterpart).
 * Common to them: fp32, bf16 and fp16 tensors (arithmetic, norms, sums and states in fp32, one rounding at the
 * end; rtn_decay_attention's products on the tensor cores round their operands as it says there); strides count elements; a call with no tokens (M, T or B of 0) returns RTN_OK and launches nothing; calls
 * only enqueue and can be captured in a graph (after a first call that sets kernel attributes).  Scratch (the operands of a
 * tensor-core linear layer, the segment states of a long prompt) comes, stream-ordered, from a memory pool per device that the library
 * makes at the first use and that keeps its memory from call to call, the most that was in use at once (a tensor-core linear layer
 * takes up to 2 GiB for its expanded operands), until rtn_release_scratch.
 * ---------------------------------------------------------------------------------------------- */
typedef enum { RTN_F32 = 0, RTN_BF16 = 1, RTN_F16 = 2 } rtn_dtype;
typedef enum { RTN_ACT_NONE = 0, RTN_ACT_RELU = 1, RTN_ACT_GELU = 2 /* erf */, RTN_ACT_GELU_TANH = 3, RTN_ACT_SILU = 4 } rtn_activation;
typedef enum { RTN_ROTARY_HALF = 0 /* pairs (i, i + R/2) */, RTN_ROTARY_INTERLEAVED = 1 /* pairs (2i, 2i + 1) */ } rtn_rotary_layout;
typedef enum { RTN_ROTARY_SCALE_NONE = 0, RTN_ROTARY_SCALE_LINEAR = 1, RTN_ROTARY_SCALE_BASE = 2, RTN_ROTARY_SCALE_PARTS = 3 } rtn_rotary_scaling;

/* Ternary linear layer: the packed product with bias, activation and residual in its epilogue.
 *     out[m][n] = act( sum_k (a_s x[m][k] + a_o)(w_s w[n][k] + w_o) + bias[n] ) + residual[m][n]
 *   a_packed ... n_wparam   as in rtn_ternary_gemm
 *   bias        NULL, or fp32 [N]
 *   residual    NULL, or [M][N] of `dtype`, rows residual_stride elements apart; may be `out` itself (same stride), to
 *               add a layer to a residual stream in place; no other overlap
 *   out         [M][N] of `dtype`, rows out_stride >= N elements apart
 * Few rows (up to 8, more where the product is small) run on a bit-plane kernel that streams the weights, some rows on a tensor-core
 * kernel that expands its own operands, both one launch; larger products take two where the operands are expanded ahead (at least two
 * row tiles of 128 or 256), else one. */
rtn_status rtn_ternary_linear(const void* a_packed, const int32_t* a_sum,
                              const void* w_packed, const int32_t* w_sum,
                              int64_t M, int64_t N, int64_t K,
                              const float* a_scale, const float* a_offset, int64_t n_aparam,
                              const float* w_scale, const float* w_offset, int64_t n_wparam,
                              const float* bias, rtn_activation act, const void* residual, int64_t residual_stride,
                              void* out, int64_t out_stride, rtn_dtype dtype, void* stream);

/* Table of a rotation: fp32 [rows][R], row p = cos(p f_i), i < R/2, then sin(p f_i), each times `amplitude`.
 * R even, >= 2.  f_i = base^(-2i/R) and, for contexts longer than the one a model was trained on,
 *   LINEAR  f_i / factor
 *   BASE    base * factor^(R/(R-2)) in place of base (R > 2)
 *   PARTS   f_i where it makes at least `high` turns over `original_context` positions, f_i / factor where it makes at
 *           most `low`, a linear ramp in the turns between (high > low)
 * Angles are computed in double.  factor, original_context, low, high are read by the kinds that name them. */
rtn_status rtn_rotary_table(float* table, int64_t rows, int64_t R, double base, rtn_rotary_scaling scaling, double factor,
                            double original_context, double low, double high, double amplitude, void* stream);

/* Norms of the query and key heads and their rotation by position, in one pass:
 *     y = x w / sqrt(mean(x^2) + eps);   the first R of the D elements rotated by row positions[t] of the table
 *   q, k        [T][Hq][D] and [T][Hk][D] of `dtype`: token t, head h starts at t*token + h*head, elements adjacent
 *   out_q,out_k same shapes with strides of their own; out_q == q with q's strides (in place) is allowed, also
 *               for k, no other overlap
 *   q_weight, k_weight   fp32 [D], or both NULL: no norm, the rotation alone
 *   table       fp32 [table_rows][R] (rtn_rotary_table), 4-byte aligned; NULL with R = 0: the norms alone
 *   positions   int64 [T], or NULL: token t is at position t
 * Hk = 0 (k NULL) is allowed.  D <= 1024, R even, R <= D.  A position outside the table makes the token's heads NaN, and
 * rtn_last_device_status reports RTN_ERR_DEVICE_INDEX once. */
rtn_status rtn_qk_norm_rotary(const void* q, int64_t q_token, int64_t q_head, const void* k, int64_t k_token, int64_t k_head,
                              void* out_q, int64_t oq_token, int64_t oq_head, void* out_k, int64_t ok_token, int64_t ok_head,
                              int64_t T, int64_t Hq, int64_t Hk, int64_t D, int64_t R, rtn_rotary_layout layout,
                              const float* q_weight, const float* k_weight, float eps,
                              const float* table, int64_t table_rows, const int64_t* positions, rtn_dtype dtype, void* stream);

/* Linear attention with a decay for each head, over whole prompts of different lengths.  Per sequence and head h:
 *     S_t = exp(log_decay[h]) S_{t-1} + k_t v_t^T,      out_t = scale q_t^T S_t
 *   q           [total][H][Dk], k [total][Hk][Dk], v [total][Hk][Dv] of `dtype` with token and head strides, elements
 *               adjacent; H a multiple of Hk, query head h reads key head h / (H/Hk)
 *   out         [total][H][Dv] of `dtype`, strides of its own, no overlap with the inputs
 *   log_decay   fp32 [H], natural logarithm, <= 0 in every intended use
 *   start       int32 [B+1], on the device: sequence b has tokens start[b] .. start[b+1]-1; lengths of 0 are allowed
 *   max_len     at least the longest length (sizes the grid)
 *   state       fp32 [n_slots][H][Dk][Dv] holding S before the first token, or NULL: zero
 *   state_out   same shape, receives S after the last token; may be `state` (in place).  Required.
 *   slots       int32 [B] (on the device): sequence b's state is slots[b]; the live slots are distinct; a negative slot
 *               is a padding entry: its out rows become zero and no state is read or written.  NULL: slot b
 * Dk, Dv <= 256.  bf16 tensors with Dk = Dv = 64 or 128, 16-byte rows and prompts of more than 16 tokens run on the tensor cores in chunks of
 * 128 tokens: there the weighted scores and the state in its product with q are rounded to 16 bits (two bf16 terms) and sums are the tensor
 * core's (fp32, towards zero), so an output is off by up to 2^-15 of its terms' magnitudes beside its own rounding (0.24 % of outputs are not the
 * bf16 value nearest to the exact one, 0.02 to 0.05 % where all is fp32); what is
 * added to the state keeps 24 bits, and the state is fp32 throughout.  Everything else runs token by token in fp32, with k scaled by up to
 * 2^8 and q by down to 2^-8 under steep decays.
 * A value that is not finite reaches no token before its own: in v it makes that column of the head not finite
 * (NaN or infinite) from its token on, in k or the state every column, in q its own token's row.
 * Bounds that do not fit (a decreasing start, a length over max_len, a slot >= n_slots) make the kernel
 * skip the sequence (its rows of out are not written), and rtn_last_device_status reports RTN_ERR_DEVICE_INDEX once. */
rtn_status rtn_decay_attention(const void* q, int64_t q_token, int64_t q_head, const void* k, int64_t k_token, int64_t k_head,
                               const void* v, int64_t v_token, int64_t v_head, void* out, int64_t o_token, int64_t o_head,
                               int64_t total, int64_t B, const int32_t* start, int64_t max_len,
                               int64_t H, int64_t Hk, int64_t Dk, int64_t Dv, const float* log_decay, float scale,
                               const float* state, float* state_out, const int32_t* slots, int64_t n_slots,
                               rtn_dtype dtype, void* stream);

/* The same for one new token of each of B sequences (token b belongs to sequence b), in fp32.  A slot >= n_slots makes the token's rows of
 * out NaN. */
rtn_status rtn_decay_attention_step(const void* q, int64_t q_token, int64_t q_head, const void* k, int64_t k_token, int64_t k_head,
                                    const void* v, int64_t v_token, int64_t v_head, void* out, int64_t o_token, int64_t o_head,
                                    int64_t B, int64_t H, int64_t Hk, int64_t Dk, int64_t Dv, const float* log_decay, float scale,
                                    const float* state, float* state_out, const int32_t* slots, int64_t n_slots,
                                    rtn_dtype dtype, void* stream);

/* ------------------------------------------------------------------------------------------------
 * A layer of routed ternary experts: the choice of experts, their products, and the norms around a block.  What is said of the layer
 * operators above holds for them as well.
 * ---------------------------------------------------------------------------------------------- */
typedef enum { RTN_SCORE_SOFTMAX = 0, RTN_SCORE_SIGMOID = 1 } rtn_score;
typedef enum { RTN_GATE_LINEAR = 0, RTN_GATE_SIGMOID = 1, RTN_GATE_SILU = 2 } rtn_gate;

/* Choice of top_k of E experts for each of T tokens, and the plan of the rows that the experts work on.
 *     s = softmax or sigmoid of the token's logits;  c = s + bias;  out of the kept groups, the top_k largest c
 *     weight = weight_scale * s   (each divided by the sum of the chosen ones' s where `renormalise`)
 *   logits      [T][E] of `dtype`, rows logits_stride elements apart
 *   bias        NULL, or fp32 [E]: moves the choice, not the weights
 *   groups      E / groups consecutive experts each; a group's value is the sum of its group_top largest c; the kept_groups groups of the
 *               largest values stay.  1 group: no such step
 *   experts     int32 [T][top_k], in the order of c, largest first
 *   weights     fp32 [T][top_k]
 *   start, tokens, place   NULL (all three), or the plan: the T*top_k (token, choice) pairs as rows sorted by expert, within an expert by
 *               token.  Expert e has rows start[e] .. start[e+1]-1 (int32 [E+1]); row r is of token tokens[r] (int32 [T*top_k]); choice j of
 *               token t is row place[t][j] (int32 [T][top_k])
 * Choices are those of exact arithmetic (a c that fp32 cannot tell from another is computed in double, and what that leaves open in pairs of
 * doubles, where a score keeps 47 bits of its distance to 0 and to 1; what is equal there goes by the logit); of equal ones the lowest
 * index comes first, for groups too.  A logit of -inf or NaN (or a bias of it) is never chosen, and +inf counts as the largest finite
 * value; a token with fewer experts to choose has -1, weight 0 and place -1 in the rest, and the rows from start[E] on are not written.
 * E <= 1024, groups <= 32 and a divisor of E, top_k <= 32 and <= the experts in the kept groups. */
rtn_status rtn_route_experts(const void* logits, int64_t logits_stride, int64_t T, int64_t E, rtn_dtype dtype, rtn_score score,
                             const float* bias, int64_t groups, int64_t kept_groups, int64_t group_top, int64_t top_k,
                             int renormalise, float weight_scale, int32_t* experts, float* weights,
                             int32_t* start, int32_t* tokens, int32_t* place, void* stream);

/* The experts' ternary products.  Expert e has rows start[e] .. start[e+1]-1 of R, a row's input is packed row tokens[r]:
 *     y[r][n] = sum_k (a_s x[tokens[r]][k] + a_o)(w_s w[e][n][k] + w_o) + bias[e][n]
 *     out[r][i] = act(y[r][i])                   F = N outputs, or
 *     out[r][i] = act(y[r][i]) * y[r][F + i]     F = N / 2 outputs where `gated`
 *   a_packed, a_sum, a_scale, a_offset   as in rtn_ternary_gemm, for T input rows (n_aparam 1 or T)
 *   tokens      int32 [R], or NULL: row r is input row r (R = T)
 *   start       int32 [E+1], on the device (rtn_route_experts); rows outside every expert are left as they were
 *   w_packed    E * N packed rows of K codes, w_sum int32 [E*N] (row 0 of rtn_pack_weights' w_sum); w_scale, w_offset: n_wparam 1 or E*N
 *   bias        NULL, or fp32 [E][N]
 *   out         NULL, or [R][F] of `dtype`, rows out_stride >= F elements apart
 *   out_packed, out_sum   NULL (both), or the codes of the outputs against thresholds, R packed rows of F codes and their sums, as
 *               rtn_ternarize_pack_act gives them: what the next product reads.  t_lo, t_hi: n_thr 1 or E.  They are the codes of the exact
 *               output (one that fp32 cannot tell from a threshold is computed in double; products of parameters that fall below fp32's normal
 *               range keep what it keeps of them); out and out_packed may both be given
 * Values are worked out in fp32 and rounded to `dtype` once; RTN_ACT_SILU by approximations, within 6 units of 2^-24 |y|.
 * Few rows run on a bit-plane kernel that streams the weights, others on the tensor cores (with scratch of R * K / 2 bytes, K rounded up to
 * 256).  Bounds that do not fit (a decreasing start, or one outside 0 .. R) leave the expert's outputs as they were, a token out of
 * range makes its row NaN (codes 0), and rtn_last_device_status reports RTN_ERR_DEVICE_INDEX once.  After such bounds the sums, and
 * rows outside start[0] .. start[E], are not to be relied on. */
rtn_status rtn_ternary_experts(const void* a_packed, const int32_t* a_sum, int64_t T, const int32_t* tokens, const int32_t* start, int64_t R,
                               const void* w_packed, const int32_t* w_sum, int64_t E, int64_t N, int64_t K,
                               const float* a_scale, const float* a_offset, int64_t n_aparam,
                               const float* w_scale, const float* w_offset, int64_t n_wparam, const float* bias,
                               rtn_activation act, int gated, void* out, int64_t out_stride, rtn_dtype dtype,
                               const float* t_lo, const float* t_hi, int64_t n_thr, void* out_packed, int32_t* out_sum, void* stream);

/* The norms after one block and before the next, with the block's gate and residual, in one pass over T tokens of W values:
 *     y = branch[t],  or  sum_j weights[t][j] branch[place[t][j]]  (the experts' weighted sum; a negative place adds nothing)
 *     u = y post_weight / sqrt(mean(y^2) + eps)                    (post_weight NULL: u = y)
 *     h = residual + scale * g(gate) * u                           (each NULL: left out)
 *     n = h norm_weight / sqrt(mean(h^2) + eps)                    (norm_weight NULL: n = h)
 *   branch      [R][W] of `dtype`, or NULL: h = residual
 *   place       int32 [T][k] with k <= 32, or NULL with k = 0: row t, R = T;  weights fp32 [T][k], or NULL: ones
 *   gate        [T][W] of `dtype`, g by gate_kind: itself, sigmoid(z) or z sigmoid(z);  scale fp32, n_scale 1 or W values
 *   residual    [T][W] of `stream_dtype`
 *   stream_out  NULL, or h in `stream_dtype`; may be `residual` (same stride), no other overlap
 *   normed      NULL, or n in `dtype` (n is computed from h before its rounding)
 *   out_packed, out_sum   NULL (both), or n's codes, T packed rows of W codes and their sums (t_lo, t_hi: n_thr 1 or W); they are the codes of
 *               the exact n (of double: a logistic function below its range is 0; factors whose product falls below fp32's normal range keep
 *               what it keeps of them)
 * h and n as values are worked out in fp32, squares too: behind post_weight or norm_weight a row is 0 where the mean of its squares is beyond fp32 (values
 * above 1.8e19), and without an eps to speak of it loses digits where that is below 1e-30.  Their codes are not touched by this.
 * Rows of every tensor are `*_stride` elements apart (0 repeats a row of an input).  W <= 16384.  A place >= R makes the token's row NaN
 * (codes 0), and rtn_last_device_status reports RTN_ERR_DEVICE_INDEX once.  With places, R may be 0 (branch is not read, and may be NULL). */
rtn_status rtn_block_norm(const void* branch, int64_t branch_stride, int64_t R, const int32_t* place, const float* weights, int64_t k,
                          const float* post_weight, const void* gate, int64_t gate_stride, rtn_gate gate_kind,
                          const float* scale, int64_t n_scale, const void* residual, int64_t residual_stride,
                          const float* norm_weight, float eps, int64_t T, int64_t W, void* stream_out, int64_t stream_stride,
                          void* normed, int64_t normed_stride, const float* t_lo, const float* t_hi, int64_t n_thr,
                          void* out_packed, int32_t* out_sum, rtn_dtype dtype, rtn_dtype stream_dtype, void* stream);

/* The variant RTN_VARIANT_AUTO resolves to for a shape (never AUTO). */
rtn_variant rtn_choose_gemm_variant(int64_t M, int64_t N, int64_t K);
/* Slices of K that RTN_VARIANT_AUTO cuts a GEMM shape into (1 = none).  A linear layer with few rows and
 * columns and a long K (linear layers are covered by the pattern of section "Efficient Computation
 * Pattern" as much as convolutions) has too few output tiles to fill the GPU: the bit-plane kernel then works on slices of K in
 * parallel, adds their exact integer parts into the output buffer and applies the affine form in place
 * (3 launches instead of 1; the integers do not depend on the order of the additions). */
int64_t rtn_gemm_k_slices(int64_t M, int64_t N, int64_t K);
/* Kernel launches of one rtn_ternary_gemm call with RTN_VARIANT_AUTO: 1; 2 when the tensor-core kernel first
 * expands the weight operand into a scratch buffer (stream-ordered allocation of about N*K bytes; shapes with
 * two or more row tiles; with two or more column tiles as well the activations too, M*K bytes more) or when K
 * is cut into slices (plus a memset). */
int64_t rtn_gemm_kernel_launches(int64_t M, int64_t N, int64_t K);
rtn_variant rtn_choose_conv_variant(int64_t B, int64_t C, int64_t H, int64_t W, int64_t N,
                                    int64_t kh, int64_t kw, int64_t stride, int64_t pad);
/* Kernel launches one rtn_ternary_conv2d call with RTN_VARIANT_AUTO makes for a shape: 1, or 2 on the
 * path that first writes the input's int8 codes to a scratch buffer. */
int64_t rtn_conv_kernel_launches(int64_t B, int64_t C, int64_t H, int64_t W, int64_t N,
                                 int64_t kh, int64_t kw, int64_t stride, int64_t pad);

/* Kernel launches of one rtn_ternary_conv2d_fused / rtn_ternary_conv2d_packed call for a shape: 1 (one-kernel
 * variant with the filters resident in shared memory), 2 (int8 codes in a scratch buffer first), or 0 if
 * the entry points do not take the shape (they would return RTN_ERR_UNSUPPORTED). */
int64_t rtn_conv_next_kernel_launches(int64_t B, int64_t C, int64_t H, int64_t W, int64_t N,
                                      int64_t kh, int64_t kw, int64_t stride, int64_t pad);

/* Synchronises `stream`, then reads and clears the device status word of the current device.
 * RTN_OK, or RTN_ERR_DEVICE_TIMEOUT if a kernel's bounded wait (on an mbarrier of the
 * tensor-core pipeline) ran out since the last call; that kernel's output is then invalid.  Else
 * RTN_ERR_DEVICE_INDEX if a layer operator met a position, slot or sequence bound out of range. */
rtn_status rtn_last_device_status(void* stream);

/* Synchronises `stream`, then gives back to the device what the current device's scratch pool keeps and no call in flight on
 * another stream uses.  The next call that needs scratch maps memory again (100 us to 1 ms). */
rtn_status rtn_release_scratch(void* stream);

/* Self-test of the bounded waits (the safety net behind RTN_ERR_DEVICE_TIMEOUT): launches one small kernel
 * whose single waiting thread polls, `polls` times (1..4096, each poll parks the thread for up to about 2 us),
 * an mbarrier that nothing arrives on, with the same wait routine the tensor-core kernels use.  The wait must
 * give up: *gave_up (device int32) receives 1, and the next rtn_last_device_status returns
 * RTN_ERR_DEVICE_TIMEOUT once.  Nothing traps or spins without limit; the context stays usable.  Only enqueues. */
rtn_status rtn_selftest_wait_timeout(int64_t polls, int32_t* gave_up, void* stream);

/* Peak probes (measurement aids; the paper has no counterpart).  The contraction kernels are judged against two
 * ceilings that no memory copy measures: the int8 tensor-pipe rate and the issue rate of the AND / XOR /
 * popcount pattern of Eq. 9.  Each probe launches rtn_probe_ctas() CTAs (one per multiprocessor) that run
 * nothing but that work on on-chip operands, and writes the SM-clock cycles of each CTA's loop to `cycles`
 * (device int64 [rtn_probe_ctas()], 8-byte aligned); time the launch with events for the rate in seconds.
 *   rtn_probe_peak_i8   n_mma (1..2^22) tcgen05.mma kind::i8 of M = 128, N = 256, K = 32 per CTA, operands in
 *                       shared memory, one accumulator; rtn_probe_i8_ops_per_mma() = 2*128*256*32 operations each.
 *                       The final wait is bounded like every other (rtn_last_device_status reports a time-out).
 *   rtn_probe_i8_rate   the same loop with accumulators of n_cols columns (a multiple of 16 in 16..256): what one
 *                       instruction of that width costs when nothing else is in the way (narrow instructions do not
 *                       get cheaper in proportion); 2*128*n_cols*32 operations each.
 *   rtn_probe_peak_popc rounds (1..2^24) rounds per thread of 64 word pairs, 1024 threads per CTA, registers
 *                       only; rtn_probe_popc_ops_per_round() operations (2 per code pair) per CTA and round.
 *                       `sink`: device int32 the kernel never writes in practice (keeps the loop alive).
 *   rtn_probe_copy      copies `bytes` (a multiple of 16; both pointers 16-byte aligned) from src to dst with two
 *                       CTAs of 1024 threads per multiprocessor, 16 bytes per thread and trip: the time a kernel
 *                       that only moves a layer's input and output takes at that size.
 * All only enqueue. */
int64_t rtn_probe_ctas(void);
int64_t rtn_probe_i8_ops_per_mma(void);
int64_t rtn_probe_popc_ops_per_round(void);
rtn_status rtn_probe_peak_i8(int64_t n_mma, int64_t* cycles, void* stream);
rtn_status rtn_probe_i8_rate(int64_t n_cols, int64_t n_mma, int64_t* cycles, void* stream);
rtn_status rtn_probe_peak_popc(int64_t rounds, int64_t* cycles, int32_t* sink, void* stream);
rtn_status rtn_probe_copy(const void* src, void* dst, int64_t bytes, void* stream);

/* Static text for a status code. */
const char* rtn_status_string(rtn_status s);

#ifdef __cplusplus
}
#endif
#endif /* RTN_H_ */
