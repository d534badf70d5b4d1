/*
 * fqvit.h -- C ABI of the MI355X (gfx950) library for the integer hot path of
 * FQ-ViT (Lin et al., "FQ-ViT: Post-Training Quantization for Fully Quantized
 * Vision Transformer", IJCAI 2022): Power-of-Two-Factor LayerNorm and
 * Log-Int-Softmax attention, the linear layers, rotary positions and
 * requantization around them, and the step over a stream of tokens: root-mean-square
 * norm, paged cache, attention over it, eviction from it.
 *
 * Conventions shared by every entry point
 *   - Tensor arguments are DEVICE pointers into memory the caller owns (for
 *     example allocated through torch).  The library allocates nothing, never
 *     synchronises, and enqueues its kernels on `stream` (a hipStream_t; NULL
 *     is the default stream).  It keeps no state between calls apart from the
 *     per-thread timing events of fq_time_next_call and the fixed device array
 *     of ptf_calibrate_noalloc.  It is re-entrant (ptf_calibrate_noalloc: see
 *     its note on overlapping calls).
 *   - Scalars are passed by value.  Tensors are dense and row-major with the
 *     shapes given below; a tensor is read or written only inside the extent
 *     its shape gives.
 *   - Every argument is validated on the host before anything is enqueued.  A
 *     failing check returns its status code and enqueues nothing.  Empty
 *     tensors (T, G or Lq equal to 0) return FQ_OK and enqueue nothing.
 *   - Integer outputs are a pure function of the arguments (no order
 *     dependence; atomics, where there are any, add integers): the same call
 *     gives the same bits every time.
 *   - Quantized activations live on the paper's unsigned b-bit grid
 *     {0 .. 2^b - 1} (Sec. 3.1, eq. 2).  The int8 containers used here hold
 *     (paper value - 2^(b-1)); zero points are shifted the same way.  Every
 *     formula uses only X_Q - zp, so results are identical on either grid.
 */
#ifndef FQVIT_H
#define FQVIT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum fq_status {
    FQ_OK = 0,
    FQ_ERR_NULL = 1,      /* a required pointer is NULL                              */
    FQ_ERR_SHAPE = 2,     /* a size is out of the supported range                    */
    FQ_ERR_PARAM = 3,     /* a scalar parameter is out of range                      */
    FQ_ERR_HEADROOM = 4,  /* the exact integer sums could overflow 64 bits           */
    FQ_ERR_HIP = 5,       /* the HIP runtime rejected a launch                       */
    FQ_ERR_SCRATCH = 6    /* the call needs more than the fixed device scratch holds */
} fq_status;

/* Static, human-readable name of a status code (never NULL). */
const char* fq_status_str(int status);

/* Library version as major * 10000 + minor * 100 + patch. */
int32_t fq_version(void);

/*
 * Instrumentation, not part of the method.  Attaches two caller-created HIP
 * events (hipEvent_t, from hipEventCreate; either may be NULL) to the kernel
 * launched by the next entry-point call made on the calling thread: `start`
 * then records that kernel's start and `stop` its end (hipExtLaunchKernel
 * semantics), so hipEventElapsedTime gives the kernel's own duration with no
 * extra packets on the stream.  Every other entry point launches one kernel.
 * ptf_calibrate, which launches four kernels, records `start` on the first and
 * `stop` on the last, so the interval covers the whole calibration; so do
 * lis_attention_paged and kv_cache_evict where they launch several.
 * The events are consumed by that next call whatever it returns; a call that
 * enqueues nothing (empty tensors, failed validation) leaves them unrecorded.
 * Always returns FQ_OK.
 */
fq_status fq_time_next_call(void* start_event, void* stop_event);

/*
 * PTF LayerNorm, integer-only (Sec. 3.2, eq. 12 for the shift; Supplement A.1
 * for the statistics M1, M2, the factors A and B, their dyadic form N2 / 2^N1
 * and the output Y_Q).
 *
 *   x_q     [T, C] int8 container of the PTF-quantized input X_Q.
 *   zp_in   layer-wise zero point, container form, in [-2^(b-1), 2^(b-1) - 1].
 *   alpha   [C] uint8 power-of-two factors; values above K are clamped to K.
 *   K       0..7 (the paper uses 3).
 *   gamma, beta  [C] float affine parameters.
 *   s_out   output scale (> 0, finite); zp_out output zero point (container).
 *   bits    b in [2, 8]; the output is clipped to the b-bit grid.
 *   y_q     [T, C] int8 container output.
 * The input scale cancels from A and B and is therefore not an argument.
 * Per row: X^ = (X_Q - zp) << alpha, M1 = sum X^, M2 = sum X^^2,
 * V = C M2 - M1^2; in IEEE double, D = sqrt(V), r = C / D, m = M1 / D,
 * A = (gamma/s_out) r, B = beta/s_out - (gamma/s_out) m (each operation
 * rounded on its own; A = 0 and B = beta/s_out when V = 0);
 * N1 = clamp(b - 1 - floor(log2|A|), 0, 30), N2 = min(floor(|A| 2^N1), 2^31 - 1)
 * (both 0 when A = 0); Y = clip(floor((sign(A) N2 X^ + rint(B 2^N1)
 * + 2^(N1-1)) / 2^N1) + zp_out) (no half term when N1 = 0).
 * Errors: FQ_ERR_NULL (x_q, alpha, gamma, beta or y_q NULL with T > 0),
 * FQ_ERR_SHAPE (T < 0, C outside [1, 8192]), FQ_ERR_PARAM (bits, K, s_out or a
 * zero point out of range).
 */
fq_status ptf_layernorm_int8(const int8_t* x_q, int64_t T, int32_t C, int32_t zp_in,
                             const uint8_t* alpha, int32_t K, const float* gamma,
                             const float* beta, float s_out, int32_t zp_out, int32_t bits,
                             int8_t* y_q, void* stream);

/*
 * Log-Int-Softmax codes (Supplement A.2: Algorithm 1, I-Exp; Algorithm 2,
 * I-Log2 and Log-Int-Softmax; the clip of the LIS equation in the same
 * section).
 *
 *   logits  [G, Lq, Lk] int32 attention logits with scale s_logit
 *           (G = attention units, e.g. batch x windows x heads).
 *   bias    NULL or [Hb, Lq, Lk] int32 added to the logits of unit g from
 *           plane g % Hb before the row maximum (Swin relative-position bias:
 *           Hb = heads; with units ordered (image, window, head), a shifted-
 *           window mask is folded in by passing the sum of mask and bias as
 *           [windows, heads, Lq, Lk] with Hb = windows x heads).
 *   s_logit in [1e-4, 0.5].
 *   bits    code width b in [1, 8]; codes are Attn_Q in [0, 2^b - 1] and the
 *           LIS output of the paper is N - Attn_Q with N = 2^b - 1, scale 2^-N.
 *   exp_n   I-Exp clamp depth n in [1, 30]: inputs below n q_ln2 are clamped.
 *   codes   [G, Lq, ld_codes] uint8 output.  b <= 4: two codes per byte, the
 *           even key in the low nibble, an odd row's last high nibble 0, bytes
 *           at and beyond ceil(Lk/2) in each row not written.  b >= 5: one
 *           code per byte, bytes at and beyond Lk not written.
 * Per row: t_j = v_j - max v, e_j = I-Exp(t_j) with q_ln2 = floor(-ln2/s),
 * q_b = floor(1.353/s), q_c = floor(0.344/((0.3585 s) s)) in IEEE double,
 * S = sum e_j, Attn_Q_j = min(I-Log2(floor((2S + e_j) / (2 e_j))), 2^b - 1).
 * Errors: FQ_ERR_NULL (logits or codes NULL with G Lq > 0), FQ_ERR_SHAPE
 * (G or Lq < 0, Lk outside [1, 4096], ld_codes below ceil(Lk/2) for b <= 4 or
 * Lk for b >= 5, Hb < 1 with a bias), FQ_ERR_PARAM (bits, exp_n or s_logit
 * out of range), FQ_ERR_HEADROOM
 * ((2 Lk + 1) (q_b^2 + q_c) 2^n >= 2^63).
 * Precondition (not checked): |logit + bias| < 2^30.
 */
fq_status lis_softmax_log4(const int32_t* logits, int64_t G, int32_t Lq, int32_t Lk,
                           const int32_t* bias, int32_t Hb, float s_logit, int32_t bits,
                           int32_t exp_n, uint8_t* codes, int32_t ld_codes, void* stream);

/*
 * BitShift Attn x V (Sec. 3.3, eq. 16-17, and its zero-point form in
 * Supplement A.2):
 *   out[g, i, c] = sum_j (v[g, j, c] - zp_v) << ((2^b - 1) - code[g, i, j]).
 *
 *   codes   [G, Lq, ld_codes] packed codes as written by lis_softmax_log4.
 *   v       [G, Lk, d] int8, zero point zp_v in [-128, 127].
 *   bits    b in [1, 4] (shifts of at most 15).
 *   out     [G, Lq, d] int32, scale s_V / 2^(2^b - 1).
 * The sum is exact; it wraps modulo 2^32 only if it leaves int32, which codes
 * produced by Log-Int-Softmax never do for Lk <= 4096.  Codes above 2^b - 1
 * (never written by lis_softmax_log4) give an unspecified result.
 * Errors: FQ_ERR_NULL, FQ_ERR_SHAPE (G or Lq < 0, Lk outside [1, 4096], d
 * outside [1, 256], ld_codes < ceil(Lk/2)), FQ_ERR_PARAM (bits, zp_v).
 */
fq_status lis_attn_v_shift(const uint8_t* codes, int32_t ld_codes, const int8_t* v,
                           int32_t zp_v, int64_t G, int32_t Lq, int32_t Lk, int32_t d,
                           int32_t bits, int32_t* out, void* stream);

/*
 * BitShift Attn x V for codes of any width b in [1, 8], including the 8-bit
 * attention maps of the paper's 8/8/8 setting (Sec. 3.3; its Table 1).  The
 * paper does not say how codes wider than 4 bits multiply V: with
 * N = 2^b - 1 the integer form (V - zp) << (N - code) would need shifts of up
 * to 255.  This product keeps the fixed output scale s_V / 2^W with
 * W = min(2^b - 1, 44):
 *   out[g, i, c] = sum_j floor((v[g, j, c] - zp_v) 2^(W - code[g, i, j])),
 * which is exact (no floor acts) for every code <= W.  Log-Int-Softmax never
 * produces a code above 44 for Lk <= 4096 and n <= 30 (round(S / e) stays
 * below 2^43 + 1), so its products are exact, and below 255 (1.5) 2^44 in
 * magnitude; for b <= 4 the result is lis_attn_v_shift's widened to int64.
 * A code above W (not one made by Log-Int-Softmax) contributes the floor of
 * its shifted value, and a sum that leaves int64 (again only for such codes)
 * wraps modulo 2^64.
 *
 *   codes   [G, Lq, ld_codes] as written by lis_softmax_log4 with the same
 *           bits: nibbles for b <= 4 (ld_codes >= ceil(Lk/2)), one byte per
 *           code for b >= 5 (ld_codes >= Lk).
 *   v       [G, Lk, d] int8, zero point zp_v in [-128, 127].
 *   out     [G, Lq, d] int64, scale s_V / 2^W.
 * Errors: FQ_ERR_NULL, FQ_ERR_SHAPE (G or Lq < 0, Lk outside [1, 4096], d
 * outside [1, 256], ld_codes below the row's bytes), FQ_ERR_PARAM (bits, zp_v).
 */
fq_status lis_attn_v_shift_wide(const uint8_t* codes, int32_t ld_codes, const int8_t* v,
                                int32_t zp_v, int64_t G, int32_t Lq, int32_t Lk, int32_t d,
                                int32_t bits, int64_t* out, void* stream);

/*
 * Fused Log-Int-Softmax and BitShift Attn x V, the integer-only attention of
 * Sec. 3.3 (the MSA dataflow of its Fig. 4): the same results as
 * lis_softmax_log4 followed by lis_attn_v_shift, with the codes kept on chip.
 * Arguments as in those two calls (bits in [1, 4]); d in [1, 256]; codes_out
 * is NULL or a [G, Lq, ld_codes] buffer that also receives the codes.
 */
fq_status lis_attention_head(const int32_t* logits, const int32_t* bias, int32_t Hb,
                             int64_t G, int32_t Lq, int32_t Lk, float s_logit, int32_t bits,
                             int32_t exp_n, const int8_t* v, int32_t zp_v, int32_t d,
                             int32_t* out, uint8_t* codes_out, int32_t ld_codes, void* stream);

/*
 * Integer-only multi-head self-attention from int8 queries and keys: the
 * MinMax-quantized MatMul of Sec. 3.1 between Q and K (an integer GEMM),
 * Log-Int-Softmax and the BitShift Attn x V of Sec. 3.3 (the dataflow of its
 * Fig. 4), with the logits and codes kept on chip:
 *   logit[g,i,j] = sum_c (q[g,i,c] - zp_q)(k[g,j,c] - zp_k) (+ bias),
 * then exactly lis_attention_head on those logits.  Log-Int-Softmax depends
 * only on the differences of a row's logits, so the result does not depend on
 * zp_k (it is still validated); the kernel drops the per-query terms.
 *
 *   q       [G, Lq, dk] int8 container, 16-byte aligned; zp_q in [-128, 127].
 *   k       [G, Lk, dk] int8 container, 16-byte aligned; zp_k in [-128, 127].
 *   dk      32 or 64.
 *   bias, Hb, s_logit, bits (in [1, 4]), exp_n, v, zp_v, out: as in
 *           lis_attention_head;
 *           s_logit is the scale of the logits (s_q s_k, with any 1/sqrt(dk)
 *           of the softmax folded in).
 * Supported: Lk in [1, 640], d in [1, 64] (rows of more than 224 keys at scales
 * outside the float path's bounds: the logits are recomputed from K in each
 * pass instead of held).
 * Errors: FQ_ERR_NULL, FQ_ERR_SHAPE (sizes, dk, or bias with Hb < 1),
 * FQ_ERR_PARAM (zero points, bits, exp_n, s_logit, or misaligned q / k),
 * FQ_ERR_HEADROOM.
 */
fq_status lis_attention_qk(const int8_t* q, const int8_t* k, int32_t zp_q, int32_t zp_k,
                           int32_t dk, const int32_t* bias, int32_t Hb, int64_t G, int32_t Lq,
                           int32_t Lk, float s_logit, int32_t bits, int32_t exp_n,
                           const int8_t* v, int32_t zp_v, int32_t d, int32_t* out, void* stream);

/*
 * PTF calibration (Sec. 3.2): the layer-wise scale and zero point of eq. (9),
 * (10) from the minimum and maximum of x, then each channel's power-of-two
 * factor alpha_c by the argmin of eq. (11) over {0 .. K}, the squared error of
 * the quantizer of eq. (8) itself (its zero point and clip included).
 *
 *   x          [T, C] float activations (finite), T in [0, 65535 * 64].
 *   bits       b in [2, 8]; K in [0, 7] (the paper uses 3).
 *   s          device double (out): s = (max - min) / (2^b - 1) / 2^K.
 *   zp         device int32 (out), container form: clip(rint(-min / (2^K s)),
 *              0, 2^b - 1) - 2^(b-1).
 *   alpha      [C] uint8 (out).
 *   workspace  device scratch of at least fq_ptf_calibrate_workspace_bytes(T,
 *              C, K) bytes, owned by the caller; its contents on entry do not
 *              matter and on return are unspecified.
 * Every operation is rounded in binary64 as written; each channel's squared
 * errors are summed in blocks of 64 consecutive rows, in order, and the block
 * sums added in order, so alpha is a pure function of x; ties of those sums go
 * to the smallest alpha.  Tie rule against the exact argmin of eq. (11): with
 * E_a the exact error of candidate a and B_a = (T + 8) 2^-53
 * sum_t (|x_tc| + 2 |deq_a(x_tc)|)^2 the bound on the rounding of its sum,
 * alpha_c is the exact argmin (ties to the smallest) unless another candidate
 * a has E_a - E_best <= B_a + B_best, in which case it may be a.  A tensor
 * whose maximum equals its minimum gets s = 0, the
 * zero point 0 of the paper's grid and alpha = 0.  T = 0 enqueues nothing and
 * leaves the outputs untouched.
 * Errors: FQ_ERR_NULL, FQ_ERR_SHAPE (T outside [0, 65535 * 64], C outside
 * [1, 8192]), FQ_ERR_PARAM (bits, K, or a workspace that is too small).
 */
size_t fq_ptf_calibrate_workspace_bytes(int64_t T, int32_t C, int32_t K);
fq_status ptf_calibrate(const float* x, int64_t T, int32_t C, int32_t bits, int32_t K, double* s,
                        int32_t* zp, uint8_t* alpha, void* workspace, size_t workspace_bytes,
                        void* stream);

/*
 * ptf_calibrate for callers that cannot allocate device memory (code under HIP
 * graph capture, tight serving loops, harnesses that forbid allocation): the
 * same kernels and results, with the workspace taken from a fixed device
 * array of FQ_NOALLOC_SCRATCH_BYTES that the library holds on each GPU it runs
 * on until the process ends.  This call allocates nothing (no hipMalloc, no
 * hipFree, no allocating library routine); on its first call on a device it
 * looks up that device's copy of the array (hipGetSymbolAddress).
 *   x, T, C, bits, K, s, zp, alpha: as ptf_calibrate.
 * Every call on one GPU shares that GPU's array, so calls that overlap on one
 * GPU (different streams, or host threads, without ordering between them)
 * race and give undefined results; calls ordered on one stream are safe.  The
 * array's contents on entry do not matter.
 * Errors: as ptf_calibrate, and FQ_ERR_SCRATCH when
 * fq_ptf_calibrate_workspace_bytes(T, C, K) exceeds FQ_NOALLOC_SCRATCH_BYTES
 * (nothing enqueued); FQ_ERR_HIP if the array cannot be looked up.
 */
#define FQ_NOALLOC_SCRATCH_BYTES ((size_t)8 << 20)
fq_status ptf_calibrate_noalloc(const float* x, int64_t T, int32_t C, int32_t bits, int32_t K,
                                double* s, int32_t* zp, uint8_t* alpha, void* stream);

/*
 * PTF quantizer (Sec. 3.2, eq. 8): X_Q = clip(rint(x / (2^alpha_c s)) + zp,
 * 0, 2^b - 1), in binary64, stored in the int8 container.
 *
 *   x      [T, C] float; s, zp: device scalars as written by ptf_calibrate
 *          (zp in container form); alpha [C] uint8; bits b in [2, 8].
 *   x_q    [T, C] int8 container output (the input of ptf_layernorm_int8).
 * s <= 0 (a degenerate calibration) stores zp everywhere.
 * Errors: FQ_ERR_NULL, FQ_ERR_SHAPE (T < 0, C outside [1, 8192]),
 * FQ_ERR_PARAM (bits).
 */
fq_status ptf_quantize_int8(const float* x, int64_t T, int32_t C, const double* s,
                            const int32_t* zp, const uint8_t* alpha, int32_t bits, int8_t* x_q,
                            void* stream);

/*
 * Dyadic requantization of an int32 accumulator to a b-bit activation, the
 * integer-only form of Supplement A.1 (a real multiplier replaced by
 * N2 / 2^N1 and a rounding shift), e.g. for the BitShift Attn x V output of
 * lis_attention_head (scale s_V / 2^(2^b - 1)) feeding the next layer.
 *
 *   q       [n] int32 with scale s_in.
 *   s_in, s_out  positive finite scales; zp_out the output zero point,
 *           container form.  bits b in [2, 8].
 *   y       [n] int8 container output.
 * With M = s_in / s_out in binary64, M = f 2^e (f in [0.5, 1)),
 * N1 = clamp(31 - e, 0, 62), N2 = min(floor(M 2^N1), 2^31 - 1):
 * y = clip(floor((N2 q + 2^(N1-1)) / 2^N1) + zp_out) (no half term when
 * N1 = 0), exact in 64-bit integers.
 * Errors: FQ_ERR_NULL, FQ_ERR_SHAPE (n < 0), FQ_ERR_PARAM (bits, a scale or
 * zp_out out of range).
 */
fq_status requant_dyadic_int8(const int32_t* q, int64_t n, float s_in, float s_out,
                              int32_t zp_out, int32_t bits, int8_t* y, void* stream);

/*
 * Linear layer: the integer matrix product that every quantized layer around
 * the attention is (Sec. 3.1), with its bias, its activation, the residual
 * branch and the requantization in the product's epilogue.  Values stand for
 *   x_real = s_x (x - zp_x),  w_real = s_w[n] w,  y_real = s_y (y - zp_y).
 *
 * linear_fold_int8 makes, once for a layer, the two vectors that the products
 * take: the bias on the accumulators' scale with the input's zero point folded
 * in, and the channels' multipliers.  In binary64, each operation rounded once:
 *   acc scale  s_n = s_x s_w[n]
 *   fold[n] = clip(rint(bias[n] / s_n), -2^30, 2^30) - zp_x sum_k w[n, k]
 *   mul[n]  = s_n / s_y rounded to binary32 (at most the largest finite one).
 * A channel whose s_w[n] is not positive and finite takes mul[n] = 0 and no
 * bias; a bias that is not a number counts as 0.
 *
 *   w      [N, K] int8 of any alignment, N in [1, 2^20], K in [1, 32768].
 *   s_w    [N] float; bias [N] float or NULL (none).
 *   zp_x   in [-128, 127]; s_x, s_y positive and finite.  s_y is the output's
 *          step, or the step of the activation's input where a table follows.
 *   fold   [N] int32 (out); mul [N] float (out) or NULL (then s_y is unused).
 * Errors: FQ_ERR_NULL, FQ_ERR_SHAPE (N or K out of range), FQ_ERR_PARAM.
 */
fq_status linear_fold_int8(const int8_t* w, int32_t N, int32_t K, const float* s_w,
                           const float* bias, int32_t zp_x, float s_x, float s_y, int32_t* fold,
                           float* mul, void* stream);

/* Activations of linear_int8. */
#define FQ_ACT_NONE 0
#define FQ_ACT_RELU 1
#define FQ_ACT_TABLE 2   /* any function, as 2^table_bits values over its input's grid */

/*
 * y = requantized (activation(x w^T + bias) + residual), in int8.
 *
 *   x      [T, K] int8, w [N, K] int8 (a row per output channel).
 *   fold, mul   [N] int32 and float, as linear_fold_int8 writes them (fold NULL:
 *          zeros).  mul >= 0 and finite.
 *   act    FQ_ACT_*; with FQ_ACT_TABLE, table is a device array of
 *          2^table_bits floats (finite), table_bits in [4, 12], zp_t in
 *          [0, 2^table_bits - 1]; else they are ignored.
 *   residual  NULL or [T, N] int8 of zero point zp_r in [-128, 127]; mul_r =
 *          s_r / s_y, in [2^-20, 2^20].
 *   zp_y, bits  the output's zero point (container form) and grid, b in [2, 8].
 *   y      [T, N] int8 container (out).  It may be the residual itself; it
 *          overlaps no other argument.
 * T >= 0, N in [1, 2^20], K in [1, 32768], fewer than 2^24 tiles of 64 x 64
 * outputs.  int8 bases of any alignment, int32 and float ones of 4 bytes; rows of x
 * and w of whole 16-byte units on 16-byte aligned bases take the fast path.
 *
 * With acc = sum_k x[t,k] w[n,k] + fold[n] exact in int32, RN = rounding to the
 * nearest binary32 and rint = to the nearest integer (ties to even in both), of
 * the exact value in its argument:
 *   a = RN(acc)
 *   without a residual:
 *     NONE   y = clip(rint(a mul + zp_y))
 *     RELU   y = clip(rint(max(a mul, 0) + zp_y))
 *     TABLE  u = clip(rint(a mul + zp_t), 0, 2^table_bits - 1)
 *            y = clip(rint(table[u] + zp_y))
 *   with one: z = RN((r + 128) mul_r + c), c = RN(zp_y - (128 + zp_r) mul_r), and
 *     NONE   y = clip(rint(RN(a mul + z)))
 *     RELU   y = clip(rint(RN(max(RN(a mul), 0) + z)))
 *     TABLE  y = clip(rint(RN(table[u] + z)))
 * clip is to the container's [-2^(b-1), 2^(b-1) - 1].  A table holds its
 * function's values in steps of the output, f(s_t (u - zp_t)) / s_y; then mul
 * was folded with the table's step s_t in the place of s_y.
 * Errors: FQ_ERR_NULL (x, w, mul, y; table with FQ_ACT_TABLE), FQ_ERR_SHAPE
 * (T, N, K or the tiles), FQ_ERR_PARAM (act, table_bits, zp_t, zero points,
 * mul_r, bits).
 */
fq_status linear_int8(const int8_t* x, int64_t T, const int8_t* w, int32_t N, int32_t K,
                      const int32_t* fold, const float* mul, int32_t act, const float* table,
                      int32_t table_bits, int32_t zp_t, const int8_t* residual, int32_t zp_r,
                      float mul_r, int32_t zp_y, int32_t bits, int8_t* y, void* stream);

/*
 * The accumulators themselves: out[t, n] = sum_k x[t,k] w[n,k] + fold[n] in
 * int32 (scale s_x s_w[n]), for class scores and layers requantized elsewhere.
 * Sizes, alignment and errors as linear_int8; fold may be NULL (zeros).  The
 * sum is exact for fold within +-2^30; it wraps modulo 2^32 where a larger one
 * takes it out of int32.
 */
fq_status linear_int32(const int8_t* x, int64_t T, const int8_t* w, int32_t N, int32_t K,
                       const int32_t* fold, int32_t* out, void* stream);

/*
 * Fills a HOST array with an activation's table for linear_int8: in binary64,
 * table[u] = f(t) / s_y rounded to binary32, t = s_t (u - zp_t), u in
 * [0, 2^table_bits - 1].  Runs on the host; enqueues nothing.
 *   kind   FQ_FN_GELU        t (1 + erf(t / sqrt 2)) / 2
 *          FQ_FN_GELU_TANH   t (1 + tanh(sqrt(2/pi) (t + 0.044715 t^3))) / 2
 *          FQ_FN_SILU        t / (1 + exp(-t))
 * Errors: FQ_ERR_NULL, FQ_ERR_PARAM (kind, table_bits, zp_t, a step not
 * positive and finite, or a value that binary32 cannot hold).
 */
#define FQ_FN_GELU 0
#define FQ_FN_GELU_TANH 1
#define FQ_FN_SILU 2
fq_status fq_activation_table(int32_t kind, float s_t, int32_t zp_t, int32_t table_bits, float s_y,
                              float* table);

/*
 * Rotary positions of several axes (time, height, width): pair p of a head
 * turns by the angle t = positions[axis[p], i] freq[p] of token i.  The table
 * holds cos and sin of every token and pair in steps of 2^-14:
 *   table[i, p] = (rint(2^14 cos t), rint(2^14 sin t)), t in binary64 (one
 * rounding), cos and sin in binary64 to within 2 units of their last place, so
 * an entry may be the other neighbour only where 2^14 cos t lies that close to
 * the middle of two integers.  Position 0 gives (2^14, 0): no turn at all.
 *
 *   positions  [axes, T] int32, axes in [1, 8], T in [0, 2^25].
 *   freq   [P] double, P in [1, 128], its products with the positions finite;
 *          axis [P] uint8 (values at or above `axes` are taken as axes - 1).
 *   table  [T, P, 2] int16 (out), 4-byte aligned.
 * Errors: FQ_ERR_NULL, FQ_ERR_SHAPE (T, axes, P), FQ_ERR_PARAM (table not
 * aligned).
 */
fq_status rope_table_int16(const int32_t* positions, int32_t axes, int64_t T, const double* freq,
                           const uint8_t* axis, int32_t P, int16_t* table, void* stream);

/*
 * The query-key-value layer's rows split into heads, queries and keys rotated
 * and requantized, as lis_attention_qk takes them.
 *
 *   qkv    [B, L, (Hq + 2 Hkv) d] int8 with scale s_x and zero point zp_x: the
 *          query heads, the key heads, the value heads.  B L in [0, 2^25], Hq, Hkv
 *          in [1, 1024], d in [1, 256].
 *   table  [table_rows, P, 2] int16, 4-byte aligned, as rope_table_int16 writes
 *          it; table_rows is L (one grid for every b) or B L.  P in [0, d / 2]
 *          pairs turn, the d - 2 P values after them do not.  P = 0: table may
 *          be NULL and table_rows is unused.
 *   interleaved  0: pair p is (x[p], x[p + P]); 1: (x[2 p], x[2 p + 1]).
 *   q      [B, Hq, L, d] int8 (out), scale s_q, zero point zp_q (container of
 *          the b-bit grid); k [B, Hkv, L, d] (out), s_k, zp_k; v [B, Hkv, L, d]
 *          (out), the values as they are.  With Hq = r Hkv, q read as
 *          [B Hkv, r L, d] are the queries of each key head.  The outputs overlap
 *          no other argument.
 * With (f, g) a pair less zp_x and (c, s) its table entry, the turned pair is
 * (f c - g s, f s + g c), exact in 32 bits for |c|, |s| <= 2^14; a value that
 * does not turn counts 2^14 times itself less zp_x.  Each, a, becomes
 * clip(rint(a m + zp)), the exact value rounded once (ties to even), with m =
 * s_x / (2^14 s_q) (s_k) in binary64 rounded to binary32.
 * Errors: FQ_ERR_NULL, FQ_ERR_SHAPE (sizes, table_rows), FQ_ERR_PARAM (scales,
 * zero points, bits, interleaved, table not aligned).
 */
fq_status rope_qkv_int8(const int8_t* qkv, int64_t B, int32_t L, int32_t Hq, int32_t Hkv, int32_t d,
                        float s_x, int32_t zp_x, const int16_t* table, int64_t table_rows, int32_t P,
                        int32_t interleaved, float s_q, int32_t zp_q, float s_k, int32_t zp_k,
                        int32_t bits, int8_t* q, int8_t* k, int8_t* v, void* stream);

/*
 * requant_dyadic_int8 of an attention result, with its heads brought back to
 * rows: q [B, H, L, d] int32 (lis_attention_qk's out) -> y [B, L, H d] int8, as
 * the projection's linear layer reads it.  The same dyadic multiplier and
 * rounding; B L in [0, 2^25], H in [1, 1024], d in [1, 256]; q 4-byte aligned, y
 * of any alignment.
 * Errors: FQ_ERR_NULL, FQ_ERR_SHAPE (B or L < 0, H, d), FQ_ERR_PARAM (bits, a
 * scale or zp_out out of range).
 */
fq_status requant_heads_int8(const int32_t* q, int64_t B, int32_t H, int32_t L, int32_t d,
                             float s_in, float s_out, int32_t zp_out, int32_t bits, int8_t* y,
                             void* stream);

/*
 * Root-mean-square norm of a stream of tokens with the addition of a branch: the
 * LayerNorm's integer form (Supplement A.1: exact sums of integers, one normaliser a
 * row) without the mean, for layers whose residual stream is kept in 16 bits.
 *
 *   x      NULL (no branch) or [T, C] int8 container of the branch, zero point zp_x in
 *          [-128, 127]; alpha NULL (zeros) or [C] uint8 power-of-two factors (Sec.
 *          3.2), values above K (0..7) are clamped to K.  m_x = s_x / s_r, the steps of
 *          branch and stream, in [2^-20, 64].
 *   r      [T, C] int16, the stream (zero point 0).
 *   gamma  [C] float, finite.  eps >= 0, finite: the norm's epsilon in steps of the
 *          stream, eps_real / s_r^2.
 *   h      [T, C] int16 (out): the stream with the branch; it may be r itself.
 *   y      [T, C] int8 container (out) of the b-bit grid, b in [2, 8].
 * T in [0, 2^24 - 1], C in [1, 8192]; other overlaps are not allowed.  With RN =
 * rounding to the nearest binary32 and rint = to the nearest integer (ties to even in
 * both) of the exact value, RN64 likewise to binary64:
 *   h = clip(r + rint((x - zp_x) 2^min(alpha, K) m_x), -32768, 32767)
 *   M2 = sum_c h^2, exact;  D = RN64(RN64(M2 / C) + eps)
 *   rho = RN64(1 / RN64(sqrt D)), 0 where D = 0
 * rmsnorm_int8, with a scale s_out (positive, finite) and zero point zp_out:
 *   y = clip(rint(h RN(gamma RN(RN64(rho / s_out))) + zp_out))
 * rmsnorm_rows_int8, with a scale for each row, scales [T] float (out), t = 2^(b-1) - 1:
 *   a = RN(gamma h), A = max_c |a|
 *   y = rint(a RN(RN64(t / A))), all 0 where A = 0;  scales = RN(RN(A RN(rho)) / t)
 * (a value that leaves binary32 on the way gives an unspecified y.)
 * Errors: FQ_ERR_NULL (r, gamma, h, y; scales), FQ_ERR_SHAPE (T, C), FQ_ERR_PARAM (bits,
 * K, zero points, m_x, eps, s_out; what is not used is not looked at).
 */
fq_status rmsnorm_int8(const int8_t* x, int32_t zp_x, const uint8_t* alpha, int32_t K, float m_x,
                       const int16_t* r, int64_t T, int32_t C, const float* gamma, float eps,
                       float s_out, int32_t zp_out, int32_t bits, int16_t* h, int8_t* y,
                       void* stream);
fq_status rmsnorm_rows_int8(const int8_t* x, int32_t zp_x, const uint8_t* alpha, int32_t K,
                            float m_x, const int16_t* r, int64_t T, int32_t C, const float* gamma,
                            float eps, int32_t bits, int16_t* h, int8_t* y, float* scales,
                            void* stream);

/*
 * A paged cache of keys and values.  Its arrays and sizes, for the three calls below:
 *
 *   k_pages  [pages, Hkv, page, d] int8, 16-byte aligned: a row for each key.
 *   v_pages  [pages, Hkv, d, page] int8, 16-byte aligned: a row for each channel.
 *   weight   [pages, Hkv, page] int64, 8-byte aligned: the attention weight that each
 *            key has received (NULL where it is not collected).
 *   table    [B, max_pages] int32: sequence b's key at place p lies in slot p % page of
 *            page table[b, p / page].  Entries behind a sequence's last key are not read.
 *   length   [B] int32: keys of each sequence, in [0, max_pages page].
 * pages in [1, 2^30], page a power of two in [16, 1024], d a multiple of 16 in
 * [16, 128], max_pages page at most 2^20, Hkv in [1, 1024], B Hkv in [0, 65536].
 * table and length are device arrays and cannot be checked here: of a longer length the
 * keys are those that the table can name, and new tokens (the last of it) may have places
 * beyond them; a length below 0 is 0.  A table entry that names no page reads as page 0 and
 * is never written through.  Sequences may share pages that no call writes.
 */

/*
 * Writes the keys and values of new tokens (as rope_qkv_int8 gives them) into a cache,
 * and a weight of 0.
 *
 *   k, v    [B, Hkv, L, d] int8, 16-byte aligned, L in [0, 2^20].
 *   n_new   NULL (L for every sequence) or [B] int32 in [0, L]: token i < n_new[b] of
 *           sequence b goes to place length[b] - n_new[b] + i, so length counts the new
 *           tokens.  Rows behind n_new[b] are not read; a token whose place is negative
 *           or beyond the table is left out.
 * All other slots are left as they were.  Places of two tokens that are one slot (pages
 * in the table twice) hold either token's bytes.
 * Errors: FQ_ERR_NULL (all but weight and n_new), FQ_ERR_SHAPE (sizes, or 2^24 or more
 * workgroups: B Hkv (L / 64 + 2)), FQ_ERR_PARAM (alignment).
 */
fq_status kv_cache_append_int8(const int8_t* k, const int8_t* v, int32_t B, int32_t Hkv, int32_t L,
                               int32_t d, const int32_t* n_new, int8_t* k_pages, int8_t* v_pages,
                               int64_t* weight, int32_t pages, int32_t page, const int32_t* table,
                               int32_t max_pages, const int32_t* length, void* stream);

/*
 * Attention of new tokens over a cache: lis_attention_qk's operator (MinMax-quantized
 * MatMul, Log-Int-Softmax, BitShift product) for rows of any length, of which each sees
 * a part, with shared key heads.
 *
 *   q       [B, Hq, L, d] int8 container, 16-byte aligned, zp_q; Hq = r Hkv, and head
 *           hq reads key head hq / r.  L in [0, 2^20], L r below 2^30.
 *   n_new   NULL (L) or [B] int32 in [0, L]: token i < n_new[b] stands at place
 *           length[b] - n_new[b] + i.  Rows behind n_new[b] are neither read nor written.
 *   causal  1: a token sees the keys up to its own place (all where that is beyond the
 *           table, none where it is negative); 0: all keys of its sequence.
 *   zp_k    does not change the result (see lis_attention_qk); it is validated.
 *   s_logit, bits (in [1, 4]), exp_n: as in lis_attention_head.
 *   out     [B, Hq, L, d] int32, 16-byte aligned: for a token that sees the keys J,
 *           out[c] = sum_{j in J} (v[j, c] - zp_v) 2^(2^b - 1 - code_j)
 *           with the codes of Log-Int-Softmax over J; 0 where J is empty.
 *   weight  NULL, or the cache's: weight[key's slot] += sum over the tokens and the r heads
 *           of its key head of 2^(2^b - 1 - code), 0 for a token that does not see it.
 *           (64-bit integer atomics: the sums do not depend on their order.)
 *   workspace  device scratch of fq_lis_attention_paged_workspace_bytes(B, Hq, Hkv, L,
 *           d, max_pages * page) bytes, 16-byte aligned, of one call at a time (NULL where that
 *           is 0); its contents on entry do not matter.  It grows with what the table can
 *           name, not with the lengths: for at most 16 rows (L r) of a key head 4 bytes for each
 *           row and key while that is at most 1 GiB in all, and never more than 17 MB beside.
 * Every row's sum is exact in 64 bits and out in 32: |out| <= 255 (1.5 2^15 + 2^20).
 * Errors: FQ_ERR_NULL, FQ_ERR_SHAPE (sizes, Hq, or 2^24 or more workgroups), FQ_ERR_PARAM
 * (zero points, causal, bits, exp_n, s_logit, alignment, workspace too small),
 * FQ_ERR_HEADROOM (that of lis_softmax_log4 with Lk = max_pages page).
 */
size_t fq_lis_attention_paged_workspace_bytes(int32_t B, int32_t Hq, int32_t Hkv, int32_t L,
                                              int32_t d, int64_t max_keys);
fq_status lis_attention_paged(const int8_t* q, int32_t B, int32_t Hq, int32_t Hkv, int32_t L,
                              int32_t d, const int32_t* n_new, const int8_t* k_pages,
                              const int8_t* v_pages, int64_t* weight, int32_t pages, int32_t page,
                              const int32_t* table, int32_t max_pages, const int32_t* length,
                              int32_t zp_q, int32_t zp_k, int32_t zp_v, int32_t causal,
                              float s_logit, int32_t bits, int32_t exp_n, int32_t* out,
                              void* workspace, size_t workspace_bytes, void* stream);

/*
 * Cuts each sequence of a cache to at most `keep` keys, by each key head on its own: the
 * `recent` last keys stay and, of the others, those of the largest weight (of equal ones
 * the first), keep in all.  They keep their order and are brought together in the
 * places [0, keep) of the pages that table_out names.
 *
 *   keep    in [1, 2^20]; recent in [0, keep].
 *   table_out  [B, max_out] int32, max_out page >= keep: table itself (then max_out =
 *           max_pages), or for each sequence the first entries of its row of table
 *           (in place: the sequence's pages are its own) or pages that nothing else in
 *           either table names.
 *   length_out [B] int32 (out): min(length, keep); it may be length itself.
 *   kept    [B, Hkv, keep] int32 (out): the places that stayed, ascending; -1 behind the last.
 *           A sequence of at most `keep` keys keeps them all (in other pages: is copied).
 * Slots behind the last key that stayed are left as they were.  The cache's weight may
 * not be NULL.
 * Errors: FQ_ERR_NULL, FQ_ERR_SHAPE (sizes, keep, max_out), FQ_ERR_PARAM (recent, alignment).
 */
fq_status kv_cache_evict(int8_t* k_pages, int8_t* v_pages, int64_t* weight, int32_t pages,
                         int32_t Hkv, int32_t page, int32_t d, const int32_t* table,
                         int32_t max_pages, const int32_t* length, int32_t B, int32_t keep,
                         int32_t recent, const int32_t* table_out, int32_t max_out,
                         int32_t* length_out, int32_t* kept, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* FQVIT_H */
