/*
 * aeris_fp8.h -- C ABI of the 8-bit path of a layer's projections (MI355X / gfx950), in the same
 * library as aeris_winattn.h and aeris_layer_ops.h.
 *
 * The projections of a transformer layer with operands of 8 bits: twice the matrix rate of bf16 and
 * half the operand bytes.  Rows come out of the operations in front of a projection in 8 bits (gated
 * residual and RMSNorm, SwiGLU gate) or are quantised by a call of their own (attention output,
 * gradients, weights); the projection multiplies them as they are.
 *
 * Quantised matrix.  The values are e4m3 (1 sign, 4 exponent, 3 mantissa bits; largest 448; no
 * infinity, 0x7f and 0xff are NaN), row-major [rows, cols], rows contiguous.  A BLOCK is
 * AERIS_FP8_BLOCK = 128 consecutive columns of one row (the last block of a row ends with it).  Every
 * block has one scale, a power of two held as one byte b that stands for 2^(b - 127); the scales are
 * [rows, aeris_fp8_scale_pitch(cols)] bytes, row-major, the entries behind the last block of a row are
 * 127 (1.0).  Scale bytes are 1 ... 254.  An entry is worth value * scale.  A block of x is quantised
 * with the smallest whole e >= -126 for which its largest finite |x| is at most 448 * 2^e:
 *     b = e + 127,   value = e4m3(x 2^-e), rounded to nearest even; NaN where x is not finite.
 * A scale that is a power of two leaves every value exact in bf16 (but below 2^-126, where bf16 has
 * multiples of 2^-133, and from 248 * 2^120 on, which rounds to 2^128), costs no precision (e4m3 keeps
 * its three mantissa bits anywhere in a block's range of 2^-14 to 1), and is applied by the matrix
 * instruction itself.
 *
 * Rows are tokens; the sample of row i is i / rows_per_sample, as in aeris_layer_ops.h.  Pointers are
 * DEVICE pointers, 16-byte aligned, owned by the caller; inputs are read-only, outputs fully
 * overwritten and, unless said otherwise, apart from the inputs.  The library allocates nothing and
 * never synchronises: calls only enqueue kernels on `hip_stream` (a hipStream_t passed as void*; NULL
 * is the default stream).  No atomics: results are bitwise reproducible.  Errors are the AERIS_ERR_*
 * codes of aeris_winattn.h; arguments are checked before anything is launched.
 */
#ifndef AERIS_FP8_H
#define AERIS_FP8_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define AERIS_FP8_BLOCK 128
/* Columns of a quantised matrix: a multiple of 64, at most this. */
#define AERIS_MAX_FP8_COLUMNS 65536

/* Bytes between the scales of consecutive rows: one per block, rounded up to a multiple of 4.
 * 0 if cols is no valid number of columns. */
int32_t aeris_fp8_scale_pitch(int32_t cols);

/*
 * Quantises x [n_rows, channels], x_dtype AERIS_DT_BF16 or AERIS_DT_F32, rows contiguous:
 *   x8, xs   : x by rows, [n_rows, channels] and its scales (blocks along the channels)
 *   xt8, xts : the transpose of x by rows, [channels, n_rows] and its scales (blocks along the rows
 *              of x); for a weight [out_features, channels], the operand of its gradient product.
 *              Needs n_rows % 64 == 0 and n_rows <= AERIS_MAX_FP8_COLUMNS.
 * Either pair may be NULL (not wanted), not both; x is read once.  channels % 64 == 0.
 */
int aeris_fp8_quantize(const void* x, int32_t x_dtype, int64_t n_rows, int32_t channels, void* x8,
                       void* xs, void* xt8, void* xts, void* hip_stream);

/*
 * Gated residual, RMSNorm and adaptive modulation in one pass over the rows, with the normalised rows
 * quantised for the projection behind them (Model Architecture section: pre-RMSNorm and the values
 * alpha, beta, gamma of the adaptive layer norm):
 *     s   = bf16(x + alpha_b y)
 *     r   = (mean_c s_c^2 + eps)^(-1/2)
 *     h_c = s_c r w_c (1 + gamma_{b,c}) + beta_{b,c},   h8, hs = h quantised
 * x, y, s [n_rows, channels] bf16; w [channels]; alpha, beta, gamma [n_samples, channels] fp32; r
 * [n_rows] fp32 or NULL (not wanted).  s may alias x or y.  Without a residual to add (y NULL): s = x,
 * alpha is not read and s not written.  fp32 arithmetic; s and r are the bits of
 * aeris_gate_residual_fwd and aeris_rmsnorm_adaln_fwd, and h is quantised without a rounding to bf16.
 * Backward: the rounding to 8 bits passes a gradient dh unchanged, so the gradients are those of
 * aeris_rmsnorm_adaln_bwd_residual on (s, r) and, from its dx, of aeris_gate_residual_bwd.
 * Limits: channels % 64 == 0, channels <= AERIS_MAX_CHANNELS, n_rows % rows_per_sample == 0, at most
 * 2^20 samples.
 */
int aeris_residual_norm_fp8_fwd(const void* x, const void* y, const float* alpha, const float* w,
                                const float* gamma, const float* beta, float eps, int64_t n_rows,
                                int64_t rows_per_sample, int32_t channels, void* s, float* r,
                                void* h8, void* hs, void* hip_stream);

/*
 * SwiGLU gate with its result quantised for the down-projection: g = silu(u) v, uv [n_rows, 2*hidden] =
 * [u | v] bf16; g8, gs = g quantised, without a rounding to bf16 before.  g is held wherever fp32 and the
 * format hold it, also where silu(u) is below the normal numbers and v is large (aeris_swiglu_fwd gives zero
 * from u = -87.4 on).  An infinite u, or a g past fp32, gives NaN.
 * hidden % 64 == 0, hidden <= AERIS_MAX_FP8_COLUMNS.  Backward: aeris_swiglu_bwd.
 */
int aeris_swiglu_fp8_fwd(const void* uv, int64_t n_rows, int32_t hidden, void* g8, void* gs,
                         void* hip_stream);

/*
 * Projection of quantised operands: y [n_rows, out_features] = x w^T, bf16, with x8, xs
 * [n_rows, channels] and w8, ws [out_features, channels] quantised by rows.
 * channels % 64 == 0, out_features % 64 == 0, both <= AERIS_MAX_FP8_COLUMNS; n_rows >= 1, and less
 * than 2^25 tiles of 64 x 64 in y.
 * Products of blocks accumulate in fp32 over the channels.  Inside the matrix instruction eight
 * neighbouring products are added before they join the accumulator, and what is below 2^-13 of the
 * largest of the eight is dropped; 16 channels at a time join it, which costs up to its last bit:
 *     |error| <= 7 * 2^-13 * (sum over groups of eight channels of the largest |x w| of the group)
 *                + (channels / 16 + 8) * 2^-23 * (sum over channels of |x w|),
 * and y is rounded to bf16 (up to 2^-8 = 4e-3 of it).  For operands of like size that is about 1e-5 of
 * the result for up to a few thousand channels; with the most channels and one large block among them
 * the second term comes to 5e-4 of the sum of magnitudes, of which 2e-4 has been seen.
 */
int aeris_linear_fp8_fwd(const void* x8, const void* xs, const void* w8, const void* ws,
                         int64_t n_rows, int32_t channels, int32_t out_features, void* y,
                         void* hip_stream);

/*
 * Gradients of that projection, given dy [n_rows, out_features] bf16:
 *     dx      [n_rows, channels]       = Q(dy) wt^T  bf16; dy quantised by rows in the workspace,
 *                                        wt8, wts [channels, out_features] the transposed weight of
 *                                        aeris_fp8_quantize; summed as in aeris_linear_fp8_fwd
 *     dweight [out_features, channels] = dy^T x      fp32, overwritten; products in bf16, in which dy
 *                                        and the values of x8, xs are exact, added as in
 *                                        aeris_linear_bwd: a gradient kept in fp32 would not be
 *                                        one after 8-bit products, which lose 1e-5 of it
 * Either output may be NULL (then its operands x8, xs or wt8, wts may be too).
 * Limits as in aeris_linear_fp8_fwd, and out_features * channels < 2^31.  workspace: at least
 * aeris_linear_fp8_bwd_workspace_bytes_for(...) bytes of the outputs that are wanted (dx alone needs
 * room for dy in 8 bits only; aeris_linear_fp8_bwd_workspace_bytes(...) is the size for both), 0 if
 * the size is not accepted; contents undefined before and after.
 */
size_t aeris_linear_fp8_bwd_workspace_bytes_for(int64_t n_rows, int32_t channels, int32_t out_features,
                                                int32_t want_dx, int32_t want_dweight);
size_t aeris_linear_fp8_bwd_workspace_bytes(int64_t n_rows, int32_t channels, int32_t out_features);
int aeris_linear_fp8_bwd(const void* x8, const void* xs, const void* wt8, const void* wts,
                         const void* dy, int64_t n_rows, int32_t channels, int32_t out_features,
                         void* dx, float* dweight, void* workspace, size_t workspace_bytes,
                         void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* AERIS_FP8_H */
