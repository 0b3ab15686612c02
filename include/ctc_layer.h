/*
 * ctc_layer.h -- the output layer around the CTC path, with its states held in 8 bits (gfx950).
 *
 * The activations that ctc_loss_and_grad and ctc_best_path read are an output layer's: a norm of the
 * network's last states, then a matrix product with a row of weights per symbol (Section 3.1 of the
 * paper).  The gradient that ctc_loss_and_grad writes is where that layer's backward pass begins.
 * The calls below are that layer for states in 8-bit integers with a scale per row:
 *
 *   forward    ctc_rms_norm_i8        residual added, root-mean-square norm, rows rounded to 8 bits
 *              ctc_linear_i8          activations from rows and weights in 8 bits
 *   backward   ctc_weight_gradient_i8 the weights' gradient from CTC's gradient and the 8-bit rows that
 *                                     the forward pass kept (its activation checkpoint)
 *              ctc_rms_norm_backward  the norm's gradient
 *   both       ctc_quantize_rows      any rows to 8 bits: weights per symbol, states to keep
 *              ctc_dequantize_rows    and back
 *              ctc_pack_frames        the list of a minibatch's frames, for all of the above
 *
 * Same library, same manner as ctc_mi355x.h: plain C ABI, every buffer is the caller's, all work is
 * enqueued on the given stream, nothing waits, nothing is allocated, errors are reported by status
 * only, and on an error found during validation nothing has been enqueued.  No call reads host
 * memory or keeps anything between calls, so all of them may be recorded into a HIP graph; a replay
 * reads every device buffer afresh.  Results are bitwise repeatable from run to run on one device.
 * Calls that may overlap in time need outputs and workspaces of their own.
 * As for the other calls, `stream` and all buffers belong to the calling thread's current device.
 *
 * Rows.  States are matrices [rows, H], activations [rows, A], the last index fastest, without gaps.
 * For a minibatch, rows = T * B and row t * B + b is frame t of utterance b, the layout [T, B, A] of
 * ctc_loss_and_grad; for single frames (streaming) rows is their number.
 *
 * Frames.  `frames` (device) [1 + rows] int32 or NULL: the rows that count.  frames[0] is their
 * number n (taken as 0 below 0 and as `rows` above), frames[1..n] their indices, in any order;
 * entries outside [0, rows) are skipped.  Rows that are not listed take no part: what they hold is of
 * no consequence, and stays.  Row-wise outputs of a row that is listed twice are those of one
 * listing, provided that no output is one of the call's inputs; sums over rows count it twice.
 * NULL: all rows.  The grids are sized by `rows`, so that n may change from replay to replay.
 *
 * Rows in 8 bits.  `q` (device, 16-byte aligned) [rows, ctc_row_pitch(H)] int8: a row's H values in
 * -127..127, then zeros up to the next multiple of 128.  `scales` (device) [rows] float: value k of
 * row r stands for q[r][k] * scales[r].  Calls that write rows in 8 bits write those zeros too; the calls that
 * multiply rows read them and rely on them.  Given the row u_0 .. u_(H-1) with m = max |u_k|, q_k is the
 * whole number nearest to 127 u_k / m in real arithmetic (of two equally near ones the even one), and
 * the scale is m / 127; a row of zeros has scale 0.  A row that holds an infinity or a NaN gets zeros
 * and the scale NaN.
 *
 * Limits.  rows, H, A >= 1; H <= CTC_MAX_STATE_WIDTH, rows <= 2^30, A <= 2^20: more is
 * refused with CTC_STATUS_UNSUPPORTED.  Pointers are aligned to their element type unless more is
 * said; a misaligned one, a null pointer not marked as allowed, and an output that overlaps another
 * buffer of the call (unless marked "may be") are refused with CTC_STATUS_INVALID_VALUE.
 */
#ifndef CTC_LAYER_H
#define CTC_LAYER_H

#include "ctc_mi355x.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Widest state: sums of 16384 products of two 8-bit numbers stay far inside 32 bits. */
#define CTC_MAX_STATE_WIDTH 16384

/* Bytes from one row in 8 bits to the next: H rounded up to a multiple of 128 (0 for H < 1 or
 * H > CTC_MAX_STATE_WIDTH).  Host computation. */
int ctc_row_pitch(int H);

/*
 * The list of a minibatch's frames, to be made once per minibatch and given to all its calls.
 *
 *   input_lengths (device) [B]; below 0 counts as 0, above T as T
 *   frames        (device) [1 + T*B]: receives the number n of frames and the n rows t * B + b with
 *                 t < input_lengths[b], ascending: frame by frame, a frame's in the order of the
 *                 utterances; what lies behind them stays.
 *   B is at most 65535 (as for ctc_loss_and_grad), T * B at most 2^30
 */
ctc_status_t ctc_pack_frames(const int32_t *input_lengths, int T, int B, int32_t *frames, hipStream_t stream);

/*
 * Rows to 8 bits.
 *
 *   x       (device) [rows, H] of type dtype
 *   q       (device) [rows, ctc_row_pitch(H)]
 *   scales  (device) [rows]
 */
ctc_status_t ctc_quantize_rows(const void *x, const int32_t *frames, int rows, int H, ctc_dtype_t dtype,
                               int8_t *q, float *scales, hipStream_t stream);

/* And back: out (device) [rows, H] of type dtype = q * scales, a product in fp32, rounded to dtype. */
ctc_status_t ctc_dequantize_rows(const int8_t *q, const float *scales, const int32_t *frames, int rows, int H,
                                 ctc_dtype_t dtype, void *out, hipStream_t stream);

/*
 * Residual, root-mean-square norm, 8 bits.  For each row
 *
 *     z = x + residual, rounded to dtype
 *     u_k = z_k * weight_k, rounded to fp32
 *     q, s = u in 8 bits as above;   scale = s / sqrt(mean_k z_k^2 + eps)
 *
 * (the norm's factor is common to a row, so it goes into the scale alone).
 *
 *   x         (device) [rows, H] of type dtype
 *   residual  (device) the same, or NULL: z = x
 *   weight    (device) [H] float, or NULL: ones
 *   eps       finite and > 0
 *   sum       (device) [rows, H] of type dtype: receives z, for the next layer and for
 *             ctc_rms_norm_backward; may be x or residual itself; NULL: not written
 *   q, scales as for ctc_quantize_rows
 */
ctc_status_t ctc_rms_norm_i8(const void *x, const void *residual, const float *weight, float eps,
                             const int32_t *frames, int rows, int H, ctc_dtype_t dtype,
                             void *sum, int8_t *q, float *scales, hipStream_t stream);

/*
 * Gradient of the norm, of y = z * weight * r with r = 1 / sqrt(mean z^2 + eps): the rounding to 8 bits
 * passes gradients through unchanged.
 *
 *     dsum = r (dy weight - z r^2 mean_k(dy weight z)) + dresidual
 *     dweight_k = sum over the listed rows of  dy_k z_k r
 *
 *   dy         (device) [rows, H] of type dtype: gradient of y
 *   sum        (device) [rows, H] of type dtype: the z that ctc_rms_norm_i8 stored
 *   weight, eps, frames: as in the forward call
 *   dresidual  (device) [rows, H] of type dtype, or NULL: the gradient that reaches z by other ways
 *   dsum       (device) [rows, H] of type dtype: gradient of z, and so of x and of residual each;
 *              may be dy, sum or dresidual itself
 *   dweight    (device) [H] float, or NULL: not computed.  Zeros if no row is listed.
 *   workspace  (device) 256-byte aligned, ctc_rms_norm_workspace_size bytes; NULL allowed without dweight
 */
ctc_status_t ctc_rms_norm_workspace_size(int rows, int H, size_t *bytes_out);
ctc_status_t ctc_rms_norm_backward(const void *dy, const void *sum, const float *weight, float eps,
                                   const void *dresidual, const int32_t *frames, int rows, int H,
                                   ctc_dtype_t dtype, void *dsum, float *dweight,
                                   void *workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * Activations from rows and weights in 8 bits:
 *
 *     logits[r][a] = scales[r] * weight_scales[a] * sum_k q[r][k] * weight_q[a][k]  + bias[a]
 *
 * The sums are exact; from there on all is in fp32 (the sum as such a number, the product of the scales, its product
 * with the sum and the bias added in one step), rounded to dtype at last.  Rows that are not listed are never read by ctc_loss_and_grad either.
 *
 *   q, scales                (device) [rows, ctc_row_pitch(H)], [rows]
 *   weight_q, weight_scales  (device) [A, ctc_row_pitch(H)] (16-byte aligned), [A]: the weights as
 *                            ctc_quantize_rows(weights, NULL, A, H, ...) lays them out
 *   bias                     (device) [A] float, or NULL
 *   logits                   (device) [rows, A] of type dtype
 */
ctc_status_t ctc_linear_i8(const int8_t *q, const float *scales, const int8_t *weight_q,
                           const float *weight_scales, const float *bias, const int32_t *frames,
                           int rows, int H, int A, ctc_dtype_t dtype, void *logits, hipStream_t stream);

/*
 * Gradient of the weights and of the bias, from the activations' gradient and the rows in 8 bits:
 *
 *     dweight[a][k] = sum over the listed rows of  grads[r][a] * scales[r] * q[r][k]
 *     dbias[a]      = sum over the listed rows of  grads[r][a]
 *
 * grads[r][a] * scales[r] is rounded to fp32 and enters the matrix cores in parts of 16 bits that hold it to
 * within 2^-23 of itself or 2^-133, if that is more (where symbols, states and rows are many: 2^-38 of its symbol's
 * largest, if that is more); sums are in fp32, in an order that the sizes and the list fix.  A product that is an infinity or a NaN gives
 * its symbol's row of dweight NaNs.
 *
 *   grads      (device) [rows, A] of type dtype, as ctc_loss_and_grad writes them
 *   q, scales  (device) as ctc_rms_norm_i8 or ctc_quantize_rows wrote them
 *   dweight    (device) [A, H] float.  Zeros if no row is listed.
 *   dbias      (device) [A] float, or NULL
 *   workspace  (device) 256-byte aligned, ctc_weight_gradient_workspace_size bytes
 *
 * A workspace made for the largest minibatch serves all: the size never shrinks as rows grow, and a call takes
 * one of the size for its own rows or for more (so too for ctc_rms_norm_workspace_size).
 */
ctc_status_t ctc_weight_gradient_workspace_size(int rows, int H, int A, size_t *bytes_out);
ctc_status_t ctc_weight_gradient_i8(const void *grads, const int8_t *q, const float *scales,
                                    const int32_t *frames, int rows, int H, int A, ctc_dtype_t dtype,
                                    float *dweight, float *dbias,
                                    void *workspace, size_t workspace_bytes, hipStream_t stream);

/* Raw hipError_t value of the most recent HIP failure of these calls in the calling thread (0 if none). */
int ctc_layer_last_hip_error(void);

#ifdef __cplusplus
}
#endif

#endif /* CTC_LAYER_H */
