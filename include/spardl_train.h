/* spardl_train.h -- C ABI of libspardl_train.so: training operators whose
 * gradients the calls of spardl.h synchronise, for AMD Instinct MI355X
 * (gfx950): the residual RMS norm, the gated feed-forward block and the
 * distillation loss from a teacher's top logits, each with its backward pass.
 *
 * Conventions for every call below.
 *  - Array arguments are DEVICE pointers owned by the caller.  Matrices are
 *    row-major; ld_* is the distance of two rows in elements and at least the
 *    row's length.  Elements of a row are contiguous.  Any element-aligned
 *    pointer and any ld is taken; 16-byte aligned rows are the fast case.
 *  - dtype is the type of the activations, weights and logits; what is said
 *    to be float is fp32 in every case.  All sums, softmax statistics and
 *    norms are held in fp32; results are rounded once, to nearest even.
 *    Matrices without rows may be NULL; EINVAL for one that spans more than
 *    2^60 elements or is not aligned to its elements.
 *  - The library allocates nothing, keeps no state between calls, never
 *    synchronises and never copies between host and device.  Arguments are
 *    validated on the host first; on error nothing is enqueued and a negative
 *    status of spardl.h is returned (spardl_strerror names it).  Otherwise
 *    kernels are enqueued on `stream` and SPARDL_OK is returned.
 *  - ws is scratch device memory of at least the bytes that the call's
 *    *_workspace_bytes function returns, 256-byte aligned (EINVAL otherwise;
 *    ECAPACITY if it is smaller).  It needs no preparation and holds nothing
 *    between calls.  Calls on different streams must use different ws.  The
 *    bytes never fall as rows or tokens grow: the largest batch's workspace
 *    serves every smaller one of the same widths.
 *  - Results are deterministic: the same arguments give the same bits.
 *  - Inputs and outputs must not overlap unless a call says so.
 */
#ifndef SPARDL_TRAIN_H
#define SPARDL_TRAIN_H

#include "spardl.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
enum { SPARDL_BF16 = 0, SPARDL_FP16 = 1, SPARDL_FP32 = 2 };

/* Activations of the gated feed-forward block: g / (1 + exp(-g)), and
 * g (1 + erf(g / sqrt 2)) / 2. */
enum { SPARDL_ACT_SILU = 0, SPARDL_ACT_GELU = 1 };

/* Longest row of the RMS norm, most teacher logits of a row. */
#define SPARDL_NORM_MAX_DIM 16384
#define SPARDL_DISTILL_MAX_TOP 1024

/* Residual RMS norm.  For every row r < rows, with s = x[r] + res[r]:
 *   sum[r] = s,   rstd[r] = 1 / sqrt(mean(s^2) + eps),
 *   y[r]   = s * rstd[r] * weight.
 * y is computed from the unrounded s.  The squares and their sum are fp32: a row
 * of |s| past about 2^63 has rstd = 0.  res may be NULL (s = x); sum may be
 * NULL, or x or res itself (with its ld).  rstd may be NULL.
 * Errors: EINVAL for NULL x, weight or y, rows < 0, dim outside
 * [1, SPARDL_NORM_MAX_DIM], ld < dim, eps not >= 0, an unknown dtype. */
int spardl_rms_norm(const void* x, int64_t ld_x, const void* res, int64_t ld_res, const void* weight, void* sum,
                    int64_t ld_sum, void* y, int64_t ld_y, float* rstd, int64_t rows, int32_t dim, float eps,
                    int32_t dtype, hipStream_t stream);

/* Its backward pass.  With xhat = sum[r] * rstd[r] and g = dy[r] * weight:
 *   dx[r]   = rstd[r] (g - xhat mean(g xhat)) + dsum[r],
 *   dweight = sum over r of dy[r] xhat             (float [dim]).
 * dx is the gradient of x and of res alike.  dsum is the gradient that
 * arrives at sum along the residual stream; NULL means none.  dx may be dy or
 * dsum itself.  rows = 0 writes dweight = 0.
 * Errors: as spardl_rms_norm, plus EINVAL for NULL dy, sum, rstd, dx or
 * dweight and a NULL or misaligned ws; ECAPACITY. */
size_t spardl_rms_norm_workspace_bytes(int64_t rows, int32_t dim);
int spardl_rms_norm_backward(const void* dy, int64_t ld_dy, const void* sum, int64_t ld_sum, const void* weight,
                             const float* rstd, const void* dsum, int64_t ld_dsum, void* dx, int64_t ld_dx,
                             float* dweight, int64_t rows, int32_t dim, int32_t dtype, void* ws, size_t ws_bytes,
                             hipStream_t stream);

/* Distillation loss from a teacher's top logits.  Row r holds the student's
 * logits z over `vocab` tokens and a sparse list of `top` slots, each a token
 * (top_idx, int32) and the teacher's logit for it (top_val, float; both
 * [rows, top] with row distance ld_top).  Slots whose token is outside
 * [0, vocab) are empty.  With the temperature t,
 *   p = softmax over the row's slots of top_val / t,
 *   q = softmax over the vocabulary of z / t,
 *   loss[r] = t^2 sum over slots with p > 0 of p (log p - log q[token]),
 *   dlogits[r][v] = dloss[r] t (q[v] - sum of p over the slots of token v).
 * A row whose slots are all empty, or all -inf, has loss 0 and gradient 0
 * whatever its logits.  Logits of -inf have q = 0; a row of nothing else, and
 * a row that holds NaN or +inf, gives NaN.  stats[r] = (max of z, sum over v
 * of exp((z[v] - max) / t)), float [rows, 2], is what the backward pass takes.
 *
 * spardl_distill_loss: loss and stats.  spardl_distill_backward: dlogits from
 * stats and dloss (float [rows]).  spardl_distill_loss_backward: all three in
 * one call, which reads dloss up front (a mean over rows: 1 / rows each).
 * dlogits may be logits itself (with its ld): the logits are then replaced.
 * Errors: EINVAL for NULL pointers, rows < 0, vocab < 1, top outside
 * [1, SPARDL_DISTILL_MAX_TOP], ld below the row's length, a temperature that
 * is not a positive normal number (2^-126 at least, finite), an unknown dtype,
 * or a NULL or misaligned ws; ECAPACITY. */
size_t spardl_distill_workspace_bytes(int64_t rows, int32_t vocab);
int spardl_distill_loss(const void* logits, int64_t ld, const int32_t* top_idx, const float* top_val, int64_t ld_top,
                        int64_t rows, int32_t vocab, int32_t top, float temperature, float* loss, float* stats,
                        int32_t dtype, void* ws, size_t ws_bytes, hipStream_t stream);
int spardl_distill_backward(const void* logits, int64_t ld, const int32_t* top_idx, const float* top_val,
                            int64_t ld_top, const float* stats, const float* dloss, int64_t rows, int32_t vocab,
                            int32_t top, float temperature, void* dlogits, int64_t ld_d, int32_t dtype,
                            hipStream_t stream);
int spardl_distill_loss_backward(const void* logits, int64_t ld, const int32_t* top_idx, const float* top_val,
                                 int64_t ld_top, const float* dloss, int64_t rows, int32_t vocab, int32_t top,
                                 float temperature, float* loss, float* stats, void* dlogits, int64_t ld_d,
                                 int32_t dtype, void* ws, size_t ws_bytes, hipStream_t stream);

/* Gated feed-forward block of `tokens` rows (SPARDL_BF16 or SPARDL_FP16):
 *   gate = x w_gate^T,  up = x w_up^T        [tokens, hidden]
 *   h    = act(gate) up
 *   y    = h w_down^T                        [tokens, dim]
 * with w_gate and w_up [hidden, dim] and w_down [dim, hidden] (w_gate and
 * w_up may be halves of one matrix).  gate and up receive what the backward
 * pass needs, with one row distance ld_hidden; both may be NULL (inference).
 * h is computed from the unrounded gate and up and rounded to dtype, as the
 * operand of the second product, for any number of tokens.
 * workspace_bytes: backward != 0 for the backward pass (which needs more);
 * unaligned != 0 if dim or hidden is a multiple of 8 and yet a row of that
 * length of x, dy or a weight may start at an address that is not a multiple
 * of 16 bytes (a view), or has a row distance of 2^21 elements or more: the
 * products then work on aligned copies in ws, as they do by themselves for
 * other dim and hidden (but not for a forward pass of up to 16 tokens, which
 * reads rows as they are).  0 on invalid sizes.
 * Errors: EINVAL for NULL x, weights or y, one of gate and up without the
 * other, tokens < 0 or >= 2^31, dim or hidden outside [1, 2^20], a product of
 * two of them past 2^36, ld below the row's length, an unknown act, a dtype
 * other than the two, or a NULL or misaligned ws; ECAPACITY (also where
 * such views meet a workspace without room for copies, for any tokens). */
size_t spardl_gated_ffn_workspace_bytes(int64_t tokens, int32_t dim, int32_t hidden, int32_t backward,
                                        int32_t unaligned);
int spardl_gated_ffn(const void* x, int64_t ld_x, const void* w_gate, int64_t ld_gate, const void* w_up,
                     int64_t ld_up, const void* w_down, int64_t ld_down, void* y, int64_t ld_y, void* gate, void* up,
                     int64_t ld_hidden, int64_t tokens, int32_t dim, int32_t hidden, int32_t act, int32_t dtype,
                     void* ws, size_t ws_bytes, hipStream_t stream);

/* Its backward pass, from the gate and up that the forward pass wrote:
 *   dh = dy w_down,  dgate = dh up act'(gate),  dup = dh act(gate),
 *   dx = dgate w_gate + dup w_up,
 *   dw_gate = dgate^T x,  dw_up = dup^T x,  dw_down = dy^T h.
 * dh stays in fp32; dgate, dup and the recomputed h are rounded to dtype, as
 * operands of the products.  The weight gradients have the weights' shapes and are of
 * dw_dtype: dtype, or SPARDL_FP32, so that they can be written straight into
 * a worker's row of a gradient matrix (spardl_residual_add).  With accumulate
 * != 0 they are added to what dw_* holds, in fp32, and rounded to dw_dtype at
 * every call.  dx may be NULL (not computed).
 * tokens = 0 writes dw_* = 0 (nothing with accumulate).
 * Errors: as spardl_gated_ffn, plus EINVAL for NULL dy, gate, up or dw_*, and
 * a dw_dtype other than dtype and SPARDL_FP32. */
int spardl_gated_ffn_backward(const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, const void* gate,
                              const void* up, int64_t ld_hidden, const void* w_gate, int64_t ld_gate,
                              const void* w_up, int64_t ld_up, const void* w_down, int64_t ld_down, void* dx,
                              int64_t ld_dx, void* dw_gate, int64_t ld_dgate, void* dw_up, int64_t ld_dup,
                              void* dw_down, int64_t ld_ddown, int32_t dw_dtype, int32_t accumulate, int64_t tokens,
                              int32_t dim, int32_t hidden, int32_t act, int32_t dtype, void* ws, size_t ws_bytes,
                              hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* SPARDL_TRAIN_H */
