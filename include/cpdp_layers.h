/*
 * cpdp_layers.h — worker-batched layers of libcpdp: the operators next to the
 * optimizer and reconcile steps that make a step's gradients, for all W
 * workers in one call.
 *
 *   norm        s = x + residual;  y = weight * s / sqrt(mean(s^2) + eps),
 *               y optionally held in 8 bits; its backward pass
 *   checkpoint  activations held in 8 bits for the backward pass, and the
 *               weight gradient that reads them: dW = dy^T x^
 *   recurrence  h_t = a_t h_(t-1) + (1 - a_t) v_t, a = sigmoid(gate); its
 *               backward pass, and its step for one token
 *
 * Layout. Arrays [W][M][D] hold worker w's M tokens (rows) of D features.
 * Features are contiguous; inputs have a worker stride and a row stride, in
 * elements (arguments x_worker, x_row and the like; both >= 0, and 0 repeats
 * a row). Outputs are contiguous unless they have a stride of their own. Weights are float32, and
 * weights and their gradients lie inside the workers' [W][N] parameter and
 * gradient rows (cpdp.h): worker w's is at pointer + w * stride, contiguous,
 * at any element alignment. Other pointers are aligned to their element.
 * Outputs must not overlap inputs or each other. An output whose own strides
 * make its parts overlap is refused.
 *
 * Types. Activations are float32 or bfloat16 (cpdp_dtype); all arithmetic,
 * sums and states are float32, and an output is rounded once (to nearest even)
 * when it is stored. Infinities and NaN follow from the formulas, except that an
 * infinite state or gradient of the recurrence may go on as NaN, where the steps
 * of a long sequence are shared out. A row whose
 * sum of squares is above the float32 range (a root mean square above
 * 1.8e19 / sqrt(D)) has the scale k = 0 in the norm.
 *
 * 8 bits. Blocks of 32 neighbouring features share an exponent e, the least
 * with max|x| <= 127 * 2^e, kept between -126 and 121; a value is held as the
 * whole number nearest to x / 2^e (ties to even), within +-127. So a value
 * that is read back is exact in bfloat16. codes: int8 [W][M][P], with
 * P = 32 * ceil(D / 32) (the padding is written as 0), 16-byte aligned;
 * exponents: uint8 [W][M][P / 32], e + 127. A block in which a value is infinite or NaN has the
 * exponent byte 255 and reads back as NaN.
 *
 * Calls launch on `stream` (a cudaStream_t; NULL is the default stream) of the
 * current device and return without waiting; they may be captured into a CUDA
 * graph. Nothing is kept between calls. A call that needs a workspace takes
 * one of at least the size that its _workspace function gives (device memory,
 * 16-byte aligned, contents of no importance), in use until the call's work on
 * the stream is done. Errors are status codes; the message is at
 * cpdp_last_error(NULL). A refused call launches nothing.
 *
 * Limits: 1 <= W <= 4096, 0 <= M, 1 <= D <= 2^30, W * M * D <= 2^40 and
 * W * M <= 2^31 - 1; further ones at each call. A call with no rows (M, B or T
 * of 0) writes the gradients or states that it owes (zeros, or the initial
 * state) and nothing else; pointers to arrays of no elements may be NULL.
 */
#ifndef CPDP_LAYERS_H
#define CPDP_LAYERS_H

#include "cpdp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rows of the norm have at most this many features. */
#define CPDP_NORM_MAX_FEATURES 16384

/* The recurrence keeps the state at every so many steps for its backward pass. */
#define CPDP_CARRY_STEPS 16

/*
 * cpdp_add_rmsnorm — the residual's addition and the norm.
 *   x, residual  [W][M][D] of dtype; residual may be NULL: s is x then
 *   weight       float32, worker w's D values at weight + w * weight_worker
 *   eps          > 0
 *   s            [W][M][D] of dtype, x + residual rounded to dtype; the norm
 *                is of the rounded s. NULL without a residual.
 *   codes, exponents  NULL, or the 8-bit form of y
 *   y            [W][M][D]: of dtype; where codes are given, bfloat16, the
 *                values that the codes stand for
 */
cpdp_status cpdp_add_rmsnorm(const void *x, int64_t x_worker, int64_t x_row,
                             const void *residual, int64_t residual_worker, int64_t residual_row,
                             const float *weight, int64_t weight_worker, cpdp_dtype dtype,
                             int W, int64_t M, int D, float eps, void *y, void *s,
                             int8_t *codes, uint8_t *exponents, void *stream);

/*
 * cpdp_add_rmsnorm_backward — gradients of the norm. With k = 1 / sqrt(mean(s^2) + eps),
 *   dx = ds + k * dy * weight - s * k^3 * mean(dy * weight * s)
 *   dweight = sum over the worker's rows of dy * s * k
 *   dy, s, ds    [W][M][D] of dtype: the gradient of y, what the forward pass
 *                gave as s (x without a residual), and the gradient that
 *                reaches s by other ways (NULL: none). Rounding y to 8 bits
 *                counts as the identity.
 *   dx           [W][M][D] of dtype: the gradient of x, and of residual
 *   dweight      dweight_dtype, worker w's at dweight + w * dweight_worker;
 *                the order of its sums is fixed by the sizes and by whether
 *                every row is one of whole 16-byte pieces
 */
size_t cpdp_add_rmsnorm_backward_workspace(int W, int64_t M, int D);
cpdp_status cpdp_add_rmsnorm_backward(const void *dy, int64_t dy_worker, int64_t dy_row,
                                      const void *s, int64_t s_worker, int64_t s_row,
                                      const void *ds, int64_t ds_worker, int64_t ds_row,
                                      const float *weight, int64_t weight_worker, cpdp_dtype dtype,
                                      int W, int64_t M, int D, float eps, void *dx,
                                      void *dweight, int64_t dweight_worker, cpdp_dtype dweight_dtype,
                                      void *workspace, size_t workspace_bytes, void *stream);

/*
 * cpdp_checkpoint — the 8-bit form of x; values (NULL: not wanted) receives
 * the values that it stands for, bfloat16 [W][M][D]. cpdp_restore writes them
 * from the 8-bit form.
 */
cpdp_status cpdp_checkpoint(const void *x, int64_t x_worker, int64_t x_row, cpdp_dtype dtype,
                            int W, int64_t M, int D, int8_t *codes, uint8_t *exponents,
                            void *values, void *stream);
cpdp_status cpdp_restore(const int8_t *codes, const uint8_t *exponents, int W, int64_t M, int D,
                         void *values, void *stream);

/*
 * cpdp_weight_gradient — dW[w][o][i] = sum over m of dy[w][m][o] * x^[w][m][i],
 * x^ the values of an 8-bit checkpoint [W][M][I].
 *   dy    [W][M][O]; float32 dy is rounded to bfloat16, the type of the
 *         product's operands
 *   dW    dW_dtype, worker w's [O][I] at dW + w * dW_worker. The tensor core
 *         sums 2,048 tokens at a time, cutting off what does not fit into
 *         float32; those sums are added in float32, rounded to nearest, in an
 *         order fixed by the sizes.
 * A dy that is not bfloat16 at a multiple of 16 bytes, with strides of whole
 * multiples of 8 elements and rows apart, is first copied to such a form in the
 * workspace.
 */
size_t cpdp_weight_gradient_workspace(const void *dy, int64_t dy_worker, int64_t dy_row, cpdp_dtype dy_dtype,
                                      int W, int64_t M, int O, int I);
cpdp_status cpdp_weight_gradient(const void *dy, int64_t dy_worker, int64_t dy_row, cpdp_dtype dy_dtype,
                                 const int8_t *codes, const uint8_t *exponents,
                                 int W, int64_t M, int O, int I,
                                 void *dW, int64_t dW_worker, cpdp_dtype dW_dtype,
                                 void *workspace, size_t workspace_bytes, void *stream);

/*
 * cpdp_gated_recurrence — h_t = a_t h_(t-1) + (1 - a_t) v_t with
 * a = sigmoid(gate), for B sequences of T <= 2^30 steps and D channels.
 *   gate, value  [B][T][D] of dtype, with a sequence and a step stride
 *   h0           float32 [B][D], the states before the first step (NULL: 0)
 *   lengths      int32 [B], each sequence's number of steps, clamped to 0..T
 *                (NULL: T for all). Nothing is read beyond a length; h is 0
 *                there and the state stays.
 *   h            [B][T][D] of dtype
 *   h_last       float32 [B][D], the states after the last step
 *   carry        NULL, or float32 [B][ceil(T / CPDP_CARRY_STEPS)][D]: the
 *                states before steps 0, CPDP_CARRY_STEPS, ..., for the
 *                backward pass (defined up to each sequence's length)
 */
size_t cpdp_gated_recurrence_workspace(int B, int64_t T, int D);
cpdp_status cpdp_gated_recurrence(const void *gate, int64_t gate_seq, int64_t gate_step,
                                  const void *value, int64_t value_seq, int64_t value_step,
                                  cpdp_dtype dtype, int B, int64_t T, int D,
                                  const float *h0, const int32_t *lengths,
                                  void *h, float *h_last, float *carry,
                                  void *workspace, size_t workspace_bytes, void *stream);

/*
 * cpdp_gated_recurrence_backward — with G_t = dh_t + a_(t+1) G_(t+1), started
 * by dh_last after a sequence's last step:
 *   dvalue_t = (1 - a_t) G_t,  dgate_t = G_t (h_(t-1) - v_t) a_t (1 - a_t),
 *   dh0 = a_0 G_0
 *   dh              [B][T][D] of dtype, with strides; not read beyond a length
 *   dh_last         float32 [B][D] (NULL: 0)
 *   carry           what the forward pass wrote; the states between are made
 *                   again from gate and value
 *   dgate, dvalue   of dtype, with one sequence and one step stride for both
 *                   (two halves of one [B][T][2 D], say; all of a sequence's
 *                   steps between two sequences, or all sequences between two
 *                   steps); 0 beyond a length
 *   dh0             float32 [B][D] (NULL: not wanted)
 * The workspace is that of the forward pass.
 */
cpdp_status cpdp_gated_recurrence_backward(const void *dh, int64_t dh_seq, int64_t dh_step,
                                           const void *gate, int64_t gate_seq, int64_t gate_step,
                                           const void *value, int64_t value_seq, int64_t value_step,
                                           cpdp_dtype dtype, int B, int64_t T, int D,
                                           const float *carry, const float *dh_last, const int32_t *lengths,
                                           void *dgate, void *dvalue, int64_t grad_seq, int64_t grad_step,
                                           float *dh0, void *workspace, size_t workspace_bytes, void *stream);

/*
 * cpdp_gated_recurrence_step — one token for each of B sequences: state
 * (float32 [B][D]) is replaced by the next one, and h ([B][D] of dtype)
 * receives it rounded. gate, value: [B][D] of dtype with a sequence stride.
 */
cpdp_status cpdp_gated_recurrence_step(const void *gate, int64_t gate_seq, const void *value, int64_t value_seq,
                                       cpdp_dtype dtype, int B, int D, float *state, void *h, void *stream);

/*
 * cpdp_layer_timeouts — the number of bounded waits that ran out since the last
 * call (0 expected): the weight gradient's warps wait for the slots of a ring,
 * for some seconds at most. A block in which one ran out writes NaN for all of
 * its tile of dW. Waits for the device.
 */
cpdp_status cpdp_layer_timeouts(int64_t *count);

#ifdef __cplusplus
}
#endif

#endif /* CPDP_LAYERS_H */
