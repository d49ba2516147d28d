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
 *   loss        softmax cross entropy over a vocabulary from the activations
 *               and the head's weight, without the logits; its backward pass
 *   convolution y_t = silu(bias + sum_k weight_k x_(t-K+1+k)) over time, for each
 *               channel; its backward pass, and its step for one token
 *   scan        h_t = exp(-dt exp(a_log)) h_(t-1) + dt u_t b_t for some states per
 *               channel, y_t = (sum_n c_t h_t + skip u_t) silu(z_t); its backward
 *               pass, and its step for one token
 *   clipping    the norm of each worker's gradient row, and the row scaled down
 *               to a largest norm
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
 * cpdp_linear_cross_entropy — for each token, with the logits l = weight x
 * over the vocabulary's V words,
 *   lse = log(sum(exp(l))),  loss = lse - l[target]
 *   x        [W][M][D] of dtype
 *   weight   [W][V][D] of dtype, with a worker and a row stride
 *   targets  int64 [W][M], contiguous. Where a target is negative the token is
 *            ignored: its loss is 0 (lse is not). Where it is V or more its loss
 *            is NaN.
 *   loss, lse  float32 [W][M]
 * The logits are float32 sums and stay on the chip. float32 operands of more than
 * 24 tokens are split into three bfloat16 parts each, and products below 2^-24 of
 * the largest part's are left out; an infinite operand gives NaN there where the
 * formula has an infinity. M and V are at most 2^30; W * V and the elements of [W][M][V] are
 * bounded as those of an array.
 */
size_t cpdp_linear_cross_entropy_workspace(const void *x, int64_t x_worker, int64_t x_row,
                                           const void *weight, int64_t weight_worker, int64_t weight_row,
                                           cpdp_dtype dtype, int W, int64_t M, int V, int D);
cpdp_status cpdp_linear_cross_entropy(const void *x, int64_t x_worker, int64_t x_row,
                                      const void *weight, int64_t weight_worker, int64_t weight_row,
                                      const int64_t *targets, cpdp_dtype dtype, int W, int64_t M, int V, int D,
                                      float *loss, float *lse, void *workspace, size_t workspace_bytes, void *stream);

/*
 * cpdp_linear_cross_entropy_backward — with d = dloss (exp(l - lse) - onehot(target)),
 *   dx = d weight,  dweight = d^T x
 * The logits are made again, for a piece of the vocabulary at a time.
 *   dloss    float32 [W][M]: the gradient of each token's loss
 *   lse      what the forward pass gave
 *   dx       [W][M][D] of dtype; 0 in the rows of ignored tokens, whose x, dloss
 *            and lse reach nothing, infinite and NaN ones included
 *   dweight  dweight_dtype, worker w's [V][D] at dweight + w * dweight_worker
 * d is float32, held in three bfloat16 parts (what of it is below 2^-133 counts
 * as 0) that stay below 1 GiB at a time or hold 256 words. float32 operands are
 * split into three parts for any number of tokens, where an infinite dloss or
 * operand gives NaN in the place of an infinity. Sums are float32, in an order
 * fixed by the sizes, by whether weight is read in place (16-byte pieces), and by
 * the type.
 */
size_t cpdp_linear_cross_entropy_backward_workspace(const void *x, int64_t x_worker, int64_t x_row,
                                                    const void *weight, int64_t weight_worker, int64_t weight_row,
                                                    cpdp_dtype dtype, int W, int64_t M, int V, int D);
cpdp_status cpdp_linear_cross_entropy_backward(const float *dloss, const void *x, int64_t x_worker, int64_t x_row,
                                               const void *weight, int64_t weight_worker, int64_t weight_row,
                                               const int64_t *targets, const float *lse,
                                               cpdp_dtype dtype, int W, int64_t M, int V, int D, void *dx,
                                               void *dweight, int64_t dweight_worker, cpdp_dtype dweight_dtype,
                                               void *workspace, size_t workspace_bytes, void *stream);

/*
 * cpdp_clip_gradients — norm = sqrt(sum(g^2)) of each worker's row of N
 * gradients, and g * min(1, max_norm / norm).
 *   grads     of dtype, worker w's N values at grads + w * grads_worker, at any
 *             element alignment
 *   max_norm  > 0; infinity: every row stays as it is, to the bit, whatever its
 *             norm
 *   norms     float32 [W]. The sum of squares is float32, in an order fixed by
 *             the sizes and the rows' alignment, and neither overflows nor
 *             vanishes where the norm itself is a float32 number.
 *   out       of dtype, with a worker stride; or grads itself, with the same
 *             stride: rows whose norm is not above max_norm are not written then.
 *             Other rows that overlap those of grads are refused.
 * A row whose norm is above the float32 range, or that has an infinite value, has
 * the norm infinity; one with a NaN has the norm NaN. Under a finite max_norm the
 * first becomes 0 (its infinite values NaN) and the second NaN throughout. W * N is
 * at most 2^40; with N = 0 the norms are 0.
 */
size_t cpdp_clip_gradients_workspace(int W, int64_t N);
cpdp_status cpdp_clip_gradients(const void *grads, int64_t grads_worker, cpdp_dtype dtype, int W, int64_t N,
                                float max_norm, float *norms, void *out, int64_t out_worker,
                                void *workspace, size_t workspace_bytes, void *stream);

/* Taps of the convolution: 2 to this many. */
#define CPDP_CONV_MAX_TAPS 4

/*
 * cpdp_causal_conv — for B sequences of T <= 2^30 steps and D channels,
 *   y_t = v_t * sigmoid(v_t),  v_t = bias + sum over k < K of weight[k] * x_(t-K+1+k)
 * Worker w's weights are those of the sequences w * B / W to (w + 1) * B / W - 1
 * (W divides B).
 *   x        [B][T][D] of dtype, with a sequence and a step stride
 *   weight   float32, worker w's [D][K] at weight + w * weight_worker
 *   bias     float32, worker w's [D] at bias + w * bias_worker
 *   state    [B][K - 1][D] of dtype, contiguous: the inputs before the first step
 *            (NULL: 0)
 *   lengths  int32 [B], each sequence's number of steps, clamped to 0..T (NULL: T
 *            for all). Nothing is read beyond a length; y is 0 there.
 *   y        [B][T][D] of dtype
 *   last     [B][K - 1][D] of dtype: the last K - 1 inputs, of state and x
 *            (NULL: not wanted)
 */
cpdp_status cpdp_causal_conv(const void *x, int64_t x_seq, int64_t x_step,
                             const float *weight, int64_t weight_worker, const float *bias, int64_t bias_worker,
                             const void *state, const int32_t *lengths,
                             cpdp_dtype dtype, int W, int B, int64_t T, int D, int K,
                             void *y, void *last, void *stream);

/*
 * cpdp_causal_conv_backward — with dv_t = dy_t * silu'(v_t), dx_t = sum over k of
 * weight[k] * dv_(t+K-1-k), dweight[k] = sum over t of dv_t * x_(t-K+1+k) and
 * dbias = sum over t of dv_t, over a worker's sequences.
 *   dy       [B][T][D] of dtype, with strides; not read beyond a length
 *   dlast    [B][K - 1][D] of dtype: the gradient of last (NULL: 0)
 *   dx       [B][T][D] of dtype; 0 beyond a length
 *   dstate   [B][K - 1][D] of dtype (NULL: not wanted)
 *   dweight, dbias  dweight_dtype, worker w's [D][K] and [D] at + w * their
 *            strides; sums are float32, in an order fixed by the sizes and by
 *            whether every row is one of whole pieces of 4 elements
 */
size_t cpdp_causal_conv_backward_workspace(int W, int B, int64_t T, int D, int K);
cpdp_status cpdp_causal_conv_backward(const void *dy, int64_t dy_seq, int64_t dy_step,
                                      const void *x, int64_t x_seq, int64_t x_step,
                                      const float *weight, int64_t weight_worker, const float *bias, int64_t bias_worker,
                                      const void *state, const void *dlast, const int32_t *lengths,
                                      cpdp_dtype dtype, int W, int B, int64_t T, int D, int K,
                                      void *dx, void *dstate, void *dweight, int64_t dweight_worker,
                                      void *dbias, int64_t dbias_worker, cpdp_dtype dweight_dtype,
                                      void *workspace, size_t workspace_bytes, void *stream);

/*
 * cpdp_causal_conv_step — one token for each of B sequences: x and y [B][D] of
 * dtype (x with a sequence stride); state [B][K - 1][D] is moved on by x.
 */
cpdp_status cpdp_causal_conv_step(const void *x, int64_t x_seq, const float *weight, int64_t weight_worker,
                                  const float *bias, int64_t bias_worker, cpdp_dtype dtype,
                                  int W, int B, int D, int K, void *state, void *y, void *stream);

/* States per channel of the scan: 1 to this many. */
#define CPDP_SCAN_MAX_STATES 32

/*
 * Inputs of the scan of B sequences of T <= 2^30 steps, D channels and N states
 * per channel. Worker w's weights are those of the sequences w * B / W to
 * (w + 1) * B / W - 1 (W divides B).
 *   u, delta, z  [B][T][D] of dtype, each with a sequence and a step stride; z
 *            NULL: no gate, silu(z) is 1
 *   b, c     [B][T][N] of dtype, with strides. Step strides are below 2^28 where
 *            T > 1.
 *   a_log, skip, bias  float32, worker w's [D][N], [D] and [D] at + w * their
 *            strides
 *   lengths  int32 [B], each sequence's number of steps, clamped to 0..T (NULL: T
 *            for all)
 */
typedef struct cpdp_scan_inputs {
    const void *u;
    int64_t u_seq, u_step;
    const void *delta;
    int64_t delta_seq, delta_step;
    const void *z;
    int64_t z_seq, z_step;
    const void *b;
    int64_t b_seq, b_step;
    const void *c;
    int64_t c_seq, c_step;
    const float *a_log;
    int64_t a_log_worker;
    const float *skip;
    int64_t skip_worker;
    const float *bias;
    int64_t bias_worker;
    const int32_t *lengths;
} cpdp_scan_inputs;

/*
 * cpdp_selective_scan — with dt = log(1 + exp(delta + bias)),
 *   h_t[n] = exp(-dt_t exp(a_log[n])) h_(t-1)[n] + dt_t u_t b_t[n]
 *   y_t = (sum over n of c_t[n] h_t[n] + skip u_t) z_t sigmoid(z_t)
 *   h0       float32 [B][D][N], the states before the first step (NULL: 0)
 *   y        [B][T][D] of dtype; nothing is read beyond a length, y is 0 there
 *            and the states stay
 *   last     float32 [B][D][N], the states after the last step
 *   carry    NULL, or float32 [B][ceil(T / CPDP_CARRY_STEPS)][D][N]: the states
 *            before steps 0, CPDP_CARRY_STEPS, ..., for the backward pass
 *            (defined up to each sequence's length)
 * States and sums are float32. A decay x = exp(-p) is off by at most
 * (2 + 2 p) 2^-23 of it; one across a segment of a split sequence, whose dt are
 * summed first, by (2 + 10 p) 2^-23. An exp(a_log) above the float32 range counts as its end:
 * a step of no size (dt of 0) leaves the state, any other forgets it. Where dt, u, z, b or c is infinite, an output may be NaN
 * that the formula has infinite. B * T * D is at most 2^34.
 */
size_t cpdp_selective_scan_workspace(int B, int64_t T, int D, int N);
cpdp_status cpdp_selective_scan(const cpdp_scan_inputs *inputs, cpdp_dtype dtype, int W, int B, int64_t T, int D, int N,
                                const float *h0, void *y, float *last, float *carry,
                                void *workspace, size_t workspace_bytes, void *stream);

/*
 * cpdp_selective_scan_backward — the gradients of all inputs of the scan.
 *   dy       [B][T][D] of dtype, with strides; not read beyond a length
 *   carry    what the forward pass wrote; the states between are made again
 *   dlast    float32 [B][D][N], the gradient of last (NULL: 0)
 *   du, ddelta, dz  [B][T][D] of dtype; 0 beyond a length; dz may be NULL where
 *            there is no z
 *   db, dc   [B][T][N] of dtype; 0 beyond a length
 *   dh0      float32 [B][D][N] (NULL: not wanted)
 *   da_log, dskip, dbias  dweight_dtype, worker w's [D][N], [D] and [D] at + w *
 *            their strides. Sums are float32, in an order fixed by the sizes.
 */
size_t cpdp_selective_scan_backward_workspace(int B, int64_t T, int D, int N);
cpdp_status cpdp_selective_scan_backward(const void *dy, int64_t dy_seq, int64_t dy_step,
                                         const cpdp_scan_inputs *inputs, cpdp_dtype dtype,
                                         int W, int B, int64_t T, int D, int N,
                                         const float *carry, const float *dlast,
                                         void *du, void *ddelta, void *dz, void *db, void *dc, float *dh0,
                                         void *da_log, int64_t da_log_worker, void *dskip, int64_t dskip_worker,
                                         void *dbias, int64_t dbias_worker, cpdp_dtype dweight_dtype,
                                         void *workspace, size_t workspace_bytes, void *stream);

/*
 * cpdp_selective_scan_step — one token for each of B sequences: inputs of one
 * step ([B][D] and [B][N], with the sequence strides; lengths and step strides
 * are not looked at); state (float32 [B][D][N]) is replaced by the next one, and
 * y ([B][D] of dtype) receives the output.
 */
cpdp_status cpdp_selective_scan_step(const cpdp_scan_inputs *inputs, cpdp_dtype dtype, int W, int B, int D, int N,
                                     float *state, void *y, void *stream);

/*
 * cpdp_layer_timeouts — the number of bounded waits that ran out since the last
 * call (0 expected): the warps of the weight gradient and of the loss wait for
 * the slots of a ring, for some seconds at most. A block in which one ran out
 * writes NaN: the weight gradient's for all of its tile of dW, the loss's for the
 * tile at hand and those that it would have come to. Waits for the device.
 */
cpdp_status cpdp_layer_timeouts(int64_t *count);

#ifdef __cplusplus
}
#endif

#endif /* CPDP_LAYERS_H */
