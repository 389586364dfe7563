/*
 * esrnn_state_space.h - C ABI of the operators of a selective state space layer in the MI355X (gfx950) library: what a
 * network needs beside the layer operators of esrnn_layers.h for layers whose channels have several states each, and whose
 * steps, inputs and outputs are chosen position by position.
 *
 *   short causal convolution   depthwise, with activation: whole sequences, its reverse pass, and single positions
 *   selective scan             the recurrence over whole sequences, its reverse pass, and single positions
 *   block norm                 gate, norm behind a block, residual, norm before the next block, and its reverse pass
 *
 * Conventions are those of esrnn_layers.h: every function returns an esrnn_status and nothing throws or aborts; arguments are
 * checked before any kernel is launched; all arrays are DEVICE pointers of the caller unless said otherwise; the library
 * allocates no device memory; all work is enqueued on `stream` and no call waits for the device.  Calls that overlap must not
 * share a workspace.  Equal calls give equal results bit for bit: no sum depends on the order in which workgroups run.
 *
 * Element types: activations and their gradients in fp32, bf16 or fp16, all of one call alike (the residual stream may be fp32 beside
 * 16-bit activations); states, statistics, parameters, their gradients and every sum in fp32.  Results are rounded to the element type
 * once, to nearest.  Alignment: that of one element (workspaces and saved states 256 bytes).
 * Arrays that a call writes must not overlap others; those that begin at one place, or that share elements as far as equal strides of rows or positions show it, and
 * rows that reach into a pool of states, are refused.
 *
 * lengths [B] int32 or NULL (all T): positions that exist; values outside 0 .. T are clamped.  Past its length a sequence is not read into
 * arithmetic, and results are zero there.
 * slots [rows] int32 or NULL (request i has row i): rows of a pool of states, distinct.  A request whose slot lies outside the pool gets
 * zeros and changes nothing (padding of a batch of fixed size: -1).
 */
#ifndef ESRNN_STATE_SPACE_H
#define ESRNN_STATE_SPACE_H

#include "esrnn_layers.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Short causal convolution of every channel with K taps of its own, 2 <= K <= 8, over T positions of B sequences:
 *   u_t = bias + sum_{j < K} weight[j] x_{t-K+1+j},   out = u  or  u sigmoid(u)      (esrnn_norm_activation)
 * The K - 1 inputs before the first position are `initial`, oldest first, or zero.  At most 2^24 - 1 tiles of 64 channels of 128 positions of a sequence.
 */
typedef struct {
    int32_t B, T, C, K;
    int32_t activation;       /* esrnn_norm_activation */
    int32_t dtype;            /* esrnn_dtype of x, out, initial, last and the gradients of x and out */
    int64_t x_stride[2], out_stride[2];                 /* {sequence, position}; channels lie next to each other */
    int64_t grad_out_stride[2], grad_x_stride[2];       /* read by the reverse pass only */
} esrnn_convolution_shape;

/* Bytes of the workspace of a reverse pass.  Host-only; strides are not read. */
esrnn_status esrnn_convolution_workspace_bytes(const esrnn_convolution_shape *shape, size_t *bytes);
/*
 *   weight   [C][K] fp32, bias [C] fp32 or NULL (zero)
 *   initial  [B][K-1][C] or NULL (zero)
 *   last     [B][K-1][C] or NULL: the last K - 1 inputs of every sequence, those of `initial` among them where it is shorter
 */
esrnn_status esrnn_convolution_forward(const esrnn_convolution_shape *shape, const void *x, const int32_t *lengths, const float *weight,
                                       const float *bias, const void *initial, void *out, void *last, void *stream);
/*
 * Reverse pass for the operands of a forward pass.  grad_last [B][K-1][C] fp32 or NULL (zero); grad_weight [C][K] fp32; grad_bias [C] fp32 or
 * NULL; grad_initial [B][K-1][C] fp32 or NULL.  Outputs are overwritten.
 */
esrnn_status esrnn_convolution_backward(const esrnn_convolution_shape *shape, const void *x, const int32_t *lengths, const float *weight,
                                        const float *bias, const void *initial, const void *grad_out, const float *grad_last, void *grad_x,
                                        float *grad_weight, float *grad_bias, float *grad_initial, void *workspace, void *stream);

/* One position for each of `rows` requests: x, out [rows] at their strides; state [pool][K-1][C] in the element type, oldest first, moved on
 * in place.  rows == 0 is no work. */
typedef struct {
    int32_t rows, pool, C, K;
    int32_t activation, dtype;
    int64_t x_stride, out_stride;
} esrnn_convolution_step_shape;
esrnn_status esrnn_convolution_step(const esrnn_convolution_step_shape *shape, const void *x, const float *weight, const float *bias,
                                    const int32_t *slots, void *state, void *out, void *stream);

/*
 * Selective scan: C channels of N states each, 1 <= N <= 64, over T positions of B sequences.  b and c belong to G groups of C / G neighbouring
 * channels.  For a channel of group g, with d = softplus(delta + bias) or delta + bias:
 *   h_t[n] = exp(d_t A[n]) h_{t-1}[n] + d_t x_t b_t[g][n],    out_t = sum_n c_t[g][n] h_t[n] + D x_t
 * A is used as it is (rates of decay are negative; minus infinity keeps nothing of a state from steps of 2^-119 on, and a step of size zero changes nothing.  The
 * gradient of a smaller step of a channel with an infinite rate leaves out what decays: it has no derivative there).
 * Operands that exist are finite; an infinity makes its channel's states, or its group's, infinite or NaN from there on.  At most 2^20 lines, of 64 channels of a
 * sequence and of a group, and 2^15 of them side by side.
 */
typedef enum { ESRNN_DELTA_SOFTPLUS = 0, ESRNN_DELTA_GIVEN = 1 } esrnn_delta_kind;

typedef struct {
    int32_t B, T, C, N, G;
    int32_t delta_kind;       /* esrnn_delta_kind */
    int32_t dtype;            /* esrnn_dtype of x, delta, b, c, out and their gradients */
    int64_t x_stride[2], delta_stride[2], b_stride[2], c_stride[2], out_stride[2];     /* {sequence, position}; b, c: [G][N] contiguous */
    int64_t grad_out_stride[2], grad_x_stride[2], grad_delta_stride[2], grad_b_stride[2], grad_c_stride[2];    /* reverse pass only */
} esrnn_selective_shape;

/* Bytes of the workspace of a forward pass, with `reverse` of a forward or a reverse pass, and of the states that the forward pass leaves for the
 * reverse pass (one fp32 state for every eight positions).  Host-only; strides are not read. */
esrnn_status esrnn_selective_workspace_bytes(const esrnn_selective_shape *shape, int32_t reverse, size_t *bytes);
esrnn_status esrnn_selective_saved_bytes(const esrnn_selective_shape *shape, size_t *bytes);
/*
 *   A        [C][N] fp32, D [C] fp32 or NULL (zero), bias [C] fp32 or NULL (zero)
 *   initial  [B][C][N] fp32 or NULL (zero): h before the first position
 *   last     [B][C][N] fp32 or NULL: h at the last position; that of a sequence of length zero is its initial state
 *   saved    esrnn_selective_saved_bytes, or NULL if no reverse pass follows
 */
esrnn_status esrnn_selective_forward(const esrnn_selective_shape *shape, const void *x, const void *delta, const float *A, const void *b,
                                     const void *c, const float *D, const float *bias, const int32_t *lengths, const float *initial,
                                     void *out, float *last, void *saved, void *workspace, void *stream);
/*
 * Reverse pass for the operands and `saved` of a forward pass of the same shape.  grad_last [B][C][N] fp32 or NULL (zero).  grad_A [C][N] fp32;
 * grad_D, grad_bias [C] fp32 or NULL; grad_initial [B][C][N] fp32 or NULL.  Outputs are overwritten.
 */
typedef struct {
    void *x, *delta, *b, *c;
    float *A, *D, *bias, *initial;
} esrnn_selective_grads;
esrnn_status esrnn_selective_backward(const esrnn_selective_shape *shape, const void *x, const void *delta, const float *A, const void *b,
                                      const void *c, const float *D, const float *bias, const int32_t *lengths, const void *saved,
                                      const void *grad_out, const float *grad_last, const esrnn_selective_grads *grads, void *workspace,
                                      void *stream);

/* One position for each of `rows` requests: x, delta, b, c, out [rows] at their strides; state [pool][C][N] fp32, updated in place.  rows == 0
 * is no work. */
typedef struct {
    int32_t rows, pool, C, N, G;
    int32_t delta_kind, dtype;
    int64_t x_stride, delta_stride, b_stride, c_stride, out_stride;
} esrnn_selective_step_shape;
esrnn_status esrnn_selective_step(const esrnn_selective_step_shape *shape, const void *x, const void *delta, const float *A, const void *b,
                                  const void *c, const float *D, const float *bias, const int32_t *slots, float *state, void *out,
                                  void *stream);

/*
 * Block norm: what stands between one block's result y and the next block's input, for every row of C channels by itself, C <= 8192:
 *   v = y silu(gate) (ESRNN_GATE_BEFORE) or y;    p = v / sqrt(mean(v^2) + eps) post_weight, or v without post_weight
 *   e = p silu(gate) (ESRNN_GATE_AFTER) or p;     sum = residual + scale e  (without residual 0, without scale 1)
 *   out = sum / sqrt(mean(sum^2) + eps) pre_weight
 * Without pre_weight there is no second norm: with a residual `sum` is the result and out is NULL, without one the result is out = scale e.
 * The second norm takes the sum before it is rounded.  Squares are summed in fp32: a row whose mean square is beyond it has a root of infinity and gives zeros.
 */
typedef enum { ESRNN_GATE_NONE = 0, ESRNN_GATE_BEFORE = 1, ESRNN_GATE_AFTER = 2 } esrnn_gate_position;

typedef struct {
    int32_t rows, C;
    int32_t gate;             /* esrnn_gate_position */
    int32_t dtype;            /* esrnn_dtype of y, gate, out and their gradients */
    int32_t stream_dtype;     /* of residual, sum and their gradients: dtype or ESRNN_F32 */
    float eps;                /* > 0 */
    int64_t y_stride, gate_stride, residual_stride, sum_stride, out_stride;                                /* of a row */
    int64_t grad_out_stride, grad_sum_stride, grad_y_stride, grad_gate_stride, grad_residual_stride;       /* reverse pass only */
} esrnn_block_norm_shape;

/* What both passes read.  Pointers that are NULL leave their part out; gate goes with the shape's `gate`. */
typedef struct {
    const void *y, *gate, *residual;
    const int32_t *exists;    /* [rows] or NULL: rows with 0 are not read into arithmetic, give zeros and add nothing to any gradient */
    const float *post_weight, *scale, *pre_weight;      /* [C] */
} esrnn_block_norm_operands;

/* Bytes of the workspace of a reverse pass.  Host-only; strides are not read. */
esrnn_status esrnn_block_norm_workspace_bytes(const esrnn_block_norm_shape *shape, size_t *bytes);
/* stats [rows][2] fp32, left for the reverse pass, or NULL if none follows; then `sum` may be `residual` itself, at its strides. */
esrnn_status esrnn_block_norm_forward(const esrnn_block_norm_shape *shape, const esrnn_block_norm_operands *in, void *sum, void *out,
                                      float *stats, void *stream);
/* grad_out as out, grad_sum as sum or NULL (zero).  The gradients of absent operands are NULL; those of the weights [C] fp32, sums over rows.
 * Outputs are overwritten. */
typedef struct {
    void *y, *gate, *residual;
    float *post_weight, *scale, *pre_weight;
} esrnn_block_norm_grads;
esrnn_status esrnn_block_norm_backward(const esrnn_block_norm_shape *shape, const esrnn_block_norm_operands *in, const float *stats,
                                       const void *grad_out, const void *grad_sum, const esrnn_block_norm_grads *grads, void *workspace,
                                       void *stream);

#ifdef __cplusplus
}
#endif
#endif
