/*
 * esrnn_layers.h - C ABI of the layer operators of the MI355X (gfx950) library:
 * what a network of linear recurrent layers needs beside the ES-RNN step of
 * esrnn.h to be trained on long sequences and to be served position by position.
 *
 *   gated linear recurrence   a scan over long sequences, its reverse pass, and its form for single positions
 *   group norm + activation   channels last, with its reverse pass
 *   AdamW                     one update of many tensors, moments in 32 or in 8 bits
 *
 * Conventions are those of esrnn.h: every function returns an esrnn_status and nothing throws or aborts; arguments are
 * checked before any kernel is launched; all arrays are DEVICE pointers of the caller unless said otherwise; the library
 * allocates no device memory; all work is enqueued on `stream` and no call waits for the device.  Calls that overlap must not
 * share a workspace.  Equal calls give equal results bit for bit: no sum depends on the order in which workgroups run.
 *
 * Element types: activations and their gradients in fp32, bf16 or fp16, all of one call alike; states, statistics, parameters
 * of the norm and every sum in fp32.  Results are rounded to the element type once, to nearest.
 * Alignment: arrays of elements need that of one element only (fp32 arrays four bytes, workspaces 256); base, strides and C that are multiples of
 * four elements are faster.
 */
#ifndef ESRNN_LAYERS_H
#define ESRNN_LAYERS_H

#include "esrnn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { ESRNN_F32 = 0, ESRNN_BF16 = 1, ESRNN_F16 = 2 } esrnn_dtype;

/*
 * Gated linear recurrence over T positions, for B sequences and C channels, each channel on its own:
 *   ESRNN_RECURRENCE_SMOOTH   h_t = (1 - z_t) h_{t-1} + z_t x_t,  z = sigmoid(gate)
 *       (exponential smoothing, Section 3.1 Eq. (1), with a coefficient of its own at every position)
 *   ESRNN_RECURRENCE_DECAY    h_t = a_t h_{t-1} + x_t,            a = sigmoid(gate)
 * Strides are in elements, of a sequence and of a position; channels are contiguous.  Any order of B and T, gaps, and
 * x and gate as parts of one array are fine; a written array must not overlap itself or another (last initial, say, or grad_x x): refused where
 * arrays begin at one place or have the same strides.
 */
typedef enum { ESRNN_RECURRENCE_SMOOTH = 0, ESRNN_RECURRENCE_DECAY = 1 } esrnn_recurrence_kind;

typedef struct {
    int32_t B, T, C;
    int32_t kind;             /* esrnn_recurrence_kind */
    int32_t dtype;            /* esrnn_dtype of x, gate, out and their gradients */
    int64_t x_stride[2], gate_stride[2], out_stride[2];                /* {sequence, position} */
    int64_t grad_out_stride[2], grad_x_stride[2], grad_gate_stride[2]; /* read by the reverse pass only */
} esrnn_recurrence_shape;

/* Bytes of the workspace of one call, and of the states that the forward pass leaves for the reverse pass (one fp32 state
 * per block of positions).  Host-only; strides are not read. */
esrnn_status esrnn_recurrence_workspace_bytes(const esrnn_recurrence_shape *shape, size_t *bytes);
esrnn_status esrnn_recurrence_saved_bytes(const esrnn_recurrence_shape *shape, size_t *bytes);

/*
 *   lengths  [B] int32 or NULL (all T): positions that exist; values outside 0 .. T are clamped.  Past its length a sequence
 *            is not read into arithmetic, and out is zero there.
 *   initial  [B][C] fp32 or NULL (zero): h before the first position.
 *   last     [B][C] fp32 or NULL: h at the last position; that of a sequence of length zero is its initial state.
 *   saved    esrnn_recurrence_saved_bytes, or NULL if no reverse pass follows.
 */
esrnn_status esrnn_recurrence_forward(const esrnn_recurrence_shape *shape, const void *x, const void *gate, const int32_t *lengths,
                                      const float *initial, void *out, float *last, void *saved, void *workspace, void *stream);
/*
 * Reverse pass for x, gate, lengths and saved of a forward pass of the same shape.  grad_last [B][C] fp32 or NULL (zero).
 * grad_x and grad_gate are zero past the lengths; grad_initial [B][C] fp32 or NULL.  Outputs are overwritten.
 */
esrnn_status esrnn_recurrence_backward(const esrnn_recurrence_shape *shape, const void *x, const void *gate, const int32_t *lengths,
                                       const void *saved, const void *grad_out, const float *grad_last, void *grad_x,
                                       void *grad_gate, float *grad_initial, void *workspace, void *stream);

/*
 * One position for each of `rows` requests, whose states are rows of a pool: state [pool][C] fp32, updated in place.
 *   slots  [rows] int32 or NULL (request i has row i): rows of the pool, distinct.  A request whose slot lies outside the pool gets
 *          zeros and changes nothing (padding of a batch of fixed size: -1).
 * x, gate, out [rows] at their strides, in elements.  rows == 0 is no work.
 */
esrnn_status esrnn_recurrence_step(int32_t kind, int32_t dtype, int32_t rows, int32_t pool, int32_t C, const void *x, int64_t x_stride,
                                   const void *gate, int64_t gate_stride, const int32_t *slots, float *state, void *out,
                                   int64_t out_stride, void *stream);

/*
 * Group norm with activation, channels last: x, out [N][T][C] contiguous, G groups of C / G neighbouring channels.  Over the
 * positions of a sample and the channels of a group:
 *   xhat = (x - mean) / sqrt(var + eps),  u = xhat scale[c] + shift[c],  out = u  or  u sigmoid(u)
 * T = 1 normalises every position by itself.  lengths [N] int32 or NULL as above: positions past the length take no part, and out and
 * grad_x are zero there; a sample of length zero adds nothing to any gradient.
 * stats [N][G][2] fp32: mean and 1 / sqrt(var + eps), left by the forward pass for the reverse pass; NULL if none follows.
 */
typedef enum { ESRNN_NORM_NONE = 0, ESRNN_NORM_SILU = 1 } esrnn_norm_activation;

typedef struct {
    int32_t N, T, C, G;
    int32_t activation;       /* esrnn_norm_activation */
    int32_t dtype;            /* esrnn_dtype of x, out and their gradients */
    float eps;                /* > 0 */
} esrnn_group_norm_shape;

esrnn_status esrnn_group_norm_workspace_bytes(const esrnn_group_norm_shape *shape, size_t *bytes);
esrnn_status esrnn_group_norm_forward(const esrnn_group_norm_shape *shape, const void *x, const int32_t *lengths, const float *scale,
                                      const float *shift, void *out, float *stats, void *workspace, void *stream);
/* grad_x [N][T][C]; grad_scale, grad_shift [C] fp32, sums over all samples; all overwritten. */
esrnn_status esrnn_group_norm_backward(const esrnn_group_norm_shape *shape, const void *x, const int32_t *lengths, const float *scale,
                                       const float *shift, const float *stats, const void *grad_out, void *grad_x,
                                       float *grad_scale, float *grad_shift, void *workspace, void *stream);

/*
 * AdamW (Adam of esrnn_adam_update with the decay taken from the parameter itself: Loshchilov & Hutter 2019, Algorithm 2)
 * over a list of tensors at once:
 *   g <- g min(1, clip_norm / (||g|| + 1e-6)),  ||g|| over all tensors of the list
 *   m <- beta1 m + (1 - beta1) g,  v <- beta2 v + (1 - beta2) g^2
 *   p <- p (1 - lr weight_decay) - lr (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps)
 * With clip_norm > 0, a gradient whose norm is not finite changes nothing at all; the norm is left where `norm` says.
 * Without, such a gradient makes its own elements NaN (in 8 bits: the moments of its block of 256, and that a gradient beyond 1e19 does too, whose
 * square is infinite in fp32).  An eps of zero gives 0 / 0 where a gradient has always been zero.
 *
 * Moments live in flat arrays over all tensors; a tensor's elements begin at a multiple of ESRNN_ADAMW_BLOCK, in list order.
 *   32 bits: m, v fp32.   8 bits: m and r = sqrt(v) in OCP e4m3 (one byte), in units of one fp32 scale for each
 *   block of ESRNN_ADAMW_BLOCK elements (its largest magnitude / 448).  They are rounded up or down at random with the mean kept: to
 *   nearest, a moving average would stand still as soon as its step is less than half a code.  The 16 + 16 random bits are a hash of
 *   seed, step and the element's place, so a repeated call repeats its result.  A root that is not zero keeps at least
 *   the smallest code (a block whose largest is below 2^-91 is zero).  The step itself uses the moments before they are rounded.
 *
 * `step` is an argument of the call: an update captured into a graph has the step number of its capture in every replay (and all of `opt`), in
 * both bias corrections and, with 8-bit moments, in the random bits, so that every element is rounded with the same bits each time and the mean is not kept.
 * Updates belong outside a graph that is replayed from step to step (or, with 32 bits, into one captured so late that the corrections are 1).
 */
#define ESRNN_ADAMW_BLOCK 256

typedef struct {
    float *param;             /* fp32 */
    const void *grad;         /* grad_dtype */
    void *copy;               /* the updated parameter in copy_dtype, or NULL */
    int64_t n;                /* elements, >= 1 */
    float weight_decay;       /* of this tensor, >= 0 */
    int32_t grad_dtype, copy_dtype;   /* esrnn_dtype; the copy bf16 or fp16 */
} esrnn_adamw_tensor;

typedef struct {
    double lr, beta1, beta2, eps;     /* double: 1 - beta2 and the bias corrections lose digits that a float beta2 has dropped */
    double clip_norm;         /* <= 0: no clipping, and no norm */
    uint32_t seed;            /* of the rounding of 8-bit moments */
} esrnn_adamw_config;

typedef struct esrnn_adamw esrnn_adamw;

/* `tensors`: HOST array of `count` tensors, copied; its pointers are not dereferenced on the host, and no two written arrays may overlap.  state_bits:
 * 32 or 8.  Gradients are read at these addresses at every step; gradients at others need a new handle, bound again. */
esrnn_status esrnn_adamw_create(const esrnn_adamw_tensor *tensors, int32_t count, int32_t state_bits, esrnn_adamw **out);
esrnn_status esrnn_adamw_destroy(esrnn_adamw *h);
/* Elements of each flat moment array: a multiple of ESRNN_ADAMW_BLOCK. */
esrnn_status esrnn_adamw_state_elements(const esrnn_adamw *h, size_t *n);
esrnn_status esrnn_adamw_workspace_bytes(const esrnn_adamw *h, size_t *bytes);
/* Writes the list of tensors into the workspace.  Once, ordered before the first update, which returns ESRNN_ERR_ORDER without it or with
 * another workspace than the last one bound; nothing else may write to the workspace from then on. */
esrnn_status esrnn_adamw_bind(esrnn_adamw *h, void *workspace, void *stream);
/* step counts from 1.  Moments are zero before the first step: 32 bits m, v; 8 bits m, r, m_scale, r_scale (v NULL), else
 * r and the scales NULL.  norm: one float or NULL; written if clip_norm > 0. */
esrnn_status esrnn_adamw_update(const esrnn_adamw *h, const esrnn_adamw_config *opt, int32_t step, void *m, float *v, void *r,
                                float *m_scale, float *r_scale, float *norm, void *workspace, void *stream);

#ifdef __cplusplus
}
#endif
#endif
