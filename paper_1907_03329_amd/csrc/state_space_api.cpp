// C ABI of the operators of a selective state space layer (include/esrnn_state_space.h): argument checks and the launches of each call.
#include "layers_checks.h"
#include "state_space_internal.h"

using namespace esrnn;

namespace {

constexpr int64_t kMostWorkgroups = (int64_t(1) << 24) - 1;     // of 256 threads: a launch has less than 2^32

bool sequences(int64_t B, int64_t T, int64_t C) { return B >= 1 && T >= 1 && C >= 1 && T <= (1 << 30) && C <= (1 << 24) && B <= (1 << 30); }
bool activation(int kind) { return kind == ESRNN_NORM_NONE || kind == ESRNN_NORM_SILU; }
bool delta(int kind) { return kind == ESRNN_DELTA_SOFTPLUS || kind == ESRNN_DELTA_GIVEN; }

bool convolution_sizes(const esrnn_convolution_shape &s)
{
    // workgroups: tiles of 64 channels, at least 128 positions
    return sequences(s.B, s.T, s.C) && s.K >= 2 && s.K <= 8 && activation(s.activation) && element_type(s.dtype) &&
           (int64_t)s.B * ((s.T + 127) / 128) <= kMostWorkgroups / ((s.C + 63) / 64);
}

bool selective_sizes(const esrnn_selective_shape &s)
{
    if (!sequences(s.B, s.T, s.C) || s.N < 1 || s.N > 64 || s.G < 1 || s.C % s.G != 0 || !delta(s.delta_kind) || !element_type(s.dtype)) return false;
    // lines of 64 channels, and their columns of partial sums (up to 72 x 64): workgroups of up to 1024 threads, less than 2^32 in a launch
    const int64_t tiles = (int64_t)s.G * ((s.C / s.G + 63) / 64), positions = (int64_t)s.B * (s.T + 7);
    return tiles <= (1 << 15) && (int64_t)s.B * tiles <= (1 << 20) && positions <= (int64_t(1) << 36) / (s.G * int64_t(64)) &&
           (int64_t)s.B * tiles * 64 <= kMostElements / s.T;
}

// Of the last states and gradients [B][C][N] and the like.
size_t states_of(const esrnn_selective_shape &s) { return (size_t)s.B * s.C * s.N; }

bool block_norm_sizes(const esrnn_block_norm_shape &s)
{
    return s.rows >= 1 && s.rows <= (1 << 30) && s.C >= 1 && s.C <= kBlockNormMostChannels && s.gate >= ESRNN_GATE_NONE && s.gate <= ESRNN_GATE_AFTER &&
           element_type(s.dtype) && (s.stream_dtype == s.dtype || s.stream_dtype == ESRNN_F32) && s.eps > 0.0f && s.eps < __builtin_inff();
}
// An array of rows, or one that is left out.
struct Rows {
    const void *p;
    int64_t stride;
    int dtype;
    bool written;
};
esrnn_status check_rows(const esrnn_block_norm_shape &s, const Rows *rows, int n, bool in_place)
{
    for (int i = 0; i < n; ++i) {
        if (!rows[i].p) continue;
        if (rows[i].stride < 0 || rows[i].stride > kMostElements / s.rows || (rows[i].written && s.rows > 1 && rows[i].stride < s.C) ||
            !element_aligned(rows[i].p, rows[i].dtype))
            return ESRNN_ERR_CONFIG;
    }
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < n; ++j) {
            const Rows &w = rows[i], &o = rows[j];
            if (i == j || !w.written || !w.p || !o.p) continue;
            if (in_place && w.p == o.p && w.stride == o.stride && w.dtype == o.dtype && !o.written) continue;
            const RowsShape shape{1, s.rows, s.C, w.dtype};
            const int64_t ws[2] = {0, w.stride}, os[2] = {0, o.stride};
            if (w.p == o.p || (w.dtype == o.dtype && rows_overlap(shape, w.p, ws, o.p, os))) return ESRNN_ERR_CONFIG;
        }
    return ESRNN_OK;
}

// What single positions read or write of each request: `width` elements next to each other.
struct StepRows {
    const void *p;
    int64_t stride, width;
};
// Whether one of them shares elements with a pool of states, which has no gaps.
bool reach_into(const StepRows &r, int64_t rows, int64_t element, const void *pool, int64_t bytes)
{
    const int64_t first = reinterpret_cast<intptr_t>(r.p) - reinterpret_cast<intptr_t>(pool), step = r.stride * element, end = first + r.width * element;
    if (bytes == 0 || (end <= 0 && step == 0)) return false;
    const int64_t i = end > 0 ? 0 : -end / step + 1;        // the first that ends behind the pool's beginning
    return i < rows && first + i * step < bytes;
}
bool step_overlaps(int64_t rows, int dtype, const StepRows &out, std::initializer_list<StepRows> read, const void *pool, int64_t bytes)
{
    const int64_t element = (int64_t)element_bytes(dtype), written[2] = {0, out.stride};
    if (reach_into(out, rows, element, pool, bytes)) return true;
    for (const StepRows &r : read) {
        const int64_t stride[2] = {0, r.stride};
        if (rows_overlap(RowsShape{1, rows, out.width, dtype}, out.p, written, r.p, stride, r.width) || reach_into(r, rows, element, pool, bytes)) return true;
    }
    return false;
}

}  // namespace

extern "C" {

esrnn_status esrnn_convolution_workspace_bytes(const esrnn_convolution_shape *shape, size_t *bytes)
{
    if (!shape || !bytes) return ESRNN_ERR_NULL;
    if (!convolution_sizes(*shape)) return ESRNN_ERR_CONFIG;
    *bytes = (convolution_workspace_floats(*shape) * sizeof(float) + 255) / 256 * 256;
    return ESRNN_OK;
}

esrnn_status esrnn_convolution_forward(const esrnn_convolution_shape *shape, const void *x, const int32_t *lengths, const float *weight,
                                       const float *bias, const void *initial, void *out, void *last, void *stream)
{
    if (!shape || !x || !weight || !out) return ESRNN_ERR_NULL;
    const esrnn_convolution_shape &s = *shape;
    if (!convolution_sizes(s) || !readable_strides(s, s.x_stride) || !writable_strides(s, s.out_stride)) return ESRNN_ERR_CONFIG;
    if (!element_aligned(x, s.dtype) || !element_aligned(out, s.dtype) || !element_aligned(initial, s.dtype) || !element_aligned(last, s.dtype) ||
        !floats_aligned(lengths) || !floats_aligned(weight) || !floats_aligned(bias))
        return ESRNN_ERR_CONFIG;
    // (windows of all sequences are one row)
    const RowsShape windows{1, 1, (int64_t)s.B * (s.K - 1) * s.C, s.dtype};
    const int64_t none[2] = {0, 0};
    if (rows_overlap(s, out, s.out_stride, x, s.x_stride) || (last && initial && rows_overlap(windows, last, none, initial, none)) ||
        one_place({out, last}, {x, lengths, weight, bias, initial}))
        return ESRNN_ERR_CONFIG;
    ConvolutionArgs a{};
    a.x = x, a.lengths = lengths, a.weight = weight, a.bias = bias, a.initial = initial, a.out = out, a.last = last;
    ESRNN_TRY(launch_convolution_forward(s, a, static_cast<hipStream_t>(stream)));
    return ESRNN_OK;
}

esrnn_status esrnn_convolution_backward(const esrnn_convolution_shape *shape, const void *x, const int32_t *lengths, const float *weight,
                                        const float *bias, const void *initial, const void *grad_out, const float *grad_last, void *grad_x,
                                        float *grad_weight, float *grad_bias, float *grad_initial, void *workspace, void *stream)
{
    if (!shape || !x || !weight || !grad_out || !grad_x || !grad_weight || !workspace) return ESRNN_ERR_NULL;
    const esrnn_convolution_shape &s = *shape;
    if (!convolution_sizes(s) || !readable_strides(s, s.x_stride) || !readable_strides(s, s.grad_out_stride) || !writable_strides(s, s.grad_x_stride))
        return ESRNN_ERR_CONFIG;
    if (!element_aligned(x, s.dtype) || !element_aligned(grad_out, s.dtype) || !element_aligned(grad_x, s.dtype) || !element_aligned(initial, s.dtype) ||
        !floats_aligned(lengths) || !floats_aligned(weight) || !floats_aligned(bias) || !floats_aligned(grad_last) || !floats_aligned(grad_weight) ||
        !floats_aligned(grad_bias) || !floats_aligned(grad_initial))
        return ESRNN_ERR_CONFIG;
    if (!aligned_to(workspace, 256)) return ESRNN_ERR_WORKSPACE;
    const size_t windows = (size_t)s.B * (s.K - 1) * s.C, taps = (size_t)s.C * s.K;
    if (rows_overlap(s, grad_x, s.grad_x_stride, x, s.x_stride) || rows_overlap(s, grad_x, s.grad_x_stride, grad_out, s.grad_out_stride) ||
        one_place({grad_x, grad_weight, grad_bias, grad_initial, workspace}, {x, lengths, weight, bias, initial, grad_out, grad_last}) ||
        floats_overlap(grad_initial, windows, grad_last, windows) || floats_overlap(grad_weight, taps, weight, taps) ||
        floats_overlap(grad_bias, s.C, bias, s.C) || floats_overlap(grad_weight, taps, grad_bias, s.C) || floats_overlap(grad_weight, taps, bias, s.C) ||
        floats_overlap(grad_bias, s.C, weight, taps))
        return ESRNN_ERR_CONFIG;
    ConvolutionArgs a{};
    a.x = x, a.lengths = lengths, a.weight = weight, a.bias = bias, a.initial = initial, a.grad_out = grad_out, a.grad_last = grad_last;
    a.grad_x = grad_x, a.grad_weight = grad_weight, a.grad_bias = grad_bias, a.grad_initial = grad_initial, a.parts = static_cast<float *>(workspace);
    ESRNN_TRY(launch_convolution_backward(s, a, static_cast<hipStream_t>(stream)));
    return ESRNN_OK;
}

esrnn_status esrnn_convolution_step(const esrnn_convolution_step_shape *shape, const void *x, const float *weight, const float *bias,
                                    const int32_t *slots, void *state, void *out, void *stream)
{
    if (!shape) return ESRNN_ERR_NULL;
    const esrnn_convolution_step_shape &s = *shape;
    if (s.K < 2 || s.K > 8 || !activation(s.activation) || !element_type(s.dtype) || s.rows < 0 || s.pool < 0 || s.C < 1 || s.C > (1 << 24) ||
        (int64_t)s.rows * ((s.C + 1023) / 1024) > (1 << 23) || (!slots && s.rows > s.pool))
        return ESRNN_ERR_CONFIG;
    if (s.rows == 0) return ESRNN_OK;
    if (!x || !weight || !state || !out) return ESRNN_ERR_NULL;
    if (s.x_stride < 0 || s.out_stride < 0 || s.x_stride > kMostElements / s.rows || s.out_stride > kMostElements / s.rows ||
        (s.rows > 1 && s.out_stride < s.C) || !element_aligned(x, s.dtype) || !element_aligned(out, s.dtype) || !element_aligned(state, s.dtype) ||
        !floats_aligned(weight) || !floats_aligned(bias) || !floats_aligned(slots) || one_place({state, out}, {x, weight, bias, slots}) ||
        step_overlaps(s.rows, s.dtype, {out, s.out_stride, s.C}, {{x, s.x_stride, s.C}}, state, (int64_t)s.pool * (s.K - 1) * s.C * (int64_t)element_bytes(s.dtype)))
        return ESRNN_ERR_CONFIG;
    ESRNN_TRY(launch_convolution_step(s, x, weight, bias, slots, state, out, static_cast<hipStream_t>(stream)));
    return ESRNN_OK;
}

esrnn_status esrnn_selective_workspace_bytes(const esrnn_selective_shape *shape, int32_t reverse, size_t *bytes)
{
    if (!shape || !bytes) return ESRNN_ERR_NULL;
    if (!selective_sizes(*shape)) return ESRNN_ERR_CONFIG;
    *bytes = (selective_workspace_floats(*shape, reverse != 0) * sizeof(float) + 255) / 256 * 256;
    return ESRNN_OK;
}

esrnn_status esrnn_selective_saved_bytes(const esrnn_selective_shape *shape, size_t *bytes)
{
    if (!shape || !bytes) return ESRNN_ERR_NULL;
    if (!selective_sizes(*shape)) return ESRNN_ERR_CONFIG;
    *bytes = selective_saved_floats(*shape) * sizeof(float);
    return ESRNN_OK;
}

esrnn_status esrnn_selective_forward(const esrnn_selective_shape *shape, const void *x, const void *delta, const float *A, const void *b,
                                     const void *c, const float *D, const float *bias, const int32_t *lengths, const float *initial,
                                     void *out, float *last, void *saved, void *workspace, void *stream)
{
    if (!shape || !x || !delta || !A || !b || !c || !out || !workspace) return ESRNN_ERR_NULL;
    const esrnn_selective_shape &s = *shape;
    if (!selective_sizes(s)) return ESRNN_ERR_CONFIG;
    const RowsShape shared{s.B, s.T, (int64_t)s.G * s.N, s.dtype};
    if (!readable_strides(s, s.x_stride) || !readable_strides(s, s.delta_stride) || !readable_strides(shared, s.b_stride) ||
        !readable_strides(shared, s.c_stride) || !writable_strides(s, s.out_stride))
        return ESRNN_ERR_CONFIG;
    for (const void *p : {x, delta, b, c, static_cast<const void *>(out)})
        if (!element_aligned(p, s.dtype)) return ESRNN_ERR_CONFIG;
    if (!floats_aligned(A) || !floats_aligned(D) || !floats_aligned(bias) || !floats_aligned(lengths) || !floats_aligned(initial) || !floats_aligned(last))
        return ESRNN_ERR_CONFIG;
    if (!aligned_to(workspace, 256) || !aligned_to(saved, 256)) return ESRNN_ERR_WORKSPACE;
    if (one_place({out, last, saved, workspace}, {x, delta, A, b, c, D, bias, lengths, initial}) || rows_overlap(s, out, s.out_stride, x, s.x_stride) ||
        rows_overlap(s, out, s.out_stride, delta, s.delta_stride) ||
        rows_overlap(s, out, s.out_stride, b, s.b_stride, shared.C) || rows_overlap(s, out, s.out_stride, c, s.c_stride, shared.C) ||
        floats_overlap(last, states_of(s), initial, states_of(s)) || floats_overlap(last, states_of(s), A, (size_t)s.C * s.N))
        return ESRNN_ERR_CONFIG;
    SelectiveArgs a{};
    a.x = x, a.delta = delta, a.b = b, a.c = c, a.A = A, a.D = D, a.bias = bias, a.initial = initial, a.lengths = lengths, a.out = out, a.last = last;
    a.saved = static_cast<float *>(saved), a.workspace = static_cast<float *>(workspace);
    ESRNN_TRY(launch_selective_forward(s, a, static_cast<hipStream_t>(stream)));
    return ESRNN_OK;
}

esrnn_status esrnn_selective_backward(const esrnn_selective_shape *shape, const void *x, const void *delta, const float *A, const void *b,
                                      const void *c, const float *D, const float *bias, const int32_t *lengths, const void *saved,
                                      const void *grad_out, const float *grad_last, const esrnn_selective_grads *grads, void *workspace,
                                      void *stream)
{
    if (!shape || !x || !delta || !A || !b || !c || !saved || !grad_out || !grads || !workspace) return ESRNN_ERR_NULL;
    const esrnn_selective_shape &s = *shape;
    const esrnn_selective_grads &g = *grads;
    if (!g.x || !g.delta || !g.b || !g.c || !g.A) return ESRNN_ERR_NULL;
    if (!selective_sizes(s)) return ESRNN_ERR_CONFIG;
    const RowsShape wide{s.B, s.T, s.C, s.dtype}, shared{s.B, s.T, (int64_t)s.G * s.N, s.dtype};
    const struct {
        const void *p;
        const int64_t *stride;
        const RowsShape &rows;
        bool written;
    } arrays[] = {{x, s.x_stride, wide, false}, {delta, s.delta_stride, wide, false}, {b, s.b_stride, shared, false}, {c, s.c_stride, shared, false},
                  {grad_out, s.grad_out_stride, wide, false}, {g.x, s.grad_x_stride, wide, true}, {g.delta, s.grad_delta_stride, wide, true},
                  {g.b, s.grad_b_stride, shared, true}, {g.c, s.grad_c_stride, shared, true}};
    for (const auto &w : arrays)
        if (!(w.written ? writable_strides(w.rows, w.stride) : readable_strides(w.rows, w.stride)) || !element_aligned(w.p, s.dtype)) return ESRNN_ERR_CONFIG;
    if (!floats_aligned(A) || !floats_aligned(D) || !floats_aligned(bias) || !floats_aligned(lengths) || !floats_aligned(grad_last) || !floats_aligned(g.A) ||
        !floats_aligned(g.D) || !floats_aligned(g.bias) || !floats_aligned(g.initial))
        return ESRNN_ERR_CONFIG;
    if (!aligned_to(workspace, 256) || !aligned_to(saved, 256)) return ESRNN_ERR_WORKSPACE;
    for (const auto &w : arrays)
        for (const auto &o : arrays)
            if (w.written && &w != &o && rows_overlap(w.rows, w.p, w.stride, o.p, o.stride, o.rows.C)) return ESRNN_ERR_CONFIG;
    if (one_place({g.x, g.delta, g.b, g.c, g.A, g.D, g.bias, g.initial, workspace}, {x, delta, A, b, c, D, bias, lengths, saved, grad_out, grad_last}))
        return ESRNN_ERR_CONFIG;
    const size_t n = states_of(s), rates = (size_t)s.C * s.N, channels = s.C;
    if (floats_overlap(g.initial, n, grad_last, n) || floats_overlap(g.A, rates, A, rates) || floats_overlap(g.D, channels, D, channels) ||
        floats_overlap(g.bias, channels, bias, channels) || floats_overlap(g.D, channels, g.bias, channels) || floats_overlap(g.A, rates, g.D, channels) ||
        floats_overlap(g.A, rates, g.bias, channels) || floats_overlap(g.initial, n, g.A, rates))
        return ESRNN_ERR_CONFIG;
    SelectiveArgs a{};
    a.x = x, a.delta = delta, a.b = b, a.c = c, a.A = A, a.D = D, a.bias = bias, a.lengths = lengths, a.grad_out = grad_out, a.grad_last = grad_last;
    a.saved = static_cast<float *>(const_cast<void *>(saved));
    a.grad_x = g.x, a.grad_delta = g.delta, a.grad_b = g.b, a.grad_c = g.c, a.grad_A = g.A, a.grad_D = g.D, a.grad_bias = g.bias, a.grad_initial = g.initial;
    a.workspace = static_cast<float *>(workspace);
    ESRNN_TRY(launch_selective_backward(s, a, static_cast<hipStream_t>(stream)));
    return ESRNN_OK;
}

esrnn_status esrnn_selective_step(const esrnn_selective_step_shape *shape, const void *x, const void *delta_, const float *A, const void *b,
                                  const void *c, const float *D, const float *bias, const int32_t *slots, float *state, void *out,
                                  void *stream)
{
    if (!shape) return ESRNN_ERR_NULL;
    const esrnn_selective_step_shape &s = *shape;
    if (s.rows < 0 || s.pool < 0 || s.C < 1 || s.C > (1 << 20) || s.N < 1 || s.N > 64 || s.G < 1 || s.C % s.G != 0 || !delta(s.delta_kind) ||
        !element_type(s.dtype) || s.rows > (1 << 30) || (!slots && s.rows > s.pool))
        return ESRNN_ERR_CONFIG;
    if (s.rows == 0) return ESRNN_OK;
    if (!x || !delta_ || !A || !b || !c || !state || !out) return ESRNN_ERR_NULL;
    for (const int64_t stride : {s.x_stride, s.delta_stride, s.b_stride, s.c_stride, s.out_stride})
        if (stride < 0 || stride > kMostElements / s.rows) return ESRNN_ERR_CONFIG;
    for (const void *p : {x, delta_, b, c, static_cast<const void *>(out)})
        if (!element_aligned(p, s.dtype)) return ESRNN_ERR_CONFIG;
    if (one_place({state, out}, {x, delta_, A, b, c, D, bias, slots})) return ESRNN_ERR_CONFIG;
    if ((s.rows > 1 && s.out_stride < s.C) || !floats_aligned(A) || !floats_aligned(D) || !floats_aligned(bias) || !floats_aligned(slots) || !floats_aligned(state))
        return ESRNN_ERR_CONFIG;
    const int64_t shared = (int64_t)s.G * s.N;
    if (step_overlaps(s.rows, s.dtype, {out, s.out_stride, s.C}, {{x, s.x_stride, s.C}, {delta_, s.delta_stride, s.C}, {b, s.b_stride, shared}, {c, s.c_stride, shared}},
                      state, (int64_t)s.pool * s.C * s.N * (int64_t)sizeof(float)))
        return ESRNN_ERR_CONFIG;
    const SelectiveStep a{x, delta_, b, c, A, D, bias, slots, state, out};
    ESRNN_TRY(launch_selective_step(s, a, static_cast<hipStream_t>(stream)));
    return ESRNN_OK;
}

esrnn_status esrnn_block_norm_workspace_bytes(const esrnn_block_norm_shape *shape, size_t *bytes)
{
    if (!shape || !bytes) return ESRNN_ERR_NULL;
    if (!block_norm_sizes(*shape)) return ESRNN_ERR_CONFIG;
    *bytes = (block_norm_workspace_floats(*shape) * sizeof(float) + 255) / 256 * 256;
    return ESRNN_OK;
}

esrnn_status esrnn_block_norm_forward(const esrnn_block_norm_shape *shape, const esrnn_block_norm_operands *in, void *sum, void *out,
                                      float *stats, void *stream)
{
    if (!shape || !in || !in->y) return ESRNN_ERR_NULL;
    const esrnn_block_norm_shape &s = *shape;
    if (!block_norm_sizes(s)) return ESRNN_ERR_CONFIG;
    // what there has to be, and what must not
    const bool needs_out = in->pre_weight || !in->residual;
    if ((s.gate != ESRNN_GATE_NONE && !in->gate) || (in->residual && !sum) || (needs_out && !out)) return ESRNN_ERR_NULL;
    if ((s.gate == ESRNN_GATE_NONE && in->gate) || (!in->residual && sum) || (!needs_out && out)) return ESRNN_ERR_CONFIG;
    const Rows rows[] = {{in->y, s.y_stride, s.dtype, false}, {in->gate, s.gate_stride, s.dtype, false}, {in->residual, s.residual_stride, s.stream_dtype, false},
                         {out, s.out_stride, s.dtype, true}, {sum, s.sum_stride, s.stream_dtype, true}};
    // (the sum in place of the residual, when no reverse pass will ask for it)
    if (sum && sum == in->residual && (stats || s.sum_stride != s.residual_stride)) return ESRNN_ERR_CONFIG;
    if (const esrnn_status e = check_rows(s, rows, 4, false); e != ESRNN_OK) return e;
    const Rows with_sum[] = {rows[0], rows[1], rows[3], rows[4], rows[2]};
    if (const esrnn_status e = check_rows(s, with_sum, 4, false); e != ESRNN_OK) return e;
    const Rows residual_and_sum[] = {rows[2], rows[4]};
    if (const esrnn_status e = check_rows(s, residual_and_sum, 2, true); e != ESRNN_OK) return e;
    if (!floats_aligned(in->exists) || !floats_aligned(in->post_weight) || !floats_aligned(in->scale) || !floats_aligned(in->pre_weight) || !floats_aligned(stats) ||
        one_place({sum, out, stats}, {in->y, in->gate, sum == in->residual ? nullptr : in->residual, in->exists, in->post_weight, in->scale, in->pre_weight}))
        return ESRNN_ERR_CONFIG;
    BlockNormArgs a{};
    a.y = in->y, a.gate = in->gate, a.residual = in->residual, a.exists = in->exists;
    a.post_weight = in->post_weight, a.scale = in->scale, a.pre_weight = in->pre_weight, a.sum = sum, a.out = out, a.stats = stats;
    ESRNN_TRY(launch_block_norm_forward(s, a, static_cast<hipStream_t>(stream)));
    return ESRNN_OK;
}

esrnn_status esrnn_block_norm_backward(const esrnn_block_norm_shape *shape, const esrnn_block_norm_operands *in, const float *stats,
                                       const void *grad_out, const void *grad_sum, const esrnn_block_norm_grads *grads, void *workspace,
                                       void *stream)
{
    if (!shape || !in || !in->y || !stats || !grads || !grads->y || !workspace) return ESRNN_ERR_NULL;
    const esrnn_block_norm_shape &s = *shape;
    const esrnn_block_norm_grads &g = *grads;
    if (!block_norm_sizes(s)) return ESRNN_ERR_CONFIG;
    const bool needs_out = in->pre_weight || !in->residual;
    if ((s.gate != ESRNN_GATE_NONE && (!in->gate || !g.gate)) || (in->residual && !g.residual) || (needs_out && !grad_out) || (in->post_weight && !g.post_weight) ||
        (in->scale && !g.scale) || (in->pre_weight && !g.pre_weight))
        return ESRNN_ERR_NULL;
    if ((s.gate == ESRNN_GATE_NONE && (in->gate || g.gate)) || (!in->residual && (g.residual || grad_sum)) || (!needs_out && grad_out) ||
        (!in->post_weight && g.post_weight) || (!in->scale && g.scale) || (!in->pre_weight && g.pre_weight))
        return ESRNN_ERR_CONFIG;
    const Rows rows[] = {{in->y, s.y_stride, s.dtype, false}, {in->gate, s.gate_stride, s.dtype, false}, {in->residual, s.residual_stride, s.stream_dtype, false},
                         {grad_out, s.grad_out_stride, s.dtype, false}, {grad_sum, s.grad_sum_stride, s.stream_dtype, false}, {g.y, s.grad_y_stride, s.dtype, true},
                         {g.gate, s.grad_gate_stride, s.dtype, true}, {g.residual, s.grad_residual_stride, s.stream_dtype, true}};
    if (const esrnn_status e = check_rows(s, rows, 8, false); e != ESRNN_OK) return e;
    const float *weights[] = {in->post_weight, in->scale, in->pre_weight}, *sums[] = {g.post_weight, g.scale, g.pre_weight};
    if (!floats_aligned(in->exists) || !floats_aligned(stats) ||
        one_place({g.y, g.gate, g.residual, g.post_weight, g.scale, g.pre_weight, workspace},
                  {in->y, in->gate, in->residual, in->exists, in->post_weight, in->scale, in->pre_weight, stats, grad_out, grad_sum}))
        return ESRNN_ERR_CONFIG;
    for (int i = 0; i < 3; ++i) {
        if (!floats_aligned(weights[i]) || !floats_aligned(sums[i])) return ESRNN_ERR_CONFIG;
        for (int j = 0; j < 3; ++j)
            if (floats_overlap(sums[i], s.C, weights[j], s.C) || (i != j && floats_overlap(sums[i], s.C, sums[j], s.C))) return ESRNN_ERR_CONFIG;
    }
    if (!aligned_to(workspace, 256)) return ESRNN_ERR_WORKSPACE;
    BlockNormArgs a{};
    a.y = in->y, a.gate = in->gate, a.residual = in->residual, a.exists = in->exists;
    a.post_weight = in->post_weight, a.scale = in->scale, a.pre_weight = in->pre_weight, a.stats_in = stats;
    a.grad_out = grad_out, a.grad_sum = grad_sum, a.grad_y = g.y, a.grad_gate = g.gate, a.grad_residual = g.residual;
    a.grad_post_weight = g.post_weight, a.grad_scale = g.scale, a.grad_pre_weight = g.pre_weight, a.parts = static_cast<float *>(workspace);
    ESRNN_TRY(launch_block_norm_backward(s, a, static_cast<hipStream_t>(stream)));
    return ESRNN_OK;
}

}  // extern "C"
