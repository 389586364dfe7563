// C ABI of the layer operators (include/esrnn_layers.h): argument checks and the launches of each call.
#include "layers_internal.h"

using namespace esrnn;

#define ESRNN_TRY(expr)                              \
    do {                                             \
        hipError_t e_ = (expr);                      \
        if (e_ != hipSuccess) return ESRNN_ERR_HIP;  \
    } while (0)

namespace {

constexpr int64_t kMostElements = int64_t(1) << 40;     // of an array, gaps included: sizes in bytes and addresses stay far from overflow

bool element_type(int dtype) { return dtype == ESRNN_F32 || dtype == ESRNN_BF16 || dtype == ESRNN_F16; }
bool element_aligned(const void *p, int dtype) { return aligned_to(p, element_bytes(dtype)); }
bool floats_aligned(const void *p) { return aligned_to(p, 4); }     // (of a null pointer too)

bool recurrence_sizes(const esrnn_recurrence_shape &s)
{
    // workgroups along the first dimension of the grid: (sequence, tile of 64 channels)
    return s.B >= 1 && s.T >= 1 && s.C >= 1 && s.T <= (1 << 30) && s.C <= (1 << 24) &&
           (int64_t)s.B * ((s.C + 63) / 64) <= (1 << 23) &&
           (s.kind == ESRNN_RECURRENCE_SMOOTH || s.kind == ESRNN_RECURRENCE_DECAY) && element_type(s.dtype);
}

// Strides of a read array: any that keep it within kMostElements (zero for one sequence that is used for all of them, say).
bool readable_strides(const esrnn_recurrence_shape &s, const int64_t st[2])
{
    return st[0] >= 0 && st[1] >= 0 && st[0] <= kMostElements / s.B && st[1] <= kMostElements / s.T;
}
// Of a written one: distinct elements, in either order.
bool writable_strides(const esrnn_recurrence_shape &s, const int64_t st[2])
{
    if (!readable_strides(s, st)) return false;
    const bool positions_inside = (s.T == 1 || st[1] >= s.C) && (s.B == 1 || st[0] >= (s.T == 1 ? 0 : (int64_t)(s.T - 1) * st[1]) + s.C);
    const bool sequences_inside = (s.B == 1 || st[0] >= s.C) && (s.T == 1 || st[1] >= (s.B == 1 ? 0 : (int64_t)(s.B - 1) * st[0]) + s.C);
    return positions_inside || sequences_inside;
}

}  // namespace

extern "C" {

esrnn_status esrnn_recurrence_workspace_bytes(const esrnn_recurrence_shape *shape, size_t *bytes)
{
    if (!shape || !bytes) return ESRNN_ERR_NULL;
    if (!recurrence_sizes(*shape)) return ESRNN_ERR_CONFIG;
    const RecurrencePlan p = recurrence_plan(*shape);
    // at least something to allocate
    *bytes = p.segments > 1 ? (size_t)shape->B * p.segments * 2 * shape->C * sizeof(float) : 256;
    return ESRNN_OK;
}

esrnn_status esrnn_recurrence_saved_bytes(const esrnn_recurrence_shape *shape, size_t *bytes)
{
    if (!shape || !bytes) return ESRNN_ERR_NULL;
    if (!recurrence_sizes(*shape)) return ESRNN_ERR_CONFIG;
    *bytes = (size_t)shape->B * recurrence_plan(*shape).blocks * shape->C * sizeof(float);
    return ESRNN_OK;
}

esrnn_status esrnn_recurrence_forward(const esrnn_recurrence_shape *shape, const void *x, const void *gate, const int32_t *lengths,
                                      const float *initial, void *out, float *last, void *saved, void *workspace, void *stream)
{
    if (!shape || !x || !gate || !out || !workspace) return ESRNN_ERR_NULL;
    const esrnn_recurrence_shape &s = *shape;
    if (!recurrence_sizes(s) || !readable_strides(s, s.x_stride) || !readable_strides(s, s.gate_stride) || !writable_strides(s, s.out_stride))
        return ESRNN_ERR_CONFIG;
    if (!element_aligned(x, s.dtype) || !element_aligned(gate, s.dtype) || !element_aligned(out, s.dtype) || !floats_aligned(lengths) ||
        !floats_aligned(initial) || !floats_aligned(last) || !floats_aligned(saved))
        return ESRNN_ERR_CONFIG;
    if (!aligned_to(workspace, 256)) return ESRNN_ERR_WORKSPACE;
    const RecurrenceForward f{x, gate, lengths, initial, out, last, static_cast<float *>(saved), static_cast<float *>(workspace)};
    ESRNN_TRY(launch_recurrence_forward(s, f, static_cast<hipStream_t>(stream)));
    return ESRNN_OK;
}

esrnn_status esrnn_recurrence_backward(const esrnn_recurrence_shape *shape, const void *x, const void *gate, const int32_t *lengths,
                                       const void *saved, const void *grad_out, const float *grad_last, void *grad_x,
                                       void *grad_gate, float *grad_initial, void *workspace, void *stream)
{
    if (!shape || !x || !gate || !saved || !grad_out || !grad_x || !grad_gate || !workspace) return ESRNN_ERR_NULL;
    const esrnn_recurrence_shape &s = *shape;
    if (!recurrence_sizes(s) || !readable_strides(s, s.x_stride) || !readable_strides(s, s.gate_stride) ||
        !readable_strides(s, s.grad_out_stride) || !writable_strides(s, s.grad_x_stride) || !writable_strides(s, s.grad_gate_stride))
        return ESRNN_ERR_CONFIG;
    if (!element_aligned(x, s.dtype) || !element_aligned(gate, s.dtype) || !element_aligned(grad_out, s.dtype) ||
        !element_aligned(grad_x, s.dtype) || !element_aligned(grad_gate, s.dtype) || !floats_aligned(lengths) || !floats_aligned(saved) ||
        !floats_aligned(grad_last) || !floats_aligned(grad_initial))
        return ESRNN_ERR_CONFIG;
    if (!aligned_to(workspace, 256)) return ESRNN_ERR_WORKSPACE;
    const RecurrenceBackward f{x, gate, lengths, static_cast<const float *>(saved), grad_out, grad_last, grad_x, grad_gate, grad_initial,
                               static_cast<float *>(workspace)};
    ESRNN_TRY(launch_recurrence_backward(s, f, static_cast<hipStream_t>(stream)));
    return ESRNN_OK;
}

esrnn_status esrnn_recurrence_step(int32_t kind, int32_t dtype, int32_t rows, int32_t pool, int32_t C, const void *x, int64_t x_stride,
                                   const void *gate, int64_t gate_stride, const int32_t *slots, float *state, void *out,
                                   int64_t out_stride, void *stream)
{
    if ((kind != ESRNN_RECURRENCE_SMOOTH && kind != ESRNN_RECURRENCE_DECAY) || !element_type(dtype) || rows < 0 || pool < 0 || C < 1 ||
        C > (1 << 24) || (int64_t)rows * ((C + 1023) / 1024) > (1 << 23) || (!slots && rows > pool))
        return ESRNN_ERR_CONFIG;
    if (rows == 0) return ESRNN_OK;
    if (!x || !gate || !state || !out) return ESRNN_ERR_NULL;
    if (x_stride < 0 || gate_stride < 0 || out_stride < 0 || x_stride > kMostElements / rows || gate_stride > kMostElements / rows ||
        out_stride > kMostElements / rows || (rows > 1 && out_stride < C) || !element_aligned(x, dtype) || !element_aligned(gate, dtype) ||
        !element_aligned(out, dtype) || !floats_aligned(slots) || !floats_aligned(state))
        return ESRNN_ERR_CONFIG;
    const RecurrenceStep a{x, gate, x_stride, gate_stride, out_stride, slots, state, out, rows, pool, C};
    ESRNN_TRY(launch_recurrence_step(kind, dtype, a, static_cast<hipStream_t>(stream)));
    return ESRNN_OK;
}

}  // extern "C"
