// C ABI of the layer operators (include/esrnn_layers.h): argument checks and the launches of each call.
#include <algorithm>
#include <cmath>
#include <limits>
#include <new>

#include "layers_checks.h"

using namespace esrnn;

namespace {

bool recurrence_sizes(const esrnn_recurrence_shape &s)
{
    // workgroups along the first dimension of the grid: (sequence, tile of channels)
    return s.B >= 1 && s.T >= 1 && s.C >= 1 && s.T <= (1 << 30) && s.C <= (1 << 24) &&
           (int64_t)s.B * ((s.C + 63) / 64) <= (1 << 22) &&
           (s.kind == ESRNN_RECURRENCE_SMOOTH || s.kind == ESRNN_RECURRENCE_DECAY) && element_type(s.dtype);
}

bool group_norm_sizes(const esrnn_group_norm_shape &s)
{
    if (!(s.N >= 1 && s.T >= 1 && s.C >= 1 && s.G >= 1 && s.C <= (1 << 20) && s.T <= (1 << 30) && s.C % s.G == 0)) return false;
    // single positions by some thousand workgroups, whatever N is: offsets of samples are 64 bits, their numbers 32
    // anything else by a workgroup or more for (sample, tile of channels)
    const bool fits = group_norm_single_positions(s) ? s.N <= (1 << 30) && s.C <= kMostElements / s.N
                                                     : (int64_t)s.N * s.T <= (int64_t(1) << 31) &&
                                                           (int64_t)s.N * ((s.C + 63) / 64) <= (1 << 22) && (int64_t)s.N * s.G <= (1 << 25);
    return fits && (s.activation == ESRNN_NORM_NONE || s.activation == ESRNN_NORM_SILU) && element_type(s.dtype) && s.eps > 0.0f &&
           s.eps < __builtin_inff();
}

}  // namespace

struct esrnn_adamw {
    AdamWEntry *entry;
    int count, state_bits, chunk, chunks;       // elements of a chunk, chunks
    int64_t elements;           // of a flat moment array
    const void *bound;          // the workspace that has the table, or null
};

namespace {

// The workspace: partial sums of squares, the tensors, the tensor of every chunk.
size_t adamw_entries_at() { return kAdamWNormBlocks * sizeof(double); }
size_t adamw_owner_at(const esrnn_adamw &h) { return (adamw_entries_at() + h.count * sizeof(AdamWEntry) + 255) / 256 * 256; }

}  // namespace

extern "C" {

esrnn_status esrnn_recurrence_workspace_bytes(const esrnn_recurrence_shape *shape, size_t *bytes)
{
    if (!shape || !bytes) return ESRNN_ERR_NULL;
    if (!recurrence_sizes(*shape)) return ESRNN_ERR_CONFIG;
    const RecurrencePlan p = recurrence_plan(*shape);
    // at least something to allocate
    *bytes = p.ahead ? p.words * sizeof(float) : 256;
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
    const size_t states = (size_t)s.B * s.C, kept = states * recurrence_plan(s).blocks;
    const float *left = static_cast<const float *>(saved);
    if (rows_overlap(s, out, s.out_stride, x, s.x_stride) || rows_overlap(s, out, s.out_stride, gate, s.gate_stride) ||
        floats_overlap(last, states, initial, states) || floats_overlap(left, kept, initial, states) || floats_overlap(left, kept, last, states))
        return ESRNN_ERR_CONFIG;
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
    const size_t states = (size_t)s.B * s.C, kept = states * recurrence_plan(s).blocks;
    if (rows_overlap(s, grad_x, s.grad_x_stride, grad_gate, s.grad_gate_stride) || floats_overlap(grad_initial, states, grad_last, states) ||
        floats_overlap(grad_initial, states, static_cast<const float *>(saved), kept))
        return ESRNN_ERR_CONFIG;
    const struct {
        const void *p;
        const int64_t *stride;
    } read[3] = {{x, s.x_stride}, {gate, s.gate_stride}, {grad_out, s.grad_out_stride}};
    for (const auto &r : read)
        if (rows_overlap(s, grad_x, s.grad_x_stride, r.p, r.stride) || rows_overlap(s, grad_gate, s.grad_gate_stride, r.p, r.stride)) return ESRNN_ERR_CONFIG;
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

esrnn_status esrnn_group_norm_workspace_bytes(const esrnn_group_norm_shape *shape, size_t *bytes)
{
    if (!shape || !bytes) return ESRNN_ERR_NULL;
    if (!group_norm_sizes(*shape)) return ESRNN_ERR_CONFIG;
    *bytes = (group_norm_workspace_floats(*shape) * sizeof(float) + 255) / 256 * 256;
    return ESRNN_OK;
}

esrnn_status esrnn_group_norm_forward(const esrnn_group_norm_shape *shape, const void *x, const int32_t *lengths, const float *scale,
                                      const float *shift, void *out, float *stats, void *workspace, void *stream)
{
    if (!shape || !x || !scale || !shift || !out || !workspace) return ESRNN_ERR_NULL;
    const esrnn_group_norm_shape &s = *shape;
    if (!group_norm_sizes(s) || !element_aligned(x, s.dtype) || !element_aligned(out, s.dtype) || !floats_aligned(lengths) ||
        !floats_aligned(scale) || !floats_aligned(shift) || !floats_aligned(stats))
        return ESRNN_ERR_CONFIG;
    if (!aligned_to(workspace, 256)) return ESRNN_ERR_WORKSPACE;
    GroupNormArgs a{};
    a.x = x, a.lengths = lengths, a.scale = scale, a.shift = shift, a.out = out, a.stats = stats, a.parts = static_cast<float *>(workspace);
    ESRNN_TRY(launch_group_norm_forward(s, a, static_cast<hipStream_t>(stream)));
    return ESRNN_OK;
}

esrnn_status esrnn_group_norm_backward(const esrnn_group_norm_shape *shape, const void *x, const int32_t *lengths, const float *scale,
                                       const float *shift, const float *stats, const void *grad_out, void *grad_x,
                                       float *grad_scale, float *grad_shift, void *workspace, void *stream)
{
    if (!shape || !x || !scale || !shift || !stats || !grad_out || !grad_x || !grad_scale || !grad_shift || !workspace) return ESRNN_ERR_NULL;
    const esrnn_group_norm_shape &s = *shape;
    if (!group_norm_sizes(s) || !element_aligned(x, s.dtype) || !element_aligned(grad_out, s.dtype) || !element_aligned(grad_x, s.dtype) ||
        !floats_aligned(lengths) || !floats_aligned(scale) || !floats_aligned(shift) || !floats_aligned(stats) || !floats_aligned(grad_scale) ||
        !floats_aligned(grad_shift))
        return ESRNN_ERR_CONFIG;
    if (!aligned_to(workspace, 256)) return ESRNN_ERR_WORKSPACE;
    GroupNormArgs a{};
    a.x = x, a.lengths = lengths, a.scale = scale, a.shift = shift, a.stats_in = stats, a.grad_out = grad_out, a.grad_x = grad_x;
    a.grad_scale = grad_scale, a.grad_shift = grad_shift, a.parts = static_cast<float *>(workspace);
    ESRNN_TRY(launch_group_norm_backward(s, a, static_cast<hipStream_t>(stream)));
    return ESRNN_OK;
}

esrnn_status esrnn_adamw_create(const esrnn_adamw_tensor *tensors, int32_t count, int32_t state_bits, esrnn_adamw **out)
{
    if (!out) return ESRNN_ERR_NULL;
    *out = nullptr;
    if (!tensors) return ESRNN_ERR_NULL;
    if (count < 1 || count > (1 << 20) || (state_bits != 32 && state_bits != 8)) return ESRNN_ERR_CONFIG;
    esrnn_adamw *h = new (std::nothrow) esrnn_adamw{};
    AdamWEntry *entry = new (std::nothrow) AdamWEntry[count];
    if (!h || !entry) {
        delete h;
        delete[] entry;
        return ESRNN_ERR_HIP;
    }
    h->entry = entry;
    h->bound = nullptr;
    esrnn_status st = ESRNN_OK;
    int64_t flat = 0, chunks = 0;
    for (int32_t i = 0; i < count && st == ESRNN_OK; ++i) {
        const esrnn_adamw_tensor &t = tensors[i];
        if (!t.param || !t.grad) st = ESRNN_ERR_NULL;
        else if (t.n < 1 || t.n > kMostElements || !(t.weight_decay >= 0.0f && t.weight_decay < __builtin_inff()) || !element_type(t.grad_dtype) ||
                 (t.copy && t.copy_dtype != ESRNN_BF16 && t.copy_dtype != ESRNN_F16) || !floats_aligned(t.param) ||
                 !element_aligned(t.grad, t.grad_dtype) || !aligned_to(t.copy, 2))
            st = ESRNN_ERR_CONFIG;
        else {
            AdamWEntry &e = entry[i];
            e = AdamWEntry{};
            e.param = t.param, e.grad = t.grad, e.copy = t.copy, e.n = t.n, e.flat = flat;
            e.weight_decay = t.weight_decay;
            e.grad_dtype = (unsigned char)t.grad_dtype, e.copy_dtype = (unsigned char)t.copy_dtype;
            flat += (t.n + ESRNN_ADAMW_BLOCK - 1) / ESRNN_ADAMW_BLOCK * ESRNN_ADAMW_BLOCK;
            chunks += (t.n + kAdamWChunk - 1) / kAdamWChunk;
            if (chunks > (1 << 23)) st = ESRNN_ERR_CONFIG;      // (workgroups of a launch; 1.7e10 elements)
        }
    }
    if (st != ESRNN_OK) {
        delete[] entry;
        delete h;
        return st;
    }
    h->chunk = chunks <= kAdamWFewChunks ? kAdamWSmallChunk : kAdamWChunk;
    chunks = 0;
    for (int32_t i = 0; i < count; ++i) {
        entry[i].first_chunk = (int)chunks;
        chunks += (entry[i].n + h->chunk - 1) / h->chunk;
    }
    h->count = count, h->state_bits = state_bits, h->chunks = (int)chunks, h->elements = flat;
    *out = h;
    return ESRNN_OK;
}

esrnn_status esrnn_adamw_destroy(esrnn_adamw *h)
{
    if (!h) return ESRNN_ERR_NULL;
    delete[] h->entry;
    delete h;
    return ESRNN_OK;
}

esrnn_status esrnn_adamw_state_elements(const esrnn_adamw *h, size_t *n)
{
    if (!h || !n) return ESRNN_ERR_NULL;
    *n = (size_t)h->elements;
    return ESRNN_OK;
}

esrnn_status esrnn_adamw_workspace_bytes(const esrnn_adamw *h, size_t *bytes)
{
    if (!h || !bytes) return ESRNN_ERR_NULL;
    *bytes = adamw_owner_at(*h) + ((size_t)h->chunks * sizeof(int) + 255) / 256 * 256;
    return ESRNN_OK;
}

esrnn_status esrnn_adamw_bind(esrnn_adamw *h, void *workspace, void *stream)
{
    if (!h || !workspace) return ESRNN_ERR_NULL;
    if (!aligned_to(workspace, 256)) return ESRNN_ERR_WORKSPACE;
    char *ws = static_cast<char *>(workspace);
    ESRNN_TRY(launch_adamw_bind(h->entry, h->count, reinterpret_cast<AdamWEntry *>(ws + adamw_entries_at()),
                                reinterpret_cast<int *>(ws + adamw_owner_at(*h)), h->chunks, static_cast<hipStream_t>(stream)));
    h->bound = workspace;
    return ESRNN_OK;
}

esrnn_status esrnn_adamw_update(const esrnn_adamw *h, const esrnn_adamw_config *opt, int32_t step, void *m, float *v, void *r,
                                float *m_scale, float *r_scale, float *norm, void *workspace, void *stream)
{
    if (!h || !opt || !m || !workspace) return ESRNN_ERR_NULL;
    if (h->state_bits == 32 ? !v : !r || !m_scale || !r_scale) return ESRNN_ERR_NULL;
    const auto rate = [](double b) { return b >= 0.0 && b < 1.0; };
    if (step < 1 || !rate(opt->beta1) || !rate(opt->beta2) || !(opt->lr >= 0.0) || !(opt->eps >= 0.0) || !(opt->lr < __builtin_inf()) ||
        opt->clip_norm != opt->clip_norm)
        return ESRNN_ERR_CONFIG;
    // whole groups of four moments
    if (!aligned_to(m, h->state_bits == 32 ? 16 : 4) || !aligned_to(v, 16) || !aligned_to(r, 4) || !floats_aligned(m_scale) ||
        !floats_aligned(r_scale) || !floats_aligned(norm))
        return ESRNN_ERR_CONFIG;
    if (workspace != h->bound) return ESRNN_ERR_ORDER;
    char *ws = static_cast<char *>(workspace);
    AdamWUpdate u{};
    u.entries = reinterpret_cast<const AdamWEntry *>(ws + adamw_entries_at());
    u.owner = reinterpret_cast<const int *>(ws + adamw_owner_at(*h));
    u.lr = (float)opt->lr;
    // Both at least the smallest normal number, unless they are zero.  Clipping to less than that stays clipping; and of eps the hardware's reciprocal is infinite
    // where it is smaller, and zero times that NaN where a gradient has always been zero (roots that are not zero are above 2^-75, and the sum with
    // them is the same).
    u.clip_norm = opt->clip_norm > 0.0 ? std::max((float)opt->clip_norm, std::numeric_limits<float>::min()) : 0.0f;
    u.eps = opt->eps > 0.0 ? std::max((float)opt->eps, std::numeric_limits<float>::min()) : 0.0f;
    u.beta1 = (float)opt->beta1, u.new1 = (float)(1.0 - opt->beta1), u.beta2 = (float)opt->beta2, u.new2 = (float)(1.0 - opt->beta2);
    u.rate = (float)(opt->lr / (1.0 - std::pow(opt->beta1, (double)step)));
    u.root_correction = (float)(1.0 / std::sqrt(1.0 - std::pow(opt->beta2, (double)step)));
    u.key = opt->seed * 0x9E3779B1u + (uint32_t)step * 0x85EBCA77u;
    u.m = m, u.v = v, u.r = r, u.m_scale = m_scale, u.r_scale = r_scale, u.norm = norm;
    ESRNN_TRY(launch_adamw_update(u, h->chunk, h->chunks, reinterpret_cast<double *>(ws), h->state_bits, static_cast<hipStream_t>(stream)));
    return ESRNN_OK;
}

}  // extern "C"
