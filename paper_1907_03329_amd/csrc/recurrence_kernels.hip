// Gated linear recurrence (include/esrnn_layers.h): h_t = a_t h_{t-1} + b_t for every channel, with a and b from a gate.
//
// Two positions one behind the other are again such a map, (A2, B2) after (A1, B1) = (A2 A1, A2 B1 + B2), and putting maps
// together is associative: a sequence is cut into pieces, every piece's map is computed at the same time, and the states between
// the pieces follow.  Here a thread has kSteps neighbouring positions of four channels in registers, sixteen threads side by side a
// row of 64 channels, so a wave has four pieces and a block of positions is 4 or 16 of them, put together by shuffles within a wave and
// through LDS between the waves.  A workgroup takes the blocks of a segment one behind the other with the state in registers.
// Sequences with few channels in all have several segments, each a workgroup: their maps come first (kMaps, reading x and
// gate once more), then every workgroup puts together the maps before its own.
//
// The reverse pass runs the same maps from the end: mu_t = a_t (d_t + mu_{t+1}), with d the gradient of out.  The states h_{t-1} that the
// gradient of the gate needs are computed again, in fp32, from the state before the block that the forward pass leaves: reading
// out instead would be one array more, and rounded to its element type.
#include <algorithm>

#include "layers_internal.h"

namespace esrnn {

namespace {

constexpr int kSteps = 8;       // positions of a thread
constexpr int kTile = 64;       // channels of a workgroup

struct Args {
    const void *x, *gate, *grad_out;
    void *out, *grad_x, *grad_gate;
    long long xb, xt, gb, gt, ob, ot, db, dt, gxb, gxt, ggb, ggt;      // strides of a sequence and of a position
    const int32_t *lengths;
    const float *initial, *saved_in, *grad_last;
    float *last, *saved, *grad_initial;
    float *parts;               // [B][segments][2][C]: maps of the segments
    int B, T, C, tiles, blocks, per_segment, segments;
};

__device__ __forceinline__ f32x4 splat(float v) { return f32x4{v, v, v, v}; }
__device__ __forceinline__ f32x4 shift_up(f32x4 v, int lanes)
{
    f32x4 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = __shfl_up(v[k], lanes, 64);
    return r;
}
__device__ __forceinline__ f32x4 from_lane(f32x4 v, int lane)
{
    f32x4 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = __shfl(v[k], lane, 64);
    return r;
}
__device__ __forceinline__ f32x4 shift_down(f32x4 v, int lanes)
{
    f32x4 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = __shfl_down(v[k], lanes, 64);
    return r;
}

// The maps of the pieces of a block, one of each thread, in order of time (or against it): what comes in at this thread's piece when
// `in` comes in at the first, and what comes out of the last.  All threads of the workgroup; `lds` is not written again before
// the next barrier but one.
template <int NW, bool kReverse>
struct Pieces {
    f32x4 A, B;             // of the pieces of this wave before this thread's
    f32x4 wave_A, wave_B;   // of the whole wave
    __device__ __forceinline__ Pieces(f32x4 a, f32x4 b, int row, int lane16)
    {
#pragma unroll
        for (int off = 1; off < 4; off *= 2) {
            const f32x4 pa = kReverse ? shift_down(a, 16 * off) : shift_up(a, 16 * off);
            const f32x4 pb = kReverse ? shift_down(b, 16 * off) : shift_up(b, 16 * off);
            if (kReverse ? row + off < 4 : row >= off) {
                b = a * pb + b;
                a = a * pa;
            }
        }
        const int end = (kReverse ? 0 : 48) + lane16;
        wave_A = from_lane(a, end);
        wave_B = from_lane(b, end);
        A = kReverse ? shift_down(a, 16) : shift_up(a, 16);
        B = kReverse ? shift_down(b, 16) : shift_up(b, 16);
        if (row == (kReverse ? 3 : 0)) {
            A = splat(1.0f);
            B = splat(0.0f);
        }
    }
    __device__ __forceinline__ void leave(f32x4 (*lds)[2][16], int wave, int row, int lane16) const
    {
        if (NW > 1 && row == 0) {
            lds[wave][0][lane16] = wave_A;
            lds[wave][1][lane16] = wave_B;
        }
    }
    // behind a barrier: `in` of this thread's piece; carry: in of the block, then out of it
    __device__ __forceinline__ f32x4 enter(f32x4 &carry, const f32x4 (*lds)[2][16], int wave, int lane16) const
    {
        if (NW == 1) {
            const f32x4 in = A * carry + B;
            carry = wave_A * carry + wave_B;
            return in;
        }
        f32x4 h = carry, mine = carry;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const int w = kReverse ? NW - 1 - i : i;
            if (w == wave) mine = h;
            h = lds[w][0][lane16] * h + lds[w][1][lane16];
        }
        carry = h;
        return A * mine + B;
    }
};

// The state behind the segments first .. end - 1 (kReverse: before them, from the last to the first) that `in` enters: their maps are dealt to the
// threads' rows in runs of neighbours and put together like the pieces of a block.
template <int NW, bool kReverse, bool kAligned>
__device__ __forceinline__ f32x4 through_segments(const float *parts, int C, int first, int end, f32x4 in, const Channels<kAligned, 16> &ch,
                                                  f32x4 (*lds)[2][16], int wave, int row, int lane16)
{
    const int n = end - first, run = (n + 4 * NW - 1) / (4 * NW);
    const int from = min((wave * 4 + row) * run, n), to = min(from + run, n);
    f32x4 A = splat(1.0f), B = splat(0.0f);
    for (int i = from; i < to; ++i) {
        const float *p = parts + (size_t)(first + (kReverse ? to - 1 - (i - from) : i)) * 2 * C;
        const f32x4 a = ch.load(p), b = ch.load(p + C);
        B = a * B + b;
        A = a * A;
    }
    const Pieces<NW, kReverse> pieces(A, B, row, lane16);
    pieces.leave(lds, wave, row, lane16);
    if (NW > 1) __syncthreads();
    (void)pieces.enter(in, lds, wave, lane16);
    if (NW > 1) __syncthreads();
    return in;
}

template <int kKind>
__device__ __forceinline__ void maps_of(f32x4 g, f32x4 x, bool inside, f32x4 &a, f32x4 &z, f32x4 &b)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const Sigmoids s = sigmoids(g[k]);
        const float keep = kKind == ESRNN_RECURRENCE_SMOOTH ? s.of_minus : s.of;
        const float take = kKind == ESRNN_RECURRENCE_SMOOTH ? s.of : s.of_minus;
        a[k] = inside ? keep : 1.0f;
        z[k] = inside ? take : 0.0f;
        b[k] = inside ? (kKind == ESRNN_RECURRENCE_SMOOTH ? take * x[k] : x[k]) : 0.0f;
    }
}

// Channels of fp32 arrays [..][C] follow the dealing of the elements'.
template <bool kAligned>
__device__ __forceinline__ f32x4 load_state(const float *p, const Channels<kAligned, 16> &ch)
{
    f32x4 v;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = p[ch.readable(k)];
    return v;
}
template <bool kAligned>
__device__ __forceinline__ void store_state(float *p, f32x4 v, const Channels<kAligned, 16> &ch)
{
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (ch.exists(k)) p[ch.channel(k)] = v[k];
}


// kMaps: the map of every segment but the last, nothing else.
template <class E, bool kAligned, int kKind, int NW, bool kMaps>
__global__ void __launch_bounds__(64 * NW) recurrence_forward_kernel(Args a)
{
    constexpr int kBlock = 4 * kSteps * NW;
    __shared__ f32x4 lds[2][NW][2][16];
    const int lane16 = threadIdx.x & 15, row = (threadIdx.x >> 4) & 3, wave = threadIdx.x >> 6;
    const int b = blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles, segment = blockIdx.y;
    const Channels<kAligned, 16> ch(lane16, tile * kTile, a.C);
    const int length = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
    const int first = segment * a.per_segment, end = min(first + a.per_segment, a.blocks);
    const E *x = static_cast<const E *>(a.x) + b * a.xb, *gate = static_cast<const E *>(a.gate) + b * a.gb;
    E *out = static_cast<E *>(a.out) + b * a.ob;
    float *parts = a.parts + (size_t)b * a.segments * 2 * a.C;

    f32x4 carry = splat(0.0f), decay = splat(1.0f);
    if (!kMaps) {
        if (a.initial) carry = load_state(a.initial + (size_t)b * a.C, ch);
        if (segment > 0) carry = through_segments<NW, false>(parts, a.C, 0, segment, carry, ch, lds[0], wave, row, lane16);
    }
    for (int block = first; block < end; ++block) {
        const int t0 = block * kBlock + (wave * 4 + row) * kSteps;
        if (block * kBlock >= length) {     // nothing left of the sequence
            if (kMaps) break;
            for (int i = 0; i < kSteps; ++i)
                if (t0 + i < a.T) ch.store(out + (t0 + i) * a.ot, Vec4<E>{});
            continue;
        }
        Vec4<E> xs[kSteps], gs[kSteps];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const long long t = min(t0 + i, length - 1);
            xs[i] = ch.load(x + t * a.xt);
            gs[i] = ch.load(gate + t * a.gt);
        }
        f32x4 as[kSteps], bs[kSteps], A = splat(1.0f), B = splat(0.0f);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            f32x4 z;
            maps_of<kKind>(to_f32<E>(gs[i]), to_f32<E>(xs[i]), t0 + i < length, as[i], z, bs[i]);
            B = as[i] * B + bs[i];
            A = as[i] * A;
        }
        const Pieces<NW, false> pieces(A, B, row, lane16);
        auto &shared = lds[block & 1];
        pieces.leave(shared, wave, row, lane16);
        if (NW > 1) __syncthreads();
        if (!kMaps && a.saved && wave == 0 && row == 0)
            store_state(a.saved + ((size_t)b * a.blocks + block) * a.C, carry, ch);
        if (kMaps) {        // the product of all a as well: the map of zero, without what it adds
            f32x4 factor = pieces.wave_A;
            if (NW > 1) {
                factor = splat(1.0f);
                for (int w = 0; w < NW; ++w) factor = factor * shared[w][0][lane16];
            }
            decay = decay * factor;
        }
        f32x4 h = pieces.enter(carry, shared, wave, lane16);
        if (kMaps) continue;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            h = as[i] * h + bs[i];
            if (t0 + i < a.T) ch.store(out + (t0 + i) * a.ot, from_f32<E>(t0 + i < length ? h : splat(0.0f)));
        }
    }
    if (wave != 0 || row != 0) return;
    if (kMaps) {
        store_state(parts + (size_t)segment * 2 * a.C, decay, ch);
        store_state(parts + ((size_t)segment * 2 + 1) * a.C, carry, ch);
    } else if (a.last && segment == a.segments - 1) {
        store_state(a.last + (size_t)b * a.C, carry, ch);
    }
}

// kMaps: the map of every segment but the first, against time.
template <class E, bool kAligned, int kKind, int NW, bool kMaps>
__global__ void __launch_bounds__(64 * NW) recurrence_backward_kernel(Args a)
{
    constexpr int kBlock = 4 * kSteps * NW;
    constexpr bool kSmooth = kKind == ESRNN_RECURRENCE_SMOOTH;
    __shared__ f32x4 lds[2][2][NW][2][16];
    const int lane16 = threadIdx.x & 15, row = (threadIdx.x >> 4) & 3, wave = threadIdx.x >> 6;
    const int b = blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles, segment = blockIdx.y + (kMaps ? 1 : 0);
    const Channels<kAligned, 16> ch(lane16, tile * kTile, a.C);
    const int length = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
    const int first = segment * a.per_segment, end = min(first + a.per_segment, a.blocks);
    const E *x = static_cast<const E *>(a.x) + b * a.xb, *gate = static_cast<const E *>(a.gate) + b * a.gb;
    const E *grad_out = static_cast<const E *>(a.grad_out) + b * a.db;
    E *grad_x = static_cast<E *>(a.grad_x) + b * a.gxb, *grad_gate = static_cast<E *>(a.grad_gate) + b * a.ggb;
    float *parts = a.parts + (size_t)b * a.segments * 2 * a.C;

    f32x4 carry = splat(0.0f), decay = splat(1.0f);
    if (!kMaps) {
        if (a.grad_last) carry = load_state(a.grad_last + (size_t)b * a.C, ch);
        if (segment < a.segments - 1)
            carry = through_segments<NW, true>(parts, a.C, segment + 1, a.segments, carry, ch, lds[0][0], wave, row, lane16);
    }
    for (int block = end - 1; block >= first; --block) {
        const int t0 = block * kBlock + (wave * 4 + row) * kSteps;
        if (block * kBlock >= length) {
            if (kMaps) continue;
            for (int i = 0; i < kSteps; ++i)
                if (t0 + i < a.T) {
                    ch.store(grad_x + (t0 + i) * a.gxt, Vec4<E>{});
                    ch.store(grad_gate + (t0 + i) * a.ggt, Vec4<E>{});
                }
            continue;
        }
        Vec4<E> xs[kSteps], gs[kSteps], ds[kSteps];
        f32x4 before;
        if (!kMaps) before = load_state(a.saved_in + ((size_t)b * a.blocks + block) * a.C, ch);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const long long t = min(t0 + i, length - 1);
            gs[i] = ch.load(gate + t * a.gt);
            ds[i] = ch.load(grad_out + t * a.dt);
            if (!kMaps) xs[i] = ch.load(x + t * a.xt);
        }
        f32x4 as[kSteps], zs[kSteps], A = splat(1.0f), B = splat(0.0f), M = splat(0.0f);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            f32x4 add;
            maps_of<kKind>(to_f32<E>(gs[i]), kMaps ? splat(0.0f) : to_f32<E>(xs[i]), t0 + i < length, as[i], zs[i], add);
            B = as[i] * B + add;
            A = as[i] * A;
        }
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i) M = as[i] * ((t0 + i < length ? to_f32<E>(ds[i]) : splat(0.0f)) + M);
        const Pieces<NW, true> back(A, M, row, lane16);
        auto &shared = lds[block & 1];
        back.leave(shared[1], wave, row, lane16);
        if (kMaps) {
            if (NW > 1) __syncthreads();
            f32x4 factor = back.wave_A;
            if (NW > 1) {
                factor = splat(1.0f);
                for (int w = NW - 1; w >= 0; --w) factor = factor * shared[1][w][0][lane16];
            }
            decay = decay * factor;
            (void)back.enter(carry, shared[1], wave, lane16);
            continue;
        }
        const Pieces<NW, false> forth(A, B, row, lane16);
        forth.leave(shared[0], wave, row, lane16);
        if (NW > 1) __syncthreads();
        f32x4 mu = back.enter(carry, shared[1], wave, lane16);
        f32x4 h = forth.enter(before, shared[0], wave, lane16);
        f32x4 hs[kSteps];       // the state before each position
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            hs[i] = h;
            const f32x4 xi = to_f32<E>(xs[i]);
            h = as[i] * h + (kSmooth ? (t0 + i < length ? zs[i] * xi : splat(0.0f)) : (t0 + i < length ? xi : splat(0.0f)));
        }
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i) {
            const bool inside = t0 + i < length;
            const f32x4 lambda = (inside ? to_f32<E>(ds[i]) : splat(0.0f)) + mu;
            mu = as[i] * lambda;
            if (t0 + i < a.T) {
                const f32x4 gx = kSmooth ? zs[i] * lambda : lambda;
                const f32x4 gg = mu * zs[i] * (kSmooth ? to_f32<E>(xs[i]) - hs[i] : hs[i]);
                ch.store(grad_x + (t0 + i) * a.gxt, from_f32<E>(inside ? gx : splat(0.0f)));
                ch.store(grad_gate + (t0 + i) * a.ggt, from_f32<E>(inside ? gg : splat(0.0f)));
            }
        }
    }
    if (wave != 0 || row != 0) return;
    if (kMaps) {
        store_state(parts + (size_t)segment * 2 * a.C, decay, ch);
        store_state(parts + ((size_t)segment * 2 + 1) * a.C, carry, ch);
    } else if (a.grad_initial && segment == 0) {
        store_state(a.grad_initial + (size_t)b * a.C, carry, ch);
    }
}

// One position: a workgroup has 1024 neighbouring channels of a request.
template <class E, bool kAligned, int kKind>
__global__ void __launch_bounds__(256) recurrence_step_kernel(RecurrenceStep a, int tiles)
{
    const int i = blockIdx.x / tiles, tile = blockIdx.x % tiles;
    const Channels<kAligned, 256> ch(threadIdx.x, tile * 1024, a.C);
    if (!ch.exists(0)) return;
    const int slot = a.slots ? a.slots[i] : i;
    E *out = static_cast<E *>(a.out) + i * a.out_stride;
    if (slot < 0 || slot >= a.pool) {
        ch.store(out, Vec4<E>{});
        return;
    }
    const f32x4 x = to_f32<E>(ch.load(static_cast<const E *>(a.x) + i * a.x_stride));
    const f32x4 g = to_f32<E>(ch.load(static_cast<const E *>(a.gate) + i * a.gate_stride));
    float *state = a.state + (size_t)slot * a.C;
    f32x4 keep, take, add;
    maps_of<kKind>(g, x, true, keep, take, add);
    const f32x4 h = keep * ch.load(state) + add;
    ch.store(state, h);
    ch.store(out, from_f32<E>(h));
}

template <int v>
using Int = std::integral_constant<int, v>;

template <class F>
void with_variant(bool aligned, int kind, F &&f)
{
    const auto of_kind = [&](auto al) {
        if (kind == ESRNN_RECURRENCE_SMOOTH) f(al, Int<ESRNN_RECURRENCE_SMOOTH>{});
        else f(al, Int<ESRNN_RECURRENCE_DECAY>{});
    };
    if (aligned) of_kind(std::true_type{});
    else of_kind(std::false_type{});
}

Args args_of(const esrnn_recurrence_shape &s, const RecurrencePlan &p)
{
    Args r{};
    r.xb = s.x_stride[0], r.xt = s.x_stride[1], r.gb = s.gate_stride[0], r.gt = s.gate_stride[1];
    r.ob = s.out_stride[0], r.ot = s.out_stride[1];
    r.db = s.grad_out_stride[0], r.dt = s.grad_out_stride[1];
    r.gxb = s.grad_x_stride[0], r.gxt = s.grad_x_stride[1], r.ggb = s.grad_gate_stride[0], r.ggt = s.grad_gate_stride[1];
    r.B = s.B, r.T = s.T, r.C = s.C;
    r.tiles = (s.C + kTile - 1) / kTile;
    r.blocks = p.blocks, r.per_segment = p.per_segment, r.segments = p.segments;
    return r;
}

bool groups_of_four(const void *p, const int64_t stride[2], int dtype)
{
    return aligned_to(p, 4 * element_bytes(dtype)) && (stride[0] | stride[1]) % 4 == 0;
}

}  // namespace

RecurrencePlan recurrence_plan(const esrnn_recurrence_shape &s)
{
    RecurrencePlan p;
    p.waves = s.T <= 64 ? 1 : 4;
    p.block = 4 * kSteps * p.waves;
    p.blocks = (s.T + p.block - 1) / p.block;
    const long long rows = (long long)s.B * ((s.C + kTile - 1) / kTile);
    const long long wanted = std::max<long long>(1, std::min<long long>(p.blocks, 1024 / rows));
    p.per_segment = (int)((p.blocks + wanted - 1) / wanted);
    p.segments = (p.blocks + p.per_segment - 1) / p.per_segment;
    return p;
}

hipError_t launch_recurrence_forward(const esrnn_recurrence_shape &s, const RecurrenceForward &f, hipStream_t st)
{
    const RecurrencePlan p = recurrence_plan(s);
    Args a = args_of(s, p);
    a.x = f.x, a.gate = f.gate, a.out = f.out, a.lengths = f.lengths, a.initial = f.initial, a.last = f.last, a.saved = f.saved, a.parts = f.parts;
    const bool aligned = s.C % 4 == 0 && groups_of_four(f.x, s.x_stride, s.dtype) && groups_of_four(f.gate, s.gate_stride, s.dtype) &&
                         groups_of_four(f.out, s.out_stride, s.dtype);
    return with_element(s.dtype, [&](auto e) {
        using E = decltype(e);
        with_variant(aligned, s.kind, [&](auto al, auto kind) {
            const unsigned rows = (unsigned)(s.B * a.tiles);
            const dim3 maps(rows, a.segments - 1), all(rows, a.segments);
            if (p.waves == 1) {
                if (maps.y) recurrence_forward_kernel<E, al(), kind(), 1, true><<<maps, 64, 0, st>>>(a);
                recurrence_forward_kernel<E, al(), kind(), 1, false><<<all, 64, 0, st>>>(a);
            } else {
                if (maps.y) recurrence_forward_kernel<E, al(), kind(), 4, true><<<maps, 256, 0, st>>>(a);
                recurrence_forward_kernel<E, al(), kind(), 4, false><<<all, 256, 0, st>>>(a);
            }
        });
        return hipGetLastError();
    });
}

hipError_t launch_recurrence_backward(const esrnn_recurrence_shape &s, const RecurrenceBackward &f, hipStream_t st)
{
    const RecurrencePlan p = recurrence_plan(s);
    Args a = args_of(s, p);
    a.x = f.x, a.gate = f.gate, a.grad_out = f.grad_out, a.grad_x = f.grad_x, a.grad_gate = f.grad_gate, a.lengths = f.lengths;
    a.saved_in = f.saved, a.grad_last = f.grad_last, a.grad_initial = f.grad_initial, a.parts = f.parts;
    const bool aligned = s.C % 4 == 0 && groups_of_four(f.x, s.x_stride, s.dtype) && groups_of_four(f.gate, s.gate_stride, s.dtype) &&
                         groups_of_four(f.grad_out, s.grad_out_stride, s.dtype) && groups_of_four(f.grad_x, s.grad_x_stride, s.dtype) &&
                         groups_of_four(f.grad_gate, s.grad_gate_stride, s.dtype);
    return with_element(s.dtype, [&](auto e) {
        using E = decltype(e);
        with_variant(aligned, s.kind, [&](auto al, auto kind) {
            const unsigned rows = (unsigned)(s.B * a.tiles);
            const dim3 maps(rows, a.segments - 1), all(rows, a.segments);
            if (p.waves == 1) {
                if (maps.y) recurrence_backward_kernel<E, al(), kind(), 1, true><<<maps, 64, 0, st>>>(a);
                recurrence_backward_kernel<E, al(), kind(), 1, false><<<all, 64, 0, st>>>(a);
            } else {
                if (maps.y) recurrence_backward_kernel<E, al(), kind(), 4, true><<<maps, 256, 0, st>>>(a);
                recurrence_backward_kernel<E, al(), kind(), 4, false><<<all, 256, 0, st>>>(a);
            }
        });
        return hipGetLastError();
    });
}

hipError_t launch_recurrence_step(int kind, int dtype, const RecurrenceStep &a, hipStream_t st)
{
    const int64_t strides[3][2] = {{a.x_stride, 0}, {a.gate_stride, 0}, {a.out_stride, 0}};
    const bool aligned = a.C % 4 == 0 && groups_of_four(a.x, strides[0], dtype) && groups_of_four(a.gate, strides[1], dtype) &&
                         groups_of_four(a.out, strides[2], dtype) && aligned_to(a.state, 16);
    const int tiles = (a.C + 1023) / 1024;
    return with_element(dtype, [&](auto e) {
        using E = decltype(e);
        with_variant(aligned, kind, [&](auto al, auto k) {
            recurrence_step_kernel<E, al(), k()><<<(unsigned)(a.rows * tiles), 256, 0, st>>>(a, tiles);
        });
        return hipGetLastError();
    });
}

}  // namespace esrnn
