// Gated linear recurrence (include/esrnn_layers.h): h_t = a_t h_{t-1} + b_t for every channel, with a and b from a gate.
//
// Two positions one behind the other are again such a map, (A2, B2) after (A1, B1) = (A2 A1, A2 B1 + B2), and putting maps
// together is associative: a sequence is cut into pieces, every piece's map is computed at the same time, and the states between
// the pieces follow.  Here a thread has kSteps neighbouring positions of four channels in registers, sixteen threads side by side a
// row of 64 channels, so a wave has four pieces and a block of positions is 4 or 16 of them, put together by shuffles within a wave and
// through LDS between the waves.
//
// Many sequences and channels: a workgroup takes all blocks of its 64 channels one behind the other, the state in registers.
// Few: every block has a workgroup of its own (kAhead), which reads its positions once, hands its map on through memory, and puts together
// the maps of the blocks before it, which are under way at the same time.  (As two launches, maps first and then x and gate once more, 8
// sequences of 4096 positions and 2048 channels took 146 us forward and 198 us in reverse.)
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
// rows of 64 channels from which a workgroup takes a whole sequence
constexpr int kLinesAlone = 1024;

struct Args {
    const void *x, *gate, *grad_out;
    void *out, *grad_x, *grad_gate;
    long long xb, xt, gb, gt, ob, ot, db, dt, gxb, gxt, ggb, ggt;      // strides of a sequence and of a position
    const int32_t *lengths;
    const float *initial, *saved_in, *grad_last;
    float *last, *saved, *grad_initial;
    float *words;               // kAhead: the ticket (256 bytes), then for each 64 channels of a sequence the maps of its blocks
    int B, T, C, tiles, blocks, groups, log_group;      // and of their groups of 2^log_group blocks, [blocks + groups][2][64]
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

// The maps of the pieces of a block, one of each thread, in order of time (or against it: then the caller counts waves from the last one
// as well): what comes in at this thread's piece when `carry` comes in at the first, and what comes out of the last.  All threads of the
// workgroup; `lds` is not written again before the next barrier but one.
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
        for (int w = 0; w < NW; ++w) {
            if (w == wave) mine = h;
            h = lds[w][0][lane16] * h + lds[w][1][lane16];
        }
        carry = h;
        return A * mine + B;
    }
};

// Maps that pass from workgroup to workgroup.
//
// They are written through to memory and read past the caches, and every float tells by itself whether it is there: the words are
// filled with kEmpty before the launch (no result has this pattern, one of the NaNs).  Which maps a block puts together, and how, depends on
// its number alone: those of the whole groups before its own, then those of the blocks before it in its group; the last block of a group
// hands on the group's map, and waits for no other group for that.  So results do not depend on who was first, a block waits for two
// others one behind the other at most, and reads 2 sqrt(blocks) maps at most.
// Every wait ends: blocks are taken by ticket, in the order in which they follow each other, whoever waits waits for lower tickets only, and
// a block's own map waits for nobody.  (A wait that goes on for seconds all the same, because calls overlap on one workspace, is given
// up, once for all this thread reads; its maps are NaN.)
constexpr unsigned kEmpty = 0xffffffffu;
constexpr int kMostLooks = 1 << 22, kMap = 128;     // floats of a map

struct Map {
    f32x4 A, B;
    __device__ __forceinline__ Map after(const Map &o) const { return {A * o.A, A * o.B + B}; }
};
__device__ __forceinline__ bool there(f32x4 v)
{
    const u32x4 u = __builtin_bit_cast(u32x4, v);
    return u[0] != kEmpty && u[1] != kEmpty && u[2] != kEmpty && u[3] != kEmpty;
}
// The maps of a row of 64 channels: of its blocks, behind them of their groups.  Map i is at 4 i kMap bytes.
struct Line {
    buf_rsrc at;
    int blocks;
    bool lost = false;
    __device__ __forceinline__ Line(float *words, int n_blocks, int n_groups) : at(make_rsrc(words, 4 * kMap * (n_blocks + n_groups))), blocks(n_blocks) {}

    __device__ __forceinline__ Map look(int i) const
    {
        const unsigned lane_bytes = 4 * kMap * i + 16 * (threadIdx.x & 15);
        return {__builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(at, lane_bytes, 0, kBufShared)),
                __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(at, lane_bytes + 256, 0, kBufShared))};
    }
    // by the sixteen threads of one row
    __device__ __forceinline__ void hand_on(int i, const Map &m) const
    {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            f32x4 v = half ? m.B : m.A;
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = v[k] != v[k] ? __builtin_nanf("") : v[k];
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), at, 4 * kMap * i + 256 * half + 16 * (threadIdx.x & 15), 0, kBufShared);
        }
    }
    // map i of this thread's row
    __device__ __forceinline__ Map wait(int i)
    {
        asm volatile("" ::: "memory");
        Map m = look(i);
        for (int looks = lost ? kMostLooks : 0; !(there(m.A) && there(m.B)); ++looks) {
            asm volatile("" ::: "memory");
            if (looks == kMostLooks) {
                lost = true;
                break;
            }
            __builtin_amdgcn_s_sleep(1);
            m = look(i);
        }
        return lost ? Map{splat(__builtin_nanf("")), splat(__builtin_nanf(""))} : m;
    }
    // n maps one behind the other, the first `groups_first` of them of groups, the others of blocks from `block` on: dealt to the rows of
    // the workgroup in runs of neighbours, which are put together like the pieces of a block.  All threads; `lds` is the call's own.
    template <int NW>
    __device__ __forceinline__ Map put_together(int groups_first, int block, int n, f32x4 (*lds)[2][16], int wave, int row, int lane16)
    {
        const int run = (n + 4 * NW - 1) / (4 * NW), from = min((wave * 4 + row) * run, n), to = min(from + run, n);
        Map m{splat(1.0f), splat(0.0f)};
        for (int j = from; j < to; ++j)
            m = wait(j < groups_first ? blocks + j : block + j - groups_first).after(m);
        const Pieces<NW, false> pieces(m.A, m.B, row, lane16);
        pieces.leave(lds, wave, row, lane16);
        __syncthreads();
        return whole<NW>(lds, lane16);
    }
    // the map of a whole block from what its waves have left
    template <int NW>
    static __device__ __forceinline__ Map whole(const f32x4 (*lds)[2][16], int lane16)
    {
        Map m{lds[0][0][lane16], lds[0][1][lane16]};
#pragma unroll
        for (int w = 1; w < NW; ++w) m = Map{lds[w][0][lane16], lds[w][1][lane16]}.after(m);
        return m;
    }
    // The state that enters block k of the sequence, if `first` enters the first: hands on the block's map, and the group's.
    template <int NW>
    __device__ __forceinline__ f32x4 entering(int k, const Map &own, f32x4 first, int log_group, f32x4 (*lds)[NW][2][16], int wave, int row, int lane16)
    {
        const bool writes = wave == 0 && row == 0;
        if (writes) hand_on(k, own);
        const int group = k >> log_group, in_group = k & ((1 << log_group) - 1);
        Map m{splat(1.0f), splat(0.0f)};
        if (in_group == (1 << log_group) - 1) {
            m = put_together<NW>(0, group << log_group, in_group, lds[0], wave, row, lane16);
            if (writes) hand_on(blocks + group, own.after(m));
            if (group > 0) m = m.after(put_together<NW>(group, 0, group, lds[1], wave, row, lane16));
        } else if (k > 0) {
            m = put_together<NW>(group, group << log_group, group + in_group, lds[0], wave, row, lane16);
        }
        // (NaN for all threads of the workgroup: what one of them could not wait for has gone through LDS)
        return m.A * first + m.B;
    }
};

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


// What a workgroup works on: a row of 64 channels of a sequence, and with kAhead one of its blocks, drawn by ticket: rows side by side, block for
// block.
struct Place {
    int line, block;
};
template <bool kAhead>
__device__ __forceinline__ Place draw_place(const Args &a)
{
    if (!kAhead) return {(int)blockIdx.x, 0};
    __shared__ unsigned s_ticket;
    if (threadIdx.x == 0) s_ticket = atomicAdd(reinterpret_cast<unsigned *>(a.words), 1u);
    __syncthreads();
    // (in a workspace that another call writes, a ticket is any number: every place has to be in the launch)
    const unsigned ticket = min((unsigned)__builtin_amdgcn_readfirstlane((int)s_ticket), gridDim.x - 1), lines = (unsigned)(a.B * a.tiles);
    return {(int)(ticket % lines), (int)(ticket / lines)};
}
__device__ __forceinline__ Line line_of(const Args &a, int line)
{
    return Line(a.words + 64 + (size_t)line * (a.blocks + a.groups) * kMap, a.blocks, a.groups);
}

template <class E, bool kAligned, int kKind, int NW, bool kAhead>
__global__ void __launch_bounds__(64 * NW) recurrence_forward_kernel(Args a)
{
    constexpr int kBlock = 4 * kSteps * NW;
    __shared__ f32x4 lds[2][NW][2][16];
    __shared__ f32x4 lds_ahead[kAhead ? 2 : 1][NW][2][16];
    const int lane16 = threadIdx.x & 15, row = (threadIdx.x >> 4) & 3, wave = threadIdx.x >> 6;
    const Place place = draw_place<kAhead>(a);
    const int b = place.line / a.tiles, tile = place.line % a.tiles;
    const Channels<kAligned, 16> ch(lane16, tile * kTile, a.C);
    const int length = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
    const E *x = static_cast<const E *>(a.x) + b * a.xb, *gate = static_cast<const E *>(a.gate) + b * a.gb;
    E *out = static_cast<E *>(a.out) + b * a.ob;
    const bool writes = wave == 0 && row == 0;

    f32x4 carry = splat(0.0f);
    if (a.initial) carry = load_state(a.initial + (size_t)b * a.C, ch);
    if (length == 0 && place.block == 0 && writes && a.last) store_state(a.last + (size_t)b * a.C, carry, ch);
    const int end = kAhead ? place.block + 1 : a.blocks;
    for (int block = place.block; block < end; ++block) {
        const int t0 = block * kBlock + (wave * 4 + row) * kSteps;
        if (block * kBlock >= length) {     // nothing left of the sequence
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
        auto &shared = lds[kAhead ? 0 : block & 1];
        pieces.leave(shared, wave, row, lane16);
        if (NW > 1) __syncthreads();
        if constexpr (kAhead)
            carry = line_of(a, place.line).template entering<NW>(block, Line::whole<NW>(shared, lane16), carry, a.log_group, lds_ahead, wave, row, lane16);
        if (a.saved && writes) store_state(a.saved + ((size_t)b * a.blocks + block) * a.C, carry, ch);
        f32x4 h = pieces.enter(carry, shared, wave, lane16);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            h = as[i] * h + bs[i];
            if (t0 + i < a.T) ch.store(out + (t0 + i) * a.ot, from_f32<E>(t0 + i < length ? h : splat(0.0f)));
        }
        if (block == (length - 1) / kBlock && writes && a.last) store_state(a.last + (size_t)b * a.C, carry, ch);
    }
}

template <class E, bool kAligned, int kKind, int NW, bool kAhead>
__global__ void __launch_bounds__(64 * NW, NW / 2) recurrence_backward_kernel(Args a)
{
    constexpr int kBlock = 4 * kSteps * NW;
    constexpr bool kSmooth = kKind == ESRNN_RECURRENCE_SMOOTH;
    __shared__ f32x4 lds[2][2][NW][2][16];
    __shared__ f32x4 lds_ahead[kAhead ? 2 : 1][NW][2][16];
    const int lane16 = threadIdx.x & 15, row = (threadIdx.x >> 4) & 3, wave = threadIdx.x >> 6;
    const Place place = draw_place<kAhead>(a);
    const int b = place.line / a.tiles, tile = place.line % a.tiles;
    const Channels<kAligned, 16> ch(lane16, tile * kTile, a.C);
    const int length = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T, top = (length - 1) / kBlock;       // the last block with positions
    const E *x = static_cast<const E *>(a.x) + b * a.xb, *gate = static_cast<const E *>(a.gate) + b * a.gb;
    const E *grad_out = static_cast<const E *>(a.grad_out) + b * a.db;
    E *grad_x = static_cast<E *>(a.grad_x) + b * a.gxb, *grad_gate = static_cast<E *>(a.grad_gate) + b * a.ggb;
    const bool writes = wave == 0 && row == 0;

    f32x4 carry = splat(0.0f);
    if (a.grad_last) carry = load_state(a.grad_last + (size_t)b * a.C, ch);
    const int last = kAhead ? a.blocks - 1 - place.block : a.blocks - 1, first = kAhead ? last : 0;
    for (int block = last; block >= first; --block) {
        const int t0 = block * kBlock + (wave * 4 + row) * kSteps;
        if (block * kBlock >= length) {
            for (int i = 0; i < kSteps; ++i)
                if (t0 + i < a.T) {
                    ch.store(grad_x + (t0 + i) * a.gxt, Vec4<E>{});
                    ch.store(grad_gate + (t0 + i) * a.ggt, Vec4<E>{});
                }
            if (block == 0 && writes && a.grad_initial) store_state(a.grad_initial + (size_t)b * a.C, carry, ch);
            continue;
        }
        Vec4<E> xs[kSteps], gs[kSteps], ds[kSteps];
        f32x4 before = load_state(a.saved_in + ((size_t)b * a.blocks + block) * a.C, ch);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const long long t = min(t0 + i, length - 1);
            gs[i] = ch.load(gate + t * a.gt);
            ds[i] = ch.load(grad_out + t * a.dt);
            xs[i] = ch.load(x + t * a.xt);
        }
        f32x4 as[kSteps], zs[kSteps], A = splat(1.0f), B = splat(0.0f), M = splat(0.0f);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            f32x4 add;
            maps_of<kKind>(to_f32<E>(gs[i]), to_f32<E>(xs[i]), t0 + i < length, as[i], zs[i], add);
            B = as[i] * B + add;
            A = as[i] * A;
        }
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i) M = as[i] * ((t0 + i < length ? to_f32<E>(ds[i]) : splat(0.0f)) + M);
        const Pieces<NW, true> back(A, M, row, lane16);
        auto &shared = lds[kAhead ? 0 : block & 1];
        // (the last wave first, as the maps against time follow each other)
        back.leave(shared[1], NW - 1 - wave, row, lane16);
        const Pieces<NW, false> forth(A, B, row, lane16);
        forth.leave(shared[0], wave, row, lane16);
        if (NW > 1) __syncthreads();
        if constexpr (kAhead)
            carry = line_of(a, place.line).template entering<NW>(top - block, Line::whole<NW>(shared[1], lane16), carry, a.log_group, lds_ahead, wave, row, lane16);
        f32x4 mu = back.enter(carry, shared[1], NW - 1 - wave, lane16);
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
        if (block == 0 && writes && a.grad_initial) store_state(a.grad_initial + (size_t)b * a.C, carry, ch);
    }
}

// Before a launch with kAhead: no ticket drawn, no map there.
__global__ void __launch_bounds__(256) recurrence_words_kernel(u32x4 *words, long long n)
{
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i < n) words[i] = i < 16 ? u32x4{0, 0, 0, 0} : u32x4{kEmpty, kEmpty, kEmpty, kEmpty};
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
    r.blocks = p.blocks, r.groups = p.groups, r.log_group = p.log_group;
    return r;
}

bool groups_of_four(const void *p, const int64_t stride[2], int dtype)
{
    return aligned_to(p, 4 * element_bytes(dtype)) && (stride[0] | stride[1]) % 4 == 0;
}

}  // namespace

RecurrencePlan recurrence_plan(const esrnn_recurrence_shape &s)
{
    RecurrencePlan p{};
    p.waves = s.T <= 64 ? 1 : 4;
    p.block = 4 * kSteps * p.waves;
    p.blocks = (s.T + p.block - 1) / p.block;
    const long long lines = (long long)s.B * ((s.C + kTile - 1) / kTile);
    p.ahead = p.waves == 4 && p.blocks > 1 && lines < kLinesAlone && lines * p.blocks <= (1 << 21);
    if (p.ahead) {
        for (p.log_group = 4; 1LL << 2 * p.log_group < p.blocks; ++p.log_group) {}
        p.groups = p.blocks >> p.log_group;
        p.words = 64 + (size_t)lines * (p.blocks + p.groups) * kMap;
    }
    return p;
}

namespace {

// f(kAhead) behind the clearing of the words
template <class F>
hipError_t with_words(const RecurrencePlan &p, float *words, hipStream_t st, F &&f)
{
    if (!p.ahead) return f(std::false_type{});
    recurrence_words_kernel<<<(unsigned)((p.words / 4 + 255) / 256), 256, 0, st>>>(reinterpret_cast<u32x4 *>(words), (long long)(p.words / 4));
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? f(std::true_type{}) : e;
}

}  // namespace

hipError_t launch_recurrence_forward(const esrnn_recurrence_shape &s, const RecurrenceForward &f, hipStream_t st)
{
    const RecurrencePlan p = recurrence_plan(s);
    Args a = args_of(s, p);
    a.x = f.x, a.gate = f.gate, a.out = f.out, a.lengths = f.lengths, a.initial = f.initial, a.last = f.last, a.saved = f.saved, a.words = f.words;
    const bool aligned = s.C % 4 == 0 && groups_of_four(f.x, s.x_stride, s.dtype) && groups_of_four(f.gate, s.gate_stride, s.dtype) &&
                         groups_of_four(f.out, s.out_stride, s.dtype);
    return with_words(p, f.words, st, [&](auto ahead) {
        return with_element(s.dtype, [&](auto e) {
            using E = decltype(e);
            with_variant(aligned, s.kind, [&](auto al, auto kind) {
                const unsigned lines = (unsigned)(s.B * a.tiles);
                if constexpr (ahead()) recurrence_forward_kernel<E, al(), kind(), 4, true><<<lines * p.blocks, 256, 0, st>>>(a);
                else if (p.waves == 1) recurrence_forward_kernel<E, al(), kind(), 1, false><<<lines, 64, 0, st>>>(a);
                else recurrence_forward_kernel<E, al(), kind(), 4, false><<<lines, 256, 0, st>>>(a);
            });
            return hipGetLastError();
        });
    });
}

hipError_t launch_recurrence_backward(const esrnn_recurrence_shape &s, const RecurrenceBackward &f, hipStream_t st)
{
    const RecurrencePlan p = recurrence_plan(s);
    Args a = args_of(s, p);
    a.x = f.x, a.gate = f.gate, a.grad_out = f.grad_out, a.grad_x = f.grad_x, a.grad_gate = f.grad_gate, a.lengths = f.lengths;
    a.saved_in = f.saved, a.grad_last = f.grad_last, a.grad_initial = f.grad_initial, a.words = f.words;
    const bool aligned = s.C % 4 == 0 && groups_of_four(f.x, s.x_stride, s.dtype) && groups_of_four(f.gate, s.gate_stride, s.dtype) &&
                         groups_of_four(f.grad_out, s.grad_out_stride, s.dtype) && groups_of_four(f.grad_x, s.grad_x_stride, s.dtype) &&
                         groups_of_four(f.grad_gate, s.grad_gate_stride, s.dtype);
    return with_words(p, f.words, st, [&](auto ahead) {
        return with_element(s.dtype, [&](auto e) {
            using E = decltype(e);
            with_variant(aligned, s.kind, [&](auto al, auto kind) {
                const unsigned lines = (unsigned)(s.B * a.tiles);
                if constexpr (ahead()) recurrence_backward_kernel<E, al(), kind(), 4, true><<<lines * p.blocks, 256, 0, st>>>(a);
                else if (p.waves == 1) recurrence_backward_kernel<E, al(), kind(), 1, false><<<lines, 64, 0, st>>>(a);
                else recurrence_backward_kernel<E, al(), kind(), 4, false><<<lines, 256, 0, st>>>(a);
            });
            return hipGetLastError();
        });
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
