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
// the maps of the blocks before it, which are under way at the same time.
//
// The reverse pass runs the same maps from the end: mu_t = a_t (d_t + mu_{t+1}), with d the gradient of out.  The states h_{t-1} that the
// gradient of the gate needs are computed again, in fp32, from the state before the block that the forward pass leaves: reading
// out instead would be one array more, and rounded to its element type.
//
// Every array is read once and written once, 3 arrays forward and 5 in reverse, so memory is the bound: in bf16, 8 sequences of 4096 positions
// and 2048 channels take 95 us forward and 162 us in reverse among other passes, 4.2 TB/s both (a copy reaches 5.1), and 102 and 165 us as single dispatches under
// the profiler.  Under the profiler too: 501 ragged sequences of up to 240 positions of 50 channels, fp32, 17 and 26 us; one sequence of 131072 positions of
// 256 channels 69 and 102 us behind 5 us each that clear the words below, 2.9 and 3.3 TB/s.  The vector ALU is busy for 40 % of the cycles.  Maps, states and
// their sums are fp32; out and the gradients are rounded once, to nearest, as they are stored.
#include <algorithm>

#include "layers_internal.h"

namespace esrnn {

namespace {

// Channels of a workgroup: 128 bytes of 16 bits, a whole cache line.  Lines of fewer leave lanes idle: 64 x 16384 x 16 bf16 takes 74 and 134 us for bytes
// that a copy moves in 20 and 33, 18 x 108288 x 33 192 and 316 for 76 and 126.
constexpr int kTile = 64;
// Lines (64 channels of a sequence) from which a workgroup takes a whole sequence.  Alone against ahead, bf16, forward and reverse: 8 x 4096 x 2048
// (256 lines) 96 and 160 us against 107 and 180, 240 lines of 2048 positions 39 and 73 against 41 and 79, of 512 12 and 20 against 15 and 24; 192 of
// 2048 37 and 60 against 35 and 55, of 512 11 and 18 against 12 and 21; 128 of 2048 35 and 51 against 27 and 40, 32 30 and 48 against 11 and 14.
constexpr int kLinesAlone = 192;

struct Args {
    const void *x, *gate, *grad_out;
    void *out, *grad_x, *grad_gate;
    long long xb, xt, gb, gt, ob, ot, db, dt, gxb, gxt, ggb, ggt;      // strides of a sequence and of a position
    const int32_t *lengths;
    const float *initial, *saved_in, *grad_last;
    float *last, *saved, *grad_initial;
    float *words;               // kAhead: the tickets of the lines (64 channels of a sequence), then for each line the maps of its blocks
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
    __device__ __forceinline__ Pieces(f32x4 a, f32x4 b, int row, int lane)
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
        const int end = (kReverse ? 0 : 48) + lane;
        wave_A = from_lane(a, end);
        wave_B = from_lane(b, end);
        A = kReverse ? shift_down(a, 16) : shift_up(a, 16);
        B = kReverse ? shift_down(b, 16) : shift_up(b, 16);
        if (row == (kReverse ? 3 : 0)) {
            A = splat(1.0f);
            B = splat(0.0f);
        }
    }
    __device__ __forceinline__ void leave(f32x4 (*lds)[2][16], int wave, int row, int lane) const
    {
        if (NW > 1 && row == 0) {
            lds[wave][0][lane] = wave_A;
            lds[wave][1][lane] = wave_B;
        }
    }
    // behind a barrier: `in` of this thread's piece; carry: in of the block, then out of it
    __device__ __forceinline__ f32x4 enter(f32x4 &carry, const f32x4 (*lds)[2][16], int wave, int lane) const
    {
        if (NW == 1) {
            const f32x4 in = A * carry + B;
            carry = wave_A * carry + wave_B;
            return in;
        }
        f32x4 h = carry, mine = carry;
#pragma unroll 2        // (all at once they would take the registers of the waves' maps)
        for (int w = 0; w < NW; ++w) {
            if (w == wave) mine = h;
            h = lds[w][0][lane] * h + lds[w][1][lane];
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
// others one behind the other at most, and reads some 3 sqrt(blocks) maps at most: sqrt(blocks) of groups, 2 sqrt(blocks) of blocks (up to 256 blocks, 31).
// Every wait ends: the blocks of a line are taken by ticket, in the order in which they follow each other, whoever waits waits for lower
// tickets of its line only, and a block's own map waits for nobody.  (A wait that goes on for seconds all the same, because calls overlap on one workspace, is given
// up, once for all this thread reads; its maps are NaN.)
constexpr unsigned kEmpty = 0xffffffffu;
constexpr int kMostLooks = 1 << 22, kMap = 128, kTicket = 64;       // floats of a map, and of a ticket's place

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
    // map i, which `m` has been read from, once it is there
    __device__ __forceinline__ Map wait(int i, Map m)
    {
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
        const auto index = [&](int j) { return j < groups_first ? blocks + j : block + j - groups_first; };
        asm volatile("" ::: "memory");
        for (int j = from; j < to; j += 2) {        // (two looks under way)
            const int second = min(j + 1, to - 1);
            const Map m0 = look(index(j)), m1 = look(index(second));
            m = wait(index(j), m0).after(m);
            if (j + 1 < to) m = wait(index(second), m1).after(m);
        }
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

// a, z = 1 - a and b of four channels.  Where there is no position, a gate that keeps everything (kNoGate) and x = 0 make it the map that
// changes nothing.
template <int kKind>
constexpr float kNoGate = kKind == ESRNN_RECURRENCE_SMOOTH ? -__builtin_inff() : __builtin_inff();
template <int kKind>
__device__ __forceinline__ void maps_of(f32x4 g, f32x4 x, f32x4 &a, f32x4 &z, f32x4 &b)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const Sigmoids s = sigmoids(g[k]);
        a[k] = kKind == ESRNN_RECURRENCE_SMOOTH ? s.of_minus : s.of;
        z[k] = kKind == ESRNN_RECURRENCE_SMOOTH ? s.of : s.of_minus;
    }
    b = kKind == ESRNN_RECURRENCE_SMOOTH ? z * x : x;
}

// How a call's channels are read, by the least aligned of its arrays:
//   kFast         groups of four elements at multiples of four bytes, blocks of less than 2 GiB: from scalar bases (Positions)
//   kFour alone   at least four channels: groups of four at the alignment of one element, 64-bit addresses
//   neither       one by one
// Scalar bases leave fewer registers to addresses, which workgroups of one or two waves need: 2048 x 100 x 64 bf16 forward 16 us with kFast, 19.5 with
// kFour alone, 4096 x 30 x 64 9.9 and 10.7; 8 x 4096 x 2048 95 and 160 us forward and reverse with either.  kFour alone against one by one: 8 x 4096 x
// 2047 135 and 232 us against 168 and 256, 18 x 108288 x 33 192 and 316 against 244 and 407.
enum Access { kOneByOne, kByFours, kByFoursFast };

// Four neighbouring channels of a line for each of sixteen lanes; the last lane with channels has the last four there are, so that two lanes may
// have the same channel.  kFour: C is 4 at least.
template <bool kFour>
struct LineChannels {
    int first, count;
    __device__ __forceinline__ LineChannels(int lane, int begin, int C) : first(begin + 4 * lane), count(C)
    {
        if (kFour && first < C) first = min(first, C - 4);
    }
    __device__ __forceinline__ int channel(int k) const { return first + k; }
    __device__ __forceinline__ bool exists(int k) const { return channel(k) < count; }
    // a channel that can be read in the place of one that does not exist
    __device__ __forceinline__ int readable(int k) const { return kFour ? min(first, count - 4) + k : min(first + k, count - 1); }
    // (at the alignment of one element, which the hardware's global accesses allow)
    template <class E>
    __device__ __forceinline__ Vec4<E> load(const E *row) const
    {
        if constexpr (kFour) return *reinterpret_cast<const typename Loose<E>::Four *>(row + readable(0));
        Vec4<E> v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = row[readable(k)];
        return v;
    }
    template <class E>
    __device__ __forceinline__ void store(E *row, Vec4<E> v) const
    {
        if constexpr (kFour) {
            if (exists(0)) *reinterpret_cast<typename Loose<E>::Four *>(row + first) = v;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (exists(k)) row[channel(k)] = v[k];
        }
    }
};

// The kSteps positions of this thread in one array: four channels of position i.  kFast: the block begins at a scalar base, the thread's place in
// it never changes, position i is a scalar offset, and lanes without channels or positions lie outside the buffer, so that they
// read zeros and write nothing: no address is left to compute on the vector ALU, whose cycles the maps need.
template <class E, bool kFast, bool kFour>
struct Positions {
    E *base, *mine;         // of the block, and of this thread's first position
    long long stride;
    const LineChannels<kFour> &ch;
    __device__ __forceinline__ Positions(const E *b, long long s, int first, const LineChannels<kFour> &c)
        : base(const_cast<E *>(b)), mine(base + first * s), stride(s), ch(c)
    {
    }
    // What is not there is read from the block's first position, which is, and masked out.  (A mask that the compiler does not see through: of a
    // selection it makes a branch around the load, and then every load is waited for by itself.)
    __device__ __forceinline__ Vec4<E> load(int i, bool there) const
    {
        using Bits = unsigned __attribute__((ext_vector_type(sizeof(E))));
        unsigned mask = there ? 0xffffffffu : 0u;
        asm("" : "+v"(mask));
        return __builtin_bit_cast(Vec4<E>, __builtin_bit_cast(Bits, ch.load(there ? mine + i * stride : base)) & mask);
    }
    __device__ __forceinline__ void store(int i, bool there, Vec4<E> v) const
    {
        if (there) ch.store(mine + i * stride, v);
    }
};
template <class E>
struct Positions<E, true, true> {
    buf_rsrc rsrc;
    unsigned at, step;
    const LineChannels<true> &ch;
    // of one block: `base` is the block's first position, `first` this thread's in the block
    __device__ __forceinline__ Positions(const E *base, long long stride, int first, const LineChannels<true> &c)
        : rsrc(make_base(base)), at(c.exists(0) ? (first * (unsigned)stride + c.first) * sizeof(E) : kOutside),
          step((unsigned)stride * sizeof(E)), ch(c)
    {
    }
    __device__ __forceinline__ Vec4<E> load(int i, bool there) const
    {
        return load_four<E>(rsrc, there ? at : kOutside, i * step);
    }
    __device__ __forceinline__ void store(int i, bool there, Vec4<E> v) const
    {
        const unsigned to = there ? at : kOutside;
        // (four dwords: no scalar offset, see buf_store4)
        if constexpr (sizeof(E) == 4) buf_store4(rsrc, to == kOutside ? kOutside : to + i * step, v);
        else __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, v), rsrc, to, i * step, 0);
    }
};
// Channels of fp32 arrays [..][C] follow the dealing of the elements'.
template <bool kFour>
__device__ __forceinline__ f32x4 load_state(const float *p, const LineChannels<kFour> &ch)
{
    f32x4 v;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = p[ch.readable(k)];
    return v;
}
template <bool kFour>
__device__ __forceinline__ void store_state(float *p, f32x4 v, const LineChannels<kFour> &ch)
{
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (ch.exists(k)) p[ch.channel(k)] = v[k];
}


// What a workgroup works on: a line (64 channels of a sequence), and with kAhead one of its blocks, drawn by ticket.  Every line has a ticket
// of its own, in a cache line of its own: one for all of them is counted up once in 15 to 18 ns, which is what launches of thousands of
// workgroups then took (131072 positions of 256 channels: 76 us forward).
struct Place {
    int line, block;
};
template <bool kAhead>
__device__ __forceinline__ Place draw_place(const Args &a)
{
    if (!kAhead) return {(int)blockIdx.x, 0};
    __shared__ unsigned s_ticket;
    const unsigned line = blockIdx.x % (unsigned)(a.B * a.tiles);
    if (threadIdx.x == 0) s_ticket = atomicAdd(reinterpret_cast<unsigned *>(a.words) + kTicket * line, 1u);
    __syncthreads();
    // (in a workspace that another call writes, a ticket is any number: every place has to be in the launch)
    return {(int)line, (int)min((unsigned)__builtin_amdgcn_readfirstlane((int)s_ticket), (unsigned)a.blocks - 1)};
}
__device__ __forceinline__ Line line_of(const Args &a, int line)
{
    return Line(a.words + kTicket * (size_t)(a.B * a.tiles) + (size_t)line * (a.blocks + a.groups) * kMap, a.blocks, a.groups);
}

template <class E, bool kFast, int kKind, int kSteps, int NW, bool kAhead, bool kFour>
__global__ void __launch_bounds__(64 * NW, !kFour && NW < 8 ? 1 : NW == 8 || !kFast ? 2 : kAhead ? 3 : 4) recurrence_forward_kernel(Args a)
{
    constexpr int kBlock = 4 * kSteps * NW;
    __shared__ f32x4 lds[2][NW][2][16];
    __shared__ f32x4 lds_ahead[kAhead ? 2 : 1][NW][2][16];
    const int lane = threadIdx.x & 15, row = (threadIdx.x >> 4) & 3, wave = threadIdx.x >> 6;
    const Place place = draw_place<kAhead>(a);
    const int b = place.line / a.tiles;
    const LineChannels<kFour> ch(lane, place.line % a.tiles * kTile, a.C);
    const int length = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
    const E *x = static_cast<const E *>(a.x) + b * a.xb, *gate = static_cast<const E *>(a.gate) + b * a.gb;
    E *out = static_cast<E *>(a.out) + b * a.ob;
    const bool writes = wave == 0 && row == 0;

    f32x4 carry = splat(0.0f);
    if (a.initial) carry = load_state(a.initial + (size_t)b * a.C, ch);
    if (length == 0 && place.block == 0 && writes && a.last) store_state(a.last + (size_t)b * a.C, carry, ch);
    const int end = kAhead ? place.block + 1 : a.blocks;
    const int first = (wave * 4 + row) * kSteps;
    for (int block = place.block; block < end; ++block) {
        const int begin = block * kBlock, left = length - begin - first, rest = a.T - begin - first;      // positions from this thread's first on
        const Positions<E, kFast, kFour> to(out + begin * a.ot, a.ot, first, ch);
        if (begin >= length) {     // nothing left of the sequence
#pragma unroll
            for (int i = 0; i < kSteps; ++i) to.store(i, i < rest, Vec4<E>{});
            continue;
        }
        const Positions<E, kFast, kFour> of_x(x + begin * a.xt, a.xt, first, ch), of_gate(gate + begin * a.gt, a.gt, first, ch);
        Vec4<E> xs[kSteps], gs[kSteps];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            xs[i] = of_x.load(i, i < left);
            gs[i] = of_gate.load(i, i < left);
        }
        f32x4 as[kSteps], bs[kSteps], A = splat(1.0f), B = splat(0.0f);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            f32x4 z;
            maps_of<kKind>(to_f32<E>(i < left ? gs[i] : from_f32<E>(splat(kNoGate<kKind>))), to_f32<E>(xs[i]), as[i], z, bs[i]);
            B = as[i] * B + bs[i];
            A = as[i] * A;
        }
        const Pieces<NW, false> pieces(A, B, row, lane);
        auto &shared = lds[kAhead ? 0 : block & 1];
        pieces.leave(shared, wave, row, lane);
        if (NW > 1) __syncthreads();
        if constexpr (kAhead)
            carry = line_of(a, place.line).template entering<NW>(block, Line::whole<NW>(shared, lane), carry, a.log_group, lds_ahead, wave, row, lane);
        if (a.saved && writes) store_state(a.saved + ((size_t)b * a.blocks + block) * a.C, carry, ch);
        f32x4 h = pieces.enter(carry, shared, wave, lane);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            h = as[i] * h + bs[i];
            to.store(i, i < rest, i < left ? from_f32<E>(h) : Vec4<E>{});
        }
        if (block == (length - 1) / kBlock && writes && a.last) store_state(a.last + (size_t)b * a.C, carry, ch);
    }
}

template <class E, bool kFast, int kKind, int kSteps, int NW, bool kAhead, bool kFour>
__global__ void __launch_bounds__(64 * NW, 2) recurrence_backward_kernel(Args a)
{
    constexpr int kBlock = 4 * kSteps * NW;
    constexpr bool kSmooth = kKind == ESRNN_RECURRENCE_SMOOTH;
    __shared__ f32x4 lds[2][2][NW][2][16];
    __shared__ f32x4 lds_ahead[kAhead ? 2 : 1][NW][2][16];
    const int lane = threadIdx.x & 15, row = (threadIdx.x >> 4) & 3, wave = threadIdx.x >> 6;
    const Place place = draw_place<kAhead>(a);
    const int b = place.line / a.tiles;
    const LineChannels<kFour> ch(lane, place.line % a.tiles * kTile, a.C);
    const int length = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T, top = (length - 1) / kBlock;       // the last block with positions
    const E *x = static_cast<const E *>(a.x) + b * a.xb, *gate = static_cast<const E *>(a.gate) + b * a.gb;
    const E *grad_out = static_cast<const E *>(a.grad_out) + b * a.db;
    E *grad_x = static_cast<E *>(a.grad_x) + b * a.gxb, *grad_gate = static_cast<E *>(a.grad_gate) + b * a.ggb;
    const bool writes = wave == 0 && row == 0;

    f32x4 carry = splat(0.0f);
    if (a.grad_last) carry = load_state(a.grad_last + (size_t)b * a.C, ch);
    const int last = kAhead ? a.blocks - 1 - place.block : a.blocks - 1, end = kAhead ? last : 0;
    const int first = (wave * 4 + row) * kSteps;
    for (int block = last; block >= end; --block) {
        const int begin = block * kBlock, left = length - begin - first, rest = a.T - begin - first;
        const Positions<E, kFast, kFour> to_x(grad_x + begin * a.gxt, a.gxt, first, ch), to_gate(grad_gate + begin * a.ggt, a.ggt, first, ch);
        if (begin >= length) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                to_x.store(i, i < rest, Vec4<E>{});
                to_gate.store(i, i < rest, Vec4<E>{});
            }
            if (block == 0 && writes && a.grad_initial) store_state(a.grad_initial + (size_t)b * a.C, carry, ch);
            continue;
        }
        const Positions<E, kFast, kFour> of_x(x + begin * a.xt, a.xt, first, ch), of_gate(gate + begin * a.gt, a.gt, first, ch),
            of_out(grad_out + begin * a.dt, a.dt, first, ch);
        Vec4<E> xs[kSteps], gs[kSteps], ds[kSteps];
        f32x4 before = load_state(a.saved_in + ((size_t)b * a.blocks + block) * a.C, ch);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            gs[i] = of_gate.load(i, i < left);
            ds[i] = of_out.load(i, i < left);
            xs[i] = of_x.load(i, i < left);
        }
        f32x4 as[kSteps], zs[kSteps], A = splat(1.0f), B = splat(0.0f), M = splat(0.0f);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            f32x4 add;
            maps_of<kKind>(to_f32<E>(i < left ? gs[i] : from_f32<E>(splat(kNoGate<kKind>))), to_f32<E>(xs[i]), as[i], zs[i], add);
            B = as[i] * B + add;
            A = as[i] * A;
        }
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i) M = as[i] * (to_f32<E>(ds[i]) + M);
        __builtin_amdgcn_sched_barrier(0);      // (or conversions move up from below, and with them registers)
        const Pieces<NW, true> back(A, M, row, lane);
        auto &shared = lds[kAhead ? 0 : block & 1];
        // (the last wave first, as the maps against time follow each other)
        back.leave(shared[1], NW - 1 - wave, row, lane);
        const Pieces<NW, false> forth(A, B, row, lane);
        forth.leave(shared[0], wave, row, lane);
        if (NW > 1) __syncthreads();
        if constexpr (kAhead)
            carry = line_of(a, place.line).template entering<NW>(top - block, Line::whole<NW>(shared[1], lane), carry, a.log_group, lds_ahead, wave, row, lane);
        f32x4 mu = back.enter(carry, shared[1], NW - 1 - wave, lane);
        f32x4 h = forth.enter(before, shared[0], wave, lane);
        f32x4 rate[kSteps];     // of the state that comes in, with the gate, but for a factor a
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const f32x4 xi = to_f32<E>(xs[i]);
            rate[i] = zs[i] * (kSmooth ? xi - h : h);
            h = as[i] * h + (kSmooth ? zs[i] * xi : xi);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i) {
            const f32x4 lambda = to_f32<E>(ds[i]) + mu;
            mu = as[i] * lambda;
            to_x.store(i, i < rest, i < left ? from_f32<E>(kSmooth ? zs[i] * lambda : lambda) : Vec4<E>{});
            to_gate.store(i, i < rest, i < left ? from_f32<E>(mu * rate[i]) : Vec4<E>{});
        }
        if (block == 0 && writes && a.grad_initial) store_state(a.grad_initial + (size_t)b * a.C, carry, ch);
    }
}

// Before a launch with kAhead: no ticket drawn, no map there.
__global__ void __launch_bounds__(256) recurrence_words_kernel(u32x4 *words, long long tickets, long long n)
{
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i < n) words[i] = i < tickets ? u32x4{0, 0, 0, 0} : u32x4{kEmpty, kEmpty, kEmpty, kEmpty};
}

// One position: a workgroup has 1024 neighbouring channels of a request.  Reads x, gate and the state, writes out and the state, nothing waits for
// anything else: 1024 requests of 2048 channels in bf16 are 29 MB, 5.8 us at the rate of a copy, and the call takes 7.1 us, 6.3 of which the host
// needs to make it; 7 requests of 240 channels take the same.
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
    maps_of<kKind>(g, x, keep, take, add);
    const f32x4 h = keep * ch.load(state) + add;
    ch.store(state, h);
    ch.store(out, from_f32<E>(h));
}

template <int v>
using Int = std::integral_constant<int, v>;

template <class F>
void with_kind(int kind, F &&f)
{
    if (kind == ESRNN_RECURRENCE_SMOOTH) f(Int<ESRNN_RECURRENCE_SMOOTH>{});
    else f(Int<ESRNN_RECURRENCE_DECAY>{});
}
template <class F>
void with_access(Access access, int kind, F &&f)
{
    with_kind(kind, [&](auto k) {
        switch (access) {
        case kOneByOne: return f(std::false_type{}, std::false_type{}, k);
        case kByFours: return f(std::false_type{}, std::true_type{}, k);
        default: return f(std::true_type{}, std::true_type{}, k);
        }
    });
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
Access access_of(const void *p, const int64_t stride[2], const esrnn_recurrence_shape &s, const RecurrencePlan &plan)
{
    const bool dwords = s.dtype == ESRNN_F32 || (aligned_to(p, 4) && (stride[0] | stride[1] | s.C) % 2 == 0);
    return s.C < 4 ? kOneByOne : dwords && plan.block * stride[1] + s.C < (int64_t(1) << 29) ? kByFoursFast : kByFours;
}

}  // namespace

RecurrencePlan recurrence_plan(const esrnn_recurrence_shape &s)
{
    RecurrencePlan p{};
    const long long lines = (long long)s.B * ((s.C + kTile - 1) / kTile);
    // Ahead from 257 positions on: up to 256 the second block costs less than clearing the words (32 lines of 256 positions 7 and 10 us against 8
    // and 10, of 512 9 and 14 against 8 and 10).  2^21 blocks: their maps are 1 GiB.
    p.ahead = s.T > 256 && lines < kLinesAlone && lines * ((s.T + 127) / 128) <= (1 << 21);
    // The block is the sequence where that is short; in long ones 8 waves have more bytes on their way, but short ones leave them idle.  Forward and
    // reverse, bf16: 16 lines of 72 positions 5.8 us forward with 2 waves, 4.7 with 4; 2048 x 100 x 64 (2048 lines) 18 and 31 with 2, 18 and 34 with 4,
    // 25 and 62 with 8; 501 x 240 x 50 fp32 16 and 26 with 4, 16 and 32 with 8; 128 x 512 x 1024 86 and 160 with 8, 95 and 154 with 4.
    // A thread has 8 positions, or 2 where 4 threads hold the sequence with that: 4096 x 8 x 512 40 and 87 us with 8, 19 and 30 with 2.
    p.waves = p.ahead ? 4 : s.T <= 32 ? 1 : s.T <= 64 || (s.T <= 128 && lines >= 1024) ? 2 : s.T <= 256 ? 4 : 8;
    p.steps = s.T <= 8 ? 2 : 8;
    p.block = 4 * p.steps * p.waves;
    p.blocks = (s.T + p.block - 1) / p.block;
    if (p.ahead) {
        for (p.log_group = 4; 1LL << 2 * p.log_group < p.blocks; ++p.log_group) {}
        p.groups = p.blocks >> p.log_group;
        p.tickets = (size_t)lines * kTicket;
        p.words = p.tickets + (size_t)lines * (p.blocks + p.groups) * kMap;
    }
    return p;
}

namespace {

// f(kAhead) behind the clearing of the words
template <class F>
hipError_t with_words(const RecurrencePlan &p, float *words, hipStream_t st, F &&f)
{
    if (!p.ahead) return f(std::false_type{});
    recurrence_words_kernel<<<(unsigned)((p.words / 4 + 255) / 256), 256, 0, st>>>(reinterpret_cast<u32x4 *>(words), (long long)(p.tickets / 4),
                                                                                   (long long)(p.words / 4));
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? f(std::true_type{}) : e;
}

}  // namespace

hipError_t launch_recurrence_forward(const esrnn_recurrence_shape &s, const RecurrenceForward &f, hipStream_t st)
{
    const RecurrencePlan p = recurrence_plan(s);
    Args a = args_of(s, p);
    a.x = f.x, a.gate = f.gate, a.out = f.out, a.lengths = f.lengths, a.initial = f.initial, a.last = f.last, a.saved = f.saved, a.words = f.words;
    const Access access = std::min({access_of(f.x, s.x_stride, s, p), access_of(f.gate, s.gate_stride, s, p), access_of(f.out, s.out_stride, s, p)});
    return with_words(p, f.words, st, [&](auto ahead) {
        return with_element(s.dtype, [&](auto e) {
            using E = decltype(e);
            with_access(access, s.kind, [&](auto fast, auto four, auto kind) {
                const unsigned lines = (unsigned)(s.B * a.tiles);
                const auto launch = [&](auto steps, auto waves) {
                    recurrence_forward_kernel<E, fast(), kind(), steps(), waves(), ahead(), four()><<<ahead() ? lines * p.blocks : lines, 64 * waves(), 0, st>>>(a);
                };
                if constexpr (ahead()) launch(Int<8>{}, Int<4>{});
                else if (p.steps == 2) launch(Int<2>{}, Int<1>{});
                else switch (p.waves) {
                case 1: return launch(Int<8>{}, Int<1>{});
                case 2: return launch(Int<8>{}, Int<2>{});
                case 4: return launch(Int<8>{}, Int<4>{});
                default: return launch(Int<8>{}, Int<8>{});
                }
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
    const Access access = std::min({access_of(f.x, s.x_stride, s, p), access_of(f.gate, s.gate_stride, s, p), access_of(f.grad_out, s.grad_out_stride, s, p),
                                    access_of(f.grad_x, s.grad_x_stride, s, p), access_of(f.grad_gate, s.grad_gate_stride, s, p)});
    return with_words(p, f.words, st, [&](auto ahead) {
        return with_element(s.dtype, [&](auto e) {
            using E = decltype(e);
            with_access(access, s.kind, [&](auto fast, auto four, auto kind) {
                const unsigned lines = (unsigned)(s.B * a.tiles);
                const auto launch = [&](auto steps, auto waves) {
                    recurrence_backward_kernel<E, fast(), kind(), steps(), waves(), ahead(), four()><<<ahead() ? lines * p.blocks : lines, 64 * waves(), 0, st>>>(a);
                };
                if constexpr (ahead()) launch(Int<8>{}, Int<4>{});
                else if (p.steps == 2) launch(Int<2>{}, Int<1>{});
                else switch (p.waves) {
                case 1: return launch(Int<8>{}, Int<1>{});
                case 2: return launch(Int<8>{}, Int<2>{});
                case 4: return launch(Int<8>{}, Int<4>{});
                default: return launch(Int<8>{}, Int<8>{});
                }
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
        with_kind(kind, [&](auto k) {
            if (aligned) recurrence_step_kernel<E, true, k()><<<(unsigned)(a.rows * tiles), 256, 0, st>>>(a, tiles);
            else recurrence_step_kernel<E, false, k()><<<(unsigned)(a.rows * tiles), 256, 0, st>>>(a, tiles);
        });
        return hipGetLastError();
    });
}

}  // namespace esrnn
