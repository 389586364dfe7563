// What the kernels of the selective scan (include/esrnn_state_space.h) share: how a sequence is cut up, the operands of a piece of eight
// positions, and where states lie in the workspace.
//
// A lane has one channel with its N states in registers (up to 16; a channel of more has two or four lanes of as many waves, the slices), so a
// wave has 64 channels, and what all of them share, b and c of a position, comes through the scalar cache into scalar registers: the vector
// ALU takes it from there in the instruction that needs it.  Nothing is summed over lanes but the gradients of b and c.
//
// A sequence is cut into segments, which are as many waves: with a_t = exp(d_t A) a segment's map is h -> exp(A sum d) h + (its own last state from
// zero), so a first launch leaves the last states and sums of d of all segments, and a second one has every segment put together the maps before its
// own (where these are many, a launch between the two does that for all of them), and then walk its positions again.  Sequences and channels that fill
// the chip need no segments, and no first launch.  Forward, where sequences are short or lines (64 channels of a sequence) many, a line is a workgroup, whose
// waves have neighbouring pieces, and maps go through LDS: one launch, and every position is read once.
//
// exp(d A) is the hardware's power of two of d (A log2 e).  In the place of positions past a length, and of channels that a tile lacks, the last one there is
// is read again, with d (and in the reverse pass the gradient of out) masked to zero where that matters: states rest behind a sequence, and what lies
// there is never read.
#pragma once

#include "state_space_internal.h"

namespace esrnn {

constexpr long long kCopyWorkgroups = 1 << 20;      // at most, of 256 threads, that copy b and c
constexpr int kPiece = 8;               // positions of a piece; the forward pass leaves the state before each for the reverse pass
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct SelectivePlan {
    int states, slices, padded;         // states of a lane, slices of a channel, and their product
    int tiles;                          // of 64 channels of a group
    int pieces, segments, span;         // of a sequence; pieces of a segment
    bool widened;                       // b and c, as far as the pass reads rows of them, are copied to fp32 rows of `padded` states first
    int copies;                         // of how many it does: both forward; in reverse the maps read those of c, and nothing else does
    bool carried;                       // the maps of segments are put together by a launch of their own
    int line_waves;                     // forward, a workgroup for a whole sequence of a tile's channels: its waves, or 0
    // floats of the workspace: maps of segments, widened b and c, both by pieces, partial gradients of b and c, of A, D and bias
    size_t maps, rows, arranged, part_rows, part_sums;
};
SelectivePlan selective_plan(const esrnn_selective_shape &s, bool reverse);

struct Scan {
    SelectiveArgs a;
    const void *b, *c;                  // of which the kernels read rows: as given, or widened (where they do)
    long long xb, xt, db, dt, ob, ot;   // strides of a sequence and of a position
    long long bb, bt, cb, ct, group;    // of rows of b and c, and of a group in both
    long long gb, gt, gxb, gxt, gdb, gdt;
    const void *arranged;               // in the reverse pass: b and c by pieces and fours of states, [..][8 positions][4 of b, 4 of c]
    float *maps, *part_rows, *part_sums;
    int B, T, C, N, G;
    bool softplus, carried;
    int group_channels, tiles, pieces, segments, span;
};
Scan scan_arguments(const esrnn_selective_shape &s, const SelectiveArgs &a, SelectivePlan &p);      // (sets p.widened)
// Puts the state that enters each segment (against time: the gradient behind it) in the place of its map.
hipError_t launch_selective_carry(const esrnn_selective_shape &s, const SelectivePlan &p, const Scan &k, bool reverse, hipStream_t st);
// Copies b and c, or c alone, to rows of fp32 where the kernels cannot read them as they are.
hipError_t launch_selective_widen(const esrnn_selective_shape &s, const SelectiveArgs &a, const SelectivePlan &p, const Scan &k, hipStream_t st);

// f(element type tag, type of b and c, states of a lane, slices)
template <class F>
hipError_t with_scan(const esrnn_selective_shape &s, const SelectivePlan &p, F &&f)
{
    const auto sized = [&](auto e, auto bc) {
        if (p.slices == 4) return f(e, bc, std::integral_constant<int, 16>{}, std::integral_constant<int, 4>{});
        if (p.slices == 2) return f(e, bc, std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{});
        if (p.states == 16) return f(e, bc, std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
        if (p.states == 8) return f(e, bc, std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
        return f(e, bc, std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{});
    };
    if (s.dtype == ESRNN_F32) return sized(float{}, float{});
    if (s.dtype == ESRNN_F16) return sized(_Float16{}, float{});
    return p.widened ? sized(__bf16{}, float{}) : sized(__bf16{}, __bf16{});
}

// What a wave works on: all the same in its lanes but `channel` and `lane_mask`.
struct ScanPlace {
    int slice, tile, group, segment, b, length;
    unsigned channel;                   // of the array; the last one of the group where the tile has none
    unsigned lane_mask;                 // zero there
    __device__ __forceinline__ ScanPlace(const Scan &k, int segments)
    {
        const int lane = threadIdx.x & 63;
        slice = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        unsigned rest = blockIdx.x;
        tile = rest % (unsigned)(k.G * k.tiles), rest /= (unsigned)(k.G * k.tiles);
        segment = rest % (unsigned)segments, b = rest / (unsigned)segments;
        group = tile / k.tiles;
        const int in_group = tile % k.tiles * 64 + lane;
        lane_mask = in_group < k.group_channels ? 0xffffffffu : 0u;
        asm("" : "+v"(lane_mask));
        channel = group * k.group_channels + min(in_group, k.group_channels - 1);
        length = k.a.lengths ? min(max(__builtin_amdgcn_readfirstlane(k.a.lengths[b]), 0), k.T) : k.T;
    }
};

__device__ __forceinline__ float masked(float v, unsigned mask) { return __builtin_bit_cast(float, __builtin_bit_cast(unsigned, v) & mask); }

// NP states of b or c at one position, the same in all lanes: scalar registers, through the scalar cache.
template <class T>
using Constant = const __attribute__((address_space(4))) T;
template <class BC, int NP>
__device__ __forceinline__ void load_shared(const BC *row, float (&v)[NP])
{
    if constexpr (sizeof(BC) == 4) {
        typedef float Whole __attribute__((ext_vector_type(NP), aligned(4)));
        const Whole w = *(Constant<Whole> *)(uintptr_t)row;
#pragma unroll
        for (int n = 0; n < NP; ++n) v[n] = w[n];
    } else {        // pairs of bf16: the upper halves of floats
        typedef unsigned Whole __attribute__((ext_vector_type(NP / 2), aligned(4)));
        const Whole w = *(Constant<Whole> *)(uintptr_t)row;
#pragma unroll
        for (int n = 0; n < NP; ++n) v[n] = __builtin_bit_cast(float, n & 1 ? w[n / 2] & 0xffff0000u : w[n / 2] << 16);
    }
}

// A number that is the same in all lanes, and that the compiler takes for a new one wherever this stands: addresses made from it are computed on
// the scalar unit when they are needed, and not carried along as dozens of pointers, which scalar registers do not hold.
__device__ __forceinline__ int fresh(int v)
{
    v = __builtin_amdgcn_readfirstlane(v);
    asm volatile("" : "+s"(v));
    return v;
}

// Values that are complete here: or the compiler moves the whole sums behind the condition under which they are stored, and with them everything
// that they are made of has to be kept.
template <int N>
__device__ __forceinline__ void complete(float (&v)[N], int from = 0, int count = N)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i >= from && i < from + count) asm volatile("" : "+v"(v[i]));
}

// Four states of b and c at the eight positions of a piece, [8][4 of b, 4 of c] in memory: few wide loads, as every wait for the scalar cache is one for all
// that is under way.
template <class BC>
struct PieceRows {
    static constexpr int kLoads = 4 * (int)sizeof(BC) / 4;
    typedef unsigned Whole __attribute__((ext_vector_type(16), aligned(4)));
    Whole w[kLoads];
    __device__ __forceinline__ explicit PieceRows(const BC *p)
    {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) w[i] = *(Constant<Whole> *)(uintptr_t)(p + i * (64 / sizeof(BC)));
    }
    // of position i, b (0) or c (1), state n
    __device__ __forceinline__ float get(int i, int which, int n) const
    {
        const int at = 8 * i + 4 * which + n;
        // (a copy first: the builtin takes an element of a vector for the vector's first)
        unsigned bits = sizeof(BC) == 4 ? w[at / 16][at % 16] : w[at / 32][at / 2 % 16];
        if (sizeof(BC) == 2) bits = at & 1 ? bits & 0xffff0000u : bits << 16;
        return __builtin_bit_cast(float, bits);
    }
};

// The elements of one channel at eight positions; behind the sequence's last one that one again.
template <class E>
struct Column {
    E v[kPiece];
    __device__ __forceinline__ void request(const E *base, long long stride, int from, int length, unsigned channel)
    {
        const int first = fresh(from), left = length - 1 - first;
        const E *p = base + first * stride;
#pragma unroll
        for (int i = 0; i < kPiece; ++i) v[i] = (p + min(i, left) * stride)[channel];
    }
};
// Row i of b or c behind `p`, which belongs to the first position of a piece.
template <class BC, int NP>
__device__ __forceinline__ void load_shared(const BC *p, long long stride, int i, int left, float (&v)[NP])
{
    load_shared<BC, NP>(p + min(i, left) * stride, v);
}

// Rows of states [NP / 4][64 lanes][4] in saved states and maps; a map's sum of d follows.
template <int NP>
__device__ __forceinline__ void store_states(float *at, const float (&h)[NP])
{
#pragma unroll
    for (int q = 0; q < NP / 4; ++q)
        *reinterpret_cast<f32x4 *>(at + 256 * q + 4 * (threadIdx.x & 63)) = f32x4{h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3]};
}
template <int NP>
__device__ __forceinline__ void load_states(const float *at, float (&h)[NP])
{
#pragma unroll
    for (int q = 0; q < NP / 4; ++q) {
        const f32x4 v = *reinterpret_cast<const f32x4 *>(at + 256 * q + 4 * (threadIdx.x & 63));
#pragma unroll
        for (int r = 0; r < 4; ++r) h[4 * q + r] = v[r];
    }
}
template <int NP>
constexpr int kMapFloats = (NP + 1) * 64;
template <int NP, int SL>
__device__ __forceinline__ float *map_of(const Scan &k, const ScanPlace &at, int segment)
{
    return k.maps + ((((size_t)at.b * k.segments + segment) * (k.G * k.tiles) + at.tile) * SL + at.slice) * kMapFloats<NP>;
}
template <int NP, int SL>
__device__ __forceinline__ float *saved_of(const Scan &k, const ScanPlace &at, int piece)
{
    return k.a.saved + ((((size_t)at.b * k.pieces + piece) * (k.G * k.tiles) + at.tile) * SL + at.slice) * (NP * 64);
}

// A log2 e, of which exp(d A) is the power of two with d.  An infinite rate of decay forgets everything in a step and nothing in one of size zero, which is
// what positions past a length are: so it is a finite one, which leaves nothing from a step of kLeastStep on (2^-256 is zero).
constexpr float kForgetsAll = -0x1p127f, kLeastStep = 0x1p-119f;
__device__ __forceinline__ float exponent_rate(float A)
{
    const float rate = A * kLog2e;
    return rate == -__builtin_inff() ? kForgetsAll : rate;
}

// This lane's states of arrays [..][C][N]; those that do not exist are zero.
template <int NP>
__device__ __forceinline__ void load_own(const float *of_channel, int slice, int N, unsigned lane_mask, float (&v)[NP])
{
#pragma unroll
    for (int n = 0; n < NP; ++n) v[n] = masked(of_channel[min(NP * slice + n, N - 1)], NP * slice + n < N ? lane_mask : 0u);
}
template <int NP>
__device__ __forceinline__ void store_own(float *of_channel, int slice, int N, unsigned lane_mask, const float (&v)[NP])
{
    if (!lane_mask) return;
#pragma unroll
    for (int n = 0; n < NP; ++n)
        if (NP * slice + n < N) of_channel[NP * slice + n] = v[n];
}

// The step size of a channel at one position, and its derivative.
template <class E>
__device__ __forceinline__ Softplus step_size(E delta, float bias, bool softplus_kind)
{
    const float v = (float)delta + bias;
    const Softplus s = softplus(v);
    return {softplus_kind ? s.of : v, softplus_kind ? s.slope : 1.0f};
}

}  // namespace esrnn
