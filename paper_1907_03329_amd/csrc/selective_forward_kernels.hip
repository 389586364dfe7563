// Selective scan over whole sequences, forward (include/esrnn_state_space.h; selective_scan.h has the way it is cut up):
//   h_t = exp(d_t A) h_{t-1} + d_t x_t b_t,  out_t = c_t . h_t + D x_t.
// A state costs a power of two, which takes the vector ALU as long as two other instructions, and four of these, where x, delta and out are six bytes for sixteen
// states: instructions are the bound, and no matrix instruction fits, for every channel has decays of its own.  4 x 4096 x 2048, 16 states, bf16, 103 segments:
// maps 110 us, of which the SIMDs issue vector instructions for 104, putting them together 24 (122 MB), outputs 153 (127 of instructions; 336 MB written, of them
// 268 states for the reverse pass).  1 x 65536 x 256: 160 us in all.  501 x 240 x 50 ragged fp32 in one launch: 67 us.
#include <algorithm>
#include <cmath>

#include "selective_scan.h"

namespace esrnn {

namespace {

constexpr int kThreadsOfRows = 256;

// kMaps: the map of a segment, which needs neither c nor the output.
template <class E, class BC, int NP, int SL, bool kMaps>
__global__ void __launch_bounds__(64 * SL) selective_forward_kernel(Scan k)
{
    __shared__ float s_y[SL > 1 && !kMaps ? 2 : 1][SL > 1 && !kMaps ? SL : 1][kPiece][64];
    const int segments = kMaps ? k.segments - 1 : k.segments;       // (nothing follows the last one)
    const ScanPlace at(k, segments);
    const int lane = threadIdx.x & 63;
    const int begin = at.segment * k.span * kPiece, end = min(begin + k.span * kPiece, k.T);
    const E *x = static_cast<const E *>(k.a.x) + at.b * k.xb, *delta = static_cast<const E *>(k.a.delta) + at.b * k.db;
    E *out = static_cast<E *>(k.a.out) + at.b * k.ob;
    const BC *b = static_cast<const BC *>(k.b) + at.b * k.bb + at.group * k.group + NP * at.slice;
    const BC *c = static_cast<const BC *>(k.c) + at.b * k.cb + at.group * k.group + NP * at.slice;
    const size_t own = ((size_t)at.b * k.C + at.channel) * k.N;

    float A[NP], h[NP];
    load_own<NP>(k.a.A + (size_t)at.channel * k.N, at.slice, k.N, at.lane_mask, A);
#pragma unroll
    for (int n = 0; n < NP; ++n) A[n] = exponent_rate(A[n]), h[n] = 0.0f;
    const float bias = k.a.bias ? k.a.bias[at.channel] : 0.0f, D = k.a.D ? k.a.D[at.channel] : 0.0f;
    if (!kMaps && k.carried && at.segment > 0) {
        if (begin < at.length) load_states<NP>(map_of<NP, SL>(k, at, at.segment), h);
    } else if (!kMaps && (begin < at.length || begin == 0)) {
        if (k.a.initial) load_own<NP>(k.a.initial + own, at.slice, k.N, at.lane_mask, h);
        for (int s = 0; s < at.segment; ++s) {
            const float *map = map_of<NP, SL>(k, at, s);
            float local[NP];
            load_states<NP>(map, local);
            const float sum = map[64 * NP + lane];
#pragma unroll
            for (int n = 0; n < NP; ++n) h[n] = fmaf(__builtin_amdgcn_exp2f(sum * A[n]), h[n], local[n]);
        }
    }
    float sum = 0.0f;
    Column<E> xs, ds, next_xs, next_ds;
    if (begin < at.length) {
        xs.request(x, k.xt, begin, at.length, at.channel);
        ds.request(delta, k.dt, begin, at.length, at.channel);
    }
    int turn = 0;
    for (int t0 = begin; t0 < min(end, at.length); t0 += kPiece, turn ^= 1) {
        next_xs.request(x, k.xt, t0 + kPiece, at.length, at.channel);
        next_ds.request(delta, k.dt, t0 + kPiece, at.length, at.channel);
        if (!kMaps && k.a.saved) store_states<NP>(saved_of<NP, SL>(k, at, t0 / kPiece), h);
        float y[kPiece];
        const int t = fresh(t0), left = at.length - 1 - t;
        const BC *b0 = b + t * k.bt, *c0 = c + t * k.ct;
#pragma unroll
        for (int i = 0; i < kPiece; ++i) {
            const float d = masked(step_size(ds.v[i], bias, k.softplus).of, i <= left ? 0xffffffffu : 0u), xi = (float)xs.v[i], u = d * xi;
            float bs[NP], cs[NP];
            load_shared<BC, NP>(b0, k.bt, i, left, bs);
            if (kMaps) {
                sum += d;
            } else {
                load_shared<BC, NP>(c0, k.ct, i, left, cs);
            }
            float part[4] = {at.slice == 0 ? D * xi : 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int n = 0; n < NP; ++n) {
                h[n] = fmaf(__builtin_amdgcn_exp2f(d * A[n]), h[n], u * bs[n]);
                if (!kMaps) part[n & 3] = fmaf(cs[n], h[n], part[n & 3]);
            }
            y[i] = (part[0] + part[1]) + (part[2] + part[3]);
        }
        if constexpr (!kMaps) {
            complete(y);
            if constexpr (SL > 1) {
#pragma unroll
                for (int i = 0; i < kPiece; ++i) s_y[turn][at.slice][i][lane] = y[i];
                lds_barrier();      // (requests for the next piece go on)
#pragma unroll
                for (int i = 0; i < kPiece; ++i)
                    if (i % SL == at.slice) {
                        y[i] = 0.0f;
#pragma unroll
                        for (int s = 0; s < SL; ++s) y[i] += s_y[turn][s][i][lane];
                    }
            }
#pragma unroll
            for (int i = 0; i < kPiece; ++i)
                if (t + i < end && i % SL == at.slice && at.lane_mask) (out + (t + i) * k.ot)[at.channel] = (E)(i <= left ? y[i] : 0.0f);
        }
        xs = next_xs, ds = next_ds;
    }
    if constexpr (kMaps) {
        float *map = map_of<NP, SL>(k, at, at.segment);
        store_states<NP>(map, h);
        map[64 * NP + lane] = sum;
    } else {
        // positions past the length, from the first piece that has none of the sequence on
        for (int t = max(begin, (at.length + kPiece - 1) / kPiece * kPiece); t < end; ++t)
            if (t % SL == at.slice && at.lane_mask) (out + t * k.ot)[at.channel] = (E)0.0f;
        const int last_segment = max(at.length - 1, 0) / (k.span * kPiece);
        if (k.a.last && at.segment == last_segment) store_own<NP>(k.a.last + own, at.slice, k.N, at.lane_mask, h);
    }
}

// A workgroup for a whole line: its waves have neighbouring pieces, whose step sizes stay in registers while the maps of all of them are put together through
// LDS, four states by each of the first waves, who keep what enters the next block of pieces.
template <class E, class BC, int NP, int kWaves>
__global__ void __launch_bounds__(64 * kWaves) selective_line_kernel(Scan k)
{
    __shared__ f32x4 s_local[kWaves][NP / 4][64];
    __shared__ float s_sum[kWaves][64];
    ScanPlace at(k, 1);
    const int lane = threadIdx.x & 63, wave = at.slice, waves = blockDim.x >> 6;
    at.slice = 0;
    const E *x = static_cast<const E *>(k.a.x) + at.b * k.xb, *delta = static_cast<const E *>(k.a.delta) + at.b * k.db;
    E *out = static_cast<E *>(k.a.out) + at.b * k.ob;
    const BC *b = static_cast<const BC *>(k.b) + at.b * k.bb + at.group * k.group, *c = static_cast<const BC *>(k.c) + at.b * k.cb + at.group * k.group;
    const size_t own = ((size_t)at.b * k.C + at.channel) * k.N;
    const bool composes = wave < NP / 4;

    float A[NP];
    load_own<NP>(k.a.A + (size_t)at.channel * k.N, 0, k.N, at.lane_mask, A);
#pragma unroll
    for (int n = 0; n < NP; ++n) A[n] = exponent_rate(A[n]);
    f32x4 rates = {}, carry = {};       // of states 4 wave ..
    if (composes)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int n = 4 * wave + r;
            const unsigned mask = n < k.N ? at.lane_mask : 0u;
            rates[r] = exponent_rate(masked(k.a.A[(size_t)at.channel * k.N + min(n, k.N - 1)], mask));
            if (k.a.initial) carry[r] = masked(k.a.initial[own + min(n, k.N - 1)], mask);
        }
    const float bias = k.a.bias ? k.a.bias[at.channel] : 0.0f, D = k.a.D ? k.a.D[at.channel] : 0.0f;
    for (int block = 0; block < at.length; block += waves * kPiece) {
        const int t = fresh(block + wave * kPiece), left = at.length - 1 - t;
        const bool active = left >= 0;
        const BC *b0 = b + t * k.bt, *c0 = c + t * k.ct;
        float d[kPiece], u[kPiece], y[kPiece], h[NP], sum = 0.0f;
#pragma unroll
        for (int n = 0; n < NP; ++n) h[n] = 0.0f;
        if (active) {
            Column<E> xs, ds;
            xs.request(x, k.xt, t, at.length, at.channel);
            ds.request(delta, k.dt, t, at.length, at.channel);
#pragma unroll
            for (int i = 0; i < kPiece; ++i) {
                const float xi = (float)xs.v[i];
                d[i] = masked(step_size(ds.v[i], bias, k.softplus).of, i <= left ? 0xffffffffu : 0u), u[i] = d[i] * xi, y[i] = D * xi;
                sum += d[i];
                float bs[NP];
                load_shared<BC, NP>(b0, k.bt, i, left, bs);
#pragma unroll
                for (int n = 0; n < NP; ++n) h[n] = fmaf(__builtin_amdgcn_exp2f(d[i] * A[n]), h[n], u[i] * bs[n]);
            }
        }
#pragma unroll
        for (int q = 0; q < NP / 4; ++q) s_local[wave][q][lane] = f32x4{h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3]};
        s_sum[wave][lane] = sum;
        lds_barrier();
        if (composes) {
#pragma unroll 4
            for (int w = 0; w < waves; ++w) {
                const f32x4 local = s_local[w][wave][lane];
                const float total = s_sum[w][lane];
                s_local[w][wave][lane] = carry;
#pragma unroll
                for (int r = 0; r < 4; ++r) carry[r] = fmaf(__builtin_amdgcn_exp2f(total * rates[r]), carry[r], local[r]);
            }
        }
        lds_barrier();
        if (!active) continue;
#pragma unroll
        for (int q = 0; q < NP / 4; ++q) {
            const f32x4 entering = s_local[wave][q][lane];
#pragma unroll
            for (int r = 0; r < 4; ++r) h[4 * q + r] = entering[r];
        }
        if (k.a.saved) store_states<NP>(saved_of<NP, 1>(k, at, t / kPiece), h);
#pragma unroll
        for (int i = 0; i < kPiece; ++i) {
            float bs[NP], cs[NP];
            load_shared<BC, NP>(b0, k.bt, i, left, bs);
            load_shared<BC, NP>(c0, k.ct, i, left, cs);
            float part[4] = {y[i], 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int n = 0; n < NP; ++n) {
                h[n] = fmaf(__builtin_amdgcn_exp2f(d[i] * A[n]), h[n], u[i] * bs[n]);
                part[n & 3] = fmaf(cs[n], h[n], part[n & 3]);
            }
            y[i] = (part[0] + part[1]) + (part[2] + part[3]);
        }
        complete(y);
#pragma unroll
        for (int i = 0; i < kPiece; ++i)
            if (t + i < k.T && at.lane_mask) (out + (t + i) * k.ot)[at.channel] = (E)(i <= left ? y[i] : 0.0f);
    }
    for (int t = (at.length + kPiece - 1) / kPiece * kPiece + wave; t < k.T; t += waves)
        if (at.lane_mask) (out + t * k.ot)[at.channel] = (E)0.0f;
    if (k.a.last && composes && at.lane_mask)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (4 * wave + r < k.N) k.a.last[own + 4 * wave + r] = carry[r];
}

// A lane has a run of neighbouring segments, in their order or against it, and four states of a channel: first the run's own map, then, behind those of the
// runs before it, what enters each of its segments.  A workgroup has kColumns channels, 64 and 16 runs or, where segments are many, 8 and 128 runs: maps stay
// in registers between the two where a run has no more than kBatch.  That is the rule between both, for it is reads that bound this: 1 x 65536 x 256, 1024
// segments, whole forward pass 202 us with 64 channels, of which one compute unit reads the maps of 64 channels for four states, and 160 with 8; 4 x 4096 x 2048,
// 86 segments, 275 and 363, as every read is an eighth of a row.
constexpr int kCarryWaves = 16, kBatch = 8, kFewColumns = 8;
template <int NP, int SL, int kColumns>
__global__ void __launch_bounds__(64 * kCarryWaves) selective_carry_kernel(Scan k, int reverse)
{
    constexpr int kWaveRuns = 64 / kColumns, kRuns = kCarryWaves * kWaveRuns;
    __shared__ __attribute__((aligned(16))) f32x4 s_local[kCarryWaves][kColumns];
    __shared__ float s_sum[kCarryWaves][kColumns];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int column = lane % kColumns, wave_run = lane / kColumns, run = wave * kWaveRuns + wave_run;
    unsigned rest = blockIdx.x;
    const int in_tile = rest % kWaveRuns * kColumns + column;
    rest /= kWaveRuns;
    const int quad = rest % (NP / 4), slice = rest / (NP / 4) % SL;
    const unsigned line = rest / (NP / 4 * SL);
    const int tiles = k.G * k.tiles, tile = line % tiles, b = line / tiles;
    const int in_group = tile % k.tiles * 64 + in_tile, channel = tile / k.tiles * k.group_channels + min(in_group, k.group_channels - 1);
    const unsigned lane_mask = in_group < k.group_channels ? 0xffffffffu : 0u;
    const int length = k.a.lengths ? min(max(__builtin_amdgcn_readfirstlane(k.a.lengths[b]), 0), k.T) : k.T;
    const int last_segment = max(length - 1, 0) / (k.span * kPiece);
    const int each = (k.segments + kRuns - 1) / kRuns, from = min(run * each, k.segments), to = min(from + each, k.segments);
    // the place of number p, and whether it has a map: none comes in behind the last segment with positions, or from the last of all in their order
    const auto segment = [&](int p) { return reverse ? k.segments - 1 - p : p; };
    const auto has_map = [&](int p) { return p < k.segments - 1 && segment(p) <= last_segment; };
    const auto place = [&](int p) { return k.maps + ((((size_t)b * k.segments + segment(p)) * tiles + tile) * SL + slice) * kMapFloats<NP>; };
    float A[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int n = NP * slice + 4 * quad + r;
        A[r] = exponent_rate(masked(k.a.A[(size_t)channel * k.N + min(n, k.N - 1)], n < k.N ? lane_mask : 0u));
    }
    const auto apply = [&](f32x4 h, f32x4 local, float sum) {
#pragma unroll
        for (int r = 0; r < 4; ++r) h[r] = fmaf(__builtin_amdgcn_exp2f(sum * A[r]), h[r], local[r]);
        return h;
    };
    // kBatch maps from number p on; those that a run has not are the map that changes nothing
    f32x4 local[kBatch];
    float sum[kBatch];
    const auto read = [&](int p) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const float *map = place(min(p + i, k.segments - 1));
            local[i] = *reinterpret_cast<const f32x4 *>(map + 256 * quad + 4 * in_tile), sum[i] = map[64 * NP + in_tile];
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const unsigned mask = p + i < to && has_map(p + i) ? 0xffffffffu : 0u;
            sum[i] = masked(sum[i], mask);
#pragma unroll
            for (int r = 0; r < 4; ++r) local[i][r] = masked(local[i][r], mask);
        }
    };
    f32x4 h = {};
    float total = 0.0f;
    for (int p = 0; p < each; p += kBatch) {
        read(from + p);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) h = apply(h, local[i], sum[i]), total += sum[i];
    }
    // the runs of a wave: each one's map behind those before it, and then only those before it
    const auto from_before = [&](float v, int off) {
        const float other = __shfl_up(v, off, 64);      // (of all lanes, so outside the condition)
        return masked(other, lane >= off ? 0xffffffffu : 0u);
    };
#pragma unroll
    for (int off = kColumns; off < 64; off *= 2) {
        f32x4 before;
#pragma unroll
        for (int r = 0; r < 4; ++r) before[r] = from_before(h[r], off);
        const float sum_before = from_before(total, off);
        h = apply(before, h, total), total += sum_before;
    }
    if (wave_run == kWaveRuns - 1) s_local[wave][column] = h, s_sum[wave][column] = total;
    f32x4 in_wave = {};
    float sum_in_wave = 0.0f;
    if constexpr (kWaveRuns > 1) {
#pragma unroll
        for (int r = 0; r < 4; ++r) in_wave[r] = from_before(h[r], kColumns);
        sum_in_wave = from_before(total, kColumns);
    }
    __syncthreads();
    const float *first = reverse ? k.a.grad_last : k.a.initial;
    h = f32x4{};
    if (first)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int n = NP * slice + 4 * quad + r;
            h[r] = masked(first[((size_t)b * k.C + channel) * k.N + min(n, k.N - 1)], n < k.N ? lane_mask : 0u);
        }
    for (int r = 0; r < wave; ++r) h = apply(h, s_local[r][column], s_sum[r][column]);
    if constexpr (kWaveRuns > 1) h = apply(h, in_wave, sum_in_wave);
    for (int p = 0; p < each; p += kBatch) {
        if (each > kBatch) read(from + p);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            if (from + p + i < to) *reinterpret_cast<f32x4 *>(place(from + p + i) + 256 * quad + 4 * in_tile) = h;
            h = apply(h, local[i], sum[i]);
        }
    }
}

// b and c, or c alone, in rows of `padded` fp32 states, zeros behind the N there are: [copies][B][T][G][padded].
template <class E>
__global__ void __launch_bounds__(kThreadsOfRows) selective_widen_kernel(const E *b, const E *c, long long bb, long long bt, long long cb, long long ct, int copies,
                                                                         int B, int T, int G, int N, int padded, float *rows)
{
    const long long half = (long long)B * T * G * padded, first_of_c = (copies - 1) * half;
    for (long long i = (long long)blockIdx.x * kThreadsOfRows + threadIdx.x; i < copies * half; i += (long long)gridDim.x * kThreadsOfRows) {
        const bool second = i >= first_of_c;
        long long rest = second ? i - first_of_c : i;
        const int n = rest % padded;
        rest /= padded;
        const int g = rest % G;
        rest /= G;
        const int t = rest % T, s = rest / T;
        const E *from = second ? c + s * cb + t * ct : b + s * bb + t * bt;
        rows[i] = n < N ? (float)from[(long long)g * N + n] : 0.0f;
    }
}

}  // namespace

// From how many segments on their maps are put together by a launch of their own, and not by every wave (0.08 us for each).
constexpr int kSegmentsAlone = 32, kReadOnce = 64 / kFewColumns * kCarryWaves * kBatch;

// How many segments a sequence is cut into, by what its launches take in microseconds, fitted to what they took (14 shapes, 1 to 1024 segments): a piece takes
// what one wave needs for it and what the other waves of its SIMD need, a wave something to begin with, and a share of the maps before its own; the reverse
// kernel, of which a SIMD holds two waves, takes whole rounds of them, one wave little less than two, and leaves sums for every wave.  Measured in us, * what this takes:
//   4 x 4096 x 2048 bf16, 16 states    forward 371 with 16 segments, 291 with 32, 275 with 86 and with 103*; reverse 543 with 16, 510 with 32, 499 with 64*
//   1 x 65536 x 256 bf16, 16 states    forward 185 with 512, 160 with 1024, 164 with 2048*; reverse 315 with 512, 294 with 1024*, 323 with 1280
//   1 x 3000 x 256 bf16, 16 states     forward 43 with 96, 33 with 188*, 35 with 375; reverse 78 with 96, 59 with 188*, 53 with 375
//   240 x 122 x 240 bf16, 16 states    reverse 188 with 1, 157 with 2*, 179 with 8
//   4 x 4096 x 1024 bf16, 32 states    reverse 513 with 16, 578 with 32, 506 with 47, 527 with 64*
static int best_segments(long long lines, int pieces, bool reverse, double &least)
{
    int best = 1;
    least = 1e30;
    for (int segments = 1; segments <= pieces && (segments == 1 || lines * segments <= 16384); segments += std::max(1, segments / 32)) {
        const int span = (pieces + segments - 1) / segments, cut = (pieces + span - 1) / span;
        const double waves = lines * (double)cut / 1024.0, maps = waves * (cut - 1) / cut;      // of a SIMD
        const double rounds = std::floor(waves / 2), rest = waves - 2 * rounds, share = cut > kSegmentsAlone ? 0.0 : 0.08 * cut;
        double time = reverse ? (rounds + (rest > 1 ? 1.0 : rest > 0 ? 0.9 : 0.0)) * (11.5 * span + 3.0 + share) + 1.1 * waves
                              : 2.8 * span + waves * (1.9 * span + 1.2 + share);
        if (cut > 1) time += (reverse ? 2.0 : 2.2) * span + maps * (span * 1.5 + 1.2) + 4.0;
        if (cut > kSegmentsAlone) time += (reverse ? 4.0 : 8.0) * ((cut + kReadOnce - 1) / kReadOnce);
        if (time < least) least = time, best = segments;
    }
    return best;
}

constexpr int kLineWaves = 16;          // of a workgroup for a whole line

SelectivePlan selective_plan(const esrnn_selective_shape &s, bool reverse)
{
    SelectivePlan p{};
    p.states = s.N <= 4 ? 4 : s.N <= 8 ? 8 : 16;
    p.slices = s.N <= 16 ? 1 : s.N <= 32 ? 2 : 4;
    p.padded = p.states * p.slices;
    p.tiles = (s.C / s.G + 63) / 64;
    p.pieces = (s.T + kPiece - 1) / kPiece;
    const long long lines = (long long)s.B * s.G * p.tiles * p.slices;
    double cut;
    p.segments = best_segments(lines, p.pieces, reverse, cut);
    // A workgroup a line, in the same terms: 16 waves where every line has a compute unit of its own, else 8, two workgroups a compute unit.  In us, forward, cut /
    // 16 waves / 8 waves: 8 x 1024 x 2048 bf16 (256 lines) 151, 122, 150; 501 x 240 x 50 ragged fp32 88, 75, 66; 200 x 72 x 40 fp32 32, 17, 17; 16 x 72 x 40 17,
    // 16, 17; 2000 x 72 x 40 74, 118, 108; 4 x 300 x 256 bf16 (16 lines) 26, 42, 47.
    p.line_waves = 0;
    if (!reverse && p.slices == 1) {
        const int most = lines <= 256 ? kLineWaves : kLineWaves / 2, blocks = (p.pieces + most - 1) / most;
        const int waves = std::max((p.pieces + blocks - 1) / blocks, p.states / 4);
        const double rounds = std::ceil(std::ceil(lines / 256.0) / 2);
        const double line = lines <= 256 ? std::max(0.8 * p.pieces, 6.0 * blocks) : rounds * blocks * (1.6 * waves + 2.0);
        if (line < cut) p.line_waves = waves, p.segments = 1;
    }
    p.span = (p.pieces + p.segments - 1) / p.segments;
    p.segments = (p.pieces + p.span - 1) / p.span;
    p.carried = p.segments > kSegmentsAlone;
    const size_t tiles = (size_t)s.G * p.tiles;
    p.maps = p.segments > 1 ? (size_t)s.B * p.segments * tiles * p.slices * (p.states + 1) * 64 : 0;
    p.copies = !reverse ? 2 : p.segments > 1 ? 1 : 0;
    p.rows = p.copies * (size_t)s.B * s.T * s.G * p.padded;
    if (reverse) {
        p.arranged = (size_t)s.B * p.pieces * s.G * p.padded / 4 * 64;      // (or half of it in bf16)
        p.part_rows = (size_t)p.tiles * s.B * p.pieces * kPiece * s.G * 2 * p.padded;
        p.part_sums = (size_t)s.B * p.segments * tiles * p.slices * (p.states + 2) * 64;
    }
    return p;
}

size_t selective_workspace_floats(const esrnn_selective_shape &s, bool reverse)
{
    // (the two passes cut sequences in ways of their own)
    const auto floats = [&](bool which) {
        const SelectivePlan p = selective_plan(s, which);
        return 64 + p.maps + p.rows + p.arranged + p.part_rows + p.part_sums;
    };
    return reverse ? std::max(floats(false), floats(true)) : floats(false);
}
size_t selective_saved_floats(const esrnn_selective_shape &s)
{
    const SelectivePlan p = selective_plan(s, false);
    return (size_t)s.B * p.pieces * s.G * p.tiles * p.padded * 64;
}

// Rows of b and c that the kernels read as they are: whole groups of states, at multiples of four bytes.  (fp16 is no upper half of a float.)
static bool shared_as_given(const esrnn_selective_shape &s, const SelectivePlan &p, const void *row, const int64_t stride[2])
{
    if (s.N != p.padded || s.dtype == ESRNN_F16) return false;
    return s.dtype == ESRNN_F32 || (aligned_to(row, 4) && stride[0] % 2 == 0 && stride[1] % 2 == 0);
}

Scan scan_arguments(const esrnn_selective_shape &s, const SelectiveArgs &a, SelectivePlan &p)
{
    Scan k{};
    k.a = a;
    k.xb = s.x_stride[0], k.xt = s.x_stride[1], k.db = s.delta_stride[0], k.dt = s.delta_stride[1], k.ob = s.out_stride[0], k.ot = s.out_stride[1];
    k.gb = s.grad_out_stride[0], k.gt = s.grad_out_stride[1], k.gxb = s.grad_x_stride[0], k.gxt = s.grad_x_stride[1];
    k.gdb = s.grad_delta_stride[0], k.gdt = s.grad_delta_stride[1];
    k.B = s.B, k.T = s.T, k.C = s.C, k.N = s.N, k.G = s.G, k.softplus = s.delta_kind == ESRNN_DELTA_SOFTPLUS;
    k.group_channels = s.C / s.G, k.tiles = p.tiles, k.pieces = p.pieces, k.segments = p.segments, k.span = p.span, k.carried = p.carried;
    k.maps = a.workspace;
    float *rows = a.workspace + p.maps;
    k.arranged = rows + p.rows, k.part_rows = rows + p.rows + p.arranged, k.part_sums = k.part_rows + p.part_rows;
    p.widened = !(shared_as_given(s, p, a.b, s.b_stride) && shared_as_given(s, p, a.c, s.c_stride));
    if (p.widened) {
        const long long position = (long long)s.G * p.padded, sequence = s.T * position;
        k.b = rows, k.c = p.copies == 2 ? rows + s.B * sequence : rows;
        k.bb = k.cb = sequence, k.bt = k.ct = position, k.group = p.padded;
    } else {
        k.b = a.b, k.c = a.c;
        k.bb = s.b_stride[0], k.bt = s.b_stride[1], k.cb = s.c_stride[0], k.ct = s.c_stride[1], k.group = s.N;
    }
    return k;
}

hipError_t launch_selective_widen(const esrnn_selective_shape &s, const SelectiveArgs &a, const SelectivePlan &p, const Scan &k, hipStream_t st)
{
    if (!p.widened || p.copies == 0) return hipSuccess;
    return with_element(s.dtype, [&](auto e) {
        typedef decltype(e) E;
        selective_widen_kernel<E><<<dim3((unsigned)std::min<long long>((p.rows + kThreadsOfRows - 1) / kThreadsOfRows, kCopyWorkgroups)), kThreadsOfRows, 0, st>>>(
            static_cast<const E *>(a.b), static_cast<const E *>(a.c), s.b_stride[0], s.b_stride[1], s.c_stride[0], s.c_stride[1], p.copies, s.B, s.T, s.G,
            s.N, p.padded, const_cast<float *>(static_cast<const float *>(k.b)));
        return hipGetLastError();
    });
}

hipError_t launch_selective_carry(const esrnn_selective_shape &s, const SelectivePlan &p, const Scan &k, bool reverse, hipStream_t st)
{
    if (!p.carried) return hipSuccess;
    const unsigned lines = (unsigned)(s.B * s.G * p.tiles);
    const auto launch = [&](auto states, auto slices) {
        constexpr int NP = decltype(states)::value, SL = decltype(slices)::value;
        const unsigned columns = lines * SL * (NP / 4);
        if (p.segments > kCarryWaves * kBatch) selective_carry_kernel<NP, SL, kFewColumns><<<dim3(columns * (64 / kFewColumns)), 64 * kCarryWaves, 0, st>>>(k, reverse);
        else selective_carry_kernel<NP, SL, 64><<<dim3(columns), 64 * kCarryWaves, 0, st>>>(k, reverse);
        return hipGetLastError();
    };
    if (p.slices == 4) return launch(std::integral_constant<int, 16>{}, std::integral_constant<int, 4>{});
    if (p.slices == 2) return launch(std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{});
    if (p.states == 16) return launch(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
    if (p.states == 8) return launch(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
    return launch(std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{});
}

hipError_t launch_selective_forward(const esrnn_selective_shape &s, const SelectiveArgs &a, hipStream_t st)
{
    SelectivePlan p = selective_plan(s, false);
    const Scan k = scan_arguments(s, a, p);
    if (const hipError_t e = launch_selective_widen(s, a, p, k, st); e != hipSuccess) return e;
    const unsigned lines = (unsigned)(s.B * s.G * p.tiles);
    return with_scan(s, p, [&](auto e, auto bc, auto states, auto slices) {
        typedef decltype(e) E;
        typedef decltype(bc) BC;
        constexpr int NP = decltype(states)::value, SL = decltype(slices)::value;
        if constexpr (SL == 1)
            if (p.line_waves) {
                selective_line_kernel<E, BC, NP, kLineWaves><<<dim3(lines), 64 * p.line_waves, 0, st>>>(k);
                return hipGetLastError();
            }
        if (p.segments > 1) {
            selective_forward_kernel<E, BC, NP, SL, true><<<dim3(lines * (p.segments - 1)), 64 * SL, 0, st>>>(k);
            if (const hipError_t failed = launch_selective_carry(s, p, k, false, st); failed != hipSuccess) return failed;
        }
        selective_forward_kernel<E, BC, NP, SL, false><<<dim3(lines * p.segments), 64 * SL, 0, st>>>(k);
        return hipGetLastError();
    });
}

}  // namespace esrnn
