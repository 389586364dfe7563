// Selective scan over whole sequences, reverse pass (include/esrnn_state_space.h; selective_scan.h has the way it is cut up).
//
// With lambda_t the gradient of h_t and mu_t = a_t lambda_t that of what a_t multiplies, from the end:
//   lambda_t = g_t c_t + mu_{t+1}        (g: gradient of out; behind the last position: that of the last state)
//   grad c_t = sum over channels of g_t h_t,   grad b_t = sum over channels of lambda_t d_t x_t
//   grad x_t = d_t sum_n lambda_t b_t + D g_t,  grad d_t = sum_n mu_t h_{t-1} A + x_t sum_n lambda_t b_t,  grad delta_t = grad d_t softplus'
//   grad A = sum_t mu_t h_{t-1} d_t,  grad D = sum_t g_t x_t,  grad bias = sum_t grad delta_t,  grad initial = mu at the first position.
// The states h are computed again, piece by piece, from the one before each piece that the forward pass has left; for a piece they stay in
// registers, four of a lane's states at a time.  Sums over channels go through LDS within a wave and over tiles in a second launch; those over positions
// stay in a lane and go over segments in the same.
//
// A state takes a power of two and some 13 instructions, with the sums over channels, of the vector ALU, which is the bound: 4 x 4096 x 2048, 16 states,
// bf16, 64 segments: 493 us in all.  Dispatch by dispatch under the profiler, where they take a tenth longer together: maps 114 (101 of instructions), putting them
// together 21, b and c by pieces 5, gradients 379 (285 of instructions; 531 MB read), sums 23.  1 x 65536 x 256: 281 us in all; 501 x 240 x 50 ragged fp32: 159;
// 4 x 2048 x 1024, 64 states, bf16: 474.  Tried and slower: two states at a
// time (699 us for the gradients, for twice the scalar loads and sums); b and c as they are given, 559 us in all, for a piece's are 32 narrow scalar loads and
// not 8 wide ones; one tile's gradients of b and c without the second launch, which takes 40 registers that there are not.
#include <algorithm>

#include "selective_scan.h"

namespace esrnn {

namespace {

// Sums over the lanes of a wave go through LDS: a lane leaves its four values for b and four for c at each of eight positions; then a lane has one of
// eight positions, b or c, and adds up every fourth lane's, four states at a time, and the four lanes of a quad put their sums together, a state each.
// That is 8.6 vector instructions for a position's eight values where exchanges between lanes alone, each of which halves the lanes and the values, take
// 18; the vector ALU is the bound here and LDS is not.  Rows are 64 lanes x 16 bytes and 64 bytes more, so that the sixteen lanes of a read have all banks.
constexpr int kSumRow = 64 * 4 + 16;
// Between accesses of a wave's lanes to what other lanes of it have: the hardware serves a wave's LDS accesses in their order, and the compiler has to keep it.
// (No instruction of its own.)
__device__ __forceinline__ void ordered_in_wave()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
// Sums of the quad's lanes, the first value in the lane 0, ..
__device__ __forceinline__ float exchanged(float keep, float send, std::integral_constant<int, 2>)
{
    return keep + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, send), 0x4e, 0xf, 0xf, true));     // lane ^ 2
}
__device__ __forceinline__ float exchanged(float keep, float send, std::integral_constant<int, 1>)
{
    return keep + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, send), 0xb1, 0xf, 0xf, true));     // lane ^ 1
}
__device__ __forceinline__ float sum_of_quad(f32x4 v)
{
    const bool upper = threadIdx.x & 2, odd = threadIdx.x & 1;
    const std::integral_constant<int, 2> two;
    const std::integral_constant<int, 1> one;
    const float p = exchanged(upper ? v[2] : v[0], upper ? v[0] : v[2], two), q = exchanged(upper ? v[3] : v[1], upper ? v[1] : v[3], two);
    return exchanged(odd ? q : p, odd ? p : q, one);
}

// mu behind the last position of a segment, of the sequence's last segment with positions: the gradient of the last state.
template <int NP, int SL>
__device__ __forceinline__ void arriving(const Scan &k, const ScanPlace &at, size_t own, const float (&A)[NP], float (&mu)[NP])
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int n = 0; n < NP; ++n) mu[n] = 0.0f;
    if (k.carried) return load_states<NP>(map_of<NP, SL>(k, at, at.segment), mu);
    if (k.a.grad_last) load_own<NP>(k.a.grad_last + own, at.slice, k.N, at.lane_mask, mu);
    for (int s = max(at.length - 1, 0) / (k.span * kPiece); s > at.segment; --s) {
        const float *map = map_of<NP, SL>(k, at, s);
        float local[NP];
        load_states<NP>(map, local);
        const float sum = map[64 * NP + lane];
#pragma unroll
        for (int n = 0; n < NP; ++n) mu[n] = fmaf(__builtin_amdgcn_exp2f(sum * A[n]), mu[n], local[n]);
    }
}

// The maps of all segments but the first, against time.
template <class E, class BC, int NP, int SL>
__global__ void __launch_bounds__(64 * SL) selective_back_maps_kernel(Scan k)
{
    ScanPlace at(k, k.segments - 1);
    ++at.segment;
    const int lane = threadIdx.x & 63;
    const int begin = at.segment * k.span * kPiece, end = min(min(begin + k.span * kPiece, k.T), at.length);
    if (begin >= end) return;
    const E *delta = static_cast<const E *>(k.a.delta) + at.b * k.db, *grad = static_cast<const E *>(k.a.grad_out) + at.b * k.gb;
    const BC *c = static_cast<const BC *>(k.c) + at.b * k.cb + at.group * k.group + NP * at.slice;
    float A[NP], mu[NP];
    load_own<NP>(k.a.A + (size_t)at.channel * k.N, at.slice, k.N, at.lane_mask, A);
#pragma unroll
    for (int n = 0; n < NP; ++n) A[n] = exponent_rate(A[n]), mu[n] = 0.0f;
    const float bias = k.a.bias ? k.a.bias[at.channel] : 0.0f;
    float sum = 0.0f;
    Column<E> ds, gs, next_ds, next_gs;
    const int top = begin + (end - 1 - begin) / kPiece * kPiece;
    ds.request(delta, k.dt, top, at.length, at.channel);
    gs.request(grad, k.gt, top, at.length, at.channel);
    for (int t0 = top; t0 >= begin; t0 -= kPiece) {
        next_ds.request(delta, k.dt, max(t0 - kPiece, 0), at.length, at.channel);
        next_gs.request(grad, k.gt, max(t0 - kPiece, 0), at.length, at.channel);
        const int t = fresh(t0), left = at.length - 1 - t;
        const BC *c0 = c + t * k.ct;
#pragma unroll
        for (int i = kPiece - 1; i >= 0; --i) {
            const unsigned mask = i <= left ? 0xffffffffu : 0u;
            const float d = masked(step_size(ds.v[i], bias, k.softplus).of, mask), g = masked((float)gs.v[i], mask);
            float cs[NP];
            load_shared<BC, NP>(c0, k.ct, i, left, cs);
            sum += d;
#pragma unroll
            for (int n = 0; n < NP; ++n) mu[n] = __builtin_amdgcn_exp2f(d * A[n]) * fmaf(cs[n], g, mu[n]);
        }
        ds = next_ds, gs = next_gs;
    }
    float *map = map_of<NP, SL>(k, at, at.segment);
    store_states<NP>(map, mu);
    map[64 * NP + lane] = sum;
}

// b and c in the order of PieceRows, zeros for states and positions that there are not: [B][pieces][G][fours of states][8][2][4], four a thread.
template <class E, class BC>
__global__ void __launch_bounds__(256) selective_arrange_kernel(Scan k, const E *b, const E *c, long long bb, long long bt, long long cb, long long ct, int fours,
                                                                long long count, Vec4<BC> *to)
{
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < count; i += (long long)gridDim.x * 256) {
        const int which = i & 1, position = i >> 1 & 7;
        long long rest = i >> 4;
        const int n = 4 * (int)(rest % fours);
        rest /= fours;
        const int group = rest % k.G;
        rest /= k.G;
        const int t = (int)(rest % k.pieces) * kPiece + position, s = (int)(rest / k.pieces);
        const int length = k.a.lengths ? min(max(k.a.lengths[s], 0), k.T) : k.T;
        const E *from = (which ? c + s * cb + (long long)min(t, k.T - 1) * ct : b + s * bb + (long long)min(t, k.T - 1) * bt) + (long long)group * k.N;
        Vec4<BC> v;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float value = (float)from[min(n + r, k.N - 1)];
            v[r] = (BC)(n + r < k.N && t < length ? value : 0.0f);
        }
        to[i] = v;
    }
}

template <class E, class BC, int NP, int SL>
__global__ void __launch_bounds__(64 * SL, SL > 1 ? 1 : 2) selective_backward_kernel(Scan k)
{
    constexpr int kPart = 4, kPadded = NP * SL;     // (states at a time: theirs at nine positions and their decays at eight take 68 registers)
    __shared__ __attribute__((aligned(16))) float s_shared[SL][2 * kPiece][kSumRow];
    __shared__ float s_steepest[SL > 1 ? SL : 1][64];
    const ScanPlace at(k, k.segments);
    const int lane = threadIdx.x & 63;
    const int begin = at.segment * k.span * kPiece, end = min(begin + k.span * kPiece, k.T);
    const E *x = static_cast<const E *>(k.a.x) + at.b * k.xb, *delta = static_cast<const E *>(k.a.delta) + at.b * k.db;
    const E *grad = static_cast<const E *>(k.a.grad_out) + at.b * k.gb;
    E *grad_x = static_cast<E *>(k.a.grad_x) + at.b * k.gxb, *grad_delta = static_cast<E *>(k.a.grad_delta) + at.b * k.gdb;
    const BC *shared_rows = static_cast<const BC *>(k.arranged) + ((size_t)at.b * k.pieces * k.G + at.group) * (kPadded / 4 * 64) + at.slice * (NP / 4 * 64);
    const size_t own = ((size_t)at.b * k.C + at.channel) * k.N;

    float A[NP], mu[NP], dA[NP], dD = 0.0f, dbias = 0.0f;
    load_own<NP>(k.a.A + (size_t)at.channel * k.N, at.slice, k.N, at.lane_mask, A);
#pragma unroll
    for (int n = 0; n < NP; ++n) A[n] = exponent_rate(A[n]), dA[n] = 0.0f;
    const float bias = k.a.bias ? k.a.bias[at.channel] : 0.0f, D = k.a.D ? k.a.D[at.channel] : 0.0f;
    if (begin < at.length || begin == 0) arriving<NP, SL>(k, at, own, A, mu);

    // what a lane has after all additions: position lane / 8, b or c, state lane % 4; rows of [2][padded] for every position and group
    const float *parts = k.part_rows + (((size_t)(at.tile % k.tiles) * k.B + at.b) * k.pieces * kPiece * k.G + at.group) * (2 * kPadded) + NP * at.slice;
    const unsigned part_position = (unsigned)k.G * (2 * kPadded);
    const unsigned part_at = 4 * ((lane >> 3) * part_position + (lane >> 2 & 1) * kPadded + (lane & 3));
    float(*shared)[kSumRow] = s_shared[at.slice];
    // The largest rate of the channel, which may make an infinity of what a slope of zero is multiplied by.
    float steepest = 0.0f;
#pragma unroll
    for (int n = 0; n < NP; ++n) steepest = fminf(steepest, A[n]);
    if constexpr (SL > 1) s_steepest[at.slice][lane] = steepest;        // (the other slices read it behind the barrier of a piece)
    const float *shared_read = &shared[lane >> 2][4 * (lane & 3)];

    const int last = min(end, at.length);
    if (begin < last) {
        const int top = begin + (last - 1 - begin) / kPiece * kPiece;
        // the next piece's elements are requested while this one is worked on, and the next four states while these are
        Column<E> xs, ds, gs;
        xs.request(x, k.xt, top, at.length, at.channel);
        ds.request(delta, k.dt, top, at.length, at.channel);
        gs.request(grad, k.gt, top, at.length, at.channel);
        f32x4 next_states = *reinterpret_cast<const f32x4 *>(saved_of<NP, SL>(k, at, top / kPiece) + 4 * lane);
        for (int t0 = top; t0 >= begin; t0 -= kPiece) {
            const int t = fresh(t0), left = at.length - 1 - t;
            const float *saved = saved_of<NP, SL>(k, at, t / kPiece);
            const BC *rows = shared_rows + (size_t)(t / kPiece) * k.G * (kPadded / 4 * 64);
            const buf_rsrc to_parts = make_base(parts + (size_t)t * part_position);
            float d[kPiece], slope[kPiece], xi[kPiece], g[kPiece], through[kPiece], rate[kPiece];   // through: sum lambda b; rate: sum mu h_{t-1} A log2(e)
#pragma unroll
            for (int i = 0; i < kPiece; ++i) {
                const unsigned mask = i <= left ? 0xffffffffu : 0u;
                const Softplus s = step_size(ds.v[i], bias, k.softplus);
                d[i] = masked(masked(s.of, at.lane_mask), mask), g[i] = masked(masked((float)gs.v[i], at.lane_mask), mask);
                slope[i] = masked(s.slope, mask), xi[i] = (float)xs.v[i];
                through[i] = rate[i] = 0.0f;
            }
            const int before_t = max(t0 - kPiece, begin);
            xs.request(x, k.xt, before_t, at.length, at.channel);
            ds.request(delta, k.dt, before_t, at.length, at.channel);
            gs.request(grad, k.gt, before_t, at.length, at.channel);
#pragma unroll
            for (int n0 = 0; n0 < NP; n0 += kPart) {
                // (or the parts' registers add up, and the loads of all of them become one)
                __builtin_amdgcn_sched_barrier(0);
                const PieceRows<BC> bc(rows + 64 * fresh(n0 / 4));
                float h[kPiece + 1][kPart], decay[kPiece][kPart];
                const f32x4 before = next_states;
                next_states = *reinterpret_cast<const f32x4 *>((n0 + kPart < NP ? saved + 64 * (n0 + kPart) : saved_of<NP, SL>(k, at, before_t / kPiece)) + 4 * lane);
#pragma unroll
                for (int n = 0; n < kPart; ++n) h[0][n] = before[n];
#pragma unroll
                for (int i = 0; i < kPiece; ++i) {
                    const float u = d[i] * xi[i];
#pragma unroll
                    for (int n = 0; n < kPart; ++n) {
                        decay[i][n] = __builtin_amdgcn_exp2f(d[i] * A[n0 + n]);
                        h[i + 1][n] = fmaf(decay[i][n], h[i][n], u * bc.get(i, 0, n));
                    }
                }
#pragma unroll
                for (int i = kPiece - 1; i >= 0; --i) {
                    float of_b[kPart], of_c[kPart];
                    const float u = d[i] * xi[i];
#pragma unroll
                    for (int n = 0; n < kPart; ++n) {
                        const float lambda = fmaf(bc.get(i, 1, n), g[i], mu[n0 + n]);
                        of_c[n] = g[i] * h[i + 1][n];
                        of_b[n] = u * lambda;
                        through[i] = fmaf(bc.get(i, 0, n), lambda, through[i]);
                        mu[n0 + n] = decay[i][n] * lambda;
                        const float m = mu[n0 + n] * h[i][n];
                        rate[i] = fmaf(m, A[n0 + n], rate[i]);
                        dA[n0 + n] = fmaf(m, d[i], dA[n0 + n]);
                    }
                    *reinterpret_cast<f32x4 *>(&shared[2 * i][4 * lane]) = f32x4{of_b[0], of_b[1], of_b[2], of_b[3]};
                    *reinterpret_cast<f32x4 *>(&shared[2 * i + 1][4 * lane]) = f32x4{of_c[0], of_c[1], of_c[2], of_c[3]};
                }
                ordered_in_wave();
                f32x4 sum[2] = {*reinterpret_cast<const f32x4 *>(shared_read), *reinterpret_cast<const f32x4 *>(shared_read + 16)};
#pragma unroll
                for (int c = 2; c < 16; ++c) sum[c & 1] += *reinterpret_cast<const f32x4 *>(shared_read + 16 * c);
                ordered_in_wave();
                buf_store(to_parts, part_at, 4 * n0, sum_of_quad(sum[0] + sum[1]));
                complete(through);
                complete(rate);
                complete(dA, n0, kPart);
            }
            float of_channel = SL > 1 ? 0.0f : steepest;
            if constexpr (SL > 1) {
                // the wave has read its rows: they hold its shares of the sums over all states until every slice has read those of its positions
#pragma unroll
                for (int i = 0; i < kPiece; ++i) shared[i][lane] = through[i], shared[kPiece + i][lane] = rate[i];
                lds_barrier();      // (requests for the next piece go on)
#pragma unroll
                for (int s = 0; s < SL; ++s) of_channel = fminf(of_channel, s_steepest[s][lane]);
#pragma unroll
                for (int i = 0; i < kPiece; ++i)
                    if (i % SL == at.slice) {
                        through[i] = rate[i] = 0.0f;
#pragma unroll
                        for (int s = 0; s < SL; ++s) through[i] += s_shared[s][i][lane], rate[i] += s_shared[s][kPiece + i][lane];
                    }
                lds_barrier();
            }
            // Slopes are zero past the length, too.  And steps below kLeastStep get no gradient from decays where a rate is infinite: it has no derivative there, and behind
            // larger steps nothing is left that would go by it.  (Behind a condition for the wave: selections at every piece cost 1 to 5 % of the kernel.)
            if (__any(of_channel < -0x1p64f)) {
                const float least = of_channel == kForgetsAll ? kLeastStep : 0.0f;
#pragma unroll
                for (int i = 0; i < kPiece; ++i) rate[i] = fabsf(d[i]) < least || slope[i] == 0.0f ? 0.0f : rate[i];
            }
#pragma unroll
            for (int i = 0; i < kPiece; ++i) {
                if (i % SL != at.slice || t + i >= end) continue;
                const float to_x = fmaf(d[i], through[i], D * g[i]), to_delta = fmaf(rate[i], kLn2, xi[i] * through[i]) * slope[i];
                dbias += to_delta;
                dD = fmaf(g[i], xi[i], dD);
                if (at.lane_mask) {
                    (grad_x + (t + i) * k.gxt)[at.channel] = (E)to_x;
                    (grad_delta + (t + i) * k.gdt)[at.channel] = (E)to_delta;
                }
            }
        }
    }
    if (at.segment == 0 && k.a.grad_initial) store_own<NP>(k.a.grad_initial + own, at.slice, k.N, at.lane_mask, mu);
    for (int t = max(begin, (at.length + kPiece - 1) / kPiece * kPiece); t < end; ++t)
        if (t % SL == at.slice && at.lane_mask) {
            (grad_x + t * k.gxt)[at.channel] = (E)0.0f;
            (grad_delta + t * k.gdt)[at.channel] = (E)0.0f;
        }
    if constexpr (SL > 1) {
        // (every slice has its share of the positions; the first one leaves the sums)
        shared[0][lane] = dD, shared[1][lane] = dbias;
        lds_barrier();
        if (at.slice == 0)
#pragma unroll
            for (int s = 1; s < SL; ++s) dD += s_shared[s][0][lane], dbias += s_shared[s][1][lane];
    }
    float *sums = k.part_sums + ((((size_t)at.b * k.segments + at.segment) * (k.G * k.tiles) + at.tile) * SL + at.slice) * ((NP + 2) * 64);
#pragma unroll
    for (int n = 0; n < NP; ++n) sums[64 * n + lane] = dA[n];
    sums[64 * NP + lane] = dD;
    sums[64 * (NP + 1) + lane] = dbias;
}

// The sums over segments of the gradients of A, D and bias (the first workgroups; rows of [tile][slice][states + 2][64]) and those over tiles of the
// gradients of b and c (the others; [tile][position][group][2][padded]).
constexpr int kSumWorkgroups = 768;     // about, each with neighbouring positions of a sequence
template <class E, int kCols>
__global__ void __launch_bounds__(1024) selective_sum_kernel(Scan k, int states, int slices, unsigned first_rows, int positions, E *grad_b, E *grad_c,
                                                             long long gbb, long long gbt, long long gcb, long long gct)
{
    if (blockIdx.x < first_rows) {
        const int wave = (states + 2) * 64;
        const long long cols = (long long)k.G * k.tiles * slices * wave, rows = (long long)k.B * k.segments;
        sum_columns<kCols>(k.part_sums, rows, cols, (long long)blockIdx.x * kCols, [&](long long col, float v) {
            const int lane = col % 64, n = (int)(col / 64) % (states + 2), slice = (int)(col / wave) % slices, tile = (int)(col / wave / slices);
            const int in_group = tile % k.tiles * 64 + lane, channel = tile / k.tiles * k.group_channels + in_group;
            if (in_group >= k.group_channels) return;
            if (n < states) {
                if (slice * states + n < k.N) k.a.grad_A[(size_t)channel * k.N + slice * states + n] = v;
            } else if (float *to = n == states ? k.a.grad_D : k.a.grad_bias) {
                if (slice == 0) to[channel] = v;
            }
        });
        return;
    }
    const unsigned padded = states * slices, width = k.G * 2 * padded, place = blockIdx.x - first_rows;
    const int whole = k.pieces * kPiece, runs = (k.T + positions - 1) / positions, b = place / (unsigned)runs, t0 = place % (unsigned)runs * positions;
    const int length = k.a.lengths ? min(max(k.a.lengths[b], 0), k.T) : k.T;
    const size_t tile_apart = (size_t)k.B * whole * width;
    const float *from = k.part_rows + ((size_t)b * whole + t0) * width;
    grad_b += b * gbb, grad_c += b * gcb;
    // (four states a thread, which share the divisions: rows are whole fours of them)
    const unsigned fours = width / 4;
    for (unsigned i = threadIdx.x; i < min(positions, k.T - t0) * fours; i += 1024) {
        const unsigned t = t0 + i / fours, within = 4 * (i % fours), n = within % padded, group = within / (2 * padded);
        if (n >= (unsigned)k.N) continue;
        f32x4 v = {};
        if (t < (unsigned)length) {
            const float *tile = from + 4 * (size_t)i;
            v = *reinterpret_cast<const f32x4 *>(tile);
#pragma unroll 8
            for (int q = 1; q < k.tiles; ++q) v += *reinterpret_cast<const f32x4 *>(tile += tile_apart);
        }
        E *to = (within / padded & 1 ? grad_c + t * gct : grad_b + t * gbt) + (size_t)group * k.N + n;
        typedef E Four __attribute__((ext_vector_type(4), aligned(sizeof(E))));
        if (n + 4 <= (unsigned)k.N) {
            *reinterpret_cast<Four *>(to) = Four{(E)v[0], (E)v[1], (E)v[2], (E)v[3]};
        } else {
#pragma unroll
            for (unsigned r = 0; r < 3; ++r)
                if (n + r < (unsigned)k.N) to[r] = (E)v[r];
        }
    }
}

}  // namespace

hipError_t launch_selective_backward(const esrnn_selective_shape &s, const SelectiveArgs &a, hipStream_t st)
{
    SelectivePlan p = selective_plan(s, true);
    const Scan k = scan_arguments(s, a, p);
    if (const hipError_t e = launch_selective_widen(s, a, p, k, st); e != hipSuccess) return e;
    const unsigned lines = (unsigned)(s.B * s.G * p.tiles);
    const hipError_t failed = with_scan(s, p, [&](auto e, auto bc, auto states, auto slices) {
        typedef decltype(e) E;
        typedef decltype(bc) BC;
        constexpr int NP = decltype(states)::value, SL = decltype(slices)::value;
        if (p.segments > 1) {
            selective_back_maps_kernel<E, BC, NP, SL><<<dim3(lines * (p.segments - 1)), 64 * SL, 0, st>>>(k);
            if (const hipError_t stopped = launch_selective_carry(s, p, k, true, st); stopped != hipSuccess) return stopped;
        }
        const long long count = (long long)s.B * p.pieces * s.G * p.padded / 4 * 16;
        selective_arrange_kernel<E, BC><<<dim3((unsigned)std::min((count + 255) / 256, kCopyWorkgroups)), 256, 0, st>>>(
            k, static_cast<const E *>(a.b), static_cast<const E *>(a.c), s.b_stride[0], s.b_stride[1], s.c_stride[0], s.c_stride[1], p.padded / 4, count,
            static_cast<Vec4<BC> *>(const_cast<void *>(k.arranged)));
        selective_backward_kernel<E, BC, NP, SL><<<dim3(lines * p.segments), 64 * SL, 0, st>>>(k);
        return hipGetLastError();
    });
    if (failed != hipSuccess) return failed;
    const long long columns = (long long)s.G * p.tiles * p.slices * (p.states + 2) * 64;
    const int positions = (int)(((long long)s.B * s.T + kSumWorkgroups - 1) / kSumWorkgroups);
    const unsigned runs = (unsigned)s.B * ((s.T + positions - 1) / positions);
    return with_element(s.dtype, [&](auto e) {
        return with_columns(columns, [&](auto cols) {
            typedef decltype(e) E;
            constexpr int kCols = decltype(cols)::value;
            const unsigned first = (unsigned)(columns / kCols);
            selective_sum_kernel<E, kCols><<<dim3(first + runs), 1024, 0, st>>>(k, p.states, p.slices, first, positions, static_cast<E *>(a.grad_b), static_cast<E *>(a.grad_c),
                                                                              s.grad_b_stride[0], s.grad_b_stride[1], s.grad_c_stride[0], s.grad_c_stride[1]);
            return hipGetLastError();
        });
    });
}

}  // namespace esrnn
