// Short causal convolution of every channel with activation (include/esrnn_state_space.h).
//
// A lane has 8 or 16 bytes of neighbouring channels and walks a run of positions with the last K - 1 inputs in registers; 64 channels are a
// tile, and a workgroup has a tile of many runs.  Eight positions are requested at a time, four in the reverse pass.
//
// The reverse pass computes u again from x, and walks K - 1 positions past its run for the gradient of its last inputs:
//   du_t = d_t act'(u_t),  dx_s = sum_i weight[K-1-i] du_{s+i},  dweight[j] = sum_t du_t x_{t-K+1+j},  dbias = sum_t du_t.
// A lane's sums for the weights are put together within its workgroup and then over all workgroups by a second launch, in a fixed order.
//
// Reads and writes are the bound, 2 K + 5 operations an element forward and 4 K + 10 in reverse are not: 8 x 4096 x 2048 bf16, 4 taps, forward 60 us (275 MB, 4.6 TB/s),
// reverse 101 + 5 us (413 MB, 4.1 TB/s).  Runs rather than a position a lane, so that inputs are read once and not K times; their K - 1 first positions are read
// twice, which is a tenth at the shortest runs.  501 x 240 x 50 ragged fp32: 13 and 20 + 5 us.
#include <algorithm>

#include "state_space_internal.h"

namespace esrnn {

namespace {

constexpr int kGroup = 8, kBackGroup = 4, kThreads = 256, kTile = 64;

struct Args {
    ConvolutionArgs a;
    long long xb, xt, ob, ot, db, dt, gb, gt;       // strides of a sequence and of a position
    int B, T, C, silu;
    int tiles, blocks, run;     // tiles of 64 channels; blocks of positions, one for each workgroup; positions of a lane, a multiple of kGroup
};

// What a workgroup works on, and a lane of it.
template <class E, bool kReverse>
struct Place {
    static constexpr int V = kReverse ? 4 : 16 / (int)sizeof(E), kLanes = kTile / V, kRuns = kThreads / kLanes;
    int tile, b, block, lane, begin;        // begin: first position of this lane's run
    __device__ __forceinline__ Place(const Args &p)
    {
        tile = blockIdx.x % p.tiles;
        const unsigned rest = blockIdx.x / (unsigned)p.tiles;
        block = rest % p.blocks, b = rest / p.blocks;
        lane = threadIdx.x % kLanes;
        begin = (block * kRuns + (int)(threadIdx.x / kLanes)) * p.run;
    }
};

// G positions from `from` on: zeros where there is none (outside 0 .. length - 1).  What does not exist is read from a place that does, and
// masked out: loads behind a condition would be waited for one by one.
template <class E, int V, bool kWide, int G>
struct Rows {
    typedef Neighbours<E, V> N;
    typename N::Values v[G];
    __device__ __forceinline__ void request(const E *base, long long stride, int from, int length, const Overlapping<E, V, kWide> &ch)
    {
#pragma unroll
        for (int i = 0; i < G; ++i) v[i] = ch.load(base + (long long)max(min(from + i, length - 1), 0) * stride);
    }
    __device__ __forceinline__ typename N::Floats get(int i, int from, int length) const
    {
        unsigned mask = (unsigned)(from + i) < (unsigned)length ? 0xffffffffu : 0u;
        asm("" : "+v"(mask));
        return N::widen(__builtin_bit_cast(typename N::Values, __builtin_bit_cast(typename N::Bits, v[i]) & mask));
    }
};

template <class F>
__device__ __forceinline__ F splat_f(float v)
{
    F r;
#pragma unroll
    for (int k = 0; k < (int)(sizeof(F) / 4); ++k) r[k] = v;
    return r;
}

template <class E, int V, bool kWide, int K>
__device__ __forceinline__ void load_weights(const Args &p, const Overlapping<E, V, kWide> &ch, typename Neighbours<E, V>::Floats (&w)[K],
                                             typename Neighbours<E, V>::Floats &bias)
{
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int c = ch.channel(k);
#pragma unroll
        for (int j = 0; j < K; ++j) w[j][k] = p.a.weight[(long long)c * K + j];
        bias[k] = p.a.bias ? p.a.bias[c] : 0.0f;
    }
}

// seen[j], j < K - 1: the inputs before `begin`, oldest first.
template <class E, int V, bool kWide, int K>
__device__ __forceinline__ void load_past(const Args &p, const E *x, int b, int begin, int length, const Overlapping<E, V, kWide> &ch,
                                          typename Neighbours<E, V>::Floats (&seen)[K])
{
    typedef Neighbours<E, V> N;
#pragma unroll
    for (int j = 0; j < K - 1; ++j) {
        const int at = begin - (K - 1) + j;
        seen[j] = splat_f<typename N::Floats>(0.0f);
        if (at >= 0 && at < length) seen[j] = N::widen(ch.load(x + at * p.xt));
        else if (at < 0 && p.a.initial) seen[j] = N::widen(ch.load(static_cast<const E *>(p.a.initial) + ((long long)b * (K - 1) + K - 1 + at) * p.C));
    }
}

template <class E, int K, bool kWide>
__global__ void __launch_bounds__(kThreads) convolution_forward_kernel(Args p)
{
    typedef Place<E, false> Here;
    constexpr int V = Here::V;
    typedef Neighbours<E, V> N;
    typedef typename N::Floats F;
    const Here at(p);
    const Overlapping<E, V, kWide> ch(at.tile * kTile + at.lane * V, p.C);
    if (!ch.some()) return;
    const int length = p.a.lengths ? min(max(p.a.lengths[at.b], 0), p.T) : p.T;
    const E *x = static_cast<const E *>(p.a.x) + at.b * p.xb;
    E *out = static_cast<E *>(p.a.out) + at.b * p.ob;

    // the last inputs, by the last run of the first block, which has the least else to do in short sequences
    if (p.a.last && at.block == 0 && threadIdx.x / Here::kLanes == Here::kRuns - 1) {
        E *last = static_cast<E *>(p.a.last) + (long long)at.b * (K - 1) * p.C;
#pragma unroll
        for (int j = 0; j < K - 1; ++j) {
            const int t = length - (K - 1) + j;
            typename N::Values v = {};
            if (t >= 0) v = ch.load(x + t * p.xt);
            else if (p.a.initial) v = ch.load(static_cast<const E *>(p.a.initial) + ((long long)at.b * (K - 1) + K - 1 + t) * p.C);
            ch.store(last + (long long)j * p.C, v);
        }
    }
    const int end = min(at.begin + p.run, p.T);
    if (at.begin >= end) return;
    if (at.begin >= length) {       // nothing left of the sequence
        for (int t = at.begin; t < end; ++t) ch.store(out + t * p.ot, typename N::Values{});
        return;
    }
    F w[K], bias, seen[K];          // seen[K - 1]: the newest
    load_weights<E, V, kWide, K>(p, ch, w, bias);
    Rows<E, V, kWide, kGroup> rows;
    load_past<E, V, kWide, K>(p, x, at.b, at.begin, length, ch, seen);
    for (int t0 = at.begin; t0 < end; t0 += kGroup) {
        rows.request(x, p.xt, t0, length, ch);
#pragma unroll
        for (int i = 0; i < kGroup; ++i) {
            seen[K - 1] = rows.get(i, t0, length);
            F u = bias;
#pragma unroll
            for (int j = 0; j < K; ++j) u += w[j] * seen[j];
#pragma unroll
            for (int j = 0; j < K - 1; ++j) seen[j] = seen[j + 1];
            if (p.silu)
#pragma unroll
                for (int k = 0; k < V; ++k) u[k] = silu(u[k]).of;
            if (t0 + i < end) ch.store(out + (t0 + i) * p.ot, t0 + i < length ? N::round(u) : typename N::Values{});
        }
    }
}

// A run gives the gradients of its inputs, which need du up to K - 1 positions behind them: it begins with du of its first K - 1 positions, and then has du at
// t = s + K - 1 for the input at s.  The sums for the weights count the latter, and those of the first K - 1 positions of the sequence.
template <class E, int K, bool kWide>
__global__ void __launch_bounds__(kThreads, K <= 4 ? 3 : 2) convolution_backward_kernel(Args p)
{
    typedef Place<E, true> Here;
    constexpr int V = Here::V, kLanes = Here::kLanes, G = kBackGroup;
    typedef Neighbours<E, V> N;
    typedef typename N::Floats F;
    __shared__ float s_sum[kThreads / 64][K + 1][kTile];
    const Here at(p);
    const Overlapping<E, V, kWide> ch(at.tile * kTile + at.lane * V, p.C);
    const int length = p.a.lengths ? min(max(p.a.lengths[at.b], 0), p.T) : p.T;
    const E *x = static_cast<const E *>(p.a.x) + at.b * p.xb, *grad_out = static_cast<const E *>(p.a.grad_out) + at.b * p.db;
    E *grad_x = static_cast<E *>(p.a.grad_x) + at.b * p.gb;
    const int end = min(at.begin + p.run, p.T);

    F dw[K], dbias = splat_f<F>(0.0f);
#pragma unroll
    for (int j = 0; j < K; ++j) dw[j] = splat_f<F>(0.0f);
    // the share that grad_last has in the gradient of the input at s, negative ones those of `initial`
    const auto add_last = [&](int s, F &d) {
        const int tail = s - (length - (K - 1));
        if (p.a.grad_last && tail >= 0 && s < length) {
            const float *g = p.a.grad_last + ((long long)at.b * (K - 1) + tail) * p.C;
#pragma unroll
            for (int k = 0; k < V; ++k) d[k] += g[ch.channel(k)];
        }
    };
    const auto put_initial = [&](int s, F d) {
        if (!p.a.grad_initial) return;
        add_last(s, d);
        float *g = p.a.grad_initial + ((long long)at.b * (K - 1) + K - 1 + s) * p.C;
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (kWide || ch.first + k < p.C) g[ch.first + k] = d[k];
    };
    if (ch.some() && at.begin < end) {
        if (at.begin >= length) {
            for (int t = at.begin; t < end; ++t) ch.store(grad_x + t * p.gt, typename N::Values{});
            if (at.begin == 0)      // an empty sequence hands the gradient of `last` to `initial`
#pragma unroll
                for (int j = 0; j < K - 1; ++j) put_initial(j - (K - 1), splat_f<F>(0.0f));
        } else {
            F w[K], bias, seen[K], du[K];       // seen[K - 1], du[K - 1]: the newest
            load_weights<E, V, kWide, K>(p, ch, w, bias);
            load_past<E, V, kWide, K>(p, x, at.b, at.begin, length, ch, seen);
#pragma unroll
            for (int j = 0; j < K; ++j) du[j] = splat_f<F>(0.0f);
            // the next position: `d` of out, whose u is made of seen[0 .. K - 1]
            const auto advance = [&](F d, bool counts) {
                if (p.silu) {
                    F u = bias;
#pragma unroll
                    for (int j = 0; j < K; ++j) u += w[j] * seen[j];
#pragma unroll
                    for (int k = 0; k < V; ++k) d[k] *= silu(u[k]).slope;
                }
                du[K - 1] = d;
                if (counts) {
                    dbias += d;
#pragma unroll
                    for (int j = 0; j < K; ++j) dw[j] += d * seen[j];
                }
            };
            // the gradient of the input K - 1 positions before the newest, and then one position on
            const auto gradient = [&] {
                F dx = w[K - 1] * du[0];
#pragma unroll
                for (int j = 1; j < K; ++j) dx += w[K - 1 - j] * du[j];
#pragma unroll
                for (int j = 0; j < K - 1; ++j) seen[j] = seen[j + 1], du[j] = du[j + 1];
                return dx;
            };
            {
                Rows<E, V, kWide, K - 1> rows, ds;
                rows.request(x, p.xt, at.begin, length, ch);
                ds.request(grad_out, p.dt, at.begin, length, ch);
#pragma unroll
                for (int i = 0; i < K - 1; ++i) {
                    seen[K - 1] = rows.get(i, at.begin, length);
                    advance(ds.get(i, at.begin, length), at.begin == 0);
                    const F dx = gradient();
                    if (at.begin == 0) put_initial(i - (K - 1), dx);
                }
            }
            for (int s0 = at.begin; s0 < end; s0 += G) {
                const int t0 = s0 + K - 1;
                Rows<E, V, kWide, G> rows, ds;
                rows.request(x, p.xt, t0, length, ch);
                ds.request(grad_out, p.dt, t0, length, ch);
                typename N::Values to[G];
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    seen[K - 1] = rows.get(i, t0, length);
                    advance(ds.get(i, t0, length), true);
                    F dx = gradient();
                    if (s0 + G > length - (K - 1)) add_last(s0 + i, dx);
                    to[i] = N::round(dx);
                }
#pragma unroll
                for (int i = 0; i < G; ++i)
                    if (s0 + i < end) ch.store(grad_x + (s0 + i) * p.gt, s0 + i < length ? to[i] : typename N::Values{});
            }
        }
    }
    // sums over the runs of the workgroup: within a wave, then over its waves
    const int wave = threadIdx.x / 64;
#pragma unroll
    for (int j = 0; j <= K; ++j)
#pragma unroll
        for (int k = 0; k < V; ++k) {
            float v = j < K ? dw[j < K ? j : 0][k] : dbias[k];
#pragma unroll
            for (int off = kLanes; off < 64; off *= 2) v += __shfl_xor(v, off, 64);
            // (a channel that another lane or tile has too: the same sum, or that tile's)
            const int place = ch.first + k - at.tile * kTile;
            if ((threadIdx.x & 63) < kLanes && place >= 0 && place < kTile) s_sum[wave][j][place] = v;
        }
    __syncthreads();
    float *parts = p.a.parts + ((long long)(at.b * p.blocks + at.block) * p.tiles + at.tile) * (K + 1) * kTile;
    for (int i = threadIdx.x; i < (K + 1) * kTile; i += kThreads) {
        float v = 0.0f;
#pragma unroll
        for (int q = 0; q < kThreads / 64; ++q) v += s_sum[q][i / kTile][i % kTile];
        parts[i] = v;
    }
}

// Rows of partial sums: [tile][K + 1][64] each.
template <int kCols>
__global__ void __launch_bounds__(1024) convolution_sum_kernel(const float *__restrict__ parts, long long rows, int tiles, int K, int C, float *grad_weight,
                                                               float *grad_bias)
{
    sum_columns<kCols>(parts, rows, (long long)tiles * (K + 1) * kTile, (long long)blockIdx.x * kCols, [&](long long col, float v) {
        const int j = (int)(col / kTile) % (K + 1), c = (int)(col / ((K + 1) * kTile)) * kTile + (int)(col % kTile);
        if (c >= C) return;
        if (j < K) grad_weight[(long long)c * K + j] = v;
        else if (grad_bias) grad_bias[c] = v;
    });
}

// One position of many requests: a lane has 16 bytes of neighbouring channels of one request.
template <class E, int K>
__global__ void __launch_bounds__(kThreads) convolution_step_kernel(esrnn_convolution_step_shape s, const E *x, const float *__restrict__ weight,
                                                                    const float *__restrict__ bias, const int32_t *slots, E *state, E *out, int tiles)
{
    constexpr int V = 16 / sizeof(E);
    typedef Neighbours<E, V> N;
    const int i = blockIdx.x / tiles;
    const N ch{(int)((blockIdx.x % tiles) * kThreads + threadIdx.x) * V, s.C};
    if (!ch.some()) return;
    const int slot = slots ? slots[i] : i;
    E *to = out + i * s.out_stride;
    if (slot < 0 || slot >= s.pool) {
        ch.store(to, typename N::Values{});
        return;
    }
    E *own = state + (long long)slot * (K - 1) * s.C;
    typename N::Values seen[K];
#pragma unroll
    for (int j = 0; j < K - 1; ++j) seen[j] = ch.load(own + (long long)j * s.C);
    seen[K - 1] = ch.load(x + i * s.x_stride);
    typename N::Floats u;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int c = min(ch.first + k, s.C - 1);
        u[k] = bias ? bias[c] : 0.0f;
#pragma unroll
        for (int j = 0; j < K; ++j) u[k] = fmaf(weight[(long long)c * K + j], (float)seen[j][k], u[k]);
        if (s.activation == ESRNN_NORM_SILU) u[k] = silu(u[k]).of;
    }
#pragma unroll
    for (int j = 0; j < K - 1; ++j) ch.store(own + (long long)j * s.C, seen[j + 1]);
    ch.store(to, N::round(u));
}

// f(std::integral_constant<int, K>)
template <class F>
hipError_t with_taps(int K, F &&f)
{
    switch (K) {
    case 2: return f(std::integral_constant<int, 2>{});
    case 3: return f(std::integral_constant<int, 3>{});
    case 4: return f(std::integral_constant<int, 4>{});
    case 5: return f(std::integral_constant<int, 5>{});
    case 6: return f(std::integral_constant<int, 6>{});
    case 7: return f(std::integral_constant<int, 7>{});
    default: return f(std::integral_constant<int, 8>{});
    }
}

// Positions of a lane's run: the longest of which there are 500 workgroups, two for each compute unit, as a run's first K - 1 positions are work of its own.
// Forward and reverse in us, bf16, with runs of 8, 16, 32, 64, 128: 8 x 4096 x 2048 (512 workgroups at 64 and at 128) 56, 51, 53, 49, 53 and 136, 106, 99, 105,
// 95; 1 x 65536 x 256 (512 at 16 and at 32) 20, 16, 18, 27, 46 and 38, 33, 31, 35, 59; 2 x 4096 x 64 (as many as there are at 8) 7, 9, 14, 23, 42 and
// 12, 14, 20, 30, 52.
Args arguments(const esrnn_convolution_shape &s, const ConvolutionArgs &a, bool reverse)
{
    Args p{};
    p.a = a;
    p.B = s.B, p.T = s.T, p.C = s.C, p.silu = s.activation == ESRNN_NORM_SILU;
    p.xb = s.x_stride[0], p.xt = s.x_stride[1], p.ob = s.out_stride[0], p.ot = s.out_stride[1];
    p.db = s.grad_out_stride[0], p.dt = s.grad_out_stride[1], p.gb = s.grad_x_stride[0], p.gt = s.grad_x_stride[1];
    p.tiles = (s.C + kTile - 1) / kTile;
    const int runs = reverse ? Place<float, true>::kRuns : s.dtype == ESRNN_F32 ? Place<float, false>::kRuns : Place<__bf16, false>::kRuns;
    const auto blocks = [&](int run) { return ((long long)s.T + runs * run - 1) / (runs * run); };
    p.run = kGroup;
    while (p.run < 128 && runs * p.run < s.T && s.B * p.tiles * blocks(2 * p.run) >= 500) p.run *= 2;
    p.blocks = (int)blocks(p.run);
    return p;
}

// f(element type tag, taps, whether a lane's channels are there at least once)
template <class F>
hipError_t with_access(const esrnn_convolution_shape &s, int reverse, F &&f)
{
    return with_element(s.dtype, [&](auto e) {
        return with_taps(s.K, [&](auto k) {
            if (s.C >= (reverse ? 4 : 16 / (int)sizeof(e))) return f(e, k, std::true_type{});
            return f(e, k, std::false_type{});
        });
    });
}

}  // namespace

size_t convolution_workspace_floats(const esrnn_convolution_shape &s)
{
    const Args p = arguments(s, ConvolutionArgs{}, true);
    return (size_t)s.B * p.blocks * p.tiles * (s.K + 1) * kTile;
}

hipError_t launch_convolution_forward(const esrnn_convolution_shape &s, const ConvolutionArgs &a, hipStream_t st)
{
    const Args p = arguments(s, a, false);
    return with_access(s, false, [&](auto e, auto k, auto wide) {
        convolution_forward_kernel<decltype(e), decltype(k)::value, decltype(wide)::value><<<dim3(p.B * p.blocks * p.tiles), kThreads, 0, st>>>(p);
        return hipGetLastError();
    });
}

hipError_t launch_convolution_backward(const esrnn_convolution_shape &s, const ConvolutionArgs &a, hipStream_t st)
{
    const Args p = arguments(s, a, true);
    const hipError_t failed = with_access(s, true, [&](auto e, auto k, auto wide) {
        convolution_backward_kernel<decltype(e), decltype(k)::value, decltype(wide)::value><<<dim3(p.B * p.blocks * p.tiles), kThreads, 0, st>>>(p);
        return hipGetLastError();
    });
    if (failed != hipSuccess) return failed;
    return with_columns((long long)p.tiles * (s.K + 1) * kTile, [&](auto cols) {
        constexpr int kCols = decltype(cols)::value;
        convolution_sum_kernel<kCols><<<dim3(p.tiles * (s.K + 1) * (kTile / kCols)), 1024, 0, st>>>(a.parts, (long long)p.B * p.blocks, p.tiles, s.K, s.C,
                                                                                                 a.grad_weight, a.grad_bias);
        return hipGetLastError();
    });
}

hipError_t launch_convolution_step(const esrnn_convolution_step_shape &s, const void *x, const float *weight, const float *bias, const int32_t *slots,
                                   void *state, void *out, hipStream_t st)
{
    return with_element(s.dtype, [&](auto e) {
        typedef decltype(e) E;
        constexpr int kWide = kThreads * 16 / (int)sizeof(E);
        const int tiles = (s.C + kWide - 1) / kWide;
        return with_taps(s.K, [&](auto k) {
            convolution_step_kernel<E, decltype(k)::value><<<dim3(s.rows * tiles), kThreads, 0, st>>>(
                s, static_cast<const E *>(x), weight, bias, slots, static_cast<E *>(state), static_cast<E *>(out), tiles);
            return hipGetLastError();
        });
    });
}

}  // namespace esrnn
