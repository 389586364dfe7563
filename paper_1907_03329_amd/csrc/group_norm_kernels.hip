// Group norm with activation, channels last (include/esrnn_layers.h), forward and reverse.
//
//   forward   mean and variance of a group (positions of a sample x neighbouring channels), then  u = xhat scale + shift,  out = act(u)
//   reverse   du = grad_out act'(u);  P1_c = sum over positions of du, P2_c of du xhat;  grad_shift, grad_scale: their sums over samples;
//             S1 = sum over the group's channels of scale P1, S2 of scale P2;  grad_x = rstd (scale du - (S1 + xhat S2) / M),
//             M the elements of the group that exist
//
// Four ways, by size alone, all with sums in fp32 and variances from differences to a mean (of the group where the data stay on
// chip, else of a thread's rows, put together pairwise by count: sums of squares would lose the variance of data far from zero); out and grad_x are
// rounded once, to nearest, as they are stored:
//   sample   a workgroup holds all positions of some groups of a sample in registers: x is read once, one launch.  16 x 72 x 40 fp32: 6.9 us with its
//            launch, of which the call on the host is 5.5.
//   position T = 1: a wave has one or several samples with all their channels; sums over a group pass through the wave's own LDS.
//            16384 x 2048 bf16 in 16 groups: forward 30 us among other passes, 4.5 TB/s, reverse 46 us with the sums over samples (under the profiler 32
//            and 44 + 5); the vector ALU is busy for all (forward) and 86 % of the cycles, with the sigmoid, its derivative and the conversions of 16 bits.
//   wide     T = 1, groups of 513 to 4096 channels: a workgroup has a group.  16384 x 2048 bf16 in one group: 27 and 60 us, the latter for bytes that
//            a copy moves in 40, and why has not been measured (a wave for each group: 68, 245).
//   stream   anything else: sums per channel and chunk of positions, sums per group (and of the gradients over samples), the result; three launches,
//            x read twice, the second time from the last-level cache where it fits.  6 ragged samples of up to 16384 positions of 256 channels, bf16:
//            forward 11 + 5 + 18 us, reverse 22 + 6 + 27, where 25 M elements at most are 50 MB an array.  Memory and last-level cache are the bound,
//            and the vector ALU near it (68 to 79 % of the cycles).
#include <algorithm>

#include "layers_internal.h"

namespace esrnn {

namespace {

__device__ __forceinline__ f32x4 splat(float v) { return f32x4{v, v, v, v}; }

struct Norm {
    const void *x, *grad_out;
    void *out, *grad_x;
    const int32_t *lengths;
    const float *scale, *shift, *stats_in;
    float *stats, *parts, *grad_scale, *grad_shift;
    int N, T, C, G, D;          // D channels a group
    int silu;
    float eps;
    int tile, tiles, log_w;     // channels of a workgroup, workgroups of a sample, log2 of the lanes side by side (sample way)
    int chunk, chunks;          // positions of a workgroup, workgroups along positions (stream way)
    int wave_pairs;             // LDS of a wave (position way)
};

__device__ __forceinline__ int length_of(const Norm &a, int n) { return a.lengths ? min(max(a.lengths[n], 0), a.T) : a.T; }

// (zero where exp(-u) is above 2^126, u < -87.3)
__device__ __forceinline__ float sigmoid_of(float u) { return fast_rcp(1.0f + __builtin_amdgcn_exp2f(u * kSigmoidExponent)); }
__device__ __forceinline__ float activate(float u, int silu) { return silu ? u * sigmoid_of(u) : u; }
// derivative of u s, s = sigmoid(u): s + u s (1 - s).  (Of 1 - s only as much counts as the sum has room for.)
__device__ __forceinline__ float slope(float u, int silu)
{
    if (!silu) return 1.0f;
    const float s = sigmoid_of(u);
    return u * s * (1.0f - s) + s;
}

// 1 / sqrt, to a unit in the last place.  The hardware's reciprocal root is infinite for denormals, and eps may be one where a constant group has no
// variance.  (Root and division as the compiler rounds them take the wide way's forward pass from 27 to 30 us, 16384 x 2048 bf16.)
__device__ __forceinline__ float rstd_of(float variance_and_eps)
{
    const int up = variance_and_eps < 0x1p-100f ? 32 : 0;
    return __builtin_ldexpf(__builtin_amdgcn_rsqf(__builtin_ldexpf(variance_and_eps, 2 * up)), up);
}

// The gradient of an input, from du, the sums over its group (by the group's elements) and what is normalised.  The product is rounded before the
// first sum is taken off, as it was in that sum: a group of one element has no gradient, and gets exactly none.
__device__ __forceinline__ f32x4 input_gradient(f32x4 rstd, f32x4 scale, f32x4 du, f32x4 s1, f32x4 xhat, f32x4 s2)
{
    f32x4 own;
    {
#pragma clang fp contract(off)
        own = scale * du;
    }
    return rstd * ((own - s1) - xhat * s2);
}

// ---- sample ------------------------------------------------------------------------------------------------------
// Channels of a tile [begin, begin + count), dealt to w = 2^log_w lanes; w and the tile are the launch's.
template <bool kAligned>
struct TileChannels {
    int begin, count, w, lane;
    __device__ __forceinline__ int at(int k) const { return kAligned ? 4 * lane + k : lane + w * k; }
    __device__ __forceinline__ bool exists(int k) const { return at(k) < count; }
    template <class E>
    __device__ __forceinline__ Vec4<E> load(const E *row) const     // of channel 0; some channel of the tile for those that do not exist
    {
        if constexpr (kAligned) return *reinterpret_cast<const Vec4<E> *>(row + begin + min(4 * lane, count - 4));
        Vec4<E> v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = row[begin + min(at(k), count - 1)];
        return v;
    }
    template <class E>
    __device__ __forceinline__ void store(E *row, Vec4<E> v) const
    {
        if constexpr (kAligned) {
            if (exists(0)) *reinterpret_cast<Vec4<E> *>(row + begin + 4 * lane) = v;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (exists(k)) row[begin + at(k)] = v[k];
        }
    }
    __device__ __forceinline__ f32x4 parameters(const float *p) const       // (any alignment)
    {
        f32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = p[begin + min(at(k), count - 1)];
        return v;
    }
};

// Sums over the workgroup's rows, and over the channels of each group.  NV values a channel.
template <int NT, int NV, bool kAligned>
struct TileSums {
    // channel sums of each wave [slots][NV][tile], of the workgroup [NV][tile] (in the first slot's place), sums of groups [groups][NV]
    float *part, *group;
    int slots, tile, D;
    __device__ __forceinline__ void channels(f32x4 (&v)[NV], const TileChannels<kAligned> &ch, int log_w)
    {
        const int w = 1 << log_w, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        for (int off = w; off < 64; off *= 2)
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) v[i][k] += __shfl_xor(v[i][k], off, 64);
        const int slot = w >= 64 ? (int)threadIdx.x >> log_w : wave;
        if (lane < w)
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (ch.exists(k)) part[(slot * NV + i) * tile + ch.at(k)] = v[i][k];
        __syncthreads();
        for (int at = threadIdx.x; at < NV * tile; at += NT) {
            float sum[4] = {part[at], 0.0f, 0.0f, 0.0f};
            int s = 1;
            for (; s + 4 <= slots; s += 4)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] += part[(s + i) * NV * tile + at];
            for (; s < slots; ++s) sum[0] += part[s * NV * tile + at];
            part[at] = (sum[0] + sum[1]) + (sum[2] + sum[3]);
        }
        __syncthreads();
    }
    __device__ __forceinline__ float channel(int i, int c) const { return part[i * tile + c]; }
    // behind channels(): a wave a group; weight: of a channel
    template <class W>
    __device__ __forceinline__ void groups(W &&weight)
    {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        for (int g = wave; g * D < tile; g += NT / 64) {
            float sum[NV] = {};
            for (int c = lane; c < D; c += 64) {
                const float f = weight(g * D + c);
#pragma unroll
                for (int i = 0; i < NV; ++i) sum[i] += f * channel(i, g * D + c);
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                sum[i] = wave_sum(sum[i]);
                if (lane == 0) group[g * NV + i] = sum[i];
            }
        }
        __syncthreads();
    }
};

// channels of a workgroup of the sample way
constexpr int most_tile(int threads) { return threads * 4 < 1024 ? threads * 4 : 1024; }

template <class E, bool kAligned, int NT, int K, bool kSilu>
__global__ void __launch_bounds__(NT) norm_sample_forward_kernel(Norm a)
{
    __shared__ float part[NT / 64 * 256], group[most_tile(NT)];
    const int n = blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles, rows = NT >> a.log_w, row = (int)threadIdx.x >> a.log_w;
    const TileChannels<kAligned> ch{tile * a.tile, min(a.tile, a.C - tile * a.tile), 1 << a.log_w, (int)threadIdx.x & ((1 << a.log_w) - 1)};
    const int length = length_of(a, n);
    const E *x = static_cast<const E *>(a.x) + (size_t)n * a.T * a.C;
    E *out = static_cast<E *>(a.out) + (size_t)n * a.T * a.C;
    Vec4<E> xs[K];
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (K == 1 || k * rows < a.T) xs[k] = ch.load(x + (size_t)min(row + k * rows, a.T - 1) * a.C);
    const f32x4 scale = ch.parameters(a.scale), shift = ch.parameters(a.shift);
    TileSums<NT, 1, kAligned> sums{part, group, a.log_w >= 6 ? rows : NT / 64, ch.count, a.D};
    int g[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) g[k] = min(ch.at(k), ch.count - 1) / a.D;
    const float inverse = length > 0 ? 1.0f / ((float)length * (float)a.D) : 0.0f;
    f32x4 mean, rstd, v[1] = {splat(0.0f)};
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (row + k * rows < length) v[0] += to_f32<E>(xs[k]);
    sums.channels(v, ch, a.log_w);
    sums.groups([](int) { return 1.0f; });
#pragma unroll
    for (int k = 0; k < 4; ++k) mean[k] = group[g[k]] * inverse;
    v[0] = splat(0.0f);
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (row + k * rows < length) {
            const f32x4 d = to_f32<E>(xs[k]) - mean;
            v[0] += d * d;
        }
    sums.channels(v, ch, a.log_w);      // (a barrier between the reads of `group` above and its next writes)
    sums.groups([](int) { return 1.0f; });
#pragma unroll
    for (int k = 0; k < 4; ++k) rstd[k] = 1.0f / sqrtf(group[g[k]] * inverse + a.eps);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int t = row + k * rows;
        if (t >= a.T) break;
        f32x4 y = (to_f32<E>(xs[k]) - mean) * rstd * scale + shift;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = activate(y[i], kSilu);
        ch.store(out + (size_t)t * a.C, from_f32<E>(t < length ? y : splat(0.0f)));
    }
    if (a.stats && row == 0)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (ch.exists(k) && ch.at(k) % a.D == 0) {
                float *s = a.stats + ((size_t)n * a.G + tile * a.tile / a.D + g[k]) * 2;
                s[0] = mean[k];
                s[1] = rstd[k];
            }
}

template <class E, bool kAligned, int NT, int K, bool kSilu>
__global__ void __launch_bounds__(NT) norm_sample_backward_kernel(Norm a)
{
    __shared__ float part[NT / 64 * 256 * 2], group[most_tile(NT) * 2];
    const int n = blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles, rows = NT >> a.log_w, row = (int)threadIdx.x >> a.log_w;
    const TileChannels<kAligned> ch{tile * a.tile, min(a.tile, a.C - tile * a.tile), 1 << a.log_w, (int)threadIdx.x & ((1 << a.log_w) - 1)};
    const int length = length_of(a, n);
    const size_t base = (size_t)n * a.T * a.C;
    const E *x = static_cast<const E *>(a.x) + base, *grad_out = static_cast<const E *>(a.grad_out) + base;
    E *grad_x = static_cast<E *>(a.grad_x) + base;
    Vec4<E> xs[K], ds[K];
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (K == 1 || k * rows < a.T) {
            const size_t at = (size_t)min(row + k * rows, a.T - 1) * a.C;
            xs[k] = ch.load(x + at);
            ds[k] = ch.load(grad_out + at);
        }
    const f32x4 scale = ch.parameters(a.scale), shift = ch.parameters(a.shift);
    f32x4 mean, rstd;
    int g[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        g[k] = min(ch.at(k), ch.count - 1) / a.D;
        const float *s = a.stats_in + ((size_t)n * a.G + tile * a.tile / a.D + g[k]) * 2;
        mean[k] = s[0];
        rstd[k] = s[1];
    }
    TileSums<NT, 2, kAligned> sums{part, group, a.log_w >= 6 ? rows : NT / 64, ch.count, a.D};
    f32x4 v[2] = {splat(0.0f), splat(0.0f)};
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (row + k * rows < length) {
            const f32x4 xhat = (to_f32<E>(xs[k]) - mean) * rstd, u = xhat * scale + shift;
            f32x4 du = to_f32<E>(ds[k]);
#pragma unroll
            for (int i = 0; i < 4; ++i) du[i] *= slope(u[i], kSilu);
            v[0] += du;
            v[1] += du * xhat;
        }
    sums.channels(v, ch, a.log_w);
    for (int c = threadIdx.x; c < ch.count; c += NT) {      // sums of the sample, to be added up over the samples
        a.parts[((size_t)n * 2) * a.C + ch.begin + c] = sums.channel(0, c);
        a.parts[((size_t)n * 2 + 1) * a.C + ch.begin + c] = sums.channel(1, c);
    }
    sums.groups([&](int c) { return a.scale[ch.begin + c]; });
    const float inverse = length > 0 ? 1.0f / ((float)length * (float)a.D) : 0.0f;
    f32x4 s1, s2;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        s1[k] = group[2 * g[k]] * inverse;
        s2[k] = group[2 * g[k] + 1] * inverse;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int t = row + k * rows;
        if (t >= a.T) break;
        const f32x4 xhat = (to_f32<E>(xs[k]) - mean) * rstd, u = xhat * scale + shift;
        f32x4 du = to_f32<E>(ds[k]);
#pragma unroll
        for (int i = 0; i < 4; ++i) du[i] *= slope(u[i], kSilu);
        const f32x4 gx = input_gradient(rstd, scale, du, s1, xhat, s2);
        ch.store(grad_x + (size_t)t * a.C, from_f32<E>(t < length ? gx : splat(0.0f)));
    }
}

// ---- position ----------------------------------------------------------------------------------------------------
// T = 1.  Groups of one sample have nothing to do with each other, so a wave has a tile of whole groups, some 256 channels, of R samples at
// once, or of R 64 / w where w < 64 lanes hold the tile's channels.  What a group adds up goes through the wave's own part of LDS: of
// four channels together where groups consist of such fours (kQuads), else channel by channel.  A group wider than 256 channels
// is a tile, in J chunks of 256, and is added up over the lanes.  No other wave takes part, so nothing waits at a barrier.
struct Pair {
    float a, b;
};
template <bool kAligned, bool kQuads, int J, int R>
struct Tile {
    static_assert(kAligned || !kQuads || J > 1, "");
    static constexpr int kEach = kQuads ? 1 : 4;        // entries of a lane and chunk
    int begin, count, D, groups, log_w, lane, row, rows;        // first channel, channels; row: of the wave's `rows` for each of R
    Pair *entries, *sums;
    int n, log_s, part, item_row, item_group;

    __device__ __forceinline__ Tile(const Norm &a, Pair *lds)
        : begin(blockIdx.x % a.tiles * a.tile), count(min(a.tile, a.C - begin)), D(a.D), groups(count / a.D), log_w(a.log_w),
          lane(threadIdx.x & ((1 << a.log_w) - 1)), row((threadIdx.x & 63) >> a.log_w), rows(64 >> a.log_w)
    {
        entries = lds + (threadIdx.x >> 6) * a.wave_pairs;
        sums = entries + R * rows * row_entries();
        n = kQuads ? D / 4 : D;
        const int items = R * rows * groups;
        for (log_s = 0; items << (log_s + 1) <= 64 && 1 << log_s < n; ++log_s) {}      // lanes that share a group
        const int l = threadIdx.x & 63;
        part = l & ((1 << log_s) - 1);
        item_row = (l >> log_s) / groups;
        item_group = (l >> log_s) - item_row * groups;
    }
    __device__ __forceinline__ int channel(int j, int k) const { return (j << (log_w + 2)) + (kAligned ? 4 * lane + k : lane + (k << log_w)); }
    __device__ __forceinline__ bool exists(int j, int k) const { return channel(j, k) < count; }
    // samples first + r rows, r = 0 .. R - 1, and the wave's others behind each; `there`: this lane's sample exists
    template <class E>
    __device__ __forceinline__ Vec4<E> load(const E *x, int first, int r, int j, bool there, int C) const
    {
        const E *p = x + (size_t)(first + r * rows) * C + begin;
        if constexpr (kAligned) return load_four<E>(make_base(p), there && exists(j, 0) ? (row * C + channel(j, 0)) * (unsigned)sizeof(E) : kOutside);
        Vec4<E> v = {};
        if (there)
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = p[(size_t)row * C + min(channel(j, k), count - 1)];
        return v;
    }
    template <class E>
    __device__ __forceinline__ void store(E *x, int first, int r, int j, bool there, int C, Vec4<E> v) const
    {
        E *p = x + (size_t)(first + r * rows) * C + begin;
        if constexpr (kAligned) {
            store_four<E>(make_base(p), there && exists(j, 0) ? (row * C + channel(j, 0)) * (unsigned)sizeof(E) : kOutside, v);
        } else if (there) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (exists(j, k)) p[(size_t)row * C + channel(j, k)] = v[k];
        }
    }
    __device__ __forceinline__ f32x4 parameters(const float *p, int j) const
    {
        f32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = p[begin + min(channel(j, k), count - 1)];
        return v;
    }
    __device__ __forceinline__ int group(int j, int k) const { return min(channel(j, k), count - 1) / D; }
    __device__ __forceinline__ f32x4 existing(f32x4 v, int j) const
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = exists(j, k) ? v[k] : 0.0f;
        return v;
    }

    // Entries of a group lie side by side; a place of padding after 16 keeps lanes that read at the distance of a group off each other's banks.
    __device__ static __forceinline__ int padded(int i) { return i + (i >> 4); }
    __device__ __forceinline__ int row_entries() const { return padded(J * kEach << log_w); }
    __device__ __forceinline__ Pair &entry(int r, int j, int k) const
    {
        return entries[(r * rows + row) * row_entries() + padded(kQuads ? (j << log_w) + lane : channel(j, k))];
    }
    __device__ __forceinline__ Pair sum(int r, int g) const { return sums[(r * rows + row) * groups + g]; }
    // f(entries of a group, this lane's first one, step between them, group's place in sums, whether this lane writes it) for every group of the
    // wave; the lanes of a group follow each other, 2^log_s of them
    template <class F>
    __device__ __forceinline__ void for_groups(F &&f) const
    {
        ordered();
        int r = item_row, g = item_group;
        for (int item = 0; item < R * rows * groups; item += 64 >> log_s) {
            const bool there = r < R * rows;
            const Pair *mine = entries + (there ? r : 0) * row_entries();
            const int at = (there ? g : 0) * n;
            f([&](int i) { return mine[padded(at + i)]; }, there, r * groups + g);
            g += 64 >> log_s;
            while (g >= groups) {
                g -= groups;
                ++r;
            }
        }
        ordered();
    }
    __device__ __forceinline__ float over_lanes(float v) const
    {
        for (int off = 1; off < 1 << log_s; off *= 2) v += __shfl_xor(v, off, 64);
        return v;
    }
    __device__ static __forceinline__ void ordered()
    {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
};

extern __shared__ float s_dynamic[];

template <class E, bool kAligned, bool kQuads, int J, int R, bool kSilu>
__global__ void __launch_bounds__(256) norm_position_forward_kernel(Norm a)
{
    constexpr int kEach = kQuads ? 1 : 4;
    const Tile<kAligned, kQuads, J, R> tile(a, reinterpret_cast<Pair *>(s_dynamic));
    int g[J][kEach];
    f32x4 scale[J], shift[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
#pragma unroll
        for (int k = 0; k < kEach; ++k) g[j][k] = tile.group(j, k);
        scale[j] = tile.parameters(a.scale, j);
        shift[j] = tile.parameters(a.shift, j);
    }
    const float inverse = 1.0f / (float)a.D;
    const int stride = R * tile.rows, step = (int)(gridDim.x / a.tiles) * 4 * stride;
    const E *x = static_cast<const E *>(a.x);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int first = ((int)(blockIdx.x / a.tiles) * 4 + wave) * stride; first < a.N; first += step) {
        Vec4<E> xs[R][J];
        bool there[R], valid[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int n = first + r * tile.rows + tile.row;
            there[r] = n < a.N;
            valid[r] = there[r] && length_of(a, min(n, a.N - 1)) > 0;
#pragma unroll
            for (int j = 0; j < J; ++j) xs[r][j] = tile.load(x, first, r, j, there[r], a.C);
        }
        Pair only{0.0f, 0.0f};      // J > 1: mean and rstd of the one group
        if constexpr (J > 1) {
            f32x4 sum = splat(0.0f);
#pragma unroll
            for (int j = 0; j < J; ++j) sum += tile.existing(to_f32<E>(xs[0][j]), j);
            only.a = wave_sum((sum[0] + sum[1]) + (sum[2] + sum[3])) * inverse;
            sum = splat(0.0f);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const f32x4 d = tile.existing(to_f32<E>(xs[0][j]) - only.a, j);
                sum += d * d;
            }
            only.b = rstd_of(wave_sum((sum[0] + sum[1]) + (sum[2] + sum[3])) * inverse + a.eps);
            if (a.stats && (threadIdx.x & 63) == 0) reinterpret_cast<Pair *>(a.stats)[(size_t)first * a.G + tile.begin / a.D] = only;
        }
        // four channels: their mean and the sum of squared differences to it; a channel by itself: its value
#pragma unroll
        for (int r = 0; r < R && J == 1; ++r)
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const f32x4 v = to_f32<E>(xs[r][j]);
                if (kQuads) {
                    const float mean = 0.25f * ((v[0] + v[1]) + (v[2] + v[3]));
                    const f32x4 d = v - mean;
                    tile.entry(r, j, 0) = Pair{mean, (d[0] * d[0] + d[1] * d[1]) + (d[2] * d[2] + d[3] * d[3])};
                } else {
#pragma unroll
                    for (int k = 0; k < kEach; ++k) tile.entry(r, j, k) = Pair{v[k], 0.0f};
                }
            }
        if constexpr (J == 1) tile.for_groups([&](auto &&entry, bool there, int to) {
            float sum = 0.0f, square = 0.0f;
            for (int i = tile.part; i < tile.n; i += 1 << tile.log_s) sum += entry(i).a;
            const float mean = tile.over_lanes(sum) * (kQuads ? 4.0f * inverse : inverse);
            for (int i = tile.part; i < tile.n; i += 1 << tile.log_s) {
                const Pair e = entry(i);
                const float d = e.a - mean;
                square += kQuads ? e.b + 4.0f * d * d : d * d;
            }
            const float rstd = rstd_of(tile.over_lanes(square) * inverse + a.eps);
            if (there && tile.part == 0) tile.sums[to] = Pair{mean, rstd};
        });
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const f32x4 v = to_f32<E>(xs[r][j]);
                f32x4 y;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const Pair s = J > 1 ? only : tile.sum(r, g[j][kQuads ? 0 : k]);
                    y[k] = activate((v[k] - s.a) * s.b * scale[j][k] + shift[j][k], kSilu);
                }
                tile.store(static_cast<E *>(a.out), first, r, j, there[r], a.C, valid[r] ? from_f32<E>(y) : Vec4<E>{});
            }
        }
        if (a.stats && J == 1)
            for (int i = threadIdx.x & 63; i < stride * tile.groups; i += 64) {
                const int r = i / tile.groups;
                if (first + r < a.N) reinterpret_cast<Pair *>(a.stats)[(size_t)(first + r) * a.G + tile.begin / a.D + i - r * tile.groups] = tile.sums[i];
            }
        tile.ordered();
    }
}

template <class E, bool kAligned, bool kQuads, int J, int R, bool kSilu>
__global__ void __launch_bounds__(256) norm_position_backward_kernel(Norm a)
{
    constexpr int kEach = kQuads ? 1 : 4;
    const Tile<kAligned, kQuads, J, R> tile(a, reinterpret_cast<Pair *>(s_dynamic));
    int g[J][kEach];
    f32x4 scale[J], shift[J], p1[J], p2[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
#pragma unroll
        for (int k = 0; k < kEach; ++k) g[j][k] = tile.group(j, k);
        scale[j] = tile.parameters(a.scale, j);
        shift[j] = tile.parameters(a.shift, j);
        p1[j] = p2[j] = splat(0.0f);
    }
    const float inverse = 1.0f / (float)a.D;
    const int stride = R * tile.rows, step = (int)(gridDim.x / a.tiles) * 4 * stride;
    const E *x = static_cast<const E *>(a.x), *grad_out = static_cast<const E *>(a.grad_out);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int first = ((int)(blockIdx.x / a.tiles) * 4 + wave) * stride; first < a.N; first += step) {
        Vec4<E> xs[R][J], ds[R][J];
        Pair stats[R][J][kEach];        // (of four channels: of their group)
        bool there[R], valid[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int at = first + r * tile.rows + tile.row, n = min(at, a.N - 1);
            there[r] = at < a.N;
            valid[r] = there[r] && length_of(a, n) > 0;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                xs[r][j] = tile.load(x, first, r, j, there[r], a.C);
                ds[r][j] = tile.load(grad_out, first, r, j, there[r], a.C);
#pragma unroll
                for (int k = 0; k < kEach; ++k)
                    stats[r][j][k] = reinterpret_cast<const Pair *>(a.stats_in)[(size_t)n * a.G + tile.begin / a.D + g[j][k]];
            }
        }
        f32x4 xhat[R][J], du[R][J];
        Pair only{0.0f, 0.0f};
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const f32x4 v = to_f32<E>(xs[r][j]), d = to_f32<E>(ds[r][j]);
                f32x4 own;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const Pair s = stats[r][j][kQuads ? 0 : k];
                    xhat[r][j][k] = (v[k] - s.a) * s.b;
                    du[r][j][k] = d[k] * slope(xhat[r][j][k] * scale[j][k] + shift[j][k], kSilu);
                }
                if (!valid[r]) xhat[r][j] = du[r][j] = splat(0.0f);
                p1[j] += du[r][j];
                p2[j] += du[r][j] * xhat[r][j];
                {
#pragma clang fp contract(off)
                    own = scale[j] * du[r][j];      // (as in input_gradient)
                }
                const f32x4 along = own * xhat[r][j];
                if (J > 1) {
                    const f32x4 o = tile.existing(own, j), l = tile.existing(along, j);
                    only.a += (o[0] + o[1]) + (o[2] + o[3]);
                    only.b += (l[0] + l[1]) + (l[2] + l[3]);
                } else if (kQuads) tile.entry(r, j, 0) = Pair{(own[0] + own[1]) + (own[2] + own[3]), (along[0] + along[1]) + (along[2] + along[3])};
                else
#pragma unroll
                    for (int k = 0; k < kEach; ++k) tile.entry(r, j, k) = Pair{own[k], along[k]};
            }
        if (J > 1) only = Pair{wave_sum(only.a) * inverse, wave_sum(only.b) * inverse};
        if constexpr (J == 1) tile.for_groups([&](auto &&entry, bool there, int to) {
            Pair sum{0.0f, 0.0f};
            for (int i = tile.part; i < tile.n; i += 1 << tile.log_s) {
                const Pair e = entry(i);
                sum.a += e.a;
                sum.b += e.b;
            }
            sum.a = tile.over_lanes(sum.a) * inverse;
            sum.b = tile.over_lanes(sum.b) * inverse;
            if (there && tile.part == 0) tile.sums[to] = sum;
        });
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int j = 0; j < J; ++j) {
                f32x4 s1, s2, rstd;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const Pair s = J > 1 ? only : tile.sum(r, g[j][kQuads ? 0 : k]);
                    s1[k] = s.a;
                    s2[k] = s.b;
                    rstd[k] = stats[r][j][kQuads ? 0 : k].b;
                }
                const f32x4 gx = input_gradient(rstd, scale[j], du[r][j], s1, xhat[r][j], s2);
                tile.store(static_cast<E *>(a.grad_x), first, r, j, there[r], a.C, valid[r] ? from_f32<E>(gx) : Vec4<E>{});
            }
        }
        tile.ordered();
    }
    // the wave's rows, then the waves one behind the other: parts [workgroups of a tile][2][C]
    for (int off = 1 << a.log_w; off < 64; off *= 2)
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                p1[j][k] += __shfl_xor(p1[j][k], off, 64);
                p2[j][k] += __shfl_xor(p2[j][k], off, 64);
            }
    for (int w = 0; w < 4; ++w) {
        __syncthreads();
        if (wave != w || tile.row != 0) continue;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (tile.exists(j, k)) {
                    const int c = tile.channel(j, k);
                    s_dynamic[c] = w ? s_dynamic[c] + p1[j][k] : p1[j][k];
                    s_dynamic[a.tile + c] = w ? s_dynamic[a.tile + c] + p2[j][k] : p2[j][k];
                }
    }
    __syncthreads();
    float *parts = a.parts + (size_t)(blockIdx.x / a.tiles) * 2 * a.C + tile.begin;
    for (int c = threadIdx.x; c < tile.count; c += 256) {
        parts[c] = s_dynamic[c];
        parts[a.C + c] = s_dynamic[a.tile + c];
    }
}

// Groups of more than 512 channels: a workgroup has one group of R samples, J chunks of 1024 channels, and adds up over its waves.
template <bool kAligned, int J>
struct WideRow {
    int begin, count;
    __device__ __forceinline__ int channel(int j, int k) const { return 1024 * j + (kAligned ? 4 * (int)threadIdx.x + k : (int)threadIdx.x + 256 * k); }
    __device__ __forceinline__ bool exists(int j, int k) const { return channel(j, k) < count; }
    template <class E>
    __device__ __forceinline__ Vec4<E> load(const E *p, int j) const
    {
        if constexpr (kAligned) return *reinterpret_cast<const Vec4<E> *>(p + begin + min(channel(j, 0), count - 4));
        Vec4<E> v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = p[begin + min(channel(j, k), count - 1)];
        return v;
    }
    template <class E>
    __device__ __forceinline__ void store(E *p, int j, Vec4<E> v) const
    {
        if constexpr (kAligned) {
            if (exists(j, 0)) *reinterpret_cast<Vec4<E> *>(p + begin + channel(j, 0)) = v;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (exists(j, k)) p[begin + channel(j, k)] = v[k];
        }
    }
    __device__ __forceinline__ f32x4 parameters(const float *p, int j) const
    {
        f32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = p[begin + min(channel(j, k), count - 1)];
        return v;
    }
    __device__ __forceinline__ f32x4 existing(f32x4 v, int j) const
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = exists(j, k) ? v[k] : 0.0f;
        return v;
    }
};
// N sums over the workgroup at once; `shared`: [4][N], not written again before the next barrier but one
template <int N>
__device__ __forceinline__ void workgroup_sums(float (&v)[N], float (*shared)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = wave_sum(v[i]);
        if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6][i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (shared[0][i] + shared[1][i]) + (shared[2][i] + shared[3][i]);
}
__device__ __forceinline__ float across(f32x4 v) { return (v[0] + v[1]) + (v[2] + v[3]); }

template <class E, bool kAligned, int J, bool kSilu>
__global__ void __launch_bounds__(256) norm_wide_forward_kernel(Norm a)
{
    constexpr int R = 4 / J;
    __shared__ float s_sum[2][4][R];
    const int g = blockIdx.x % a.G;
    const WideRow<kAligned, J> row{g * a.D, a.D};
    f32x4 scale[J], shift[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        scale[j] = row.parameters(a.scale, j);
        shift[j] = row.parameters(a.shift, j);
    }
    const float inverse = 1.0f / (float)a.D;
    const E *x = static_cast<const E *>(a.x);
    for (int first = (int)(blockIdx.x / a.G) * R; first < a.N; first += (int)(gridDim.x / a.G) * R) {
        f32x4 v[R][J];
        float sum[R], square[R];
        {
            Vec4<E> xs[R][J];
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int j = 0; j < J; ++j) xs[r][j] = row.load(x + (size_t)min(first + r, a.N - 1) * a.C, j);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                f32x4 all = splat(0.0f);
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    v[r][j] = to_f32<E>(xs[r][j]);
                    all += row.existing(v[r][j], j);
                }
                sum[r] = across(all);
            }
        }
        workgroup_sums(sum, s_sum[0]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            f32x4 all = splat(0.0f);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                v[r][j] -= sum[r] * inverse;
                const f32x4 d = row.existing(v[r][j], j);
                all += d * d;
            }
            square[r] = across(all);
        }
        workgroup_sums(square, s_sum[1]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int n = first + r;
            if (n >= a.N) break;
            const float rstd = rstd_of(square[r] * inverse + a.eps);
            const bool valid = length_of(a, n) > 0;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                f32x4 y = v[r][j] * rstd * scale[j] + shift[j];
#pragma unroll
                for (int k = 0; k < 4; ++k) y[k] = activate(y[k], kSilu);
                row.store(static_cast<E *>(a.out) + (size_t)n * a.C, j, valid ? from_f32<E>(y) : Vec4<E>{});
            }
            if (a.stats && threadIdx.x == 0) reinterpret_cast<Pair *>(a.stats)[(size_t)n * a.G + g] = Pair{sum[r] * inverse, rstd};
        }
    }
}

template <class E, bool kAligned, int J, bool kSilu>
__global__ void __launch_bounds__(256) norm_wide_backward_kernel(Norm a)
{
    constexpr int R = 4 / J;
    __shared__ float s_sum[2][4][2 * R];
    const int g = blockIdx.x % a.G;
    const WideRow<kAligned, J> row{g * a.D, a.D};
    f32x4 scale[J], shift[J], p1[J], p2[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        scale[j] = row.parameters(a.scale, j);
        shift[j] = row.parameters(a.shift, j);
        p1[j] = p2[j] = splat(0.0f);
    }
    const float inverse = 1.0f / (float)a.D;
    const E *x = static_cast<const E *>(a.x), *grad_out = static_cast<const E *>(a.grad_out);
    int turn = 0;
    for (int first = (int)(blockIdx.x / a.G) * R; first < a.N; first += (int)(gridDim.x / a.G) * R) {
        Vec4<E> xs[R][J], ds[R][J];
        Pair stats[R];
        f32x4 xhat[R][J], du[R][J];
        float sum[2 * R];
        bool valid[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int n = min(first + r, a.N - 1);
            valid[r] = first + r < a.N && length_of(a, n) > 0;
            stats[r] = reinterpret_cast<const Pair *>(a.stats_in)[(size_t)n * a.G + g];
#pragma unroll
            for (int j = 0; j < J; ++j) {
                xs[r][j] = row.load(x + (size_t)n * a.C, j);
                ds[r][j] = row.load(grad_out + (size_t)n * a.C, j);
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            f32x4 s1 = splat(0.0f), s2 = splat(0.0f);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                xhat[r][j] = (to_f32<E>(xs[r][j]) - stats[r].a) * stats[r].b;
                du[r][j] = to_f32<E>(ds[r][j]);
                f32x4 own;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    du[r][j][k] *= slope(xhat[r][j][k] * scale[j][k] + shift[j][k], kSilu);
                    if (!(valid[r] && row.exists(j, k))) du[r][j][k] = xhat[r][j][k] = 0.0f;
                }
                p1[j] += du[r][j];
                p2[j] += du[r][j] * xhat[r][j];
                own = scale[j] * du[r][j];
                s1 += own;
                s2 += own * xhat[r][j];
            }
            sum[2 * r] = across(s1);
            sum[2 * r + 1] = across(s2);
        }
        workgroup_sums(sum, s_sum[turn]);
        turn ^= 1;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int n = first + r;
            if (n >= a.N) break;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const f32x4 gx = input_gradient(splat(stats[r].b), scale[j], du[r][j], splat(sum[2 * r] * inverse), xhat[r][j], splat(sum[2 * r + 1] * inverse));
                row.store(static_cast<E *>(a.grad_x) + (size_t)n * a.C, j, valid[r] ? from_f32<E>(gx) : Vec4<E>{});
            }
        }
    }
    float *parts = a.parts + (size_t)(blockIdx.x / a.G) * 2 * a.C + row.begin;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (row.exists(j, k)) {
                parts[row.channel(j, k)] = p1[j][k];
                parts[a.C + row.channel(j, k)] = p2[j][k];
            }
}

// Sums of 64 channels over `rows` rows at a distance of 2 C, by a workgroup of NW waves, which take every NW-th row.
template <int NW>
__device__ __forceinline__ void sum_rows_of_tile(const float *__restrict__ parts, int rows, int C, int tile, float *__restrict__ to)
{
    __shared__ float s_sum[NW][64];
    constexpr int kAtOnce = 8;
    const int lane = threadIdx.x & 63, c = tile * 64 + lane, wave = threadIdx.x >> 6;
    const float *p = parts + min(c, C - 1);
    float sum[kAtOnce] = {};
    int r = wave;
    for (; r + (kAtOnce - 1) * NW < rows; r += kAtOnce * NW)
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) sum[i] += p[(size_t)(r + NW * i) * 2 * C];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i)
        if (r + NW * i < rows) sum[i] += p[(size_t)(r + NW * i) * 2 * C];
    s_sum[wave][lane] = ((sum[0] + sum[1]) + (sum[2] + sum[3])) + ((sum[4] + sum[5]) + (sum[6] + sum[7]));
    __syncthreads();
    if (wave != 0 || c >= C) return;
    float all = 0.0f;
    for (int w = 0; w < NW; ++w) all += s_sum[w][lane];
    to[c] = all;
}
// [rows][2][C], in gridDim.z runs: of several to [runs][2][C], of one to the gradients
__global__ void __launch_bounds__(1024) norm_sum_rows_kernel(const float *__restrict__ parts, int rows, int C, float *to_shift, float *to_scale)
{
    const int run = (rows + (int)gridDim.z - 1) / (int)gridDim.z, first = min((int)blockIdx.z * run, rows);
    sum_rows_of_tile<16>(parts + ((size_t)first * 2 + blockIdx.y) * C, min(run, rows - first), C, blockIdx.x,
                         (blockIdx.y ? to_scale : to_shift) + (size_t)blockIdx.z * 2 * C);
}

// ---- stream ------------------------------------------------------------------------------------------------------
// mean of n values, and the sum of squared differences to it
struct Moments {
    float n, mean, square;
    __device__ __forceinline__ void add(const Moments &o)
    {
        const float all = n + o.n, share = all > 0.0f ? o.n / all : 0.0f, delta = o.mean - mean;
        if (o.n > 0.0f) {
            mean += delta * share;
            square += o.square + delta * delta * n * share;
        }
        n = all;
    }
};

constexpr int kRows = 8;        // positions that a thread has in registers at once

// parts [N][chunks][2][C]: mean and sum of squared differences of a channel over a chunk's positions
template <class E, bool kAligned>
__global__ void __launch_bounds__(256) norm_moments_kernel(Norm a)
{
    __shared__ float s_mean[16][64], s_square[16][64];
    __shared__ int s_n[16];
    const int lane16 = threadIdx.x & 15, row = threadIdx.x >> 4;
    const int n = blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles, chunk = blockIdx.y;
    const Channels<kAligned, 16> ch(lane16, tile * 64, a.C);
    const int first = chunk * a.chunk, end = min(min(first + a.chunk, a.T), length_of(a, n));
    const E *x = static_cast<const E *>(a.x) + (size_t)n * a.T * a.C;
    f32x4 mean = splat(0.0f), square = splat(0.0f);
    int count = 0;
    for (int t0 = first; t0 < end; t0 += 16 * kRows) {
        Vec4<E> xs[kRows];
#pragma unroll
        for (int k = 0; k < kRows; ++k) xs[k] = ch.load(x + (size_t)min(t0 + row + 16 * k, end - 1) * a.C);
        int have = 0;
        f32x4 sum = splat(0.0f), sq = splat(0.0f);
#pragma unroll
        for (int k = 0; k < kRows; ++k)
            if (t0 + row + 16 * k < end) {
                sum += to_f32<E>(xs[k]);
                ++have;
            }
        if (!have) break;
        const f32x4 m = sum * (1.0f / (float)have);
#pragma unroll
        for (int k = 0; k < kRows; ++k)
            if (t0 + row + 16 * k < end) {
                const f32x4 d = to_f32<E>(xs[k]) - m;
                sq += d * d;
            }
        const float share = (float)have / (float)(count + have);
        const f32x4 delta = m - mean;
        square += sq + delta * delta * ((float)count * share);
        mean += delta * share;
        count += have;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        s_mean[row][kAligned ? 4 * lane16 + k : lane16 + 16 * k] = mean[k];
        s_square[row][kAligned ? 4 * lane16 + k : lane16 + 16 * k] = square[k];
    }
    if (lane16 == 0) s_n[row] = count;
    __syncthreads();
    const int c = tile * 64 + (int)threadIdx.x;
    if (threadIdx.x >= 64 || c >= a.C) return;
    Moments all{0.0f, 0.0f, 0.0f};
    for (int r = 0; r < 16; ++r) all.add(Moments{(float)s_n[r], s_mean[r][threadIdx.x], s_square[r][threadIdx.x]});
    float *p = a.parts + ((size_t)n * a.chunks + chunk) * 2 * a.C + c;
    p[0] = all.mean;
    p[a.C] = all.square;
}

__device__ __forceinline__ int positions_in(const Norm &a, int chunk, int length)
{
    return max(min(min((chunk + 1) * a.chunk, a.T), length) - chunk * a.chunk, 0);
}

// f(chunk, channel of the group) for this thread's share of the entries of a group, by a workgroup of 256
template <class F>
__device__ __forceinline__ void for_entries(const Norm &a, F &&f)
{
    int chunk = threadIdx.x / a.D, c = threadIdx.x % a.D;
    const int chunks_on = 256 / a.D, c_on = 256 % a.D;
    while (chunk < a.chunks) {
        f(chunk, c);
        chunk += chunks_on;
        c += c_on;
        if (c >= a.D) {
            c -= a.D;
            ++chunk;
        }
    }
}
// sum over a workgroup of 256; `shared`: four words of the call's own
__device__ __forceinline__ float workgroup_sum(float v, float *shared)
{
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
    __syncthreads();
    return (shared[0] + shared[1]) + (shared[2] + shared[3]);
}

// Workgroups of the sums over groups, one a group up to this many: a launch has to have fewer than 2^32 threads.
constexpr int kMostGroupWorkgroups = 1 << 22;
unsigned group_workgroups(const esrnn_group_norm_shape &s) { return (unsigned)std::min<int64_t>((int64_t)s.N * s.G, kMostGroupWorkgroups); }

// stats [N][G][2]: a workgroup a group
__global__ void __launch_bounds__(256) norm_stats_kernel(Norm a)
{
    // (two places in turn: a barrier lies between the reads of one and its next writes)
    __shared__ float s_sum[2][4];
    for (int item = blockIdx.x; item < a.N * a.G; item += gridDim.x) {
        const int n = item / a.G, g = item % a.G, length = length_of(a, n);
        const float *p = a.parts + (size_t)n * a.chunks * 2 * a.C + g * a.D;
        // the mean first, then what lies off it: sums whose terms do not wait for each other
        const float inverse = length > 0 ? 1.0f / ((float)length * (float)a.D) : 0.0f;
        float sum = 0.0f, square = 0.0f;
        for_entries(a, [&](int chunk, int c) { sum += (float)positions_in(a, chunk, length) * p[(size_t)chunk * 2 * a.C + c]; });
        const float mean = workgroup_sum(sum, s_sum[0]) * inverse;
        for_entries(a, [&](int chunk, int c) {
            const int here = positions_in(a, chunk, length);
            const float d = p[(size_t)chunk * 2 * a.C + c] - mean;
            if (here > 0) square += p[((size_t)chunk * 2 + 1) * a.C + c] + (float)here * d * d;
        });
        square = workgroup_sum(square, s_sum[1]);
        if (threadIdx.x == 0) {
            float *s = a.stats + (size_t)item * 2;
            s[0] = mean;
            s[1] = 1.0f / sqrtf(square * inverse + a.eps);
        }
    }
}

// mean and rstd of the groups of four channels of a lane
template <bool kAligned>
__device__ __forceinline__ void group_stats(const Norm &a, const float *stats, int n, const Channels<kAligned, 16> &ch, f32x4 &mean, f32x4 &rstd)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float *s = stats + ((size_t)n * a.G + ch.readable(k) / a.D) * 2;
        mean[k] = s[0];
        rstd[k] = s[1];
    }
}
template <bool kAligned>
__device__ __forceinline__ f32x4 parameters(const float *p, const Channels<kAligned, 16> &ch)
{
    return f32x4{p[ch.readable(0)], p[ch.readable(1)], p[ch.readable(2)], p[ch.readable(3)]};
}

template <class E, bool kAligned, bool kSilu>
__global__ void __launch_bounds__(256) norm_apply_kernel(Norm a)
{
    const int lane16 = threadIdx.x & 15, row = threadIdx.x >> 4;
    const int n = blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles;
    const Channels<kAligned, 16> ch(lane16, tile * 64, a.C);
    const int length = length_of(a, n), first = blockIdx.y * a.chunk, end = min(first + a.chunk, a.T);
    const E *x = static_cast<const E *>(a.x) + (size_t)n * a.T * a.C;
    E *out = static_cast<E *>(a.out) + (size_t)n * a.T * a.C;
    f32x4 mean, rstd;
    group_stats(a, a.stats, n, ch, mean, rstd);
    const f32x4 scale = parameters(a.scale, ch), shift = parameters(a.shift, ch);
    for (int t0 = first; t0 < end; t0 += 16 * kRows) {
        Vec4<E> xs[kRows];
        if (t0 < length)
#pragma unroll
            for (int k = 0; k < kRows; ++k) xs[k] = ch.load(x + (size_t)min(t0 + row + 16 * k, length - 1) * a.C);
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            const int t = t0 + row + 16 * k;
            f32x4 y = (to_f32<E>(xs[k]) - mean) * rstd * scale + shift;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = activate(y[i], kSilu);
            if (t < end) ch.store(out + (size_t)t * a.C, from_f32<E>(t < length ? y : splat(0.0f)));
        }
    }
}

// parts [N][chunks][2][C]: P1 and P2 of a chunk's positions
template <class E, bool kAligned, bool kSilu>
__global__ void __launch_bounds__(256) norm_gradient_sums_kernel(Norm a)
{
    __shared__ float s_p1[16][64], s_p2[16][64];
    const int lane16 = threadIdx.x & 15, row = threadIdx.x >> 4;
    const int n = blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles, chunk = blockIdx.y;
    const Channels<kAligned, 16> ch(lane16, tile * 64, a.C);
    const int first = chunk * a.chunk, end = min(min(first + a.chunk, a.T), length_of(a, n));
    const E *x = static_cast<const E *>(a.x) + (size_t)n * a.T * a.C, *grad_out = static_cast<const E *>(a.grad_out) + (size_t)n * a.T * a.C;
    f32x4 mean, rstd, p1 = splat(0.0f), p2 = splat(0.0f);
    group_stats(a, a.stats_in, n, ch, mean, rstd);
    const f32x4 scale = parameters(a.scale, ch), shift = parameters(a.shift, ch);
    for (int t0 = first; t0 < end; t0 += 16 * kRows) {
        Vec4<E> xs[kRows], ds[kRows];
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            const size_t at = (size_t)min(t0 + row + 16 * k, end - 1) * a.C;
            xs[k] = ch.load(x + at);
            ds[k] = ch.load(grad_out + at);
        }
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            const f32x4 xhat = (to_f32<E>(xs[k]) - mean) * rstd, u = xhat * scale + shift;
            f32x4 du = to_f32<E>(ds[k]);
#pragma unroll
            for (int i = 0; i < 4; ++i) du[i] *= slope(u[i], kSilu);
            if (t0 + row + 16 * k < end) {
                p1 += du;
                p2 += du * xhat;
            }
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        s_p1[row][kAligned ? 4 * lane16 + k : lane16 + 16 * k] = p1[k];
        s_p2[row][kAligned ? 4 * lane16 + k : lane16 + 16 * k] = p2[k];
    }
    __syncthreads();
    const int c = threadIdx.x & 63, which = threadIdx.x >> 6;
    if (which >= 2 || tile * 64 + c >= a.C) return;
    float sum = 0.0f;
    for (int r = 0; r < 16; ++r) sum += (which ? s_p2 : s_p1)[r][c];
    a.parts[(((size_t)n * a.chunks + chunk) * 2 + which) * a.C + tile * 64 + c] = sum;
}

// sums [N][G][2] behind parts: S1 / M and S2 / M, a workgroup a group; in the same launch, by the first `channel_groups` workgroups, the
// sums over all samples and chunks (where there is one run of them)
__global__ void __launch_bounds__(256) norm_group_sums_kernel(Norm a, int channel_groups)
{
    __shared__ float s_sum[2][4];
    if ((int)blockIdx.x < channel_groups) {
        const int tiles = channel_groups / 2, which = blockIdx.x / tiles;
        sum_rows_of_tile<4>(a.parts + (size_t)which * a.C, a.N * a.chunks, a.C, blockIdx.x % tiles, which ? a.grad_scale : a.grad_shift);
        return;
    }
    for (int item = (int)blockIdx.x - channel_groups; item < a.N * a.G; item += (int)gridDim.x - channel_groups) {
        const int n = item / a.G, g = item % a.G, length = length_of(a, n);
        const float *p = a.parts + (size_t)n * a.chunks * 2 * a.C + g * a.D, *scale = a.scale + g * a.D;
        float s1 = 0.0f, s2 = 0.0f;
        for_entries(a, [&](int chunk, int c) {
            s1 += scale[c] * p[(size_t)chunk * 2 * a.C + c];
            s2 += scale[c] * p[((size_t)chunk * 2 + 1) * a.C + c];
        });
        s1 = workgroup_sum(s1, s_sum[0]);
        s2 = workgroup_sum(s2, s_sum[1]);
        if (threadIdx.x == 0) {
            const float inverse = length > 0 ? 1.0f / ((float)length * (float)a.D) : 0.0f;
            float *s = a.parts + (size_t)a.N * a.chunks * 2 * a.C + (size_t)item * 2;
            s[0] = s1 * inverse;
            s[1] = s2 * inverse;
        }
    }
}

template <class E, bool kAligned, bool kSilu>
__global__ void __launch_bounds__(256) norm_gradient_kernel(Norm a)
{
    const int lane16 = threadIdx.x & 15, row = threadIdx.x >> 4;
    const int n = blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles;
    const Channels<kAligned, 16> ch(lane16, tile * 64, a.C);
    const int length = length_of(a, n), first = blockIdx.y * a.chunk, end = min(first + a.chunk, a.T);
    const E *x = static_cast<const E *>(a.x) + (size_t)n * a.T * a.C, *grad_out = static_cast<const E *>(a.grad_out) + (size_t)n * a.T * a.C;
    E *grad_x = static_cast<E *>(a.grad_x) + (size_t)n * a.T * a.C;
    f32x4 mean, rstd, s1, s2;
    group_stats(a, a.stats_in, n, ch, mean, rstd);
    group_stats(a, a.parts + (size_t)a.N * a.chunks * 2 * a.C, n, ch, s1, s2);
    const f32x4 scale = parameters(a.scale, ch), shift = parameters(a.shift, ch);
    for (int t0 = first; t0 < end; t0 += 16 * kRows) {
        Vec4<E> xs[kRows], ds[kRows];
        if (t0 < length)
#pragma unroll
            for (int k = 0; k < kRows; ++k) {
                const size_t at = (size_t)min(t0 + row + 16 * k, length - 1) * a.C;
                xs[k] = ch.load(x + at);
                ds[k] = ch.load(grad_out + at);
            }
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            const int t = t0 + row + 16 * k;
            const f32x4 xhat = (to_f32<E>(xs[k]) - mean) * rstd, u = xhat * scale + shift;
            f32x4 du = to_f32<E>(ds[k]);
#pragma unroll
            for (int i = 0; i < 4; ++i) du[i] *= slope(u[i], kSilu);
            const f32x4 gx = input_gradient(rstd, scale, du, s1, xhat, s2);
            if (t < end) ch.store(grad_x + (size_t)t * a.C, from_f32<E>(t < length ? gx : splat(0.0f)));
        }
    }
}

// ---- which way, and its sizes ------------------------------------------------------------------------------------
enum Kind { kPosition, kWide, kSample, kStream };
struct Way {
    Kind kind;
    int threads, rows_each;     // sample: of a workgroup; positions a thread
    int tile, tiles, log_w, chunk, chunks;
    int pieces;                 // position: chunks of four channels a lane
    int forward_groups, backward_groups;        // position: workgroups of a tile
    int part_rows;              // rows [2][C] of channel sums that the reverse pass leaves
};

// Channels of a group: of a wave; of a workgroup (four chunks of 1024 is the widest that was built, not a bound that was found: beyond it the stream way takes
// single positions too, with one of its sixteen rows of threads at work and workgroups of few bytes: 8192 x 8192 bf16 in one group 2.9 and 5.9 ms for bytes
// that a copy moves in 53 and 79 us); samples at once (of groups up to 256).
constexpr int kMostPositionTile = 512, kMostWideTile = 4096, kPositionRows = 4;

// Rows are added up in two launches, the first in kRuns runs, from this many on: one alone reads them with 2 C / 64 workgroups (reverse pass of
// 8000 x 16 x 128 bf16 62 us, with one launch 81; 2048 x 16 x 64 fp32 20 against 22).
constexpr int kManyRows = 1024, kRuns = 64;

Way way_of(const esrnn_group_norm_shape &s)
{
    Way w{};
    const int D = s.C / s.G;
    if (s.T == 1 && D > kMostPositionTile && D <= kMostWideTile) {
        // (a wave for each group needs more registers than it has beyond 512 channels: figures above)
        w.kind = kWide;
        w.tiles = s.G;
        w.pieces = D <= 1024 ? 1 : D <= 2048 ? 2 : 4;
        const int64_t most = ((int64_t)s.N * w.pieces + 3) / 4;
        w.forward_groups = (int)std::min<int64_t>(most, std::max(1, 2048 / s.G));
        w.backward_groups = (int)std::min<int64_t>(most, std::max(1, 1024 / s.G));
        w.part_rows = w.backward_groups;
        return w;
    }
    if (s.T == 1 && D <= kMostPositionTile) {
        // whole groups up to 256 channels, of which a few groups less may be whole groups of four channels
        int groups = std::max(1, std::min(s.G, 256 / D));
        for (int fewer = groups; fewer > std::max(1, groups - 4); --fewer)
            if (fewer * D % 4 == 0) {
                groups = fewer;
                break;
            }
        w.kind = kPosition;
        w.tile = groups * D;
        w.tiles = (s.G + groups - 1) / groups;
        for (w.log_w = 0; w.log_w < 6 && 4 << w.log_w < w.tile; ++w.log_w) {}
        for (w.pieces = 1; w.pieces * 256 < w.tile; w.pieces *= 2) {}
        const int rows = 4 * (w.pieces == 1 ? kPositionRows : 1) * (64 >> w.log_w);     // of a workgroup
        const int64_t most = ((int64_t)s.N + rows - 1) / rows;
        // (16384 x 2048 bf16, the one size that they were tried at: forward with 1024, 2048, 3000, 4096 workgroups 34, 32, 30, 31 us; reverse with
        // 512, 1024, 2048 54, 45, 47)
        w.forward_groups = (int)std::min<int64_t>(most, std::max(1, 3000 / w.tiles));
        w.backward_groups = (int)std::min<int64_t>(most, std::max(1, 1024 / w.tiles));
        w.part_rows = w.backward_groups;
        return w;
    }
    // sample: whole groups side by side up to 64 channels (a run of 128 bytes of bf16), as many positions as fit.  Against the stream way, forward and
    // reverse: 512 x 72 x 64 fp32 10 and 13 us against 16 and 20, 64 x 512 x 512 bf16 26 and 42 against 26 and 42.
    // A wave by itself waits at no barrier, but has all groups of the tile to add up: up to 16 positions, from 2048 workgroups on (4096 x 16 x 64 fp32 15
    // and 25 us, with 256 threads 22 and 38; 2048 12 and 18 against 13 and 22; 1024 10 and 16 against 9 and 13; 3000 x 4 x 256 bf16 17 and 25
    // against 44 and 50).
    // Up to 32 channels only for few workgroups, where the launches of the stream way are what counts (2 samples of 1000 x 96 fp32, forward 11
    // against 15 us; 64 of 1024 x 512 bf16: 58 against 46).
    constexpr int kSplits[6][3] = {{64, 64, 4}, {64, 256, 4}, {64, 256, 16}, {64, 1024, 4}, {64, 1024, 8}, {32, 1024, 8}};   // channels, threads, positions each
    for (const auto &split : kSplits) {
        if (split[0] < 64 && (int64_t)s.N * s.C > 256 * 32) break;
        int groups = std::max(1, std::min(s.G, split[0] / D));
        for (int fewer = groups; fewer > 1; --fewer)        // (whole groups of four channels, if a few groups less give them)
            if (fewer * D % 4 == 0) {
                groups = fewer;
                break;
            }
        w.tile = groups * D;
        for (w.log_w = 0; 4 << w.log_w < w.tile; ++w.log_w) {}
        w.tiles = (s.G + groups - 1) / groups;
        if (split[1] == 64 && (int64_t)s.N * w.tiles < 2048) continue;
        if (w.tile <= most_tile(split[1]) && split[1] >> w.log_w >= 1 && (int64_t)s.N * w.tiles * split[1] <= (int64_t(1) << 31) &&
            (int64_t)s.T <= (int64_t)(split[1] >> w.log_w) * split[2]) {
            w.kind = kSample;
            w.threads = split[1], w.rows_each = split[2];
            break;
        }
    }
    w.part_rows = s.N;
    if (w.kind == kSample) return w;
    w.kind = kStream;
    // some 2048 workgroups (1024 to 8192 make no difference), of 128 positions at least
    w.tiles = (s.C + 63) / 64;
    const int64_t columns = (int64_t)s.N * w.tiles;
    int64_t chunks = std::max<int64_t>(1, std::min<int64_t>((s.T + 127) / 128, 2048 / columns));
    w.chunk = (int)(((s.T + chunks - 1) / chunks + 127) / 128 * 128);
    w.chunks = (s.T + w.chunk - 1) / w.chunk;
    w.part_rows = s.N * w.chunks;
    return w;
}

Norm norm_of(const esrnn_group_norm_shape &s, const GroupNormArgs &f, const Way &w)
{
    Norm a{};
    a.x = f.x, a.grad_out = f.grad_out, a.out = f.out, a.grad_x = f.grad_x, a.lengths = f.lengths, a.scale = f.scale, a.shift = f.shift;
    a.stats_in = f.stats_in, a.stats = f.stats, a.parts = f.parts, a.grad_scale = f.grad_scale, a.grad_shift = f.grad_shift;
    a.N = s.N, a.T = s.T, a.C = s.C, a.G = s.G, a.D = s.C / s.G, a.silu = s.activation == ESRNN_NORM_SILU, a.eps = s.eps;
    a.tile = w.tile, a.tiles = w.tiles, a.log_w = w.log_w, a.chunk = w.chunk, a.chunks = w.chunks;
    return a;
}

template <class F>
void with_flags(bool aligned, bool silu, F &&f)
{
    if (aligned) silu ? f(std::true_type{}, std::true_type{}) : f(std::true_type{}, std::false_type{});
    else silu ? f(std::false_type{}, std::true_type{}) : f(std::false_type{}, std::false_type{});
}


// LDS of a wave of the position way, in pairs: entries of its rows, sums of their groups (as Tile has them)
int position_pairs(const esrnn_group_norm_shape &s, const Way &w, bool quads)
{
    if (w.pieces > 1) return 0;
    const int rows = kPositionRows * (64 >> w.log_w), entries = (quads ? 1 : 4) << w.log_w;
    return rows * (entries + entries / 16 + w.tile / (s.C / s.G));
}

// f(pieces, samples at once, aligned, quads)
template <class F>
void with_pieces(int pieces, bool aligned, bool quads, F &&f)
{
    const auto layout = [&](auto j, auto r) {
        // (of one group in chunks there is nothing to tell apart)
        if (aligned && (quads || j() > 1)) f(j, r, std::true_type{}, std::true_type{});
        else if (aligned) f(j, r, std::true_type{}, std::bool_constant<(j() > 1)>{});
        else f(j, r, std::false_type{}, std::bool_constant<(j() > 1)>{});
    };
    using One = std::integral_constant<int, 1>;
    switch (pieces) {
    case 1: return layout(One{}, std::integral_constant<int, kPositionRows>{});
    default: return layout(std::integral_constant<int, 2>{}, One{});
    }
}

template <class E, bool kSilu>
void position_forward(const esrnn_group_norm_shape &s, Norm a, const Way &w, bool aligned, hipStream_t st)
{
    const bool fours = aligned && w.tile % 4 == 0, quads = fours && a.D % 4 == 0;
    a.wave_pairs = position_pairs(s, w, quads);
    with_pieces(w.pieces, fours, quads, [&](auto j, auto r, auto al, auto q) {
        norm_position_forward_kernel<E, al(), q(), j(), r(), kSilu><<<w.tiles * w.forward_groups, 256, 4 * sizeof(Pair) * a.wave_pairs, st>>>(a);
    });
}

template <class E, bool kSilu>
void position_backward(const esrnn_group_norm_shape &s, Norm a, const Way &w, bool aligned, hipStream_t st)
{
    const bool fours = aligned && w.tile % 4 == 0, quads = fours && a.D % 4 == 0;
    a.wave_pairs = position_pairs(s, w, quads);
    const size_t lds = std::max(4 * sizeof(Pair) * a.wave_pairs, 2 * sizeof(float) * a.tile);
    with_pieces(w.pieces, fours, quads, [&](auto j, auto r, auto al, auto q) {
        norm_position_backward_kernel<E, al(), q(), j(), r(), kSilu><<<w.tiles * w.backward_groups, 256, lds, st>>>(a);
    });
}

template <class F>
void with_wide_pieces(int pieces, F &&f)
{
    switch (pieces) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    default: return f(std::integral_constant<int, 4>{});
    }
}

// The sums over `rows` rows at parts; `more`: room for kRuns rows.
void sum_rows(const Norm &a, int rows, float *more, hipStream_t st)
{
    const unsigned tiles = (a.C + 63) / 64;
    if (rows >= kManyRows) {
        norm_sum_rows_kernel<<<dim3(tiles, 2, kRuns), 1024, 0, st>>>(a.parts, rows, a.C, more, more + a.C);
        norm_sum_rows_kernel<<<dim3(tiles, 2, 1), 1024, 0, st>>>(more, kRuns, a.C, a.grad_shift, a.grad_scale);
    } else {
        norm_sum_rows_kernel<<<dim3(tiles, 2, 1), 1024, 0, st>>>(a.parts, rows, a.C, a.grad_shift, a.grad_scale);
    }
}

// The workspace: channel sums [part_rows][2][C] of the reverse pass (of the stream way's forward pass: moments), statistics or group sums
// [N][G][2] of the stream way, runs of channel sums.
size_t groups_at(const esrnn_group_norm_shape &s, const Way &w) { return (size_t)w.part_rows * 2 * s.C; }
size_t runs_at(const esrnn_group_norm_shape &s, const Way &w) { return groups_at(s, w) + (w.kind == kStream ? (size_t)s.N * s.G * 2 : 0); }

}  // namespace

bool group_norm_single_positions(const esrnn_group_norm_shape &s) { return s.T == 1 && s.C / s.G <= kMostWideTile; }

size_t group_norm_workspace_floats(const esrnn_group_norm_shape &s)
{
    const Way w = way_of(s);
    return runs_at(s, w) + (w.part_rows >= kManyRows ? (size_t)kRuns * 2 * s.C : 0);
}

hipError_t launch_group_norm_forward(const esrnn_group_norm_shape &s, const GroupNormArgs &f, hipStream_t st)
{
    const Way w = way_of(s);
    Norm a = norm_of(s, f, w);
    const size_t group = 4 * element_bytes(s.dtype);
    const bool aligned = s.C % 4 == 0 && aligned_to(f.x, group) && aligned_to(f.out, group), fours = aligned && a.D % 4 == 0;
    return with_element(s.dtype, [&](auto e) {
        using E = decltype(e);
        with_flags(aligned && (w.kind != kSample || w.tile % 4 == 0), a.silu, [&](auto al, auto silu) {
            if (w.kind == kPosition) {
                position_forward<E, silu()>(s, a, w, aligned, st);
                return;
            }
            if (w.kind == kWide) {
                with_wide_pieces(w.pieces, [&](auto j) {
                    if (fours) norm_wide_forward_kernel<E, true, j(), silu()><<<s.G * w.forward_groups, 256, 0, st>>>(a);
                    else norm_wide_forward_kernel<E, false, j(), silu()><<<s.G * w.forward_groups, 256, 0, st>>>(a);
                });
                return;
            }
            if (w.kind == kSample) {
                const unsigned grid = (unsigned)(s.N * w.tiles);
                if (w.threads == 64) norm_sample_forward_kernel<E, al(), 64, 4, silu()><<<grid, 64, 0, st>>>(a);
                else if (w.threads == 256 && w.rows_each == 4) norm_sample_forward_kernel<E, al(), 256, 4, silu()><<<grid, 256, 0, st>>>(a);
                else if (w.threads == 256) norm_sample_forward_kernel<E, al(), 256, 16, silu()><<<grid, 256, 0, st>>>(a);
                else if (w.rows_each == 4) norm_sample_forward_kernel<E, al(), 1024, 4, silu()><<<grid, 1024, 0, st>>>(a);
                else norm_sample_forward_kernel<E, al(), 1024, 8, silu()><<<grid, 1024, 0, st>>>(a);
                return;
            }
            if (!a.stats) a.stats = a.parts + groups_at(s, w);
            const dim3 grid((unsigned)(s.N * w.tiles), w.chunks);
            norm_moments_kernel<E, al()><<<grid, 256, 0, st>>>(a);
            norm_stats_kernel<<<group_workgroups(s), 256, 0, st>>>(a);
            norm_apply_kernel<E, al(), silu()><<<grid, 256, 0, st>>>(a);
        });
        return hipGetLastError();
    });
}

hipError_t launch_group_norm_backward(const esrnn_group_norm_shape &s, const GroupNormArgs &f, hipStream_t st)
{
    const Way w = way_of(s);
    const Norm a = norm_of(s, f, w);
    const size_t group = 4 * element_bytes(s.dtype);
    const bool aligned = s.C % 4 == 0 && aligned_to(f.x, group) && aligned_to(f.grad_out, group) && aligned_to(f.grad_x, group);
    const bool fours = aligned && a.D % 4 == 0;
    return with_element(s.dtype, [&](auto e) {
        using E = decltype(e);
        with_flags(aligned && (w.kind != kSample || w.tile % 4 == 0), a.silu, [&](auto al, auto silu) {
            float *runs = a.parts + runs_at(s, w);
            if (w.kind == kPosition) {
                position_backward<E, silu()>(s, a, w, aligned, st);
                sum_rows(a, w.part_rows, runs, st);
                return;
            }
            if (w.kind == kWide) {
                with_wide_pieces(w.pieces, [&](auto j) {
                    if (fours) norm_wide_backward_kernel<E, true, j(), silu()><<<s.G * w.backward_groups, 256, 0, st>>>(a);
                    else norm_wide_backward_kernel<E, false, j(), silu()><<<s.G * w.backward_groups, 256, 0, st>>>(a);
                });
                sum_rows(a, w.part_rows, runs, st);
                return;
            }
            if (w.kind == kSample) {
                const unsigned grid = (unsigned)(s.N * w.tiles);
                if (w.threads == 64) norm_sample_backward_kernel<E, al(), 64, 4, silu()><<<grid, 64, 0, st>>>(a);
                else if (w.threads == 256 && w.rows_each == 4) norm_sample_backward_kernel<E, al(), 256, 4, silu()><<<grid, 256, 0, st>>>(a);
                else if (w.threads == 256) norm_sample_backward_kernel<E, al(), 256, 16, silu()><<<grid, 256, 0, st>>>(a);
                else if (w.rows_each == 4) norm_sample_backward_kernel<E, al(), 1024, 4, silu()><<<grid, 1024, 0, st>>>(a);
                else norm_sample_backward_kernel<E, al(), 1024, 8, silu()><<<grid, 1024, 0, st>>>(a);
                sum_rows(a, w.part_rows, runs, st);
                return;
            }
            const dim3 grid((unsigned)(s.N * w.tiles), w.chunks);
            norm_gradient_sums_kernel<E, al(), silu()><<<grid, 256, 0, st>>>(a);
            const int channel_groups = w.part_rows < kManyRows ? 2 * ((s.C + 63) / 64) : 0;
            norm_group_sums_kernel<<<channel_groups + group_workgroups(s), 256, 0, st>>>(a, channel_groups);
            if (!channel_groups) sum_rows(a, w.part_rows, runs, st);
            norm_gradient_kernel<E, al(), silu()><<<grid, 256, 0, st>>>(a);
        });
        return hipGetLastError();
    });
}

}  // namespace esrnn
