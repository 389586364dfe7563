// Block norm: gate, norm behind a block, residual, norm before the next block, for every row by itself (include/esrnn_state_space.h).
//
// A row is held in registers by L lanes of a wave, or by one or several whole waves, whose sums go through LDS; a workgroup takes rows one behind
// the other (in reverse each is requested while the one before is worked on), so that a lane's weights are read once, and so that the gradients of the
// weights add up in its registers.  Forward, with act = silu(gate):
//   v = y act | y,  r1 = 1 / sqrt(mean v^2 + eps),  p = v r1 post,  e = p act | p,  s = residual + scale e,  r2 = 1 / sqrt(mean s^2 + eps),  out = s r2 pre.
// Reverse, with that = s r2, vhat = v r1 and the gradients D of out and S of sum:
//   ds = S + r2 (D pre - that mean(D pre that)),  de = ds scale,  dp = de act | de,  dv = r1 (dp post - vhat mean(dp post vhat)),  dy = dv act | dv,
//   dgate = silu'(gate) (dv y | de p),  dpre = sum D that,  dscale = sum ds e,  dpost = sum dp vhat.
// The reverse pass computes s again from the residual, in fp32, rather than read the rounded sum.
//
// Reads and writes are the bound, every operand once: 32768 rows of 2048, bf16, gate and both norms, forward 137-144 us (673 MB, 4.8 TB/s), reverse 226-256 + 5 us
// (1089 MB, 4.5 TB/s); 120240 rows of 50, fp32, 21 and 28 + 5 us.
#include <algorithm>
#include <limits>

#include "state_space_internal.h"

namespace esrnn {

namespace {

constexpr int kWavesForward = 8192, kWavesReverse = 4096;

struct Args {
    BlockNormArgs a;
    long long y, gate, residual, sum, out, grad_out, grad_sum, grad_y, grad_gate, grad_residual;       // strides of a row
    int rows, C, before, after;         // where the gate is
    float eps, inverse;                 // 1 / C
};

// How a row is held: L lanes of each of NW waves, M groups of four neighbouring channels a lane; RW rows of a workgroup at a time.
// kAhead: rows are requested ahead.
template <int L_, int NW_, int M_ = 1, bool kAhead_ = true>
struct Layout {
    static constexpr bool kAhead = kAhead_;
    static constexpr int L = L_, NW = NW_, M = M_, kThreads = NW > 1 ? 64 * NW : 256, RW = kThreads / (L * NW), kChannels = 4 * M * L * NW;
};

// Sums over the lanes of a row, the same in all of them.  `slot`: two sums that follow each other have different ones.
template <class Y>
__device__ __forceinline__ float row_sum(float v, float (*lds)[16], int slot)
{
#pragma unroll
    for (int off = Y::L / 2; off > 0; off /= 2) v += __shfl_xor(v, off, 64);
    if constexpr (Y::NW > 1) {
        if ((threadIdx.x & 63) == 0) lds[slot][threadIdx.x >> 6] = v;
        lds_barrier();          // (requests for the next row go on)
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < Y::NW; ++w) v += lds[slot][w];
    }
    return v;
}

// A lane's channels: group m begins at 4 (m T + lane), T the lanes of a row.  A row is requested while the one before it is worked on.
template <class Y, class E>
struct Row {
    typename Neighbours<E, 4>::Values v[Y::M];
    __device__ __forceinline__ void request(const void *base, long long at, int lane, int C)
    {
        if (!base) return;
        const E *row = static_cast<const E *>(base) + at;
#pragma unroll
        for (int m = 0; m < Y::M; ++m) v[m] = Neighbours<E, 4>{4 * (m * Y::L * Y::NW + lane), C}.load(row);
    }
    __device__ __forceinline__ void get(bool there, f32x4 (&to)[Y::M]) const
    {
#pragma unroll
        for (int m = 0; m < Y::M; ++m) to[m] = there ? to_f32<E>(v[m]) : f32x4{};
    }
};
template <class Y, class E>
__device__ __forceinline__ void store_row(void *base, long long at, int lane, int C, const f32x4 (&v)[Y::M])
{
    E *row = static_cast<E *>(base) + at;
#pragma unroll
    for (int m = 0; m < Y::M; ++m) {
        const Neighbours<E, 4> ch{4 * (m * Y::L * Y::NW + lane), C};
        ch.store(row, from_f32<E>(v[m]));
    }
}
// Weights of a lane's channels, ones where there are none.
template <class Y>
__device__ __forceinline__ f32x4 load_weight(const float *w, int m, int lane, int C)
{
    if (!w) return f32x4{1.0f, 1.0f, 1.0f, 1.0f};
    return Neighbours<float, 4>{4 * (m * Y::L * Y::NW + lane), C}.load(w);
}
template <class Y>
struct Weights {
    f32x4 v[Y::M];
    __device__ __forceinline__ Weights(const float *w, int lane, int C)
    {
#pragma unroll
        for (int m = 0; m < Y::M; ++m) v[m] = load_weight<Y>(w, m, lane, C);
    }
    __device__ __forceinline__ f32x4 operator[](int m) const { return v[m]; }
};
template <class Y>
__device__ __forceinline__ float squares(const f32x4 (&v)[Y::M])
{
    f32x4 s = {};
#pragma unroll
    for (int m = 0; m < Y::M; ++m) s += v[m] * v[m];
    return (s[0] + s[1]) + (s[2] + s[3]);
}
template <class Y>
__device__ __forceinline__ float products(const f32x4 (&v)[Y::M], const f32x4 (&u)[Y::M])
{
    f32x4 s = {};
#pragma unroll
    for (int m = 0; m < Y::M; ++m) s += v[m] * u[m];
    return (s[0] + s[1]) + (s[2] + s[3]);
}
// 1 / sqrt(mean + eps): a square root and a division, each rounded once
__device__ __forceinline__ float inverse_root(float sum, const Args &p) { return 1.0f / sqrtf(fmaf(sum, p.inverse, p.eps)); }

template <class E, class R, class Y>
__global__ void __launch_bounds__(Y::kThreads) block_norm_forward_kernel(Args p)
{
    __shared__ float s_sums[4][16];
    const int lane = threadIdx.x % (Y::L * Y::NW), in_group = threadIdx.x / (Y::L * Y::NW);
    const Weights<Y> post(p.a.post_weight, lane, p.C), scale(p.a.scale, lane, p.C), pre(p.a.pre_weight, lane, p.C);
    Row<Y, E> ys, gates;
    Row<Y, R> residuals;
    bool exists = false;
    const auto request = [&](int first) {
        const long long row = min(first + in_group, p.rows - 1);
        exists = !p.a.exists || p.a.exists[row] != 0;
        ys.request(p.a.y, row * p.y, lane, p.C);
        gates.request(p.a.gate, row * p.gate, lane, p.C);
        residuals.request(p.a.residual, row * p.residual, lane, p.C);
    };
    int turn = 0;
    const int step = gridDim.x * Y::RW;
    if (Y::kAhead) request(blockIdx.x * Y::RW);
    for (int first = blockIdx.x * Y::RW; first < p.rows; first += step, turn ^= 2) {
        const long long row = first + in_group;
        const bool mine = row < p.rows;
        if (!Y::kAhead) request(first);
        f32x4 v[Y::M], act[Y::M], s[Y::M] = {};
        ys.get(exists, v);
        if (p.a.gate) gates.get(exists, act);
        if (p.a.residual) residuals.get(exists, s);
        if (Y::kAhead && first + step < p.rows) request(first + step);
        if (p.a.gate) {
#pragma unroll
            for (int m = 0; m < Y::M; ++m)
#pragma unroll
                for (int k = 0; k < 4; ++k) act[m][k] = silu(act[m][k]).of;
        }
        if (p.before)
#pragma unroll
            for (int m = 0; m < Y::M; ++m) v[m] *= act[m];
        float r1 = 1.0f, r2 = 1.0f;
        if (p.a.post_weight) {
            r1 = inverse_root(row_sum<Y>(squares<Y>(v), s_sums, turn), p);
#pragma unroll
            for (int m = 0; m < Y::M; ++m) v[m] = v[m] * r1 * post[m];
        }
        if (p.after)
#pragma unroll
            for (int m = 0; m < Y::M; ++m) v[m] *= act[m];
#pragma unroll
        for (int m = 0; m < Y::M; ++m) s[m] += scale[m] * v[m];
        if (p.a.residual && mine) store_row<Y, R>(p.a.sum, row * p.sum, lane, p.C, s);
        if (p.a.pre_weight) {
            r2 = inverse_root(row_sum<Y>(squares<Y>(s), s_sums, turn + 1), p);
#pragma unroll
            for (int m = 0; m < Y::M; ++m) s[m] = s[m] * r2 * pre[m];
        }
        if (p.a.out && mine) store_row<Y, E>(p.a.out, row * p.out, lane, p.C, s);
        if (p.a.stats && mine && lane == 0) {
            p.a.stats[2 * row] = r1;
            p.a.stats[2 * row + 1] = r2;
        }
    }
}

template <class E, class R, class Y>
__global__ void __launch_bounds__(Y::kThreads) block_norm_backward_kernel(Args p)
{
    constexpr int M = Y::M;
    __shared__ float s_sums[4][16];
    __shared__ __attribute__((aligned(16))) float s_parts[Y::RW > 1 ? Y::RW : 1][Y::RW > 1 ? Y::kChannels : 1];
    const int lane = threadIdx.x % (Y::L * Y::NW), in_group = threadIdx.x / (Y::L * Y::NW);
    const Weights<Y> post(p.a.post_weight, lane, p.C), scale(p.a.scale, lane, p.C), pre(p.a.pre_weight, lane, p.C);
    // (sixteen waves of a row have at most 128 registers, which requests in fp32 would exceed)
    constexpr bool kAhead = Y::kAhead && !(Y::NW == 16 && sizeof(R) == 4);
    f32x4 dpost[M] = {}, dscale[M] = {}, dpre[M] = {};
    Row<Y, E> ys, gates, ds_out;
    Row<Y, R> residuals, ds_sum;
    bool exists = false;
    float next_r1 = 0.0f, next_r2 = 0.0f;
    const auto request = [&](int first) {
        const long long row = min(first + in_group, p.rows - 1);
        exists = first + in_group < p.rows && (!p.a.exists || p.a.exists[row] != 0);
        ys.request(p.a.y, row * p.y, lane, p.C);
        gates.request(p.a.gate, row * p.gate, lane, p.C);
        residuals.request(p.a.residual, row * p.residual, lane, p.C);
        ds_out.request(p.a.grad_out, row * p.grad_out, lane, p.C);
        ds_sum.request(p.a.grad_sum, row * p.grad_sum, lane, p.C);
        next_r1 = p.a.stats_in[2 * row], next_r2 = p.a.stats_in[2 * row + 1];
    };
    int turn = 0;
    const int step = gridDim.x * Y::RW;
    if (kAhead) request(blockIdx.x * Y::RW);
    for (int first = blockIdx.x * Y::RW; first < p.rows; first += step, turn ^= 2) {
        const long long row = first + in_group;
        const bool mine = row < p.rows;
        if (!kAhead) request(first);
        f32x4 y[M], gate[M] = {}, s[M] = {}, d[M] = {}, ds[M] = {};
        const float r1 = exists ? next_r1 : 0.0f, r2 = exists ? next_r2 : 0.0f;
        ys.get(exists, y);
        if (p.a.gate) gates.get(exists, gate);
        if (p.a.residual) residuals.get(exists, s);
        if (p.a.grad_out) ds_out.get(exists, d);
        if (p.a.grad_sum) ds_sum.get(exists, ds);
        if (kAhead && first + step < p.rows) request(first + step);
        f32x4 act[M], slope[M], vhat[M], e[M];
#pragma unroll
        for (int m = 0; m < M; ++m) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const Silu g = silu(gate[m][k]);
                act[m][k] = g.of, slope[m][k] = g.slope;
            }
            vhat[m] = (p.before ? y[m] * act[m] : y[m]) * r1;
            e[m] = vhat[m] * post[m];       // p, for now
            s[m] += scale[m] * (p.after ? e[m] * act[m] : e[m]);
        }
        if (p.a.pre_weight) {
            f32x4 weighted[M];
#pragma unroll
            for (int m = 0; m < M; ++m) {
                s[m] *= r2;                 // that
                dpre[m] += d[m] * s[m];
                weighted[m] = d[m] * pre[m];
            }
            const float mean = row_sum<Y>(products<Y>(weighted, s), s_sums, turn) * p.inverse;
#pragma unroll
            for (int m = 0; m < M; ++m) ds[m] += r2 * (weighted[m] - s[m] * mean);
        } else if (!p.a.residual) {
#pragma unroll
            for (int m = 0; m < M; ++m) ds[m] = d[m];
        }
        if (p.a.grad_residual && mine) store_row<Y, R>(p.a.grad_residual, row * p.grad_residual, lane, p.C, ds);
        f32x4 dgate[M], weighted[M];
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const f32x4 of_e = p.after ? e[m] * act[m] : e[m];
            dscale[m] += ds[m] * of_e;
            const f32x4 de = ds[m] * scale[m];
            dgate[m] = de * e[m];
            const f32x4 dp = p.after ? de * act[m] : de;
            dpost[m] += dp * vhat[m];
            weighted[m] = dp * post[m];
        }
        if (p.a.post_weight) {
            const float mean = row_sum<Y>(products<Y>(weighted, vhat), s_sums, turn + 1) * p.inverse;
#pragma unroll
            for (int m = 0; m < M; ++m) weighted[m] = r1 * (weighted[m] - vhat[m] * mean);
        }
        if (p.before)
#pragma unroll
            for (int m = 0; m < M; ++m) {
                dgate[m] = weighted[m] * y[m];
                weighted[m] *= act[m];
            }
        if (mine) {
            store_row<Y, E>(p.a.grad_y, row * p.grad_y, lane, p.C, weighted);
            if (p.a.grad_gate) {
#pragma unroll
                for (int m = 0; m < M; ++m) dgate[m] *= slope[m];
                store_row<Y, E>(p.a.grad_gate, row * p.grad_gate, lane, p.C, dgate);
            }
        }
    }
    // the workgroup's sums, rows of [3][C]
#pragma unroll
    for (int which = 0; which < 3; ++which) {
        f32x4 sum[M];
#pragma unroll
        for (int m = 0; m < M; ++m) sum[m] = which == 0 ? dpost[m] : which == 1 ? dscale[m] : dpre[m];
        float *to = p.a.parts + ((size_t)blockIdx.x * 3 + which) * p.C;
        if constexpr (Y::RW > 1) {
            __syncthreads();
#pragma unroll
            for (int m = 0; m < M; ++m) *reinterpret_cast<f32x4 *>(&s_parts[in_group][4 * (m * Y::L + lane)]) = sum[m];
            __syncthreads();
            for (int c = threadIdx.x; c < p.C; c += Y::kThreads) {
                float v = 0.0f;
                for (int r = 0; r < Y::RW; ++r) v += s_parts[r][c];
                to[c] = v;
            }
        } else {
            store_row<Y, float>(to, 0, lane, p.C, sum);
        }
    }
}

// Rows of more than 4096 channels, of which registers do not hold what is made of them: every one of the three steps (the sum for the second norm, that for the first,
// the gradients) reads the row again, from the caches, and the sums over rows are in LDS.  4000 rows of 8192 channels, bf16: some 250 us, where 109 would be those of a
// copy.  The operands alone would fit (eight channels of five arrays: 20 registers in 16 bits, 40 in fp32, of 128) and could be read once, the terms made of them at every
// step: not built.
template <class E, class R, class Y>
__global__ void __launch_bounds__(Y::kThreads) block_norm_wide_backward_kernel(Args p)
{
    constexpr int M = Y::M;
    __shared__ float s_sums[4][16];
    __shared__ f32x4 s_weights[3][M][Y::kThreads];
    const int lane = threadIdx.x;
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int which = 0; which < 3; ++which) s_weights[which][m][lane] = f32x4{};
    int turn = 0;
    for (long long row = blockIdx.x; row < p.rows; row += gridDim.x, turn ^= 2) {
        const bool exists = !p.a.exists || p.a.exists[row] != 0;
        const float r1 = exists ? p.a.stats_in[2 * row] : 0.0f, r2 = exists ? p.a.stats_in[2 * row + 1] : 0.0f;
        const auto ch = [&](int m) { return 4 * (m * Y::kThreads + lane); };
        // (converted behind the condition on `base`, and all requests of a step together, or each would be waited for by itself)
        const auto read = [&](auto e, const void *base, long long at, int m) {
            typedef decltype(e) T;
            Vec4<T> v = {};
            if (base) v = Neighbours<T, 4>{ch(m), p.C}.load(static_cast<const T *>(base) + at);
            return v;
        };
        const auto widen = [&](auto v) { return exists ? __builtin_convertvector(v, f32x4) : f32x4{}; };
        struct Terms {
            f32x4 y, act, slope, vhat, e, that, d, ds;  // e: p, before a gate behind the norm
        };
        const auto terms = [&](int m, bool with_sum) {
            Terms t;
            const auto y = read(E{}, p.a.y, row * p.y, m), d = read(E{}, p.a.grad_out, row * p.grad_out, m), g = read(E{}, p.a.gate, row * p.gate, m);
            const auto residual = read(R{}, p.a.residual, row * p.residual, m), ds = read(R{}, with_sum ? p.a.grad_sum : nullptr, row * p.grad_sum, m);
            const f32x4 gate = widen(g);
            t.y = widen(y), t.d = widen(d), t.ds = widen(ds);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const Silu a = silu(gate[k]);
                t.act[k] = a.of, t.slope[k] = a.slope;
            }
            t.vhat = (p.before ? t.y * t.act : t.y) * r1;
            t.e = t.vhat * load_weight<Y>(p.a.post_weight, m, lane, p.C);
            t.that = (widen(residual) + load_weight<Y>(p.a.scale, m, lane, p.C) * (p.after ? t.e * t.act : t.e)) * r2;
            return t;
        };
        const auto dot = [](f32x4 a, f32x4 b) {
            const f32x4 v = a * b;
            return (v[0] + v[1]) + (v[2] + v[3]);
        };
        float mean2 = 0.0f, mean1 = 0.0f;
        if (p.a.pre_weight) {
#pragma unroll
            for (int m = 0; m < M; ++m) {
                const Terms t = terms(m, false);
                mean2 += dot(t.d * load_weight<Y>(p.a.pre_weight, m, lane, p.C), t.that);
            }
            mean2 = row_sum<Y>(mean2, s_sums, turn) * p.inverse;
        }
        const auto of_sum = [&](int m, const Terms &t) {
            if (!p.a.residual && !p.a.pre_weight) return t.d;
            return p.a.pre_weight ? t.ds + r2 * (t.d * load_weight<Y>(p.a.pre_weight, m, lane, p.C) - t.that * mean2) : t.ds;
        };
        if (p.a.post_weight) {
#pragma unroll
            for (int m = 0; m < M; ++m) {
                const Terms t = terms(m, true);
                const f32x4 de = of_sum(m, t) * load_weight<Y>(p.a.scale, m, lane, p.C);
                mean1 += dot((p.after ? de * t.act : de) * load_weight<Y>(p.a.post_weight, m, lane, p.C), t.vhat);
            }
            mean1 = row_sum<Y>(mean1, s_sums, turn + 1) * p.inverse;
        }
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const Terms t = terms(m, true);
            const f32x4 ds = of_sum(m, t), de = ds * load_weight<Y>(p.a.scale, m, lane, p.C), dp = p.after ? de * t.act : de;
            if (p.a.pre_weight) s_weights[2][m][lane] += t.d * t.that;
            s_weights[1][m][lane] += ds * (p.after ? t.e * t.act : t.e);
            s_weights[0][m][lane] += dp * t.vhat;
            f32x4 dv = dp * load_weight<Y>(p.a.post_weight, m, lane, p.C);
            if (p.a.post_weight) dv = r1 * (dv - t.vhat * mean1);
            const f32x4 dgate = (p.before ? dv * t.y : de * t.e) * t.slope;
            if (p.before) dv *= t.act;
            if (p.a.grad_residual) Neighbours<R, 4>{ch(m), p.C}.store(static_cast<R *>(p.a.grad_residual) + row * p.grad_residual, from_f32<R>(ds));
            Neighbours<E, 4>{ch(m), p.C}.store(static_cast<E *>(p.a.grad_y) + row * p.grad_y, from_f32<E>(dv));
            if (p.a.grad_gate) Neighbours<E, 4>{ch(m), p.C}.store(static_cast<E *>(p.a.grad_gate) + row * p.grad_gate, from_f32<E>(dgate));
        }
    }
#pragma unroll
    for (int which = 0; which < 3; ++which)
#pragma unroll
        for (int m = 0; m < M; ++m)
            Neighbours<float, 4>{4 * (m * Y::kThreads + lane), p.C}.store(p.a.parts + ((size_t)blockIdx.x * 3 + which) * p.C, s_weights[which][m][lane]);
}

template <int kCols>
__global__ void __launch_bounds__(1024) block_norm_sum_kernel(const float *__restrict__ parts, int rows, int C, float *grad_post, float *grad_scale, float *grad_pre)
{
    sum_columns<kCols>(parts, rows, 3ll * C, (long long)blockIdx.x * kCols, [=](long long col, float v) {
        if (col < C) {
            if (grad_post) grad_post[col] = v;
        } else if (col < 2ll * C) {
            if (grad_scale) grad_scale[col - C] = v;
        } else if (grad_pre) {
            grad_pre[col - 2ll * C] = v;
        }
    });
}

Args arguments(const esrnn_block_norm_shape &s, const BlockNormArgs &a)
{
    Args p{};
    p.a = a;
    p.y = s.y_stride, p.gate = s.gate_stride, p.residual = s.residual_stride, p.sum = s.sum_stride, p.out = s.out_stride;
    p.grad_out = s.grad_out_stride, p.grad_sum = s.grad_sum_stride, p.grad_y = s.grad_y_stride, p.grad_gate = s.grad_gate_stride;
    p.grad_residual = s.grad_residual_stride;
    p.rows = s.rows, p.C = s.C, p.before = s.gate == ESRNN_GATE_BEFORE, p.after = s.gate == ESRNN_GATE_AFTER;
    // (at least the smallest normal number, or the root of a row of zeros is zero)
    p.eps = std::max(s.eps, std::numeric_limits<float>::min()), p.inverse = 1.0f / s.C;
    return p;
}

// In reverse four channels a lane, requested ahead: 32768 rows of 2048 channels, bf16, 236 us by eight waves, 264 by four with eight channels, 411 by two with
// sixteen.  Forward eight channels, by as many waves as the registers allow, which need no requests ahead: 134 us by four waves (144 ahead), 145 by
// eight with four channels; 30000 rows of 500 channels 32 by one wave, 46 by two.
template <bool kReverse, class F>
hipError_t with_layout(int C, F &&f)
{
    if (C <= 64) return f(Layout<16, 1>{});
    if (C <= 128) return f(Layout<32, 1>{});
    if (C <= 256) return f(Layout<64, 1>{});
    if constexpr (kReverse) {
        if (C <= 512) return f(Layout<64, 2>{});
        if (C <= 1024) return f(Layout<64, 4>{});
        if (C <= 2048) return f(Layout<64, 8>{});
        if (C <= 4096) return f(Layout<64, 16>{});
        return f(Layout<64, 16, 2, false>{});
    } else {
        if (C <= 512) return f(Layout<64, 1, 2, false>{});
        if (C <= 1024) return f(Layout<64, 2, 2, false>{});
        if (C <= 2048) return f(Layout<64, 4, 2, false>{});
        if (C <= 4096) return f(Layout<64, 8, 2, false>{});
        return f(Layout<64, 16, 2, false>{});
    }
}
template <class F>
hipError_t with_types(const esrnn_block_norm_shape &s, F &&f)
{
    return with_element(s.dtype, [&](auto e) {
        if (s.stream_dtype == s.dtype) return f(e, e);
        return f(e, float{});
    });
}
// As many workgroups as the chip holds: some 8 waves a SIMD forward, 4 in reverse (32768 x 2048 bf16 in reverse 367 us with half as many, 30000 x 500 125
// for 82).
template <class Y>
int workgroups(int rows, bool reverse)
{
    return (int)std::min<long long>(((long long)rows + Y::RW - 1) / Y::RW, (reverse ? kWavesReverse : kWavesForward) / (Y::kThreads / 64));
}

}  // namespace

size_t block_norm_workspace_floats(const esrnn_block_norm_shape &s)
{
    size_t rows = 0;
    with_layout<true>(s.C, [&](auto y) {
        rows = workgroups<decltype(y)>(s.rows, true);
        return hipSuccess;
    });
    return rows * 3 * s.C;
}

hipError_t launch_block_norm_forward(const esrnn_block_norm_shape &s, const BlockNormArgs &a, hipStream_t st)
{
    const Args p = arguments(s, a);
    return with_types(s, [&](auto e, auto r) {
        return with_layout<false>(s.C, [&](auto y) {
            typedef decltype(y) Y;
            block_norm_forward_kernel<decltype(e), decltype(r), Y><<<dim3(workgroups<Y>(s.rows, false)), Y::kThreads, 0, st>>>(p);
            return hipGetLastError();
        });
    });
}

hipError_t launch_block_norm_backward(const esrnn_block_norm_shape &s, const BlockNormArgs &a, hipStream_t st)
{
    const Args p = arguments(s, a);
    int rows = 0;
    const hipError_t failed = with_types(s, [&](auto e, auto r) {
        return with_layout<true>(s.C, [&](auto y) {
            typedef decltype(y) Y;
            rows = workgroups<Y>(s.rows, true);
            if constexpr (Y::M > 1) block_norm_wide_backward_kernel<decltype(e), decltype(r), Y><<<dim3(rows), Y::kThreads, 0, st>>>(p);
            else block_norm_backward_kernel<decltype(e), decltype(r), Y><<<dim3(rows), Y::kThreads, 0, st>>>(p);
            return hipGetLastError();
        });
    });
    if (failed != hipSuccess || !(a.grad_post_weight || a.grad_scale || a.grad_pre_weight)) return failed;
    return with_columns(3ll * s.C, [&](auto cols) {
        constexpr int kCols = decltype(cols)::value;
        block_norm_sum_kernel<kCols><<<dim3((3 * s.C + kCols - 1) / kCols), 1024, 0, st>>>(a.parts, rows, s.C, a.grad_post_weight, a.grad_scale, a.grad_pre_weight);
        return hipGetLastError();
    });
}

}  // namespace esrnn
