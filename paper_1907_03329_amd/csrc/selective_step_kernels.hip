// Selective scan, one position of many requests (include/esrnn_state_space.h): a lane has four states of a channel, so that a pool's rows are read and
// written by 16 bytes a lane, all lanes of a wave side by side.  A workgroup keeps its channels' rates of decay in registers and takes requests one behind
// the other.  States are the bound, read and written once: 1024 requests of 2048 channels of 16 states, bf16, 281 MB, 46 us (6.2 TB/s) over and over on a few
// pools, which the last-level cache holds in part, and 67 us (4.2 TB/s) in turn with other work.
#include <algorithm>

#include "selective_scan.h"

namespace esrnn {

namespace {

constexpr int kThreads = 256;

// L lanes of a channel, 4 L >= N; kFours: N = 4 L, and states at multiples of 16 bytes.
template <class E, int L, bool kFours>
__global__ void __launch_bounds__(kThreads) selective_step_kernel(esrnn_selective_step_shape s, SelectiveStep a, int tiles)
{
    constexpr int kChannels = kThreads / L;
    const int tile = blockIdx.x % tiles, first_row = blockIdx.x / tiles, rows_apart = gridDim.x / tiles;
    const int part = threadIdx.x % L, n0 = 4 * part, in_tile = tile * kChannels + (int)threadIdx.x / L;
    const bool exists = in_tile < s.C;
    const int channel = min(in_tile, s.C - 1), group = channel / (s.C / s.G);
    float A[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) A[r] = n0 + r < s.N ? exponent_rate(a.A[(size_t)channel * s.N + n0 + r]) : 0.0f;
    const float bias = a.bias ? a.bias[channel] : 0.0f, D = a.D ? a.D[channel] : 0.0f;
    for (int i = first_row; i < s.rows; i += rows_apart) {
        const int slot = a.slots ? a.slots[i] : i;
        E *out = static_cast<E *>(a.out) + i * s.out_stride;
        if (slot < 0 || slot >= s.pool) {
            if (exists && part == 0) out[channel] = (E)0.0f;
            continue;
        }
        float *state = a.state + ((size_t)slot * s.C + channel) * s.N + n0;
        const E *b = static_cast<const E *>(a.b) + i * s.b_stride + (size_t)group * s.N + n0, *c = static_cast<const E *>(a.c) + i * s.c_stride + (size_t)group * s.N + n0;
        float h[4], bs[4], cs[4];
        if constexpr (kFours) {
            const f32x4 v = *reinterpret_cast<const f32x4 *>(state);
#pragma unroll
            for (int r = 0; r < 4; ++r) h[r] = v[r], bs[r] = (float)b[r], cs[r] = (float)c[r];
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const bool there = n0 + r < s.N;
                h[r] = there ? state[r] : 0.0f, bs[r] = there ? (float)b[r] : 0.0f, cs[r] = there ? (float)c[r] : 0.0f;
            }
        }
        const float x = (float)(static_cast<const E *>(a.x) + i * s.x_stride)[channel];
        const float d = step_size((static_cast<const E *>(a.delta) + i * s.delta_stride)[channel], bias, s.delta_kind == ESRNN_DELTA_SOFTPLUS).of, u = d * x;
        float y = part == 0 ? D * x : 0.0f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            h[r] = fmaf(__builtin_amdgcn_exp2f(d * A[r]), h[r], u * bs[r]);
            y = fmaf(cs[r], h[r], y);
        }
        if (exists) {
            if constexpr (kFours) {
                *reinterpret_cast<f32x4 *>(state) = f32x4{h[0], h[1], h[2], h[3]};
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (n0 + r < s.N) state[r] = h[r];
            }
        }
#pragma unroll
        for (int off = 1; off < L; off *= 2) y += __shfl_xor(y, off, 64);
        if (exists && part == 0) out[channel] = (E)y;
    }
}

}  // namespace

hipError_t launch_selective_step(const esrnn_selective_step_shape &s, const SelectiveStep &a, hipStream_t st)
{
    const auto launch = [&](auto e, auto lanes) {
        typedef decltype(e) E;
        constexpr int L = decltype(lanes)::value;
        const int tiles = (s.C + kThreads / L - 1) / (kThreads / L);
        const int rows = (int)std::min<long long>(s.rows, std::max(1, 4096 / tiles));
        const dim3 grid((unsigned)(tiles * rows));
        if (s.N == 4 * L && aligned_to(a.state, 16)) selective_step_kernel<E, L, true><<<grid, kThreads, 0, st>>>(s, a, tiles);
        else selective_step_kernel<E, L, false><<<grid, kThreads, 0, st>>>(s, a, tiles);
        return hipGetLastError();
    };
    return with_element(s.dtype, [&](auto e) {
        if (s.N <= 4) return launch(e, std::integral_constant<int, 1>{});
        if (s.N <= 8) return launch(e, std::integral_constant<int, 2>{});
        if (s.N <= 16) return launch(e, std::integral_constant<int, 4>{});
        if (s.N <= 32) return launch(e, std::integral_constant<int, 8>{});
        return launch(e, std::integral_constant<int, 16>{});
    });
}

}  // namespace esrnn
