// What the operators of a selective state space layer (include/esrnn_state_space.h) share: channels of a lane, sums over rows of partial
// results, the softplus, and the launch functions that state_space_api.cpp calls.
#pragma once

#include "esrnn_state_space.h"
#include "layers_internal.h"

namespace esrnn {

// V neighbouring channels of a lane from `first` on, of `count` in all: one access of 16 bytes at the alignment of one element where all of them
// exist, one by one in the last lane of a row that they do not fill.
template <class E, int V>
struct Neighbours {
    typedef E LooseValues __attribute__((ext_vector_type(V), aligned(sizeof(E))));
    typedef E Values __attribute__((ext_vector_type(V)));
    typedef unsigned Bits __attribute__((ext_vector_type(V * sizeof(E) / 4)));
    typedef float Floats __attribute__((ext_vector_type(V)));
    int first, count;
    __device__ __forceinline__ bool some() const { return first < count; }
    __device__ __forceinline__ bool all() const { return first + V <= count; }
    // zeros where there are no channels
    __device__ __forceinline__ Values load(const E *row) const
    {
        Values v = {};
        if (all()) {
            v = *reinterpret_cast<const LooseValues *>(row + first);
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (first + k < count) v[k] = row[first + k];
        }
        return v;
    }
    __device__ __forceinline__ void store(E *row, Values v) const
    {
        if (all()) {
            *reinterpret_cast<LooseValues *>(row + first) = v;
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (first + k < count) row[first + k] = v[k];
        }
    }
    static __device__ __forceinline__ Floats widen(Values v) { return __builtin_convertvector(v, Floats); }
    static __device__ __forceinline__ Values round(Floats v) { return __builtin_convertvector(v, Values); }
};

// The same where kWide says that there are V channels at least: then the last lane with channels has the last V there are, so that two lanes may
// have the same channel, compute the same and write the same.  Else one by one, and the last channel in the place of those that do not exist.
template <class E, int V, bool kWide>
struct Overlapping {
    typedef Neighbours<E, V> N;
    int first, count;
    __device__ __forceinline__ Overlapping(int begin, int C) : first(kWide && begin < C ? min(begin, C - V) : begin), count(C) {}
    __device__ __forceinline__ bool some() const { return first < count; }
    __device__ __forceinline__ int channel(int k) const { return kWide ? min(first, count - V) + k : min(first + k, count - 1); }
    __device__ __forceinline__ typename N::Values load(const E *row) const
    {
        typename N::Values v;
        if constexpr (kWide) {
            v = *reinterpret_cast<const typename N::LooseValues *>(row + channel(0));
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k) v[k] = row[channel(k)];
        }
        return v;
    }
    // (by lanes with channels)
    __device__ __forceinline__ void store(E *row, typename N::Values v) const
    {
        if constexpr (kWide) {
            *reinterpret_cast<typename N::LooseValues *>(row + first) = v;
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (first + k < count) row[first + k] = v[k];
        }
    }
};

// Sums of `rows` rows of `cols` partial results, in a fixed order, for kCols columns from `first` on: by a workgroup of 1024 threads, 1024 / kCols rows at
// a time; store(column, sum) by the threads of the first row.  Few columns need narrow workgroups to be many, many columns whole cache lines: 1024 rows of 150
// columns 3.9 us by 16 columns and 9.3 by 64, 512 rows of 6144 columns 20 us by 16 and 14 by 64.
template <int kCols, class F>
__device__ __forceinline__ void sum_columns(const float *__restrict__ parts, long long rows, long long cols, long long first, F &&store)
{
    constexpr int kRows = 1024 / kCols;
    __shared__ float s_sum[kRows][kCols];
    const int lane = threadIdx.x % kCols, row = threadIdx.x / kCols;
    const long long col = first + lane;
    constexpr int kBatch = 8;       // loads under way
    float v[kBatch] = {};
    if (col < cols) {
        long long r = row;
        for (; r + (kBatch - 1) * kRows < rows; r += kBatch * kRows)
#pragma unroll
            for (int k = 0; k < kBatch; ++k) v[k] += parts[(r + kRows * k) * cols + col];
        for (; r < rows; r += kRows) v[0] += parts[r * cols + col];
    }
    s_sum[row][lane] = ((v[0] + v[4]) + (v[2] + v[6])) + ((v[1] + v[5]) + (v[3] + v[7]));
    __syncthreads();
#pragma unroll
    for (int half = kRows / 2; half > 0; half /= 2) {
        if (row < half) s_sum[row][lane] += s_sum[row + half][lane];
        __syncthreads();
    }
    if (row == 0 && col < cols) store(col, s_sum[0][lane]);
}
// f(std::integral_constant<int, kCols>)
template <class F>
hipError_t with_columns(long long cols, F &&f)
{
    if (cols >= 6000) return f(std::integral_constant<int, 64>{});
    if (cols >= 2048) return f(std::integral_constant<int, 32>{});
    return f(std::integral_constant<int, 16>{});
}

// softplus(v) = max(v, 0) + log(1 + exp(-|v|)) and its derivative sigmoid(v).  Of w = 1 + e, rounded, log(1 + e) = log(w) + (e - (w - 1)) / (1 + ..),
// where the second term is what the rounding has lost of e, without which small e would lose all digits; its divisor is left out, as the term is below 2^-24
// where that is not 1.  The hardware's logarithm is off by 2^-23 of itself at w near 1 too (all floats from 1 to 2 in steps of eight tried).
// exp(-|v|) is zero below 2^-126.
struct Softplus {
    float of, slope;
};
__device__ __forceinline__ Softplus softplus(float v)
{
    const float e = __builtin_amdgcn_exp2f(fabsf(v) * kSigmoidExponent), w = 1.0f + e, r = fast_rcp(w);
    const float l = fmaf(__builtin_amdgcn_logf(w), 0.69314718055994531f, e - (w - 1.0f));
    return {fmaxf(v, 0.0f) + l, v < 0.0f ? e * r : r};
}

// u sigmoid(u) and its derivative, p (1 + u (1 - p)).  An infinite u gives -0 and 0, or itself and 1, not the product of zero and infinity.
struct Silu {
    float of, slope;
};
__device__ __forceinline__ Silu silu(float u)
{
    const Sigmoids s = sigmoids(u);
    const float of = s.of == 0.0f ? -0.0f : u * s.of;
    return {of, fmaf(fminf(of, 0x1p127f), s.of_minus, s.of)};
}

// ---- short causal convolution (convolution_kernels.hip) ----
struct ConvolutionArgs {
    const void *x, *grad_out, *initial;
    const int32_t *lengths;
    const float *weight, *bias, *grad_last;
    void *out, *last, *grad_x;
    float *grad_weight, *grad_bias, *grad_initial;
    float *parts;               // the workspace: (K + 1) sums of every channel for every workgroup
};
size_t convolution_workspace_floats(const esrnn_convolution_shape &s);
hipError_t launch_convolution_forward(const esrnn_convolution_shape &s, const ConvolutionArgs &a, hipStream_t st);
hipError_t launch_convolution_backward(const esrnn_convolution_shape &s, const ConvolutionArgs &a, hipStream_t st);
hipError_t launch_convolution_step(const esrnn_convolution_step_shape &s, const void *x, const float *weight, const float *bias, const int32_t *slots,
                                   void *state, void *out, hipStream_t st);

// ---- selective scan (selective_forward_kernels.hip, selective_backward_kernels.hip, selective_step_kernels.hip) ----
struct SelectiveArgs {
    const void *x, *delta, *b, *c, *grad_out;
    const float *A, *D, *bias, *initial, *grad_last;
    const int32_t *lengths;
    void *out, *grad_x, *grad_delta, *grad_b, *grad_c;
    float *last, *saved, *grad_A, *grad_D, *grad_bias, *grad_initial;
    float *workspace;
};
size_t selective_workspace_floats(const esrnn_selective_shape &s, bool reverse);
size_t selective_saved_floats(const esrnn_selective_shape &s);
hipError_t launch_selective_forward(const esrnn_selective_shape &s, const SelectiveArgs &a, hipStream_t st);
hipError_t launch_selective_backward(const esrnn_selective_shape &s, const SelectiveArgs &a, hipStream_t st);
struct SelectiveStep {
    const void *x, *delta, *b, *c;
    const float *A, *D, *bias;
    const int32_t *slots;
    float *state;
    void *out;
};
hipError_t launch_selective_step(const esrnn_selective_step_shape &s, const SelectiveStep &a, hipStream_t st);

// ---- block norm (block_norm_kernels.hip) ----
struct BlockNormArgs {
    const void *y, *gate, *residual, *grad_out, *grad_sum;
    const int32_t *exists;
    const float *post_weight, *scale, *pre_weight, *stats_in;
    void *sum, *out, *grad_y, *grad_gate, *grad_residual;
    float *stats, *grad_post_weight, *grad_scale, *grad_pre_weight;
    float *parts;               // the workspace: three sums of every channel for every workgroup
};
constexpr int kBlockNormMostChannels = 8192;
size_t block_norm_workspace_floats(const esrnn_block_norm_shape &s);
hipError_t launch_block_norm_forward(const esrnn_block_norm_shape &s, const BlockNormArgs &a, hipStream_t st);
hipError_t launch_block_norm_backward(const esrnn_block_norm_shape &s, const BlockNormArgs &a, hipStream_t st);

}  // namespace esrnn
