// What the layer operators (include/esrnn_layers.h) share: element types, aligned and unaligned groups of four channels,
// the sigmoid in both directions, and the launch functions that layers_api.cpp calls.
#pragma once

#include "device_utils.h"
#include "esrnn_layers.h"

namespace esrnn {

template <class E>
using Vec4 = E __attribute__((ext_vector_type(4)));
// the same at the alignment of one element: the hardware's global accesses ask for no more
template <class E>
struct Loose {
    typedef E Four __attribute__((ext_vector_type(4), aligned(sizeof(E))));
};

// f(element type tag) for the element type of a call (checked before)
template <class F>
hipError_t with_element(int dtype, F &&f)
{
    switch (dtype) {
    case ESRNN_F32: return f(float{});
    case ESRNN_BF16: return f(__bf16{});
    default: return f(_Float16{});
    }
}

template <class E>
__device__ __forceinline__ f32x4 to_f32(Vec4<E> v)
{
    return __builtin_convertvector(v, f32x4);
}
template <class E>
__device__ __forceinline__ Vec4<E> from_f32(f32x4 v)
{
    return __builtin_convertvector(v, Vec4<E>);
}

// Groups of four elements at a scalar base and a lane's offset in bytes, at multiples of four bytes: no address is left to compute on the vector
// ALU.  A lane at kOutside reads zeros and writes nothing; a base reaches over less than 2 GiB.
constexpr unsigned kOutside = 0x80000000u;
__device__ __forceinline__ buf_rsrc make_base(const void *p) { return make_rsrc(p, 0x7fffffff); }
template <class E>
__device__ __forceinline__ Vec4<E> load_four(buf_rsrc base, unsigned lane_bytes, unsigned scalar_bytes = 0)
{
    if constexpr (sizeof(E) == 4) return __builtin_bit_cast(Vec4<E>, __builtin_amdgcn_raw_buffer_load_b128(base, lane_bytes, scalar_bytes, 0));
    else return __builtin_bit_cast(Vec4<E>, __builtin_amdgcn_raw_buffer_load_b64(base, lane_bytes, scalar_bytes, 0));
}
// (four dwords: no scalar offset, see buf_store4)
template <class E>
__device__ __forceinline__ void store_four(buf_rsrc base, unsigned lane_bytes, Vec4<E> v)
{
    if constexpr (sizeof(E) == 4) buf_store4(base, lane_bytes, v);
    else __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, v), base, lane_bytes, 0, 0);
}

// A lane has four channels of a row of tiles of 4 W channels, W lanes side by side.  Aligned: neighbours, one wide access; the last lane of a
// row whose channels are no multiple of four has the last four of them, so that two lanes have the same channel (C >= 4).  Else
// the channels lane, lane + W, ..: every access of the W lanes is one run of neighbouring elements.
template <bool kAligned, int W>
struct Channels {
    int first, count;       // first channel of this lane, and how many there are in all
    __device__ __forceinline__ Channels(int lane, int begin, int C) : first(begin + (kAligned ? 4 * lane : lane)), count(C)
    {
        if (kAligned && first < C) first = min(first, C - 4);
    }
    __device__ __forceinline__ int channel(int k) const { return first + (kAligned ? k : W * k); }
    __device__ __forceinline__ bool exists(int k) const { return channel(k) < count; }
    // a channel that can be read in the place of one that does not exist
    __device__ __forceinline__ int readable(int k) const
    {
        return kAligned ? min(first, count - 4) + k : min(channel(k), count - 1);
    }
    template <class E>
    __device__ __forceinline__ Vec4<E> load(const E *row) const
    {
        if constexpr (kAligned) return *reinterpret_cast<const Vec4<E> *>(row + readable(0));
        Vec4<E> v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = row[readable(k)];
        return v;
    }
    template <class E>
    __device__ __forceinline__ void store(E *row, Vec4<E> v) const
    {
        if constexpr (kAligned) {
            if (exists(0)) *reinterpret_cast<Vec4<E> *>(row + first) = v;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (exists(k)) row[channel(k)] = v[k];
        }
    }
};

// sigmoid(g) and sigmoid(-g) (1 - sigmoid would lose the digits of the small one): with E = exp(-g), 1 / (1 + E) and E / (1 + E).  The hardware's
// reciprocal gives no denormals: where 1 + E is above 2^126 (g < -87.3) it is zero, which is what the first is then taken to be; in the second 2^-126
// stands in its place, so that the product is 1 or more, up to infinity, and the minimum makes the 1 it has to be.  (The minimum that keeps a NaN:
// a gate that is NaN makes both of them NaN.)  The larger of the two is off by about a unit in the last place; the smaller one by up to |g| units of 2^-24
// more, as the exponent is one rounded product: 29 at |g| = 30.  Infinite gates give exactly 0 and 1.
struct Sigmoids {
    float of, of_minus;
};
__device__ __forceinline__ Sigmoids sigmoids(float g)
{
    const float e = __builtin_amdgcn_exp2f(g * kSigmoidExponent), r = fast_rcp(1.0f + e);
    return Sigmoids{r, __builtin_elementwise_minimum(e * fmaxf(r, 0x1p-126f), 1.0f)};
}

inline bool aligned_to(const void *p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
inline size_t element_bytes(int dtype) { return dtype == ESRNN_F32 ? 4 : 2; }

// ---- gated linear recurrence (recurrence_kernels.hip) ----
// Waves of a workgroup, positions of a thread and of a block, the blocks of a sequence; ahead: every block has a workgroup of its own, and its maps go
// through `words` floats of the workspace, by whole groups of 2^log_group blocks too.
struct RecurrencePlan {
    int waves, steps, block, blocks;
    bool ahead;
    int log_group, groups;
    size_t tickets, words;
};
RecurrencePlan recurrence_plan(const esrnn_recurrence_shape &s);
struct RecurrenceForward {
    const void *x, *gate;
    const int32_t *lengths;
    const float *initial;
    void *out;
    float *last, *saved, *words;
};
struct RecurrenceBackward {
    const void *x, *gate;
    const int32_t *lengths;
    const float *saved;
    const void *grad_out;
    const float *grad_last;
    void *grad_x, *grad_gate;
    float *grad_initial, *words;
};
hipError_t launch_recurrence_forward(const esrnn_recurrence_shape &s, const RecurrenceForward &a, hipStream_t st);
hipError_t launch_recurrence_backward(const esrnn_recurrence_shape &s, const RecurrenceBackward &a, hipStream_t st);
struct RecurrenceStep {
    const void *x, *gate;
    long long x_stride, gate_stride, out_stride;
    const int32_t *slots;
    float *state;
    void *out;
    int rows, pool, C;
};
hipError_t launch_recurrence_step(int kind, int dtype, const RecurrenceStep &a, hipStream_t st);

// ---- AdamW over many tensors (adamw_kernels.hip) ----
// Elements of a workgroup: 2048, or 1024 in lists of up to 512 chunks, that do not fill the chip (40 tensors of 3000 elements, norm and update:
// 5.0 + 4.5 us with 2048, 3.7 + 3.7 with 1024; 73 M elements, update alone: 360, 373 with 4096).
constexpr int kAdamWChunk = 2048, kAdamWSmallChunk = 1024, kAdamWFewChunks = 512, kAdamWNormBlocks = 256, kAdamWEntriesAtOnce = 56;
struct AdamWEntry {
    float *param;
    const void *grad;
    void *copy;
    long long n, flat;          // elements; where the tensor begins in the moments
    float weight_decay;
    int first_chunk;
    unsigned char grad_dtype, copy_dtype;
};
struct AdamWUpdate {
    const AdamWEntry *entries;
    const int *owner;           // tensor of every chunk
    const double *partial;      // sums of squares, or null without clipping
    int n_partial;
    float lr, beta1, new1, beta2, new2, eps, clip_norm;     // new1 = 1 - beta1, new2 = 1 - beta2
    float rate, root_correction;        // lr / (1 - beta1^step), 1 / sqrt(1 - beta2^step)
    unsigned key;               // of the random bits
    void *m;
    float *v;
    void *r;
    float *m_scale, *r_scale, *norm;
};
hipError_t launch_adamw_bind(const AdamWEntry *host, int count, AdamWEntry *entries, int *owner, int chunks, hipStream_t st);
hipError_t launch_adamw_update(const AdamWUpdate &u, int chunk, int chunks, double *partial, int state_bits, hipStream_t st);

// ---- group norm + activation (group_norm_kernels.hip) ----
struct GroupNormArgs {
    const void *x, *grad_out;
    const int32_t *lengths;
    const float *scale, *shift, *stats_in;
    void *out, *grad_x;
    float *stats, *grad_scale, *grad_shift;
    float *parts;               // the workspace
};
// Whether every position is normalised by itself, by kernels of their own (T = 1 and groups that they hold).
bool group_norm_single_positions(const esrnn_group_norm_shape &s);
size_t group_norm_workspace_floats(const esrnn_group_norm_shape &s);
hipError_t launch_group_norm_forward(const esrnn_group_norm_shape &s, const GroupNormArgs &a, hipStream_t st);
hipError_t launch_group_norm_backward(const esrnn_group_norm_shape &s, const GroupNormArgs &a, hipStream_t st);

}  // namespace esrnn
