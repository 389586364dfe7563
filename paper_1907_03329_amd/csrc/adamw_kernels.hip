// AdamW over many tensors at once (include/esrnn_layers.h).
//
// All tensors are one list of chunks of 2048 elements (of 1024 in short lists), a workgroup each, so that a list of any length is one launch (two with
// clipping: sums of squares in a fixed order first, which every workgroup of the update adds up in the same order).  A chunk finds its
// tensor through a table in the workspace.  A wave has whole blocks of 256 elements, four neighbours a lane: the block of an 8-bit
// moment's scale is one wave's, and its largest magnitude takes six steps within the wave.
//
// fp32 moments: memory is the bound.  73 M elements with bf16 gradients and a bf16 copy, 28 bytes each, take 360 us, 5.7 TB/s; the norm reads the
// gradients once more, 2 bytes each, in 57 us, behind the write-back of what the program before it left in the caches (25 us by itself).
// 8-bit moments: the same elements without a copy, 14 bytes each, take 190 us among other passes (178 to 215 as single dispatches), 5.4 TB/s, and the vector ALU
// is as near its bound, with some 80 instructions an element: roots rounded correctly, 32 random bits, two codes.  40 tensors of some 3000 elements:
// launches, 3.7 us for each of the two kernels.
//
// The moments are fp32; 8 bits are a choice of the caller's: m and r = sqrt(v), which has half of v's range, as e4m3 with a scale for 256
// neighbours, rounded up with the probability of what is cut off, so that small changes are not lost over many steps.
#include <algorithm>
#include <cmath>

#include "layers_internal.h"

namespace esrnn {

namespace {

// magnitude of e4m3's largest number, and the factor that brings its exponents to those at a float's lower end (exponent bias
// 7 against 127): the upper 12 bits of the scaled magnitude, denormal or not, are the code
constexpr float kMostE4m3 = 448.0f, kToCode = 0x1p-120f, kLeastScale = 0x1p-100f;

// N groups of four neighbours of this lane, 256 elements apart, of a tensor of n elements; `whole`: all of the wave's groups are in it (the same
// in all lanes).  Pointers out of a table are told to be global memory.
template <class E, int N>
__device__ __forceinline__ void load_groups(const void *base, long long first, long long n, bool whole, f32x4 (&v)[N])
{
    typedef typename Loose<E>::Four Four;
    const auto *p = (const __attribute__((address_space(1))) E *)base + first;
    if (whole) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = to_f32<E>(*reinterpret_cast<const __attribute__((address_space(1))) Four *>(p + 256 * j));
        return;
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) v[j][k] = first + 256 * j + k < n ? (float)p[256 * j + k] : 0.0f;
}
// one of them
template <class E>
__device__ __forceinline__ void store_group(void *base, long long at, long long n, bool whole, f32x4 v)
{
    typedef typename Loose<E>::Four Four;
    auto *p = (__attribute__((address_space(1))) E *)base + at;
    const Vec4<E> r = from_f32<E>(v);
    if (whole) {
        *reinterpret_cast<__attribute__((address_space(1))) Four *>(p) = r;
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (at + k < n) p[k] = r[k];
}
template <int N>
__device__ __forceinline__ void load_grad(const AdamWEntry &e, long long first, bool whole, f32x4 (&g)[N])
{
    if (e.grad_dtype == ESRNN_BF16) load_groups<__bf16>(e.grad, first, e.n, whole, g);
    else if (e.grad_dtype == ESRNN_F16) load_groups<_Float16>(e.grad, first, e.n, whole, g);
    else load_groups<float>(e.grad, first, e.n, whole, g);
}

// Sums of squares in fp64, by 256 workgroups of 16 waves however many chunks there are: their partial sums are few enough for each workgroup of the
// update to add up by itself, so that no third launch stands between the two.
template <int kChunk>
__global__ void __launch_bounds__(1024) adamw_norm_kernel(const AdamWEntry *__restrict__ entries, const int *__restrict__ owner, int chunks,
                                                          double *__restrict__ partial)
{
    constexpr int kGroups = kChunk / 256;
    __shared__ double s_wave[16];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    double acc = 0.0;       // (squares of fp32 numbers do not overflow)
    const int step = gridDim.x * 16;
    int chunk = __builtin_amdgcn_readfirstlane(blockIdx.x * 16 + wave);
    // the next chunk's tensor is looked up while this one's elements are under way
    AdamWEntry e = chunk < chunks ? entries[owner[chunk]] : AdamWEntry{};
    while (chunk < chunks) {
        const int next = chunk + step;
        const long long first = (long long)(chunk - e.first_chunk) * kChunk;
        f32x4 g[kGroups];
        load_grad(e, first + 4 * lane, first + kChunk <= e.n, g);
        e = entries[owner[min(next, chunks - 1)]];
#pragma unroll
        for (int j = 0; j < kGroups; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) acc += (double)g[j][k] * (double)g[j][k];
        chunk = next;
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) acc += __shfl_xor(acc, off, 64);
    if (lane == 0) s_wave[wave] = acc;
    __syncthreads();
    if (threadIdx.x == 0) {
        double sum = 0.0;
        for (int w = 0; w < 16; ++w) sum += s_wave[w];
        partial[blockIdx.x] = sum;
    }
}

// largest of the wave's 64 (bit patterns of magnitudes: a NaN is above infinity, and that above all numbers)
__device__ __forceinline__ int wave_max_bits(int v)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v = max(v, __shfl_xor(v, off, 64));
    return v;
}

// of a place's lower word, and the key with what its upper word adds
__device__ __forceinline__ unsigned key_of(long long place, unsigned key) { return (unsigned)(place >> 32) * 0xC2B2AE35u ^ key; }
__device__ __forceinline__ unsigned random_word(unsigned place, unsigned key)
{
    unsigned w = place ^ key;
    w = (w ^ w >> 16) * 0x7FEB352Du;
    w = (w ^ w >> 15) * 0x846CA68Bu;
    return w ^ w >> 16;
}

// sqrt, correctly rounded from 2^-104 on and to a unit in the last place below: the hardware's root is off by one unit at most, and which of the
// three it has to be shows in the sign of x - root (root +- a unit), of which nothing may be left in a float below 2^-104.  Zero, infinity and NaN stay.
__device__ __forceinline__ float root_of(float x)
{
    const float s = __builtin_amdgcn_sqrtf(x);
    const float below = __builtin_bit_cast(float, __builtin_bit_cast(int, s) - 1), above = __builtin_bit_cast(float, __builtin_bit_cast(int, s) + 1);
    const float down = __builtin_fmaf(-below, s, x), up = __builtin_fmaf(-above, s, x);
    return up > 0.0f ? above : down <= 0.0f ? below : s;
}

struct Scale {
    float scale, inverse;
    bool finite;
};
__device__ __forceinline__ Scale scale_of(int most_bits)
{
    const float scale = __builtin_bit_cast(float, most_bits) * (1.0f / kMostE4m3);
    if (most_bits >= 0x7f800000) return {__builtin_nanf(""), 0.0f, false};
    return scale > kLeastScale ? Scale{scale, 1.0f / scale, true} : Scale{0.0f, 0.0f, true};
}
// a magnitude in units of the scale (not zero unless magnitude or scale are) as the float whose upper 12 bits are its code, rounded down
__device__ __forceinline__ unsigned scaled(float units) { return __builtin_bit_cast(unsigned, units * kToCode); }
// 16 random bits behind the three of the code's mantissa, of the 20 that are cut off: up with the probability of what is cut off
__device__ __forceinline__ unsigned code_of(unsigned y, unsigned bits16) { return (y + (bits16 << 4)) >> 20; }

// Every operation rounded by itself, as an elementwise program rounds them: which of two codes a moment takes hangs on its last bits.
__device__ __forceinline__ void moments(f32x4 &m, f32x4 &v, f32x4 g, const AdamWUpdate &u)
{
#pragma clang fp contract(off)
    m = u.beta1 * m + u.new1 * g;
    v = u.beta2 * v + u.new2 * (g * g);
}

// kBits: of the moments.
template <int kBits, int kChunk>
__global__ void __launch_bounds__(256) adamw_update_kernel(AdamWUpdate u)
{
    constexpr int kGroups = kChunk / 1024;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, chunk = blockIdx.x;
    const AdamWEntry e = u.entries[u.owner[chunk]];
    const long long first = (long long)(chunk - e.first_chunk) * kChunk + wave * (256 * kGroups) + 4 * lane;
    const long long flat = e.flat + first;      // place in the moments

    const bool whole = first - 4 * lane + 256 * kGroups <= e.n;
    f32x4 p[kGroups], g[kGroups], m[kGroups], v[kGroups];
    unsigned m8[kGroups], r8[kGroups];
    float m_scale[kGroups], r_scale[kGroups];
    load_groups<float>(e.param, first, e.n, whole, p);
    load_grad(e, first, whole, g);
#pragma unroll
    for (int j = 0; j < kGroups; ++j) {
        const bool block = first - 4 * lane + 256 * j < e.n;        // (uniform: the wave has a block here)
        if (kBits == 32) {
            m[j] = v[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            if (block) {
                m[j] = *reinterpret_cast<const f32x4 *>(static_cast<const float *>(u.m) + flat + 256 * j);
                v[j] = *reinterpret_cast<const f32x4 *>(u.v + flat + 256 * j);
            }
        } else {
            m8[j] = r8[j] = 0;
            m_scale[j] = r_scale[j] = 0.0f;
            if (block) {
                m8[j] = reinterpret_cast<const unsigned *>(u.m)[(flat + 256 * j) >> 2];
                r8[j] = reinterpret_cast<const unsigned *>(u.r)[(flat + 256 * j) >> 2];
                m_scale[j] = u.m_scale[(flat + 256 * j) >> 8];
                r_scale[j] = u.r_scale[(flat + 256 * j) >> 8];
            }
        }
    }
    float scale = 1.0f;
    if (u.partial) {
        __shared__ double s_sum[4];
        static_assert(kAdamWNormBlocks <= 256, "");
        double sum = (int)threadIdx.x < u.n_partial ? u.partial[threadIdx.x] : 0.0;
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
        if (lane == 0) s_sum[wave] = sum;
        __syncthreads();
        const float norm = (float)sqrt((s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]));
        if (u.norm && blockIdx.x == 0 && threadIdx.x == 0) *u.norm = norm;
        if (!(norm < __builtin_inff())) return;     // infinite or NaN: nothing changes
        scale = fminf(1.0f, u.clip_norm / (norm + 1e-6f));
    }
    const float keep = 1.0f - u.lr * e.weight_decay;
#pragma unroll
    for (int j = 0; j < kGroups; ++j) {
        if (first + 256 * j - 4 * lane >= e.n) break;
        if (kBits == 8) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(m8[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(m8[j], true);
            const auto rlo = __builtin_amdgcn_cvt_pk_f32_fp8(r8[j], false), rhi = __builtin_amdgcn_cvt_pk_f32_fp8(r8[j], true);
            m[j] = f32x4{lo[0], lo[1], hi[0], hi[1]} * m_scale[j];
            const f32x4 r = f32x4{rlo[0], rlo[1], rhi[0], rhi[1]} * r_scale[j];
            v[j] = r * r;
        }
        f32x4 root;
        moments(m[j], v[j], g[j] * scale, u);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            root[k] = root_of(v[j][k]);
            p[j][k] = keep * p[j][k] - u.rate * m[j][k] * fast_rcp(root[k] * u.root_correction + u.eps);
        }
        store_group<float>(e.param, first + 256 * j, e.n, whole, p[j]);
        if (e.copy) {
            if (e.copy_dtype == ESRNN_BF16) store_group<__bf16>(e.copy, first + 256 * j, e.n, whole, p[j]);
            else store_group<_Float16>(e.copy, first + 256 * j, e.n, whole, p[j]);
        }
        if (kBits == 32) {
            *reinterpret_cast<f32x4 *>(static_cast<float *>(u.m) + flat + 256 * j) = m[j];
            *reinterpret_cast<f32x4 *>(u.v + flat + 256 * j) = v[j];
            continue;
        }
        int most_m = 0, most_r = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            most_m = max(most_m, __builtin_bit_cast(int, fabsf(m[j][k])));
            most_r = max(most_r, __builtin_bit_cast(int, fabsf(root[k])));
        }
        const Scale sm = scale_of(wave_max_bits(most_m)), sr = scale_of(wave_max_bits(most_r));
        unsigned m_codes = 0, r_codes = 0;
        const unsigned place = (unsigned)(flat + 256 * j), key = key_of(flat + 256 * j, u.key);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const unsigned w = random_word(place + k, key);      // (a multiple of four: no carry into the upper word)
            const float mk = m[j][k];       // (a bit cast of the vector's element itself is one of its first element)
            const float units = root[k] * sr.inverse;
            const unsigned ym = scaled(fabsf(mk) * sm.inverse), yr = scaled(units), sign = __builtin_bit_cast(unsigned, mk) >> 24 & 0x80u;
            m_codes |= (code_of(ym, w >> 16) | sign) << 8 * k;
            // (at least one for any root: `yr` itself may be too small for a float)
            r_codes |= max(code_of(yr, w & 0xffffu), min(__builtin_bit_cast(unsigned, units), 1u)) << 8 * k;
        }
        if (!sm.finite) m_codes = 0x7f7f7f7fu;
        if (!sr.finite) r_codes = 0x7f7f7f7fu;
        reinterpret_cast<unsigned *>(u.m)[(flat + 256 * j) >> 2] = m_codes;
        reinterpret_cast<unsigned *>(u.r)[(flat + 256 * j) >> 2] = r_codes;
        if (lane == 0) {
            u.m_scale[(flat + 256 * j) >> 8] = sm.scale;
            u.r_scale[(flat + 256 * j) >> 8] = sr.scale;
        }
    }
}

// The table comes to the device as arguments of launches: no copy from host memory that might still be read after the call.
struct Some {
    AdamWEntry entry[kAdamWEntriesAtOnce];
};
__global__ void __launch_bounds__(64) adamw_entries_kernel(Some some, int n, AdamWEntry *to)
{
    if ((int)threadIdx.x < n) to[threadIdx.x] = some.entry[threadIdx.x];
}
__global__ void __launch_bounds__(256) adamw_owners_kernel(const AdamWEntry *entries, int count, int *owner, int chunks)
{
    const int chunk = blockIdx.x * 256 + threadIdx.x;
    if (chunk >= chunks) return;
    int lo = 0, hi = count;         // the last entry whose first chunk is not behind this one
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (entries[mid].first_chunk <= chunk) lo = mid;
        else hi = mid;
    }
    owner[chunk] = lo;
}

}  // namespace

hipError_t launch_adamw_bind(const AdamWEntry *host, int count, AdamWEntry *entries, int *owner, int chunks, hipStream_t st)
{
    for (int first = 0; first < count; first += kAdamWEntriesAtOnce) {
        Some some{};
        const int n = std::min(kAdamWEntriesAtOnce, count - first);
        std::copy(host + first, host + first + n, some.entry);
        adamw_entries_kernel<<<1, 64, 0, st>>>(some, n, entries + first);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    adamw_owners_kernel<<<(chunks + 255) / 256, 256, 0, st>>>(entries, count, owner, chunks);
    return hipGetLastError();
}

namespace {

template <int kChunk>
hipError_t launch_update(AdamWUpdate u, int chunks, double *partial, int state_bits, hipStream_t st)
{
    if (u.clip_norm > 0.0f) {
        u.partial = partial;
        u.n_partial = std::min((chunks + 15) / 16, kAdamWNormBlocks);
        adamw_norm_kernel<kChunk><<<u.n_partial, 1024, 0, st>>>(u.entries, u.owner, chunks, partial);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (state_bits == 32) adamw_update_kernel<32, kChunk><<<chunks, 256, 0, st>>>(u);
    else adamw_update_kernel<8, kChunk><<<chunks, 256, 0, st>>>(u);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_adamw_update(const AdamWUpdate &u, int chunk, int chunks, double *partial, int state_bits, hipStream_t st)
{
    return chunk == kAdamWChunk ? launch_update<kAdamWChunk>(u, chunks, partial, state_bits, st)
                                : launch_update<kAdamWSmallChunk>(u, chunks, partial, state_bits, st);
}

}  // namespace esrnn
