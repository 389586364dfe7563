// Argument checks that the entry points of the layer operators share (layers_api.cpp, state_space_api.cpp).
#pragma once

#include <initializer_list>
#include <utility>

#include "layers_internal.h"

#define ESRNN_TRY(expr)                              \
    do {                                             \
        hipError_t e_ = (expr);                      \
        if (e_ != hipSuccess) return ESRNN_ERR_HIP;  \
    } while (0)

namespace esrnn {

constexpr int64_t kMostElements = int64_t(1) << 40;     // of an array, gaps included: sizes in bytes and addresses stay far from overflow

inline bool element_type(int dtype) { return dtype == ESRNN_F32 || dtype == ESRNN_BF16 || dtype == ESRNN_F16; }
inline bool element_aligned(const void *p, int dtype) { return aligned_to(p, element_bytes(dtype)); }
inline bool floats_aligned(const void *p) { return aligned_to(p, 4); }     // (of a null pointer too)

// Arrays of B sequences of T positions of C elements next to each other, at strides of a sequence and of a position.  S has B, T, C and dtype.
struct RowsShape {
    int64_t B, T, C;
    int dtype;
};

// Strides of a read array: any that keep it within kMostElements (zero for one sequence that is used for all of them, say).
template <class S>
bool readable_strides(const S &s, const int64_t st[2])
{
    return st[0] >= 0 && st[1] >= 0 && st[0] <= kMostElements / s.B && st[1] <= kMostElements / s.T;
}
// Of a written one: distinct elements, in either order.
template <class S>
bool writable_strides(const S &s, const int64_t st[2])
{
    if (!readable_strides(s, st)) return false;
    const bool positions_inside = (s.T == 1 || st[1] >= s.C) && (s.B == 1 || st[0] >= (s.T == 1 ? 0 : (int64_t)(s.T - 1) * st[1]) + s.C);
    const bool sequences_inside = (s.B == 1 || st[0] >= s.C) && (s.T == 1 || st[1] >= (s.B == 1 ? 0 : (int64_t)(s.B - 1) * st[0]) + s.C);
    return positions_inside || sequences_inside;
}

// Whether an array that is written shares elements with another one of its type, with rows of `other_row` elements, as far as strides show it:
// arrays that begin at one place, or have the same strides and lie within each other's reach.  (Those with strides of their own that reach into
// each other are taken to be the caller's design.)
template <class S>
bool rows_overlap(const S &s, const void *written, const int64_t written_stride[2], const void *other, const int64_t other_stride[2], int64_t other_row)
{
    if (written == other) return true;
    const int64_t e = (int64_t)element_bytes(s.dtype), row = s.C * e, row2 = other_row * e;
    const auto reach = [&](const int64_t st[2], int64_t r) { return ((s.B - 1) * st[0] + (s.T - 1) * st[1]) * e + r; };
    const int64_t apart = reinterpret_cast<intptr_t>(other) - reinterpret_cast<intptr_t>(written);
    if (apart >= reach(written_stride, row) || -apart >= reach(other_stride, row2)) return false;
    if ((s.B > 1 && written_stride[0] != other_stride[0]) || (s.T > 1 && written_stride[1] != other_stride[1])) return false;
    // Rows of the one are those of the other, moved.  Strides of a written array nest: all rows of the inner dimension lie within one step of the
    // outer one, so only the two nearest steps of each can bring two rows together.
    int64_t count[2] = {s.B, s.T}, step[2] = {s.B > 1 ? written_stride[0] * e : 0, s.T > 1 ? written_stride[1] * e : 0};
    if (step[0] < step[1]) std::swap(count[0], count[1]), std::swap(step[0], step[1]);
    for (int i = 0; i < 2; ++i) {
        const int64_t outer = step[0] ? (apart < 0 ? -(-apart / step[0]) - 1 : apart / step[0]) + i : 0, rest = apart - outer * step[0];
        for (int j = 0; j < 2; ++j) {
            const int64_t inner = step[1] ? (rest < 0 ? -(-rest / step[1]) - 1 : rest / step[1]) + j : 0, left = rest - inner * step[1];
            if (outer > -count[0] && outer < count[0] && inner > -count[1] && inner < count[1] && left > -row2 && left < row) return true;
        }
    }
    return false;
}
template <class S>
bool rows_overlap(const S &s, const void *written, const int64_t written_stride[2], const void *other, const int64_t other_stride[2])
{
    return rows_overlap(s, written, written_stride, other, other_stride, s.C);
}
// Whether an array that is written begins where another one does.  Null pointers are no arrays.
inline bool one_place(std::initializer_list<const void *> written, std::initializer_list<const void *> read)
{
    for (const void *const *w = written.begin(); w != written.end(); ++w) {
        if (!*w) continue;
        for (const void *const *o = w + 1; o != written.end(); ++o)
            if (*o == *w) return true;
        for (const void *o : read)
            if (o == *w) return true;
    }
    return false;
}
// of fp32 arrays of n and m elements, either of which may be null
inline bool floats_overlap(const float *a, size_t n, const float *b, size_t m) { return a && b && a < b + m && b < a + n; }

}  // namespace esrnn
