// Checks of arguments that the entry points of the operators on values share.
#pragma once

#include "values.h"

namespace dgn {

constexpr int64_t kMaxCount = 2147483646;
#define DGN_HIP(expr)                                         \
    do {                                                      \
        hipError_t e__ = (expr);                              \
        if (e__ != hipSuccess) return note_hip_error(e__);    \
    } while (0)

inline size_t round256(size_t v) { return (v + 255) & ~(size_t)255; }
inline bool misaligned(const void *p, size_t to) { return ((uintptr_t)p & (to - 1)) != 0; }
inline bool type_known(int32_t dtype) { return dtype == DGN_F32 || dtype == DGN_F16 || dtype == DGN_BF16; }

// Rows in memory, in bytes.  Two of them meet if they have a byte in common; rows of one buffer may lie between each other's (columns of
// a wider matrix), if they are as far apart.
struct Span { const void *at; int64_t rows, stride, width; };
inline bool meet(Span a, Span b)
{
    if (!a.at || !b.at || a.rows <= 0 || b.rows <= 0 || a.width <= 0 || b.width <= 0) return false;
    if (a.rows == 1) a.stride = b.rows == 1 ? a.width : b.stride;
    if (b.rows == 1) b.stride = a.stride;
    const uintptr_t pa = (uintptr_t)a.at, pb = (uintptr_t)b.at;
    if (pa > pb) return meet(b, a);
    const uint64_t apart = pb - pa;
    if (apart >= (unsigned __int128)(a.rows - 1) * (uint64_t)a.stride + (uint64_t)a.width) return false;
    if (a.stride != b.stride) return true;
    const int64_t off = (int64_t)(apart % (uint64_t)a.stride);
    return off < a.width || a.stride - off < b.width;
}
template <int N> bool meets(Span a, const Span (&others)[N])
{
    for (int i = 0; i < N; i++) if (meet(a, others[i])) return true;
    return false;
}
inline Span dense(const void *p, int64_t rows, int64_t row_bytes) { return Span{p, rows, row_bytes, row_bytes}; }      // (no gaps)

}  // namespace dgn
