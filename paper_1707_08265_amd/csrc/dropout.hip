// Dropout from a counter, added to a residual:  y = residual + keep x scale.
//
// The draws are those of Philox 4x32 with ten rounds (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random numbers: as easy as 1, 2, 3",
// 2011): a block of four 32-bit words is a function of a 64-bit key and a 128-bit counter, so that a thread makes the eight 16-bit draws of its
// eight elements from their place alone, and the backward pass makes the same ones again.  16 bits a draw: with 32, twice the integer work, it
// would be bound by that work (20 products and about 60 other instructions a block) and not by memory.  65 537 x 1 024 in bf16: with a residual 403
// MB in 73 us (5.5 TB/s), without 268 MB in 44 (6.0; a copy has 6.2), both together 118 as well on tensors of which the last-level cache has nothing.
#include "layer.h"
#include "rows.h"

namespace dgn {

constexpr int kDraws = 8, kDropThreads = 256;

__device__ __forceinline__ void philox(u64 block, u64 seed, u64 offset, uint32_t (&c)[4])
{
    c[0] = (uint32_t)block;
    c[1] = (uint32_t)(block >> 32);
    c[2] = (uint32_t)offset;
    c[3] = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; r++) {
        const u64 p = (u64)0xD2511F53u * c[0], q = (u64)0xCD9E8D57u * c[2];
        c[0] = (uint32_t)(q >> 32) ^ c[1] ^ k0;
        c[1] = (uint32_t)q;
        c[2] = (uint32_t)(p >> 32) ^ c[3] ^ k1;
        c[3] = (uint32_t)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

// kFlat: rows without gaps, taken as one.  Otherwise eight neighbours may be of two rows or more.
template <class T, bool kResidual, bool kFlat, bool kStream>
__global__ __launch_bounds__(kDropThreads) void k_dropout(DropArgs a)
{
    typedef typename T::Store S;
    constexpr int kPart = 16 / (int)sizeof(S), kParts = kDraws / kPart;
    const int64_t n = a.rows * a.columns, blocks = (n + kDraws - 1) / kDraws;
    const u64 seed = a.key[0], offset = a.key[1];
    const S *x = static_cast<const S *>(a.x), *residual = static_cast<const S *>(a.residual);
    S *y = static_cast<S *>(a.y);
    for (int64_t b = (int64_t)blockIdx.x * kDropThreads + threadIdx.x; b < blocks; b += (int64_t)gridDim.x * kDropThreads) {
        const int64_t e = b * kDraws, row = kFlat ? 0 : divide(e, a.columns), column = e - row * a.columns;
        const bool whole = kFlat ? e + kDraws <= n : column + kDraws <= a.columns;
        uint32_t w[4];
        if (whole) {
            Pack<T, kPart> in[kParts], to[kParts];
#pragma unroll
            for (int i = 0; i < kParts; i++) {
                in[i].load(x + row * a.x_stride + column + i * kPart);
                if (kResidual) to[i].load(residual + row * a.residual_stride + column + i * kPart);
            }
            philox(b, seed, offset, w);
#pragma unroll
            for (int i = 0; i < kParts; i++) {
                float out[kPart];
#pragma unroll
                for (int k = 0; k < kPart; k++) {
                    const int d = i * kPart + k;
                    const bool keep = (d % 2 ? w[d / 2] >> 16 : w[d / 2] & 0xffff) >= a.drop;
                    const float v = keep ? in[i].get(k) * a.scale : 0.0f;
                    out[k] = kResidual ? v + to[i].get(k) : v;
                }
                to[i].set(out);
                to[i].template store<kStream>(y + row * a.y_stride + column + i * kPart);
            }
            continue;
        }
        philox(b, seed, offset, w);
        for (int d = 0; d < kDraws && e + d < n; d++) {
            const int64_t at_row = kFlat ? 0 : divide(e + d, a.columns), at = e + d - at_row * a.columns;
            const uint32_t word = d < 4 ? (d < 2 ? w[0] : w[1]) : (d < 6 ? w[2] : w[3]);
            const bool keep = (d % 2 ? word >> 16 : word & 0xffff) >= a.drop;
            const float v = keep ? (float)x[at_row * a.x_stride + at] * a.scale : 0.0f;
            y[at_row * a.y_stride + at] = (S)(kResidual ? v + (float)residual[at_row * a.residual_stride + at] : v);
        }
    }
}

template <class T> static void go_dropout(const DropArgs &a, hipStream_t s)
{
    const int64_t c = a.columns, groups = (a.rows * c + kDraws * kDropThreads - 1) / (kDraws * kDropThreads);
    const dim3 grid((unsigned)(groups < (1 << 23) ? groups : 1 << 23)), threads(kDropThreads);
    const bool flat = a.rows == 1 || (a.x_stride == c && a.y_stride == c && (!a.residual || a.residual_stride == c));
    // results of calls that are larger than the last-level cache go past it (65 537 x 1 024: 75.3 -> 72.7 us with a residual, 44.9 -> 44.4)
    const bool stream = flat && (size_t)(a.rows * c) * (a.residual ? 3 : 2) * sizeof(typename T::Store) > kStreamBytes;
#define DGN_GO(R, F, P) hipLaunchKernelGGL((k_dropout<T, R, F, P>), grid, threads, 0, s, a)
    if (a.residual) {
        if (stream) DGN_GO(true, true, true);
        else if (flat) DGN_GO(true, true, false);
        else DGN_GO(true, false, false);
    } else {
        if (stream) DGN_GO(false, true, true);
        else if (flat) DGN_GO(false, true, false);
        else DGN_GO(false, false, false);
    }
#undef DGN_GO
}
hipError_t launch_dropout(int dtype, const DropArgs &a, hipStream_t s)
{
#define DGN_GO(T) go_dropout<T>(a, s)
    DGN_BY_DTYPE(dtype, DGN_GO);
#undef DGN_GO
    return hipGetLastError();
}

__global__ __launch_bounds__(256) void k_zero(float *out, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) out[i] = 0.0f;
}
hipError_t launch_zero(float *out, int64_t n, hipStream_t s)
{
    if (!out || n <= 0) return hipSuccess;
    const int64_t groups = (n + 255) / 256;
    hipLaunchKernelGGL(k_zero, dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(256), 0, s, out, n);
    return hipGetLastError();
}

}  // namespace dgn
