// Rows of ragged sequences and packed elements: what the operators on values share.
#pragma once

#include "values.h"

#include <type_traits>

namespace dgn {

__device__ __forceinline__ int64_t row_bound(int64_t v, int64_t tokens) { return v < 0 ? 0 : v > tokens ? tokens : v; }

__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

typedef uint32_t Word __attribute__((aligned(2)));
typedef uint32_t Pair __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t Quad4 __attribute__((ext_vector_type(4), aligned(4)));

// V neighbouring elements, at an address that is aligned to one, as they are in memory.
template <class T, int V> struct Pack {
    typedef typename T::Store S;
    static constexpr int kBytes = V * (int)sizeof(S), kWords = kBytes < 4 ? 1 : kBytes / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const S *p)
    {
        if (kBytes == 2) w[0] = *reinterpret_cast<const uint16_t *>(p);
        else if (kBytes == 4) w[0] = *reinterpret_cast<const Word *>(p);
        else if (kBytes == 8) { const Pair v = *reinterpret_cast<const Pair *>(p); w[0] = v[0]; w[1 % kWords] = v[1]; }
        else {
            const Quad4 v = take<false, sizeof(S), Quad4>(p);
#pragma unroll
            for (int i = 0; i < 4; i++) w[i % kWords] = v[i];
        }
    }
    template <bool kStream = false> __device__ __forceinline__ void store(S *p) const
    {
        if (kBytes == 2) put<kStream, sizeof(S)>(p, (uint16_t)w[0]);
        else if (kBytes == 4) put<kStream, sizeof(S)>(p, (Word)w[0]);
        else if (kBytes == 8) put<kStream, sizeof(S)>(p, Pair{w[0], w[1 % kWords]});
        else put<kStream, sizeof(S)>(p, Quad4{w[0], w[1 % kWords], w[2 % kWords], w[3 % kWords]});
    }
    __device__ __forceinline__ float get(int i) const
    {
        if (sizeof(S) == 4) return __uint_as_float(w[i]);
        const uint16_t h = (uint16_t)(w[i / 2 % kWords] >> (i % 2 * 16));
        return (float)__builtin_bit_cast(typename std::conditional<sizeof(S) == 2, S, _Float16>::type, h);
    }
    __device__ __forceinline__ void set(const float (&f)[V])
    {
        if (sizeof(S) == 4) {
#pragma unroll
            for (int i = 0; i < V; i++) w[i % kWords] = __float_as_uint(f[i]);
        } else {
            typedef typename std::conditional<sizeof(S) == 2, S, _Float16>::type H;
            typedef H H2 __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int i = 0; i < V; i += 2) w[i / 2 % kWords] = __builtin_bit_cast(uint32_t, H2{(H)f[i], (H)f[i + 1 < V ? i + 1 : i]});
        }
    }
    // From here on the compiler knows nothing of the value.
    __device__ __forceinline__ void forget()
    {
#pragma unroll
        for (int i = 0; i < kWords; i++) asm volatile("" : "+v"(w[i]));
    }
};

__device__ __forceinline__ int64_t uniform(int64_t v)
{
    return (int64_t)((u64)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)v));
}
__device__ __forceinline__ int64_t divide(int64_t n, int64_t by)       // (both fit 32 bits but in the largest of calls)
{
    return n >> 32 || by >> 32 ? n / by : (int64_t)((uint32_t)n / (uint32_t)by);
}

// Number of rowptr[0 .. n-1] below `value`; one wave, 64 looks at a time.
__device__ __forceinline__ int64_t rows_below(const int64_t *rowptr, int64_t n, int64_t value)
{
    int64_t l = 0, r = n;
    while (l < r) {
        const int64_t step = (r - l + kWave - 1) / kWave, at = l + lane_id() * step;
        const int below = __popcll(__ballot(at < r && rowptr[at < r ? at : l] < value));
        if (below == 0) return l;
        const int64_t top = l + below * step;
        l += (below - 1) * step + 1;
        r = top < r ? top : r;
    }
    return l;
}

// The sequences of 64 rows from row0 on, one row to a lane: its number, first row and the row after its last, or -1.  One wave; own: room
// for kWave numbers in LDS, a wave's own.  Row pointers that do not ascend give sequences that mean nothing, with first <= row < end.
struct RowSeq { int32_t q; int64_t first, end; };
__device__ __forceinline__ RowSeq sequences_of(const int64_t *rowptr, int64_t seqs, int64_t tokens, int64_t row0, int32_t *own)
{
    const int lane = lane_id();
    own[lane] = -1;
    wave_fence();
    const int64_t row = row0 + lane;
    if (seqs < kWave) {                 // all pointers in one look (rows are fewer than 2^31)
        const int32_t p = (int32_t)row_bound(lane <= seqs ? rowptr[lane] : tokens, tokens);
        const int64_t at = p - row0;
        if (lane <= seqs && at >= 0 && at < kWave) atomicMax(&own[at], lane);
        wave_fence();
        const int q0 = __popcll(__ballot(lane <= seqs && p <= row0)) - 1;
        int q = wave_incl_max(own[lane]);
        q = q < q0 ? q0 : q;
        const int32_t first = __shfl(p, q < 0 ? 0 : q, kWave), end = __shfl(p, q < 0 ? 0 : q + 1 < kWave ? q + 1 : q, kWave);
        return q >= 0 && q < seqs && row < tokens && first <= row && row < end ? RowSeq{q, first, end} : RowSeq{-1, 0, 0};
    }
    const int64_t q0 = uniform(rows_below(rowptr, seqs + 1, row0 + 1)) - 1;       // the last pointer that is not past row0
    for (int64_t at = q0 + 1;; at += kWave) {
        const int64_t q = at + lane;
        const int64_t p = q <= seqs ? row_bound(rowptr[q], tokens) - row0 : kWave;
        if (p >= 0 && p < kWave) atomicMax(&own[p], (int32_t)q);                  // (of sequences without rows and the one after them: that one)
        if (!__all(p < kWave)) break;
    }
    wave_fence();
    int32_t q = wave_incl_max(own[lane]);
    q = q < (int32_t)q0 ? (int32_t)q0 : q;
    RowSeq r = {-1, 0, 0};
    if (q >= 0 && q < seqs && row < tokens) {
        const int64_t first = row_bound(rowptr[q], tokens), end = row_bound(rowptr[q + 1], tokens);
        if (first <= row && row < end) r = RowSeq{q, first, end};
    }
    return r;
}

// States of sequences without rows, `width` elements each: out = in (or zero).  A unit is kCopySlice elements of every kCopyPhases-th of those
// among 64 sequences; one after the other they are taken by the waves of the launch that are left for it.  (What is read goes to registers first:
// for all that the compiler knows in may be out, and each read would wait for the write before it.  14 of 96 sequences, 32 768 floats each, by one wave for 64 sequences: 2 089 us,
// the launch without them 355.)
constexpr int64_t kCopySlice = 1024, kCopyPhases = 8, kMostCopyGroups = 1024;
inline int64_t copy_groups(int64_t seqs, int64_t width, int waves)     // workgroups of so many waves
{
    const int64_t units = (seqs + kWave - 1) / kWave * kCopyPhases * ((width + kCopySlice - 1) / kCopySlice), n = (units + waves - 1) / waves;
    return n < kMostCopyGroups ? n : kMostCopyGroups;
}
template <class S> __device__ __forceinline__ void copy_empties(const int64_t *rowptr, int64_t seqs, int64_t tokens, int64_t width, const S *in, S *out,
                                                                int64_t wave, int64_t waves)
{
    constexpr int kEach = kCopySlice / kWave;
    const int64_t slices = (width + kCopySlice - 1) / kCopySlice, units = (seqs + kWave - 1) / kWave * kCopyPhases * slices;
    for (int64_t unit = wave; unit < units; unit += waves) {
        const int64_t some_of = divide(unit, slices), block = some_of / kCopyPhases, from = (unit - some_of * slices) * kCopySlice, q = block * kWave + lane_id();
        const int phase = (int)(some_of % kCopyPhases);
        const bool empty = q < seqs && row_bound(rowptr[q], tokens) >= row_bound(rowptr[q + 1], tokens);
        int number = 0;
        for (u64 some = __ballot(empty); some; some &= some - 1, number++) {
            if (number % kCopyPhases != phase) continue;
            const int64_t at = (block * kWave + __builtin_ctzll(some)) * width + from + lane_id(), left = width - from - lane_id();
            S v[kEach];
#pragma unroll
            for (int k = 0; k < kEach; k++) v[k] = in && k * kWave < left ? in[at + k * kWave] : (S)0.0f;
#pragma unroll
            for (int k = 0; k < kEach; k++) if (k * kWave < left) out[at + k * kWave] = v[k];
        }
    }
}

}  // namespace dgn
