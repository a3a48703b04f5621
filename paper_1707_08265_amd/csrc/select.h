// What the kernels of the selective scan share (select_forward.hip, select_backward.hip).
//
// For each channel, with N states and d = log(1 + exp(delta + bias)), a = exp(d A):
//   h_t[n] = a h_{t-1}[n] + d x B_t[n],   y = (sum_n C_t[n] h_t[n] + D x) z sigma(z)
//
// The rows, whatever sequences they belong to, are cut into strips; a wave takes a strip of some channels.  What a strip does to the state that
// comes into it is h -> exp(A sum d) h + E (E its end from a state of zero), or h -> E if a sequence begins in it.  Three launches: the
// strips' (sum d, E), which only the rows from the last beginning on have a part in, and none where the strip's last row ends a sequence; the
// states between strips; the strips again, now with the state that comes into each (two launches for few strips, one for a single one).
// It is bound by vector instructions: a state and row takes an exponential, which costs two others (3.5 ns an instruction and SIMD; a
// multiply-add 1.5), and three or four more in each of the two passes over the rows.
#pragma once

#include "layer.h"
#include "rows.h"

namespace dgn {

constexpr int kSelectWaves = 4;         // of a workgroup; each works by itself
constexpr int kSelectBatch = 8;         // rows that a wave has in registers at a time
constexpr int kSelectMostRows = 64;     // of a strip
// Sums over the channels of a workgroup wait in memory for those of the others, [blocks of channels][rows][2 states], which is as much as the
// square of the states: backward a launch takes as many strips as these many bytes have room for, but those of so many workgroups at
// least, for what the last of a launch leave idle (backward of 16 384 x 2 048 in bf16, ms, in one launch, in ones of 256 MiB, of 4 096
// workgroups, and as it is: 128 states 8.22, 7.87, 7.87 and 7.85, for 4.8 and 1.3 GiB of scratch; 256 states 21.1, 24.0, 22.1 and 21.7, for 17.5
// and 2.5 GiB).
constexpr int64_t kSharedBytes = (int64_t)256 << 20, kSharedGroups = 8192;
constexpr int kSelectKeep = 16;         // rows between two states that the forward pass keeps for the backward pass
// Up to so many strips each applies the ones before it itself, half as many where a lane has 16 states (forward with that and with the launch
// between, us: 32 strips of 512 x 2 048 x 16 27.0 and 32.5; 64 of 1 024 x 512, four states a lane, 22.3 and 23.7; 64 of 1 024 x 2 048, 16
// states, 47.2 and 38.9; 128 of 2 048 x 512, four states, 37.6 and 34.7).
constexpr int64_t kFewSelectStrips = 64;
constexpr float kLog2e = 1.44269504088896340736f, kLog2eLow = 1.92596299112661746887e-8f, kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float exp2_of(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float inverse(float v) { return __builtin_amdgcn_rcpf(v); }

// log(1 + exp(v)) = max(v, 0) + 2 artanh(s), s = q / (2 + q), q = exp(-|v|); artanh(s) / s is 1 + s^2 times a polynomial in s^2 <= 1/9 (by least
// squares at Chebyshev's points, 2^-25.9 off).  The argument of the exponential is carried in two parts.  And its derivative sigma(v).
__device__ __forceinline__ float small_exp(float v)     // exp(-|v|)
{
    const float w = -fabsf(v), t = w * kLog2e, e = fmaf(w, kLog2eLow, fmaf(w, kLog2e, -t)), q = exp2_of(t);
    return t < -126.0f ? 0.0f : fmaf(q, e * kLn2, q);       // (w of -inf: e is NaN)
}
struct Step { float d, slope; };
__device__ __forceinline__ Step step_and_slope(float v)
{
    const float q = small_exp(v), s = q * inverse(2.0f + q), r = s * s, k = inverse(1.0f + q);
    float p = fmaf(r, 0.13433805108070374f, 0.1411697268486023f);
    p = fmaf(r, p, 0.2000383585691452f);
    p = fmaf(r, p, 0.33333319425582886f);
    const float half = fmaf(s * r, p, s), positive = v > 0.0f ? v : 0.0f;
    return Step{fmaf(2.0f, half, positive), v > 0.0f ? k : q * k};
}
__device__ __forceinline__ float step_of(float v) { return step_and_slope(v).d; }
// sigma(z): of 32 bits by a rounded exponential and quotient.
template <class T> __device__ __forceinline__ float gate_of(float z)
{
    if (sizeof(typename T::Store) == 4) return 1.0f / (1.0f + expf(-z));
    return inverse(1.0f + exp2_of(z * -kLog2e));
}

// What a strip does to a state.  Its sum of d says so if a sequence begins in it (sums are at least 0, or no numbers).  A sum of finite steps that
// passes the range of floats is its end: infinity times an A of 0, or that of a state that there is not, would be no number.  (A step that
// is no number is in the strip's end too.)
constexpr float kCutSpan = -1.0f, kMostSpan = 3.402823466e38f;
__device__ __forceinline__ float kept_span(float span) { return fminf(span, kMostSpan); }
__device__ __forceinline__ float apply_strip(float span, float end, float A2, float h)
{
    return span == kCutSpan ? end : fmaf(exp2_of(span * A2), h, end);
}

// Sum over the L lanes of a channel, L a power of two: inside a row of 16 lanes by moves (quads, then mirrors of lanes that agree).
template <int kControl> __device__ __forceinline__ float moved(float v)
{
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), kControl, 0xf, 0xf, true));
}
template <int L> __device__ __forceinline__ float sum_channel(float v)
{
    if (L > 1) v += moved<0xB1>(v);         // lanes 1 0 3 2 of a quad
    if (L > 2) v += moved<0x4E>(v);         // lanes 2 3 0 1
    if (L > 4) v += moved<0x141>(v);        // lanes 7 .. 0 of eight
    if (L > 8) v += moved<0x140>(v);        // lanes 15 .. 0 of sixteen
    if (L > 16) v += __shfl_xor(v, 16, kWave);
    if (L > 32) v += __shfl_xor(v, 32, kWave);
    return v;
}

// The strip of a wave; the channel and the S of its states that a lane has, L lanes a channel.
template <int S, int L> struct Lane {
    static constexpr int kWide = S * L;     // states of a channel with those that there are not, which stay 0
    static constexpr int kChannels = kWave / L;
    int64_t row0, c, group, strip;
    int32_t rows, n0, part, count;          // first state, place among the channel's lanes, states that there are
    bool active;                            // lanes past the group's end do what its last channel's do, and write nothing
    u64 valid, begin, end;
    int32_t seq;

    __device__ __forceinline__ bool find(const SelectArgs &a, int64_t number)
    {
        if (number >= a.strips * a.blocks) return false;
        strip = divide(number, a.blocks);
        place(a, number - strip * a.blocks);
        row0 = strip * a.rows;
        const int64_t left = a.tokens - row0;
        rows = (int32_t)(left < a.rows ? left : a.rows);
        return true;
    }
    __device__ __forceinline__ void place(const SelectArgs &a, int64_t block) { place(a, block, divide(block, a.group_blocks)); }
    __device__ __forceinline__ void place(const SelectArgs &a, int64_t block, int64_t group_)
    {
        group = group_;
        const int64_t share = a.channels / a.groups, at = (block - group * a.group_blocks) * kChannels + lane_id() / L;
        active = at < share;
        c = group * share + (active ? at : share - 1);
        part = lane_id() % L;
        n0 = part * S;
        const int64_t some = a.states - n0;
        count = some < 0 ? 0 : some > S ? S : (int32_t)some;
    }
    __device__ __forceinline__ void mark(const SelectArgs &a, int32_t *own)
    {
        const RowSeq s = sequences_of(a.rowptr, a.seqs, a.tokens, row0, own);
        const int64_t row = row0 + lane_id();
        const bool mine = s.q >= 0 && lane_id() < rows;
        seq = s.q;
        valid = __ballot(mine);
        begin = __ballot(mine && s.first == row);
        end = __ballot(mine && s.end == row + 1);
    }
    __device__ __forceinline__ int64_t q(int k) const { return __builtin_amdgcn_readlane(seq, k); }
    // The lane's states in arrays of [..][channels][states].
    __device__ __forceinline__ void load(const SelectArgs &a, const float *p, int64_t row, float (&h)[S]) const
    {
        const float *at = p + (row * a.channels + c) * a.states + n0;
        if (p && a.states % 4 == 0) {
#pragma unroll
            for (int i = 0; i < S; i += 4) {
                Pack<F32, 4> v = {};
                if (i < count) v.load(at + i);
#pragma unroll
                for (int k = 0; k < 4; k++) h[i + k] = v.get(k);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < S; i++) h[i] = p && i < count ? at[i] : 0.0f;
    }
    template <bool kStream = false> __device__ __forceinline__ void store(const SelectArgs &a, float *p, int64_t row, const float (&h)[S]) const
    {
        float *at = p + (row * a.channels + c) * a.states + n0;
        if (a.states % 4 == 0) {
#pragma unroll
            for (int i = 0; i < S; i += 4) {
                const float some[4] = {h[i], h[i + 1], h[i + 2], h[i + 3]};
                Pack<F32, 4> v;
                v.set(some);
                if (active && i < count) v.template store<kStream>(at + i);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < S; i++) if (active && i < count) at[i] = h[i];
    }
    // The same in the library's own arrays of [..][channels][kWide], 16 bytes at a time.
    __device__ __forceinline__ int64_t own(const SelectArgs &a, int64_t row) const { return (row * a.channels + c) * kWide + n0; }
    __device__ __forceinline__ void load_own(const float *p, float (&h)[S]) const
    {
#pragma unroll
        for (int i = 0; i < S; i += 4) {
            const float4 v = *reinterpret_cast<const float4 *>(p + i);
            h[i] = v.x, h[i + 1] = v.y, h[i + 2] = v.z, h[i + 3] = v.w;
        }
    }
    __device__ __forceinline__ void store_own(float *p, const float (&h)[S]) const
    {
        if (!active) return;
#pragma unroll
        for (int i = 0; i < S; i += 4) *reinterpret_cast<float4 *>(p + i) = make_float4(h[i], h[i + 1], h[i + 2], h[i + 3]);
    }
    // A log2(e), so that exp(d A) is the base-2 exponential of a product.
    __device__ __forceinline__ void decays(const SelectArgs &a, float (&A2)[S]) const
    {
        load(a, a.A, 0, A2);
#pragma unroll
        for (int i = 0; i < S; i++) A2[i] *= kLog2e;
    }
    // The state that comes into the strip: the launch between has left it, or (few strips) those before it are applied here.
    template <bool kBack> __device__ __forceinline__ void before(const SelectArgs &a, const float (&A2)[S], float (&h)[S]) const
    {
        if (a.before) { load_own((kBack ? a.back : a.before) + own(a, strip), h); return; }
#pragma unroll
        for (int i = 0; i < S; i++) h[i] = 0.0f;
        const int64_t n = kBack ? a.strips - 1 - strip : strip;
        constexpr int kAhead = S == 4 ? 8 : 2;          // (strips that are asked for at once)
#pragma unroll kAhead
        for (int64_t k = 0; k < n; k++) {
            const int64_t at = kBack ? a.strips - 1 - k : k;
            float e[S];
            load_own(a.ends + own(a, at), e);
            const float span = a.spans[at * a.channels + c];
#pragma unroll
            for (int i = 0; i < S; i++) h[i] = apply_strip(span, e[i], A2[i], h[i]);
        }
    }
};

// Rows of B or C, kSelectBatch of them, from memory to a wave's own LDS [rows][kWide] as floats; states that there are not are 0.
template <class T, int kWide, int kRows> struct Shared {
    typedef typename T::Store E;
    static constexpr int kEach = (kRows * kWide + kWave - 1) / kWave;
    E v[kEach];
    __device__ __forceinline__ void load(const void *p, int64_t stride, int64_t row0, const SelectArgs &a, int64_t group)
    {
#pragma unroll
        for (int i = 0; i < kEach; i++) {
            const int e = i * kWave + lane_id(), n = e % kWide;
            int64_t row = row0 + e / kWide;
            row = row < a.tokens ? row : a.tokens - 1;
            v[i] = n < a.states ? static_cast<const E *>(p)[row * stride + group * a.states + n] : (E)0.0f;
        }
    }
    __device__ __forceinline__ void put(float *lds) const
    {
#pragma unroll
        for (int i = 0; i < kEach; i++) if (kEach * kWave == kRows * kWide || i * kWave + lane_id() < kRows * kWide) lds[i * kWave + lane_id()] = (float)v[i];
    }
};
// A lane's S of a row of it.
template <int S> __device__ __forceinline__ void take_states(const float *lds, float (&v)[S])
{
#pragma unroll
    for (int i = 0; i < S; i += 4) {
        const float4 f = *reinterpret_cast<const float4 *>(lds + i);
        v[i] = f.x, v[i + 1] = f.y, v[i + 2] = f.z, v[i + 3] = f.w;
    }
}
// A lane's channel in kRows rows of an array.
template <class T, int kRows> struct Column {
    typedef typename T::Store E;
    E v[kRows];
    __device__ __forceinline__ void load(const void *p, int64_t stride, int64_t row0, int64_t c, int64_t tokens)
    {
        const E *at = static_cast<const E *>(p) + c;
#pragma unroll
        for (int k = 0; k < kRows; k++) v[k] = at[(row0 + k < tokens ? row0 + k : tokens - 1) * stride];
    }
    __device__ __forceinline__ float get(int k) const { return (float)v[k]; }
};

// The arguments of the kernel (its first parameter) from where the launch has put them.  They do not fit the scalar registers of a wave that
// also has a loop's own values there; what a part of the loop needs of them it asks for anew, and the compiler does not keep it from part to part.
__device__ __forceinline__ SelectArgs asked_again()
{
    typedef const __attribute__((address_space(4))) SelectArgs *At;
    At p = (At)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const SelectArgs *)p;
}

// How lanes and strips are cut.
struct SelectLayout {
    int S, L;                       // forward; backward has four states a lane
    int64_t group_blocks, blocks, rows, strips;
    int64_t back_group_blocks, back_blocks, slice;
    int wide;
    size_t spans, ends, before, partial, shared, copy, forward_bytes, bytes, carry;
};
SelectLayout select_layout(const SelectArgs &a);
void select_states(const SelectArgs &a, int wide, bool back, hipStream_t s);
void select_forward(int dtype, const SelectArgs &a, const SelectLayout &l, hipStream_t s);
void select_backward(int dtype, const SelectArgs &a, const SelectLayout &l, hipStream_t s);

// call(S, L): the forms that select_layout may choose.
#define DGN_BY_LANES(S, L, call)                                                         \
    do {                                                                                 \
        if ((S) == 16) {                                                                 \
            switch (L) {                                                                 \
            case 1: call(16, 1); break;                                                  \
            case 2: call(16, 2); break;                                                  \
            case 4: call(16, 4); break;                                                  \
            case 8: call(16, 8); break;                                                  \
            default: call(16, 16);                                                       \
            }                                                                            \
        } else {                                                                         \
            switch (L) {                                                                 \
            case 1: call(4, 1); break;                                                   \
            case 2: call(4, 2); break;                                                   \
            case 4: call(4, 4); break;                                                   \
            case 8: call(4, 8); break;                                                   \
            case 16: call(4, 16); break;                                                 \
            case 32: call(4, 32); break;                                                 \
            default: call(4, 64);                                                        \
            }                                                                            \
        }                                                                                \
    } while (0)

}  // namespace dgn
