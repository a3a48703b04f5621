// Selective scan over ragged sequences: the forward pass, the states between strips, and one token (see select.h).
#include "select.h"

namespace dgn {

// First launch: what a strip does to the state that comes into it.  Bound by vector instructions, 99 a row and wave of 64
// channels x 16 states, 64 of them the states' (an exponential takes two slots of four cycles): 16 384 x 1 024 x 16 in bf16 63 us, 80 % of its
// cycles; its waves, four a SIMD, are for 14 % of their time behind memory or LDS.
template <class T, int S, int L>
__global__ __launch_bounds__(kSelectWaves *kWave) void k_select_ends(SelectArgs a)
{
    typedef Lane<S, L> Mine;
    __shared__ int32_t s_own[kSelectWaves][kWave];
    __shared__ __attribute__((aligned(16))) float s_b[kSelectWaves][kSelectBatch * Mine::kWide];
    float *lds = s_b[wave_id()];
    Mine ln;
    if (!ln.find(a, (int64_t)blockIdx.x * kSelectWaves + wave_id())) return;
    ln.mark(a, s_own[wave_id()]);
    if (!((ln.valid & ~ln.end) >> (ln.rows - 1) & 1)) {         // (nothing goes on past it; without a beginning no row belongs to a sequence)
        const float none[S] = {};
        ln.store_own(a.ends + ln.own(a, ln.strip), none);
        if (ln.active && ln.part == 0) a.spans[ln.strip * a.channels + ln.c] = kCutSpan;
        return;
    }
    const int from = ln.begin ? 63 - __builtin_clzll(ln.begin) : 0;
    float A2[S], h[S], span = 0.0f;
    ln.decays(a, A2);
#pragma unroll
    for (int i = 0; i < S; i++) h[i] = 0.0f;
    if (ln.begin) ln.load(a, a.h0, ln.q(from), h);
    const float bias = a.delta_bias ? a.delta_bias[ln.c] : 0.0f;
    Column<T, kSelectBatch> x, delta;
    Shared<T, Mine::kWide, kSelectBatch> B;
    const auto fetch = [&](int k0) {
        x.load(a.x, a.x_stride, ln.row0 + k0, ln.c, a.tokens);
        delta.load(a.delta, a.delta_stride, ln.row0 + k0, ln.c, a.tokens);
        B.load(a.B, a.b_stride, ln.row0 + k0, a, ln.group);
    };
    fetch(from);
    for (int k0 = from; k0 < ln.rows; k0 += kSelectBatch) {
        wave_fence();
        B.put(lds);
        wave_fence();
        const Column<T, kSelectBatch> x1 = x, d1 = delta;
        if (k0 + kSelectBatch < ln.rows) fetch(k0 + kSelectBatch);
        const auto rows = [&](auto some) {
#pragma unroll
            for (int k = 0; k < kSelectBatch; k++) {
                if (some.value && k0 + k >= ln.rows) break;
                const float d = step_of(d1.get(k) + bias), u = d * x1.get(k);
                float b[S];
                take_states(lds + k * Mine::kWide + ln.n0, b);
#pragma unroll
                for (int i = 0; i < S; i++) h[i] = fmaf(exp2_of(d * A2[i]), h[i], u * b[i]);
                span += d;
            }
        };
        if (k0 + kSelectBatch <= ln.rows) rows(std::false_type());
        else rows(std::true_type());
    }
    ln.store_own(a.ends + ln.own(a, ln.strip), h);
    if (ln.active && ln.part == 0) a.spans[ln.strip * a.channels + ln.c] = ln.begin ? kCutSpan : kept_span(span);
}

// Second launch: the state that comes into each strip.  A workgroup has 64 neighbouring states and a wave for each of 16 pieces of the strips: each
// is put together, the pieces before are applied one after the other, and each is gone through again: up to kEach strips of a piece with what
// they do in registers, so that it is asked for once and all at once (kEach 0: any number).  256 strips of 16 384 states: 29 us without, 313 of
// 6 400 15.6, and 12.9 with; with 32 a piece registers are spilled.
constexpr int kStateThreads = 1024;
template <int kEach>
__global__ __launch_bounds__(kStateThreads) void k_select_states(SelectArgs a, int wide, bool back)
{
    constexpr int kPieces = kStateThreads / kWave;
    __shared__ float s_end[kPieces][kWave], s_span[kPieces][kWave];
    const int lane = lane_id(), piece = wave_id();
    const int64_t slots = a.channels * wide, slot = (int64_t)blockIdx.x * kWave + lane, at = slot < slots ? slot : slots - 1;
    const int64_t c = divide(at, wide), n = at - c * wide;
    const float A2 = n < a.states ? a.A[c * a.states + n] * kLog2e : 0.0f;
    const int64_t each = (a.strips + kPieces - 1) / kPieces, from = piece * each, to = from + each < a.strips ? from + each : a.strips;
    float *out = back ? a.back : a.before;
    const auto strip_of = [&](int64_t k) { return back ? a.strips - 1 - k : k; };
    float end[kEach ? kEach : 1], step[kEach ? kEach : 1];
#pragma unroll
    for (int k = 0; k < kEach; k++) {
        const int64_t strip = strip_of(from + k < to ? from + k : 0);
        end[k] = a.ends[strip * slots + at];
        step[k] = a.spans[strip * a.channels + c];
    }
    float h = 0.0f, span = 0.0f;
    bool cut = false;
    const auto every = [&](auto write) {
        const auto one = [&](int64_t k, float e, float d) {
            if (write.value) { if (slot < slots) out[strip_of(k) * slots + slot] = h; }
            h = apply_strip(d, e, A2, h);
            span += d;
            cut = cut || d == kCutSpan;
        };
        if (kEach) {
#pragma unroll
            for (int k = 0; k < kEach; k++) if (from + k < to) one(from + k, end[k], step[k]);
            return;
        }
#pragma unroll 4
        for (int64_t k = from; k < to; k++) one(k, a.ends[strip_of(k) * slots + at], a.spans[strip_of(k) * a.channels + c]);
    };
    every(std::false_type());
    s_end[piece][lane] = h;
    s_span[piece][lane] = cut ? kCutSpan : kept_span(span);
    __syncthreads();
    h = 0.0f;
#pragma unroll 4
    for (int p = 0; p < piece; p++) h = apply_strip(s_span[p][lane], s_end[p][lane], A2, h);
    every(std::true_type());
}
void select_states(const SelectArgs &a, int wide, bool back, hipStream_t s)
{
    const int64_t slots = a.channels * wide;
    const dim3 threads(kStateThreads), few((unsigned)((slots + 63) / 64));
    if (a.strips <= 64) hipLaunchKernelGGL((k_select_states<4>), few, threads, 0, s, a, wide, back);
    else if (a.strips <= 256) hipLaunchKernelGGL((k_select_states<16>), few, threads, 0, s, a, wide, back);
    else if (a.strips <= 384) hipLaunchKernelGGL((k_select_states<24>), few, threads, 0, s, a, wide, back);
    else hipLaunchKernelGGL((k_select_states<0>), few, threads, 0, s, a, wide, back);
}

// Third launch: 143 instructions a row and wave of 64 channels x 16 states, 80 of them the states'.  16 384 x 1 024 x 16 in bf16 95 us, 76 % of the
// cycles in vector instructions, waves for 20 % of their time behind memory or LDS; 32 771 x 2 048 x 16 316 to 338 us.
// (Four states a lane instead of 16 do what belongs to a row and channel four times over, but are four times as many waves: the rule is at
// select_layout.)
template <class T, int S, int L>
__global__ __launch_bounds__(kSelectWaves *kWave) void k_select_outputs(SelectArgs args)
{
    const SelectArgs &a = args;
    typedef Lane<S, L> Mine;
    typedef typename T::Store E;
    __shared__ int32_t s_own[kSelectWaves][kWave];
    __shared__ __attribute__((aligned(16))) float s_bc[kSelectWaves][2][kSelectBatch * Mine::kWide];
    const int64_t number = (int64_t)blockIdx.x * kSelectWaves + wave_id(), strips = (a.strips * a.blocks + kSelectWaves - 1) / kSelectWaves;
    if (blockIdx.x >= strips) {
        if (a.final)
            copy_empties(a.rowptr, a.seqs, a.tokens, a.channels * a.states, a.h0, a.final, number - strips * kSelectWaves, (gridDim.x - strips) * kSelectWaves);
        return;
    }
    float (&lds)[2][kSelectBatch * Mine::kWide] = s_bc[wave_id()];
    Mine ln;
    if (!ln.find(a, number)) return;
    float A2[S], h[S];
    ln.decays(a, A2);
    ln.template before<false>(a, A2, h);
    const float bias = a.delta_bias ? a.delta_bias[ln.c] : 0.0f, D = a.D ? a.D[ln.c] : 0.0f;
    Column<T, kSelectBatch> x, delta, z;
    Shared<T, Mine::kWide, kSelectBatch> B, C;
    const auto fetch = [&](int k0) {
        const SelectArgs a = asked_again();
        x.load(a.x, a.x_stride, ln.row0 + k0, ln.c, a.tokens);
        delta.load(a.delta, a.delta_stride, ln.row0 + k0, ln.c, a.tokens);
        if (a.z) z.load(a.z, a.z_stride, ln.row0 + k0, ln.c, a.tokens);
        B.load(a.B, a.b_stride, ln.row0 + k0, a, ln.group);
        C.load(a.C, a.c_stride, ln.row0 + k0, a, ln.group);
    };
    fetch(0);
    ln.mark(a, s_own[wave_id()]);                               // (with the first rows on their way)
    for (int k0 = 0; k0 < ln.rows; k0 += kSelectBatch) {
        wave_fence();
        B.put(lds[0]);
        C.put(lds[1]);
        wave_fence();
        const Column<T, kSelectBatch> x1 = x, d1 = delta, z1 = z;
        if (k0 + kSelectBatch < ln.rows) fetch(k0 + kSelectBatch);
        const SelectArgs a = asked_again();
        if (a.kept && k0 % kSelectKeep == 0) ln.store_own(a.kept + ln.own(a, (ln.row0 + k0) / kSelectKeep), h);
        const uint32_t valid = ln.valid >> k0 & 0xff, begin = ln.begin >> k0 & 0xff, end = ln.end >> k0 & 0xff;
        E *to = static_cast<E *>(a.y) + (ln.row0 + k0) * a.y_stride + ln.c;
        const auto rows = [&](auto some) {
#pragma unroll
            for (int k = 0; k < kSelectBatch; k++) {
                if (some.value && !(valid >> k & 1)) continue;
                const float d = step_of(d1.get(k) + bias), u = d * x1.get(k);
                if (some.value && (begin >> k & 1)) ln.load(a, a.h0, ln.q(k0 + k), h);
                float b[S], c[S], y = 0.0f;
                take_states(lds[0] + k * Mine::kWide + ln.n0, b);
                take_states(lds[1] + k * Mine::kWide + ln.n0, c);
#pragma unroll
                for (int i = 0; i < S; i++) {
                    h[i] = fmaf(exp2_of(d * A2[i]), h[i], u * b[i]);
                    y = fmaf(c[i], h[i], y);
                }
                y = sum_channel<L>(y);
                if (a.D) y = fmaf(D, x1.get(k), y);
                if (a.z) y *= z1.get(k) * gate_of<T>(z1.get(k));
                if (ln.active && ln.part == 0) to[k * a.y_stride] = (E)y;
                if (some.value && (end >> k & 1) && a.final) ln.store(a, a.final, ln.q(k0 + k), h);
            }
        };
        // (most rows are in the middle of a sequence)
        if (valid == 0xff && (begin | end) == 0) rows(std::false_type());
        else rows(std::true_type());
    }
}

template <class T, int S, int L> static void go_forward(const SelectArgs &a, hipStream_t s)
{
    const int64_t groups = (a.strips * a.blocks + kSelectWaves - 1) / kSelectWaves;
    const int64_t empties = a.final ? copy_groups(a.seqs, a.channels * a.states, kSelectWaves) : 0;
    const dim3 threads(kSelectWaves * kWave);
    if (a.strips > 1) {
        hipLaunchKernelGGL((k_select_ends<T, S, L>), dim3((unsigned)groups), threads, 0, s, a);
        if (a.before) select_states(a, S * L, false, s);
    }
    if (groups + empties > 0) hipLaunchKernelGGL((k_select_outputs<T, S, L>), dim3((unsigned)(groups + empties)), threads, 0, s, a);
}
void select_forward(int dtype, const SelectArgs &a, const SelectLayout &l, hipStream_t s)
{
#define DGN_CALL(S, L) go_forward<Type, S, L>(a, s)
#define DGN_GO(T)                                   \
    do {                                            \
        typedef T Type;                             \
        DGN_BY_LANES(l.S, l.L, DGN_CALL);           \
    } while (0)
    DGN_BY_DTYPE(dtype, DGN_GO);
#undef DGN_GO
#undef DGN_CALL
}

// The value of lane k of each group of K (1, 2 or 4 neighbouring lanes).
template <int K> __device__ __forceinline__ float of_lane(float v, int k)
{
    if (K == 1) return v;
    if (K == 2) return k == 0 ? moved<0xA0>(v) : moved<0xF5>(v);
    return k == 0 ? moved<0x00>(v) : k == 1 ? moved<0x55>(v) : k == 2 ? moved<0xAA>(v) : moved<0xFF>(v);
}
// One token for each row: four states a lane, kBlocks of a row's channel blocks a wave.  Bound by memory: all that is read is asked for before
// anything is made of it, and what belongs to a channel (step, input, outer gate) is made by one lane: lane k of the first kBlocks for block k.
// kFours: a multiple of four states.  States of calls larger than the last-level cache go past it: 1 024 rows of 2 048 x 16, 278 MB, 65 us on a
// pool that is not in that cache (4.3 TB/s; a copy has 6.2; A, 131 KB, is read from L2 for each row, another 134 MB).  On one pool again and
// again, half of it in that cache, 46 to 54 (else 64; with what belongs to a channel made by all its lanes 82, and with a block a wave 88).
template <class T, int L, int kBlocks, bool kFours, bool kStream>
__global__ __launch_bounds__(256) void k_select_step(SelectStepArgs s)
{
    static_assert(kBlocks <= L, "a lane for each block");
    constexpr int S = 4;
    typedef typename T::Store E;
    const SelectArgs &a = s.in;
    const int64_t group_pieces = (a.group_blocks + kBlocks - 1) / kBlocks, pieces = group_pieces * a.groups;
    for (int64_t number = (int64_t)blockIdx.x * 4 + wave_id(); number < a.tokens * pieces; number += (int64_t)gridDim.x * 4) {
        const int64_t row = divide(number, pieces), piece = number - row * pieces, slot = s.slot ? s.slot[row] : row;
        const int64_t group = divide(piece, group_pieces), block0 = group * a.group_blocks + (piece - group * group_pieces) * kBlocks;
        Lane<S, L> ln[kBlocks], own;                    // own: whose channel the lane answers for
        own.place(a, block0 + lane_id() % L % kBlocks, group);
        const bool here = slot >= 0 && slot < s.slots;
        float y = 0.0f;
        if (here) {
            float h[kBlocks][S], A[kBlocks][S], b[S], c[S];
#pragma unroll
            for (int k = 0; k < kBlocks; k++) {
                ln[k].place(a, block0 + k, group);
                ln[k].load(a, s.state_in, slot, h[k]);
            }
            const E delta = static_cast<const E *>(a.delta)[row * a.delta_stride + own.c], xe = static_cast<const E *>(a.x)[row * a.x_stride + own.c],
                    ze = a.z ? static_cast<const E *>(a.z)[row * a.z_stride + own.c] : (E)0.0f;
#pragma unroll
            for (int k = 0; k < kBlocks; k++) ln[k].load(a, a.A, 0, A[k]);
            const float bias = a.delta_bias ? a.delta_bias[own.c] : 0.0f, D = a.D ? a.D[own.c] : 0.0f;
            const E *be = static_cast<const E *>(a.B) + row * a.b_stride + group * a.states + own.n0,
                    *ce = static_cast<const E *>(a.C) + row * a.c_stride + group * a.states + own.n0;
            if (kFours) {
                Pack<T, S> bs = {}, cs = {};
                if (own.count) {
                    bs.load(be);
                    cs.load(ce);
                }
#pragma unroll
                for (int i = 0; i < S; i++) b[i] = bs.get(i), c[i] = cs.get(i);
            } else {
#pragma unroll
                for (int i = 0; i < S; i++) b[i] = i < own.count ? (float)be[i] : 0.0f, c[i] = i < own.count ? (float)ce[i] : 0.0f;
            }
            const float d = step_of((float)delta + bias), x = (float)xe, u = d * x, z = (float)ze;
#pragma unroll
            for (int k = 0; k < kBlocks; k++) {
                const float dk = of_lane<kBlocks>(d, k) * kLog2e, uk = of_lane<kBlocks>(u, k);
                float yk = 0.0f;
#pragma unroll
                for (int i = 0; i < S; i++) {
                    h[k][i] = fmaf(exp2_of(dk * A[k][i]), h[k][i], uk * b[i]);
                    yk = fmaf(c[i], h[k][i], yk);
                }
                ln[k].template store<kStream>(a, s.state_out, slot, h[k]);
                yk = sum_channel<L>(yk);
                if (lane_id() % L % kBlocks == k) y = yk;
            }
            if (a.D) y = fmaf(D, x, y);
            if (a.z) y *= z * gate_of<T>(z);
        }
        if (own.active && own.part < kBlocks) static_cast<E *>(a.y)[row * a.y_stride + own.c] = (E)y;
    }
}

// Lanes: 16 states each where that gives kManyWaves waves of kSelectKeep rows, else four, and from 64 states on, which four a lane spread over
// many lanes, half as many waves (forward, us with 16 and with four: 512 x 512 x 16, 256 waves, 28.1 and 17.0; 1 024 x 512 x 16, 512 waves, 25.4 and
// 23.8; 2 048 x 512 x 16, 1 024 waves, 31.3 and 34.7; 300 x 256 x 128, 608 waves, 27.3 and 34.7; training step of 512 x 2 048 x 16, 1 024 waves, 85 and 78).
// Rows of a strip: as few as give kSelectStrips waves, from kSelectKeep to kSelectMostRows (8 192 waves: the states between strips of 16 384 x 1 024
// x 16 take 29 us instead of 12, its gradients 350 instead of 328).
constexpr int64_t kSelectStrips = 4096, kManyWaves = 1024;
SelectLayout select_layout(const SelectArgs &a)
{
    SelectLayout l;
    l.wide = 4;
    while (l.wide < a.states) l.wide *= 2;
    const int64_t share = a.channels / a.groups;
    const auto blocks = [&](int S) { const int64_t width = kWave / (l.wide / S); return (share + width - 1) / width; };
    const int64_t back = l.wide <= 16 ? 64 : 1024 / l.wide;             // channels of a workgroup of the backward pass
    l.back_group_blocks = (share + back - 1) / back;
    l.back_blocks = l.back_group_blocks * a.groups;
    l.S = l.wide >= 16 && blocks(16) * a.groups * ((a.tokens + kSelectKeep - 1) / kSelectKeep) >= (l.wide < 64 ? kManyWaves : kManyWaves / 2) ? 16 : 4;
    l.L = l.wide / l.S;
    l.group_blocks = blocks(l.S);
    l.blocks = l.group_blocks * a.groups;
    l.rows = a.tokens * l.blocks / kSelectStrips / kSelectKeep * kSelectKeep;
    l.rows = l.rows < kSelectKeep ? kSelectKeep : l.rows > kSelectMostRows ? kSelectMostRows : l.rows;
    l.strips = (a.tokens + l.rows - 1) / l.rows;
    const size_t state = (size_t)a.channels * l.wide * sizeof(float), chunks = (size_t)((a.tokens + kSelectKeep - 1) / kSelectKeep);
    const auto room = [](size_t v) { return (v + 255) / 256 * 256; };
    l.carry = chunks * state;
    l.ends = 0;
    l.before = l.ends + room(l.strips * state);
    l.spans = l.before + room(l.strips * state);
    l.partial = l.spans + room((size_t)l.strips * a.channels * sizeof(float));
    l.copy = l.partial;             // (the one forward, the other backward)
    l.shared = l.partial + room(l.strips * (state + 2 * a.channels * sizeof(float)));
    const int64_t strip_sums = l.back_blocks * l.rows * 2 * l.wide * (int64_t)sizeof(float);
    const int64_t fitting = kSharedBytes / strip_sums, least = (kSharedGroups + l.back_blocks - 1) / l.back_blocks;
    l.slice = fitting > least ? fitting : least;
    const int64_t slice_rows = l.slice * l.rows < a.tokens ? l.slice * l.rows : a.tokens;
    l.forward_bytes = l.copy + (size_t)a.seqs * a.channels * a.states * sizeof(float);
    const size_t sums = l.shared + (size_t)(l.back_blocks * slice_rows) * 2 * l.wide * sizeof(float);
    l.bytes = l.forward_bytes > sums ? l.forward_bytes : sums;
    return l;
}
bool select_fits(int, const SelectArgs &a)          // launches of less than 2^32 threads
{
    const SelectLayout l = select_layout(a);
    const int64_t most = l.blocks > l.back_blocks ? l.blocks : l.back_blocks;
    return l.strips * most < ((int64_t)1 << 24) - kMostCopyGroups && a.channels * l.wide < ((int64_t)1 << 25);
}
size_t select_scratch_bytes(const SelectArgs &a, bool forward_only)
{
    const SelectLayout l = select_layout(a);
    return forward_only ? l.forward_bytes : l.bytes;
}
size_t select_carry_bytes(const SelectArgs &a) { return select_layout(a).carry; }

__global__ __launch_bounds__(256) void k_copy_floats(const float *from, float *to, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) to[i] = from[i];
}

hipError_t launch_select(int dtype, bool back, const SelectArgs &args, void *carry, void *scratch, hipStream_t s)
{
    const SelectLayout l = select_layout(args);
    SelectArgs a = args;
    char *mem = static_cast<char *>(scratch);
    const auto at = [&](size_t v) { return reinterpret_cast<float *>(mem + v); };
    a.strips = l.strips;
    a.blocks = back ? l.back_blocks : l.blocks;
    a.group_blocks = (int32_t)(back ? l.back_group_blocks : l.group_blocks);
    a.rows = (int32_t)l.rows;
    a.ends = at(l.ends);
    a.spans = at(l.spans);
    a.before = a.back = l.strips > (l.S == 4 ? kFewSelectStrips : kFewSelectStrips / 2) ? at(l.before) : nullptr;
    a.kept = static_cast<float *>(carry);
    a.partial = at(l.partial);
    a.shared = at(l.shared);
    if (back) {
        select_backward(dtype, a, l, s);
        return hipGetLastError();
    }
    const int64_t n = a.seqs * a.channels * a.states;
    if (a.h0 && a.final && a.h0 < a.final + n && a.final < a.h0 + n) {      // (strips read and write states in any order)
        const int64_t groups = (n + 255) / 256;
        hipLaunchKernelGGL(k_copy_floats, dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(256), 0, s, a.h0, at(l.copy), n);
        a.h0 = at(l.copy);
    }
    select_forward(dtype, a, l, s);
    return hipGetLastError();
}

// Waves, of one block each, from which on they take several: 64 and 128 rows of 2 048 x 16, 8 192 and 16 384 waves, are as long as the call either
// way; 256 rows take 16.4 us, with a block a wave 21.5.
constexpr int64_t kManySteps = 8192;
hipError_t launch_select_step(int dtype, const SelectStepArgs &args, hipStream_t s)
{
    const SelectLayout l = select_layout(args.in);
    SelectStepArgs a = args;
    const int64_t width = kWave / (l.wide / 4), share = a.in.channels / a.in.groups;
    a.in.group_blocks = (int32_t)((share + width - 1) / width);
    a.in.blocks = a.in.group_blocks * a.in.groups;
    const bool many = a.in.states % 4 == 0 && a.in.tokens * a.in.blocks >= kManySteps;
    const bool stream = many && (size_t)a.in.tokens * a.in.channels * (a.in.states * 2 * sizeof(float) + 3 * element_size(dtype)) > kStreamBytes;
    const int64_t each = !many ? 1 : l.wide < 16 ? l.wide / 4 : 4;
    const int64_t n = (a.in.tokens * ((a.in.group_blocks + each - 1) / each) * a.in.groups + 3) / 4;
    const dim3 grid((unsigned)(n < (1 << 22) ? n : 1 << 22)), threads(256);
#define DGN_STEP(L, N, F, P) hipLaunchKernelGGL((k_select_step<Type, L, N, F, P>), grid, threads, 0, s, a)
#define DGN_CALL(S, L)                                              \
    do {                                                            \
        if (a.in.states % 4 == 0) {                                 \
            if (stream) DGN_STEP(L, (L < 4 ? L : 4), true, true);   \
            else if (many) DGN_STEP(L, (L < 4 ? L : 4), true, false); \
            else DGN_STEP(L, 1, true, false);                       \
        } else DGN_STEP(L, 1, false, false);                        \
    } while (0)
#define DGN_GO(T)                                   \
    do {                                            \
        typedef T Type;                             \
        switch (l.wide / 4) {                       \
        case 1: DGN_CALL(4, 1); break;              \
        case 2: DGN_CALL(4, 2); break;              \
        case 4: DGN_CALL(4, 4); break;              \
        case 8: DGN_CALL(4, 8); break;              \
        case 16: DGN_CALL(4, 16); break;            \
        case 32: DGN_CALL(4, 32); break;            \
        default: DGN_CALL(4, 64);                   \
        }                                           \
    } while (0)
    DGN_BY_DTYPE(dtype, DGN_GO);
#undef DGN_GO
#undef DGN_CALL
#undef DGN_STEP
    return hipGetLastError();
}

}  // namespace dgn
