// Selective scan over ragged sequences, forward, backward and for one token.  For each channel, with N states and
//   d = log(1 + exp(delta + bias)):
//   h_t[n] = exp(d A[n]) h_{t-1}[n] + d x B_t[n],   y = (sum_n C_t[n] h_t[n] + D x) z sigma(z)
// and, with o = dy z sigma(z) and e_t the gradient of h_t (what reaches y_t and what comes back from h_{t+1}),
//   e_t[n] = o C_t[n] + a_{t+1}[n] e_{t+1}[n],   dh0 = a_0 e_0,   a = exp(d A)
//   dC = sum_c o h,   dB = sum_c e d x,   dx = D o + d sum_n e B,   dA = sum_t e d a h_{t-1},   dD = sum_t o x
//   dd = sum_n e (A a h_{t-1} + B x),   ddelta = dd sigma(delta + bias),   dz = dy y sigma(z) (1 + z (1 - sigma(z)))
//
// A lane has kStates states of a channel, 2^k neighbouring lanes a channel.  The rows, whatever sequences they belong to, are cut into strips;
// what a strip does to the state that comes into it is h -> exp(A sum d) h + E (E its end from a state of zero), or h -> E if a sequence
// begins in it: three launches, the strips' (sum d, E), the states between strips, the strips again.
#include "layer.h"
#include "rows.h"

namespace dgn {

constexpr int kStates = 4;              // of a lane
constexpr int kSelectRows = 16;         // of a strip
constexpr int kSelectWaves = 4;
constexpr float kLog2e = 1.44269504088896340736f;

// log(1 + exp(v)) = max(v, 0) + 2 artanh(s), s = q / (2 + q), q = exp(-|v|), by the series s + s^3 / 3 + ... (s <= 1/3: what is left out
// is below 2^-26); and its derivative.
struct Step { float d, slope; };
__device__ __forceinline__ Step step_of(float v)
{
    const float q = expf(-fabsf(v)), s = q / (2.0f + q), r = s * s;
    float p = fmaf(r, 1.0f / 15.0f, 1.0f / 13.0f);
    p = fmaf(r, p, 1.0f / 11.0f);
    p = fmaf(r, p, 1.0f / 9.0f);
    p = fmaf(r, p, 1.0f / 7.0f);
    p = fmaf(r, p, 1.0f / 5.0f);
    p = fmaf(r, p, 1.0f / 3.0f);
    const float l = 2.0f * fmaf(s * r, p, s);
    const float k = 1.0f / (1.0f + q);
    return Step{v > 0.0f ? v + l : l, v > 0.0f ? k : q * k};      // (NaN: l and q are NaN)
}
__device__ __forceinline__ float gate_of(float z) { return 1.0f / (1.0f + expf(-z)); }

// The strip of a wave, the channel and the states of a lane.
template <int L> struct Lane {
    int64_t row0, c, group, slot;       // slot: the lane's place in arrays of [strips][blocks][64]
    int64_t block;
    int32_t rows, n0, part, count;      // first state, place among the channel's lanes, states that there are
    bool active;                        // lanes past the group's end do what its last channel's do, and write nothing
    u64 valid, begin, end;
    RowSeq seq;

    __device__ __forceinline__ bool find(const SelectArgs &a, int64_t number)
    {
        if (number >= a.strips * a.blocks) return false;
        const int64_t strip = divide(number, a.blocks);
        place(a, number - strip * a.blocks);
        row0 = strip * a.rows;
        const int64_t left = a.tokens - row0;
        rows = (int32_t)(left < a.rows ? left : a.rows);
        slot = number * kWave + lane_id();
        return true;
    }
    __device__ __forceinline__ void place(const SelectArgs &a, int64_t block_)
    {
        constexpr int kWidth = kWave / L;
        block = block_;
        group = divide(block, a.group_blocks);
        const int64_t share = a.channels / a.groups, at = (block - group * a.group_blocks) * kWidth + lane_id() / L;
        active = at < share;
        c = group * share + (active ? at : share - 1);
        part = lane_id() % L;
        n0 = part * kStates;
        const int64_t some = a.states - n0;
        count = some < 0 ? 0 : some > kStates ? kStates : (int32_t)some;
    }
    __device__ __forceinline__ void mark(const SelectArgs &a, int32_t *own)
    {
        seq = sequences_of(a.rowptr, a.seqs, a.tokens, row0, own);
        const int64_t row = row0 + lane_id();
        const bool mine = seq.q >= 0 && lane_id() < rows;
        valid = __ballot(mine);
        begin = __ballot(mine && seq.first == row);
        end = __ballot(mine && seq.end == row + 1);
    }
    __device__ __forceinline__ int64_t q(int k) const { return __builtin_amdgcn_readlane(seq.q, k); }
    // States of the lane in arrays of [..][channels][states]; those that there are not are 0.
    __device__ __forceinline__ void load(const SelectArgs &a, const float *p, int64_t row, float (&h)[kStates]) const
    {
        const float *at = p + (row * a.channels + c) * a.states + n0;
#pragma unroll
        for (int i = 0; i < kStates; i++) h[i] = p && i < count ? at[i] : 0.0f;
    }
    __device__ __forceinline__ void store(const SelectArgs &a, float *p, int64_t row, const float (&h)[kStates]) const
    {
        float *at = p + (row * a.channels + c) * a.states + n0;
#pragma unroll
        for (int i = 0; i < kStates; i++) if (active && i < count) at[i] = h[i];
    }
    template <class T> __device__ __forceinline__ void wide(const void *p, int64_t stride, int64_t row, const SelectArgs &a, float (&v)[kStates]) const
    {
        const typename T::Store *at = static_cast<const typename T::Store *>(p) + row * stride + group * a.states + n0;
#pragma unroll
        for (int i = 0; i < kStates; i++) v[i] = i < count ? (float)at[i] : 0.0f;
    }
    template <class T> __device__ __forceinline__ float one(const void *p, int64_t stride, int64_t row) const
    {
        return (float)static_cast<const typename T::Store *>(p)[row * stride + c];
    }
    template <class T> __device__ __forceinline__ void put_one(void *p, int64_t stride, int64_t row, float v) const
    {
        if (active && part == 0) static_cast<typename T::Store *>(p)[row * stride + c] = (typename T::Store)v;
    }
};
template <int L> __device__ __forceinline__ float sum_channel(float v)
{
#pragma unroll
    for (int d = 1; d < L; d <<= 1) v += __shfl_xor(v, d, kWave);
    return v;
}
template <int L> __device__ __forceinline__ float sum_channels(float v)        // over the lanes of the same states
{
#pragma unroll
    for (int d = L; d < kWave; d <<= 1) v += __shfl_xor(v, d, kWave);
    return v;
}
__device__ __forceinline__ void scaled(const float (&A)[kStates], float (&A2)[kStates])
{
#pragma unroll
    for (int i = 0; i < kStates; i++) A2[i] = A[i] * kLog2e;
}

// First launch: what a strip does to a state.  kBack: to a gradient, from its last row to its first.
template <class T, int L, bool kBack>
__global__ __launch_bounds__(kSelectWaves *kWave) void k_select_ends(SelectArgs a)
{
    __shared__ int32_t s_own[kSelectWaves][kWave];
    Lane<L> ln;
    if (!ln.find(a, (int64_t)blockIdx.x * kSelectWaves + wave_id())) return;
    ln.mark(a, s_own[wave_id()]);
    float A[kStates], A2[kStates], h[kStates], span = 0.0f;
    ln.load(a, a.A, 0, A);
    scaled(A, A2);
#pragma unroll
    for (int i = 0; i < kStates; i++) h[i] = 0.0f;
    const float bias = a.delta_bias ? a.delta_bias[ln.c] : 0.0f;
    for (int t = 0; t < ln.rows; t++) {
        const int k = kBack ? ln.rows - 1 - t : t;
        if (!(ln.valid >> k & 1)) continue;
        const int64_t row = ln.row0 + k;
        const Step st = step_of(ln.template one<T>(a.delta, a.delta_stride, row) + bias);
        float v[kStates];
        if (kBack) {
            float o = ln.template one<T>(a.dy, a.dy_stride, row);
            if (a.z) {
                const float z = ln.template one<T>(a.z, a.z_stride, row);
                o *= z * gate_of(z);
            }
            ln.template wide<T>(a.C, a.c_stride, row, a, v);
            if (ln.end >> k & 1) ln.load(a, a.dfinal, ln.q(k), h);
#pragma unroll
            for (int i = 0; i < kStates; i++) h[i] = exp2f(st.d * A2[i]) * fmaf(o, v[i], h[i]);
        } else {
            const float u = st.d * ln.template one<T>(a.x, a.x_stride, row);
            ln.template wide<T>(a.B, a.b_stride, row, a, v);
            if (ln.begin >> k & 1) ln.load(a, a.h0, ln.q(k), h);
#pragma unroll
            for (int i = 0; i < kStates; i++) h[i] = fmaf(exp2f(st.d * A2[i]), h[i], u * v[i]);
        }
        span += st.d;
    }
#pragma unroll
    for (int i = 0; i < kStates; i++) a.ends[ln.slot * kStates + i] = h[i];
    a.spans[ln.slot] = span;
    if (ln.block == 0 && lane_id() == 0) a.cuts[ln.row0 / a.rows] = (kBack ? ln.end : ln.begin) != 0;
}

// Second launch: the state that comes into each strip.
template <int L, bool kBack>
__global__ __launch_bounds__(kWave) void k_select_states(SelectArgs a)
{
    Lane<L> ln;
    ln.place(a, blockIdx.x);
    float A[kStates], A2[kStates], h[kStates];
    ln.load(a, a.A, 0, A);
    scaled(A, A2);
#pragma unroll
    for (int i = 0; i < kStates; i++) h[i] = 0.0f;
    float *to = kBack ? a.back : a.before;
    for (int64_t t = 0; t < a.strips; t++) {
        const int64_t strip = kBack ? a.strips - 1 - t : t, at = (strip * a.blocks + blockIdx.x) * kWave + lane_id();
        const bool cut = a.cuts[strip];
        const float span = a.spans[at];
#pragma unroll
        for (int i = 0; i < kStates; i++) {
            to[at * kStates + i] = h[i];
            const float end = a.ends[at * kStates + i];
            h[i] = cut ? end : fmaf(exp2f(span * A2[i]), h[i], end);
        }
    }
}

// Sequences without rows: out = in (or zero).
__device__ __forceinline__ void copy_empty_states(const SelectArgs &a, const float *in, float *out, int64_t wave, int64_t waves)
{
    const int64_t width = a.channels * a.states;
    for (int64_t q0 = wave * kWave; q0 < a.seqs; q0 += waves * kWave) {
        const int64_t q = q0 + lane_id();
        const bool empty = q < a.seqs && row_bound(a.rowptr[q], a.tokens) >= row_bound(a.rowptr[q + 1], a.tokens);
        for (u64 some = __ballot(empty); some; some &= some - 1) {
            const int64_t at = (q0 + __builtin_ctzll(some)) * width;
            for (int64_t i = lane_id(); i < width; i += kWave) out[at + i] = in ? in[at + i] : 0.0f;
        }
    }
}

// Third launch, forward.
template <class T, int L>
__global__ __launch_bounds__(kSelectWaves *kWave) void k_select_outputs(SelectArgs a)
{
    __shared__ int32_t s_own[kSelectWaves][kWave];
    const int64_t number = (int64_t)blockIdx.x * kSelectWaves + wave_id(), strips = (a.strips * a.blocks + kSelectWaves - 1) / kSelectWaves;
    if (blockIdx.x >= strips) {
        if (a.final) copy_empty_states(a, a.h0, a.final, number - strips * kSelectWaves, (gridDim.x - strips) * kSelectWaves);
        return;
    }
    Lane<L> ln;
    if (!ln.find(a, number)) return;
    ln.mark(a, s_own[wave_id()]);
    float A[kStates], A2[kStates], h[kStates];
    ln.load(a, a.A, 0, A);
    scaled(A, A2);
#pragma unroll
    for (int i = 0; i < kStates; i++) h[i] = a.before[ln.slot * kStates + i];
    const float bias = a.delta_bias ? a.delta_bias[ln.c] : 0.0f, D = a.D ? a.D[ln.c] : 0.0f;
    for (int k = 0; k < ln.rows; k++) {
        if (!(ln.valid >> k & 1)) continue;
        const int64_t row = ln.row0 + k;
        const Step st = step_of(ln.template one<T>(a.delta, a.delta_stride, row) + bias);
        const float x = ln.template one<T>(a.x, a.x_stride, row), u = st.d * x;
        float B[kStates], C[kStates], y = 0.0f;
        ln.template wide<T>(a.B, a.b_stride, row, a, B);
        ln.template wide<T>(a.C, a.c_stride, row, a, C);
        if (ln.begin >> k & 1) ln.load(a, a.h0, ln.q(k), h);
#pragma unroll
        for (int i = 0; i < kStates; i++) {
            h[i] = fmaf(exp2f(st.d * A2[i]), h[i], u * B[i]);
            y = fmaf(C[i], h[i], y);
        }
        y = sum_channel<L>(y);
        if (a.D) y = fmaf(D, x, y);
        if (a.z) {
            const float z = ln.template one<T>(a.z, a.z_stride, row);
            y *= z * gate_of(z);
        }
        ln.template put_one<T>(a.y, a.y_stride, row, y);
        if ((ln.end >> k & 1) && a.final) ln.store(a, a.final, ln.q(k), h);
    }
}

// Third launch, backward: a strip's states again from the one that comes into it, then the gradients from the one that comes back into it.
// Sums over rows: partial [strips][blocks][64][kStates + 2], over a block's channels: shared [group_blocks][tokens][groups][2 L kStates].
template <class T, int L>
__global__ __launch_bounds__(kSelectWaves *kWave) void k_select_gradients(SelectArgs a)
{
    __shared__ int32_t s_own[kSelectWaves][kWave];
    const int64_t number = (int64_t)blockIdx.x * kSelectWaves + wave_id(), strips = (a.strips * a.blocks + kSelectWaves - 1) / kSelectWaves;
    if (blockIdx.x >= strips) {
        if (a.dh0) copy_empty_states(a, a.dfinal, a.dh0, number - strips * kSelectWaves, (gridDim.x - strips) * kSelectWaves);
        return;
    }
    Lane<L> ln;
    if (!ln.find(a, number)) return;
    ln.mark(a, s_own[wave_id()]);
    float A[kStates], A2[kStates], h[kStates], e[kStates], dA[kStates], dD = 0.0f, dbias = 0.0f;
    ln.load(a, a.A, 0, A);
    scaled(A, A2);
#pragma unroll
    for (int i = 0; i < kStates; i++) {
        h[i] = a.before[ln.slot * kStates + i];
        e[i] = a.back[ln.slot * kStates + i];
        dA[i] = 0.0f;
    }
    const float bias = a.delta_bias ? a.delta_bias[ln.c] : 0.0f, D = a.D ? a.D[ln.c] : 0.0f;
    float before[kSelectRows][kStates];
#pragma unroll
    for (int k = 0; k < kSelectRows; k++) {
        if (!(ln.valid >> k & 1)) continue;
        const int64_t row = ln.row0 + k;
        const Step st = step_of(ln.template one<T>(a.delta, a.delta_stride, row) + bias);
        const float u = st.d * ln.template one<T>(a.x, a.x_stride, row);
        float B[kStates];
        ln.template wide<T>(a.B, a.b_stride, row, a, B);
        if (ln.begin >> k & 1) ln.load(a, a.h0, ln.q(k), h);
#pragma unroll
        for (int i = 0; i < kStates; i++) {
            before[k][i] = h[i];
            h[i] = fmaf(exp2f(st.d * A2[i]), h[i], u * B[i]);
        }
    }
    const int64_t wide = (int64_t)L * kStates;
#pragma unroll
    for (int k = kSelectRows - 1; k >= 0; k--) {
        if (!(ln.valid >> k & 1)) continue;
        const int64_t row = ln.row0 + k;
        const Step st = step_of(ln.template one<T>(a.delta, a.delta_stride, row) + bias);
        const float x = ln.template one<T>(a.x, a.x_stride, row), u = st.d * x, dy = ln.template one<T>(a.dy, a.dy_stride, row);
        float B[kStates], C[kStates];
        ln.template wide<T>(a.B, a.b_stride, row, a, B);
        ln.template wide<T>(a.C, a.c_stride, row, a, C);
        float z = 0.0f, s = 0.0f, o = dy;
        if (a.z) {
            z = ln.template one<T>(a.z, a.z_stride, row);
            s = gate_of(z);
            o = dy * z * s;
        }
        if (ln.end >> k & 1) ln.load(a, a.dfinal, ln.q(k), e);
        float y = 0.0f, eb = 0.0f, ea = 0.0f, dB[kStates], dC[kStates];
#pragma unroll
        for (int i = 0; i < kStates; i++) {
            const float g = exp2f(st.d * A2[i]), ah = g * before[k][i], now = fmaf(u, B[i], ah);
            e[i] = fmaf(o, C[i], e[i]);
            y = fmaf(C[i], now, y);
            dC[i] = o * now;
            dB[i] = e[i] * u;
            eb = fmaf(e[i], B[i], eb);
            const float w = e[i] * ah;
            ea = fmaf(A[i], w, ea);
            dA[i] = fmaf(st.d, w, dA[i]);
            e[i] *= g;
        }
        y = sum_channel<L>(y);
        eb = sum_channel<L>(eb);
        ea = sum_channel<L>(ea);
        if (a.D) y = fmaf(D, x, y);
        const float dx = a.D ? fmaf(D, o, st.d * eb) : st.d * eb, dd = fmaf(eb, x, ea) * st.slope;
        dD = fmaf(o, x, dD);
        dbias += dd;
        ln.template put_one<T>(a.dx, a.dx_stride, row, dx);
        ln.template put_one<T>(a.ddelta, a.ddelta_stride, row, dd);
        if (a.z) ln.template put_one<T>(a.dz, a.dz_stride, row, dy * y * s * fmaf(z, 1.0f - s, 1.0f));
        if ((ln.begin >> k & 1) && a.dh0) ln.store(a, a.dh0, ln.q(k), e);
        float *shared = a.shared + (((ln.block - ln.group * a.group_blocks) * a.tokens + row) * a.groups + ln.group) * (2 * wide) + ln.n0;
#pragma unroll
        for (int i = 0; i < kStates; i++) {
            const float b = sum_channels<L>(ln.active ? dB[i] : 0.0f), c = sum_channels<L>(ln.active ? dC[i] : 0.0f);
            if (lane_id() < L) {
                shared[i] = b;
                shared[wide + i] = c;
            }
        }
    }
    float *partial = a.partial + ln.slot * (kStates + 2);
#pragma unroll
    for (int i = 0; i < kStates; i++) partial[i] = dA[i];
    partial[kStates] = dD;
    partial[kStates + 1] = dbias;
}

// Sums over rows, in 64 bits: a wave has a channel block's lanes.
template <int L>
__global__ __launch_bounds__(kWave) void k_select_sums(SelectArgs a)
{
    Lane<L> ln;
    ln.place(a, blockIdx.x);
    double sum[kStates + 2] = {};
    for (int64_t strip = 0; strip < a.strips; strip++) {
        const float *p = a.partial + ((strip * a.blocks + blockIdx.x) * kWave + lane_id()) * (kStates + 2);
#pragma unroll
        for (int i = 0; i < kStates + 2; i++) sum[i] += (double)p[i];
    }
    float dA[kStates];
#pragma unroll
    for (int i = 0; i < kStates; i++) dA[i] = (float)sum[i];
    ln.store(a, a.dA, 0, dA);
    if (ln.part || !ln.active) return;
    if (a.dD) a.dD[ln.c] = (float)sum[kStates];
    if (a.ddelta_bias) a.ddelta_bias[ln.c] = (float)sum[kStates + 1];
}

// Sums over the blocks of a group's channels.
template <class T>
__global__ __launch_bounds__(256) void k_select_shared(SelectArgs a, int32_t wide)
{
    typedef typename T::Store S;
    const int64_t low = row_bound(a.rowptr[0], a.tokens), high = row_bound(a.rowptr[a.seqs], a.tokens), width = a.groups * a.states;
    for (int64_t i = low * width + (int64_t)blockIdx.x * 256 + threadIdx.x; i < high * width; i += (int64_t)gridDim.x * 256) {
        const int64_t row = divide(i, width), at = i - row * width, group = divide(at, a.states), n = at - group * a.states;
        float b = 0.0f, c = 0.0f;
        for (int64_t p = 0; p < a.group_blocks; p++) {
            const float *from = a.shared + ((p * a.tokens + row) * a.groups + group) * (2 * wide) + n;
            b += from[0];
            c += from[wide];
        }
        static_cast<S *>(a.dB)[row * a.db_stride + at] = (S)b;
        static_cast<S *>(a.dC)[row * a.dc_stride + at] = (S)c;
    }
}

__global__ __launch_bounds__(256) void k_copy_floats(const float *from, float *to, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) to[i] = from[i];
}

// One token for each row: lanes as above, of a row's channel block.
template <class T, int L>
__global__ __launch_bounds__(256) void k_select_step(SelectStepArgs s)
{
    const SelectArgs &a = s.in;
    for (int64_t number = (int64_t)blockIdx.x * 4 + wave_id(); number < a.tokens * a.blocks; number += (int64_t)gridDim.x * 4) {
        const int64_t row = divide(number, a.blocks), slot = s.slot ? s.slot[row] : row;
        Lane<L> ln;
        ln.place(a, number - row * a.blocks);
        float y = 0.0f;
        if (slot >= 0 && slot < s.slots) {
            float A[kStates], A2[kStates], h[kStates], B[kStates], C[kStates];
            ln.load(a, s.state_in, slot, h);
            ln.load(a, a.A, 0, A);
            scaled(A, A2);
            const Step st = step_of(ln.template one<T>(a.delta, a.delta_stride, row) + (a.delta_bias ? a.delta_bias[ln.c] : 0.0f));
            const float x = ln.template one<T>(a.x, a.x_stride, row), u = st.d * x;
            ln.template wide<T>(a.B, a.b_stride, row, a, B);
            ln.template wide<T>(a.C, a.c_stride, row, a, C);
#pragma unroll
            for (int i = 0; i < kStates; i++) {
                h[i] = fmaf(exp2f(st.d * A2[i]), h[i], u * B[i]);
                y = fmaf(C[i], h[i], y);
            }
            ln.store(a, s.state_out, slot, h);
            y = sum_channel<L>(y);
            if (a.D) y = fmaf(a.D[ln.c], x, y);
            if (a.z) {
                const float z = ln.template one<T>(a.z, a.z_stride, row);
                y *= z * gate_of(z);
            }
        }
        ln.template put_one<T>(a.y, a.y_stride, row, y);
    }
}

static int lanes_of(int64_t states)
{
    int L = 1;
    while (L * kStates < states) L *= 2;
    return L;
}
struct SelectLayout { int L; int64_t group_blocks, blocks, strips; size_t spans, cuts, ends, before, back, partial, shared, copy, bytes; };
static SelectLayout select_layout(const SelectArgs &a)
{
    SelectLayout l;
    l.L = lanes_of(a.states);
    const int64_t width = kWave / l.L, share = a.channels / a.groups;
    l.group_blocks = (share + width - 1) / width;
    l.blocks = l.group_blocks * a.groups;
    l.strips = (a.tokens + kSelectRows - 1) / kSelectRows;
    const size_t slots = (size_t)l.strips * l.blocks * kWave, states = slots * kStates * sizeof(float);
    l.ends = 0;
    l.before = l.ends + states;
    l.back = l.before;                  // (the forward pass keeps its own in carry, or here)
    l.spans = l.before + states;
    l.cuts = l.spans + slots * sizeof(float);
    l.partial = l.cuts + ((size_t)l.strips * sizeof(int32_t) + 255) / 256 * 256;
    l.shared = l.partial + slots * (kStates + 2) * sizeof(float);
    l.copy = l.partial;                 // (forward only)
    const size_t copied = (size_t)a.seqs * a.channels * a.states * sizeof(float),
                 sums = slots * (kStates + 2) * sizeof(float) + (size_t)l.group_blocks * a.tokens * a.groups * 2 * l.L * kStates * sizeof(float);
    l.bytes = l.partial + (copied > sums ? copied : sums);
    return l;
}
bool select_fits(int, const SelectArgs &a)
{
    const SelectLayout l = select_layout(a);
    return l.strips * l.blocks < ((int64_t)1 << 25) && l.blocks < ((int64_t)1 << 25);
}
size_t select_scratch_bytes(int, const SelectArgs &a) { return select_layout(a).bytes; }
size_t select_carry_bytes(int, const SelectArgs &a)
{
    const SelectLayout l = select_layout(a);
    return (size_t)l.strips * l.blocks * kWave * kStates * sizeof(float);
}

template <class T, int L> static void go_select(bool back, const SelectArgs &a, hipStream_t s)
{
    const int64_t groups = (a.strips * a.blocks + kSelectWaves - 1) / kSelectWaves, empties = (a.seqs + 255) / 256;
    const dim3 grid((unsigned)groups), more((unsigned)(groups + (empties < 256 ? empties : 256))), threads(kSelectWaves * kWave);
    const dim3 blocks((unsigned)a.blocks), wave(kWave);
    if (!back) {
        if (a.strips > 0) {
            hipLaunchKernelGGL((k_select_ends<T, L, false>), grid, threads, 0, s, a);
            hipLaunchKernelGGL((k_select_states<L, false>), blocks, wave, 0, s, a);
        }
        hipLaunchKernelGGL((k_select_outputs<T, L>), more, threads, 0, s, a);
        return;
    }
    if (a.strips > 0) {
        hipLaunchKernelGGL((k_select_ends<T, L, true>), grid, threads, 0, s, a);
        hipLaunchKernelGGL((k_select_states<L, true>), blocks, wave, 0, s, a);
    }
    hipLaunchKernelGGL((k_select_gradients<T, L>), more, threads, 0, s, a);
    hipLaunchKernelGGL((k_select_sums<L>), blocks, wave, 0, s, a);
    if (a.strips > 0) {
        const int64_t n = (a.tokens * a.groups * a.states + 255) / 256;
        hipLaunchKernelGGL((k_select_shared<T>), dim3((unsigned)(n < 8192 ? n : 8192)), dim3(256), 0, s, a, L * kStates);
    }
}
#define DGN_BY_LANES(L, call)       \
    do {                            \
        switch (L) {                \
        case 1: call(1); break;     \
        case 2: call(2); break;     \
        case 4: call(4); break;     \
        case 8: call(8); break;     \
        case 16: call(16); break;   \
        case 32: call(32); break;   \
        default: call(64);          \
        }                           \
    } while (0)

hipError_t launch_select(int dtype, bool back, const SelectArgs &args, void *carry, void *scratch, hipStream_t s)
{
    const SelectLayout l = select_layout(args);
    SelectArgs a = args;
    char *mem = static_cast<char *>(scratch);
    const auto at = [&](size_t v) { return reinterpret_cast<float *>(mem + v); };
    a.strips = l.strips;
    a.blocks = l.blocks;
    a.group_blocks = (int32_t)l.group_blocks;
    a.rows = kSelectRows;
    a.ends = at(l.ends);
    a.spans = at(l.spans);
    a.cuts = reinterpret_cast<int32_t *>(mem + l.cuts);
    a.before = carry ? static_cast<float *>(carry) : at(l.before);
    a.back = at(l.back);
    a.partial = at(l.partial);
    a.shared = at(l.shared);
    const int64_t n = a.seqs * a.channels * a.states;
    if (!back && a.h0 && a.final && a.h0 < a.final + n && a.final < a.h0 + n) {
        const int64_t groups = (n + 255) / 256;
        hipLaunchKernelGGL(k_copy_floats, dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(256), 0, s, a.h0, at(l.copy), n);
        a.h0 = at(l.copy);
    }
#define DGN_GO(T)                                   \
    do {                                            \
        const auto call = [&](auto lanes) { go_select<T, decltype(lanes)::value>(back, a, s); }; \
        DGN_BY_LANES(l.L, DGN_CALL);                \
    } while (0)
#define DGN_CALL(n) call(std::integral_constant<int, n>())
    DGN_BY_DTYPE(dtype, DGN_GO);
#undef DGN_GO
    return hipGetLastError();
}

hipError_t launch_select_step(int dtype, const SelectStepArgs &args, hipStream_t s)
{
    const SelectLayout l = select_layout(args.in);
    SelectStepArgs a = args;
    a.in.blocks = l.blocks;
    a.in.group_blocks = (int32_t)l.group_blocks;
    const int64_t n = (a.in.tokens * l.blocks + 3) / 4;
    const dim3 grid((unsigned)(n < (1 << 22) ? n : 1 << 22)), threads(256);
#define DGN_GO(T)                                   \
    do {                                            \
        const auto call = [&](auto lanes) { hipLaunchKernelGGL((k_select_step<T, decltype(lanes)::value>), grid, threads, 0, s, a); }; \
        DGN_BY_LANES(l.L, DGN_CALL);                \
    } while (0)
    DGN_BY_DTYPE(dtype, DGN_GO);
#undef DGN_GO
#undef DGN_CALL
    return hipGetLastError();
}

}  // namespace dgn
