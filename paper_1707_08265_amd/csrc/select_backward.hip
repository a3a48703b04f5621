// Selective scan over ragged sequences: the backward pass (see select.h).  With o = dy z sigma(z) and e_t the gradient of h_t (what reaches y_t
// and what comes back from h_{t+1}),
//   e_t[n] = o C_t[n] + a_{t+1}[n] e_{t+1}[n],   dh0 = a_0 e_0
//   dC = sum_c o h,   dB = sum_c e d x,   dx = D o + d sum_n e B,   dA = sum_t e d a h_{t-1},   dD = sum_t o x
//   dd = sum_n e (A a h_{t-1} + B x),   ddelta = dd sigma(delta + bias),   dz = dy y sigma(z) (1 + z (1 - sigma(z)))
// What comes back over strips is put together as the states are: a e -> exp(A sum d) (a e) + F, or F where a sequence ends.
#include "select.h"

namespace dgn {

// First launch (110 instructions a row and wave of 64 channels x 16 states, 73 % of its cycles): what a strip does to what comes back into it, from its last row to its first; only the rows up to the first end have a part
// in it, and none where the strip's first row begins a sequence.
template <class T, int S, int L>
__global__ __launch_bounds__(kSelectWaves *kWave) void k_select_back_ends(SelectArgs a)
{
    typedef Lane<S, L> Mine;
    __shared__ int32_t s_own[kSelectWaves][kWave];
    __shared__ __attribute__((aligned(16))) float s_c[kSelectWaves][kSelectBatch * Mine::kWide];
    float *lds = s_c[wave_id()];
    Mine ln;
    if (!ln.find(a, (int64_t)blockIdx.x * kSelectWaves + wave_id())) return;
    ln.mark(a, s_own[wave_id()]);
    if (!(ln.valid & ~ln.begin & 1)) {
        const float none[S] = {};
        ln.store_own(a.ends + ln.own(a, ln.strip), none);
        if (ln.active && ln.part == 0) a.spans[ln.strip * a.channels + ln.c] = kCutSpan;
        return;
    }
    const int to = ln.end ? __builtin_ctzll(ln.end) + 1 : ln.rows;      // rows 0 .. to - 1 are of one sequence
    float A2[S], h[S], span = 0.0f;
    ln.decays(a, A2);
#pragma unroll
    for (int i = 0; i < S; i++) h[i] = 0.0f;
    if (ln.end) ln.load(a, a.dfinal, ln.q(to - 1), h);
    const float bias = a.delta_bias ? a.delta_bias[ln.c] : 0.0f;
    Column<T, kSelectBatch> dy, delta, z;
    Shared<T, Mine::kWide, kSelectBatch> C;
    const auto fetch = [&](int k0) {
        dy.load(a.dy, a.dy_stride, ln.row0 + k0, ln.c, a.tokens);
        delta.load(a.delta, a.delta_stride, ln.row0 + k0, ln.c, a.tokens);
        if (a.z) z.load(a.z, a.z_stride, ln.row0 + k0, ln.c, a.tokens);
        C.load(a.C, a.c_stride, ln.row0 + k0, a, ln.group);
    };
    const int last = (to - 1) / kSelectBatch * kSelectBatch;
    fetch(last);
    for (int k0 = last; k0 >= 0; k0 -= kSelectBatch) {
        wave_fence();
        C.put(lds);
        wave_fence();
        const Column<T, kSelectBatch> y1 = dy, d1 = delta, z1 = z;
        if (k0 > 0) fetch(k0 - kSelectBatch);
        const auto rows = [&](auto some) {
#pragma unroll
            for (int k = kSelectBatch - 1; k >= 0; k--) {
                if (some.value && k0 + k >= to) continue;
                const float d = step_of(d1.get(k) + bias);
                float o = y1.get(k), c[S];
                if (a.z) o *= z1.get(k) * gate_of<T>(z1.get(k));
                take_states(lds + k * Mine::kWide + ln.n0, c);
#pragma unroll
                for (int i = 0; i < S; i++) h[i] = exp2_of(d * A2[i]) * fmaf(o, c[i], h[i]);
                span += d;
            }
        };
        if (k0 + kSelectBatch <= to) rows(std::false_type());
        else rows(std::true_type());
    }
    ln.store_own(a.ends + ln.own(a, ln.strip), h);
    if (ln.active && ln.part == 0) a.spans[ln.strip * a.channels + ln.c] = ln.end ? kCutSpan : kept_span(span);
}

// Sums of N values a lane over the lanes that are a multiple of L apart.  Lanes 32, then 16 apart share out what is left (an exchange of halves
// between two registers and an addition for two values): returned are N / kShare of them, by the lane's place (see shared_row).
template <int kDistance> __device__ __forceinline__ void exchange(float &a, float &b)
{
    typedef uint32_t Two __attribute__((ext_vector_type(2)));
    Two r;
    if (kDistance == 32) r = __builtin_bit_cast(Two, __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false));
    else r = __builtin_bit_cast(Two, __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false));
    a = __uint_as_float(r[0]);
    b = __uint_as_float(r[1]);
}
// v: [4 rows][8].  Afterwards rows 0 (and 1, without an exchange at 16; and 2, 3, without any) hold the sums; row r of a lane is row
// r + (lane / 32) * 2 + (lane / 16 % 2) of the four, as far as halves have been exchanged.
template <int L> __device__ __forceinline__ void sum_rows(float (&v)[4][8])
{
    if (L <= 32) {
#pragma unroll
        for (int r = 0; r < 2; r++)
#pragma unroll
            for (int i = 0; i < 8; i++) {
                exchange<32>(v[r][i], v[r + 2][i]);
                v[r][i] += v[r + 2][i];
            }
    }
    if (L <= 16) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            exchange<16>(v[0][i], v[1][i]);
            v[0][i] += v[1][i];
        }
    }
    if (L <= 8) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            v[0][i] += moved<0x128>(v[0][i]);                   // lanes turned by 8 in a row of 16
            if (L <= 4) v[0][i] += moved<0x124>(v[0][i]);       // by 4
            if (L <= 2) v[0][i] += moved<0x4E>(v[0][i]);
            if (L <= 1) v[0][i] += moved<0xB1>(v[0][i]);
        }
    }
}

// Third launch: a strip, kSelectKeep rows at a time, the last first: their states again from the one that is kept, with their decays, in
// registers, then the gradients.  A workgroup has up to 64 channels; what belongs to a row and channel (step, input, gradient of the output) is
// made once, by one thread, and handed on in LDS, and the sums over a channel's states come back the same way.
// Bound by vector instructions: 119 a row and wave of 16 channels x 16 states, 77 % of the cycles with the exponentials' second slots, waves for
// 24 % of their time behind memory, LDS or the others of their workgroup (16 384 x 1 024 x 16 in bf16: 312 us).  The next rows are asked for while the ones after them are worked on (402 us without), and the same 16 rows with branches for
// what begins and ends in them only where something does (497 without).
// partial: [strips][channels][kWide], then [strips][2][channels]; shared: [parts of a group's channels][rows of the launch][groups][2 kWide].
template <int L> struct Back {
    static constexpr int kWaves = L < 4 ? L : 4, kThreads = kWaves * kWave, kWide = 4 * L;
    static constexpr int kChannels = kThreads / L;                              // of a workgroup
    static constexpr int kItems = (kSelectKeep * kChannels + kThreads - 1) / kThreads;    // rows and channels of a thread
    static constexpr int kSumRows = kWide <= 64 ? kSelectKeep : 4;              // rows whose sums over channels are in LDS at a time (up to 32 KiB)
};
template <class T, int L>
__global__ __launch_bounds__(Back<L>::kThreads, Back<L>::kWaves == 4 ? 2 : 1) void k_select_gradients(SelectArgs args)
{
    typedef Lane<4, L> Mine;
    typedef Back<L> G;
    typedef typename T::Store E;
    constexpr int kRows = kSelectKeep, kWide = G::kWide;
    __shared__ int32_t s_own[G::kWaves][kWave];
    __shared__ float4 s_item[kRows][G::kChannels];                                // step, input, gradient; then sums of e B, A e a h, C h
    __shared__ __attribute__((aligned(16))) float s_bc[2][kRows * kWide];
    __shared__ __attribute__((aligned(16))) float s_sum[G::kWaves][G::kSumRows][2 * kWide];
    const SelectArgs &a = args;
    const int64_t strips = a.slice_strips * a.blocks;
    if (blockIdx.x >= strips) {
        if (a.dh0)
            copy_empties(a.rowptr, a.seqs, a.tokens, a.channels * a.states, a.dfinal, a.dh0, (blockIdx.x - strips) * G::kWaves + wave_id(),
                         (gridDim.x - strips) * G::kWaves);
        return;
    }
    Mine ln;
    // the workgroup's channels from c0 on, of which there are `width`
    ln.strip = divide(blockIdx.x, a.blocks);
    const int64_t block = blockIdx.x - ln.strip * a.blocks;
    ln.strip += a.slice;
    ln.group = divide(block, a.group_blocks);
    const int64_t share = a.channels / a.groups, part = block - ln.group * a.group_blocks, c0 = ln.group * share + part * G::kChannels;
    const int width = (int)(share - part * G::kChannels < G::kChannels ? share - part * G::kChannels : G::kChannels);
    const int lane_channel = threadIdx.x / L;
    ln.active = lane_channel < width;
    ln.c = c0 + (ln.active ? lane_channel : width - 1);
    ln.part = lane_id() % L;
    ln.n0 = ln.part * 4;
    ln.count = a.states - ln.n0 < 0 ? 0 : a.states - ln.n0 > 4 ? 4 : (int32_t)(a.states - ln.n0);
    ln.row0 = ln.strip * a.rows;
    ln.rows = (int32_t)(a.tokens - ln.row0 < a.rows ? a.tokens - ln.row0 : a.rows);
    float A2[4], e[4], dA[4] = {};
    ln.decays(a, A2);
    ln.template before<true>(a, A2, e);
    ln.mark(a, s_own[wave_id()]);

    // the thread's rows and channel where it makes what belongs to a row and channel
    const int item_channel = threadIdx.x % G::kChannels, item_row = G::kChannels == kWave ? wave_id() : (int)threadIdx.x / G::kChannels;
    constexpr int kItemStep = G::kThreads / G::kChannels;
    const bool item = item_channel < width && item_row < kRows;
    const uint32_t own = item_channel < width ? item_channel : width - 1;
    const int64_t ci = c0 + own;
    const float bias = a.delta_bias ? a.delta_bias[ci] : 0.0f, D = a.D ? a.D[ci] : 0.0f;
    float dD = 0.0f, dbias = 0.0f;

    // what the next rows are made of: asked for while the ones after them are worked on
    constexpr int kShared = (kRows * kWide + G::kThreads - 1) / G::kThreads;
    E x1[G::kItems], delta1[G::kItems], dy1[G::kItems], z1[G::kItems], b1[kShared], c1[kShared];
    float h1[4];
    const auto fetch = [&](int64_t row0) {
        const SelectArgs a = asked_again();
#pragma unroll
        for (int j = 0; j < G::kItems; j++) {
            int64_t row = row0 + item_row + j * kItemStep;
            row = row < a.tokens ? row : a.tokens - 1;
            x1[j] = (static_cast<const E *>(a.x) + row * a.x_stride + c0)[own];
            delta1[j] = (static_cast<const E *>(a.delta) + row * a.delta_stride + c0)[own];
            dy1[j] = (static_cast<const E *>(a.dy) + row * a.dy_stride + c0)[own];
            z1[j] = a.z ? (static_cast<const E *>(a.z) + row * a.z_stride + c0)[own] : (E)0.0f;
        }
#pragma unroll
        for (int j = 0; j < kShared; j++) {
            const int at = j * G::kThreads + threadIdx.x, n = at % kWide;
            int64_t row = row0 + at / kWide;
            row = row < a.tokens ? row : a.tokens - 1;
            b1[j] = n < a.states ? static_cast<const E *>(a.B)[row * a.b_stride + ln.group * a.states + n] : (E)0.0f;
            c1[j] = n < a.states ? static_cast<const E *>(a.C)[row * a.c_stride + ln.group * a.states + n] : (E)0.0f;
        }
        ln.load_own(a.kept + ln.own(a, row0 / kRows), h1);
    };
    const int top = (ln.rows - 1) / kRows * kRows;
    fetch(ln.row0 + top);
    for (int k0 = top; k0 >= 0; k0 -= kRows) {
        const uint32_t valid = ln.valid >> k0 & ((1u << kRows) - 1), begin = ln.begin >> k0 & ((1u << kRows) - 1), end = ln.end >> k0 & ((1u << kRows) - 1);
        const int64_t row0 = ln.row0 + k0;
        E x[G::kItems], delta[G::kItems], dy[G::kItems], z[G::kItems];
        float h[4], slope[G::kItems], sigma[G::kItems];
#pragma unroll
        for (int j = 0; j < G::kItems; j++) x[j] = x1[j], delta[j] = delta1[j], dy[j] = dy1[j], z[j] = z1[j];
#pragma unroll
        for (int i = 0; i < 4; i++) h[i] = h1[i];
#pragma unroll
        for (int j = 0; j < kShared; j++) {
            const int at = j * G::kThreads + threadIdx.x;
            if (kShared * G::kThreads == kRows * kWide || at < kRows * kWide) {
                s_bc[0][at] = (float)b1[j];
                s_bc[1][at] = (float)c1[j];
            }
        }
        if (k0 > 0) fetch(row0 - kRows);
        if (valid == 0) { __syncthreads(); continue; }
        const SelectArgs a = asked_again();
#pragma unroll
        for (int j = 0; j < G::kItems; j++) {
            const Step st = step_and_slope((float)delta[j] + bias);
            const float d = st.d, zj = (float)z[j];
            slope[j] = st.slope;
            sigma[j] = a.z ? gate_of<T>(zj) : 0.0f;
            const float o = a.z ? (float)dy[j] * (zj * sigma[j]) : (float)dy[j];
            // (channels that there are not have no part in the sums over channels)
            if (item_row + j * kItemStep < kRows)
                s_item[item_row + j * kItemStep][item_channel] = item_channel < width ? make_float4(d, d * (float)x[j], o, 0.0f) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
        __syncthreads();
        const auto rows = [&](auto inside) {
            const SelectArgs a = asked_again();
            float before[kRows][4], decay[kRows][4];
#pragma unroll
            for (int k = 0; k < kRows; k++) {
                if (!inside.value && !(valid >> k & 1)) continue;
                const float2 du = *reinterpret_cast<const float2 *>(&s_item[k][lane_channel]);
                float b[4];
                take_states(s_bc[0] + k * kWide + ln.n0, b);
                if (!inside.value && (begin >> k & 1)) ln.load(a, a.h0, ln.q(k0 + k), h);
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    before[k][i] = h[i];
                    decay[k][i] = exp2_of(du.x * A2[i]);
                    h[i] = fmaf(decay[k][i], h[i], du.y * b[i]);
                }
            }
#pragma unroll
            for (int k4 = kRows - 4; k4 >= 0; k4 -= 4) {
                float sums[4][8];
#pragma unroll
                for (int r = 3; r >= 0; r--) {
                    const int k = k4 + r;
                    if (!inside.value && !(valid >> k & 1)) {
#pragma unroll
                        for (int i = 0; i < 8; i++) sums[r][i] = 0.0f;
                        continue;
                    }
                    const float4 it = s_item[k][lane_channel];
                    const float d = it.x, u = it.y, o = it.z;
                    float b[4], c[4], y = 0.0f, eb = 0.0f, ea = 0.0f;
                    take_states(s_bc[0] + k * kWide + ln.n0, b);
                    take_states(s_bc[1] + k * kWide + ln.n0, c);
                    if (!inside.value && (end >> k & 1)) ln.load(a, a.dfinal, ln.q(k0 + k), e);
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const float ah = decay[k][i] * before[k][i], now = fmaf(u, b[i], ah);
                        e[i] = fmaf(o, c[i], e[i]);
                        y = fmaf(c[i], now, y);
                        sums[r][i] = e[i] * u;
                        sums[r][4 + i] = o * now;
                        eb = fmaf(e[i], b[i], eb);
                        const float w = e[i] * ah;
                        ea = fmaf(A2[i], w, ea);
                        dA[i] = fmaf(d, w, dA[i]);
                        e[i] *= decay[k][i];
                    }
                    y = sum_channel<L>(y);
                    eb = sum_channel<L>(eb);
                    ea = sum_channel<L>(ea);
                    wave_fence();
                    if (ln.part == 0) *reinterpret_cast<float4 *>(&s_item[k][lane_channel]) = make_float4(eb, ea * kLn2, y, d);
                    if (!inside.value && (begin >> k & 1) && a.dh0) ln.store(a, a.dh0, ln.q(k0 + k), e);
                }
                sum_rows<L>(sums);
                // (lanes of the same states hold the same sums: those of the first channel of their part of the wave write)
                constexpr int kLeft = L <= 16 ? 1 : L <= 32 ? 2 : 4, kPart = L <= 16 ? 16 : L <= 32 ? 32 : 64;
                const int first = k4 % G::kSumRows + (L <= 32 ? lane_id() / 32 * 2 : 0) + (L <= 16 ? lane_id() / 16 % 2 : 0);
                if (lane_id() % kPart < L) {
#pragma unroll
                    for (int r = 0; r < kLeft; r++) {
                        float *to = s_sum[wave_id()][first + r];
                        *reinterpret_cast<float4 *>(to + ln.n0) = make_float4(sums[r][0], sums[r][1], sums[r][2], sums[r][3]);
                        *reinterpret_cast<float4 *>(to + kWide + ln.n0) = make_float4(sums[r][4], sums[r][5], sums[r][6], sums[r][7]);
                    }
                }
                if (k4 % G::kSumRows == 0) {
                    __syncthreads();
                    float *to = a.shared + ((part * a.slice_rows + row0 - a.slice * a.rows + k4) * a.groups + ln.group) * (2 * kWide);
                    for (int at = threadIdx.x; at < G::kSumRows * 2 * kWide; at += G::kThreads) {
                        const int r = at / (2 * kWide), n = at % (2 * kWide);
                        float sum = 0.0f;
#pragma unroll
                        for (int w = 0; w < G::kWaves; w++) sum += s_sum[w][r][n];
                        if (inside.value || k0 + k4 + r < ln.rows) to[r * a.groups * (2 * kWide) + n] = sum;
                    }
                    if (G::kSumRows < kRows) __syncthreads();
                }
            }
        };
        // (most rows are in the middle of a sequence: those ask for nothing, so that the next ones can be under way)
        if (valid == (1u << kRows) - 1 && (begin | end) == 0) rows(std::true_type());
        else rows(std::false_type());
        if (G::kSumRows < kRows) __syncthreads();
        const SelectArgs b = asked_again();
#pragma unroll
        for (int j = 0; j < G::kItems; j++) {
            const int k = item_row + j * kItemStep;
            if (!item || k >= kRows || !(valid >> k & 1)) continue;
            const int64_t row = row0 + k;
            const float4 got = s_item[k][item_channel];
            const float xj = (float)x[j], dyj = (float)dy[j], zj = (float)z[j], eb = got.x, d = got.w;
            float o = dyj, y = got.z;
            if (b.D) y = fmaf(D, xj, y);
            if (b.z) {
                const float s = sigma[j];
                o = dyj * (zj * s);
                (static_cast<E *>(b.dz) + row * b.dz_stride + c0)[own] = (E)(dyj * y * (s * fmaf(zj, 1.0f - s, 1.0f)));
            }
            const float dx = b.D ? fmaf(D, o, d * eb) : d * eb, dd = fmaf(eb, xj, got.y) * slope[j];
            (static_cast<E *>(b.dx) + row * b.dx_stride + c0)[own] = (E)dx;
            (static_cast<E *>(b.ddelta) + row * b.ddelta_stride + c0)[own] = (E)dd;
            dD = fmaf(o, xj, dD);
            dbias += dd;
        }
        __syncthreads();
    }
    ln.store_own(a.partial + ln.own(a, ln.strip), dA);
    // (the threads of a channel, one after the other)
    constexpr bool kItemsFit = sizeof(s_item) >= G::kThreads * sizeof(float2);
    static_assert(kItemsFit || sizeof(s_sum) >= G::kThreads * sizeof(float2), "a pair for each thread");
    float2 *pair = kItemsFit ? reinterpret_cast<float2 *>(&s_item[0][0]) : reinterpret_cast<float2 *>(&s_sum[0][0][0]);
    pair[threadIdx.x] = make_float2(dD, dbias);
    __syncthreads();
    if ((int)threadIdx.x < width) {
        float2 sum = make_float2(0.0f, 0.0f);
        for (int r = 0; r < kItemStep; r++) {
            const float2 v = pair[threadIdx.x + r * G::kChannels];
            sum.x += v.x;
            sum.y += v.y;
        }
        float *to = a.partial + a.strips * a.channels * kWide + ln.strip * 2 * a.channels + c0 + threadIdx.x;
        to[0] = sum.x;
        to[a.channels] = sum.y;
    }
}

// Sums over strips, in 64 bits: a wave has 64 neighbours of a strip's, kSumPieces waves a share of the strips each.
constexpr int kSumPieces = 16;
__global__ __launch_bounds__(kSumPieces *kWave) void k_select_sums(SelectArgs a, int wide)
{
    __shared__ double s_sum[kSumPieces][kWave];
    const int64_t first = a.channels * wide, slot = (int64_t)blockIdx.x * kWave + lane_id();
    const bool tail = slot >= first;
    const int64_t stride = tail ? 2 * a.channels : first;
    const float *from = tail ? a.partial + a.strips * first + (slot - first) : a.partial + slot;
    const bool there = slot < first + 2 * a.channels;
    double sum = 0.0;
    if (there) {
#pragma unroll 4
        for (int64_t k = wave_id(); k < a.strips; k += kSumPieces) sum += (double)from[k * stride];
    }
    s_sum[wave_id()][lane_id()] = sum;
    __syncthreads();
    if (wave_id() || !there) return;
    for (int w = 1; w < kSumPieces; w++) sum += s_sum[w][lane_id()];
    if (!tail) {
        const int64_t c = divide(slot, wide), n = slot - c * wide;
        if (n < a.states) a.dA[c * a.states + n] = (float)sum;
        return;
    }
    const int64_t c = slot - first;
    if (c < a.channels) { if (a.dD) a.dD[c] = (float)sum; }
    else if (a.ddelta_bias) a.ddelta_bias[c - a.channels] = (float)sum;
}

// Sums over the parts of a group's channels, of the rows of the launch before it.
template <class T>
__global__ __launch_bounds__(256) void k_select_shared(SelectArgs a, int wide)
{
    typedef typename T::Store E;
    const int64_t first = a.slice * a.rows, past = first + a.slice_rows, from0 = row_bound(a.rowptr[0], a.tokens), to0 = row_bound(a.rowptr[a.seqs], a.tokens);
    const int64_t low = from0 > first ? from0 : first, high = to0 < past ? to0 : past, width = a.groups * a.states;
    for (int64_t i = low * width + (int64_t)blockIdx.x * 256 + threadIdx.x; i < high * width; i += (int64_t)gridDim.x * 256) {
        const int64_t row = divide(i, width), at = i - row * width, group = divide(at, a.states), n = at - group * a.states;
        float b = 0.0f, c = 0.0f;
#pragma unroll 4
        for (int64_t p = 0; p < a.group_blocks; p++) {
            const float *from = a.shared + ((p * a.slice_rows + row - first) * a.groups + group) * (2 * wide) + n;
            b += from[0];
            c += from[wide];
        }
        static_cast<E *>(a.dB)[row * a.db_stride + at] = (E)b;
        static_cast<E *>(a.dC)[row * a.dc_stride + at] = (E)c;
    }
}

template <class T, int S, int L> static void go_back_ends(const SelectArgs &a, const SelectLayout &l, hipStream_t s)
{
    SelectArgs f = a;                       // (cut as the forward pass is)
    f.blocks = l.blocks;
    f.group_blocks = (int32_t)l.group_blocks;
    const int64_t groups = (f.strips * f.blocks + kSelectWaves - 1) / kSelectWaves;
    hipLaunchKernelGGL((k_select_back_ends<T, S, L>), dim3((unsigned)groups), dim3(kSelectWaves * kWave), 0, s, f);
    if (a.before) select_states(f, l.wide, true, s);
}
template <class T, int L> static void go_gradients(const SelectArgs &a, hipStream_t s)
{
    const int64_t groups = a.slice_strips * a.blocks + (a.dh0 && a.slice == 0 ? copy_groups(a.seqs, a.channels * a.states, Back<L>::kWaves) : 0);
    if (groups > 0) hipLaunchKernelGGL((k_select_gradients<T, L>), dim3((unsigned)groups), dim3(Back<L>::kThreads), 0, s, a);
}
template <class T> static void go_backward(SelectArgs a, const SelectLayout &l, hipStream_t s)
{
    if (a.strips > 1) {
#define DGN_CALL(S, L) go_back_ends<T, S, L>(a, l, s)
        DGN_BY_LANES(l.S, l.L, DGN_CALL);
#undef DGN_CALL
    }
    for (a.slice = 0; a.slice == 0 || a.slice < a.strips; a.slice += l.slice) {     // (without rows: what belongs to sequences alone)
        a.slice_strips = a.strips - a.slice < l.slice ? a.strips - a.slice : l.slice;
        a.slice_rows = a.tokens - a.slice * a.rows < l.slice * a.rows ? a.tokens - a.slice * a.rows : l.slice * a.rows;
        switch (l.wide / 4) {
        case 1: go_gradients<T, 1>(a, s); break;
        case 2: go_gradients<T, 2>(a, s); break;
        case 4: go_gradients<T, 4>(a, s); break;
        case 8: go_gradients<T, 8>(a, s); break;
        case 16: go_gradients<T, 16>(a, s); break;
        case 32: go_gradients<T, 32>(a, s); break;
        default: go_gradients<T, 64>(a, s);
        }
        if (a.strips == 0) break;
        const int64_t n = (a.slice_rows * a.groups * a.states + 255) / 256;
        hipLaunchKernelGGL((k_select_shared<T>), dim3((unsigned)(n < 8192 ? n : 8192)), dim3(256), 0, s, a, l.wide);
    }
    const int64_t sums = (a.channels * (l.wide + 2) + kWave - 1) / kWave;
    hipLaunchKernelGGL(k_select_sums, dim3((unsigned)sums), dim3(kSumPieces * kWave), 0, s, a, l.wide);
}
void select_backward(int dtype, const SelectArgs &a, const SelectLayout &l, hipStream_t s)
{
#define DGN_GO(T) go_backward<T>(a, l, s)
    DGN_BY_DTYPE(dtype, DGN_GO);
#undef DGN_GO
}

}  // namespace dgn
