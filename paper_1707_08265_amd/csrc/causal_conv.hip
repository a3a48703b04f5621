// Short causal convolution over ragged sequences, forward, backward and for one token, channel by channel:
//   p_t = bias + sum_j w_j x_{t-(K-1)+j},   y = p or p sigma(p)
// and, with g_t = dy_t y'(p_t) (zero from the sequence's end on),
//   dx_t = sum_i w_{K-1-i} g_{t+i} (+ dfinal, in the last K-1 rows),   dw_j = sum_t g_t x_{t-(K-1)+j},   dbias = sum_t g_t,
// and dstate0 by dx's sum for the K-1 rows before a sequence.
//
// A wave takes a run of rows of 64 V channels and goes down (backward: up) it, eight rows in registers with the K-1 before them.  Which
// rows sequences begin and end with is the same for the wave; eight rows in the middle of a sequence ask for nothing, rows whose window reaches
// into a state look there.  Bound by memory: training step of 65 301 x 1 024 in f16, 268 MB forward in 54 us (4.9 TB/s; a copy has 6.2), vector units
// 46 % busy, and 403 MB backward in 93 to 96 (4.2 to 4.3), 58 % busy with under three waves a SIMD, which wait for memory 39 % of their time.
// (Times of calls on the same tensors, half of whose inputs the last-level cache has kept; a training step on others is 3 us longer.)
#include "layer.h"
#include "rows.h"

namespace dgn {

constexpr int kConvRows = 56;           // rows of a run, at most: with those that a backward pass looks ahead to, a lane for each
constexpr int kConvBatch = 8, kConvWaves = 4;

__device__ __forceinline__ int64_t conv_low(int64_t a, int64_t b) { return a < b ? a : b; }

// sigma(p): 32-bit results by a rounded exponential and quotient, of 16 bits by the card's approximations (a few 2^-24 of them).
template <class T> __device__ __forceinline__ float conv_sigmoid(float p)
{
    if (sizeof(typename T::Store) == 4) return 1.0f / (1.0f + expf(-p));
    return __builtin_amdgcn_rcpf(1.0f + __expf(-p));
}

// What a wave has of a run: its rows, its channels, and the sequences of its rows, one row to a lane.
template <int V> struct Run {
    int64_t run, row0, c;
    RowSeq seq;
    u64 valid, begin, end, early, late;  // (early: less than K - 1 rows into its sequence; late: less than K - 1 before its last)
    int32_t rows, place, left;          // place of the lane's row in its sequence, and rows from it to the end

    __device__ __forceinline__ bool find(const ConvArgs &a, int64_t block, int64_t run_)
    {
        run = run_;
        row0 = run * a.rows;
        rows = (int32_t)conv_low(a.tokens - row0, a.rows);
        const int64_t at = (block * kWave + lane_id()) * V;
        c = at + V <= a.channels ? at : a.channels - V;         // (lanes past the end do what the last does, to the same places)
        return rows > 0;
    }
    __device__ __forceinline__ void mark(const ConvArgs &a, int32_t *own)
    {
        seq = sequences_of(a.rowptr, a.seqs, a.tokens, row0, own);
        const int64_t row = row0 + lane_id();
        valid = __ballot(seq.q >= 0);
        begin = __ballot(seq.q >= 0 && seq.first == row);
        end = __ballot(seq.q >= 0 && seq.end == row + 1);
        place = (int32_t)conv_low(row - seq.first, kWave);
        left = (int32_t)conv_low(seq.end - row, kWave);
        early = __ballot(place < a.taps - 1);
        late = __ballot(left < a.taps);
    }
    __device__ __forceinline__ int64_t q(int k) const { return __builtin_amdgcn_readlane(seq.q, k); }
};

// Rows k0 - (K-1) .. k0 + 7 of a run.
template <class T, int V, int K> struct Window {
    typedef typename T::Store S;
    Pack<T, V> x[kConvBatch + K - 1];
    __device__ __forceinline__ void load(const ConvArgs &a, int64_t row, int64_t c)
    {
#pragma unroll
        for (int k = 0; k < kConvBatch + K - 1; k++) {
            int64_t r = row + k - (K - 1);
            r = r < 0 ? 0 : conv_low(r, a.tokens - 1);
            x[k].load(static_cast<const S *>(a.x) + r * a.x_stride + c);
        }
    }
    // The eight rows after those that it has, from `row` on.
    __device__ __forceinline__ void follow(const ConvArgs &a, int64_t row, int64_t c)
    {
#pragma unroll
        for (int k = 0; k < K - 1; k++) x[k] = x[kConvBatch + k];
#pragma unroll
        for (int k = 0; k < kConvBatch; k++) x[K - 1 + k].load(static_cast<const S *>(a.x) + conv_low(row + k, a.tokens - 1) * a.x_stride + c);
    }
    // The eight rows before those that it has, from `row` on.
    __device__ __forceinline__ void precede(const ConvArgs &a, int64_t row, int64_t c)
    {
#pragma unroll
        for (int k = K - 2; k >= 0; k--) x[kConvBatch + k] = x[k];
#pragma unroll
        for (int k = 0; k < kConvBatch; k++) {
            const int64_t r = row + k - (K - 1);
            x[k].load(static_cast<const S *>(a.x) + (r < 0 ? 0 : r) * a.x_stride + c);
        }
    }
    // The K rows that row k's result is made of, oldest first.
    template <bool kInside> __device__ __forceinline__ void at(const ConvArgs &a, const Run<V> &run, int k0, int k, float (&w)[K][V]) const
    {
#pragma unroll
        for (int j = 0; j < K; j++)
#pragma unroll
            for (int i = 0; i < V; i++) w[j][i] = x[k + j].get(i);
        if (kInside || !(run.early >> (k0 + k) & 1)) return;
        const int place = __builtin_amdgcn_readlane(run.place, k0 + k);
        const S *state = static_cast<const S *>(a.state0) + run.q(k0 + k) * (K - 1) * a.channels + run.c;
#pragma unroll
        for (int s = 1; s < K; s++) {
            if (place >= s) continue;
#pragma unroll
            for (int i = 0; i < V; i++) w[K - 1 - s][i] = a.state0 ? (float)state[(K - 1 + place - s) * a.channels + i] : 0.0f;
        }
    }
};

template <int V, int K> struct Taps {
    float w[K][V], bias[V];
    __device__ __forceinline__ void load(const float *weight, const float *b, int64_t c)
    {
#pragma unroll
        for (int i = 0; i < V; i++) {
#pragma unroll
            for (int j = 0; j < K; j++) w[j][i] = weight[(c + i) * K + j];
            bias[i] = b ? b[c + i] : 0.0f;
        }
    }
    __device__ __forceinline__ float sum(const float (&x)[K][V], int i) const
    {
        float p = bias[i];
#pragma unroll
        for (int j = 0; j < K; j++) p = fmaf(w[j][i], x[j][i], p);
        return p;
    }
};

template <class T, int V, bool kStream = false> __device__ __forceinline__ void conv_store(void *base, int64_t at, const float (&v)[V])
{
    Pack<T, V> p;
    p.set(v);
    p.template store<kStream>(static_cast<typename T::Store *>(base) + at);
}

template <class T, int V, int K, bool kSilu, bool kStream>
__global__ __launch_bounds__(kConvWaves *kWave) void k_conv_forward(ConvArgs a)
{
    __shared__ int32_t s_own[kConvWaves][kWave];
    const int64_t groups = (a.runs + kConvWaves - 1) / kConvWaves;
    if (blockIdx.x >= groups * a.blocks) {
        typedef typename T::Store S;
        if (a.final)
            copy_empties(a.rowptr, a.seqs, a.tokens, (K - 1) * a.channels, static_cast<const S *>(a.state0), static_cast<S *>(a.final),
                         (blockIdx.x - groups * a.blocks) * kConvWaves + wave_id(), (gridDim.x - groups * a.blocks) * kConvWaves);
        return;
    }
    const int64_t group = divide(blockIdx.x, a.blocks), block = blockIdx.x - group * a.blocks;
    Run<V> run;
    if (!run.find(a, block, group * kConvWaves + wave_id())) return;
    Window<T, V, K> next;
    next.load(a, run.row0, run.c);
    Taps<V, K> taps;
    taps.load(a.weight, a.bias, run.c);
    run.mark(a, s_own[wave_id()]);
    for (int k0 = 0; k0 < run.rows; k0 += kConvBatch) {
        const Window<T, V, K> win = next;
        if (k0 + kConvBatch < run.rows) next.follow(a, run.row0 + k0 + kConvBatch, run.c);
        const u64 odd = ~run.valid | run.early | run.end;
        const auto rows = [&](auto inside) {
#pragma unroll
            for (int k = 0; k < kConvBatch; k++) {
                if (!inside.value && (k0 + k >= run.rows || !(run.valid >> (k0 + k) & 1))) continue;
                float x[K][V], y[V];
                win.template at<inside.value>(a, run, k0, k, x);
#pragma unroll
                for (int i = 0; i < V; i++) {
                    y[i] = taps.sum(x, i);
                    if (kSilu) y[i] *= conv_sigmoid<T>(y[i]);
                }
                conv_store<T, V, kStream>(a.y, (run.row0 + k0 + k) * a.y_stride + run.c, y);
                if (!inside.value && (run.end >> (k0 + k) & 1) && a.final) {
#pragma unroll
                    for (int j = 1; j < K; j++) conv_store<T, V>(a.final, (run.q(k0 + k) * (K - 1) + j - 1) * a.channels + run.c, x[j]);
                }
            }
        };
        // (most rows are in the middle of a sequence)
        if ((odd >> k0 & 0xff) == 0 && k0 + kConvBatch <= run.rows) rows(std::true_type());
        else rows(std::false_type());
    }
}

// Backward.  A run begins with the K-1 rows after it, whose g the gradients of its last rows are made of.
template <class T, int V, int K, bool kSilu, bool kStream>
__global__ __launch_bounds__(kConvWaves *kWave) void k_conv_backward(ConvArgs a)
{
    typedef typename T::Store S;
    __shared__ int32_t s_own[kConvWaves][kWave];
    __shared__ float s_sum[kConvWaves][K + 1][V][kWave];
    const int64_t groups = (a.runs + kConvWaves - 1) / kConvWaves;
    if (blockIdx.x >= groups * a.blocks) {
        if (a.dstate0)
            copy_empties(a.rowptr, a.seqs, a.tokens, (K - 1) * a.channels, static_cast<const S *>(a.dfinal), static_cast<S *>(a.dstate0),
                         (blockIdx.x - groups * a.blocks) * kConvWaves + wave_id(), (gridDim.x - groups * a.blocks) * kConvWaves);
        return;
    }
    const int64_t group = divide(blockIdx.x, a.blocks), block = blockIdx.x - group * a.blocks;
    float dw[K + 1][V];                 // (the last: of the bias)
#pragma unroll
    for (int j = 0; j <= K; j++)
#pragma unroll
        for (int i = 0; i < V; i++) dw[j][i] = 0.0f;
    Run<V> run;
    const S *dfinal = static_cast<const S *>(a.dfinal);
    if (run.find(a, block, group * kConvWaves + wave_id())) {
        Taps<V, K> taps;
        taps.load(a.weight, a.bias, run.c);
        float g[K][V];                  // g_t .. g_{t+K-1}
#pragma unroll
        for (int j = 0; j < K; j++)
#pragma unroll
            for (int i = 0; i < V; i++) g[j][i] = 0.0f;
        // (without rows after it, from its last batch on)
        const int top = run.rows < a.rows ? (run.rows - 1) / kConvBatch * kConvBatch : a.rows;
        Window<T, V, K> next;
        Pack<T, V> dy_next[kConvBatch];
        const auto fetch = [&](int k0) {
#pragma unroll
            for (int k = 0; k < kConvBatch; k++)
                dy_next[k].load(static_cast<const S *>(a.dy) + conv_low(run.row0 + k0 + k, a.tokens - 1) * a.dy_stride + run.c);
        };
        next.load(a, run.row0 + top, run.c);
        fetch(top);
        run.mark(a, s_own[wave_id()]);
        for (int k0 = top; k0 >= 0; k0 -= kConvBatch) {
            const bool ahead = k0 == a.rows;
            const int some = ahead ? K - 1 : kConvBatch;
            const Window<T, V, K> win = next;
            Pack<T, V> dy[kConvBatch];
#pragma unroll
            for (int k = 0; k < kConvBatch; k++) dy[k] = dy_next[k];
            if (k0 > 0) {
                next.precede(a, run.row0 + k0 - kConvBatch, run.c);
                fetch(k0 - kConvBatch);
            }
            const u64 odd = ~run.valid | run.early | run.late;
            const auto rows = [&](auto inside) {
#pragma unroll
                for (int k = kConvBatch - 1; k >= 0; k--) {
                    if (!inside.value && (k >= some || !(run.valid >> (k0 + k) & 1))) continue;
                    const int64_t row = run.row0 + k0 + k;
                    float x[K][V];
                    win.template at<inside.value>(a, run, k0, k, x);
                    const bool last = !inside.value && (run.end >> (k0 + k) & 1);
#pragma unroll
                    for (int j = K - 1; j > 0; j--)
#pragma unroll
                        for (int i = 0; i < V; i++) g[j][i] = last ? 0.0f : g[j - 1][i];
#pragma unroll
                    for (int i = 0; i < V; i++) {
                        g[0][i] = dy[k].get(i);
                        if (kSilu) {
                            const float p = taps.sum(x, i), s = conv_sigmoid<T>(p);
                            g[0][i] *= s * fmaf(p, 1.0f - s, 1.0f);
                        }
                    }
                    if (!inside.value && ahead) continue;
                    float dx[V];
#pragma unroll
                    for (int i = 0; i < V; i++) {
                        dx[i] = 0.0f;
#pragma unroll
                        for (int j = 0; j < K; j++) {
                            dx[i] = fmaf(taps.w[K - 1 - j][i], g[j][i], dx[i]);
                            dw[j][i] = fmaf(g[0][i], x[j][i], dw[j][i]);
                        }
                        dw[K][i] += g[0][i];
                    }
                    const int left = inside.value ? kWave : __builtin_amdgcn_readlane(run.left, k0 + k);
                    if (dfinal && left <= K - 1) {
                        const S *d = dfinal + (run.q(k0 + k) * (K - 1) + K - 1 - left) * a.channels + run.c;
#pragma unroll
                        for (int i = 0; i < V; i++) dx[i] += (float)d[i];
                    }
                    conv_store<T, V, kStream>(a.dx, row * a.dx_stride + run.c, dx);
                    if (inside.value || !(run.begin >> (k0 + k) & 1) || !a.dstate0) continue;
#pragma unroll
                    for (int m = 1; m < K; m++) {           // the row m before the first; the sequence has `left` rows
                        float ds[V];
#pragma unroll
                        for (int i = 0; i < V; i++) {
                            ds[i] = 0.0f;
#pragma unroll
                            for (int j = m; j < K; j++) ds[i] = fmaf(taps.w[K - 1 - j][i], g[j - m][i], ds[i]);
                        }
                        if (dfinal && left + m <= K - 1) {
                            const S *d = dfinal + (run.q(k0 + k) * (K - 1) + K - 1 - left - m) * a.channels + run.c;
#pragma unroll
                            for (int i = 0; i < V; i++) ds[i] += (float)d[i];
                        }
                        conv_store<T, V>(a.dstate0, (run.q(k0 + k) * (K - 1) + K - 1 - m) * a.channels + run.c, ds);
                    }
                }
            };
            if (!ahead && (odd >> k0 & 0xff) == 0) rows(std::true_type());
            else rows(std::false_type());
        }
    }
#pragma unroll
    for (int j = 0; j <= K; j++)
#pragma unroll
        for (int i = 0; i < V; i++) s_sum[wave_id()][j][i][lane_id()] = dw[j][i];
    __syncthreads();
    for (int at = threadIdx.x; at < (K + 1) * V * kWave; at += kConvWaves * kWave) {
        const int lane = at % kWave, i = at / kWave % V, j = at / (kWave * V);
        float sum = 0.0f;
        for (int w = 0; w < kConvWaves; w++) sum += s_sum[w][j][i][lane];
        const int64_t c = (block * kWave + lane) * V + i;
        // (of lanes past the end only the last channels' own places count)
        if (c < a.channels && (block * kWave + lane + 1) * V <= a.channels) a.partial[(group * (K + 1) + j) * a.channels + c] = sum;
        else if (c < a.channels) {
            // the last lane is moved back to end with the last channel: its channel c is V - (channels - first) places further on
            const int64_t first = (block * kWave + lane) * V, moved = first + V - a.channels;
            float tail = 0.0f;
            for (int w = 0; w < kConvWaves; w++) tail += s_sum[w][j][i + (int)moved][lane];
            a.partial[(group * (K + 1) + j) * a.channels + c] = tail;
        }
    }
}

// The sums over all rows, in 64 bits (341 parts of 1 024 channels: 5.3 us): a workgroup has 64 channels of one tap (or the bias), each of its waves a share of the parts.
constexpr int kSumWaves = 16;
__global__ __launch_bounds__(kSumWaves *kWave) void k_conv_sums(ConvArgs a, int64_t parts)
{
    __shared__ double s_sum[kSumWaves][kWave];
    const int64_t c = (int64_t)blockIdx.x * kWave + lane_id(), j = blockIdx.y;
    double sum = 0.0;
    if (c < a.channels)
#pragma unroll 8
        for (int64_t p = wave_id(); p < parts; p += kSumWaves) sum += (double)a.partial[(p * (a.taps + 1) + j) * a.channels + c];
    s_sum[wave_id()][lane_id()] = sum;
    __syncthreads();
    if (wave_id() || c >= a.channels) return;
    for (int w = 1; w < kSumWaves; w++) sum += s_sum[w][lane_id()];
    if (j < a.taps) a.dweight[c * a.taps + j] = (float)sum;
    else if (a.dbias) a.dbias[c] = (float)sum;
}

// A copy of the states that come in, for calls whose states go out to the same memory: runs read and write them in any order.
template <class S> __global__ __launch_bounds__(256) void k_copy_rows(const S *from, S *to, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) to[i] = from[i];
}

// One token: a row of the batch is cut into pieces of 256 V channels.  512 rows of 2 048 channels in bf16: 16 MB in 6.4 us.
template <class T, int V, int K, bool kSilu>
__global__ __launch_bounds__(256) void k_conv_step(ConvStepArgs a)
{
    typedef typename T::Store S;
    for (int64_t at = blockIdx.x; at < a.rows * a.pieces; at += gridDim.x) {
        const int64_t row = divide(at, a.pieces), c = (at - row * a.pieces) * (256 * V) + threadIdx.x * V;
        if (c >= a.channels) continue;
        const int64_t slot = a.slot ? a.slot[row] : row;
        float y[V];
#pragma unroll
        for (int i = 0; i < V; i++) y[i] = 0.0f;
        if (slot >= 0 && slot < a.slots) {
            Pack<T, V> x[K];
            const int64_t state = slot * (K - 1) * a.channels + c;
#pragma unroll
            for (int j = 0; j < K - 1; j++) x[j].load(static_cast<const S *>(a.state_in) + state + j * a.channels);
            x[K - 1].load(static_cast<const S *>(a.x) + row * a.x_stride + c);
            Taps<V, K> taps;
            taps.load(a.weight, a.bias, c);
            float w[K][V];
#pragma unroll
            for (int j = 0; j < K; j++)
#pragma unroll
                for (int i = 0; i < V; i++) w[j][i] = x[j].get(i);
#pragma unroll
            for (int i = 0; i < V; i++) {
                y[i] = taps.sum(w, i);
                if (kSilu) y[i] *= conv_sigmoid<T>(y[i]);
            }
#pragma unroll
            for (int j = 1; j < K; j++) x[j].store(static_cast<S *>(a.state_out) + state + (j - 1) * a.channels);
        }
        conv_store<T, V>(a.y, row * a.y_stride + c, y);
    }
}

// Four bytes of a row a lane (eight: training step of 65 301 x 1 024, forward 56 instead of 53 us, backward 119 instead of 102); rows that are shorter
// than that one element.
static int conv_width(int dtype, int64_t channels)
{
    const int V = dtype == DGN_F32 ? 1 : 2;
    return channels >= V ? V : 1;
}
// Rows of a run: as few as give kConvRuns waves (16 384: the training step's 104 us backward become 118), from kConvBatch to kConvRows.
constexpr int64_t kConvRuns = 8192;
struct ConvLayout { int V; int64_t blocks, rows, runs, groups; size_t before, bytes; };
static ConvLayout conv_layout(int dtype, const ConvArgs &a)
{
    ConvLayout l;
    l.V = conv_width(dtype, a.channels);
    l.blocks = (a.channels + kWave * l.V - 1) / (kWave * l.V);
    l.rows = a.tokens * l.blocks / kConvRuns / kConvBatch * kConvBatch;
    l.rows = l.rows < kConvBatch ? kConvBatch : l.rows > kConvRows ? kConvRows : l.rows;
    l.runs = (a.tokens + l.rows - 1) / l.rows;
    l.groups = (l.runs + kConvWaves - 1) / kConvWaves;
    l.before = (size_t)l.groups * (a.taps + 1) * a.channels * sizeof(float);
    l.bytes = l.before + (size_t)a.seqs * (a.taps - 1) * a.channels * element_size(dtype);
    return l;
}
bool conv_fits(int dtype, const ConvArgs &a)        // launches of less than 2^32 threads
{
    const ConvLayout l = conv_layout(dtype, a);
    return l.groups * l.blocks < ((int64_t)1 << 24) - kMostCopyGroups && a.channels <= ((int64_t)1 << 28) - kWave;
}
size_t conv_scratch_bytes(int dtype, const ConvArgs &a) { return conv_layout(dtype, a).bytes; }

template <class T, int V, int K, bool kSilu, bool kStream> static void go_conv(bool back, const ConvArgs &a, const ConvLayout &l, hipStream_t s)
{
    const int64_t empties = (back ? a.dstate0 : a.final) ? copy_groups(a.seqs, (K - 1) * a.channels, kConvWaves) : 0;
    const dim3 grid((unsigned)(l.groups * l.blocks + empties)), threads(kConvWaves * kWave);
    const bool any = a.seqs > 0 && grid.x > 0;
    if (!back) {
        if (any) hipLaunchKernelGGL((k_conv_forward<T, V, K, kSilu, kStream>), grid, threads, 0, s, a);
        return;
    }
    if (any) hipLaunchKernelGGL((k_conv_backward<T, V, K, kSilu, kStream>), grid, threads, 0, s, a);
    const dim3 sums((unsigned)((a.channels + kWave - 1) / kWave), (unsigned)(a.taps + 1));
    hipLaunchKernelGGL(k_conv_sums, sums, dim3(kSumWaves * kWave), 0, s, a, a.seqs > 0 ? l.groups : 0);
}
// Results of calls that are larger than the last-level cache go past it (65 301 x 1 024 backward, 403 MB: 102 -> 93 us).
template <class T, int K, bool kSilu> static void by_width(bool back, const ConvArgs &a, const ConvLayout &l, hipStream_t s)
{
    constexpr int V = 4 / (int)sizeof(typename T::Store);
    const bool stream = (size_t)a.tokens * a.channels * (back ? 3 : 2) * sizeof(typename T::Store) > kStreamBytes;
    if (l.V != V) go_conv<T, 1, K, kSilu, false>(back, a, l, s);
    else if (stream) go_conv<T, V, K, kSilu, true>(back, a, l, s);
    else go_conv<T, V, K, kSilu, false>(back, a, l, s);
}
template <class T, bool kSilu> static void by_taps(bool back, const ConvArgs &a, const ConvLayout &l, hipStream_t s)
{
    if (a.taps == 2) by_width<T, 2, kSilu>(back, a, l, s);
    else if (a.taps == 3) by_width<T, 3, kSilu>(back, a, l, s);
    else by_width<T, 4, kSilu>(back, a, l, s);
}
template <class T> static hipError_t go(int activation, bool back, ConvArgs a, void *scratch, hipStream_t s)
{
    const ConvLayout l = conv_layout(sizeof(typename T::Store) == 4 ? DGN_F32 : DGN_F16, a);
    char *mem = static_cast<char *>(scratch);
    a.runs = l.runs;
    a.blocks = l.blocks;
    a.rows = (int32_t)l.rows;
    a.partial = reinterpret_cast<float *>(mem);
    typedef typename T::Store S;
    const int64_t n = a.seqs * (a.taps - 1) * a.channels;
    const S *in = static_cast<const S *>(a.state0), *out = static_cast<const S *>(a.final);
    if (!back && in && out && in < out + n && out < in + n) {
        S *copy = reinterpret_cast<S *>(mem + l.before);
        const int64_t groups = (n + 255) / 256;
        hipLaunchKernelGGL(k_copy_rows<S>, dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(256), 0, s, in, copy, n);
        a.state0 = copy;
    }
    if (activation == DGN_ACT_SILU) by_taps<T, true>(back, a, l, s);
    else by_taps<T, false>(back, a, l, s);
    return hipGetLastError();
}
hipError_t launch_conv(int dtype, int activation, bool back, const ConvArgs &a, void *scratch, hipStream_t s)
{
#define DGN_GO(T) return go<T>(activation, back, a, scratch, s)
    DGN_BY_DTYPE(dtype, DGN_GO);
#undef DGN_GO
}

template <class T, bool kSilu> static void go_step(int taps, ConvStepArgs a, hipStream_t s)
{
    constexpr int kMost = 8 / (int)sizeof(typename T::Store);
    const int V = a.channels % kMost == 0 ? kMost : 1;          // (a row's last lane has as many as the others)
    a.pieces = (a.channels + 256 * V - 1) / (256 * V);
    const int64_t n = a.rows * a.pieces;
    const dim3 grid((unsigned)(n < (1 << 22) ? n : 1 << 22)), threads(256);
    if (V == 1) {
        if (taps == 2) hipLaunchKernelGGL((k_conv_step<T, 1, 2, kSilu>), grid, threads, 0, s, a);
        else if (taps == 3) hipLaunchKernelGGL((k_conv_step<T, 1, 3, kSilu>), grid, threads, 0, s, a);
        else hipLaunchKernelGGL((k_conv_step<T, 1, 4, kSilu>), grid, threads, 0, s, a);
    } else {
        if (taps == 2) hipLaunchKernelGGL((k_conv_step<T, kMost, 2, kSilu>), grid, threads, 0, s, a);
        else if (taps == 3) hipLaunchKernelGGL((k_conv_step<T, kMost, 3, kSilu>), grid, threads, 0, s, a);
        else hipLaunchKernelGGL((k_conv_step<T, kMost, 4, kSilu>), grid, threads, 0, s, a);
    }
}
hipError_t launch_conv_step(int dtype, int activation, int taps, const ConvStepArgs &a, hipStream_t s)
{
#define DGN_GO(T)                                                    \
    if (activation == DGN_ACT_SILU) go_step<T, true>(taps, a, s);   \
    else go_step<T, false>(taps, a, s)
    DGN_BY_DTYPE(dtype, DGN_GO);
#undef DGN_GO
    return hipGetLastError();
}

}  // namespace dgn
