// Gated linear recurrence over ragged sequences, forward, backward and for one token.
//   decay:    a_t = gate_t,          u_t = x_t
//   sigmoid:  a_t = sigma(gate_t),   u_t = (1 - a_t) x_t
//   h_t = a_t h_{t-1} + u_t
// and, with e_t the gradient of h_t (what reaches y_t and what comes back from h_{t+1}),
//   e_t = dy_t + a_{t+1} e_{t+1},   dh0 = a_0 e_0
//   decay:    dx = e,               dgate = e_t h_{t-1}
//   sigmoid:  dx = (1 - a) e,       dgate = a (1 - a) e_t (h_{t-1} - x_t)
// A gate may be shared by `group` channels; its gradient is then the sum over them.
//
// Both directions go over their data once.  The rows, whatever sequences they belong to, are cut into tiles; a workgroup
// takes a tile of some channels into registers, kTokens rows to a thread.  What a run of rows does to the state that comes
// into it is h -> A h + B (A the product of its gates, B its end from a state of zero), or h -> B if a sequence begins in
// it.  The waves of a workgroup put their (A, B) together in LDS; the workgroups through a word of 64 bits per tile and
// channel in memory: first the tile's (A, B), then, once the state that comes into the tile is known, the state that
// leaves it.  A workgroup looks at up to kWindow tiles before its own, takes the state that left the first of them and
// applies the (A, B) of the others in their order.  Tiles are handed out by a counter, in order, so that whoever is waited
// for is already running and, waiting only for tiles before its own, gets there.  The state that goes into a tile is the
// same chain of operations wherever the chain is picked up, so the same inputs give the same bits.
#include "values.h"

namespace dgn {

enum Kind : int { kDecay = DGN_GATE_DECAY, kSigmoid = DGN_GATE_SIGMOID };

// a and 1 - a of a gate, the latter from the exponential: 1 - sigma(g) would lose the digits of a gate that is nearly open.
template <int kKind> __device__ __forceinline__ void open_gate(float g, float &a, float &b)
{
    if (kKind == kDecay) { a = g; b = 1.0f; return; }
    const float e = __expf(-fabsf(g)), r = __builtin_amdgcn_rcpf(1.0f + e), er = e * r;
    a = g < 0.0f ? er : r;                  // (NaN: r is NaN)
    b = g < 0.0f ? r : er;
}

__device__ __forceinline__ int64_t row_bound(int64_t v, int64_t tokens) { return v < 0 ? 0 : v > tokens ? tokens : v; }

// V neighbouring elements, at an address that is aligned to one.
template <class T, int V> struct Pack {
    typedef typename T::Store S;
    typedef S Vec __attribute__((ext_vector_type(V), aligned(sizeof(S))));
    Vec v;
    __device__ __forceinline__ void load(const S *p) { v = *reinterpret_cast<const Vec *>(p); }
    __device__ __forceinline__ void store(S *p) const { *reinterpret_cast<Vec *>(p) = v; }
    __device__ __forceinline__ float get(int i) const { return (float)v[i]; }
    __device__ __forceinline__ void set(int i, float f) { v[i] = (S)f; }
};
template <class T> struct Pack<T, 1> {
    typedef typename T::Store S;
    S v;
    __device__ __forceinline__ void load(const S *p) { v = *p; }
    __device__ __forceinline__ void store(S *p) const { *p = v; }
    __device__ __forceinline__ float get(int) const { return (float)v; }
    __device__ __forceinline__ void set(int, float f) { v = (S)f; }
};

// What a run of rows does to the state that comes into it: A h + B, or B alone if `cut` (a sequence begins in it).
// In memory: B in the low half, A in the high one, all bits of which are inverted, so that a cleared word is none (an A that is
// no number is written as the usual one, and as another to say `cut`).
constexpr uint32_t kNaN = 0x7fc00000u, kCut = 0x7fc00001u;
__device__ __forceinline__ u64 link_word(float A, float B, bool cut)
{
    const uint32_t bits = cut ? kCut : A != A ? kNaN : __float_as_uint(A);
    return (u64)~bits << 32 | __float_as_uint(B);
}
__device__ __forceinline__ bool word_cuts(u64 w) { return ~(uint32_t)(w >> 32) == kCut; }
__device__ __forceinline__ float apply_word(u64 w, float h)
{
    const float A = __uint_as_float(~(uint32_t)(w >> 32)), B = __uint_as_float((uint32_t)w);
    return word_cuts(w) ? B : fmaf(A, h, B);
}

constexpr int kTokens = 8;          // rows of a thread
constexpr int kLook = 2;            // tiles that a wave looks at

// Where the sequences of a tile begin and end, for all waves of its workgroup.
template <int kRows> struct TileMarks {
    int32_t begin[kRows], end[kRows];       // the sequence whose first / last row this is, or -1
    int32_t empties;
};

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

// Marks of the tile of rows from `from` on.  Sequences in no ascending order give marks that mean nothing, inside the tile.
template <int kRows, int kThreads>
__device__ __forceinline__ void mark_tile(const ScanArgs &a, int64_t from, bool last, TileMarks<kRows> &m)
{
    for (int i = threadIdx.x; i < kRows; i += kThreads) m.begin[i] = m.end[i] = -1;
    if (threadIdx.x == 0) m.empties = 0;
    int64_t first = 0;
    if (a.seqs > 4 * kThreads) {            // (up to here all are looked at)
        first = rows_below(a.rowptr, a.seqs + 1, from) - 1;
        if (first < 0) first = 0;
    }
    __syncthreads();
    for (int64_t q = first + threadIdx.x; q < a.seqs; q += kThreads) {
        const int64_t p = row_bound(a.rowptr[q], a.tokens), e = row_bound(a.rowptr[q + 1], a.tokens);
        if (p > from + kRows && !last) break;
        if (p < e) {
            if (p >= from && p < from + kRows) m.begin[p - from] = (int32_t)q;
            if (e > from && e <= from + kRows) m.end[e - 1 - from] = (int32_t)q;
        } else if (p >= from && (p < from + kRows || last)) m.empties = 1;
    }
    __syncthreads();
}

// The sequences without rows whose place is in the tile: out = in (or zero).
template <int V, int kRows, int kWaves>
__device__ __forceinline__ void copy_empties(const ScanArgs &a, int64_t from, bool last, int64_t c, bool active,
                                             const float *in, float *out)
{
    int64_t first = 0;
    if (a.seqs > 4 * kWaves) {              // (mark_tile may have looked at all)
        first = rows_below(a.rowptr, a.seqs + 1, from) - 1;
        if (first < 0) first = 0;
    }
    for (int64_t q = first + (threadIdx.x >> 6); q < a.seqs; q += kWaves) {
        const int64_t p = row_bound(a.rowptr[q], a.tokens), e = row_bound(a.rowptr[q + 1], a.tokens);
        if (p > from + kRows && !last) break;
        if (p < e || p < from || (p >= from + kRows && !last) || !active) continue;
#pragma unroll
        for (int i = 0; i < V; i++) out[q * a.channels + c + i] = in ? in[q * a.channels + c + i] : 0.0f;
    }
}

template <int V> __device__ __forceinline__ void load_state(const float *p, int64_t at, float (&h)[V])
{
#pragma unroll
    for (int i = 0; i < V; i++) h[i] = p ? p[at + i] : 0.0f;
}

// The state that comes into this tile: out of the words of the tiles before it (`step` of the direction: -1 or +1).  All waves;
// `window`: room for a word per tile looked at, lane and element.  The result is wave 0's.
template <int V, int kWaves>
__device__ __forceinline__ void state_before(const u64 *words, int64_t row_words, int64_t tile, int64_t step, int64_t tiles,
                                             u64 *window, float (&h)[V])
{
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    constexpr int kWindow = kWaves * kLook;
#pragma unroll
    for (int l = 0; l < kLook; l++) {
        const int far = wave * kLook + l;                   // 0: the tile next to this one
        const int64_t j = tile + (far + 1) * step;
        u64 w[V];
        if (j >= 0 && j < tiles) {
            const u64 *at = words + j * row_words + lane * V;
            for (;;) {
                bool there = true;
#pragma unroll
                for (int i = 0; i < V; i++) {
                    w[i] = load_coherent(at + i);
                    // the farthest has to be a state: what is nearer can then be applied to it
                    there = there && (far == kWindow - 1 ? w[i] != 0 && word_cuts(w[i]) : w[i] != 0);
                }
                if (__all(there)) break;
                __builtin_amdgcn_s_sleep(1);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; i++) w[i] = link_word(0.0f, 0.0f, true);
        }
#pragma unroll
        for (int i = 0; i < V; i++) window[(far * V + i) * kWave + lane] = w[i];
    }
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (int i = 0; i < V; i++) h[i] = 0.0f;
#pragma unroll
        for (int far = kWindow - 1; far >= 0; far--) {
#pragma unroll
            for (int i = 0; i < V; i++) h[i] = apply_word(window[(far * V + i) * kWave + lane], h[i]);
        }
    }
}

// How the channels are cut: a workgroup takes up to 64 V of them.  Shared gates: whole heads if they fit, else a part of a head
// (then the parts' sums of a gate's gradient are added up afterwards).
struct Cut { int64_t blocks; int32_t width; int32_t parts; };
inline Cut cut_channels(int64_t channels, int64_t group, int V)
{
    const int64_t room = 64 * V;
    if (group == 1) return Cut{(channels + room - 1) / room, (int32_t)room, 1};
    if (group <= room) {
        const int64_t width = room / group * group;
        return Cut{(channels + width - 1) / width, (int32_t)width, 1};
    }
    const int64_t parts = (group + room - 1) / room;
    return Cut{channels / group * parts, (int32_t)room, (int32_t)parts};
}
// First channel of a block, how many it has, and which part of its head it is.
struct Block { int64_t c; int32_t width, part; };
__device__ __forceinline__ Block block_of(const ScanArgs &a, int64_t block)
{
    if (a.parts == 1) {
        const int64_t c = block * a.width, left = a.channels - c;
        return Block{c, (int32_t)(left < a.width ? left : a.width), 0};
    }
    const int64_t head = block / a.parts, part = block % a.parts, at = part * a.width, left = a.group - at;
    return Block{head * a.group + at, (int32_t)(left < a.width ? left : a.width), (int32_t)part};
}

// The next tile and block of channels of a workgroup.  With words in memory the counter hands them out in order.
template <bool kBack>
__device__ __forceinline__ bool take_work(const ScanArgs &a, int64_t turn, int64_t &tile, int64_t &block, int64_t *s_ticket)
{
    int64_t at = blockIdx.x + turn * gridDim.x;
    if (turn > 0) __syncthreads();                      // nobody still reads what the last tile left in LDS
    if (a.words) {
        if (threadIdx.x == 0) *s_ticket = (int64_t)atomicAdd(a.ticket, 1ull);
        __syncthreads();
        at = *s_ticket;
    }
    if (at >= a.tiles * a.blocks) return false;
    tile = at / a.blocks;
    block = at - tile * a.blocks;
    if (kBack) tile = a.tiles - 1 - tile;
    return true;
}

template <class T, int kKind, int V, bool kShared, int kWaves>
__global__ __launch_bounds__(kWaves *kWave) void k_scan_forward(ScanArgs a)
{
    typedef typename T::Store S;
    constexpr int kRows = kWaves * kTokens, kThreads = kWaves * kWave;
    __shared__ TileMarks<kRows> marks;
    __shared__ u64 s_link[kWaves * V * kWave];
    __shared__ u64 s_window[kWaves * kLook * V * kWave];
    __shared__ float s_state[kWaves * V * kWave];
    __shared__ int64_t s_ticket;
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    int64_t tile, block;
    for (int64_t turn = 0; take_work<false>(a, turn, tile, block, &s_ticket); turn++) {
        const Block bl = block_of(a, block);
        const bool active = lane * V < bl.width;
        const int64_t c = bl.c + (active ? lane * V : 0), from = tile * kRows, row0 = from + wave * kTokens;
        const bool last = tile == a.tiles - 1;
        // all of the tile's rows are asked for at once (rows past the end: the last one again)
        Pack<T, V> x[kTokens], y;
        Pack<T, kShared ? 1 : V> g[kTokens];
        if (a.tokens > 0) {
#pragma unroll
            for (int k = 0; k < kTokens; k++) {
                const int64_t t = row0 + k < a.tokens ? row0 + k : a.tokens - 1;
                x[k].load(static_cast<const S *>(a.x) + t * a.x_stride + c);
                g[k].load(static_cast<const S *>(a.gate) + t * a.gate_stride + (kShared ? c / a.group : c));
            }
        }
        mark_tile<kRows, kThreads>(a, from, last, marks);
        const int64_t low = row_bound(a.rowptr[0], a.tokens), high = row_bound(a.rowptr[a.seqs], a.tokens);
        const int mark = lane < kTokens ? marks.begin[wave * kTokens + lane] : -1;
        const int stop = lane < kTokens ? marks.end[wave * kTokens + lane] : -1;
        const uint32_t begins = (uint32_t)__ballot(mark >= 0), ends = (uint32_t)__ballot(stop >= 0);
        if (marks.empties && a.final) copy_empties<V, kRows, kWaves>(a, from, last, c, active, a.h0, a.final);

        float ga[kTokens][V], u[kTokens][V], A[V], h[V];
#pragma unroll
        for (int i = 0; i < V; i++) { A[i] = 1.0f; h[i] = 0.0f; }
#pragma unroll
        for (int k = 0; k < kTokens; k++) {
            if (begins >> k & 1) load_state<V>(a.h0, (int64_t)__builtin_amdgcn_readlane(mark, k) * a.channels + c, h);
            float b;
#pragma unroll
            for (int i = 0; i < V; i++) {
                if (!kShared || i == 0) open_gate<kKind>(g[k].get(i), ga[k][i], b);
                else ga[k][i] = ga[k][0];
                u[k][i] = kKind == kDecay ? x[k].get(i) : b * x[k].get(i);
                A[i] *= ga[k][i];
                h[i] = fmaf(ga[k][i], h[i], u[k][i]);
            }
        }
#pragma unroll
        for (int i = 0; i < V; i++) s_link[(wave * V + i) * kWave + lane] = link_word(A[i], h[i], begins != 0);
        __syncthreads();

        float in[V];                                    // (wave 0) the state that comes into the tile
#pragma unroll
        for (int i = 0; i < V; i++) in[i] = 0.0f;
        const bool closed = marks.begin[0] >= 0 || tile == 0;       // nothing comes into it
        u64 *mine = a.words ? a.words + tile * a.row_words + block * (V * kWave) + lane * V : nullptr;
        float tA[V], tB[V];
        bool cut = false;
        if (wave == 0 && a.words) {
#pragma unroll
            for (int i = 0; i < V; i++) { tA[i] = 1.0f; tB[i] = 0.0f; }
#pragma unroll
            for (int w = 0; w < kWaves; w++) {
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const u64 link = s_link[(w * V + i) * kWave + lane];
                    tB[i] = apply_word(link, tB[i]);
                    tA[i] *= __uint_as_float(~(uint32_t)(link >> 32));
                    cut = cut || word_cuts(link);
                }
            }
            cut = __any(cut);
            if (!last) {
#pragma unroll
                for (int i = 0; i < V; i++) store_coherent(mine + i, link_word(tA[i], tB[i], cut || closed));
            }
        }
        if (a.words && !closed) {
            state_before<V, kWaves>(a.words + block * (V * kWave), a.row_words, tile, -1, a.tiles, s_window, in);
            if (wave == 0 && !cut && !last) {
#pragma unroll
                for (int i = 0; i < V; i++) store_coherent(mine + i, link_word(0.0f, fmaf(tA[i], in[i], tB[i]), true));
            }
        }
        if (wave == 0) {
#pragma unroll
            for (int w = 0; w < kWaves; w++) {
#pragma unroll
                for (int i = 0; i < V; i++) {
                    s_state[(w * V + i) * kWave + lane] = in[i];
                    in[i] = apply_word(s_link[(w * V + i) * kWave + lane], in[i]);
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; i++) h[i] = s_state[(wave * V + i) * kWave + lane];
        if (a.carry && row0 % kScanTile == 0 && row0 < a.tokens && active) {
#pragma unroll
            for (int i = 0; i < V; i++) a.carry[row0 / kScanTile * a.channels + c + i] = h[i];
        }
#pragma unroll
        for (int k = 0; k < kTokens; k++) {
            if (begins >> k & 1) load_state<V>(a.h0, (int64_t)__builtin_amdgcn_readlane(mark, k) * a.channels + c, h);
#pragma unroll
            for (int i = 0; i < V; i++) {
                h[i] = fmaf(ga[k][i], h[i], u[k][i]);
                y.set(i, h[i]);
            }
            if (row0 + k >= low && row0 + k < high && active) y.store(static_cast<S *>(a.y) + (row0 + k) * a.y_stride + c);
            if ((ends >> k & 1) && a.final && active) {
                const int64_t at = (int64_t)__builtin_amdgcn_readlane(stop, k) * a.channels + c;
#pragma unroll
                for (int i = 0; i < V; i++) a.final[at + i] = h[i];
            }
        }
    }
}

// Sums of kTokens values a lane over the lanes of each head (`lanes` of them, the first head's from lane 0 on); the result for token k of
// a head is in `out[k]` of its first lane.
__device__ __forceinline__ void sum_heads(float (&v)[kTokens], int lanes, int lane)
{
    if ((lanes & (lanes - 1)) == 0) {
        for (int d = lanes >> 1; d >= 1; d >>= 1) {
#pragma unroll
            for (int k = 0; k < kTokens; k++) v[k] += __shfl_xor(v[k], d, kWave);
        }
        return;
    }
    const int at = lane % lanes;
    for (int d = 1; d < lanes; d <<= 1) {
#pragma unroll
        for (int k = 0; k < kTokens; k++) {
            const float o = __shfl_down(v[k], d, kWave);
            if (at + d < lanes && lane + d < kWave) v[k] += o;
        }
    }
}

template <class T, int kKind, int V, bool kShared, int kWaves>
__global__ __launch_bounds__(kWaves *kWave) void k_scan_backward(ScanArgs a)
{
    typedef typename T::Store S;
    constexpr int kRows = kWaves * kTokens, kThreads = kWaves * kWave;
    static_assert(kRows == kScanTile, "a state is kept for each tile of the backward pass");
    __shared__ TileMarks<kRows> marks;
    __shared__ u64 s_ahead[kWaves * V * kWave], s_back[kWaves * V * kWave];
    __shared__ u64 s_window[kWaves * kLook * V * kWave];
    __shared__ float s_state[kWaves * V * kWave], s_grad[kWaves * V * kWave];
    __shared__ int64_t s_ticket;
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    int64_t tile, block;
    for (int64_t turn = 0; take_work<true>(a, turn, tile, block, &s_ticket); turn++) {
        const Block bl = block_of(a, block);
        const bool active = lane * V < bl.width;
        const int64_t c = bl.c + (active ? lane * V : 0), from = tile * kRows, row0 = from + wave * kTokens;
        const int64_t head = kShared ? c / a.group : 0;
        const bool last = tile == a.tiles - 1;
        Pack<T, V> x[kTokens], dy[kTokens];
        Pack<T, kShared ? 1 : V> g[kTokens];
        float kept[V];
        if (a.tokens > 0) {
#pragma unroll
            for (int k = 0; k < kTokens; k++) {
                const int64_t t = row0 + k < a.tokens ? row0 + k : a.tokens - 1;
                x[k].load(static_cast<const S *>(a.x) + t * a.x_stride + c);
                g[k].load(static_cast<const S *>(a.gate) + t * a.gate_stride + (kShared ? head : c));
                dy[k].load(static_cast<const S *>(a.dy) + t * a.dy_stride + c);
            }
            if (wave == 0) load_state<V>(a.carry, tile * a.channels + c, kept);
        }
        mark_tile<kRows, kThreads>(a, from, last, marks);
        const int64_t low = row_bound(a.rowptr[0], a.tokens), high = row_bound(a.rowptr[a.seqs], a.tokens);
        const int mark = lane < kTokens ? marks.begin[wave * kTokens + lane] : -1;
        const int stop = lane < kTokens ? marks.end[wave * kTokens + lane] : -1;
        const uint32_t begins = (uint32_t)__ballot(mark >= 0), ends = (uint32_t)__ballot(stop >= 0);
        if (marks.empties && a.dh0) copy_empties<V, kRows, kWaves>(a, from, last, c, active, a.dfinal, a.dh0);

        float ga[kTokens][V], gb[kTokens][V], A[V], h[V], e[V];
#pragma unroll
        for (int i = 0; i < V; i++) { A[i] = 1.0f; h[i] = e[i] = 0.0f; }
#pragma unroll
        for (int k = 0; k < kTokens; k++) {
            if (begins >> k & 1) load_state<V>(a.h0, (int64_t)__builtin_amdgcn_readlane(mark, k) * a.channels + c, h);
#pragma unroll
            for (int i = 0; i < V; i++) {
                if (!kShared || i == 0) open_gate<kKind>(g[k].get(i), ga[k][i], gb[k][i]);
                else { ga[k][i] = ga[k][0]; gb[k][i] = gb[k][0]; }
                A[i] *= ga[k][i];
                h[i] = fmaf(ga[k][i], h[i], gb[k][i] * x[k].get(i));
            }
        }
#pragma unroll
        for (int k = kTokens - 1; k >= 0; k--) {
            if (ends >> k & 1) load_state<V>(a.dfinal, (int64_t)__builtin_amdgcn_readlane(stop, k) * a.channels + c, e);
#pragma unroll
            for (int i = 0; i < V; i++) e[i] = ga[k][i] * (e[i] + dy[k].get(i));
        }
#pragma unroll
        for (int i = 0; i < V; i++) {
            s_ahead[(wave * V + i) * kWave + lane] = link_word(A[i], h[i], begins != 0);
            s_back[(wave * V + i) * kWave + lane] = link_word(A[i], e[i], ends != 0);
        }
        __syncthreads();

        float in[V];                                    // (wave 0) what comes back into the tile
#pragma unroll
        for (int i = 0; i < V; i++) in[i] = 0.0f;
        const bool closed = marks.end[kRows - 1] >= 0 || last;
        u64 *mine = a.words ? a.words + tile * a.row_words + block * (V * kWave) + lane * V : nullptr;
        float tA[V], tB[V];
        bool cut = false;
        if (wave == 0 && a.words) {
#pragma unroll
            for (int i = 0; i < V; i++) { tA[i] = 1.0f; tB[i] = 0.0f; }
#pragma unroll
            for (int w = kWaves - 1; w >= 0; w--) {
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const u64 link = s_back[(w * V + i) * kWave + lane];
                    tB[i] = apply_word(link, tB[i]);
                    tA[i] *= __uint_as_float(~(uint32_t)(link >> 32));
                    cut = cut || word_cuts(link);
                }
            }
            cut = __any(cut);
            if (tile > 0) {
#pragma unroll
                for (int i = 0; i < V; i++) store_coherent(mine + i, link_word(tA[i], tB[i], cut || closed));
            }
        }
        if (a.words && !closed) {
            state_before<V, kWaves>(a.words + block * (V * kWave), a.row_words, tile, 1, a.tiles, s_window, in);
            if (wave == 0 && !cut && tile > 0) {
#pragma unroll
                for (int i = 0; i < V; i++) store_coherent(mine + i, link_word(0.0f, fmaf(tA[i], in[i], tB[i]), true));
            }
        }
        if (wave == 0) {
#pragma unroll
            for (int w = kWaves - 1; w >= 0; w--) {
#pragma unroll
                for (int i = 0; i < V; i++) {
                    s_grad[(w * V + i) * kWave + lane] = in[i];
                    in[i] = apply_word(s_back[(w * V + i) * kWave + lane], in[i]);
                }
            }
#pragma unroll
            for (int w = 0; w < kWaves; w++) {
#pragma unroll
                for (int i = 0; i < V; i++) {
                    s_state[(w * V + i) * kWave + lane] = kept[i];
                    kept[i] = apply_word(s_ahead[(w * V + i) * kWave + lane], kept[i]);
                }
            }
        }
        __syncthreads();
        float before[kTokens][V];
#pragma unroll
        for (int i = 0; i < V; i++) { h[i] = s_state[(wave * V + i) * kWave + lane]; e[i] = s_grad[(wave * V + i) * kWave + lane]; }
#pragma unroll
        for (int k = 0; k < kTokens; k++) {
            if (begins >> k & 1) load_state<V>(a.h0, (int64_t)__builtin_amdgcn_readlane(mark, k) * a.channels + c, h);
#pragma unroll
            for (int i = 0; i < V; i++) {
                before[k][i] = h[i];
                h[i] = fmaf(ga[k][i], h[i], gb[k][i] * x[k].get(i));
            }
        }
        float sum[kTokens];
#pragma unroll
        for (int k = kTokens - 1; k >= 0; k--) {
            if (ends >> k & 1) load_state<V>(a.dfinal, (int64_t)__builtin_amdgcn_readlane(stop, k) * a.channels + c, e);
            const bool mine_row = row0 + k >= low && row0 + k < high && active;
            Pack<T, V> dx, dg;
            sum[k] = 0.0f;
#pragma unroll
            for (int i = 0; i < V; i++) {
                e[i] += dy[k].get(i);
                dx.set(i, kKind == kDecay ? e[i] : gb[k][i] * e[i]);
                const float d = kKind == kDecay ? e[i] * before[k][i] : ga[k][i] * gb[k][i] * (e[i] * (before[k][i] - x[k].get(i)));
                if (kShared) sum[k] += d;
                else dg.set(i, d);
                e[i] *= ga[k][i];
            }
            if (mine_row) {
                dx.store(static_cast<S *>(a.dx) + (row0 + k) * a.dx_stride + c);
                if (!kShared) dg.store(static_cast<S *>(a.dgate) + (row0 + k) * a.dgate_stride + c);
            }
            if ((begins >> k & 1) && a.dh0 && active) {
                const int64_t at = (int64_t)__builtin_amdgcn_readlane(mark, k) * a.channels + c;
#pragma unroll
                for (int i = 0; i < V; i++) a.dh0[at + i] = e[i];
            }
        }
        if (kShared) {
            // (a part of a head is all lanes of its block; the lanes past its end count nothing)
            if (!active) {
#pragma unroll
                for (int k = 0; k < kTokens; k++) sum[k] = 0.0f;
            }
            const int lanes = a.parts > 1 ? kWave : (int)(a.group / V);
            sum_heads(sum, lanes, lane);
            if (active && lane % lanes == 0) {
#pragma unroll
                for (int k = 0; k < kTokens; k++) {
                    const int64_t t = row0 + k;
                    if (t < low || t >= high) continue;
                    if (a.parts > 1) a.partial[(bl.part * a.tokens + t) * a.heads + head] = sum[k];
                    else static_cast<S *>(a.dgate)[t * a.dgate_stride + head] = (S)sum[k];
                }
            }
        }
    }
}

// Gates shared by more channels than a workgroup has: the sum of the parts' sums.
template <class T>
__global__ __launch_bounds__(256) void k_gate_sums(ScanArgs a)
{
    const int64_t low = row_bound(a.rowptr[0], a.tokens), high = row_bound(a.rowptr[a.seqs], a.tokens);
    for (int64_t i = low * a.heads + blockIdx.x * 256 + threadIdx.x; i < high * a.heads; i += (int64_t)gridDim.x * 256) {
        const int64_t t = i / a.heads, head = i - t * a.heads;
        float sum = 0.0f;
        for (int p = 0; p < a.parts; p++) sum += a.partial[p * a.tokens * a.heads + i];
        static_cast<typename T::Store *>(a.dgate)[t * a.dgate_stride + head] = (typename T::Store)sum;
    }
}

template <class T, int kKind>
__global__ __launch_bounds__(256) void k_scan_step(StepArgs a)
{
    typedef typename T::Store S;
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= a.channels) return;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const int64_t slot = a.slot ? a.slot[row] : row;
    float h = 0.0f;
    if (slot >= 0 && slot < a.slots) {
        float g, b;
        open_gate<kKind>((float)(static_cast<const S *>(a.gate)[row * a.gate_stride + c / a.group]), g, b);
        h = g * a.state_in[slot * a.channels + c] + b * (float)(static_cast<const S *>(a.x)[row * a.x_stride + c]);
        a.state_out[slot * a.channels + c] = h;
    }
    static_cast<S *>(a.y)[row * a.y_stride + c] = (S)h;
    }
}

// Elements a thread takes of a row: two, where the rows and the heads have an even number.
static int elements_of(const ScanArgs &a) { return a.channels % 2 == 0 && (a.group == 1 || a.group % 2 == 0) ? 2 : 1; }

constexpr int kForwardWaves = 16, kBackwardWaves = 8;
static int64_t tiles_of(int64_t tokens, int rows) { return tokens > 0 ? (tokens + rows - 1) / rows : 1; }

// Scratch: the counter (256 bytes), a word per tile and channel of the direction with the smaller tiles, the parts' sums.
struct ScanScratch { size_t words, partial, bytes; };
static ScanScratch lay_out(const ScanArgs &a)
{
    const int V = elements_of(a);
    const Cut cut = cut_channels(a.channels, a.group, V);
    ScanScratch s;
    s.words = 256;
    s.partial = s.words + (size_t)tiles_of(a.tokens, kBackwardWaves * kTokens) * cut.blocks * V * kWave * sizeof(u64);
    s.bytes = s.partial + (cut.parts > 1 ? (size_t)cut.parts * a.tokens * a.heads * sizeof(float) : 0);
    return s;
}
size_t scan_scratch_bytes(const ScanArgs &a) { return lay_out(a).bytes; }

// Sets what the kernels need to know of the cut; clears the counter and the words where there are several tiles.
static hipError_t set_up(ScanArgs &a, int rows, void *scratch, hipStream_t s)
{
    const int V = elements_of(a);
    const Cut cut = cut_channels(a.channels, a.group, V);
    const ScanScratch l = lay_out(a);
    char *mem = static_cast<char *>(scratch);
    a.blocks = cut.blocks;
    a.width = cut.width;
    a.parts = cut.parts;
    a.tiles = tiles_of(a.tokens, rows);
    a.row_words = cut.blocks * V * kWave;
    a.partial = reinterpret_cast<float *>(mem + l.partial);
    if (a.tiles == 1) return hipSuccess;
    a.ticket = reinterpret_cast<u64 *>(mem);
    a.words = reinterpret_cast<u64 *>(mem + l.words);
    const FillRegion clear = {mem, l.words + (size_t)a.tiles * a.row_words * sizeof(u64)};
    return launch_clear(&clear, 1, s);
}

static unsigned grid_of(const ScanArgs &a)
{
    const int64_t n = a.tiles * a.blocks;
    return (unsigned)(n < (1 << 20) ? n : 1 << 20);     // (a workgroup goes on until all is handed out)
}

template <class T, int kKind> static void go_forward(const ScanArgs &a, hipStream_t s)
{
    const dim3 grid(grid_of(a)), threads(kForwardWaves * kWave);
    const int V = elements_of(a);
    if (a.group == 1) {
        if (V == 2) hipLaunchKernelGGL((k_scan_forward<T, kKind, 2, false, kForwardWaves>), grid, threads, 0, s, a);
        else hipLaunchKernelGGL((k_scan_forward<T, kKind, 1, false, kForwardWaves>), grid, threads, 0, s, a);
    } else {
        if (V == 2) hipLaunchKernelGGL((k_scan_forward<T, kKind, 2, true, kForwardWaves>), grid, threads, 0, s, a);
        else hipLaunchKernelGGL((k_scan_forward<T, kKind, 1, true, kForwardWaves>), grid, threads, 0, s, a);
    }
}
template <class T, int kKind> static void go_backward(const ScanArgs &a, hipStream_t s)
{
    const dim3 grid(grid_of(a)), threads(kBackwardWaves * kWave);
    const int V = elements_of(a);
    if (a.group == 1) {
        if (V == 2) hipLaunchKernelGGL((k_scan_backward<T, kKind, 2, false, kBackwardWaves>), grid, threads, 0, s, a);
        else hipLaunchKernelGGL((k_scan_backward<T, kKind, 1, false, kBackwardWaves>), grid, threads, 0, s, a);
    } else {
        if (V == 2) hipLaunchKernelGGL((k_scan_backward<T, kKind, 2, true, kBackwardWaves>), grid, threads, 0, s, a);
        else hipLaunchKernelGGL((k_scan_backward<T, kKind, 1, true, kBackwardWaves>), grid, threads, 0, s, a);
        if (a.parts > 1 && a.tokens > 0) {
            const int64_t n = (a.tokens * a.heads + 255) / 256;
            hipLaunchKernelGGL((k_gate_sums<T>), dim3((unsigned)(n < 8192 ? n : 8192)), dim3(256), 0, s, a);
        }
    }
}

#define DGN_BY_TYPE(call)                                                                                     \
    do {                                                                                                      \
        if (dtype == DGN_F32) { typedef F32 T; if (kind == kDecay) call(T, kDecay); else call(T, kSigmoid); } \
        else if (dtype == DGN_F16) { typedef F16 T; if (kind == kDecay) call(T, kDecay); else call(T, kSigmoid); } \
        else { typedef BF16 T; if (kind == kDecay) call(T, kDecay); else call(T, kSigmoid); }                 \
    } while (0)

hipError_t launch_scan_forward(int dtype, int kind, ScanArgs a, void *scratch, hipStream_t s)
{
    const hipError_t e = set_up(a, kForwardWaves * kTokens, scratch, s);
    if (e != hipSuccess) return e;
#define DGN_GO(T, K) go_forward<T, K>(a, s)
    DGN_BY_TYPE(DGN_GO);
#undef DGN_GO
    return hipGetLastError();
}

hipError_t launch_scan_backward(int dtype, int kind, ScanArgs a, void *scratch, hipStream_t s)
{
    const hipError_t e = set_up(a, kBackwardWaves * kTokens, scratch, s);
    if (e != hipSuccess) return e;
#define DGN_GO(T, K) go_backward<T, K>(a, s)
    DGN_BY_TYPE(DGN_GO);
#undef DGN_GO
    return hipGetLastError();
}

hipError_t launch_scan_step(int dtype, int kind, const StepArgs &a, hipStream_t s)
{
    if (a.channels == 0 || a.rows == 0) return hipSuccess;
    const dim3 grid((unsigned)((a.channels + 255) / 256), (unsigned)(a.rows < 32768 ? a.rows : 32768));
#define DGN_GO(T, K) hipLaunchKernelGGL((k_scan_step<T, K>), grid, dim3(256), 0, s, a)
    DGN_BY_TYPE(DGN_GO);
#undef DGN_GO
    return hipGetLastError();
}

}  // namespace dgn
