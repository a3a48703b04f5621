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
// The rows, whatever sequences they belong to, are cut into strips; a wave takes a strip of 64 V channels.  What a strip does to the state
// that comes into it is h -> A h + B (A the product of its gates, B its end from a state of zero), or h -> B if a sequence begins in it.
// Three launches: the strips' (A, B); the states between strips, a short scan per channel; the strips again, now with the state that comes
// into each (two launches for up to 32 strips, one for up to 8).  Nothing waits for anything within a launch, and the order of all sums
// is given by the sizes alone.  It is bound by memory: forward every element of x and gate is read twice, of gate and dy backward.
// (In one launch, that reads x and gate once, a workgroup keeps its rows in registers until the workgroups before it have handed their state
// on.  All of them then load, wait and store at the same time: 65 301 x 2 048 forward in f16 253 us, 10 000 x 1 000 43 us, training step of
// 65 537 x 1 024 500 us.)
#include "rows.h"

namespace dgn {

enum Kind : int { kDecay = DGN_GATE_DECAY, kSigmoid = DGN_GATE_SIGMOID };

// a and 1 - a of a gate, the latter from the exponential: 1 - sigma(g) would lose the digits of a gate that is nearly open.  Gates of 32 bits
// by a rounded exponential and a reciprocal with one step of Newton's (training step of 20 000 x 400: 102 us; with a division 105; with what
// 16 bits have 98).  Of 16 bits by the faster exp2 of a product, which is off by |g| 2^-24 (at most 88 of
// them, then it is 0), and an approximate reciprocal: far below what the gate itself was rounded by, |g| 2^-12 and more.
template <class T, int kKind> __device__ __forceinline__ void open_gate(float g, float &a, float &b)
{
    if (kKind == kDecay) { a = g; b = 1.0f; return; }
    constexpr bool kRounded = sizeof(typename T::Store) == 4;
    const float e = kRounded ? expf(-fabsf(g)) : __expf(-fabsf(g)), d = 1.0f + e;
    float r = __builtin_amdgcn_rcpf(d);
    if (kRounded) r = fmaf(fmaf(-d, r, 1.0f), r, r);
    const float er = e * r;
    a = g < 0.0f ? er : r;                  // (NaN: r is NaN)
    b = g < 0.0f ? r : er;
}

// What a run of rows does to the state that comes into it: A h + B, or B alone if `cut` (a sequence begins in it, or for gradients ends).
// In memory: B in the low half, A in the high one (an A that is no number as the usual one, and as another to say `cut`).
constexpr uint32_t kNaN = 0x7fc00000u, kCut = 0x7fc00001u, kWide = 0x7fc00002u;       // (kWide: see k_scan_states)
__device__ __forceinline__ u64 link_word(float A, float B, bool cut)
{
    const uint32_t bits = cut ? kCut : A != A ? kNaN : __float_as_uint(A);
    return (u64)bits << 32 | __float_as_uint(B);
}
__device__ __forceinline__ bool word_cuts(u64 w) { return (uint32_t)(w >> 32) == kCut; }
__device__ __forceinline__ float apply_word(u64 w, float h)
{
    const float A = __uint_as_float((uint32_t)(w >> 32)), B = __uint_as_float((uint32_t)w);
    return word_cuts(w) ? B : fmaf(A, h, B);
}

// How the channels are cut: a wave takes up to 64 V of them.  Shared gates: whole heads if they fit, else a part of a head
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
    const int64_t head = divide(block, a.parts), part = block - head * a.parts, at = part * a.width, left = a.group - at;
    return Block{head * a.group + at, (int32_t)(left < a.width ? left : a.width), (int32_t)part};
}

constexpr int kKeep = kScanKeep;        // rows between two states that the forward pass keeps for the backward pass
constexpr int kMostRows = 64;           // rows of a strip, at most
constexpr int kStripWaves = 4;          // waves of a workgroup; each has a strip of its own

// Where sequences begin and end in the rows of a strip, a wave's own.
struct Marks {
    int32_t begin[kMostRows], end[kMostRows];       // the sequence whose first / last row this is, or -1
};
// A lane's V states of a row that is the same for the wave (nothing: zero).
template <int V> __device__ __forceinline__ void load_state(const float *row, uint32_t mine, float (&h)[V])
{
#pragma unroll
    for (int i = 0; i < V; i++) h[i] = row ? row[mine + i] : 0.0f;
}
template <int V> __device__ __forceinline__ void store_state(float *row, uint32_t mine, const float (&h)[V])
{
#pragma unroll
    for (int i = 0; i < V; i++) row[mine + i] = h[i];
}
__device__ __forceinline__ const float *row_of(const float *p, int32_t row, const ScanArgs &a, int64_t c)
{
    return p ? p + row * a.channels + c : nullptr;
}
__device__ __forceinline__ float *row_of(float *p, int32_t row, const ScanArgs &a, int64_t c) { return p + row * a.channels + c; }

// The strip of a wave: its rows, its channels, and what marks them.
template <int V, bool kShared> struct Strip {
    int64_t row0, c, head0;     // first row, first channel, and the head that has it
    int32_t rows, from, to;     // rows of it; those from `from` on, before `to`, belong to sequences
    int32_t part, width;        // which part of a head, and the channels of the block
    int64_t strip, number;      // and the number of the block
    uint32_t mine, head;        // the lane's place in the block, and its head's (32 bits: what is the same for the wave stays in scalar registers)
    bool active, last, marked, empties;

    // false: there is no such strip.  Lanes past the block's end do what lane 0 does, and store the same values to the same places.
    __device__ __forceinline__ bool find(const ScanArgs &a, int64_t at, bool back)
    {
        if (at >= a.strips * a.blocks) return false;
        strip = divide(at, a.blocks);
        const int64_t strip_block = at - strip * a.blocks;
        const Block bl = block_of(a, strip_block);
        if (back) strip = a.strips - 1 - strip;
        number = strip_block;
        c = bl.c;
        part = bl.part;
        width = bl.width;
        active = lane_id() * V < bl.width;
        mine = active ? lane_id() * V : 0;
        head = kShared ? mine / (uint32_t)a.group : 0;
        head0 = kShared ? divide(c, a.group) : 0;
        row0 = strip * a.rows;
        last = strip == a.strips - 1;
        const int64_t left = a.tokens - row0;
        rows = (int32_t)(left < a.rows ? left : a.rows);
        const int64_t low = uniform(row_bound(a.rowptr[0], a.tokens)) - row0, high = uniform(row_bound(a.rowptr[a.seqs], a.tokens)) - row0;
        from = low < 0 ? 0 : low > rows ? rows : (int32_t)low;
        to = high < 0 ? 0 : high > rows ? rows : (int32_t)high;
        return true;
    }
    // Rows that a sequence begins or ends with.  Row pointers that do not ascend give marks that mean nothing, inside the strip.
    __device__ __forceinline__ void mark(const ScanArgs &a, Marks &m)
    {
        const int lane = lane_id();
#pragma unroll
        for (int i = 0; i < kMostRows; i += kWave) m.begin[i + lane] = m.end[i + lane] = -1;
        wave_fence();
        marked = empties = false;
        for (int64_t q0 = first_sequence(a);; q0 += kWave) {
            const int64_t q = q0 + lane;
            bool more = false;
            if (q < a.seqs) {
                const int64_t p = row_bound(a.rowptr[q], a.tokens) - row0, e = row_bound(a.rowptr[q + 1], a.tokens) - row0;
                more = p <= a.rows || last;
                if (p < e) {
                    if (p >= 0 && p < rows) { m.begin[p] = (int32_t)q; marked = true; }
                    if (e > 0 && e <= rows) { m.end[e - 1] = (int32_t)q; marked = true; }
                } else empties = empties || (p >= 0 && (p < a.rows || last));
            }
            if (!__all(more)) break;
        }
        marked = __any(marked);
        empties = __any(empties);
        wave_fence();
    }
    __device__ __forceinline__ int64_t first_sequence(const ScanArgs &a) const
    {
        if (a.seqs <= kWave) return 0;
        const int64_t q = uniform(rows_below(a.rowptr, a.seqs + 1, row0)) - 1;
        return q < 0 ? 0 : q;
    }
    // The sequences without rows whose place is in the strip: out = in (or zero).
    __device__ __forceinline__ void copy_empties(const ScanArgs &a, const float *in, float *out) const
    {
        for (int64_t q0 = first_sequence(a);; q0 += kWave) {
            const int64_t q = q0 + lane_id();
            bool more = false, mine_too = false;
            if (q < a.seqs) {
                const int64_t p = row_bound(a.rowptr[q], a.tokens) - row0, e = row_bound(a.rowptr[q + 1], a.tokens) - row0;
                more = p <= a.rows || last;
                mine_too = p >= e && p >= 0 && (p < a.rows || last);
            }
            for (u64 some = __ballot(mine_too); some; some &= some - 1) {
                const int64_t row = (q0 + __builtin_ctzll(some)) * a.channels + c;
                float h[V];
                load_state<V>(in ? in + row : nullptr, mine, h);
                store_state<V>(out + row, mine, h);
            }
            if (!__all(more)) break;
        }
    }
};

// Marks of kTokens rows from row k0 of a strip on: the sequence in lane k for row k0 + k, and a bit for each.
struct Row16 { int id; uint32_t bits; };
template <int kTokens> __device__ __forceinline__ Row16 marks_of(const int32_t *marks, bool marked, int k0)
{
    Row16 r = {-1, 0};
    if (!marked) return r;
    if (lane_id() < kTokens) r.id = marks[k0 + lane_id()];
    r.bits = (uint32_t)__ballot(r.id >= 0);
    return r;
}

// The rows of a thread in one array, from row0 on; loads go on with the last row where there are no more.
struct Rows {
    int64_t at, stride;         // elements
    int32_t left;
    __device__ __forceinline__ Rows(int64_t row0, int64_t tokens, int64_t stride_, int64_t column) : stride(stride_)
    {
        const int64_t more = tokens - 1 - row0;
        at = (more < 0 ? tokens - 1 : row0) * stride + column;
        left = more > 1 << 20 ? 1 << 20 : (int32_t)more;
    }
    __device__ __forceinline__ void next(int k) { at += k < left ? stride : 0; }
};

// Rows k0 .. k0 + 7 of a strip in two arrays.
template <class T, int V, bool kShared> struct Batch {
    typedef typename T::Store S;
    static constexpr int kTokens = 8;
    Pack<T, V> x[kTokens];
    Pack<T, kShared ? 1 : V> g[kTokens];
    __device__ __forceinline__ void load(const ScanArgs &a, const Strip<V, kShared> &st, const S *in, int64_t stride, int k0)
    {
        Rows xs(st.row0 + k0, a.tokens, stride, st.c), gs(st.row0 + k0, a.tokens, a.gate_stride, kShared ? st.head0 : st.c);
#pragma unroll
        for (int k = 0; k < kTokens; k++) {
            x[k].load(in + xs.at + st.mine);
            g[k].load(static_cast<const S *>(a.gate) + gs.at + (kShared ? st.head : st.mine));
            xs.next(k);
            gs.next(k);
        }
    }
};

// The link of a strip.  kBack: of the gradients, where (A, B) of rows 0 .. n-1 is what comes back from a row after them: A the product of
// their gates, B the sum of dy_k times the gates up to k.
template <class T, int kKind, int V, bool kShared, bool kBack>
__device__ __forceinline__ void strip_link(const ScanArgs &a, Strip<V, kShared> &st, Marks &marks, u64 (&link)[V])
{
    typedef typename T::Store S;
    constexpr int kTokens = Batch<T, V, kShared>::kTokens;
    const S *in = static_cast<const S *>(kBack ? a.dy : a.x);
    const int64_t stride = kBack ? a.dy_stride : a.x_stride;
    float A[V], h[V];
#pragma unroll
    for (int i = 0; i < V; i++) { A[i] = 1.0f; h[i] = 0.0f; }
    bool cut = false;
    Batch<T, V, kShared> now, next;
    if (st.rows > 0) now.load(a, st, in, stride, 0);
    st.mark(a, marks);                                  // (with the first rows on their way)
    for (int k0 = 0; k0 < st.rows; k0 += kTokens) {
        if (k0 + kTokens < st.rows) next.load(a, st, in, stride, k0 + kTokens);
        const Row16 at = marks_of<kTokens>(kBack ? marks.end : marks.begin, st.marked, k0);
        const auto rows = [&](auto some) {
#pragma unroll
            for (int k = 0; k < kTokens; k++) {
                if (some.value && k0 + k >= st.rows) break;
                const bool here = some.value && (at.bits >> k & 1);
                if (!kBack && here) {
                    load_state<V>(row_of(a.h0, __builtin_amdgcn_readlane(at.id, k), a, st.c), st.mine, h);
                    cut = true;
                }
                float ga, gb;
#pragma unroll
                for (int i = 0; i < V; i++) {
                    if (!kShared || i == 0) open_gate<T, kKind>(now.g[k].get(i), ga, gb);
                    A[i] *= ga;
                    h[i] = kBack ? fmaf(A[i], now.x[k].get(i), h[i]) : fmaf(ga, h[i], gb * now.x[k].get(i));
                }
                if (kBack && here) {
                    float d[V];
                    load_state<V>(row_of(a.dfinal, __builtin_amdgcn_readlane(at.id, k), a, st.c), st.mine, d);
#pragma unroll
                    for (int i = 0; i < V; i++) h[i] = fmaf(A[i], d[i], h[i]);
                    cut = true;
                    break;                              // (what comes after it is another sequence's)
                }
            }
        };
        // (most rows are in the middle of a sequence: those ask for nothing, so that the next ones can stay on their way)
        if (at.bits == 0 && k0 + kTokens <= st.rows) rows(std::false_type());
        else rows(std::true_type());
        if (kBack && cut) break;
        now = next;
    }
#pragma unroll
    for (int i = 0; i < V; i++) link[i] = link_word(A[i], h[i], cut);
}

// First launch: the links of the strips.  65 537 x 1 024 in bf16: 268 MB in 56 us, 4.8 TB/s (a copy by a thread per 16 bytes: 6.2).
template <class T, int kKind, int V, bool kShared, bool kBack>
__global__ __launch_bounds__(kStripWaves *kWave, 8) void k_scan_links(ScanArgs a)
{
    __shared__ Marks s_marks[kStripWaves];
    Marks &marks = s_marks[wave_id()];
    Strip<V, kShared> st;
    const int64_t number = (int64_t)blockIdx.x * kStripWaves + wave_id();
    if (!st.find(a, number, false)) return;
    u64 link[V];
    strip_link<T, kKind, V, kShared, kBack>(a, st, marks, link);
    u64 *out = a.words + number * (kWave * V) + lane_id() * V;
#pragma unroll
    for (int i = 0; i < V; i++) out[i] = link[i];
}

// Second launch: the state that comes into each strip, states[strip][slot].  A workgroup has kSlots slots; the strips are cut into kPieces
// pieces, each is put together, the pieces' links are applied one after the other, and each is gone through again: with its words in
// registers where they are few (kEach > 0: at most so many), so that they are asked for once and all at once: 625 strips of 1 024 slots 6.9
// instead of 8.7 us.  (With 32 of them, for 1 025 strips, 21 us instead of 11: too many registers for 1 024 threads.)
// A piece has any number of gates.  Products that only fall may reach 0; where one of the strips' is above 1, their product could pass the range
// of floats though no state does (200 decays of 2, then 200 of 1/2): it is then held as a 64-bit fraction with an exponent beside it, and
// applied in 64 bits.  (In 64 bits always: 3 us more.)
constexpr int kSlots = 16, kPieces = 64;
template <int kEach>
__global__ __launch_bounds__(kSlots *kPieces) void k_scan_states(const u64 *words, float *states, int64_t strips, int64_t slots, bool back)
{
    __shared__ u64 s_link[kPieces][kSlots];
    __shared__ double s_wide[kPieces][kSlots];
    const int64_t slot = (int64_t)blockIdx.x * kSlots + threadIdx.x % kSlots;
    const int piece = threadIdx.x / kSlots;
    const int64_t each = (strips + kPieces - 1) / kPieces, from = piece * each, to = from + each < strips ? from + each : strips;
    const auto row = [&](int64_t n) { return (back ? strips - 1 - n : n) * slots + slot; };
    u64 kept[kEach > 0 ? kEach : 1];
    float A = 1.0f, B = 0.0f;
    bool cut = false, grows = false;
    if (kEach > 0) {
#pragma unroll
        for (int k = 0; k < kEach; k++) kept[k] = from + k < to ? words[row(from + k)] : link_word(1.0f, 0.0f, false);
    }
    const auto every = [&](auto join) {
        if (kEach > 0) {
#pragma unroll
            for (int k = 0; k < kEach; k++) join(kept[k]);
        } else {
#pragma unroll 8
            for (int64_t n = from; n < to; n++) join(words[row(n)]);
        }
    };
    every([&](u64 w) {
        const float a = __uint_as_float((uint32_t)(w >> 32));
        B = apply_word(w, B);
        A *= a;
        cut = cut || word_cuts(w);
        grows = grows || !(fabsf(a) <= 1.0f);
    });
    u64 link = link_word(A, B, cut);
    if (grows && !cut) {
        double wide = 1.0;
        int exponent = 0;
        every([&](u64 w) {
            wide *= (double)__uint_as_float((uint32_t)(w >> 32));
            exponent += __builtin_amdgcn_frexp_exp(wide);
            wide = __builtin_amdgcn_frexp_mant(wide);
        });
        // (from 2^1000 on every state but 0 is past the floats, from 2^-1000 down none is left)
        s_wide[piece][threadIdx.x % kSlots] = ldexp(wide, exponent < -1000 ? -1000 : exponent > 1000 ? 1000 : exponent);
        link = (u64)kWide << 32 | (uint32_t)link;
    }
    s_link[piece][threadIdx.x % kSlots] = link;
    float h = 0.0f;
    if (__syncthreads_or(grows && !cut)) {
        for (int p = 0; p < piece; p++) {
            const u64 w = s_link[p][threadIdx.x % kSlots];
            if ((uint32_t)(w >> 32) == kWide) h = (float)fma(s_wide[p][threadIdx.x % kSlots], (double)h, (double)__uint_as_float((uint32_t)w));
            else h = apply_word(w, h);
        }
    } else {
#pragma unroll 8
        for (int p = 0; p < piece; p++) h = apply_word(s_link[p][threadIdx.x % kSlots], h);
    }
    if (kEach > 0) {
#pragma unroll
        for (int k = 0; k < kEach; k++) {
            if (from + k < to) states[row(from + k)] = h;
            h = apply_word(kept[k], h);
        }
        return;
    }
#pragma unroll 8
    for (int64_t n = from; n < to; n++) {
        const u64 w = words[row(n)];
        states[row(n)] = h;
        h = apply_word(w, h);
    }
}

// The state that comes into a strip: the second launch has left it, or (few strips) the links before it are applied here.
template <int V> __device__ __forceinline__ void state_before(const ScanArgs &a, int64_t strip, int64_t block, bool back, float (&h)[V])
{
    const int64_t slots = a.blocks * (kWave * V), at = block * (kWave * V) + lane_id() * V;
#pragma unroll
    for (int i = 0; i < V; i++) h[i] = a.states ? a.states[strip * slots + at + i] : 0.0f;
    if (a.states) return;
    const int n = (int)(back ? a.strips - 1 - strip : strip);
#pragma unroll 4
    for (int k = 0; k < n; k++) {
        const u64 *w = a.words + (back ? a.strips - 1 - k : k) * slots + at;
#pragma unroll
        for (int i = 0; i < V; i++) h[i] = apply_word(w[i], h[i]);
    }
}

// The outputs of a strip, from the state that comes into it.  kMarked: its marks are there.
template <class T, int kKind, int V, bool kShared, bool kStream, bool kMarked>
__device__ __forceinline__ void strip_outputs(const ScanArgs &a, Strip<V, kShared> &st, Marks &marks, float (&h)[V])
{
    typedef typename T::Store S;
    constexpr int kTokens = Batch<T, V, kShared>::kTokens;
    if (!kMarked && st.rows == 0) st.mark(a, marks);
    S *y = static_cast<S *>(a.y) + st.row0 * a.y_stride + st.c;
    for (int k0 = 0; k0 < st.rows; k0 += kTokens) {
        Batch<T, V, kShared> now;
        now.load(a, st, static_cast<const S *>(a.x), a.x_stride, k0);
        if (!kMarked && k0 == 0) st.mark(a, marks);     // (with the first rows on their way)
        const Row16 begin = marks_of<kTokens>(marks.begin, st.marked, k0), end = marks_of<kTokens>(marks.end, st.marked, k0);
        if (a.kept && (st.row0 + k0) % kKeep == 0) store_state<V>(a.kept + (st.row0 + k0) / kKeep * a.channels + st.c, st.mine, h);
#pragma unroll
        for (int k = 0; k < kTokens; k++) {
            if (begin.bits >> k & 1) load_state<V>(row_of(a.h0, __builtin_amdgcn_readlane(begin.id, k), a, st.c), st.mine, h);
            float ga, gb;
#pragma unroll
            for (int i = 0; i < V; i++) {
                if (!kShared || i == 0) open_gate<T, kKind>(now.g[k].get(i), ga, gb);
                h[i] = fmaf(ga, h[i], gb * now.x[k].get(i));
            }
            if (k0 + k >= st.from && k0 + k < st.to) {
                Pack<T, V> out;
                out.set(h);
                out.template store<kStream>(y + st.mine);
            }
            y += a.y_stride;
            if ((end.bits >> k & 1) && a.final) store_state<V>(row_of(a.final, __builtin_amdgcn_readlane(end.id, k), a, st.c), st.mine, h);
        }
    }
    if (st.empties && a.final) st.copy_empties(a, a.h0, a.final);
}

// Third launch, forward.  The strips from the last to the first: what the first launch read last is still in the cache, and results of calls
// larger than it go past it.  65 537 x 1 024 in bf16: 402 MB in 74 us, 5.4 TB/s.
template <class T, int kKind, int V, bool kShared, bool kStream>
__global__ __launch_bounds__(kStripWaves *kWave, 8) void k_scan_outputs(ScanArgs a)
{
    __shared__ Marks s_marks[kStripWaves];
    Marks &marks = s_marks[wave_id()];
    Strip<V, kShared> st;
    if (!st.find(a, (int64_t)blockIdx.x * kStripWaves + wave_id(), true)) return;
    float h[V];
    state_before<V>(a, st.strip, st.number, false, h);
    strip_outputs<T, kKind, V, kShared, kStream, false>(a, st, marks, h);
}

// Sums of N values a lane (of rows `row` ...) over groups of 2 d lanes, handed to write(row, sum) by one lane of each.  At each step two lanes
// share out the values that are left: 17 exchanges for 16 values over 64 lanes, not 96.
template <int N, class F> __device__ __forceinline__ void sum_lanes(const float (&v)[N], int d, int row, bool writes, F write)
{
    if (d == 0) {
#pragma unroll
        for (int k = 0; k < N; k++) if (writes) write(row + k, v[k]);
        return;
    }
    const bool upper = lane_id() & d;
    if constexpr (N == 1) {
        const float both[1] = {v[0] + __shfl_xor(v[0], d, kWave)};
        sum_lanes<1>(both, d >> 1, row, writes && !upper, write);
    } else {
        float half[N / 2];
#pragma unroll
        for (int k = 0; k < N / 2; k++) half[k] = (upper ? v[k + N / 2] : v[k]) + __shfl_xor(upper ? v[k] : v[k + N / 2], d, kWave);
        sum_lanes<N / 2>(half, d >> 1, upper ? row + N / 2 : row, writes, write);
    }
}
// The same over groups of any number of lanes, the first from lane 0 on.
template <int N, class F> __device__ __forceinline__ void sum_any_lanes(float (&v)[N], int lanes, bool writes, F write)
{
    const int at = lane_id() % lanes;
    for (int d = 1; d < lanes; d <<= 1) {
#pragma unroll
        for (int k = 0; k < N; k++) {
            const float o = __shfl_down(v[k], d, kWave);
            if (at + d < lanes && lane_id() + d < kWave) v[k] += o;
        }
    }
#pragma unroll
    for (int k = 0; k < N; k++) if (writes && at == 0) write(k, v[k]);
}

// The gradients of a strip, from what comes back into it.  kKeep rows at a time, the last first: the states before each of them from the
// one that is kept, then the gradients.  sums: room for a wave's [kKeep][kWave] (shared gates).
template <class T, int kKind, int V, bool kShared, bool kStream>
__device__ __forceinline__ void strip_gradients(const ScanArgs &a, const Strip<V, kShared> &st, const Marks &marks, float *sums, float (&e)[V])
{
    typedef typename T::Store S;
    constexpr int kTokens = kKeep;
    if (st.empties && a.dh0) st.copy_empties(a, a.dfinal, a.dh0);
    for (int k0 = (st.rows - 1) / kTokens * kTokens; k0 >= 0 && st.rows > 0; k0 -= kTokens) {
        Pack<T, V> x[kTokens], dy[kTokens];
        Pack<T, kShared ? 1 : V> g[kTokens];
        const int64_t row0 = st.row0 + k0;
        Rows xs(row0, a.tokens, a.x_stride, st.c), gs(row0, a.tokens, a.gate_stride, kShared ? st.head0 : st.c),
            ys(row0, a.tokens, a.dy_stride, st.c);
#pragma unroll
        for (int k = 0; k < kTokens; k++) {
            x[k].load(static_cast<const S *>(a.x) + xs.at + st.mine);
            g[k].load(static_cast<const S *>(a.gate) + gs.at + (kShared ? st.head : st.mine));
            dy[k].load(static_cast<const S *>(a.dy) + ys.at + st.mine);
            xs.next(k);
            gs.next(k);
            ys.next(k);
        }
        float h[V];
        load_state<V>(a.kept + row0 / kKeep * a.channels + st.c, st.mine, h);
        const Row16 begin = marks_of<kTokens>(marks.begin, st.marked, k0), end = marks_of<kTokens>(marks.end, st.marked, k0);
        float before[kTokens][V], sum[kTokens];
#pragma unroll
        for (int k = 0; k < kTokens; k++) {
            if (begin.bits >> k & 1) load_state<V>(row_of(a.h0, __builtin_amdgcn_readlane(begin.id, k), a, st.c), st.mine, h);
            float ga, gb;
#pragma unroll
            for (int i = 0; i < V; i++) {
                if (!kShared || i == 0) open_gate<T, kKind>(g[k].get(i), ga, gb);
                before[k][i] = h[i];
                h[i] = fmaf(ga, h[i], gb * x[k].get(i));
            }
        }
        // (the gates are computed again: kept, they would take as many registers as the states)
#pragma unroll
        for (int k = 0; k < kTokens; k++) g[k].forget();
        S *px = static_cast<S *>(a.dx) + (row0 + kTokens - 1) * a.dx_stride + st.c,
          *pg = static_cast<S *>(a.dgate) + (row0 + kTokens - 1) * a.dgate_stride + st.c;
#pragma unroll
        for (int k = kTokens - 1; k >= 0; k--) {
            sum[k] = 0.0f;
            if (k0 + k < st.rows) {
                if (end.bits >> k & 1) load_state<V>(row_of(a.dfinal, __builtin_amdgcn_readlane(end.id, k), a, st.c), st.mine, e);
                float dx[V], dg[V], ga, gb;
#pragma unroll
                for (int i = 0; i < V; i++) {
                    if (!kShared || i == 0) open_gate<T, kKind>(g[k].get(i), ga, gb);
                    e[i] += dy[k].get(i);
                    dx[i] = kKind == kDecay ? e[i] : gb * e[i];
                    dg[i] = kKind == kDecay ? e[i] * before[k][i] : ga * gb * (e[i] * (before[k][i] - x[k].get(i)));
                    if (kShared) sum[k] += dg[i];
                    e[i] *= ga;
                }
                if (k0 + k >= st.from && k0 + k < st.to) {
                    Pack<T, V> out;
                    out.set(dx);
                    out.template store<kStream>(px + st.mine);
                    if (!kShared) {
                        out.set(dg);
                        out.template store<kStream>(pg + st.mine);
                    }
                }
                if ((begin.bits >> k & 1) && a.dh0) store_state<V>(row_of(a.dh0, __builtin_amdgcn_readlane(begin.id, k), a, st.c), st.mine, e);
            }
            px -= a.dx_stride;
            pg -= a.dgate_stride;
        }
        if (kShared) {
            // (a part of a head is all lanes of its block, and has one place; the lanes past its end count nothing)
            if (!st.active) {
#pragma unroll
                for (int k = 0; k < kTokens; k++) sum[k] = 0.0f;
            }
            const int lanes = a.parts > 1 ? kWave : (int)(a.group / V);
            const auto write = [&](int k, float v) { sums[k * kWave + st.head] = v; };     // [row][head of the block]
            const bool writes = st.active || a.parts > 1;
            if ((lanes & (lanes - 1)) == 0) sum_lanes<kTokens>(sum, lanes >> 1, 0, writes, write);
            else sum_any_lanes<kTokens>(sum, lanes, writes, write);
            wave_fence();
            const int heads = a.parts > 1 ? 1 : (int)(st.width / (int32_t)a.group);
            for (int i = lane_id(); i < kTokens * heads; i += kWave) {
                const int k = i / heads, head = i - k * heads;
                if (k0 + k < st.from || k0 + k >= st.to) continue;
                const float v = sums[k * kWave + head];
                if (a.parts > 1) a.partial[(st.part * a.tokens + row0 + k) * a.heads + st.head0] = v;
                else static_cast<S *>(a.dgate)[(row0 + k) * a.dgate_stride + st.head0 + head] = (S)v;
            }
            wave_fence();
        }
    }
}

// Third launch, backward: 65 537 x 1 024 in bf16, 688 MB in 141 us, 4.9 TB/s.  Four waves to a SIMD: with five or six, and registers spilled,
// the training step took 409 and 474 us instead of 335.
template <class T, int kKind, int V, bool kShared, bool kStream>
__global__ __launch_bounds__(kStripWaves *kWave, 4) void k_scan_gradients(ScanArgs a)
{
    __shared__ Marks s_marks[kStripWaves];
    __shared__ float s_sums[kShared ? kStripWaves : 1][kShared ? kKeep * kWave : 1];
    Marks &marks = s_marks[wave_id()];
    Strip<V, kShared> st;
    if (!st.find(a, (int64_t)blockIdx.x * kStripWaves + wave_id(), true)) return;
    float e[V];
    state_before<V>(a, st.strip, st.number, true, e);
    st.mark(a, marks);
    strip_gradients<T, kKind, V, kShared, kStream>(a, st, marks, s_sums[kShared ? wave_id() : 0], e);
}

// Short calls in one launch: a workgroup has all strips of its channels, a wave to a strip, and the links stay in LDS.  (16 x 512 forward 6.6
// us, in two launches 9.8; 128 rows 9.3 and 11.3.  With 16 waves, 256 rows, 13.0 and 12.3: one compute unit does then what many could.)
constexpr int kShortWaves = 8;
template <class T, int kKind, int V, bool kShared, bool kBack>
__global__ __launch_bounds__(kShortWaves *kWave) void k_scan_short(ScanArgs a)
{
    __shared__ Marks s_marks[kShortWaves];
    __shared__ u64 s_link[kShortWaves][V][kWave];
    __shared__ float s_sums[kShared && kBack ? kShortWaves : 1][kShared && kBack ? kKeep * kWave : 1];
    const int wave = wave_id(), lane = lane_id(), strips = (int)a.strips;
    Marks &marks = s_marks[wave];
    Strip<V, kShared> st;
    st.find(a, wave * a.blocks + blockIdx.x, false);        // (as many waves as strips)
    if (strips == 1) st.mark(a, marks);
    else {
        u64 link[V];
        strip_link<T, kKind, V, kShared, kBack>(a, st, marks, link);
#pragma unroll
        for (int i = 0; i < V; i++) s_link[wave][i][lane] = link[i];
        __syncthreads();
    }
    float h[V];
#pragma unroll
    for (int i = 0; i < V; i++) h[i] = 0.0f;
    const int before = kBack ? strips - 1 - wave : wave;
    for (int n = 0; n < before; n++) {
#pragma unroll
        for (int i = 0; i < V; i++) h[i] = apply_word(s_link[kBack ? strips - 1 - n : n][i][lane], h[i]);
    }
    if constexpr (kBack) strip_gradients<T, kKind, V, kShared, false>(a, st, marks, s_sums[kShared ? wave : 0], h);
    else strip_outputs<T, kKind, V, kShared, false, true>(a, st, marks, h);
}

// Gates shared by more channels than a wave has: the sum of the parts' sums.
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

// A copy of the states that come in, for calls whose states go out to the same memory: strips read and write them in any order.
__global__ __launch_bounds__(256) void k_copy_states(const float *from, float *to, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) to[i] = from[i];
}

// One token: a row of the batch is cut into pieces of 256 V channels, a workgroup each.  Bound by memory, and for few rows by the launch: 4 096
// rows of 2 048 channels 18.5 us, 5.3 TB/s, with four channels a thread; 32.8 us with one.
template <class T, int kKind, int V, bool kShared>
__global__ __launch_bounds__(256) void k_scan_step(StepArgs a)
{
    typedef typename T::Store S;
    for (int64_t at = blockIdx.x; at < a.rows * a.pieces; at += gridDim.x) {
        const int64_t row = divide(at, a.pieces), c = (at - row * a.pieces) * (256 * V) + threadIdx.x * V;
        if (c >= a.channels) continue;
        const int64_t slot = a.slot ? a.slot[row] : row;
        Pack<T, V> x, y;
        Pack<T, kShared ? 1 : V> g;
        x.load(static_cast<const S *>(a.x) + row * a.x_stride + c);
        g.load(static_cast<const S *>(a.gate) + row * a.gate_stride + (kShared ? c / a.group : c));
        float h[V];
#pragma unroll
        for (int i = 0; i < V; i++) h[i] = 0.0f;
        if (slot >= 0 && slot < a.slots) {
            Pack<F32, V> state;
            state.load(a.state_in + slot * a.channels + c);
            float ga, gb;
#pragma unroll
            for (int i = 0; i < V; i++) {
                if (!kShared || i == 0) open_gate<T, kKind>(g.get(i), ga, gb);
                h[i] = fmaf(ga, state.get(i), gb * x.get(i));
            }
            state.set(h);
            state.store(a.state_out + slot * a.channels + c);
        }
        y.set(h);
        y.store(static_cast<S *>(a.y) + row * a.y_stride + c);
    }
}

// Elements a thread takes of a row: four bytes of them, as the rows' and the heads' numbers allow.  (Eight bytes forward: 10 000 x 1 000
// 32.5 instead of 30.6 us, 257 x 512 14.6 instead of 12.2, with half as many waves to ask for rows.)
static int elements_of(int dtype, const ScanArgs &a)
{
    const int64_t unit = a.group == 1 ? a.channels : a.group;      // (heads that are cut into parts are cut at multiples of V)
    return dtype != DGN_F32 && unit % 2 == 0 ? 2 : 1;
}

// Rows of a strip: as few as give kStrips strips, which is what the card has waves for, and at least so many that a channel has no
// more strips than the second launch keeps in registers -- from kKeep to kMostRows.
constexpr int64_t kStrips = 8192, kChannelStrips = 1024;
// Up to so many strips each applies the links before it itself, without the launch between: 512 x 512 forward (32 strips) 12.9 us, with it
// 14.0; 768 x 512 (48) 14.4 and 14.0.
constexpr int64_t kFewStrips = 32;
struct Layout { int V; Cut cut; int64_t rows, strips; size_t words, states, partial, before, bytes; };
static Layout lay_out(int dtype, const ScanArgs &a)
{
    Layout l;
    l.V = elements_of(dtype, a);
    l.cut = cut_channels(a.channels, a.group, l.V);
    const int64_t want = a.tokens * l.cut.blocks / kStrips, least = (a.tokens + kChannelStrips - 1) / kChannelStrips;
    l.rows = want / kKeep * kKeep > least ? want / kKeep * kKeep : (least + kKeep - 1) / kKeep * kKeep;
    l.rows = l.rows < kKeep ? kKeep : l.rows > kMostRows ? kMostRows : l.rows;
    l.strips = a.tokens > 0 ? (a.tokens + l.rows - 1) / l.rows : 1;
    const size_t slots = (size_t)l.strips * l.cut.blocks * l.V * kWave;
    l.words = 0;
    l.states = l.words + slots * sizeof(u64);
    l.partial = l.states + slots * sizeof(float);
    l.before = l.partial + (l.cut.parts > 1 ? (size_t)l.cut.parts * a.tokens * a.heads * sizeof(float) : 0);
    l.bytes = l.before + (size_t)a.seqs * a.channels * sizeof(float);
    return l;
}
bool scan_fits(int dtype, const ScanArgs &a)        // launches of less than 2^32 threads
{
    const Layout l = lay_out(dtype, a);
    return l.strips * l.cut.blocks < ((int64_t)1 << 26) - kStripWaves && l.cut.blocks * l.V * kWave < ((int64_t)1 << 25);
}
size_t scan_scratch_bytes(int dtype, const ScanArgs &a) { return lay_out(dtype, a).bytes; }

static dim3 grid_of(const ScanArgs &a) { return dim3((unsigned)((a.strips * a.blocks + kStripWaves - 1) / kStripWaves)); }
static void scan_states(const ScanArgs &a, int V, bool back, hipStream_t s)
{
    const int64_t slots = a.blocks * V * kWave;
    const dim3 grid((unsigned)(slots / kSlots)), threads(kSlots * kPieces);
    if (a.strips <= 8 * kPieces) hipLaunchKernelGGL(k_scan_states<8>, grid, threads, 0, s, a.words, a.states, a.strips, slots, back);
    else if (a.strips <= 16 * kPieces) hipLaunchKernelGGL(k_scan_states<16>, grid, threads, 0, s, a.words, a.states, a.strips, slots, back);
    else hipLaunchKernelGGL(k_scan_states<0>, grid, threads, 0, s, a.words, a.states, a.strips, slots, back);
}
template <class T> static void gate_sums(const ScanArgs &a, hipStream_t s)
{
    if (a.parts == 1 || a.tokens == 0) return;
    const int64_t n = (a.tokens * a.heads + 255) / 256;
    hipLaunchKernelGGL((k_gate_sums<T>), dim3((unsigned)(n < 8192 ? n : 8192)), dim3(256), 0, s, a);
}
template <class T, int kKind, int V, bool kShared> static void go_forward(const ScanArgs &a, hipStream_t s)
{
    if (a.strips <= kShortWaves) {
        hipLaunchKernelGGL((k_scan_short<T, kKind, V, kShared, false>), dim3((unsigned)a.blocks), dim3((unsigned)a.strips * kWave), 0, s, a);
        return;
    }
    hipLaunchKernelGGL((k_scan_links<T, kKind, V, kShared, false>), grid_of(a), dim3(kStripWaves * kWave), 0, s, a);
    if (a.states) scan_states(a, V, false, s);
    // x, gate and y; x, gate, dy, dx and dgate (of the backward pass)
    if (a.tokens * (2 * a.channels + a.heads) * sizeof(typename T::Store) > kStreamBytes)
        hipLaunchKernelGGL((k_scan_outputs<T, kKind, V, kShared, true>), grid_of(a), dim3(kStripWaves * kWave), 0, s, a);
    else hipLaunchKernelGGL((k_scan_outputs<T, kKind, V, kShared, false>), grid_of(a), dim3(kStripWaves * kWave), 0, s, a);
}
template <class T, int kKind, int V, bool kShared> static void go_backward(const ScanArgs &a, hipStream_t s)
{
    if (a.strips <= kShortWaves) {
        hipLaunchKernelGGL((k_scan_short<T, kKind, V, kShared, true>), dim3((unsigned)a.blocks), dim3((unsigned)a.strips * kWave), 0, s, a);
        gate_sums<T>(a, s);
        return;
    }
    hipLaunchKernelGGL((k_scan_links<T, kKind, V, kShared, true>), grid_of(a), dim3(kStripWaves * kWave), 0, s, a);
    if (a.states) scan_states(a, V, true, s);
    if (a.tokens * (3 * a.channels + 2 * a.heads) * sizeof(typename T::Store) > kStreamBytes)
        hipLaunchKernelGGL((k_scan_gradients<T, kKind, V, kShared, true>), grid_of(a), dim3(kStripWaves * kWave), 0, s, a);
    else hipLaunchKernelGGL((k_scan_gradients<T, kKind, V, kShared, false>), grid_of(a), dim3(kStripWaves * kWave), 0, s, a);
    gate_sums<T>(a, s);
}
template <class T, int kKind, int V, bool kShared> static void go_scan(bool back, const ScanArgs &a, hipStream_t s)
{
    if (back) go_backward<T, kKind, V, kShared>(a, s);
    else go_forward<T, kKind, V, kShared>(a, s);
}
template <class T, int kKind> static hipError_t go(int dtype, bool back, ScanArgs a, void *scratch, hipStream_t s)
{
    const Layout l = lay_out(dtype, a);
    char *mem = static_cast<char *>(scratch);
    a.blocks = l.cut.blocks;
    a.width = l.cut.width;
    a.parts = l.cut.parts;
    a.rows = l.rows;
    a.strips = l.strips;
    a.partial = reinterpret_cast<float *>(mem + l.partial);
    a.words = reinterpret_cast<u64 *>(mem + l.words);
    if (a.strips > kFewStrips) a.states = reinterpret_cast<float *>(mem + l.states);
    const float *&in = back ? a.dfinal : a.h0;
    const float *out = back ? a.dh0 : a.final;
    const int64_t n = a.seqs * a.channels;
    if (in && out && in < out + n && out < in + n) {
        float *copy = reinterpret_cast<float *>(mem + l.before);
        const int64_t groups = (n + 255) / 256;
        hipLaunchKernelGGL(k_copy_states, dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(256), 0, s, in, copy, n);
        in = copy;
    }
    constexpr int kMost = sizeof(typename T::Store) == 4 ? 1 : 2;
    if (a.group == 1) {
        if (l.V == 1) go_scan<T, kKind, 1, false>(back, a, s);
        else go_scan<T, kKind, kMost, false>(back, a, s);
    } else {
        if (l.V == 1) go_scan<T, kKind, 1, true>(back, a, s);
        else go_scan<T, kKind, kMost, true>(back, a, s);
    }
    return hipGetLastError();
}

#define DGN_BY_KIND(T)                     \
    if (kind == kDecay) DGN_GO(T, kDecay); \
    else DGN_GO(T, kSigmoid)

hipError_t launch_scan(int dtype, int kind, bool back, const ScanArgs &a, void *scratch, hipStream_t s)
{
#define DGN_GO(T, K) return go<T, K>(dtype, back, a, scratch, s)
    DGN_BY_DTYPE(dtype, DGN_BY_KIND);
#undef DGN_GO
}

template <class T, int kKind> static void go_step(StepArgs a, hipStream_t s)
{
    const int V = (a.group == 1 ? a.channels : a.group) % 4 == 0 ? 4 : 1;
    a.pieces = (a.channels + 256 * V - 1) / (256 * V);
    const int64_t n = a.rows * a.pieces;
    const dim3 grid((unsigned)(n < (1 << 22) ? n : 1 << 22));
    if (a.group == 1) {
        if (V == 4) hipLaunchKernelGGL((k_scan_step<T, kKind, 4, false>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((k_scan_step<T, kKind, 1, false>), grid, dim3(256), 0, s, a);
    } else {
        if (V == 4) hipLaunchKernelGGL((k_scan_step<T, kKind, 4, true>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((k_scan_step<T, kKind, 1, true>), grid, dim3(256), 0, s, a);
    }
}
hipError_t launch_scan_step(int dtype, int kind, const StepArgs &a, hipStream_t s)
{
#define DGN_GO(T, K) go_step<T, K>(a, s)
    DGN_BY_DTYPE(dtype, DGN_BY_KIND);
#undef DGN_GO
    return hipGetLastError();
}

}  // namespace dgn
