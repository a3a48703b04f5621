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

#include <type_traits>

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

__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

typedef uint32_t Word __attribute__((aligned(2)));
typedef uint32_t Pair __attribute__((ext_vector_type(2), aligned(2)));

// V neighbouring elements, at an address that is aligned to one, as they are in memory.
template <class T, int V> struct Pack {
    typedef typename T::Store S;
    static constexpr int kBytes = V * (int)sizeof(S), kWords = kBytes < 4 ? 1 : kBytes / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const S *p)
    {
        if (kBytes == 2) w[0] = *reinterpret_cast<const uint16_t *>(p);
        else if (kBytes == 4) w[0] = *reinterpret_cast<const Word *>(p);
        else { const Pair v = *reinterpret_cast<const Pair *>(p); w[0] = v[0]; w[kWords - 1] = v[1]; }
    }
    __device__ __forceinline__ void store(S *p) const
    {
        if (kBytes == 2) *reinterpret_cast<uint16_t *>(p) = (uint16_t)w[0];
        else if (kBytes == 4) *reinterpret_cast<Word *>(p) = w[0];
        else *reinterpret_cast<Pair *>(p) = Pair{w[0], w[kWords - 1]};
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

// Before row k of a thread: what earlier rows, or an earlier pass, made of these values is not kept, and what follows is not begun
// before.  Left to itself the compiler has the gates of all rows in registers at once.
template <class... P> __device__ __forceinline__ void step(int k, P &...p)
{
    if (k % 4 == 0) __builtin_amdgcn_sched_barrier(0);
    (p.forget(), ...);
}

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

// Waves of a workgroup, rows of a thread and waves that are to fit a SIMD, for elements of 2 and of 4 bytes.
template <class T> struct Shape {
    static constexpr bool kWide = sizeof(typename T::Store) == 4;
    static constexpr int kForwardWaves = kWide ? 16 : 8, kForwardRows = kWide ? 8 : 16, kForwardResident = 4;
    static constexpr int kBackwardWaves = 8, kBackwardRows = 8, kBackwardResident = kWide ? 4 : 4;
};
constexpr int kForwardTile = 128, kBackwardTile = kScanTile;
constexpr int kGroup = 8;           // tiles of a group, and groups that are looked at

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

template <int kRows, int kThreads> __device__ __forceinline__ void clear_marks(TileMarks<kRows> &m)
{
    for (int i = threadIdx.x; i < kRows; i += kThreads) m.begin[i] = m.end[i] = -1;
    if (threadIdx.x == 0) m.empties = 0;
}

// Sequence q, of rows p .. e - 1, on the marks of the tile of rows from `from` on.  What lies past the last tile is the last tile's.
template <int kRows> __device__ __forceinline__ void mark_sequence(TileMarks<kRows> &m, int32_t q, int32_t p, int32_t e, int32_t from, bool last)
{
    const int32_t at = p - from, past = e - from;
    if (p < e) {
        if (at >= 0 && at < kRows) m.begin[at] = q;
        if (past > 0 && past <= kRows) m.end[past - 1] = q;
    } else if (at >= 0 && (at < kRows || last)) m.empties = 1;
}

template <int kRows> __device__ __forceinline__ bool any_mark(const int32_t *marks)
{
    bool some = false;
    for (int i = lane_id(); i < kRows; i += kWave) some = some || marks[i] >= 0;
    return __any(some);
}

// The sequences of a batch: up to a thread each they are in registers, the rest is looked up for each tile.  Row pointers that do
// not ascend give marks that mean nothing, inside the tile.
template <int kRows, int kThreads> struct Sequences {
    int32_t low, high, p, e;
    __device__ __forceinline__ void load(const ScanArgs &a)
    {
        low = (int32_t)row_bound(a.rowptr[0], a.tokens);
        high = (int32_t)row_bound(a.rowptr[a.seqs], a.tokens);
        p = e = -1 - kRows;                                 // (on no tile)
        if (a.seqs <= kThreads && (int)threadIdx.x < a.seqs) {
            p = (int32_t)row_bound(a.rowptr[threadIdx.x], a.tokens);
            e = (int32_t)row_bound(a.rowptr[threadIdx.x + 1], a.tokens);
        }
    }
    __device__ __forceinline__ void mark(const ScanArgs &a, int64_t from, bool last, TileMarks<kRows> &m) const
    {
        if (a.seqs <= kThreads) {
            mark_sequence(m, threadIdx.x, p, e, (int32_t)from, last);
            return;
        }
        int64_t q = rows_below(a.rowptr, a.seqs + 1, from) - 1;
        for (q = (q < 0 ? 0 : q) + threadIdx.x; q < a.seqs; q += kThreads) {
            const int64_t b = row_bound(a.rowptr[q], a.tokens);
            if (b > from + kRows && !last) break;
            mark_sequence(m, (int32_t)q, (int32_t)b, (int32_t)row_bound(a.rowptr[q + 1], a.tokens), (int32_t)from, last);
        }
    }
    // Bit k: row row0 + k belongs to some sequence.
    template <int kTokens> __device__ __forceinline__ uint32_t rows_in_use(int64_t row0) const
    {
        const int64_t l = low - row0, h = high - row0;
        const int from = l < 0 ? 0 : l > kTokens ? kTokens : (int)l, to = h < 0 ? 0 : h > kTokens ? kTokens : (int)h;
        return __builtin_amdgcn_readfirstlane(((1u << to) - 1) & ~((1u << from) - 1));
    }
};

// The sequences without rows whose place is in the tile: out = in (or zero).
template <int V, int kRows, int kWaves>
__device__ __forceinline__ void copy_empties(const ScanArgs &a, int64_t from, bool last, int64_t c, uint32_t mine, bool active, const float *in, float *out)
{
    int64_t q = 0;
    if (a.seqs > 4 * kWaves) {
        q = rows_below(a.rowptr, a.seqs + 1, from) - 1;
        if (q < 0) q = 0;
    }
    for (q += wave_id(); q < a.seqs; q += kWaves) {
        const int64_t p = row_bound(a.rowptr[q], a.tokens), e = row_bound(a.rowptr[q + 1], a.tokens);
        if (p > from + kRows && !last) break;
        if (p < e || p < from || (p >= from + kRows && !last) || !active) continue;
#pragma unroll
        for (int i = 0; i < V; i++) out[q * a.channels + c + mine + i] = in ? in[q * a.channels + c + mine + i] : 0.0f;
    }
}

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

// The links of the waves of a workgroup, or the words of the tiles it looks at: [row][lane][V].
template <int V> struct Words {
    static __device__ __forceinline__ void put(u64 *at, int row, int lane, const u64 (&w)[V])
    {
#pragma unroll
        for (int i = 0; i < V; i++) at[(row * kWave + lane) * V + i] = w[i];
    }
    static __device__ __forceinline__ void apply(const u64 *at, int row, int lane, float (&h)[V])
    {
        u64 w[V];
#pragma unroll
        for (int i = 0; i < V; i++) w[i] = at[(row * kWave + lane) * V + i];
#pragma unroll
        for (int i = 0; i < V; i++) h[i] = apply_word(w[i], h[i]);
    }
};

template <int V> __device__ __forceinline__ void publish(u64 *at, const float (&A)[V], const float (&B)[V], bool cut)
{
#pragma unroll
    for (int i = 0; i < V; i++) store_coherent(at + i, link_word(A[i], B[i], cut));
}

// Rows [from, to) of links put together, in that order, after (A, B, cut); `step`: from one to the next.
template <int V>
__device__ __forceinline__ void join_links(const u64 *links, int from, int step, int n, int lane, float (&A)[V], float (&B)[V], bool &cut)
{
    bool some = false;
#pragma unroll 4
    for (int r = 0; r < n; r++) {
#pragma unroll
        for (int i = 0; i < V; i++) {
            const u64 w = links[((from + r * step) * kWave + lane) * V + i];
            B[i] = apply_word(w, B[i]);
            A[i] *= __uint_as_float(~(uint32_t)(w >> 32));
            some = some || word_cuts(w);
        }
    }
    cut = cut || __any(some);
}

// The word at `at` for each element, once it is there (`state`: once it is a state); without one, no state.
template <int V> __device__ __forceinline__ void wait_for(const u64 *at, bool some, bool state, u64 (&w)[V])
{
#pragma unroll
    for (int i = 0; i < V; i++) w[i] = link_word(0.0f, 0.0f, true);
    while (some) {
        bool there = true;
#pragma unroll
        for (int i = 0; i < V; i++) {
            w[i] = load_coherent(at + i);
            there = there && w[i] != 0 && (!state || word_cuts(w[i]));
        }
        if (__all(there)) break;
        __builtin_amdgcn_s_sleep(1);
    }
}

// The state that comes into a tile, for all waves of its workgroup.  The tiles are a chain, in the order of the direction, `turn` the
// place in it; kGroup of them are a group.  In memory each tile leaves its link, and the last tile of a group the group's: first what
// the group does to a state, then the state that leaves it.  A tile takes the state that left the group before its own (from the nearest
// of the kGroup groups before it that has one, through the links of those between), and through the links of its group's tiles.  Which
// of them were there as states makes no difference to the bits: a group's state is always its link applied to the state before it.
//   links: the waves' (rows in the order of the chain: first + n * step); cut: a sequence begins in the tile; closed: with its first row
template <int V, int kWaves>
__device__ __forceinline__ void chain_state(const ScanArgs &a, int64_t block, int64_t turn, bool cut, bool closed, const u64 *links, int first,
                                            int step, u64 *window, float *s_state, float (&in)[V])
{
    static_assert(kWaves >= kGroup, "a wave looks at one tile and one group");
    const int lane = lane_id(), wave = wave_id(), place = (int)(turn & (kGroup - 1));
    const int64_t group = turn / kGroup;
    const bool last = turn == a.tiles - 1, ends_group = place == kGroup - 1 && !last;
    u64 *tiles = a.words + block * (V * kWave) + lane * V, *groups = tiles + a.tiles * a.row_words;
    float A[V], B[V];
#pragma unroll
    for (int i = 0; i < V; i++) { A[i] = 1.0f; B[i] = in[i] = 0.0f; }
    if (wave == 0) {
        __builtin_amdgcn_s_setprio(3);
        bool unused = false;
        join_links<V>(links, first, step, kWaves, lane, A, B, unused);
        if (place < kGroup - 1 && !last) publish<V>(tiles + turn * a.row_words, A, B, cut || closed);
        if (ends_group && (cut || closed)) publish<V>(groups + group * a.row_words, A, B, true);
        __builtin_amdgcn_s_setprio(0);
    }
    if (closed) return;
    u64 w[V];
    if (wave < kGroup) {
        wait_for<V>(tiles + (turn - place + wave) * a.row_words, wave < place, false, w);
        Words<V>::put(window, wave, lane, w);
    }
    bool group_cut = cut;
    if (ends_group && !cut) {
        __syncthreads();
        if (wave == 0) {
            __builtin_amdgcn_s_setprio(3);
            float tA[V], tB[V];
#pragma unroll
            for (int i = 0; i < V; i++) { tA[i] = A[i]; tB[i] = B[i]; A[i] = 1.0f; B[i] = 0.0f; }
            join_links<V>(window, 0, 1, kGroup - 1, lane, A, B, group_cut);
#pragma unroll
            for (int i = 0; i < V; i++) { B[i] = fmaf(tA[i], B[i], tB[i]); A[i] *= tA[i]; }
            publish<V>(groups + group * a.row_words, A, B, group_cut);
            __builtin_amdgcn_s_setprio(0);
        }
    }
    if (wave < kGroup) {
        const int64_t before = group - 1 - wave;
        wait_for<V>(groups + before * a.row_words, before >= 0, wave == kGroup - 1, w);
        Words<V>::put(window, kGroup + wave, lane, w);
    }
    __syncthreads();
    if (wave == 0) {
        __builtin_amdgcn_s_setprio(3);
#pragma unroll 4
        for (int far = kGroup - 1; far >= 0; far--) Words<V>::apply(window, kGroup + far, lane, in);
        if (ends_group && !group_cut) {
#pragma unroll
            for (int i = 0; i < V; i++) B[i] = fmaf(A[i], in[i], B[i]);
            publish<V>(groups + group * a.row_words, A, B, true);
        }
#pragma unroll 4
        for (int n = 0; n < place; n++) Words<V>::apply(window, n, lane, in);
#pragma unroll
        for (int i = 0; i < V; i++) s_state[lane * V + i] = in[i];
        __builtin_amdgcn_s_setprio(0);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; i++) in[i] = s_state[lane * V + i];
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
__device__ __forceinline__ int64_t uniform(int64_t v)
{
    return (int64_t)((u64)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)v));
}
__device__ __forceinline__ int64_t divide(int64_t n, int64_t by)       // (both fit 32 bits but in the largest of calls)
{
    return n >> 32 || by >> 32 ? n / by : (int64_t)((uint32_t)n / (uint32_t)by);
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

// Tiles and blocks of channels are handed out in order, by a counter where there are words to wait for.  The next number is asked for
// while the last one is worked on.  (A workgroup may then hold a number that it has not begun.  Of all tiles that are not done
// the first is nevertheless being worked on: its holder has nothing before it left to do.)
__device__ __forceinline__ int64_t next_number(const ScanArgs &a, int64_t last)
{
    return a.words ? (int64_t)atomicAdd(a.ticket, 1ull) : last + gridDim.x;
}

template <class T, int kKind, int V, bool kShared, int kWaves, int kTokens>
__global__ __launch_bounds__(kWaves *kWave, Shape<T>::kForwardResident) void k_scan_forward(ScanArgs a)
{
    typedef typename T::Store S;
    constexpr int kRows = kWaves * kTokens, kThreads = kWaves * kWave;
    static_assert(kRows == kForwardTile && kRows % kScanTile == 0 && kScanTile % kTokens == 0, "the backward pass's states lie between waves");
    __shared__ TileMarks<kRows> marks;
    __shared__ u64 s_link[kWaves * V * kWave];
    __shared__ u64 s_window[2 * kGroup * V * kWave];
    __shared__ float s_state[V * kWave];
    __shared__ int64_t s_number;
    const int lane = lane_id(), wave = wave_id();
    Sequences<kRows, kThreads> seqs;
    seqs.load(a);
    clear_marks<kRows, kThreads>(marks);
    int64_t ahead = 0;                                  // (thread 0) the number that comes next
    if (threadIdx.x == 0) s_number = a.words ? next_number(a, 0) : blockIdx.x;
    __syncthreads();
    for (;;) {
        const int64_t number = uniform(s_number);
        if (number >= a.tiles * a.blocks) return;
        const int64_t tile = divide(number, a.blocks), block = number - tile * a.blocks;
        const Block bl = block_of(a, block);
        const bool active = lane * V < bl.width;
        // A lane's place in the block, and its head's (32 bits: what is the same for the wave stays in scalar registers).  Lanes past the
        // block's end do what lane 0 does, and store the same values to the same places.
        const uint32_t mine = active ? lane * V : 0, head = kShared ? mine / (uint32_t)a.group : 0;
        const int64_t head0 = kShared ? divide(bl.c, a.group) : 0, from = tile * kRows, row0 = from + wave * kTokens;
        const bool last = tile == a.tiles - 1;
        // all of the tile's rows are asked for at once (rows past the end: the last one again)
        Pack<T, V> x[kTokens];
        Pack<T, kShared ? 1 : V> g[kTokens];
        if (a.tokens > 0) {
            Rows xs(row0, a.tokens, a.x_stride, bl.c), gs(row0, a.tokens, a.gate_stride, kShared ? head0 : bl.c);
#pragma unroll
            for (int k = 0; k < kTokens; k++) {
                x[k].load(static_cast<const S *>(a.x) + xs.at + mine);
                g[k].load(static_cast<const S *>(a.gate) + gs.at + (kShared ? head : mine));
                xs.next(k);
                gs.next(k);
            }
        }
        seqs.mark(a, from, last, marks);
        __syncthreads();
        const uint32_t rows = seqs.template rows_in_use<kTokens>(row0);
        const int mark = lane < kTokens ? marks.begin[wave * kTokens + lane] : -1;
        const int stop = lane < kTokens ? marks.end[wave * kTokens + lane] : -1;
        const uint32_t begins = (uint32_t)__ballot(mark >= 0), ends = (uint32_t)__ballot(stop >= 0);
        const bool closed = marks.begin[0] >= 0 || tile == 0;       // nothing comes into the tile
        const bool cut = any_mark<kRows>(marks.begin);              // a sequence begins in it
        if (marks.empties && a.final) copy_empties<V, kRows, kWaves>(a, from, last, bl.c, mine, active, a.h0, a.final);

        float A[V], h[V];
#pragma unroll
        for (int i = 0; i < V; i++) { A[i] = 1.0f; h[i] = 0.0f; }
#pragma unroll
        for (int k = 0; k < kTokens; k++) {
            if ((begins >> k & 1)) load_state<V>(row_of(a.h0, __builtin_amdgcn_readlane(mark, k), a, bl.c), mine, h);
            step(k, x[k], g[k]);
            float ga, gb;
#pragma unroll
            for (int i = 0; i < V; i++) {
                if (!kShared || i == 0) open_gate<kKind>(g[k].get(i), ga, gb);
                A[i] *= ga;
                h[i] = fmaf(ga, h[i], gb * x[k].get(i));
            }
        }
        {
            u64 w[V];
#pragma unroll
            for (int i = 0; i < V; i++) w[i] = link_word(A[i], h[i], begins != 0);
            Words<V>::put(s_link, wave, lane, w);
        }
        __syncthreads();
        clear_marks<kRows, kThreads>(marks);
        if (threadIdx.x == 0) ahead = next_number(a, number);

        float in[V];                                    // the state that comes into the tile
#pragma unroll
        for (int i = 0; i < V; i++) in[i] = 0.0f;
        if (a.words) chain_state<V, kWaves>(a, block, tile, cut, closed, s_link, 0, 1, s_window, s_state, in);
#pragma unroll
        for (int i = 0; i < V; i++) h[i] = in[i];
        for (int w = 0; w < wave; w++) Words<V>::apply(s_link, w, lane, h);
        if (a.carry && row0 % kScanTile == 0 && row0 < a.tokens)
            store_state<V>(a.carry + row0 / kScanTile * a.channels + bl.c, mine, h);
        S *y = static_cast<S *>(a.y) + row0 * a.y_stride + bl.c;
#pragma unroll
        for (int k = 0; k < kTokens; k++) {
            if ((begins >> k & 1)) load_state<V>(row_of(a.h0, __builtin_amdgcn_readlane(mark, k), a, bl.c), mine, h);
            step(k, x[k], g[k]);
            float ga, gb;
#pragma unroll
            for (int i = 0; i < V; i++) {
                if (!kShared || i == 0) open_gate<kKind>(g[k].get(i), ga, gb);
                h[i] = fmaf(ga, h[i], gb * x[k].get(i));
            }
            if (rows >> k & 1) {
                Pack<T, V> out;
                out.set(h);
                out.store(y + mine);
            }
            y += a.y_stride;
            if ((ends >> k & 1) && a.final)
                store_state<V>(row_of(a.final, __builtin_amdgcn_readlane(stop, k), a, bl.c), mine, h);
        }
        if (threadIdx.x == 0) s_number = ahead;
        __syncthreads();
    }
}

// Sums of kTokens values a lane over the lanes of each head (`lanes` of them, the first head's from lane 0 on); the result for token k of
// a head is in v[k] of its first lane.
template <int kTokens> __device__ __forceinline__ void sum_heads(float (&v)[kTokens], int lanes, int lane)
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

template <class T, int kKind, int V, bool kShared, int kWaves, int kTokens>
__global__ __launch_bounds__(kWaves *kWave, Shape<T>::kBackwardResident) void k_scan_backward(ScanArgs a)
{
    typedef typename T::Store S;
    constexpr int kRows = kWaves * kTokens, kThreads = kWaves * kWave;
    static_assert(kRows == kScanTile, "a state is kept for each tile of the backward pass");
    __shared__ TileMarks<kRows> marks;
    __shared__ u64 s_ahead[kWaves * V * kWave], s_back[kWaves * V * kWave];
    __shared__ u64 s_window[2 * kGroup * V * kWave];
    __shared__ float s_state[V * kWave];
    __shared__ int64_t s_number;
    const int lane = lane_id(), wave = wave_id();
    Sequences<kRows, kThreads> seqs;
    seqs.load(a);
    clear_marks<kRows, kThreads>(marks);
    int64_t ahead = 0;
    if (threadIdx.x == 0) s_number = a.words ? next_number(a, 0) : blockIdx.x;
    __syncthreads();
    for (;;) {
        const int64_t number = uniform(s_number);
        if (number >= a.tiles * a.blocks) return;
        const int64_t turn = divide(number, a.blocks), block = number - turn * a.blocks, tile = a.tiles - 1 - turn;
        const Block bl = block_of(a, block);
        const bool active = lane * V < bl.width;
        const uint32_t mine = active ? lane * V : 0, head = kShared ? mine / (uint32_t)a.group : 0;
        const int64_t head0 = kShared ? divide(bl.c, a.group) : 0, from = tile * kRows, row0 = from + wave * kTokens;
        const bool last = tile == a.tiles - 1;
        Pack<T, V> x[kTokens], dy[kTokens];
        Pack<T, kShared ? 1 : V> g[kTokens];
        float h[V], e[V], A[V];
        float kept[V];                                  // the state before the tile's first row
        if (a.tokens > 0) {
            Rows xs(row0, a.tokens, a.x_stride, bl.c), gs(row0, a.tokens, a.gate_stride, kShared ? head0 : bl.c),
                ys(row0, a.tokens, a.dy_stride, bl.c);
#pragma unroll
            for (int k = 0; k < kTokens; k++) {
                x[k].load(static_cast<const S *>(a.x) + xs.at + mine);
                g[k].load(static_cast<const S *>(a.gate) + gs.at + (kShared ? head : mine));
                dy[k].load(static_cast<const S *>(a.dy) + ys.at + mine);
                xs.next(k);
                gs.next(k);
                ys.next(k);
            }
            load_state<V>(static_cast<const float *>(a.carry) + tile * a.channels + bl.c, mine, kept);
        }
        seqs.mark(a, from, last, marks);
        __syncthreads();
        const uint32_t rows = seqs.template rows_in_use<kTokens>(row0);
        const int mark = lane < kTokens ? marks.begin[wave * kTokens + lane] : -1;
        const int stop = lane < kTokens ? marks.end[wave * kTokens + lane] : -1;
        const uint32_t begins = (uint32_t)__ballot(mark >= 0), ends = (uint32_t)__ballot(stop >= 0);
        const bool closed = marks.end[kRows - 1] >= 0 || last;      // nothing comes back into the tile
        const bool cut = any_mark<kRows>(marks.end);                // a sequence ends in it
        if (marks.empties && a.dh0) copy_empties<V, kRows, kWaves>(a, from, last, bl.c, mine, active, a.dfinal, a.dh0);

        // Both directions' links at once: e of the rows before k is what e of row k becomes, times the gates between, so that
        // with P the product of the gates up to k the backward sum is that of P dy.
#pragma unroll
        for (int i = 0; i < V; i++) { A[i] = 1.0f; h[i] = e[i] = 0.0f; }
#pragma unroll
        for (int k = 0; k < kTokens; k++) {
            if ((begins >> k & 1)) load_state<V>(row_of(a.h0, __builtin_amdgcn_readlane(mark, k), a, bl.c), mine, h);
            // (a sequence that ends here sends its rows' share back; what comes after it is another's)
            const bool over = (ends & ((1u << k) - 1));
            step(k, x[k], g[k], dy[k]);
            float ga, gb;
#pragma unroll
            for (int i = 0; i < V; i++) {
                if (!kShared || i == 0) open_gate<kKind>(g[k].get(i), ga, gb);
                A[i] *= ga;
                h[i] = fmaf(ga, h[i], gb * x[k].get(i));
                if (!over) e[i] = fmaf(A[i], dy[k].get(i), e[i]);
            }
            if ((ends >> k & 1) && !over) {
                float d[V];
                load_state<V>(row_of(a.dfinal, __builtin_amdgcn_readlane(stop, k), a, bl.c), mine, d);
#pragma unroll
                for (int i = 0; i < V; i++) e[i] = fmaf(A[i], d[i], e[i]);
            }
        }
        {
            u64 w[V];
#pragma unroll
            for (int i = 0; i < V; i++) w[i] = link_word(A[i], h[i], begins != 0);
            Words<V>::put(s_ahead, wave, lane, w);
#pragma unroll
            for (int i = 0; i < V; i++) w[i] = link_word(A[i], e[i], ends != 0);
            Words<V>::put(s_back, wave, lane, w);
        }
        __syncthreads();
        clear_marks<kRows, kThreads>(marks);
        if (threadIdx.x == 0) ahead = next_number(a, number);

        float in[V];                                    // what comes back into the tile
#pragma unroll
        for (int i = 0; i < V; i++) in[i] = 0.0f;
        if (a.words) chain_state<V, kWaves>(a, block, turn, cut, closed, s_back, kWaves - 1, -1, s_window, s_state, in);
#pragma unroll
        for (int i = 0; i < V; i++) { h[i] = kept[i]; e[i] = in[i]; }
        for (int w = 0; w < wave; w++) Words<V>::apply(s_ahead, w, lane, h);
        for (int w = kWaves - 1; w > wave; w--) Words<V>::apply(s_back, w, lane, e);
        float sum[kTokens];
        float before[kTokens][V];
#pragma unroll
        for (int k = 0; k < kTokens; k++) {
            if ((begins >> k & 1)) load_state<V>(row_of(a.h0, __builtin_amdgcn_readlane(mark, k), a, bl.c), mine, h);
            step(k, x[k], g[k]);
            float ga, gb;
#pragma unroll
            for (int i = 0; i < V; i++) {
                if (!kShared || i == 0) open_gate<kKind>(g[k].get(i), ga, gb);
                before[k][i] = h[i];
                h[i] = fmaf(ga, h[i], gb * x[k].get(i));
            }
        }
        S *px = static_cast<S *>(a.dx) + (row0 + kTokens - 1) * a.dx_stride + bl.c,
          *pg = static_cast<S *>(a.dgate) + (row0 + kTokens - 1) * a.dgate_stride + bl.c;
#pragma unroll
        for (int k = kTokens - 1; k >= 0; k--) {
            if ((ends >> k & 1)) load_state<V>(row_of(a.dfinal, __builtin_amdgcn_readlane(stop, k), a, bl.c), mine, e);
            step(k, x[k], g[k], dy[k]);
            float dx[V], dg[V], ga, gb;
            sum[k] = 0.0f;
#pragma unroll
            for (int i = 0; i < V; i++) {
                if (!kShared || i == 0) open_gate<kKind>(g[k].get(i), ga, gb);
                e[i] += dy[k].get(i);
                dx[i] = kKind == kDecay ? e[i] : gb * e[i];
                dg[i] = kKind == kDecay ? e[i] * before[k][i] : ga * gb * (e[i] * (before[k][i] - x[k].get(i)));
                if (kShared) sum[k] += dg[i];
                e[i] *= ga;
            }
            if (rows >> k & 1) {
                Pack<T, V> out;
                out.set(dx);
                out.store(px + mine);
                if (!kShared) {
                    out.set(dg);
                    out.store(pg + mine);
                }
            }
            px -= a.dx_stride;
            pg -= a.dgate_stride;
            if ((begins >> k & 1) && a.dh0)
                store_state<V>(row_of(a.dh0, __builtin_amdgcn_readlane(mark, k), a, bl.c), mine, e);
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
                    if (!(rows >> k & 1)) continue;
                    if (a.parts > 1) a.partial[(bl.part * a.tokens + row0 + k) * a.heads + head0 + head] = sum[k];
                    else static_cast<S *>(a.dgate)[(row0 + k) * a.dgate_stride + head0 + head] = (S)sum[k];
                }
            }
        }
        if (threadIdx.x == 0) s_number = ahead;
        __syncthreads();
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

// Elements a thread takes of a row: four of 16 bits where there are channels enough for a wave of them, else two, as the rows' and the
// heads' numbers allow.
static int elements_of(int dtype, const ScanArgs &a)
{
    const int64_t unit = a.group == 1 ? a.channels : a.group;      // (heads that are cut into parts are cut at multiples of V)
    if (dtype != DGN_F32 && unit % 4 == 0 && a.channels > 128) return 4;
    return unit % 2 == 0 ? 2 : 1;
}

static int64_t tiles_of(int64_t tokens, int rows) { return tokens > 0 ? (tokens + rows - 1) / rows : 1; }

// Scratch: the counter (256 bytes), a word per tile and channel of the direction with the smaller tiles, the parts' sums.
struct ScanScratch { size_t words, partial, bytes; };
static ScanScratch lay_out(int dtype, const ScanArgs &a)
{
    const int V = elements_of(dtype, a);
    const Cut cut = cut_channels(a.channels, a.group, V);
    ScanScratch s;
    s.words = 256;
    const int64_t tiles = tiles_of(a.tokens, kBackwardTile);
    s.partial = s.words + (size_t)(tiles + tiles / kGroup) * cut.blocks * V * kWave * sizeof(u64);
    s.bytes = s.partial + (cut.parts > 1 ? (size_t)cut.parts * a.tokens * a.heads * sizeof(float) : 0);
    return s;
}
size_t scan_scratch_bytes(int dtype, const ScanArgs &a) { return lay_out(dtype, a).bytes; }

// Sets what the kernels need to know of the cut; clears the counter and the words where there are several tiles.
static hipError_t set_up(int dtype, ScanArgs &a, int rows, void *scratch, hipStream_t s)
{
    const int V = elements_of(dtype, a);
    const Cut cut = cut_channels(a.channels, a.group, V);
    const ScanScratch l = lay_out(dtype, a);
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
    const FillRegion clear = {mem, l.words + (size_t)(a.tiles + a.tiles / kGroup) * a.row_words * sizeof(u64)};
    return launch_clear(&clear, 1, s);
}

static unsigned grid_of(const ScanArgs &a)
{
    const int64_t n = a.tiles * a.blocks;
    return (unsigned)(n < (1 << 20) ? n : 1 << 20);     // (a workgroup goes on until all is handed out)
}

template <class T, int kKind, int V> static void go_forward(const ScanArgs &a, hipStream_t s)
{
    typedef Shape<T> P;
    const dim3 grid(grid_of(a)), threads(P::kForwardWaves * kWave);
    if (a.group == 1) hipLaunchKernelGGL((k_scan_forward<T, kKind, V, false, P::kForwardWaves, P::kForwardRows>), grid, threads, 0, s, a);
    else hipLaunchKernelGGL((k_scan_forward<T, kKind, V, true, P::kForwardWaves, P::kForwardRows>), grid, threads, 0, s, a);
}
template <class T, int kKind, int V> static void go_backward(const ScanArgs &a, hipStream_t s)
{
    typedef Shape<T> P;
    const dim3 grid(grid_of(a)), threads(P::kBackwardWaves * kWave);
    if (a.group == 1) {
        hipLaunchKernelGGL((k_scan_backward<T, kKind, V, false, P::kBackwardWaves, P::kBackwardRows>), grid, threads, 0, s, a);
        return;
    }
    hipLaunchKernelGGL((k_scan_backward<T, kKind, V, true, P::kBackwardWaves, P::kBackwardRows>), grid, threads, 0, s, a);
    if (a.parts > 1 && a.tokens > 0) {
        const int64_t n = (a.tokens * a.heads + 255) / 256;
        hipLaunchKernelGGL((k_gate_sums<T>), dim3((unsigned)(n < 8192 ? n : 8192)), dim3(256), 0, s, a);
    }
}
template <class T, int kKind> static void go(bool back, int V, const ScanArgs &a, hipStream_t s)
{
    constexpr int kMost = sizeof(typename T::Store) == 4 ? 2 : 4;
    if (V == 1) { if (back) go_backward<T, kKind, 1>(a, s); else go_forward<T, kKind, 1>(a, s); }
    else if (V == 2) { if (back) go_backward<T, kKind, 2>(a, s); else go_forward<T, kKind, 2>(a, s); }
    else { if (back) go_backward<T, kKind, kMost>(a, s); else go_forward<T, kKind, kMost>(a, s); }
}

#define DGN_BY_TYPE(call)                                                                                     \
    do {                                                                                                      \
        if (dtype == DGN_F32) { typedef F32 T; if (kind == kDecay) call(T, kDecay); else call(T, kSigmoid); } \
        else if (dtype == DGN_F16) { typedef F16 T; if (kind == kDecay) call(T, kDecay); else call(T, kSigmoid); } \
        else { typedef BF16 T; if (kind == kDecay) call(T, kDecay); else call(T, kSigmoid); }                 \
    } while (0)

hipError_t launch_scan_forward(int dtype, int kind, ScanArgs a, void *scratch, hipStream_t s)
{
    const hipError_t e = set_up(dtype, a, kForwardTile, scratch, s);
    if (e != hipSuccess) return e;
#define DGN_GO(T, K) go<T, K>(false, elements_of(dtype, a), a, s)
    DGN_BY_TYPE(DGN_GO);
#undef DGN_GO
    return hipGetLastError();
}

hipError_t launch_scan_backward(int dtype, int kind, ScanArgs a, void *scratch, hipStream_t s)
{
    const hipError_t e = set_up(dtype, a, kBackwardTile, scratch, s);
    if (e != hipSuccess) return e;
#define DGN_GO(T, K) go<T, K>(true, elements_of(dtype, a), a, s)
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
