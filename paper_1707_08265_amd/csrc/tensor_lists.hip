// Operators over a list of tensors: norms of up to 64 target sets, clipping by them, and the update that applies it.
//   n_q = sqrt(sum of |g_i|^2 over the tensors i of set q),   f_i = min over its sets of min(1, max_norm / (n_q + eps))
//   m' = beta1 m + (1 - beta1) f g,   v' = beta2 v + (1 - beta2) (f g)^2,   p' = p - lr (m' / c1 / (sqrt(v' / c2) + eps) + wd p)
// A tensor is cut into chunks of kListChunk elements, which a list has a table of: address, size and type in one load.  All of it is
// bound by memory.  500 layers of 120 M elements in all: squares of bf16 240 MB in 42 us, 5.7 TB/s; clipping 482 MB in 77 us, 6.3 TB/s;
// the update 3.37 GB in 604 to 623 us, 5.4 to 5.6 TB/s (a copy by a thread per 16 bytes: 6.2, past the caches 6.5).
#include "values.h"

namespace dgn {

__device__ __forceinline__ double wave_sum_double(double v)
{
#pragma unroll
    for (int d = kWave / 2; d >= 1; d >>= 1) v += __shfl_xor(v, d, kWave);
    return v;
}

// N neighbouring elements, at an address that is aligned to one, in 32 bits.
typedef uint32_t Quad32 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t Quad16 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t Pair16 __attribute__((ext_vector_type(2), aligned(2)));
template <class T> __device__ __forceinline__ float half_of(uint32_t w, int i)
{
    return (float)__builtin_bit_cast(typename T::Store, (uint16_t)(w >> (16 * i)));
}
template <class T> __device__ __forceinline__ uint32_t two_halves(float a, float b)
{
    typedef typename T::Store H2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, H2{(typename T::Store)a, (typename T::Store)b});
}
// What a thread takes of a tensor at a time: sixteen bytes.
template <class T> struct Run;
template <> struct Run<F32> {
    static constexpr int kN = 4;
    Quad32 w;
    __device__ __forceinline__ void load(const float *p) { w = *reinterpret_cast<const Quad32 *>(p); }
    template <bool kStream> __device__ __forceinline__ void store(float *p) const { put<kStream, 4>(p, w); }
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(w[i]); }
    __device__ __forceinline__ void scale(float f)
    {
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = __float_as_uint(get(i) * f);
    }
};
template <class T> struct Run16 {
    typedef typename T::Store S;
    static constexpr int kN = 8;
    Quad16 w;
    __device__ __forceinline__ void load(const S *p) { w = *reinterpret_cast<const Quad16 *>(p); }
    template <bool kStream> __device__ __forceinline__ void store(S *p) const { put<kStream, 2>(p, w); }
    __device__ __forceinline__ float get(int i) const { return half_of<T>(w[i / 2], i % 2); }
    __device__ __forceinline__ void scale(float f)
    {
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = two_halves<T>(get(2 * i) * f, get(2 * i + 1) * f);
    }
};
template <> struct Run<F16> : Run16<F16> {};
template <> struct Run<BF16> : Run16<BF16> {};
// Four elements of any type.
template <class T> struct Four;
template <> struct Four<F32> {
    template <bool kStream> static __device__ __forceinline__ void load(const float *p, float (&f)[4])
    {
        const Quad32 w = take<kStream, 4, Quad32>(p);
#pragma unroll
        for (int i = 0; i < 4; i++) f[i] = __uint_as_float(w[i]);
    }
    template <bool kStream> static __device__ __forceinline__ void store(float *p, const float (&f)[4])
    {
        put<kStream, 4>(p, Quad32{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])});
    }
};
template <class T> struct Four16 {
    typedef typename T::Store S;
    template <bool kStream> static __device__ __forceinline__ void load(const S *p, float (&f)[4])
    {
        const Pair16 w = take<kStream, 2, Pair16>(p);
#pragma unroll
        for (int i = 0; i < 4; i++) f[i] = half_of<T>(w[i / 2], i % 2);
    }
    template <bool kStream> static __device__ __forceinline__ void store(S *p, const float (&f)[4])
    {
        put<kStream, 2>(p, Pair16{two_halves<T>(f[0], f[1]), two_halves<T>(f[2], f[3])});
    }
};
template <> struct Four<F16> : Four16<F16> {};
template <> struct Four<BF16> : Four16<BF16> {};

__device__ __forceinline__ int elements(const ListChunk &c) { return (int)(c.n_type >> 2); }
__device__ __forceinline__ int type(const ListChunk &c) { return (int)(c.n_type & 3); }

// The sets that reach an entry: its word of the mask, or that of the tensor that it stands for (none, if there is no such
// tensor); without a mask every set does.
__device__ __forceinline__ u64 reach_of(const Reach &r, int32_t entry)
{
    const u64 all = r.sets < 64 ? (1ull << r.sets) - 1 : ~0ull;
    if (!r.mask) return all;
    const int64_t at = r.ids ? r.ids[entry] : entry;
    return at >= 0 && at < r.words ? r.mask[at] & all : 0;
}

// Threads of a workgroup, and workgroups to a chunk.  The update goes over nine arrays at once, and is the faster the closer together all
// workgroups are in them: one pass of 2 048 elements each 657 us, of 1 024 690 us, four passes of 1 024 750 us or, from the last
// chunk to the first, 812.
constexpr int kListThreads = 256, kClipParts = 2;
constexpr int kAdamThreads = 512, kAdamParts = 4;

// Squares are added up in 64 bits: those of 32-bit gradients above 2e19 or below 1e-23 have no 32-bit value.
template <class T, int kThreads> __device__ __forceinline__ double squares(const typename T::Store *p, int n, int thread)
{
    constexpr int kN = Run<T>::kN, kTurn = kThreads * kN, kAhead = 2;
    double sum[2] = {0.0, 0.0};
    int i = thread * kN;
    for (; i + (kAhead - 1) * kTurn + kN <= n; i += kAhead * kTurn) {
        Run<T> r[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; u++) r[u].load(p + i + u * kTurn);
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
#pragma unroll
            for (int k = 0; k < kN; k++) { const double v = r[u].get(k); sum[k % 2] = fma(v, v, sum[k % 2]); }
        }
    }
    for (; i + kN <= n; i += kTurn) {
        Run<T> r;
        r.load(p + i);
#pragma unroll
        for (int k = 0; k < kN; k++) { const double v = r.get(k); sum[k % 2] = fma(v, v, sum[k % 2]); }
    }
    i = n / kN * kN + thread;
    if (i < n) { const double v = (float)p[i]; sum[0] = fma(v, v, sum[0]); }
    return sum[0] + sum[1];
}
__global__ __launch_bounds__(kListThreads) void k_list_squares(ListView g, double *partial, uint32_t *arrived)
{
    __shared__ double s_sum[kListThreads / kWave];
    const ListChunk c = g.chunk[blockIdx.x];
    double sum = 0.0;
#define DGN_GO(T) sum = squares<T, kListThreads>(static_cast<const typename T::Store *>(c.data), elements(c), threadIdx.x)
    DGN_BY_DTYPE(type(c), DGN_GO);
#undef DGN_GO
    sum = wave_sum_double(sum);
    if (lane_id() == 0) s_sum[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        partial[blockIdx.x] = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
        if (blockIdx.x == 0) *arrived = 0;              // for the next launch
    }
}

// The chunks' sums to the sets': a lane per set, kPerGroup chunks to a workgroup, and the workgroups' sums by the one that is done last.
// Always in the same order, so the same gradients give the same norms.
constexpr int kPerGroup = 1024;
__global__ __launch_bounds__(kPerGroup) void k_list_norms(ListView g, Reach r, const double *partial, double *sums, uint32_t *arrived, float *norms)
{
    struct Link { double sum; u64 bits; };
    __shared__ Link s_link[kPerGroup];
    __shared__ double s_sum[kPerGroup / kWave][kWave];
    __shared__ bool s_last;
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    const int32_t chunk = blockIdx.x * kPerGroup + threadIdx.x;
    const bool some = chunk < g.chunks;
    s_link[threadIdx.x] = Link{some ? partial[chunk] : 0.0, some ? reach_of(r, (int32_t)g.chunk[chunk].entry) : 0};
    __syncthreads();
    double sum = 0.0;
#pragma unroll 4
    for (int j = 0; j < kWave; j++) {
        const Link l = s_link[wave * kWave + j];
        if (l.bits >> lane & 1) sum += l.sum;           // (what a set does not need does not count, whatever it is)
    }
    s_sum[wave][lane] = sum;
    __syncthreads();
    if (wave != 0) return;
    sum = 0.0;
#pragma unroll
    for (int w = 0; w < kPerGroup / kWave; w++) sum += s_sum[w][lane];
    if (gridDim.x > 1) {
        store_coherent(reinterpret_cast<u64 *>(sums) + blockIdx.x * kWave + lane, (u64)__double_as_longlong(sum));
        __threadfence();
        if (lane == 0) s_last = atomicAdd(arrived, 1u) == gridDim.x - 1;
        wave_fence();
        if (!s_last) return;
        __threadfence();
        sum = 0.0;
#pragma unroll 8
        for (unsigned b = 0; b < gridDim.x; b++) sum += __longlong_as_double((long long)load_coherent(reinterpret_cast<const u64 *>(sums) + b * kWave + lane));
    }
    if (lane < r.sets) norms[lane] = (float)sqrt(sum);
}

// The least factor of the sets that reach a tensor (NaN if one of their norms is), 1 where none does.
__device__ __forceinline__ float clip_factor(const ClipArgs &c, u64 bits, bool &finite)
{
    const int lane = lane_id();
    float f = 1.0f;
    bool fine = true;
    if (bits >> lane & 1) {
        const float n = c.norms[lane];
        fine = fabsf(n) < INFINITY;
        f = c.max_norm / (n + c.eps);
        if (f > 1.0f || n + c.eps <= 0.0f) f = 1.0f;        // (gradients of 0, and max_norm and eps as well: nothing to scale)
        if (n == INFINITY) f = 0.0f;                        // (also if max_norm is infinite)
    }
    finite = __all(fine);
#pragma unroll
    for (int d = kWave / 2; d >= 1; d >>= 1) {
        const float o = __shfl_xor(f, d, kWave);
        f = o < f || o != o ? o : f;
    }
    return f;
}

// Lists of a few small tensors: all of it in one workgroup, a wave to a chunk, instead of two launches.  Both in us, f32, 40 calls
// in a graph: 1 chunk of 8 192 elements 4.3 and 7.3, 16 of 8 192 5.6 and 7.9, 64 of 64 4.3 and 8.4, 64 of 2 048 6.9 and 8.5, but 64 of
// 4 096 10.1 and 8.7, 128 of 64 6.8 and 8.2, 128 of 1 024 8.9 and 8.4.  In bf16 the same within a tenth.
constexpr int kSmallChunks = 64;
constexpr int64_t kSmallElements = 131072;
__global__ __launch_bounds__(1024) void k_list_norms_small(ListView g, Reach r, float *norms)
{
    __shared__ double s_sum[16][kWave];
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    double mine = 0.0;
    for (int j = wave; j < g.chunks; j += 16) {
        const ListChunk c = g.chunk[j];
        double sum = 0.0;
#define DGN_GO(T) sum = squares<T, kWave>(static_cast<const typename T::Store *>(c.data), elements(c), lane)
        DGN_BY_DTYPE(type(c), DGN_GO);
#undef DGN_GO
        sum = wave_sum_double(sum);
        if (reach_of(r, (int32_t)c.entry) >> lane & 1) mine += sum;
    }
    s_sum[wave][lane] = mine;
    __syncthreads();
    if (wave != 0) return;
    mine = 0.0;
#pragma unroll
    for (int w = 0; w < 16; w++) mine += s_sum[w][lane];
    if (lane < r.sets) norms[lane] = (float)sqrt(mine);
}

template <class T, bool kStream> __device__ __forceinline__ void scale_to(typename T::Store *out, const typename T::Store *p, int n, float f)
{
    constexpr int kN = Run<T>::kN, kTurn = kListThreads * kN, kAhead = 2;
    int i = threadIdx.x * kN;
    for (; i + (kAhead - 1) * kTurn + kN <= n; i += kAhead * kTurn) {
        Run<T> r[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; u++) r[u].load(p + i + u * kTurn);
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
            if (f != 1.0f) r[u].scale(f);
            r[u].template store<kStream>(out + i + u * kTurn);
        }
    }
    for (; i + kN <= n; i += kTurn) {
        Run<T> r;
        r.load(p + i);
        if (f != 1.0f) r.scale(f);
        r.template store<kStream>(out + i);
    }
    i = n / kN * kN + threadIdx.x;
    if (i < n) out[i] = f != 1.0f ? (typename T::Store)((float)p[i] * f) : p[i];
}
// The chunks from the last to the first: what the norms' pass read last is still in the cache.
template <bool kStream> __global__ __launch_bounds__(kListThreads) void k_list_clip(ListView g, ListView out, ClipArgs cl)
{
    const unsigned number = gridDim.x - 1 - blockIdx.x, chunk = number / kClipParts;
    const ListChunk c = g.chunk[chunk], o = out.chunk[chunk];
    const int first = (int)(number % kClipParts) * (kListChunk / kClipParts), left = elements(c) - first;
    const int n = left < kListChunk / kClipParts ? left : kListChunk / kClipParts;
    if (n <= 0) return;
    bool finite;
    const float f = clip_factor(cl, reach_of(cl.reach, (int32_t)c.entry), finite);
    if (f == 1.0f && c.data == o.data) return;
#define DGN_GO(T) scale_to<T, kStream>(static_cast<typename T::Store *>(o.data) + first, static_cast<const typename T::Store *>(c.data) + first, n, f)
    DGN_BY_DTYPE(type(c), DGN_GO);
#undef DGN_GO
}

struct AdamRow { const float *p, *m, *v; float *op, *om, *ov; };
__device__ __forceinline__ void adam_one(const AdamArgs &a, float g, float &p, float &m, float &v)
{
    m = a.beta1 * m + a.rest1 * g;
    v = a.beta2 * v + a.rest2 * (g * g);
    p -= a.decay * p + a.rate * m / (sqrtf(v * a.spread) + a.eps);
}
template <class T, bool kStream>
__device__ __forceinline__ void adam_chunk(const AdamArgs &a, const typename T::Store *g, const AdamRow &r, void *copy, int32_t copy_type, int n,
                                           float f, bool live)
{
    constexpr int kTurn = kAdamThreads * 4;
    for (int i = threadIdx.x * 4; i + 4 <= n; i += kTurn) {
        float d[4], p[4], m[4], v[4];
        Four<T>::template load<kStream>(g + i, d);
        Four<F32>::load<kStream>(r.p + i, p);
        Four<F32>::load<kStream>(r.m + i, m);
        Four<F32>::load<kStream>(r.v + i, v);
        if (live) {
#pragma unroll
            for (int k = 0; k < 4; k++) adam_one(a, d[k] * f, p[k], m[k], v[k]);
        }
        Four<F32>::store<kStream>(r.op + i, p);
        Four<F32>::store<kStream>(r.om + i, m);
        Four<F32>::store<kStream>(r.ov + i, v);
        if (copy) {
#define DGN_GO(C) Four<C>::template store<kStream>(static_cast<typename C::Store *>(copy) + i, p)
            DGN_BY_DTYPE(copy_type, DGN_GO);
#undef DGN_GO
        }
    }
    const int i = n / 4 * 4 + threadIdx.x;
    if (i < n) {
        float p = r.p[i], m = r.m[i], v = r.v[i];
        if (live) adam_one(a, (float)g[i] * f, p, m, v);
        r.op[i] = p;
        r.om[i] = m;
        r.ov[i] = v;
        if (copy) {
#define DGN_GO(C) static_cast<typename C::Store *>(copy)[i] = (typename C::Store)p
            DGN_BY_DTYPE(copy_type, DGN_GO);
#undef DGN_GO
        }
    }
}
template <bool kStream> __global__ __launch_bounds__(kAdamThreads) void k_list_adam(AdamArgs a)
{
    const unsigned chunk = blockIdx.x / kAdamParts;
    const ListChunk g = a.grad.chunk[chunk];
    const int first = (int)(blockIdx.x % kAdamParts) * (kListChunk / kAdamParts), left = elements(g) - first;
    const int n = left < kListChunk / kAdamParts ? left : kListChunk / kAdamParts;
    if (n <= 0) return;
    const u64 bits = reach_of(a.clip.reach, (int32_t)g.entry);
    bool finite = true;
    const float f = a.clip.norms ? clip_factor(a.clip, bits, finite) : 1.0f;
    const bool live = bits != 0 && (finite || !a.skip_nonfinite);
    const auto at = [&](const ListView &l) { return static_cast<float *>(l.chunk[chunk].data) + first; };
    const AdamRow r = {at(a.param), at(a.m), at(a.v), at(a.out_param), at(a.out_m), at(a.out_v)};
    void *copy = nullptr;
    int32_t copy_type = DGN_F32;
    if (a.copy.chunk) {
        const ListChunk c = a.copy.chunk[chunk];
        copy_type = type(c);
        copy = static_cast<char *>(c.data) + first * (copy_type == DGN_F32 ? 4 : 2);
    } else if (!live && r.p == r.op && r.m == r.om && r.v == r.ov) return;
#define DGN_GO(T) adam_chunk<T, kStream>(a, static_cast<const typename T::Store *>(g.data) + first, r, copy, copy_type, n, f, live)
    DGN_BY_DTYPE(type(g), DGN_GO);
#undef DGN_GO
}

// Scratch of the norms: a sum per chunk, the workgroups' sums for each set, and how many of them are done.
static int norm_groups(const ListView &g) { return (g.chunks + kPerGroup - 1) / kPerGroup; }
size_t list_norms_scratch_bytes(const ListView &g)
{
    return sizeof(double) * ((size_t)g.chunks + (size_t)norm_groups(g) * kWave) + 256;
}

hipError_t launch_list_norms(const ListView &g, const Reach &r, void *scratch, float *norms, hipStream_t s)
{
    double *partial = static_cast<double *>(scratch), *sums = partial + g.chunks;
    const int groups = norm_groups(g);
    if (g.chunks <= kSmallChunks && g.elements <= kSmallElements) {
        hipLaunchKernelGGL(k_list_norms_small, dim3(1), dim3(1024), 0, s, g, r, norms);
        return hipGetLastError();
    }
    uint32_t *arrived = reinterpret_cast<uint32_t *>(sums + (size_t)groups * kWave);
    hipLaunchKernelGGL(k_list_squares, dim3((unsigned)g.chunks), dim3(kListThreads), 0, s, g, partial, arrived);
    hipLaunchKernelGGL(k_list_norms, dim3((unsigned)groups), dim3(kPerGroup), 0, s, g, r, partial, sums, arrived, norms);
    return hipGetLastError();
}

hipError_t launch_list_clip(const ListView &g, const ListView &out, const ClipArgs &c, hipStream_t s)
{
    if (g.chunks == 0) return hipSuccess;
    if (g.bytes + out.bytes > kStreamBytes) hipLaunchKernelGGL(k_list_clip<true>, dim3((unsigned)g.chunks * kClipParts), dim3(kListThreads), 0, s, g, out, c);
    else hipLaunchKernelGGL(k_list_clip<false>, dim3((unsigned)g.chunks * kClipParts), dim3(kListThreads), 0, s, g, out, c);
    return hipGetLastError();
}

hipError_t launch_list_adam(const AdamArgs &a, hipStream_t s)
{
    if (a.grad.chunks == 0) return hipSuccess;
    const size_t bytes = a.grad.bytes + 6 * a.param.bytes + a.copy.bytes;
    if (bytes > kStreamBytes) hipLaunchKernelGGL(k_list_adam<true>, dim3((unsigned)a.grad.chunks * kAdamParts), dim3(kAdamThreads), 0, s, a);
    else hipLaunchKernelGGL(k_list_adam<false>, dim3((unsigned)a.grad.chunks * kAdamParts), dim3(kAdamThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace dgn
