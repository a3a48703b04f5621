// Operators over a list of tensors: norms of up to 64 target sets, clipping by them, and the update that applies it.
// A tensor is cut into chunks of kListChunk elements; a workgroup takes one.
#include "values.h"

namespace dgn {

__device__ __forceinline__ double wave_sum_double(double v)
{
#pragma unroll
    for (int d = kWave / 2; d >= 1; d >>= 1) v += __shfl_xor(v, d, kWave);
    return v;
}

__device__ __forceinline__ float load_at(const void *p, int dtype, int64_t i)
{
    if (dtype == DGN_F32) return static_cast<const float *>(p)[i];
    if (dtype == DGN_F16) return (float)static_cast<const _Float16 *>(p)[i];
    return (float)static_cast<const __bf16 *>(p)[i];
}
__device__ __forceinline__ void store_at(void *p, int dtype, int64_t i, float v)
{
    if (dtype == DGN_F32) static_cast<float *>(p)[i] = v;
    else if (dtype == DGN_F16) static_cast<_Float16 *>(p)[i] = (_Float16)v;
    else static_cast<__bf16 *>(p)[i] = (__bf16)v;
}

// The sets that reach an entry: its word of the mask, or that of the tensor that it stands for (none, if there is no such
// tensor); without a mask every set does.
__device__ __forceinline__ u64 reach_of(const Reach &r, int32_t entry)
{
    const u64 all = r.sets < 64 ? (1ull << r.sets) - 1 : ~0ull;
    if (!r.mask) return all;
    const int64_t at = r.ids ? r.ids[entry] : entry;
    return at >= 0 && at < r.words ? r.mask[at] & all : 0;
}

// Squares are added up in 64 bits: those of 32-bit gradients above 2e19 or below 1e-23 have no 32-bit value.
__global__ __launch_bounds__(256) void k_list_squares(ListView g, double *partial)
{
    __shared__ double s_sum[4];
    const ListChunk c = g.chunk[blockIdx.x];
    const ListEntry e = g.entry[c.entry];
    const int64_t from = (int64_t)c.index * kListChunk, to = from + kListChunk < e.numel ? from + kListChunk : e.numel;
    double sum = 0.0;
    for (int64_t i = from + threadIdx.x; i < to; i += 256) {
        const double v = load_at(e.data, e.dtype, i);
        sum += v * v;
    }
    sum = wave_sum_double(sum);
    if (lane_id() == 0) s_sum[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) partial[blockIdx.x] = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
}

// A lane per set; the chunks in a fixed order, so the same gradients give the same norms.
__global__ __launch_bounds__(1024) void k_list_norms(ListView g, Reach r, const double *partial, float *norms)
{
    __shared__ double s_sum[16][kWave];
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    double sum = 0.0;
    for (int32_t at = wave * kWave; at < g.chunks; at += 1024) {
        const bool some = at + lane < g.chunks;
        const double v = some ? partial[at + lane] : 0.0;
        const u64 bits = some ? reach_of(r, g.chunk[at + lane].entry) : 0;
        for (int j = 0; j < kWave; j++) {
            const double w = __shfl(v, j, kWave);
            if (shfl64(bits, j) >> lane & 1) sum += w;
        }
    }
    s_sum[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && lane < r.sets) {
        sum = 0.0;
        for (int w = 0; w < 16; w++) sum += s_sum[w][lane];
        norms[lane] = (float)sqrt(sum);
    }
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
        if (f > 1.0f) f = 1.0f;
    }
    finite = __all(fine);
#pragma unroll
    for (int d = kWave / 2; d >= 1; d >>= 1) {
        const float o = __shfl_xor(f, d, kWave);
        f = o < f || o != o ? o : f;
    }
    return f;
}

__global__ __launch_bounds__(256) void k_list_clip(ListView g, ListView out, ClipArgs cl)
{
    const ListChunk c = g.chunk[blockIdx.x];
    const ListEntry e = g.entry[c.entry], o = out.entry[c.entry];
    bool finite;
    const float f = clip_factor(cl, reach_of(cl.reach, c.entry), finite);
    if (f == 1.0f && e.data == o.data) return;
    const int64_t from = (int64_t)c.index * kListChunk, to = from + kListChunk < e.numel ? from + kListChunk : e.numel;
    for (int64_t i = from + threadIdx.x; i < to; i += 256) store_at(o.data, o.dtype, i, load_at(e.data, e.dtype, i) * f);
}

__global__ __launch_bounds__(256) void k_list_adam(AdamArgs a)
{
    const ListChunk c = a.grad.chunk[blockIdx.x];
    const ListEntry g = a.grad.entry[c.entry];
    const u64 bits = reach_of(a.clip.reach, c.entry);
    bool finite = true;
    const float f = a.clip.norms ? clip_factor(a.clip, bits, finite) : 1.0f;
    const bool live = bits != 0 && (finite || !a.skip_nonfinite);
    const float *p = static_cast<const float *>(a.param.entry[c.entry].data), *m = static_cast<const float *>(a.m.entry[c.entry].data),
                *v = static_cast<const float *>(a.v.entry[c.entry].data);
    float *op = static_cast<float *>(a.out_param.entry[c.entry].data), *om = static_cast<float *>(a.out_m.entry[c.entry].data),
          *ov = static_cast<float *>(a.out_v.entry[c.entry].data);
    const int64_t from = (int64_t)c.index * kListChunk, to = from + kListChunk < g.numel ? from + kListChunk : g.numel;
    for (int64_t i = from + threadIdx.x; i < to; i += 256) {
        float np = p[i], nm = m[i], nv = v[i];
        if (live) {
            const float d = load_at(g.data, g.dtype, i) * f;
            nm = a.beta1 * nm + a.rest1 * d;
            nv = a.beta2 * nv + a.rest2 * (d * d);
            np -= a.decay * np + a.rate * nm / (sqrtf(nv * a.spread) + a.eps);
        }
        op[i] = np;
        om[i] = nm;
        ov[i] = nv;
        if (a.copy.entries) store_at(a.copy.entry[c.entry].data, a.copy.entry[c.entry].dtype, i, np);
    }
}

hipError_t launch_list_norms(const ListView &g, const Reach &r, double *partial, float *norms, hipStream_t s)
{
    if (g.chunks > 0) hipLaunchKernelGGL(k_list_squares, dim3((unsigned)g.chunks), dim3(256), 0, s, g, partial);
    hipLaunchKernelGGL(k_list_norms, dim3(1), dim3(1024), 0, s, g, r, partial, norms);
    return hipGetLastError();
}

hipError_t launch_list_clip(const ListView &g, const ListView &out, const ClipArgs &c, hipStream_t s)
{
    if (g.chunks > 0) hipLaunchKernelGGL(k_list_clip, dim3((unsigned)g.chunks), dim3(256), 0, s, g, out, c);
    return hipGetLastError();
}

hipError_t launch_list_adam(const AdamArgs &a, hipStream_t s)
{
    if (a.grad.chunks > 0) hipLaunchKernelGGL(k_list_adam, dim3((unsigned)a.grad.chunks), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace dgn
