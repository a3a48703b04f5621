// Internal declarations of the operators on tensor values (gated_scan.hip, tensor_lists.hip).
#pragma once

#include "common.h"

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

namespace dgn {

// Element types in memory; arithmetic is in 32 bits throughout, conversions round to nearest, ties to even.
struct F32 { typedef float Store; };
struct F16 { typedef _Float16 Store; };
struct BF16 { typedef __bf16 Store; };

inline int element_size(int32_t dtype) { return dtype == DGN_F32 ? 4 : 2; }
// call(T) for the element type.
#define DGN_BY_DTYPE(dtype, call)                 \
    do {                                          \
        if ((dtype) == DGN_F32) { call(F32); }    \
        else if ((dtype) == DGN_F16) { call(F16); } \
        else { call(BF16); }                      \
    } while (0)

// Past the caches where kStream (see kStreamBytes).  kAlign: what the address is aligned to (a number, as a type's alignment does not pass
// through a template).
template <class V, int kAlign> struct Placed { typedef V At __attribute__((aligned(kAlign))); };
template <bool kStream, int kAlign, class V> __device__ __forceinline__ V take(const void *p)
{
    typedef typename Placed<V, kAlign>::At At;
    return kStream ? __builtin_nontemporal_load(static_cast<const At *>(p)) : *static_cast<const At *>(p);
}
template <bool kStream, int kAlign, class V> __device__ __forceinline__ void put(void *p, V v)
{
    typedef typename Placed<V, kAlign>::At At;
    if (kStream) __builtin_nontemporal_store(v, static_cast<At *>(p));
    else *static_cast<At *>(p) = v;
}
// What lanes of a wave wrote to LDS is there for the others.
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// ---- gated linear recurrence --------------------------------------------------------------------
constexpr int kScanKeep = 16;       // rows between two states that the forward pass keeps for the backward pass
struct ScanArgs {
    int64_t tokens, seqs, channels, group, heads;
    int64_t x_stride, gate_stride, y_stride, dy_stride, dx_stride, dgate_stride;
    const void *x, *gate;
    const int64_t *rowptr;
    const float *h0;
    void *y;
    float *final;
    float *kept;                    // [ceil(tokens / kScanKeep)][channels]: the state before that row
    const void *dy;
    const float *dfinal;
    void *dx, *dgate;
    float *dh0;
    // how rows and channels are cut (see gated_scan.hip), and scratch: set at the launch
    int64_t strips, blocks, rows;
    int32_t width, parts;
    u64 *words;                     // [strips][blocks][64 V]: what a strip does to a state
    float *states;                  // the same: the state that comes into it; NULL: few strips
    float *partial;                 // gates shared by more channels than a wave has: [parts][tokens][heads]
};
struct StepArgs {
    int64_t rows, slots, channels, group;
    int64_t x_stride, gate_stride, y_stride;
    const void *x, *gate;
    const int32_t *slot;
    const float *state_in;
    float *state_out;
    void *y;
    int64_t pieces;                 // set at the launch
};
bool scan_fits(int dtype, const ScanArgs &a);
size_t scan_scratch_bytes(int dtype, const ScanArgs &a);
hipError_t launch_scan(int dtype, int kind, bool back, const ScanArgs &a, void *scratch, hipStream_t s);
hipError_t launch_scan_step(int dtype, int kind, const StepArgs &a, hipStream_t s);

// ---- lists of tensors -----------------------------------------------------------------------------
constexpr int kListChunk = 8192;    // elements of a chunk
struct alignas(16) ListChunk { void *data; uint32_t entry, n_type; };    // its first element, the tensor it is of, elements * 4 + type
static_assert(sizeof(ListChunk) == 16, "a chunk is one load");
struct ListView { const ListChunk *chunk; int32_t chunks; int64_t elements; size_t bytes; };

struct Reach { const u64 *mask; int64_t words; const int32_t *ids; int32_t sets; };   // which sets reach an entry: see reach_of
struct ClipArgs { Reach reach; const float *norms; float max_norm, eps; };
struct AdamArgs {
    ListView grad, param, m, v, out_param, out_m, out_v, copy;     // copy.chunk == NULL: none
    ClipArgs clip;                                                  // norms == NULL: no clipping
    float rate, beta1, rest1, beta2, rest2, eps, decay;                           // rate = lr / (1 - beta1^t), decay = lr * weight decay, rest = 1 - beta
    float spread;                                                   // 1 / (1 - beta2^t)
    int32_t skip_nonfinite;
};
size_t list_norms_scratch_bytes(const ListView &g);
hipError_t launch_list_norms(const ListView &g, const Reach &r, void *scratch, float *norms, hipStream_t s);
hipError_t launch_list_clip(const ListView &g, const ListView &out, const ClipArgs &c, hipStream_t s);
hipError_t launch_list_adam(const AdamArgs &a, hipStream_t s);

}  // namespace dgn
