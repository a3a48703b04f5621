// Internal declarations of the operators on tensor values (gated_scan.hip, tensor_lists.hip).
#pragma once

#include "common.h"

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

namespace dgn {

// Element types in memory; arithmetic is in 32 bits throughout.
struct F32 { typedef float Store; };
struct F16 { typedef _Float16 Store; };
struct BF16 { typedef __bf16 Store; };

template <class T> __device__ __forceinline__ float to_float(typename T::Store v) { return (float)v; }
template <class T> __device__ __forceinline__ typename T::Store from_float(float v) { return (typename T::Store)v; }   // nearest, ties to even

inline int element_size(int32_t dtype) { return dtype == DGN_F32 ? 4 : 2; }

// 1 / (1 + exp(-v)): without overflow for either sign, 0 and 1 at the infinities, NaN for NaN.
__device__ __forceinline__ float sigmoid(float v) { return 1.0f / (1.0f + __expf(-v)); }

// ---- gated linear recurrence --------------------------------------------------------------------
constexpr int kScanTile = 128;      // tokens between two states that the forward pass keeps for the backward pass
struct ScanArgs {
    int64_t tokens, seqs, channels, group, heads;
    int64_t x_stride, gate_stride, y_stride, dy_stride, dx_stride, dgate_stride;
    const void *x, *gate;
    const int64_t *rowptr;
    const float *h0;
    void *y;
    float *final;
    float *carry;                   // [ceil(tokens / kScanTile)][channels]: the state before the tile's first token
    const void *dy;
    const float *dfinal;
    void *dx, *dgate;
    float *dh0;
    float *partial;                 // shared gates: a gate's gradient per channel, [tokens][channels]
};
struct StepArgs {
    int64_t rows, slots, channels, group;
    int64_t x_stride, gate_stride, y_stride;
    const void *x, *gate;
    const int32_t *slot;
    const float *state_in;
    float *state_out;
    void *y;
};
size_t scan_scratch_bytes(int64_t tokens, int64_t channels, int64_t group);
hipError_t launch_scan_forward(int dtype, int kind, const ScanArgs &a, hipStream_t s);
hipError_t launch_scan_backward(int dtype, int kind, const ScanArgs &a, hipStream_t s);
hipError_t launch_scan_step(int dtype, int kind, const StepArgs &a, hipStream_t s);

// ---- lists of tensors -----------------------------------------------------------------------------
constexpr int kListChunk = 16384;   // elements that a workgroup takes
struct ListEntry { void *data; int64_t numel; int32_t dtype, first_chunk; };
struct ListChunk { int32_t entry, index; };
struct ListView { const ListEntry *entry; const ListChunk *chunk; int32_t entries, chunks; };

struct Reach { const u64 *mask; int64_t words; const int32_t *ids; int32_t sets; };   // which sets reach an entry: see reach_of
struct ClipArgs { Reach reach; const float *norms; float max_norm, eps; };
struct AdamArgs {
    ListView grad, param, m, v, out_param, out_m, out_v, copy;     // copy.entries == 0: none
    ClipArgs clip;                                                  // norms == NULL: no clipping
    float rate, beta1, rest1, beta2, rest2, eps, decay;                           // rate = lr / (1 - beta1^t), decay = lr * weight decay, rest = 1 - beta
    float spread;                                                   // 1 / (1 - beta2^t)
    int32_t skip_nonfinite;
};
hipError_t launch_list_norms(const ListView &g, const Reach &r, double *partial, float *norms, hipStream_t s);
hipError_t launch_list_clip(const ListView &g, const ListView &out, const ClipArgs &c, hipStream_t s);
hipError_t launch_list_adam(const AdamArgs &a, hipStream_t s);

}  // namespace dgn
