// Gated linear recurrence over ragged sequences, forward, backward and for one token.
//   decay:    a_t = gate_t,          u_t = x_t
//   sigmoid:  a_t = sigma(gate_t),   u_t = (1 - a_t) x_t
//   h_t = a_t h_{t-1} + u_t
// and, with e_t the gradient of h_t (what reaches y_t and what comes back from h_{t+1}),
//   e_t = dy_t + a_{t+1} e_{t+1},   dh0 = a_0 e_0
//   decay:    dx = e,               dgate = e_t h_{t-1}
//   sigmoid:  dx = (1 - a) e,       dgate = a (1 - a) e_t (h_{t-1} - x_t)
// A gate may be shared by `group` channels; its gradient is then the sum over them.
#include "values.h"

namespace dgn {

enum Kind : int { kDecay = DGN_GATE_DECAY, kSigmoid = DGN_GATE_SIGMOID };

// a and 1 - a of a gate: sigma(-g), not 1 - sigma(g), which loses the digits of a gate that is nearly open.
template <int kKind> __device__ __forceinline__ void open_gate(float g, float &a, float &b)
{
    if (kKind == kDecay) { a = g; b = 1.0f; }
    else { a = sigmoid(g); b = sigmoid(-g); }
}

__device__ __forceinline__ int64_t row_bound(int64_t v, int64_t tokens) { return v < 0 ? 0 : v > tokens ? tokens : v; }

// A thread per sequence and channel, token after token.
template <class T, int kKind>
__global__ __launch_bounds__(64) void k_scan_forward(ScanArgs a)
{
    typedef typename T::Store S;
    const int64_t c = (int64_t)blockIdx.x * 64 + threadIdx.x;
    if (c >= a.channels) return;
    for (int64_t q = blockIdx.y; q < a.seqs; q += gridDim.y) {
    const int64_t from = row_bound(a.rowptr[q], a.tokens), to = row_bound(a.rowptr[q + 1], a.tokens);
    float h = a.h0 ? a.h0[q * a.channels + c] : 0.0f;
    for (int64_t t = from; t < to; t++) {
        if (a.carry && t % kScanTile == 0) a.carry[t / kScanTile * a.channels + c] = h;
        float g, b;
        open_gate<kKind>(to_float<T>(static_cast<const S *>(a.gate)[t * a.gate_stride + c / a.group]), g, b);
        h = g * h + b * to_float<T>(static_cast<const S *>(a.x)[t * a.x_stride + c]);
        static_cast<S *>(a.y)[t * a.y_stride + c] = from_float<T>(h);
    }
    if (a.final) a.final[q * a.channels + c] = h;
    }
}

template <class T, int kKind>
__global__ __launch_bounds__(64) void k_scan_backward(ScanArgs a)
{
    typedef typename T::Store S;
    const int64_t c = (int64_t)blockIdx.x * 64 + threadIdx.x;
    if (c >= a.channels) return;
    for (int64_t q = blockIdx.y; q < a.seqs; q += gridDim.y) {
    const int64_t from = row_bound(a.rowptr[q], a.tokens), to = row_bound(a.rowptr[q + 1], a.tokens);
    const S *x = static_cast<const S *>(a.x) + c, *gate = static_cast<const S *>(a.gate) + c / a.group;
    float e = a.dfinal ? a.dfinal[q * a.channels + c] : 0.0f;
    float before[kScanTile];
    for (int64_t end = to; end > from;) {
        const int64_t tile = (end - 1) / kScanTile, begin = tile * kScanTile > from ? tile * kScanTile : from;
        float h = begin > from ? a.carry[tile * a.channels + c] : a.h0 ? a.h0[q * a.channels + c] : 0.0f;
        for (int64_t t = begin; t < end; t++) {
            float g, b;
            open_gate<kKind>(to_float<T>(gate[t * a.gate_stride]), g, b);
            before[t - begin] = h;
            h = g * h + b * to_float<T>(x[t * a.x_stride]);
        }
        for (int64_t t = end - 1; t >= begin; t--) {
            float g, b;
            open_gate<kKind>(to_float<T>(gate[t * a.gate_stride]), g, b);
            e += to_float<T>(static_cast<const S *>(a.dy)[t * a.dy_stride + c]);
            static_cast<S *>(a.dx)[t * a.dx_stride + c] = from_float<T>(b * e);
            const float prev = before[t - begin];
            const float dg = kKind == kDecay ? e * prev : g * b * (e * (prev - to_float<T>(x[t * a.x_stride])));
            if (a.group == 1) static_cast<S *>(a.dgate)[t * a.dgate_stride + c] = from_float<T>(dg);
            else a.partial[t * a.channels + c] = dg;
            e *= g;
        }
        end = begin;
    }
    if (a.dh0) a.dh0[q * a.channels + c] = e;
    }
}

template <class T>
__global__ __launch_bounds__(64) void k_gate_sums(ScanArgs a)
{
    const int64_t head = (int64_t)blockIdx.x * 64 + threadIdx.x;
    const int64_t first = row_bound(a.rowptr[0], a.tokens), last = row_bound(a.rowptr[a.seqs], a.tokens);
    if (head >= a.heads) return;
    for (int64_t t = first + blockIdx.y; t < last; t += gridDim.y) {
        float sum = 0.0f;
        for (int64_t i = 0; i < a.group; i++) sum += a.partial[t * a.channels + head * a.group + i];
        static_cast<typename T::Store *>(a.dgate)[t * a.dgate_stride + head] = from_float<T>(sum);
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
        open_gate<kKind>(to_float<T>(static_cast<const S *>(a.gate)[row * a.gate_stride + c / a.group]), g, b);
        h = g * a.state_in[slot * a.channels + c] + b * to_float<T>(static_cast<const S *>(a.x)[row * a.x_stride + c]);
        a.state_out[slot * a.channels + c] = h;
    }
    static_cast<S *>(a.y)[row * a.y_stride + c] = from_float<T>(h);
    }
}

size_t scan_scratch_bytes(int64_t tokens, int64_t channels, int64_t group)
{
    return group == 1 ? 0 : (size_t)tokens * channels * 4;
}

#define DGN_BY_TYPE(call)                                                                                     \
    do {                                                                                                      \
        if (dtype == DGN_F32) { typedef F32 T; if (kind == kDecay) call(T, kDecay); else call(T, kSigmoid); } \
        else if (dtype == DGN_F16) { typedef F16 T; if (kind == kDecay) call(T, kDecay); else call(T, kSigmoid); } \
        else { typedef BF16 T; if (kind == kDecay) call(T, kDecay); else call(T, kSigmoid); }                 \
    } while (0)

hipError_t launch_scan_forward(int dtype, int kind, const ScanArgs &a, hipStream_t s)
{
    if (a.channels == 0 || a.seqs == 0) return hipSuccess;
    const dim3 grid((unsigned)((a.channels + 63) / 64), (unsigned)(a.seqs < 32768 ? a.seqs : 32768));
#define DGN_GO(T, K) hipLaunchKernelGGL((k_scan_forward<T, K>), grid, dim3(64), 0, s, a)
    DGN_BY_TYPE(DGN_GO);
#undef DGN_GO
    return hipGetLastError();
}

hipError_t launch_scan_backward(int dtype, int kind, const ScanArgs &a, hipStream_t s)
{
    if (a.channels == 0 || a.seqs == 0) return hipSuccess;
    const dim3 grid((unsigned)((a.channels + 63) / 64), (unsigned)(a.seqs < 32768 ? a.seqs : 32768));
#define DGN_GO(T, K) hipLaunchKernelGGL((k_scan_backward<T, K>), grid, dim3(64), 0, s, a)
    DGN_BY_TYPE(DGN_GO);
#undef DGN_GO
    if (a.group > 1 && a.tokens > 0) {
        const dim3 g((unsigned)((a.heads + 63) / 64), (unsigned)(a.tokens < 16384 ? a.tokens : 16384));
#define DGN_GO(T, K) hipLaunchKernelGGL((k_gate_sums<T>), g, dim3(64), 0, s, a)
        DGN_BY_TYPE(DGN_GO);
#undef DGN_GO
    }
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
