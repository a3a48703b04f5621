// Internal declarations of the operators of a selective recurrent layer (causal_conv.hip, select_forward.hip, select_backward.hip,
// dropout.hip).
#pragma once

#include "values.h"

namespace dgn {

// ---- short causal convolution -------------------------------------------------------------------
struct ConvArgs {
    int64_t tokens, seqs, channels;
    int64_t x_stride, y_stride, dy_stride, dx_stride;
    int32_t taps;
    const void *x;
    const float *weight, *bias;
    const int64_t *rowptr;
    const void *state0;
    void *y, *final;
    const void *dy, *dfinal;
    void *dx;
    float *dweight, *dbias;
    void *dstate0;
    // how rows and channels are cut, and scratch: set at the launch
    int64_t runs, blocks;
    int32_t rows;
    float *partial;                 // [parts][taps + 1][channels]: sums of a workgroup's rows
};
struct ConvStepArgs {
    int64_t rows, slots, channels;
    int64_t x_stride, y_stride;
    const void *x;
    const float *weight, *bias;
    const int32_t *slot;
    const void *state_in;
    void *state_out, *y;
    int64_t pieces;                 // set at the launch
};
bool conv_fits(int dtype, const ConvArgs &a);
size_t conv_scratch_bytes(int dtype, const ConvArgs &a);
hipError_t launch_conv(int dtype, int activation, bool back, const ConvArgs &a, void *scratch, hipStream_t s);
hipError_t launch_conv_step(int dtype, int activation, int taps, const ConvStepArgs &a, hipStream_t s);

// ---- selective scan -------------------------------------------------------------------------------
struct SelectArgs {
    int64_t tokens, seqs, channels, states, groups;
    int64_t x_stride, delta_stride, b_stride, c_stride, z_stride, y_stride;
    int64_t dy_stride, dx_stride, ddelta_stride, db_stride, dc_stride, dz_stride;
    const void *x, *delta, *B, *C, *z;
    const float *A, *D, *delta_bias;
    const int64_t *rowptr;
    const float *h0;
    void *y;
    float *final;
    const void *dy;
    const float *dfinal;
    void *dx, *ddelta, *dB, *dC, *dz;
    float *dA, *dD, *ddelta_bias, *dh0;
    // set at the launch
    int64_t strips, blocks;         // of rows, and of channels in all
    int32_t group_blocks;           // of channels in a group
    int32_t rows;                   // of a strip
    float *ends, *spans;            // what a strip does to a state: [strips][channels][states up to a power of two], sums of d: [strips][channels]
    float *before, *back;           // like ends: what comes into the strip, forward and backward; NULL: few strips
    float *kept;                    // like ends, of every kSelectKeep rows: the state before that row
    float *partial, *shared;        // sums over a strip's rows and over a block's channels
    int64_t slice, slice_strips, slice_rows;    // backward: first strip, strips and rows of a launch
};
struct SelectStepArgs {
    SelectArgs in;                  // tokens: rows
    int64_t slots;
    const int32_t *slot;
    const float *state_in;
    float *state_out;
};
bool select_fits(int dtype, const SelectArgs &a);
size_t select_scratch_bytes(const SelectArgs &a, bool forward_only);
size_t select_carry_bytes(const SelectArgs &a);
hipError_t launch_select(int dtype, bool back, const SelectArgs &a, void *carry, void *scratch, hipStream_t s);
hipError_t launch_select_step(int dtype, const SelectStepArgs &a, hipStream_t s);

// ---- dropout ----------------------------------------------------------------------------------------
struct DropArgs {
    int64_t rows, columns;
    int64_t x_stride, residual_stride, y_stride;
    const void *x, *residual;
    const u64 *key;
    void *y;
    uint32_t drop;                  // of 65 536
    float scale;
};
hipError_t launch_dropout(int dtype, const DropArgs &a, hipStream_t s);

// What neither pass has rows for: out = 0.
hipError_t launch_zero(float *out, int64_t n, hipStream_t s);

}  // namespace dgn
