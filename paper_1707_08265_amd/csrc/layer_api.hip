// C ABI of the operators of a selective recurrent layer (declared in dgn.h): argument checks, then the launches.
#include <math.h>

#include "checks.h"
#include "layer.h"

using namespace dgn;

namespace {

bool sizes_ok(int64_t tokens, int64_t seqs, int64_t channels) { return tokens >= 0 && seqs >= 0 && channels >= 0; }
int check_stride(int64_t stride, int64_t width)
{
    if (stride < 0 || (stride && stride < width)) return DGN_ERR_INVALID_ARG;
    return stride > ((int64_t)1 << 40) ? DGN_ERR_TOO_LARGE : DGN_OK;
}

int check_conv(const dgn_conv_desc *d)
{
    if (!d) return DGN_ERR_NULL_PTR;
    if (!sizes_ok(d->num_tokens, d->num_seqs, d->num_channels) || d->num_taps < 2 || d->num_taps > 4 || !type_known(d->dtype) ||
        (d->activation != DGN_ACT_NONE && d->activation != DGN_ACT_SILU))
        return DGN_ERR_INVALID_ARG;
    if (d->num_tokens > kMaxCount || d->num_seqs > kMaxCount || d->num_channels > kMaxCount) return DGN_ERR_TOO_LARGE;
    const int64_t stride[4] = {d->x_stride, d->y_stride, d->dy_stride, d->dx_stride};
    for (int64_t s : stride) {
        const int rc = check_stride(s, d->num_channels);
        if (rc != DGN_OK) return rc;
    }
    return DGN_OK;
}
ConvArgs conv_args(const dgn_conv_desc *d)
{
    ConvArgs a = {};
    a.tokens = d->num_tokens;
    a.seqs = d->num_seqs;
    a.channels = d->num_channels;
    a.taps = d->num_taps;
    const int64_t c = a.channels;
    a.x_stride = d->x_stride ? d->x_stride : c;
    a.y_stride = d->y_stride ? d->y_stride : c;
    a.dy_stride = d->dy_stride ? d->dy_stride : c;
    a.dx_stride = d->dx_stride ? d->dx_stride : c;
    return a;
}

int check_select(const dgn_select_desc *d)
{
    if (!d) return DGN_ERR_NULL_PTR;
    if (!sizes_ok(d->num_tokens, d->num_seqs, d->num_channels) || !type_known(d->dtype) || d->num_states < 1 || d->num_groups < 1 ||
        (d->forward_only != 0 && d->forward_only != 1))
        return DGN_ERR_INVALID_ARG;
    if (d->num_tokens > kMaxCount || d->num_seqs > kMaxCount || d->num_channels > kMaxCount || d->num_states > 256) return DGN_ERR_TOO_LARGE;
    if (d->num_channels % d->num_groups || d->num_groups > kMaxCount) return DGN_ERR_INVALID_ARG;
    const int64_t wide = d->num_groups * d->num_states;
    const int64_t stride[12] = {d->x_stride, d->delta_stride, d->z_stride, d->y_stride, d->dy_stride, d->dx_stride, d->ddelta_stride,
                                d->dz_stride, d->b_stride, d->c_stride, d->db_stride, d->dc_stride};
    for (int i = 0; i < 12; i++) {
        const int rc = check_stride(stride[i], i < 8 ? d->num_channels : wide);
        if (rc != DGN_OK) return rc;
    }
    return DGN_OK;
}
SelectArgs select_args(const dgn_select_desc *d)
{
    SelectArgs a = {};
    a.tokens = d->num_tokens;
    a.seqs = d->num_seqs;
    a.channels = d->num_channels;
    a.states = d->num_states;
    a.groups = d->num_groups;
    const int64_t c = a.channels, w = a.groups * a.states;
    const auto or_else = [](int64_t stride, int64_t width) { return stride ? stride : width; };
    a.x_stride = or_else(d->x_stride, c);
    a.delta_stride = or_else(d->delta_stride, c);
    a.z_stride = or_else(d->z_stride, c);
    a.y_stride = or_else(d->y_stride, c);
    a.dy_stride = or_else(d->dy_stride, c);
    a.dx_stride = or_else(d->dx_stride, c);
    a.ddelta_stride = or_else(d->ddelta_stride, c);
    a.dz_stride = or_else(d->dz_stride, c);
    a.b_stride = or_else(d->b_stride, w);
    a.c_stride = or_else(d->c_stride, w);
    a.db_stride = or_else(d->db_stride, w);
    a.dc_stride = or_else(d->dc_stride, w);
    return a;
}

// The inputs of a description, checked, and what they take in memory.
struct SelectSpans { Span at[9]; };
int select_inputs(const dgn_select_desc *d, const dgn_select_inputs *in, bool step, SelectArgs *a, SelectSpans *spans)
{
    if (!in) return DGN_ERR_NULL_PTR;
    if (d->num_tokens > 0 && (!in->x || !in->delta || !in->B || !in->C)) return DGN_ERR_NULL_PTR;
    if (!in->A || (!step && !in->seq_rowptr)) return DGN_ERR_NULL_PTR;
    const size_t e = element_size(d->dtype);
    if (misaligned(in->x, e) || misaligned(in->delta, e) || misaligned(in->B, e) || misaligned(in->C, e) || misaligned(in->z, e) ||
        misaligned(in->A, 4) || misaligned(in->D, 4) || misaligned(in->delta_bias, 4) ||
        (!step && (misaligned(in->h0, 4) || misaligned(in->seq_rowptr, 8))))
        return DGN_ERR_INVALID_ARG;
    a->x = in->x;
    a->delta = in->delta;
    a->A = in->A;
    a->B = in->B;
    a->C = in->C;
    a->D = in->D;
    a->delta_bias = in->delta_bias;
    a->z = in->z;
    if (!step) {
        a->rowptr = in->seq_rowptr;
        a->h0 = in->h0;
    }
    const int64_t n = a->tokens, b = e, c = a->channels, w = a->groups * a->states;
    *spans = SelectSpans{{{in->x, n, a->x_stride * b, c * b}, {in->delta, n, a->delta_stride * b, c * b}, {in->z, n, a->z_stride * b, c * b},
                          {in->B, n, a->b_stride * b, w * b}, {in->C, n, a->c_stride * b, w * b}, dense(in->A, c, a->states * 4),
                          dense(in->D, 1, c * 4), dense(in->delta_bias, 1, c * 4), dense(a->rowptr, a->seqs + 1, 8)}};
    return DGN_OK;
}

}  // namespace

extern "C" {

int dgn_conv_workspace(const dgn_conv_desc *d, size_t *scratch_bytes)
{
    const int rc = check_conv(d);
    if (rc != DGN_OK) return rc;
    if (d->num_channels > 0 && !conv_fits(d->dtype, conv_args(d))) return DGN_ERR_TOO_LARGE;
    if (scratch_bytes) *scratch_bytes = d->num_channels > 0 ? round256(conv_scratch_bytes(d->dtype, conv_args(d))) : 0;
    return DGN_OK;
}

int dgn_conv_forward(const dgn_conv_desc *d, const void *x, const float *weight, const float *bias, const int64_t *seq_rowptr,
                     const void *state0, void *y, void *final, void *scratch, size_t scratch_bytes, dgn_stream stream)
{
    size_t need = 0;
    const int rc = dgn_conv_workspace(d, &need);
    if (rc != DGN_OK) return rc;
    if (d->num_channels == 0 || d->num_seqs == 0) return DGN_OK;
    if (!weight || !seq_rowptr || (d->num_tokens > 0 && (!x || !y)) || (need > 0 && !scratch)) return DGN_ERR_NULL_PTR;
    if (scratch_bytes < need) return DGN_ERR_WORKSPACE_TOO_SMALL;
    const size_t e = element_size(d->dtype);
    if (misaligned(x, e) || misaligned(y, e) || misaligned(state0, e) || misaligned(final, e) || misaligned(weight, 4) ||
        misaligned(bias, 4) || misaligned(seq_rowptr, 8) || misaligned(scratch, 8))
        return DGN_ERR_INVALID_ARG;
    ConvArgs a = conv_args(d);
    const int64_t n = a.tokens, b = e, c = a.channels, state = (a.taps - 1) * c * b;
    const Span in[] = {{x, n, a.x_stride * b, c * b}, dense(weight, c, a.taps * 4), dense(bias, 1, c * 4), dense(seq_rowptr, a.seqs + 1, 8)};
    const Span out[] = {{y, n, a.y_stride * b, c * b}, dense(scratch, 1, (int64_t)need), dense(final, a.seqs, state)}, first = dense(state0, a.seqs, state);
    for (int i = 0; i < 3; i++) {
        if (meets(out[i], in) || (i < 2 && meet(out[i], first))) return DGN_ERR_INVALID_ARG;
        for (int k = 0; k < i; k++) if (meet(out[i], out[k])) return DGN_ERR_INVALID_ARG;
    }
    a.x = x;
    a.weight = weight;
    a.bias = bias;
    a.rowptr = seq_rowptr;
    a.state0 = state0;
    a.y = y;
    a.final = final;
    DGN_HIP(launch_conv(d->dtype, d->activation, false, a, scratch, static_cast<hipStream_t>(stream)));
    return DGN_OK;
}

int dgn_conv_backward(const dgn_conv_desc *d, const void *x, const float *weight, const float *bias, const int64_t *seq_rowptr,
                      const void *state0, const void *dy, const void *dfinal, void *dx, float *dweight, float *dbias, void *dstate0,
                      void *scratch, size_t scratch_bytes, dgn_stream stream)
{
    size_t need = 0;
    const int rc = dgn_conv_workspace(d, &need);
    if (rc != DGN_OK) return rc;
    if (d->num_channels == 0) return DGN_OK;
    if (!dweight || (need > 0 && !scratch)) return DGN_ERR_NULL_PTR;
    if (d->num_seqs > 0 && (!weight || !seq_rowptr || (d->num_tokens > 0 && (!x || !dy || !dx)))) return DGN_ERR_NULL_PTR;
    if (scratch_bytes < need) return DGN_ERR_WORKSPACE_TOO_SMALL;
    const size_t e = element_size(d->dtype);
    if (misaligned(x, e) || misaligned(dy, e) || misaligned(dx, e) || misaligned(state0, e) || misaligned(dfinal, e) ||
        misaligned(dstate0, e) || misaligned(weight, 4) || misaligned(bias, 4) || misaligned(dweight, 4) || misaligned(dbias, 4) ||
        misaligned(seq_rowptr, 8) || misaligned(scratch, 8))
        return DGN_ERR_INVALID_ARG;
    ConvArgs a = conv_args(d);
    const int64_t n = a.tokens, b = e, c = a.channels, state = (a.taps - 1) * c * b;
    const Span in[] = {{x, n, a.x_stride * b, c * b}, {dy, n, a.dy_stride * b, c * b}, dense(weight, c, a.taps * 4), dense(bias, 1, c * 4),
                       dense(seq_rowptr, a.seqs + 1, 8), dense(state0, a.seqs, state), dense(dfinal, a.seqs, state)};
    const Span out[] = {{dx, n, a.dx_stride * b, c * b}, dense(dweight, c, a.taps * 4), dense(dbias, 1, c * 4), dense(dstate0, a.seqs, state),
                        dense(scratch, 1, (int64_t)need)};
    for (int i = 0; i < 5; i++) {
        if (meets(out[i], in)) return DGN_ERR_INVALID_ARG;
        for (int k = 0; k < i; k++) if (meet(out[i], out[k])) return DGN_ERR_INVALID_ARG;
    }
    a.x = x;
    a.weight = weight;
    a.bias = bias;
    a.rowptr = seq_rowptr;
    a.state0 = state0;
    a.dy = dy;
    a.dfinal = dfinal;
    a.dx = dx;
    a.dweight = dweight;
    a.dbias = dbias;
    a.dstate0 = dstate0;
    DGN_HIP(launch_conv(d->dtype, d->activation, true, a, scratch, static_cast<hipStream_t>(stream)));
    return DGN_OK;
}

int dgn_conv_step(const dgn_conv_desc *d, int64_t num_slots, const void *x, const float *weight, const float *bias, const int32_t *slots,
                  const void *state_in, void *state_out, void *y, dgn_stream stream)
{
    const int rc = check_conv(d);
    if (rc != DGN_OK) return rc;
    if (num_slots < 0) return DGN_ERR_INVALID_ARG;
    if (num_slots > kMaxCount) return DGN_ERR_TOO_LARGE;
    if (d->num_tokens == 0 || d->num_channels == 0) return DGN_OK;
    if (!x || !weight || !y || (num_slots > 0 && (!state_in || !state_out))) return DGN_ERR_NULL_PTR;
    const size_t e = element_size(d->dtype);
    if (misaligned(x, e) || misaligned(y, e) || misaligned(state_in, e) || misaligned(state_out, e) || misaligned(weight, 4) ||
        misaligned(bias, 4) || misaligned(slots, 4))
        return DGN_ERR_INVALID_ARG;
    const ConvArgs s = conv_args(d);
    const int64_t n = s.tokens, b = e, c = s.channels, state = (s.taps - 1) * c * b;
    const Span in[] = {dense(weight, c, s.taps * 4), dense(bias, 1, c * 4), dense(slots, n, 4)};
    const Span from = {x, n, s.x_stride * b, c * b}, out = {y, n, s.y_stride * b, c * b};
    const Span old = dense(state_in, num_slots, state), now = dense(state_out, num_slots, state);
    if (meets(out, in) || meets(now, in) || meet(out, old) || meet(out, now) || meet(now, from) || (meet(now, old) && state_in != state_out))
        return DGN_ERR_INVALID_ARG;
    if (meet(out, from) && !(x == y && (n == 1 || s.x_stride == s.y_stride))) return DGN_ERR_INVALID_ARG;   // (a thread reads what it writes)
    const ConvStepArgs a = {s.tokens, num_slots, s.channels, s.x_stride, s.y_stride, x, weight, bias, slots, state_in, state_out, y, 0};
    DGN_HIP(launch_conv_step(d->dtype, d->activation, d->num_taps, a, static_cast<hipStream_t>(stream)));
    return DGN_OK;
}

int dgn_select_workspace(const dgn_select_desc *d, size_t *scratch_bytes, size_t *carry_bytes)
{
    const int rc = check_select(d);
    if (rc != DGN_OK) return rc;
    const SelectArgs a = select_args(d);
    if (a.channels > 0 && !select_fits(d->dtype, a)) return DGN_ERR_TOO_LARGE;
    if (scratch_bytes) *scratch_bytes = a.channels > 0 ? round256(select_scratch_bytes(a, d->forward_only)) : 0;
    if (carry_bytes) *carry_bytes = a.channels > 0 && !d->forward_only ? round256(select_carry_bytes(a)) : 0;
    return DGN_OK;
}

int dgn_select_forward(const dgn_select_desc *d, const dgn_select_inputs *in, void *y, float *final, void *carry, void *scratch,
                       size_t scratch_bytes, dgn_stream stream)
{
    size_t need = 0, kept = 0;
    int rc = dgn_select_workspace(d, &need, &kept);
    if (rc != DGN_OK) return rc;
    if (d->num_channels == 0 || d->num_seqs == 0) return DGN_OK;
    SelectArgs a = select_args(d);
    SelectSpans spans;
    rc = select_inputs(d, in, false, &a, &spans);
    if (rc != DGN_OK) return rc;
    if ((d->num_tokens > 0 && !y) || (need > 0 && !scratch)) return DGN_ERR_NULL_PTR;
    if (scratch_bytes < need) return DGN_ERR_WORKSPACE_TOO_SMALL;
    const size_t e = element_size(d->dtype);
    if (misaligned(y, e) || misaligned(final, 4) || misaligned(carry, 16) || misaligned(scratch, 16) || (carry && d->forward_only))
        return DGN_ERR_INVALID_ARG;
    const int64_t b = e, c = a.channels, state = c * a.states * 4;
    const Span first = dense(a.h0, a.seqs, state), last = dense(final, a.seqs, state);
    const Span out[] = {{y, a.tokens, a.y_stride * b, c * b}, dense(carry, 1, (int64_t)kept), dense(scratch, 1, (int64_t)need), last};
    for (int i = 0; i < 4; i++) {
        if (meets(out[i], spans.at) || (i < 3 && meet(out[i], first))) return DGN_ERR_INVALID_ARG;
        for (int k = 0; k < i; k++) if (meet(out[i], out[k])) return DGN_ERR_INVALID_ARG;
    }
    a.y = y;
    a.final = final;
    DGN_HIP(launch_select(d->dtype, false, a, carry, scratch, static_cast<hipStream_t>(stream)));
    return DGN_OK;
}

int dgn_select_backward(const dgn_select_desc *d, const dgn_select_inputs *in, const void *carry, const void *dy, const float *dfinal,
                        const dgn_select_grads *g, void *scratch, size_t scratch_bytes, dgn_stream stream)
{
    size_t need = 0, kept = 0;
    int rc = dgn_select_workspace(d, &need, &kept);
    if (rc != DGN_OK) return rc;
    if (d->forward_only) return DGN_ERR_INVALID_ARG;
    if (!g) return DGN_ERR_NULL_PTR;
    if (d->num_channels == 0) return DGN_OK;
    if (!g->dA) return DGN_ERR_NULL_PTR;
    if (misaligned(g->dA, 4) || misaligned(g->dD, 4) || misaligned(g->ddelta_bias, 4) || misaligned(g->dh0, 4)) return DGN_ERR_INVALID_ARG;
    SelectArgs a = select_args(d);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (d->num_seqs == 0) {             // (no rows count)
        DGN_HIP(launch_zero(g->dA, a.channels * a.states, s));
        DGN_HIP(launch_zero(g->dD, a.channels, s));
        DGN_HIP(launch_zero(g->ddelta_bias, a.channels, s));
        return DGN_OK;
    }
    SelectSpans spans;
    rc = select_inputs(d, in, false, &a, &spans);
    if (rc != DGN_OK) return rc;
    if (d->num_tokens > 0 && (!carry || !dy || !g->dx || !g->ddelta || !g->dB || !g->dC || (in->z && !g->dz))) return DGN_ERR_NULL_PTR;
    if (need > 0 && !scratch) return DGN_ERR_NULL_PTR;
    if (scratch_bytes < need) return DGN_ERR_WORKSPACE_TOO_SMALL;
    const size_t e = element_size(d->dtype);
    if (misaligned(dy, e) || misaligned(g->dx, e) || misaligned(g->ddelta, e) || misaligned(g->dB, e) || misaligned(g->dC, e) ||
        misaligned(g->dz, e) || misaligned(dfinal, 4) || misaligned(carry, 16) || misaligned(scratch, 16))
        return DGN_ERR_INVALID_ARG;
    const int64_t n = a.tokens, b = e, c = a.channels, w = a.groups * a.states, state = c * a.states * 4;
    const Span more[] = {dense(a.h0, a.seqs, state), dense(dfinal, a.seqs, state), {dy, n, a.dy_stride * b, c * b}, dense(carry, 1, (int64_t)kept)};
    const Span out[] = {{g->dx, n, a.dx_stride * b, c * b}, {g->ddelta, n, a.ddelta_stride * b, c * b},
                        {in->z ? g->dz : nullptr, n, a.dz_stride * b, c * b}, {g->dB, n, a.db_stride * b, w * b},
                        {g->dC, n, a.dc_stride * b, w * b}, dense(g->dA, c, a.states * 4), dense(g->dD, 1, c * 4),
                        dense(g->ddelta_bias, 1, c * 4), dense(g->dh0, a.seqs, state), dense(scratch, 1, (int64_t)need)};
    for (int i = 0; i < 10; i++) {
        if (meets(out[i], spans.at) || meets(out[i], more)) return DGN_ERR_INVALID_ARG;
        for (int k = 0; k < i; k++) if (meet(out[i], out[k])) return DGN_ERR_INVALID_ARG;
    }
    a.dy = dy;
    a.dfinal = dfinal;
    a.dx = g->dx;
    a.ddelta = g->ddelta;
    a.dB = g->dB;
    a.dC = g->dC;
    a.dz = in->z ? g->dz : nullptr;
    a.dA = g->dA;
    a.dD = g->dD;
    a.ddelta_bias = g->ddelta_bias;
    a.dh0 = g->dh0;
    DGN_HIP(launch_select(d->dtype, true, a, const_cast<void *>(carry), scratch, s));
    return DGN_OK;
}

int dgn_select_step(const dgn_select_desc *d, int64_t num_slots, const dgn_select_inputs *in, const int32_t *slots, const float *state_in,
                    float *state_out, void *y, dgn_stream stream)
{
    int rc = check_select(d);
    if (rc != DGN_OK) return rc;
    if (num_slots < 0) return DGN_ERR_INVALID_ARG;
    if (num_slots > kMaxCount) return DGN_ERR_TOO_LARGE;
    if (d->num_tokens == 0 || d->num_channels == 0) return DGN_OK;
    SelectStepArgs a = {};
    a.in = select_args(d);
    a.in.seqs = 0;
    SelectSpans spans;
    rc = select_inputs(d, in, true, &a.in, &spans);
    if (rc != DGN_OK) return rc;
    if (!y || (num_slots > 0 && (!state_in || !state_out))) return DGN_ERR_NULL_PTR;
    const size_t e = element_size(d->dtype);
    if (misaligned(y, e) || misaligned(state_in, 4) || misaligned(state_out, 4) || misaligned(slots, 4)) return DGN_ERR_INVALID_ARG;
    const int64_t n = a.in.tokens, b = e, c = a.in.channels, state = c * a.in.states * 4;
    const Span out = {y, n, a.in.y_stride * b, c * b}, old = dense(state_in, num_slots, state), now = dense(state_out, num_slots, state),
               which = dense(slots, n, 4);
    if (meets(now, spans.at) || meet(now, which) || meet(out, which) || meet(out, old) || meet(out, now) ||
        (meet(now, old) && state_in != state_out))
        return DGN_ERR_INVALID_ARG;
    for (int i = 0; i < 9; i++) {               // (x, delta and z: the lanes that write an element have read it, in the same wave)
        const bool same = i < 3 && spans.at[i].at == y && (n == 1 || spans.at[i].stride == out.stride);
        if (meet(out, spans.at[i]) && !same) return DGN_ERR_INVALID_ARG;
    }
    a.slots = num_slots;
    a.slot = slots;
    a.state_in = state_in;
    a.state_out = state_out;
    a.in.y = y;
    DGN_HIP(launch_select_step(d->dtype, a, static_cast<hipStream_t>(stream)));
    return DGN_OK;
}

int dgn_dropout(const dgn_dropout_desc *d, const void *x, const void *residual, const uint64_t *key, void *y, dgn_stream stream)
{
    if (!d) return DGN_ERR_NULL_PTR;
    if (d->num_rows < 0 || d->num_columns < 0 || !type_known(d->dtype) || !(d->rate >= 0.0 && d->rate <= 1.0)) return DGN_ERR_INVALID_ARG;
    if (d->num_rows > kMaxCount || d->num_columns > kMaxCount) return DGN_ERR_TOO_LARGE;
    const int64_t stride[3] = {d->x_stride, d->residual_stride, d->y_stride};
    for (int64_t s : stride) {
        const int rc = check_stride(s, d->num_columns);
        if (rc != DGN_OK) return rc;
    }
    if (d->num_rows == 0 || d->num_columns == 0) return DGN_OK;
    if (!x || !key || !y) return DGN_ERR_NULL_PTR;
    const size_t e = element_size(d->dtype);
    if (misaligned(x, e) || misaligned(residual, e) || misaligned(y, e) || misaligned(key, 8)) return DGN_ERR_INVALID_ARG;
    DropArgs a = {};
    a.rows = d->num_rows;
    a.columns = d->num_columns;
    const int64_t c = a.columns, b = e;
    a.x_stride = d->x_stride ? d->x_stride : c;
    a.residual_stride = d->residual_stride ? d->residual_stride : c;
    a.y_stride = d->y_stride ? d->y_stride : c;
    const Span out = {y, a.rows, a.y_stride * b, c * b};
    const Span in[] = {{x, a.rows, a.x_stride * b, c * b}, {residual, a.rows, a.residual_stride * b, c * b}};
    if (meet(out, dense(key, 1, 16))) return DGN_ERR_INVALID_ARG;
    for (const Span &from : in) {               // (a thread reads its elements before it writes the same ones)
        const bool same = from.at == y && (a.rows == 1 || from.stride == out.stride);
        if (meet(out, from) && !same) return DGN_ERR_INVALID_ARG;
    }
    a.x = x;
    a.residual = residual;
    a.key = reinterpret_cast<const u64 *>(key);
    a.y = y;
    a.drop = (uint32_t)floor(d->rate * 65536.0 + 0.5);
    a.scale = a.drop < 65536 ? (float)(65536.0 / (65536.0 - a.drop)) : 0.0f;
    DGN_HIP(launch_dropout(d->dtype, a, static_cast<hipStream_t>(stream)));
    return DGN_OK;
}

}  // extern "C"
