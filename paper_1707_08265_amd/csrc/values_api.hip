// C ABI of the operators on tensor values (declared in dgn.h): argument checks, then the launches.
#include <math.h>
#include <new>
#include <string.h>

#include "checks.h"

using namespace dgn;

struct dgn_list {
    ListView v;
    int64_t count;
    int64_t *numel;         // host copy: lists that are used together have to agree
    int32_t *dtype;
    bool all_f32;
};

namespace {

int check_scan(const dgn_scan_desc *d)
{
    if (!d) return DGN_ERR_NULL_PTR;
    if (d->num_tokens < 0 || d->num_seqs < 0 || d->num_channels < 0 || d->gate_group < 1) return DGN_ERR_INVALID_ARG;
    if (!type_known(d->dtype) || (d->gate_kind != DGN_GATE_DECAY && d->gate_kind != DGN_GATE_SIGMOID)) return DGN_ERR_INVALID_ARG;
    if (d->num_tokens > kMaxCount || d->num_seqs > kMaxCount || d->num_channels > kMaxCount) return DGN_ERR_TOO_LARGE;
    if (d->num_channels % d->gate_group) return DGN_ERR_INVALID_ARG;
    const int64_t heads = d->num_channels / d->gate_group;
    const int64_t stride[6] = {d->x_stride, d->y_stride, d->dy_stride, d->dx_stride, d->gate_stride, d->dgate_stride};
    for (int i = 0; i < 6; i++) {
        if (stride[i] < 0 || (stride[i] && stride[i] < (i < 4 ? d->num_channels : heads))) return DGN_ERR_INVALID_ARG;
        if (stride[i] > ((int64_t)1 << 40)) return DGN_ERR_TOO_LARGE;
    }
    return DGN_OK;
}

ScanArgs scan_args(const dgn_scan_desc *d)
{
    ScanArgs a = {};
    a.tokens = d->num_tokens;
    a.seqs = d->num_seqs;
    a.channels = d->num_channels;
    a.group = d->gate_group;
    a.heads = d->num_channels / d->gate_group;
    const int64_t c = a.channels, h = a.heads;
    a.x_stride = d->x_stride ? d->x_stride : c;
    a.y_stride = d->y_stride ? d->y_stride : c;
    a.dy_stride = d->dy_stride ? d->dy_stride : c;
    a.dx_stride = d->dx_stride ? d->dx_stride : c;
    a.gate_stride = d->gate_stride ? d->gate_stride : h;
    a.dgate_stride = d->dgate_stride ? d->dgate_stride : h;
    return a;
}

int check_reach(const dgn_reach *r, const dgn_list *l, Reach *out)
{
    *out = Reach{nullptr, 0, nullptr, 1};
    if (!r) return DGN_OK;
    if (r->num_sets < 1 || r->num_sets > DGN_MAX_SETS) return DGN_ERR_TOO_MANY_SETS;
    if (r->num_words < 0) return DGN_ERR_INVALID_ARG;
    if (misaligned(r->tensor_mask, 8) || misaligned(r->tensor_ids, 4)) return DGN_ERR_INVALID_ARG;
    if (r->tensor_mask && !r->tensor_ids && r->num_words < l->count) return DGN_ERR_INVALID_ARG;
    if (!r->tensor_mask && r->num_words > 0) return DGN_ERR_NULL_PTR;
    out->mask = reinterpret_cast<const u64 *>(r->tensor_mask);
    out->words = r->num_words;
    out->ids = r->tensor_ids;
    out->sets = r->num_sets;
    return DGN_OK;
}

bool same_sizes(const dgn_list *a, const dgn_list *b)
{
    return a == b || (a->count == b->count && (a->count == 0 || memcmp(a->numel, b->numel, sizeof(int64_t) * a->count) == 0));
}

int check_list(const dgn_list_desc *d, int64_t *chunks)
{
    if (!d) return DGN_ERR_NULL_PTR;
    if (d->count < 0) return DGN_ERR_INVALID_ARG;
    if (d->count > kMaxCount) return DGN_ERR_TOO_LARGE;
    if (d->count > 0 && (!d->data || !d->numel || !d->dtype)) return DGN_ERR_NULL_PTR;
    int64_t n = 0;
    for (int64_t i = 0; i < d->count; i++) {
        if (d->numel[i] < 0 || !type_known(d->dtype[i])) return DGN_ERR_INVALID_ARG;
        if (d->numel[i] > ((int64_t)1 << 44)) return DGN_ERR_TOO_LARGE;
        n += (d->numel[i] + kListChunk - 1) / kListChunk;
        if (n > kMaxCount / 1024) return DGN_ERR_TOO_LARGE;      // a launch holds less than 2^32 threads
        if (d->numel[i] > 0 && !d->data[i]) return DGN_ERR_NULL_PTR;
        if (misaligned(d->data[i], element_size(d->dtype[i]))) return DGN_ERR_INVALID_ARG;
    }
    *chunks = n;
    return DGN_OK;
}

size_t list_bytes_of(int64_t chunks)
{
    return round256(sizeof(ListChunk) * (size_t)chunks) + 256;
}

}  // namespace

extern "C" {

int dgn_scan_workspace(const dgn_scan_desc *d, size_t *scratch_bytes, size_t *carry_bytes)
{
    const int rc = check_scan(d);
    if (rc != DGN_OK) return rc;
    if (d->num_channels > 0 && !scan_fits(d->dtype, scan_args(d))) return DGN_ERR_TOO_LARGE;
    if (scratch_bytes) *scratch_bytes = d->num_channels > 0 ? round256(scan_scratch_bytes(d->dtype, scan_args(d))) : 0;
    if (carry_bytes) *carry_bytes = round256((size_t)((d->num_tokens + kScanKeep - 1) / kScanKeep) * d->num_channels * 4);
    return DGN_OK;
}

int dgn_scan_forward(const dgn_scan_desc *d, const void *x, const void *gate, const int64_t *seq_rowptr, const float *h0, void *y,
                     float *final, void *carry, void *scratch, size_t scratch_bytes, dgn_stream stream)
{
    int rc = check_scan(d);
    if (rc != DGN_OK) return rc;
    if (d->num_channels == 0 || d->num_seqs == 0) return DGN_OK;
    size_t need = 0;
    rc = dgn_scan_workspace(d, &need, nullptr);
    if (rc != DGN_OK) return rc;
    if (!seq_rowptr || (d->num_tokens > 0 && (!x || !gate || !y)) || (need > 0 && !scratch)) return DGN_ERR_NULL_PTR;
    if (scratch_bytes < need) return DGN_ERR_WORKSPACE_TOO_SMALL;
    const size_t e = element_size(d->dtype);
    if (misaligned(x, e) || misaligned(gate, e) || misaligned(y, e) || misaligned(h0, 4) || misaligned(final, 4) ||
        misaligned(seq_rowptr, 8) || misaligned(carry, 4) || misaligned(scratch, 8))
        return DGN_ERR_INVALID_ARG;
    ScanArgs a = scan_args(d);
    const int64_t n = a.tokens, b = e, state = a.channels * 4;
    const Span in[] = {{x, n, a.x_stride * b, a.channels * b}, {gate, n, a.gate_stride * b, a.heads * b}, dense(seq_rowptr, a.seqs + 1, 8)};
    const Span out = {y, n, a.y_stride * b, a.channels * b}, last = dense(final, a.seqs, state);
    if (meets(out, in) || meets(last, in) || meet(out, last) || meet(out, dense(h0, a.seqs, state))) return DGN_ERR_INVALID_ARG;
    a.x = x;
    a.gate = gate;
    a.rowptr = seq_rowptr;
    a.h0 = h0;
    a.y = y;
    a.final = final;
    a.kept = static_cast<float *>(carry);
    DGN_HIP(launch_scan(d->dtype, d->gate_kind, false, a, scratch, static_cast<hipStream_t>(stream)));
    return DGN_OK;
}

int dgn_scan_backward(const dgn_scan_desc *d, const void *x, const void *gate, const int64_t *seq_rowptr, const float *h0,
                      const void *carry, const void *dy, const float *dfinal, void *dx, void *dgate, float *dh0, void *scratch,
                      size_t scratch_bytes, dgn_stream stream)
{
    int rc = check_scan(d);
    if (rc != DGN_OK) return rc;
    if (d->num_channels == 0 || d->num_seqs == 0) return DGN_OK;
    size_t need = 0;
    rc = dgn_scan_workspace(d, &need, nullptr);
    if (rc != DGN_OK) return rc;
    if (!seq_rowptr || (d->num_tokens > 0 && (!x || !gate || !dy || !dx || !dgate || !carry)) || (need > 0 && !scratch))
        return DGN_ERR_NULL_PTR;
    if (scratch_bytes < need) return DGN_ERR_WORKSPACE_TOO_SMALL;
    const size_t e = element_size(d->dtype);
    if (misaligned(x, e) || misaligned(gate, e) || misaligned(dy, e) || misaligned(dx, e) || misaligned(dgate, e) ||
        misaligned(h0, 4) || misaligned(dfinal, 4) || misaligned(dh0, 4) || misaligned(seq_rowptr, 8) || misaligned(carry, 4) ||
        misaligned(scratch, 8))
        return DGN_ERR_INVALID_ARG;
    ScanArgs a = scan_args(d);
    const int64_t n = a.tokens, b = e, state = a.channels * 4;
    const Span in[] = {{x, n, a.x_stride * b, a.channels * b}, {gate, n, a.gate_stride * b, a.heads * b}, dense(seq_rowptr, a.seqs + 1, 8),
                       {dy, n, a.dy_stride * b, a.channels * b}};
    const Span states[] = {dense(h0, a.seqs, state), dense(dfinal, a.seqs, state), dense(dh0, a.seqs, state)};
    const Span wide = {dx, n, a.dx_stride * b, a.channels * b}, gates = {dgate, n, a.dgate_stride * b, a.heads * b};
    if (meets(wide, in) || meets(gates, in) || meets(states[2], in) || meet(wide, gates) || meets(wide, states) || meets(gates, states) ||
        (meet(states[2], states[0]) && dh0 != h0))              // (dh0 in h0's place: each state is read before it is written)
        return DGN_ERR_INVALID_ARG;
    a.x = x;
    a.gate = gate;
    a.rowptr = seq_rowptr;
    a.h0 = h0;
    a.kept = const_cast<float *>(static_cast<const float *>(carry));
    a.dy = dy;
    a.dfinal = dfinal;
    a.dx = dx;
    a.dgate = dgate;
    a.dh0 = dh0;
    DGN_HIP(launch_scan(d->dtype, d->gate_kind, true, a, scratch, static_cast<hipStream_t>(stream)));
    return DGN_OK;
}

int dgn_scan_step(const dgn_scan_desc *d, int64_t num_slots, const void *x, const void *gate, const int32_t *slots,
                  const float *state_in, float *state_out, void *y, dgn_stream stream)
{
    const int rc = check_scan(d);
    if (rc != DGN_OK) return rc;
    if (num_slots < 0) return DGN_ERR_INVALID_ARG;
    if (num_slots > kMaxCount) return DGN_ERR_TOO_LARGE;
    if (d->num_tokens == 0 || d->num_channels == 0) return DGN_OK;
    if (!x || !gate || !y || (num_slots > 0 && (!state_in || !state_out))) return DGN_ERR_NULL_PTR;
    const size_t e = element_size(d->dtype);
    if (misaligned(x, e) || misaligned(gate, e) || misaligned(y, e) || misaligned(state_in, 4) || misaligned(state_out, 4) ||
        misaligned(slots, 4))
        return DGN_ERR_INVALID_ARG;
    const ScanArgs s = scan_args(d);
    const int64_t n = s.tokens, b = e, state = s.channels * 4;
    const Span in[] = {{x, n, s.x_stride * b, s.channels * b}, {gate, n, s.gate_stride * b, s.heads * b}, dense(slots, n, 4)};
    const Span out = {y, n, s.y_stride * b, s.channels * b}, from = dense(state_in, num_slots, state), to = dense(state_out, num_slots, state);
    if (meets(to, in) || meet(out, to) || meet(out, from) || (meet(to, from) && state_in != state_out)) return DGN_ERR_INVALID_ARG;
    for (int k = 0; k < 3; k++) {       // (each thread reads its elements of x and gate before it writes the same ones)
        const bool same = k < 2 && in[k].at == y && in[k].width == out.width && (n == 1 || in[k].stride == out.stride);
        if (meet(out, in[k]) && !same) return DGN_ERR_INVALID_ARG;
    }
    const StepArgs a = {s.tokens, num_slots, s.channels, s.group, s.x_stride, s.gate_stride, s.y_stride, x, gate, slots, state_in,
                        state_out, y, 0};
    DGN_HIP(launch_scan_step(d->dtype, d->gate_kind, a, static_cast<hipStream_t>(stream)));
    return DGN_OK;
}

int dgn_list_workspace(const dgn_list_desc *d, size_t *list_bytes)
{
    if (!list_bytes) return DGN_ERR_NULL_PTR;
    int64_t chunks = 0;
    const int rc = check_list(d, &chunks);
    if (rc != DGN_OK) return rc;
    *list_bytes = list_bytes_of(chunks);
    return DGN_OK;
}

int dgn_list_build(const dgn_list_desc *d, void *list_mem, size_t list_bytes, dgn_stream stream, dgn_list **out)
{
    if (!out || !list_mem) return DGN_ERR_NULL_PTR;
    *out = nullptr;
    int64_t chunks = 0;
    const int rc = check_list(d, &chunks);
    if (rc != DGN_OK) return rc;
    const size_t need = list_bytes_of(chunks);
    if (list_bytes < need) return DGN_ERR_WORKSPACE_TOO_SMALL;
    if (misaligned(list_mem, 16)) return DGN_ERR_INVALID_ARG;
    dgn_list *l = new (std::nothrow) dgn_list();
    if (!l) return note_hip_error(hipErrorOutOfMemory);
    ListChunk *chunk = new (std::nothrow) ListChunk[need / sizeof(ListChunk)]();
    l->numel = new (std::nothrow) int64_t[d->count + 1];
    l->dtype = new (std::nothrow) int32_t[d->count + 1];
    if (!chunk || !l->numel || !l->dtype) {
        delete[] chunk;
        dgn_list_destroy(l);
        return note_hip_error(hipErrorOutOfMemory);
    }
    int32_t n = 0;
    l->all_f32 = true;
    for (int64_t i = 0; i < d->count; i++) {
        l->numel[i] = d->numel[i];
        l->v.elements += d->numel[i];
        l->v.bytes += (size_t)d->numel[i] * element_size(d->dtype[i]);
        l->dtype[i] = d->dtype[i];
        l->all_f32 = l->all_f32 && d->dtype[i] == DGN_F32;
        for (int64_t at = 0; at < d->numel[i]; at += kListChunk) {
            const int64_t left = d->numel[i] - at, of = left < kListChunk ? left : kListChunk;
            chunk[n++] = ListChunk{static_cast<char *>(d->data[i]) + at * element_size(d->dtype[i]), (uint32_t)i, (uint32_t)(of * 4 + d->dtype[i])};
        }
    }
    l->count = d->count;
    l->v.chunk = static_cast<const ListChunk *>(list_mem);
    l->v.chunks = n;
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = hipMemcpyAsync(list_mem, chunk, need, hipMemcpyHostToDevice, s);
    if (e == hipSuccess) e = hipStreamSynchronize(s);
    delete[] chunk;
    if (e != hipSuccess) {
        dgn_list_destroy(l);
        return note_hip_error(e);
    }
    *out = l;
    return DGN_OK;
}

void dgn_list_destroy(dgn_list *l)
{
    if (!l) return;
    delete[] l->numel;
    delete[] l->dtype;
    delete l;
}

int dgn_list_norms_workspace(const dgn_list *l, size_t *scratch_bytes)
{
    if (!l || !scratch_bytes) return DGN_ERR_NULL_PTR;
    *scratch_bytes = round256(list_norms_scratch_bytes(l->v));
    return DGN_OK;
}

int dgn_list_norms(const dgn_list *l, const dgn_reach *reach, float *norms, void *scratch, size_t scratch_bytes, dgn_stream stream)
{
    if (!l || !norms || !scratch) return DGN_ERR_NULL_PTR;
    Reach r;
    int rc = check_reach(reach, l, &r);
    if (rc != DGN_OK) return rc;
    size_t need = 0;
    rc = dgn_list_norms_workspace(l, &need);
    if (rc != DGN_OK) return rc;
    if (scratch_bytes < need) return DGN_ERR_WORKSPACE_TOO_SMALL;
    if (misaligned(scratch, 8) || misaligned(norms, 4)) return DGN_ERR_INVALID_ARG;
    DGN_HIP(launch_list_norms(l->v, r, scratch, norms, static_cast<hipStream_t>(stream)));
    return DGN_OK;
}

int dgn_list_clip(const dgn_list *l, const dgn_list *out, const dgn_reach *reach, const float *norms, float max_norm, float eps,
                  dgn_stream stream)
{
    if (!l || !out || !norms) return DGN_ERR_NULL_PTR;
    Reach r;
    const int rc = check_reach(reach, l, &r);
    if (rc != DGN_OK) return rc;
    if (!(max_norm >= 0.0f) || !(eps >= 0.0f) || misaligned(norms, 4) || !same_sizes(l, out)) return DGN_ERR_INVALID_ARG;
    if (l->count > 0 && memcmp(l->dtype, out->dtype, sizeof(int32_t) * l->count)) return DGN_ERR_INVALID_ARG;
    const ClipArgs c = {r, norms, max_norm, eps};
    DGN_HIP(launch_list_clip(l->v, out->v, c, static_cast<hipStream_t>(stream)));
    return DGN_OK;
}

int dgn_list_adam(const dgn_adam_lists *ls, const dgn_reach *reach, const float *norms, const dgn_adam_options *o, dgn_stream stream)
{
    if (!ls || !o || !ls->grad || !ls->param || !ls->m || !ls->v) return DGN_ERR_NULL_PTR;
    const dgn_list *out_p = ls->out_param ? ls->out_param : ls->param, *out_m = ls->out_m ? ls->out_m : ls->m,
                   *out_v = ls->out_v ? ls->out_v : ls->v;
    const dgn_list *all[7] = {ls->param, ls->m, ls->v, out_p, out_m, out_v, ls->copy};
    AdamArgs a = {};
    const int rc = check_reach(reach, ls->grad, &a.clip.reach);
    if (rc != DGN_OK) return rc;
    for (int i = 0; i < 7; i++) {
        if (!all[i]) continue;                                   // (no copy asked for)
        if (!same_sizes(ls->grad, all[i]) || (i < 6 && !all[i]->all_f32)) return DGN_ERR_INVALID_ARG;
    }
    if (!(o->lr >= 0.0) || !(o->beta1 >= 0.0 && o->beta1 < 1.0) || !(o->beta2 >= 0.0 && o->beta2 < 1.0) || !(o->eps >= 0.0) ||
        !(o->weight_decay >= 0.0) || o->step < 1)
        return DGN_ERR_INVALID_ARG;
    if (norms && (!(o->max_norm >= 0.0f) || !(o->clip_eps >= 0.0f) || misaligned(norms, 4))) return DGN_ERR_INVALID_ARG;
    a.grad = ls->grad->v;
    a.param = ls->param->v;
    a.m = ls->m->v;
    a.v = ls->v->v;
    a.out_param = out_p->v;
    a.out_m = out_m->v;
    a.out_v = out_v->v;
    if (ls->copy) a.copy = ls->copy->v;
    a.clip.norms = norms;
    a.clip.max_norm = o->max_norm;
    a.clip.eps = o->clip_eps;
    a.rate = (float)(o->lr / (1.0 - pow(o->beta1, (double)o->step)));
    a.spread = (float)(1.0 / (1.0 - pow(o->beta2, (double)o->step)));
    a.beta1 = (float)o->beta1;
    a.rest1 = (float)(1.0 - o->beta1);
    a.beta2 = (float)o->beta2;
    a.rest2 = (float)(1.0 - o->beta2);
    a.eps = (float)o->eps;
    a.decay = (float)(o->lr * o->weight_decay);
    a.skip_nonfinite = o->skip_nonfinite;
    DGN_HIP(launch_list_adam(a, static_cast<hipStream_t>(stream)));
    return DGN_OK;
}

}  // extern "C"
