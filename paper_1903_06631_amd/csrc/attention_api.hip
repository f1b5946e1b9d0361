// extern "C" entry points of the attention and cache operators: argument checks, workspace carving, launches.
#include <math.h>
#include <stdio.h>

#include <algorithm>
#include <initializer_list>

#include "../../include/lap.h"
#include "attn_kernels.h"

namespace {

constexpr size_t ALIGN = 256;
inline size_t up(size_t x) { return (x + ALIGN - 1) / ALIGN * ALIGN; }

#define LAP_HIP(expr)                                                                          \
    do {                                                                                       \
        const hipError_t lap_e_ = (expr);                                                      \
        if (lap_e_ != hipSuccess) {                                                            \
            fprintf(stderr, "liblap: %s failed: %s\n", #expr, hipGetErrorString(lap_e_));      \
            return LAP_E_HIP;                                                                  \
        }                                                                                      \
    } while (0)

int check_ws(void *ws, size_t have, size_t need)
{
    if (need == 0) return LAP_OK;
    return !ws || ((uintptr_t)ws % ALIGN) != 0 || have < need ? LAP_E_WORKSPACE : LAP_OK;
}

constexpr uint32_t MAX_LEN = 1u << 30, MAX_ITEMS = 1u << 30, MAX_GRID = 65535;
constexpr int64_t MAX_ROW_STRIDE = 1 << 24;

// The dimensions of rows that have more than one place; the others' strides are nobody's business.
struct Dim {
    int64_t stride, extent;
};
int dims_of(const lap_rows *x, uint64_t batch, uint64_t heads, uint64_t len, Dim (&d)[3])
{
    int n = 0;
    if (batch > 1) d[n++] = {x->batch, (int64_t)batch};
    if (heads > 1) d[n++] = {x->head, (int64_t)heads};
    if (len > 1) d[n++] = {x->row, (int64_t)len};
    return n;
}

// Whether two rows of head_dim elements, places apart by these strides, share an element.
bool rows_overlap(Dim (&d)[3], int n, int64_t head_dim)
{
    std::sort(d, d + n, [](const Dim &a, const Dim &b) { return a.stride < b.stride; });
    __int128 span = head_dim;      // the elements from the first to the last of all dimensions so far
    int i = 0;
    for (; i < n && d[i].stride >= span; ++i) span += (__int128)d[i].stride * (d[i].extent - 1);
    if (i == n) return false;      // one within the other, as views of a tensor are
    if (d[0].stride < head_dim) return true;
    // Two or three dimensions that reach into each other: two rows are nearer than head_dim if for some number of steps along
    // all dimensions but the one with most places, a number of steps along that one comes near to minus as much.
    std::sort(d, d + n, [](const Dim &a, const Dim &b) { return a.extent < b.extent; });
    const Dim last = d[n - 1], first = n == 3 ? d[0] : Dim{0, 1}, second = d[n - 2];
    for (int64_t a = 0; a < first.extent; ++a)      // (the other half are these with all signs turned round)
        for (int64_t b = a ? 1 - second.extent : 0; b < second.extent; ++b) {
            const __int128 away = (__int128)a * first.stride + (__int128)b * second.stride;
            const __int128 c = away >= 0 ? away / last.stride : -((-away + last.stride - 1) / last.stride);
            for (__int128 k = c; k <= c + 1; ++k) {
                const __int128 gap = away - k * last.stride;
                if (k > -last.extent && k < last.extent && (a || b || k) && gap > -head_dim && gap < head_dim) return true;
            }
        }
    return false;
}

// rows x of [batch, heads, len]; an output's rows have to be apart from each other
int check_rows(const lap_rows *x, uint64_t batch, uint64_t heads, uint64_t len, uint32_t head_dim, bool output)
{
    if (!x) return LAP_E_NULL;
    if (batch * heads * len == 0) return LAP_OK;
    if (!x->data) return LAP_E_NULL;
    if ((uintptr_t)x->data % 16) return LAP_E_LAYOUT;
    Dim d[3];
    const int n = dims_of(x, batch, heads, len, d);
    for (int i = 0; i < n; ++i)
        if (d[i].stride < 0 || d[i].stride % 8) return LAP_E_LAYOUT;
    if (len > 1 && x->row >= MAX_ROW_STRIDE) return LAP_E_LAYOUT;
    return output && rows_overlap(d, n, head_dim) ? LAP_E_LAYOUT : LAP_OK;
}

// An output that starts where something does that is read, or written, for other rows than those that are written.  (That
// memory is shared in other ways is not looked for: rows of one tensor may stand between those of another.)
int check_apart(const void *output, std::initializer_list<const void *> others)
{
    for (const void *x : others)
        if (x && x == output) return LAP_E_LAYOUT;
    return LAP_OK;
}

int check_shape(const lap_attention_shape *s)
{
    if (!s) return LAP_E_NULL;
    if (s->type != LAP_T_BF16 && s->type != LAP_T_F16) return LAP_E_ATTENTION;
    if (!s->batch || !s->q_heads || !s->kv_heads || !s->head_dim) return LAP_E_SIZE;
    if (s->head_dim > LAP_MAX_HEAD_DIM || s->q_len > MAX_LEN || s->k_len > MAX_LEN) return LAP_E_SIZE;
    if ((uint64_t)s->batch * s->q_heads > MAX_GRID * 16ull) return LAP_E_SIZE;
    if ((uint64_t)s->batch * s->q_heads * (((uint64_t)s->q_len + s->k_len) / 32 + 2) > MAX_ITEMS) return LAP_E_SIZE;
    if (s->head_dim % 8) return LAP_E_LAYOUT;
    if (s->q_heads % s->kv_heads) return LAP_E_ATTENTION;
    if (s->causal > 1 || (s->window && !s->causal) || s->window > MAX_LEN) return LAP_E_ATTENTION;
    if (!(s->scale > 0.f) || s->scale > 1e6f) return LAP_E_ATTENTION;
    return LAP_OK;
}

lap::AttnShape shape_of(const lap_attention_shape *s)
{
    return {s->batch, s->q_heads, s->kv_heads, s->q_len, s->k_len, s->head_dim, (int32_t)s->causal, (int32_t)s->window, s->scale,
            s->q_lens, s->k_lens, s->type == LAP_T_F16};
}
// strides of one place are not used: 0
lap::Rows rows_of(const lap_rows *x, uint64_t batch, uint64_t heads, uint64_t len)
{
    return {x->data, batch > 1 ? x->batch : 0, heads > 1 ? x->head : 0, len > 1 ? x->row : 0};
}
lap::Rows queries_of(const lap_attention_shape *s, const lap_rows *x) { return rows_of(x, s->batch, s->q_heads, s->q_len); }
lap::Rows keys_of(const lap_attention_shape *s, const lap_rows *x) { return rows_of(x, s->batch, s->kv_heads, s->k_len); }

lap::StepShape step_of(const lap_attention_shape *s)
{
    lap::StepShape p = {s->batch, s->q_heads, s->kv_heads, s->k_len, s->head_dim, s->scale, s->k_lens, s->type == LAP_T_F16, 0, 0, 0, false};
    lap::step_split(p);
    return p;
}
inline size_t padded_dim(const lap_attention_shape *s) { return s->head_dim <= 64 ? 64 : 128; }

size_t ws_stats(const lap_attention_shape *s) { return up((size_t)s->batch * s->q_heads * s->q_len * 2 * sizeof(float)); }
size_t ws_grad(const lap_attention_shape *s) { return ws_stats(s) + up(lap::grad_sums(shape_of(s))); }
size_t ws_weights(const lap_attention_shape *s)
{
    const uint32_t parts = lap::weights_parts(shape_of(s));
    return parts == 1 ? 0 : up((size_t)s->batch * s->kv_heads * parts * s->k_len * 4);
}
size_t ws_step(const lap_attention_shape *s)
{
    const lap::StepShape p = step_of(s);
    const size_t heads = (size_t)s->batch * s->q_heads;
    return p.whole ? up(heads * p.score_row * 4) : up(heads * p.splits * padded_dim(s) * 4) + up(heads * p.splits * sizeof(float2)) + up(heads * p.score_row * 4);
}

lap::Rows slots_of(const lap_cache *c, const lap_rows *x) { return rows_of(x, c->batch, c->kv_heads, c->slots); }

int check_cache(const lap_cache *c, bool output)
{
    if (!c) return LAP_E_NULL;
    if (c->type != LAP_T_BF16 && c->type != LAP_T_F16) return LAP_E_ATTENTION;
    if (!c->batch || !c->kv_heads || !c->head_dim) return LAP_E_SIZE;
    if (c->head_dim > LAP_MAX_HEAD_DIM || c->slots > MAX_LEN || (uint64_t)c->batch * c->kv_heads > MAX_GRID) return LAP_E_SIZE;
    if (c->head_dim % 8) return LAP_E_LAYOUT;
    const int rc = check_rows(&c->k, c->batch, c->kv_heads, c->slots, c->head_dim, output);
    return rc ? rc : check_rows(&c->v, c->batch, c->kv_heads, c->slots, c->head_dim, output);
}

}  // namespace

extern "C" {

size_t lap_attention_workspace_bytes(int which_call, const lap_attention_shape *s)
{
    if (check_shape(s)) return 0;
    switch (which_call) {
    case LAP_AT_FORWARD: return up(lap::forward_workspace(shape_of(s)));
    case LAP_AT_GRAD: return ws_grad(s);
    case LAP_AT_WEIGHTS: return ws_weights(s);
    case LAP_AT_STEP: return ws_step(s);
    default: return 0;
    }
}

size_t lap_cache_workspace_bytes(const lap_cache *to)
{
    if (!to) return 0;
    return up((size_t)to->batch * to->kv_heads * to->slots * 4);
}

int lap_attention(const lap_attention_shape *s, const lap_rows *q, const lap_rows *k, const lap_rows *v, const lap_rows *out, float *lse,
                  void *ws, size_t ws_bytes, void *hip_stream)
{
    int rc = check_shape(s);
    if (!rc) rc = check_rows(q, s->batch, s->q_heads, s->q_len, s->head_dim, false);
    if (!rc) rc = check_rows(k, s->batch, s->kv_heads, s->k_len, s->head_dim, false);
    if (!rc) rc = check_rows(v, s->batch, s->kv_heads, s->k_len, s->head_dim, false);
    if (!rc) rc = check_rows(out, s->batch, s->q_heads, s->q_len, s->head_dim, true);
    if (!rc && s->q_len && !lse) rc = LAP_E_NULL;
    if (!rc) rc = check_ws(ws, ws_bytes, up(lap::forward_workspace(shape_of(s))));
    if (rc || !s->q_len) return rc;
    if (s->k_len) rc = check_apart(out->data, {k->data, v->data});
    if (rc) return rc;
    LAP_HIP(lap::launch_attention(shape_of(s), queries_of(s, q), keys_of(s, k), keys_of(s, v), queries_of(s, out), lse, ws, (hipStream_t)hip_stream));
    return LAP_OK;
}

int lap_attention_grad(const lap_attention_shape *s, const lap_rows *dout, const lap_rows *q, const lap_rows *k, const lap_rows *v,
                       const lap_rows *out, const float *lse, const lap_rows *dq, const lap_rows *dk, const lap_rows *dv,
                       void *ws, size_t ws_bytes, void *hip_stream)
{
    int rc = check_shape(s);
    for (const lap_rows *x : {dout, q, out})
        if (!rc) rc = check_rows(x, s->batch, s->q_heads, s->q_len, s->head_dim, false);
    for (const lap_rows *x : {k, v})
        if (!rc) rc = check_rows(x, s->batch, s->kv_heads, s->k_len, s->head_dim, false);
    if (!rc) rc = check_rows(dq, s->batch, s->q_heads, s->q_len, s->head_dim, true);
    for (const lap_rows *x : {dk, dv})
        if (!rc) rc = check_rows(x, s->batch, s->kv_heads, s->k_len, s->head_dim, true);
    if (!rc && s->q_len && !lse) rc = LAP_E_NULL;
    if (!rc) rc = check_ws(ws, ws_bytes, ws_grad(s));
    if (rc || (!s->q_len && !s->k_len)) return rc;
    if (s->q_len && s->k_len) {      // the first kernel writes dq while it streams k and v, the second dk and dv while it streams q and dout
        rc = check_apart(dq->data, {q->data, dout->data, k->data, v->data, dk->data, dv->data});
        if (!rc) rc = check_apart(dk->data, {q->data, dout->data, dv->data});
        if (!rc) rc = check_apart(dv->data, {q->data, dout->data});
        if (rc) return rc;
    }
    LAP_HIP(lap::launch_attention_grad(shape_of(s), {queries_of(s, dout), queries_of(s, q), keys_of(s, k), keys_of(s, v), queries_of(s, out), queries_of(s, dq),
                                                     keys_of(s, dk), keys_of(s, dv), lse, (float *)ws, (float *)((char *)ws + ws_stats(s))}, (hipStream_t)hip_stream));
    return LAP_OK;
}

int lap_attention_weights(const lap_attention_shape *s, const lap_rows *q, const lap_rows *k, const float *lse, const float *before,
                          float *weights, void *ws, size_t ws_bytes, void *hip_stream)
{
    int rc = check_shape(s);
    if (!rc) rc = check_rows(q, s->batch, s->q_heads, s->q_len, s->head_dim, false);
    if (!rc) rc = check_rows(k, s->batch, s->kv_heads, s->k_len, s->head_dim, false);
    if (!rc && ((s->q_len && !lse) || (s->k_len && !weights))) rc = LAP_E_NULL;
    if (!rc) rc = check_ws(ws, ws_bytes, ws_weights(s));
    if (rc || !s->k_len) return rc;
    if (s->q_len) rc = check_apart(weights, {lse, q->data, k->data});
    if (rc) return rc;
    LAP_HIP(lap::launch_attention_weights(shape_of(s), queries_of(s, q), keys_of(s, k), lse, before, weights, (float *)ws, (hipStream_t)hip_stream));
    return LAP_OK;
}

int lap_attention_step(const lap_attention_shape *s, const lap_rows *q, const lap_rows *k, const lap_rows *v, const int32_t *positions,
                       const float *before, const lap_rows *out, float *lse, float *weights, void *ws, size_t ws_bytes, void *hip_stream)
{
    int rc = check_shape(s);
    if (!rc && (s->q_len != 1 || s->causal || s->q_lens)) rc = LAP_E_ATTENTION;
    if (!rc && (s->q_heads / s->kv_heads > lap::MAX_GROUP)) rc = LAP_E_SIZE;
    if (!rc) rc = check_rows(q, s->batch, s->q_heads, 1, s->head_dim, false);
    if (!rc) rc = check_rows(k, s->batch, s->kv_heads, s->k_len, s->head_dim, false);
    if (!rc) rc = check_rows(v, s->batch, s->kv_heads, s->k_len, s->head_dim, false);
    if (!rc) rc = check_rows(out, s->batch, s->q_heads, 1, s->head_dim, true);
    if (!rc && (!lse || (before != nullptr) != (weights != nullptr))) rc = LAP_E_NULL;
    if (!rc) rc = check_ws(ws, ws_bytes, ws_step(s));
    if (!rc && s->k_len) rc = check_apart(out->data, {k->data, v->data});
    if (rc) return rc;
    const lap::StepShape p = step_of(s);
    const size_t heads = (size_t)s->batch * s->q_heads;
    lap::StepWork w = {queries_of(s, q), keys_of(s, k), keys_of(s, v), queries_of(s, out), positions, before, lse, weights, nullptr, nullptr, nullptr};
    char *at = (char *)ws;
    if (!p.whole) {
        w.outs = (float *)at, at += up(heads * p.splits * padded_dim(s) * 4);
        w.sums = (float2 *)at, at += up(heads * p.splits * sizeof(float2));
    }
    w.scores = (float *)at;
    LAP_HIP(lap::launch_attention_step(p, w, (hipStream_t)hip_stream));
    return LAP_OK;
}

int lap_cache_evict(const lap_cache *from, const int32_t *lens, uint32_t keep, uint32_t recent, const lap_cache *to, int32_t *lens_out,
                    void *ws, size_t ws_bytes, void *hip_stream)
{
    int rc = check_cache(from, false);
    if (!rc) rc = check_cache(to, true);
    if (rc) return rc;
    if (from->type != to->type || from->batch != to->batch || from->kv_heads != to->kv_heads || from->head_dim != to->head_dim)
        return LAP_E_ATTENTION;
    if (keep == 0 || keep > to->slots || recent > keep) return LAP_E_SIZE;
    if ((from->slots && !from->weights) || !to->weights || !to->positions || !lens_out) return LAP_E_NULL;
    rc = check_ws(ws, ws_bytes, lap_cache_workspace_bytes(to));
    if (!rc) rc = check_apart(to->k.data, {to->v.data});
    if (!rc && from->slots) {
        rc = check_apart(to->k.data, {from->k.data, from->v.data});
        if (!rc) rc = check_apart(to->v.data, {from->k.data, from->v.data});
        if (!rc) rc = check_apart(to->weights, {from->weights});
        if (!rc) rc = check_apart(to->positions, {from->positions});
    }
    if (rc) return rc;
    const lap::EvictShape s = {from->batch, from->kv_heads, from->slots, to->slots, from->head_dim, keep, recent, lens};
    LAP_HIP(lap::launch_cache_evict(s, slots_of(from, &from->k), slots_of(from, &from->v), from->weights, from->positions, slots_of(to, &to->k),
                                    slots_of(to, &to->v), to->weights, to->positions, lens_out, (int32_t *)ws, (hipStream_t)hip_stream));
    return LAP_OK;
}

int lap_cache_insert(const lap_cache *c, const lap_rows *k_new, const lap_rows *v_new, const int32_t *position, uint32_t recent,
                     int32_t *slots, void *hip_stream)
{
    int rc = check_cache(c, true);
    if (rc) return rc;
    if (c->slots == 0 || recent > c->slots) return LAP_E_SIZE;
    rc = check_rows(k_new, c->batch, c->kv_heads, 1, c->head_dim, false);
    if (!rc) rc = check_rows(v_new, c->batch, c->kv_heads, 1, c->head_dim, false);
    if (rc) return rc;
    if (!c->weights || !c->positions || !position || !slots) return LAP_E_NULL;
    const lap::InsertShape s = {c->batch, c->kv_heads, c->slots, c->head_dim, recent};
    LAP_HIP(lap::launch_cache_insert(s, rows_of(k_new, c->batch, c->kv_heads, 1), rows_of(v_new, c->batch, c->kv_heads, 1),
                                     slots_of(c, &c->k), slots_of(c, &c->v), c->weights, c->positions, position,
                                     slots, (hipStream_t)hip_stream));
    return LAP_OK;
}

}  // extern "C"
