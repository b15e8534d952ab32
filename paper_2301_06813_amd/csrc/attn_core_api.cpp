// attn_core_api.cpp -- C ABI of softmax attention (include/sbp.h, "softmax
// attention"): argument checks and operand mapping, then the launches of
// attn_core_fwd.hip or attn_core_bwd.hip. Every check happens on the host before
// any HIP call.
#include <math.h>
#include <stdint.h>

#include "../../include/sbp.h"
#include "api_internal.h"
#include "attn_core.h"
#include "attn_views.h"

namespace {

using namespace sbpa;

constexpr int64_t MAX_ROWS = int64_t(1) << 29;   // i + len_k - len_q + window fits 32 bits
constexpr int64_t MAX_DIM = 128;
constexpr float MIN_SCALE = 0x1p-100f;

// check_view4, and element offsets that stay inside 62 bits.
int check_bounded(const sbp_view4_t *v) {
    int rc = check_view4(v);
    if (rc) return rc;
    const double last = (double)v->batch * (double)v->stride_b +
                        (double)v->heads * (double)v->stride_h + (double)v->rows * (double)v->ld +
                        (double)v->cols;
    return last > 1e18 ? SBP_ERR_SHAPE : SBP_OK;
}

// Two outputs of the same element size whose rows interleave in one buffer -- the
// Q, K and V parts of a fused gradient -- and so share spans but no element: equal
// row and batch strides, every head of a row inside [0, ld), and the two footprints
// disjoint within a row.
bool interleaved(const sbp_view4_t *x, const sbp_view4_t *y) {
    if (x->dtype != y->dtype || x->ld != y->ld || x->rows != y->rows) return false;
    if (x->batch > 1 && (x->stride_b != y->stride_b || x->stride_b < x->rows * x->ld)) return false;
    const int64_t fx = (x->heads - 1) * x->stride_h + x->cols;
    const int64_t fy = (y->heads - 1) * y->stride_h + y->cols;
    const sbp_view4_t *a = x, *b = y;
    int64_t fa = fx, fb = fy;
    if (reinterpret_cast<uintptr_t>(b->data) < reinterpret_cast<uintptr_t>(a->data)) {
        std::swap(a, b);
        std::swap(fa, fb);
    }
    const uintptr_t gap =
        reinterpret_cast<uintptr_t>(b->data) - reinterpret_cast<uintptr_t>(a->data);
    if (gap % elsz(a->dtype)) return false;
    const int64_t at = (int64_t)(gap / elsz(a->dtype));
    return fa <= at && at + fb <= a->ld;
}

bool outputs_clash(const sbp_view4_t *x, const sbp_view4_t *y) {
    return overlap(span4(x->data, x, x->heads), span4(y->data, y, y->heads)) && !interleaved(x, y);
}

// The call's operands on rank r: Q's heads are split in groups, one group per key
// head of the rank's share.
struct Call {
    sbpi::CoreArgs a;
    int64_t hq = 0, hk = 0;        // local heads
    int64_t q0 = 0;                // rank's first query head
    int64_t H = 0;                 // query heads of the GLOBAL views, or hq
};

sbpi::CoreView kernel_view(const sbp_view4_t *v, int64_t first_head) {
    sbpi::CoreView o;
    o.p = v->data;
    if (o.p && v->heads > 0)
        o.p = static_cast<char *>(v->data) + first_head * v->stride_h * elsz(v->dtype);
    o.sb = v->stride_b;
    o.sh = v->stride_h;
    o.ld = v->ld;
    return o;
}

// Checks Q, K, V, the options and the rank; fills the shapes and views of them.
int prepare(const sbp_view4_t *Q, const sbp_view4_t *K, const sbp_view4_t *V,
            const sbp_attn_opts_t *opts, int32_t p, int32_t r, Call *c) {
    if (!Q || !K || !V || !opts) return SBP_ERR_NULL;
    const sbp_view4_t *ins[3] = {Q, K, V};
    for (const sbp_view4_t *v : ins) {
        int rc = check_bounded(v);
        if (rc) return rc;
        if (v->dtype != SBP_BF16) return SBP_ERR_DTYPE;
        if (v->scope != SBP_GLOBAL && v->scope != SBP_LOCAL) return SBP_ERR_SHAPE;
        if (v->scope != Q->scope || v->batch != Q->batch || v->cols != Q->cols ||
            v->rows > MAX_ROWS)
            return SBP_ERR_SHAPE;
    }
    if (p < 1 || r < 0 || r >= p) return SBP_ERR_LAYOUT;
    if (Q->cols < 1 || Q->cols > MAX_DIM) return SBP_ERR_SHAPE;
    if (K->heads != V->heads || K->rows != V->rows) return SBP_ERR_SHAPE;
    if (K->heads == 0 ? Q->heads != 0 : Q->heads % K->heads != 0) return SBP_ERR_SHAPE;
    // (beyond these scales lse / scale, or the scale in base 2 times small scores, leaves fp32)
    if (!(opts->scale >= MIN_SCALE && opts->scale <= 1.f / MIN_SCALE) || opts->window < 0 ||
        (opts->causal != 0 && opts->causal != 1))
        return SBP_ERR_SHAPE;
    for (const int32_t *len : {opts->len_q, opts->len_k})
        if (reinterpret_cast<uintptr_t>(len) % 4) return SBP_ERR_ALIGN;
    const int64_t group = K->heads ? Q->heads / K->heads : 1;
    int64_t k0 = 0;
    c->hk = K->heads;
    if (Q->scope == SBP_GLOBAL) head_split(K->heads, p, r, &k0, &c->hk);
    c->hq = c->hk * group;
    c->q0 = k0 * group;
    c->H = Q->heads;
    // packed rows fit 31 bits; the launches' threads (256 for 32 packed rows or keys, or
    // for 16 rows of statistics) fit 32
    if (Q->rows * group > INT32_MAX - 128) return SBP_ERR_SHAPE;
    const double heads = (double)Q->batch * (double)c->hk;
    const double tiles = heads * (double)std::max((Q->rows * group + 31) / 32, (K->rows + 31) / 32);
    if (tiles > 16777215.0 || heads * (double)(Q->rows * group) > 268435440.0) return SBP_ERR_SHAPE;
    sbpi::CoreArgs &a = c->a;
    a = sbpi::CoreArgs{};
    a.q = kernel_view(Q, c->q0);
    a.k = kernel_view(K, k0);
    a.v = kernel_view(V, k0);
    a.batch = (int32_t)Q->batch;
    a.kv_heads = (int32_t)c->hk;
    a.group = (int32_t)group;
    a.sq = (int32_t)Q->rows;
    a.sk = (int32_t)K->rows;
    a.d = (int32_t)Q->cols;
    a.causal = opts->causal;
    // a window as long as the keys hides none of them
    a.window = opts->window >= K->rows ? 0 : opts->window;
    a.len_q = opts->len_q;
    a.len_k = opts->len_k;
    a.scale = opts->scale;
    return SBP_OK;
}

// An operand over the rank's query heads: GLOBAL (all H heads) or LOCAL.
int query_operand(const sbp_view4_t *v, const Call &c, const sbp_view4_t *Q, int64_t cols,
                  sbpi::CoreView *out) {
    int rc = check_bounded(v);
    if (rc) return rc;
    if (v->batch != Q->batch || v->rows != Q->rows || v->cols != cols) return SBP_ERR_SHAPE;
    if (v->scope == SBP_GLOBAL) {
        if (Q->scope != SBP_GLOBAL ? v->heads != c.hq : v->heads != c.H) return SBP_ERR_SHAPE;
        *out = kernel_view(v, v->heads == c.H ? c.q0 : 0);
    } else if (v->scope == SBP_LOCAL) {
        if (v->heads != c.hq) return SBP_ERR_SHAPE;
        *out = kernel_view(v, 0);
    } else {
        return SBP_ERR_SHAPE;
    }
    return SBP_OK;
}

// An output of `heads` local heads.
int output(const sbp_view4_t *v, int64_t batch, int64_t heads, int64_t rows, int64_t cols,
           sbpi::CoreView *out) {
    int rc = check_bounded(v);
    if (rc) return rc;
    if (v->batch != batch || v->heads != heads || v->rows != rows || v->cols != cols)
        return SBP_ERR_SHAPE;
    if (v->scope == SBP_ACCUMULATE && v->dtype != SBP_F32) return SBP_ERR_DTYPE;
    if (!injective(v)) return SBP_ERR_SHAPE;
    *out = kernel_view(v, 0);
    return SBP_OK;
}

std::pair<uintptr_t, uintptr_t> span_of(const sbpi::CoreView &v, const sbp_view4_t *s,
                                        int64_t heads) {
    return span4(v.p, s, heads);
}

// 16-byte rows, and tile offsets that fit a 31-bit buffer offset (256 rows at most).
bool rows16(const sbpi::CoreView &v, int64_t d) {
    return reinterpret_cast<uintptr_t>(v.p) % 16 == 0 && v.ld % 8 == 0 && v.sb % 8 == 0 &&
           v.sh % 8 == 0 && d % 8 == 0 && v.ld < (int64_t(1) << 21);
}

std::pair<uintptr_t, uintptr_t> lens_span(const int32_t *p, int64_t batch) {
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    return p ? std::make_pair(b, b + (uintptr_t)(4 * batch)) : std::make_pair(uintptr_t(0), uintptr_t(0));
}

int check_ws(const sbp_workspace_t *ws, sbpi::CoreArgs *a,
             std::pair<uintptr_t, uintptr_t> *span) {
    *span = {0, 0};
    if (!ws || ws->bytes == 0) return SBP_OK;
    if (ws->bytes < 0) return SBP_ERR_SHAPE;
    if (!ws->data) return SBP_ERR_NULL;
    const uintptr_t b = reinterpret_cast<uintptr_t>(ws->data);
    if (b & 15) return SBP_ERR_ALIGN;
    a->ws = static_cast<float *>(ws->data);
    a->ws_floats = (size_t)ws->bytes / sizeof(float);
    *span = {b, b + (uintptr_t)ws->bytes};
    return SBP_OK;
}

int finish(hipError_t e) { return e == hipSuccess ? SBP_OK : hip_error(e); }

}  // namespace

extern "C" {

int sbp_attn_core_fwd(const sbp_view4_t *Q, const sbp_view4_t *K, const sbp_view4_t *V,
                      const sbp_attn_opts_t *opts, sbp_view4_t *O, sbp_view4_t *lse, int32_t p,
                      int32_t r, const sbp_workspace_t *ws, hipStream_t stream) {
    if (!O) return SBP_ERR_NULL;
    Call c;
    int rc = prepare(Q, K, V, opts, p, r, &c);
    if (rc) return rc;
    sbpi::CoreArgs &a = c.a;
    if (O->scope == SBP_ACCUMULATE || (lse && lse->scope == SBP_ACCUMULATE)) return SBP_ERR_SHAPE;
    if ((rc = output(O, Q->batch, c.hq, Q->rows, Q->cols, &a.o))) return rc;
    a.o_f32 = O->dtype == SBP_F32;
    if (lse) {
        if ((rc = output(lse, Q->batch, c.hq, Q->rows, 1, &a.lse))) return rc;
        if (lse->dtype != SBP_F32) return SBP_ERR_DTYPE;
    }
    std::pair<uintptr_t, uintptr_t> wspan;
    if ((rc = check_ws(ws, &a, &wspan))) return rc;
    const std::pair<uintptr_t, uintptr_t> ins[5] = {
        span_of(a.q, Q, c.hq), span_of(a.k, K, c.hk), span_of(a.v, V, c.hk),
        lens_span(a.len_q, Q->batch), lens_span(a.len_k, Q->batch)};
    const auto os = span4(O->data, O, c.hq);
    const auto ls = lse ? span4(lse->data, lse, c.hq) : std::pair<uintptr_t, uintptr_t>(0, 0);
    for (const auto &x : ins)
        if (overlap(x, os) || overlap(x, ls) || overlap(x, wspan)) return SBP_ERR_ALIAS;
    if (overlap(os, ls) || overlap(os, wspan) || overlap(ls, wspan)) return SBP_ERR_ALIAS;
    if (a.batch == 0 || c.hq == 0 || a.sq == 0) return SBP_OK;
    a.aligned = rows16(a.q, a.d) && rows16(a.k, a.d) && rows16(a.v, a.d);
    return finish(sbpi::launch_core_fwd(a, stream));
}

int sbp_attn_core_bwd(const sbp_view4_t *dO, const sbp_view4_t *Q, const sbp_view4_t *K,
                      const sbp_view4_t *V, const sbp_view4_t *O, const sbp_view4_t *lse,
                      const sbp_attn_opts_t *opts, sbp_view4_t *dQ, sbp_view4_t *dK,
                      sbp_view4_t *dV, int32_t p, int32_t r, const sbp_workspace_t *ws,
                      hipStream_t stream) {
    if (!dO || !O || !lse || !dQ || !dK || !dV) return SBP_ERR_NULL;
    Call c;
    int rc = prepare(Q, K, V, opts, p, r, &c);
    if (rc) return rc;
    sbpi::CoreArgs &a = c.a;
    // one launch holds the workgroups of dK and dV and those of dQ, 256 threads for 64 keys or
    // 64 packed rows and more
    const int64_t tiles = (a.sk + int64_t(63)) / 64 + ((int64_t)a.sq * a.group + 63) / 64;
    if ((double)a.batch * a.kv_heads * (double)tiles > 16777215.0) return SBP_ERR_SHAPE;
    if ((rc = query_operand(dO, c, Q, Q->cols, &a.dout))) return rc;
    if ((rc = query_operand(O, c, Q, Q->cols, &a.o))) return rc;
    if ((rc = query_operand(lse, c, Q, 1, &a.lse))) return rc;
    if (dO->dtype != SBP_BF16 || lse->dtype != SBP_F32) return SBP_ERR_DTYPE;
    a.o_f32 = O->dtype == SBP_F32;
    if ((rc = output(dQ, Q->batch, c.hq, Q->rows, Q->cols, &a.dq))) return rc;
    if ((rc = output(dK, Q->batch, c.hk, K->rows, K->cols, &a.dk))) return rc;
    if ((rc = output(dV, Q->batch, c.hk, V->rows, V->cols, &a.dv))) return rc;
    a.dq_f32 = dQ->dtype == SBP_F32;
    a.dk_f32 = dK->dtype == SBP_F32;
    a.dv_f32 = dV->dtype == SBP_F32;
    a.dq_acc = dQ->scope == SBP_ACCUMULATE;
    a.dk_acc = dK->scope == SBP_ACCUMULATE;
    a.dv_acc = dV->scope == SBP_ACCUMULATE;
    std::pair<uintptr_t, uintptr_t> wspan;
    if ((rc = check_ws(ws, &a, &wspan))) return rc;
    const std::pair<uintptr_t, uintptr_t> ins[8] = {
        span_of(a.q, Q, c.hq),        span_of(a.k, K, c.hk),
        span_of(a.v, V, c.hk),        span_of(a.dout, dO, c.hq),
        span_of(a.o, O, c.hq),        span_of(a.lse, lse, c.hq),
        lens_span(a.len_q, Q->batch), lens_span(a.len_k, Q->batch)};
    const sbp_view4_t *const outs[3] = {dQ, dK, dV};
    for (int x = 0; x < 3; ++x) {
        const auto os = span4(outs[x]->data, outs[x], outs[x]->heads);
        for (const auto &in : ins)
            if (overlap(os, in)) return SBP_ERR_ALIAS;
        if (overlap(os, wspan)) return SBP_ERR_ALIAS;
        for (int y = 0; y < x; ++y)
            if (outputs_clash(outs[x], outs[y])) return SBP_ERR_ALIAS;
    }
    for (const auto &in : ins)
        if (overlap(in, wspan)) return SBP_ERR_ALIAS;
    if (a.batch == 0 || c.hk == 0) return SBP_OK;
    if (sbpi::core_bwd_stat_floats(a) > a.ws_floats) return SBP_ERR_WORKSPACE;
    a.aligned = rows16(a.q, a.d) && rows16(a.k, a.d) && rows16(a.v, a.d) && rows16(a.dout, a.d);
    return finish(sbpi::launch_core_bwd(a, stream));
}

}  // extern "C"
