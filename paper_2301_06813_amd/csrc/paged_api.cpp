// paged_api.cpp -- C ABI of the paged cache (include/sbp.h, "paged cache of keys and
// values"): argument checks and operand mapping, then the launches of paged_append.hip or
// paged_attn.hip. Every check happens on the host before any HIP call.
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/sbp.h"
#include "api_internal.h"
#include "paged.h"
#include "rope_checks.h"

namespace {

using namespace sbpa;

constexpr int64_t MAX_SEQS = int64_t(1) << 20;

typedef std::pair<uintptr_t, uintptr_t> Span;

int finish(hipError_t e) { return e == hipSuccess ? SBP_OK : hip_error(e); }

// Checks a bf16 operand and its scope.
int check_in(const sbp_view4_t *v, const sbp_view4_t *like) {
    int rc = check_bounded(v);
    if (rc) return rc;
    if (v->dtype != SBP_BF16) return SBP_ERR_DTYPE;
    if ((v->scope != SBP_GLOBAL && v->scope != SBP_LOCAL) || v->scope != like->scope ||
        v->cols != like->cols)
        return SBP_ERR_SHAPE;
    return SBP_OK;
}

// Checks the cache against operands of `rows` (a view of the new tokens), and the pages' arrays.
int check_cache(const sbp_view4_t *Kc, const sbp_view4_t *Vc, const sbp_pages_t *pages,
                const sbp_view4_t *rows, sbpi::Pages *at, Span arrays[4]) {
    int rc;
    if ((rc = check_in(Kc, Kc)) || (rc = check_in(Vc, Kc))) return rc;
    if (Kc->batch != Vc->batch || Kc->heads != Vc->heads || Kc->rows != Vc->rows ||
        Kc->cols != rows->cols || Kc->rows < 1)
        return SBP_ERR_SHAPE;
    if (rows->cols < 1 || rows->cols > MAX_DIM || rows->rows > MAX_ROWS) return SBP_ERR_SHAPE;
    const sbp_pages_t &g = *pages;
    if (g.seqs < 0 || g.seqs > MAX_SEQS || g.width < 0 || g.table_ld < g.width ||
        g.table_ld > (int64_t(1) << 40) || (int64_t)g.width * Kc->rows > MAX_ROWS)
        return SBP_ERR_SHAPE;
    if (g.row_q ? rows->batch != 1 || g.len_q : rows->batch != g.seqs) return SBP_ERR_SHAPE;
    for (const int32_t *p : {g.table, g.len_k, g.len_q, g.row_q})
        if (reinterpret_cast<uintptr_t>(p) % 4) return SBP_ERR_ALIGN;
    if (g.seqs > 0 && (!g.len_k || (g.width > 0 && !g.table))) return SBP_ERR_NULL;
    at->table = g.table;
    at->table_ld = g.table_ld;
    at->seqs = g.seqs;
    at->width = g.width;
    at->pages = (int32_t)Kc->batch;
    at->page = (int32_t)Kc->rows;
    at->len_k = g.len_k;
    at->len_q = g.len_q;
    at->row_q = g.row_q;
    at->rows = (int32_t)rows->rows;
    arrays[0] = lens_span(g.seqs > 0 && g.width > 0 ? g.table : nullptr,
                          (g.seqs - 1) * g.table_ld + g.width);
    arrays[1] = lens_span(g.len_k, g.seqs);
    arrays[2] = lens_span(g.len_q, g.seqs);
    arrays[3] = lens_span(g.row_q, g.seqs + 1);
    return SBP_OK;
}

}  // namespace

extern "C" {

int sbp_paged_append(const sbp_view4_t *K, const sbp_view4_t *V, const sbp_pages_t *pages,
                     const sbp_rope_t *rope, sbp_view4_t *Kc, sbp_view4_t *Vc,
                     const sbp_view4_t *Q, sbp_view4_t *Qo, int32_t p, int32_t r,
                     hipStream_t stream) {
    if (!K || !V || !pages || !Kc || !Vc || !Q != !Qo) return SBP_ERR_NULL;
    if (Q && !rope) return SBP_ERR_NULL;
    int rc;
    if ((rc = check_in(K, K)) || (rc = check_in(V, K)) || (Q && (rc = check_in(Q, K)))) return rc;
    if (p < 1 || r < 0 || r >= p) return SBP_ERR_LAYOUT;
    if (V->batch != K->batch || V->rows != K->rows || V->heads != K->heads) return SBP_ERR_SHAPE;
    if (Q && (Q->batch != K->batch || Q->rows != K->rows ||
              (K->heads == 0 ? Q->heads != 0 : Q->heads % K->heads != 0)))
        return SBP_ERR_SHAPE;
    sbpi::AppendArgs a;
    Span arrays[5];
    if ((rc = check_cache(Kc, Vc, pages, K, &a.at, arrays))) return rc;
    arrays[4] = {0, 0};
    if (rope) {
        if ((rc = check_rotation(rope, K->cols, &a.rot))) return rc;
        arrays[4] = turns_span(a.rot);
    }
    const int64_t group = Q && K->heads ? Q->heads / K->heads : 1;
    int64_t k0 = 0, hk = K->heads, c0 = 0, hc = Kc->heads;
    if (K->scope == SBP_GLOBAL) head_split(K->heads, p, r, &k0, &hk);
    if (Kc->scope == SBP_GLOBAL) head_split(Kc->heads, p, r, &c0, &hc);
    if (hk != hc || (K->scope == Kc->scope && K->heads != Kc->heads)) return SBP_ERR_SHAPE;
    const sbp_view4_t ins[3] = {share_of(K, k0, hk), share_of(V, k0, hk),
                                Q ? share_of(Q, k0 * group, hk * group) : sbp_view4_t{}};
    const sbp_view4_t cache[2] = {share_of(Kc, c0, hc), share_of(Vc, c0, hc)};
    a.k = kernel_view(&ins[0], 0);
    a.v = kernel_view(&ins[1], 0);
    a.kc = kernel_view(&cache[0], 0);
    a.vc = kernel_view(&cache[1], 0);
    a.kv_heads = (int32_t)hk;
    a.batch = (int32_t)K->batch;
    a.d = (int32_t)K->cols;
    const int n = Q ? 3 : 2;
    if (Q) {
        if ((rc = output(Qo, Q->batch, ins[2].heads, Q->rows, Q->cols, &a.qo))) return rc;
        if (Qo->scope == SBP_ACCUMULATE) return SBP_ERR_SHAPE;
        a.q = kernel_view(&ins[2], 0);
        a.q_heads = (int32_t)ins[2].heads;
        for (int x = 0; x < n; ++x)
            if (!(x == 2 && in_place(Qo, &ins[2])) && !apart(Qo, &ins[x])) return SBP_ERR_ALIAS;
        for (const Span &s : arrays)
            if (overlap(s, span4(Qo->data, Qo, Qo->heads))) return SBP_ERR_ALIAS;
    }
    for (int x = 0; x < 2; ++x) {
        if (!injective(&cache[x])) return SBP_ERR_ALIAS;
        const Span c = span4(cache[x].data, &cache[x], hc);
        for (int y = 0; y < n; ++y)
            if (overlap(c, span4(ins[y].data, &ins[y], ins[y].heads))) return SBP_ERR_ALIAS;
        for (const Span &s : arrays)
            if (overlap(s, c)) return SBP_ERR_ALIAS;
        if (Q && overlap(c, span4(Qo->data, Qo, Qo->heads))) return SBP_ERR_ALIAS;
    }
    if (!apart(&cache[0], &cache[1])) return SBP_ERR_ALIAS;
    if (a.batch == 0 || a.at.rows == 0 || a.at.seqs == 0 || hk == 0) return SBP_OK;
    if (!rotation_fits(a.batch * (double)a.at.rows, a.q_heads + 2.0 * hk, a.d)) return SBP_ERR_SHAPE;
    return finish(sbpi::launch_append(a, Q && Qo->dtype == SBP_F32, stream));
}

int sbp_paged_attn(const sbp_view4_t *Q, const sbp_view4_t *Kc, const sbp_view4_t *Vc,
                   const sbp_pages_t *pages, float scale, int32_t causal, int32_t window,
                   sbp_view4_t *O, sbp_view4_t *lse, int32_t p, int32_t r,
                   const sbp_workspace_t *ws, hipStream_t stream) {
    if (!Q || !Kc || !Vc || !pages || !O) return SBP_ERR_NULL;
    int rc;
    if ((rc = check_in(Q, Q)) || (rc = check_in(Kc, Q)) || (rc = check_in(Vc, Q))) return rc;
    if (p < 1 || r < 0 || r >= p) return SBP_ERR_LAYOUT;
    sbpi::PagedArgs a;
    Span arrays[4];
    if ((rc = check_cache(Kc, Vc, pages, Q, &a.at, arrays))) return rc;
    if (Kc->heads == 0 ? Q->heads != 0 : Q->heads % Kc->heads != 0) return SBP_ERR_SHAPE;
    if (!(scale >= MIN_SCALE && scale <= 1.f / MIN_SCALE) || window < 0 || (causal != 0 && causal != 1))
        return SBP_ERR_SHAPE;
    const int64_t group = Kc->heads ? Q->heads / Kc->heads : 1;
    int64_t k0 = 0, hk = Kc->heads;
    if (Q->scope == SBP_GLOBAL) head_split(Kc->heads, p, r, &k0, &hk);
    const int64_t hq = hk * group;
    if (Q->rows * group > INT32_MAX - 256) return SBP_ERR_SHAPE;
    // tiles of 32 packed rows, one more for each sequence of a packed batch
    const double tiles = (double)hk * (Q->batch * (double)((Q->rows * group + 31) / 32) + pages->seqs);
    if (tiles > 16777215.0) return SBP_ERR_SHAPE;
    const sbp_view4_t ins[3] = {share_of(Q, k0 * group, hq), share_of(Kc, k0, hk),
                                share_of(Vc, k0, hk)};
    a.q = kernel_view(&ins[0], 0);
    a.kc = kernel_view(&ins[1], 0);
    a.vc = kernel_view(&ins[2], 0);
    if (O->scope == SBP_ACCUMULATE || (lse && lse->scope == SBP_ACCUMULATE)) return SBP_ERR_SHAPE;
    if ((rc = output(O, Q->batch, hq, Q->rows, Q->cols, &a.o))) return rc;
    if (lse) {
        if ((rc = output(lse, Q->batch, hq, Q->rows, 1, &a.lse))) return rc;
        if (lse->dtype != SBP_F32) return SBP_ERR_DTYPE;
    }
    Span wspan;
    if ((rc = check_ws(ws, &a.ws, &a.ws_floats, &wspan))) return rc;
    const Span os = span4(O->data, O, hq), ls = lse ? span4(lse->data, lse, hq) : Span(0, 0);
    for (const Span &o : {os, ls, wspan}) {
        for (const sbp_view4_t &x : ins)
            if (overlap(o, span4(x.data, &x, x.heads))) return SBP_ERR_ALIAS;
        for (const Span &s : arrays)
            if (overlap(o, s)) return SBP_ERR_ALIAS;
    }
    if (overlap(os, ls) || overlap(os, wspan) || overlap(ls, wspan)) return SBP_ERR_ALIAS;
    a.batch = (int32_t)Q->batch;
    a.kv_heads = (int32_t)hk;
    a.group = (int32_t)group;
    a.d = (int32_t)Q->cols;
    a.causal = causal;
    // a window as long as the keys hides none of them
    a.window = window >= (int64_t)a.at.width * a.at.page ? 0 : window;
    a.scale = scale;
    a.o_f32 = O->dtype == SBP_F32;
    a.aligned = rows16(a.q, a.d) && rows16(a.kc, a.d) && rows16(a.vc, a.d);
    if (a.batch == 0 || hq == 0 || a.at.rows == 0 || a.at.seqs == 0) return SBP_OK;
    return finish(sbpi::launch_paged(a, stream));
}

}  // extern "C"
