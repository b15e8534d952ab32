// attn_views.h -- checks of the attention calls' 4-D views and their head split,
// shared by attn_api.cpp and attn_core_api.cpp.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <utility>

#include "../../include/sbp.h"

namespace sbpa {

inline int64_t elsz(int32_t dtype) { return dtype == SBP_F32 ? 4 : 2; }

// Heads [h0, h0 + hr) of H on rank r of p (the balanced split rule).
inline void head_split(int64_t H, int32_t p, int32_t r, int64_t *h0, int64_t *hr) {
    const int64_t base = H / p, rem = H % p;
    *hr = base + (r < rem ? 1 : 0);
    *h0 = (int64_t)r * base + (r < rem ? r : rem);
}

inline int check_view4(const sbp_view4_t *v) {
    if (!v) return SBP_ERR_NULL;
    if (v->dtype != SBP_BF16 && v->dtype != SBP_F32) return SBP_ERR_DTYPE;
    const int64_t ext[4] = {v->batch, v->heads, v->rows, v->cols};
    for (int64_t e : ext)
        if (e < 0 || e > INT32_MAX) return SBP_ERR_SHAPE;
    if (v->ld < v->cols || v->ld < 1 || v->stride_b < 0 || v->stride_h < 0) return SBP_ERR_SHAPE;
    if (v->ld > (int64_t(1) << 40) || v->stride_b > (int64_t(1) << 40) ||
        v->stride_h > (int64_t(1) << 40))
        return SBP_ERR_SHAPE;
    const bool empty = v->batch == 0 || v->heads == 0 || v->rows == 0 || v->cols == 0;
    if (!empty) {
        if (!v->data) return SBP_ERR_NULL;
        if (reinterpret_cast<uintptr_t>(v->data) % elsz(v->dtype)) return SBP_ERR_ALIGN;
    }
    return SBP_OK;
}

// An input operand: its rank-r base and local head count.
struct In4 {
    const char *ptr;
    int64_t heads;
    const sbp_view4_t *v;
};

// [begin, end) bytes a 4-D view with `heads` heads starting at p touches.
inline std::pair<uintptr_t, uintptr_t> span4(const void *p, const sbp_view4_t *v, int64_t heads) {
    if (!p || v->batch == 0 || heads == 0 || v->rows == 0 || v->cols == 0) return {0, 0};
    const int64_t last = (v->batch - 1) * v->stride_b + (heads - 1) * v->stride_h +
                         (v->rows - 1) * v->ld + v->cols;
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    return {b, b + (uintptr_t)(last * elsz(v->dtype))};
}

inline bool overlap(std::pair<uintptr_t, uintptr_t> a, std::pair<uintptr_t, uintptr_t> b) {
    if (a.first == a.second || b.first == b.second) return false;
    return a.first < b.second && b.first < a.second;
}

// No two elements of an output view share an address: with the outer
// dimensions sorted by stride, each stride covers the span of the smaller ones.
inline bool injective(const sbp_view4_t *v) {
    struct D {
        int64_t stride, n;
    } d[3] = {{v->ld, v->rows}, {v->stride_h, v->heads}, {v->stride_b, v->batch}};
    std::sort(d, d + 3, [](const D &a, const D &b) { return a.stride < b.stride; });
    int64_t span = v->cols;   // elements covered by the dimensions below
    for (const D &x : d) {
        if (x.n <= 1) continue;
        if (x.stride < span) return false;
        span = x.stride * (x.n - 1) + span;
    }
    return true;
}

// The call's head split: H (when some input is GLOBAL) and rank r's heads.
inline int resolve_heads(const sbp_view4_t *const *ins, int nin, int32_t p, int32_t r, int64_t *hr,
                  In4 *out) {
    if (p < 1 || r < 0 || r >= p) return SBP_ERR_LAYOUT;
    int64_t H = -1, local = -1;
    for (int i = 0; i < nin; ++i) {
        const sbp_view4_t *v = ins[i];
        if (v->scope == SBP_GLOBAL) {
            if (H >= 0 && v->heads != H) return SBP_ERR_SHAPE;
            H = v->heads;
        } else if (v->scope == SBP_LOCAL) {
            if (local >= 0 && v->heads != local) return SBP_ERR_SHAPE;
            local = v->heads;
        } else {
            return SBP_ERR_SHAPE;
        }
    }
    int64_t h0 = 0;
    if (H >= 0) {
        head_split(H, p, r, &h0, hr);
        if (local >= 0 && local != *hr) return SBP_ERR_SHAPE;
    } else {
        *hr = local;
    }
    for (int i = 0; i < nin; ++i) {
        const sbp_view4_t *v = ins[i];
        out[i].v = v;
        out[i].heads = *hr;
        out[i].ptr = static_cast<const char *>(v->data);
        if (v->scope == SBP_GLOBAL && *hr > 0 && out[i].ptr)
            out[i].ptr += h0 * v->stride_h * elsz(v->dtype);
    }
    return SBP_OK;
}

// Output checks: shape [batch][hr][rows][cols], dtype, no self-overlap, no
// overlap with the inputs' spans.
inline int check_out4(const sbp_view4_t *o, int64_t batch, int64_t hr, int64_t rows, int64_t cols,
               const In4 *ins, int nin) {
    int rc = check_view4(o);
    if (rc) return rc;
    if (o->batch != batch || o->heads != hr || o->rows != rows || o->cols != cols)
        return SBP_ERR_SHAPE;
    if (o->scope == SBP_ACCUMULATE && o->dtype != SBP_F32) return SBP_ERR_DTYPE;
    if (!injective(o)) return SBP_ERR_SHAPE;
    const auto os = span4(o->data, o, hr);
    for (int i = 0; i < nin; ++i)
        if (overlap(os, span4(ins[i].ptr, ins[i].v, ins[i].heads))) return SBP_ERR_ALIAS;
    return SBP_OK;
}

}  // namespace sbpa
