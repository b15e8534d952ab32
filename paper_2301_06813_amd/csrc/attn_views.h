// attn_views.h -- checks of the attention calls' 4-D views and their head split,
// shared by attn_api.cpp, attn_core_api.cpp, rope_api.cpp and paged_api.cpp.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <utility>

#include "../../include/sbp.h"
#include "attn_core.h"

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

constexpr int64_t MAX_ROWS = int64_t(1) << 29;   // i + len_k - len_q + window fits 32 bits
constexpr int64_t MAX_DIM = 128;
constexpr float MIN_SCALE = 0x1p-100f;

// check_view4, and element offsets that stay inside 62 bits.
inline int check_bounded(const sbp_view4_t *v) {
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
inline bool interleaved(const sbp_view4_t *x, const sbp_view4_t *y) {
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

inline bool outputs_clash(const sbp_view4_t *x, const sbp_view4_t *y) {
    return overlap(span4(x->data, x, x->heads), span4(y->data, y, y->heads)) && !interleaved(x, y);
}

inline sbpi::CoreView kernel_view(const sbp_view4_t *v, int64_t first_head) {
    sbpi::CoreView o;
    o.p = v->data;
    if (o.p && v->heads > 0)
        o.p = static_cast<char *>(v->data) + first_head * v->stride_h * elsz(v->dtype);
    o.sb = v->stride_b;
    o.sh = v->stride_h;
    o.ld = v->ld;
    return o;
}

// An output of `heads` local heads.
inline int output(const sbp_view4_t *v, int64_t batch, int64_t heads, int64_t rows, int64_t cols,
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

// The rank's heads [first, first + heads) of a view, as a view of their own.
inline sbp_view4_t share_of(const sbp_view4_t *v, int64_t first, int64_t heads) {
    sbp_view4_t s = *v;
    s.data = kernel_view(v, v->heads > 0 ? first : 0).p;
    s.heads = heads;
    return s;
}

inline bool same_strides(const sbp_view4_t *x, const sbp_view4_t *y) {
    auto same = [](int64_t n, int64_t m, int64_t s, int64_t t) { return (n <= 1 && m <= 1) || s == t; };
    return x->dtype == y->dtype && same(x->rows, y->rows, x->ld, y->ld) &&
           same(x->heads, y->heads, x->stride_h, y->stride_h) &&
           same(x->batch, y->batch, x->stride_b, y->stride_b);
}

// x is y's memory, element for element.
inline bool in_place(const sbp_view4_t *x, const sbp_view4_t *y) {
    return x->data == y->data && x->batch == y->batch && x->heads == y->heads &&
           x->rows == y->rows && x->cols == y->cols && same_strides(x, y);
}

// Two views of equal strides that share spans but no element: parts of one tensor along
// its batch, head or row dimension, or along one more dimension that both are cut out of.
inline bool parts_of_one(const sbp_view4_t *x, const sbp_view4_t *y) {
    if (!same_strides(x, y)) return false;
    if (reinterpret_cast<uintptr_t>(y->data) < reinterpret_cast<uintptr_t>(x->data)) std::swap(x, y);
    const uintptr_t bytes =
        reinterpret_cast<uintptr_t>(y->data) - reinterpret_cast<uintptr_t>(x->data);
    if (bytes % elsz(x->dtype) || bytes == 0) return false;
    const int64_t gap = (int64_t)(bytes / elsz(x->dtype));
    const int64_t nx[3] = {x->rows, x->heads, x->batch}, ny[3] = {y->rows, y->heads, y->batch};
    // a dimension of one element has the other view's stride
    auto stride = [&](int k) {
        const sbp_view4_t *v = nx[k] > 1 ? x : y;
        return k == 0 ? v->ld : k == 1 ? v->stride_h : v->stride_b;
    };
    const int64_t cols = std::max(x->cols, y->cols);
    for (int along = 0; along < 4; ++along) {   // 3: one more dimension
        std::pair<int64_t, int64_t> d[4];       // stride, extent of the tensor of both
        for (int k = 0; k < 3; ++k) d[k] = {stride(k), std::max(nx[k], ny[k])};
        d[3] = {gap, 2};
        if (along < 3) {
            const int64_t s = stride(along);
            if (s < 1 || gap % s || gap / s < nx[along]) continue;
            d[along] = {s, gap / s + ny[along]};
            d[3].second = 1;
        }
        std::sort(d, d + 4);
        int64_t span = cols;
        bool apart = true;
        for (const auto &[s, n] : d) {
            if (n <= 1) continue;
            if (s < span) apart = false;
            if ((double)s * (double)n > 4e18) apart = false;
            if (!apart) break;
            span = s * (n - 1) + span;
        }
        if (apart) return true;
    }
    return false;
}

// Two views of which one is written share no element.
inline bool apart(const sbp_view4_t *x, const sbp_view4_t *y) {
    return !overlap(span4(x->data, x, x->heads), span4(y->data, y, y->heads)) ||
           interleaved(x, y) || parts_of_one(x, y);
}

// 16-byte rows, and tile offsets that fit a 31-bit buffer offset (256 rows at most).
inline bool rows16(const sbpi::CoreView &v, int64_t d) {
    return reinterpret_cast<uintptr_t>(v.p) % 16 == 0 && v.ld % 8 == 0 && v.sb % 8 == 0 &&
           v.sh % 8 == 0 && d % 8 == 0 && v.ld < (int64_t(1) << 21);
}

inline std::pair<uintptr_t, uintptr_t> lens_span(const int32_t *p, int64_t batch) {
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    return p ? std::make_pair(b, b + (uintptr_t)(4 * batch)) : std::make_pair(uintptr_t(0), uintptr_t(0));
}

// A call's workspace (left as it was where there is none) and its span.
inline int check_ws(const sbp_workspace_t *ws, float **at, size_t *floats,
                    std::pair<uintptr_t, uintptr_t> *span) {
    *span = {0, 0};
    if (!ws || ws->bytes == 0) return SBP_OK;
    if (ws->bytes < 0) return SBP_ERR_SHAPE;
    if (!ws->data) return SBP_ERR_NULL;
    const uintptr_t b = reinterpret_cast<uintptr_t>(ws->data);
    if (b & 15) return SBP_ERR_ALIGN;
    *at = static_cast<float *>(ws->data);
    *floats = (size_t)ws->bytes / sizeof(float);
    *span = {b, b + (uintptr_t)ws->bytes};
    return SBP_OK;
}

}  // namespace sbpa
