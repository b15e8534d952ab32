// rope_api.cpp -- C ABI of rotary positions (include/sbp.h, "rotary positions"): the table
// of frequencies, argument checks and operand mapping, then the launch of rope.hip. Every
// check happens on the host before any HIP call.
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/sbp.h"
#include "api_internal.h"
#include "rope_checks.h"

namespace {

using namespace sbpa;

constexpr long double TAU = 6.283185307179586476925286766559005768L;

// The pair of a rotation with n turns over the context.
long double pair_at(long double n, long double dim, long double base, long double context) {
    return dim * logl(context / (TAU * n)) / (2 * logl(base));
}

int rope(const sbp_view4_t *Q, const sbp_view4_t *K, const sbp_rope_t *rope_, const sbp_places_t *at,
         sbp_view4_t *Qo, sbp_view4_t *Ko, int32_t p, int32_t r, int back, hipStream_t stream) {
    if (!Q || !Qo || !rope_ || !K != !Ko) return SBP_ERR_NULL;
    const int n = K ? 2 : 1;
    const sbp_view4_t *ins[2] = {Q, K};
    sbp_view4_t *outs[2] = {Qo, Ko};
    int rc;
    for (int x = 0; x < n; ++x) {
        if ((rc = check_bounded(ins[x]))) return rc;
        const sbp_view4_t *v = ins[x];
        if (v->scope != SBP_GLOBAL && v->scope != SBP_LOCAL) return SBP_ERR_SHAPE;
        if (v->scope != Q->scope || v->batch != Q->batch || v->rows != Q->rows || v->cols != Q->cols)
            return SBP_ERR_SHAPE;
        if (v->dtype != Q->dtype) return SBP_ERR_DTYPE;
    }
    if (p < 1 || r < 0 || r >= p) return SBP_ERR_LAYOUT;
    if (Q->cols < 1 || Q->cols > MAX_DIM || Q->rows > MAX_ROWS) return SBP_ERR_SHAPE;
    if (K && (K->heads == 0 ? Q->heads != 0 : Q->heads % K->heads != 0)) return SBP_ERR_SHAPE;
    sbpi::RopeArgs a;
    if ((rc = check_rotation(rope_, Q->cols, &a.rot))) return rc;
    // the rank's heads: of K, and the query heads that share them
    const sbp_view4_t *kv = K ? K : Q;
    const int64_t group = kv->heads ? Q->heads / kv->heads : 1;
    int64_t k0 = 0, hk = kv->heads;
    if (Q->scope == SBP_GLOBAL) head_split(kv->heads, p, r, &k0, &hk);
    sbp_view4_t in[2], out[2];
    in[0] = share_of(Q, k0 * group, hk * group);
    if (K) in[1] = share_of(K, k0, hk);
    for (int x = 0; x < n; ++x) {
        const sbp_view4_t *o = outs[x];
        if ((rc = output(o, Q->batch, in[x].heads, Q->rows, Q->cols, &a.out[x]))) return rc;
        if (o->scope == SBP_ACCUMULATE) return SBP_ERR_SHAPE;
        if (o->dtype != Qo->dtype || (Q->dtype == SBP_F32 && o->dtype != SBP_F32))
            return SBP_ERR_DTYPE;
        out[x] = *o;
        a.in[x] = kernel_view(&in[x], 0);
        a.heads[x] = (int32_t)in[x].heads;
    }
    a.batch = (int32_t)Q->batch;
    a.rows = (int32_t)Q->rows;
    a.d = (int32_t)Q->cols;
    a.back = back;
    std::pair<uintptr_t, uintptr_t> arrays[2] = {turns_span(a.rot), {0, 0}};
    if (at) {
        if ((at->per_row != 0 && at->per_row != 1) || at->ld < 0 ||
            (double)Q->batch * (double)at->ld > 1e18)
            return SBP_ERR_SHAPE;
        const bool some = Q->batch > 0 && Q->rows > 0;
        if (some && !at->pos) return SBP_ERR_NULL;
        if (reinterpret_cast<uintptr_t>(at->pos) % 4) return SBP_ERR_ALIGN;
        a.pos = at->pos;
        a.pos_ld = at->ld;
        a.pos_per_row = at->per_row;
        if (some)
            arrays[1] = lens_span(at->pos, (Q->batch - 1) * at->ld + (at->per_row ? Q->rows : 1));
    }
    for (int x = 0; x < n; ++x) {
        for (int y = 0; y < n; ++y)
            if (!(x == y && in_place(&out[x], &in[y])) && !apart(&out[x], &in[y])) return SBP_ERR_ALIAS;
        for (const auto &s : arrays)
            if (overlap(s, span4(out[x].data, &out[x], out[x].heads))) return SBP_ERR_ALIAS;
    }
    if (n == 2 && !apart(&out[0], &out[1])) return SBP_ERR_ALIAS;
    if (a.batch == 0 || a.rows == 0 || hk == 0) return SBP_OK;
    if (!rotation_fits(a.batch * (double)a.rows, a.heads[0] + (double)a.heads[1], a.d))
        return SBP_ERR_SHAPE;
    const hipError_t e = sbpi::launch_rope(a, Q->dtype == SBP_F32, Qo->dtype == SBP_F32, stream);
    return e == hipSuccess ? SBP_OK : hip_error(e);
}

}  // namespace

extern "C" {

int sbp_rope_turns(int32_t dim, double base, int32_t scaling, double factor, double low,
                   double high, double context, uint64_t *turns) {
    if (!turns) return SBP_ERR_NULL;
    if (dim < 2 || dim > MAX_DIM || dim % 2 || !(base > 1.0) || !isfinite(base) || scaling < 0 ||
        scaling > SBP_ROPE_BY_PAIRS)
        return SBP_ERR_SHAPE;
    const bool ramp = scaling == SBP_ROPE_BY_TURNS || scaling == SBP_ROPE_BY_PAIRS;
    if (scaling != SBP_ROPE_PLAIN && !(factor > 0.0 && isfinite(factor))) return SBP_ERR_SHAPE;
    if (ramp && !(context > 0.0 && isfinite(context) && low > 0.0 && high > low && isfinite(high)))
        return SBP_ERR_SHAPE;
    long double b = base;
    if (scaling == SBP_ROPE_BASE && dim > 2)
        b *= powl((long double)factor, (long double)dim / (dim - 2));
    const long double first = ramp ? fmaxl(0, floorl(pair_at(high, dim, base, context))) : 0;
    const long double last = ramp ? fminl(dim - 1, ceill(pair_at(low, dim, base, context))) : 0;
    for (int i = 0; i < dim / 2; ++i) {
        long double n = powl(b, -2 * (long double)i / dim) / TAU;   // turns a position
        const long double slow = n / factor;
        auto limited = [](long double w) { return fminl(1, fmaxl(0, w)); };
        if (scaling == SBP_ROPE_LINEAR) {
            n = slow;
        } else if (scaling == SBP_ROPE_BY_TURNS) {
            const long double w = limited((context * n - low) / ((long double)high - low));
            n = n * w + slow * (1 - w);
        } else if (scaling == SBP_ROPE_BY_PAIRS) {
            const long double w = limited((i - first) / fmaxl(last - first, 0.001L));
            n = n * (1 - w) + slow * w;
        }
        // whole turns a position make no difference
        const long double x = roundl((n - floorl(n)) * 0x1p64L);
        turns[i] = x >= 0x1p64L ? 0 : (uint64_t)x;
    }
    return SBP_OK;
}

int sbp_rope_fwd(const sbp_view4_t *Q, const sbp_view4_t *K, const sbp_rope_t *rope_,
                 const sbp_places_t *at, sbp_view4_t *Qo, sbp_view4_t *Ko, int32_t p, int32_t r,
                 hipStream_t stream) {
    return rope(Q, K, rope_, at, Qo, Ko, p, r, 0, stream);
}

int sbp_rope_bwd(const sbp_view4_t *dQo, const sbp_view4_t *dKo, const sbp_rope_t *rope_,
                 const sbp_places_t *at, sbp_view4_t *dQ, sbp_view4_t *dK, int32_t p, int32_t r,
                 hipStream_t stream) {
    return rope(dQo, dKo, rope_, at, dQ, dK, p, r, 1, stream);
}

}  // extern "C"
