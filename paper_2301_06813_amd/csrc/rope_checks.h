// rope_checks.h -- checks of a rotation, shared by rope_api.cpp and paged_api.cpp.
#pragma once

#include <math.h>

#include "attn_views.h"
#include "rope.h"

namespace sbpa {

inline int check_rotation(const sbp_rope_t *rope, int64_t cols, sbpi::Rotation *out) {
    if (!rope->turns) return SBP_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(rope->turns) % 8) return SBP_ERR_ALIGN;
    if (rope->dim < 2 || rope->dim % 2 || rope->dim > cols || !isfinite(rope->mul) ||
        (rope->order != SBP_ROPE_HALVES && rope->order != SBP_ROPE_PAIRS))
        return SBP_ERR_SHAPE;
    out->turns = rope->turns;
    out->dim = rope->dim;
    out->pairs = rope->order == SBP_ROPE_PAIRS;
    out->mul = rope->mul;
    return SBP_OK;
}

inline std::pair<uintptr_t, uintptr_t> turns_span(const sbpi::Rotation &r) {
    const uintptr_t b = reinterpret_cast<uintptr_t>(r.turns);
    return {b, b + (uintptr_t)(r.dim / 2 * 8)};
}

// Rows times heads times units of 8 columns and more (rotated and copied columns apart, so two
// more at most than the head dimension has) stay below 2^31.
inline bool rotation_fits(double rows, double heads, int64_t d) {
    return rows * heads * (double)((d + 23) / 8) < 2147483648.0;
}

}  // namespace sbpa
