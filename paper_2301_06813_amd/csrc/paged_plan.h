// paged_plan.h -- arithmetic of the line of items of paged_attn.hip, in host and device code: which
// units a workgroup takes and where its partial outputs lie.
#pragma once

#include <stdint.h>

namespace sbpi {

// Whether workgroup wg has a share of the line, from unit share wg on: of parts a part each, of steps
// share = (total - 1) / holders + 1 of `total` (1 of none), for as many workgroups as have room for
// their partial outputs. Rows that descend, which sequences may have in common, can make any number
// of units, past 31 bits too: whatever it is, no other workgroup takes any (share wg would wrap).
constexpr bool has_share(int total, int share, int wg, bool parts, int holders) {
    return (parts || wg < holders) && share * wg < total;
}

// The partial output of a workgroup that has one, or, in shares of steps, two: of an item that it
// began, and of one that it did not.
constexpr int64_t slot_of(int wg, bool began, bool parts) {
    return parts ? wg : 2 * (int64_t)wg + (began ? 1 : 0);
}

// The workspace in floats: each workgroup's note for the join; two statistics of each of `rows` rows
// of a slot; the slots' partial outputs of `cols` columns a row, a multiple of 4.
constexpr int CUT_FLOATS = 8;
constexpr int64_t stats_at(int groups) { return CUT_FLOATS * (int64_t)groups; }
constexpr int64_t parts_at(int groups, int slots, int rows) {
    return stats_at(groups) + 2 * (int64_t)slots * rows;
}
// Slots that fit, an even number: the partial outputs begin at 16 bytes for any number of rows.
constexpr int64_t slots_in(int64_t floats, int groups, int rows, int cols) {
    return floats < stats_at(groups) ? 0 : (floats - stats_at(groups)) / (rows * (int64_t)(2 + cols)) & ~1ll;
}

}  // namespace sbpi
