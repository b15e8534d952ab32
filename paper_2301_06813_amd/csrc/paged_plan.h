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

}  // namespace sbpi
