// paged_kernel.h -- rows of sequences and pages of their tokens (CDNA4 / gfx950),
// shared by the kernels of paged_append.hip and paged_attn*.
#pragma once

#include "paged.h"

namespace sbpk {

using sbpi::CoreView;
using sbpi::Pages;

// A sequence's rows: n of them from row `first` of batch `batch` on; and its tokens in the cache.
struct SeqRows {
    int batch, first, n, len;
};

__device__ __forceinline__ SeqRows rows_of(const Pages &p, int b) {
    SeqRows s;
    s.len = p.len_k[b];
    if (p.row_q) {
        s.batch = 0;
        s.first = min(max(p.row_q[b], 0), p.rows);
        s.n = min(max(p.row_q[b + 1], s.first), p.rows) - s.first;
    } else {
        s.batch = b;
        s.first = 0;
        s.n = p.len_q ? min(max(p.len_q[b], 0), p.rows) : p.rows;
    }
    return s;
}

// The last sequence whose first row is at or before `row` (uniform over the wave; -1: none, seqs:
// row lies behind all), of first rows that do not descend. Every step looks at 64 places
// of what is left; a whole wave calls it.
__device__ __forceinline__ int sequence_of(const Pages &p, int row) {
    const int lane = threadIdx.x & 63;
    int lo = -1, n = p.seqs + 1;      // the answer is lo or one of the next n
    while (n > 0) {
        const int step = (n + 63) / 64, at = lo + (lane + 1) * step;
        const bool in = at <= lo + n && p.row_q[at] <= row;
        const int below = __builtin_popcountll(__ballot(in));
        const int end = lo + n;
        lo += below * step;
        n = min(step - 1, end - lo);
    }
    return lo;
}

}  // namespace sbpk
