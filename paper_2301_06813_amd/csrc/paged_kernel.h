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

}  // namespace sbpk
