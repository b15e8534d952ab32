// paged.h -- a paged cache of keys and values (include/sbp.h): arguments shared by the host
// code and the kernels of paged_append.hip and paged_attn*.
#pragma once

#include "attn_core.h"
#include "rope.h"

namespace sbpi {

// Where the tokens of the sequences lie: in the rows of Q, K, V and O, and in the cache.
struct Pages {
    const int32_t *table = nullptr;
    int64_t table_ld = 0;
    int32_t seqs = 0, width = 0;          // sequences, entries of a table row
    int32_t pages = 0, page = 1;          // pages of the cache, tokens of a page
    const int32_t *len_k = nullptr, *len_q = nullptr, *row_q = nullptr;
    int32_t rows = 0;                     // of a batch (padded), or in all (packed)
};

struct AppendArgs {
    Pages at;
    CoreView k, v, q, kc, vc, qo;         // q.p NULL: none
    int32_t kv_heads = 0, q_heads = 0;
    int32_t batch = 0, d = 0;             // batches of the rows' views
    Rotation rot;                         // turns NULL: none
};

struct PagedArgs {
    Pages at;
    CoreView q, kc, vc, o, lse;           // lse.p may be NULL
    int32_t batch = 0, kv_heads = 0, group = 0, d = 0;
    int32_t causal = 0, window = 0;
    float scale = 0.f;
    int32_t o_f32 = 0, aligned = 0;       // aligned: 16-byte rows of Q and of the cache
    float *ws = nullptr;
    size_t ws_floats = 0;
};

hipError_t launch_append(const AppendArgs &a, int qo_f32, hipStream_t s);
hipError_t launch_paged(const PagedArgs &a, hipStream_t s);

}  // namespace sbpi
