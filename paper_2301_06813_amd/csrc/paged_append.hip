// paged_append.hip -- new tokens' keys and values to their places in a paged cache, with the
// rotation of K and Q on the way.
//
// A thread owns R pairs of columns of a new token and takes them in HEADS of the heads of Q, K and
// V, one after the other (rope.hip): the token's place gives both its row of the cache and its
// angles. In a packed batch a wave finds its first row's sequence by a search of 64 places at a
// time. The bound is memory, for few tokens the chain of loads from a row to its page. (7180 new
// tokens of 64 + 8 + 8 heads of 128: 87 us with one head a thread, 64 with two, 65 with three, 67
// with four, 72 with eight.)
#include "attn_core_kernel.h"
#include "paged_kernel.h"
#include "profile.h"
#include "rope_kernel.h"

namespace sbpk {

using sbpi::AppendArgs;

// Pairs of a unit: 16 bytes of Qo's type.
template <typename TQ>
constexpr int PAIRS_OF = 16 / (int)sizeof(TQ);

struct AppendLaunch {
    AppendArgs a;
    int32_t threads;                 // rows x head groups x units
    Div units, groups, rows, page;   // of a head, of a row, of a batch, tokens of a page
};

template <typename TQ, int HEADS>
__global__ __launch_bounds__(256) void paged_append_kernel(AppendLaunch f) {
    constexpr int R = PAIRS_OF<TQ>;
    const AppendArgs &a = f.a;
    const Rotation &r = a.rot;
    const uint32_t id = blockIdx.x * 256u + threadIdx.x;
    if (blockIdx.x * 256u + (threadIdx.x & ~63u) >= (uint32_t)f.threads) return;   // whole waves
    const int rest = f.units(id), ui = f.units.rest(id, rest);
    const int row = f.groups(rest), hg = f.groups.rest(rest, row);
    const bool live = id < (uint32_t)f.threads;
    int b = 0, batch = 0, i = row, n = a.at.rows, first = 0;
    if (a.at.row_q) {
        // the last sequence that begins at or before the row
        b = sequence_of(a.at, __builtin_amdgcn_readfirstlane(row));
        if (!live) return;
        while (b < a.at.seqs && a.at.row_q[b + 1] <= row) ++b;
        if (b < 0 || b >= a.at.seqs) return;
        first = max(a.at.row_q[b], 0);
        n = min(a.at.row_q[b + 1], a.at.rows) - first;
    } else {
        if (!live) return;
        b = batch = f.rows(row);
        i = f.rows.rest(row, b);
        if (a.at.len_q) n = min(max(a.at.len_q[b], 0), a.at.rows);
    }
    const int new_i = i - first;
    if (new_i < 0 || new_i >= n) return;
    const int64_t t = (int64_t)a.at.len_k[b] - n + new_i;
    const int heads = a.q_heads + 2 * a.kv_heads, step = (int)f.groups.d;
    const Unit u = unit_of<R>(r, a.d, ui);
    // head h of Q's, then K's, then V's
    Pair<uint16_t, R> x[HEADS];
#pragma unroll
    for (int k = 0; k < HEADS; ++k) {
        const int h = hg + k * step;
        const int hk = h - a.q_heads, hv = hk - a.kv_heads;
        const CoreView &v = hk < 0 ? a.q : hv < 0 ? a.k : a.v;
        const int m = hk < 0 ? h : hv < 0 ? hk : hv;
        if (h < heads) x[k].load(static_cast<const uint16_t *>(v.p) + batch * v.sb + m * v.sh + i * v.ld, u);
    }
    int page = -1, slot = 0;
    if (t >= 0 && t < (int64_t)a.at.width * a.at.page) {
        const int at = f.page((int)t);
        slot = f.page.rest((int)t, at);
        page = a.at.table[b * a.at.table_ld + at];
    }
    Angles<R> g;
    if (u.turn) g.find(r, ui, t, false);
#pragma unroll
    for (int k = 0; k < HEADS; ++k) {
        const int h = hg + k * step;
        const int hk = h - a.q_heads, hv = hk - a.kv_heads;
        if (h >= heads) continue;
        if (hk < 0) {
            put(x[k], g, u, r.pairs,
                static_cast<TQ *>(a.qo.p) + batch * a.qo.sb + h * a.qo.sh + i * a.qo.ld);
        } else if (page >= 0 && page < a.at.pages) {
            const CoreView &v = hv < 0 ? a.kc : a.vc;
            Unit w = u;
            w.turn = u.turn && hv < 0;
            put(x[k], g, w, r.pairs, static_cast<uint16_t *>(v.p) + page * v.sb +
                                         (hv < 0 ? hk : hv) * v.sh + slot * v.ld);
        }
    }
}

}  // namespace sbpk

namespace sbpi {

namespace {

template <typename TQ>
hipError_t launch(const AppendArgs &a, hipStream_t s) {
    sbpk::AppendLaunch f;
    f.a = a;
    const int64_t rows = (int64_t)a.batch * a.at.rows;
    const int heads = a.q_heads + 2 * a.kv_heads, units = sbpk::units_of<sbpk::PAIRS_OF<TQ>>(a.rot, a.d);
    const bool many = rows * heads * units > (int64_t)device_cus() * 2048;
    const int groups = many ? (heads + 1) / 2 : heads;
    f.threads = (int32_t)(rows * groups * units);
    f.units = sbpk::Div(units);
    f.groups = sbpk::Div(groups);
    f.rows = sbpk::Div(a.at.rows);
    f.page = sbpk::Div(a.at.page);
    const dim3 grid((unsigned)((f.threads + 255ll) / 256)), block(256);
    return many ? launch_kernel(sbpk::paged_append_kernel<TQ, 2>, "paged_append_kernel<2>", grid, block, s, f)
                : launch_kernel(sbpk::paged_append_kernel<TQ, 1>, "paged_append_kernel<1>", grid, block, s, f);
}

}  // namespace

hipError_t launch_append(const AppendArgs &a, int qo_f32, hipStream_t s) {
    return qo_f32 ? launch<float>(a, s) : launch<uint16_t>(a, s);
}

}  // namespace sbpi
