// rope.hip -- rotary positions of Q and K, forward and backward.
//
// A thread owns 2 R columns (R pairs) of a row and turns them in HEADS heads of Q and K, one
// after the other: the angles are computed once for these, while the heads' values are on
// the way. The bound is memory: each element is read once and written once. R values of the
// longer type are 16 bytes; angles for four heads pay for bf16 (32768 rows of 72 heads of 128: 316
// us with one head a thread, 240 with two, 237 with four, 251 with eight), for two for fp32 (16384
// such rows, the same bytes: 207 us).
#include "attn_core_kernel.h"
#include "profile.h"
#include "rope_kernel.h"

namespace sbpk {

struct RopeLaunch {
    RopeArgs a;
    int64_t threads;                 // rows x head groups x units, below 2^31
    Div units, groups, rows;         // of a head, of a row, of a sequence
};

template <typename TI, typename TO, int R, int HEADS>
__global__ __launch_bounds__(256) void rope_kernel(RopeLaunch f) {
    const RopeArgs &a = f.a;
    const Rotation &r = a.rot;
    const uint32_t id = blockIdx.x * 256u + threadIdx.x;
    if (id >= f.threads) return;
    const int rest = f.units(id), ui = f.units.rest(id, rest);
    const int row = f.groups(rest), hg = f.groups.rest(rest, row);
    const int b = f.rows(row), i = f.rows.rest(row, b);
    const Unit u = unit_of<R>(r, a.d, ui);
    const int heads = a.heads[0] + a.heads[1], step = (int)f.groups.d;
    auto at = [&](const CoreView (&v)[2], int h) {    // element offset of head h's row
        return h < a.heads[0] ? b * v[0].sb + i * v[0].ld + h * v[0].sh
                              : b * v[1].sb + i * v[1].ld + (h - a.heads[0]) * v[1].sh;
    };
    auto base = [&](const CoreView (&v)[2], int h) { return h < a.heads[0] ? v[0].p : v[1].p; };
    Pair<TI, R> x[HEADS];
#pragma unroll
    for (int k = 0; k < HEADS; ++k) {
        const int h = hg + k * step;
        if (h < heads) x[k].load(static_cast<const TI *>(base(a.in, h)) + at(a.in, h), u);
    }
    Angles<R> g;
    if (u.turn) {
        int64_t t = i;
        if (a.pos) t = a.pos_per_row ? a.pos[b * a.pos_ld + i] : (int64_t)a.pos[b * a.pos_ld] + i;
        g.find(r, ui, t, a.back);
    }
#pragma unroll
    for (int k = 0; k < HEADS; ++k) {
        const int h = hg + k * step;
        if (h < heads) put(x[k], g, u, r.pairs, static_cast<TO *>(base(a.out, h)) + at(a.out, h));
    }
}

}  // namespace sbpk

namespace sbpi {

namespace {

template <typename TI, typename TO>
hipError_t launch(const RopeArgs &a, hipStream_t s) {
    constexpr bool BF = sizeof(TO) == 2;
    constexpr int R = BF ? 8 : 4, MANY = BF ? 4 : 2;
    sbpk::RopeLaunch f;
    f.a = a;
    const int64_t rows = (int64_t)a.batch * a.rows;
    const int heads = a.heads[0] + a.heads[1], units = sbpk::units_of<R>(a.rot, a.d);
    // (one head a thread where that does not fill the chip twice over)
    const bool many = rows * heads * units > (int64_t)device_cus() * 2048;
    const int groups = many ? (heads + MANY - 1) / MANY : heads;
    f.threads = rows * groups * units;
    f.units = sbpk::Div(units);
    f.groups = sbpk::Div(groups);
    f.rows = sbpk::Div(a.rows);
    const dim3 grid((unsigned)((f.threads + 255) / 256)), block(256);
    return many ? launch_kernel(sbpk::rope_kernel<TI, TO, R, MANY>, "rope_kernel<many>", grid, block, s, f)
                : launch_kernel(sbpk::rope_kernel<TI, TO, R, 1>, "rope_kernel<1>", grid, block, s, f);
}

}  // namespace

hipError_t launch_rope(const RopeArgs &a, int in_f32, int out_f32, hipStream_t s) {
    if (in_f32) return launch<float, float>(a, s);
    if (out_f32) return launch<uint16_t, float>(a, s);
    return launch<uint16_t, uint16_t>(a, s);
}

}  // namespace sbpi
