// attn_core_fwd.hip -- softmax attention, forward.
//
// Per sequence and key head, the rows of a group of query heads that share it
// are packed as row = i * group + g (query i, head g), so K and V are read once
// for the group and a few query rows fill a tile. A workgroup owns a tile of rows
// and walks over the keys that any of them sees, 64 or 128 at a time: scores
// as S^T = K Q^T, running maximum m and sum l of each row, O^T += V^T P^T. In these
// orientations a lane holds one query's scores (half of them, the other half-wave
// the rest), so m and l are one register each, the rows' scaling needs no
// broadcast, and P^T goes from the exponentials into the second product without
// leaving its registers.
//
//   * exp(scale (s - m)) is one multiply-add and one base-2 exponential a score. That
//     multiply-add takes off m's product rounded, which is as good as the difference while
//     the product is small; where it is not (FAR) the difference is formed first, so that
//     the largest score has the weight 1 however large it is.
//     The maximum is moved only when a row's grows by more than 8 in the exponent:
//     until then sums and outputs grow by up to 2^8, far inside fp32, and rescaling
//     is skipped by the whole wave.
//   * P is rounded to bf16 for the second product (the matrix cores' type, rounded
//     like the framework's other bf16 operands); the row sum adds the fp32 values.
//   * The next block's scores are computed beside this block's exponentials, and its
//     maximum beside this block's product with V (written one after the other,
//     16 heads over 4 of 8192 x 128, causal, took 314 us; so 256, 1.07 PFLOP/s, at two
//     waves per SIMD).
//   * With KG wave groups, group k takes the k-th part of every step's keys; their
//     (m, l, O) are joined through LDS at the end. Few rows and many keys are also
//     split over workgroups, whose normalised partial outputs and row statistics
//     go through the workspace.
#include <math.h>

#include <algorithm>

#include "attn_core_walk.h"
#include "gemm.h"
#include "profile.h"

namespace sbpk {

struct FwdArgs {
    CoreArgs a;
    int32_t tiles, splits, rows;     // row tiles per (sequence, key head); rows = sq * group
    int32_t vec;                     // O allows 4-value stores
    Div per, by_split, heads, kv, group, by_rows;   // tiles x splits, splits, batch x key heads, ...
};

// The split parts' statistics, behind their partial outputs: a row's maximum and its sum of
// exponents, apart, since a large maximum has no bits left for the logarithm of the sum.
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ f32x2 *stats_of(const FwdArgs &f, int64_t d4) {
    return reinterpret_cast<f32x2 *>(f.a.ws +
                                     (int64_t)f.splits * f.a.batch * f.a.kv_heads * f.rows * d4);
}

template <int DP, int KG, int KT, int NW, int WPS, bool DMA>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(WPS, WPS)))
void attn_core_fwd_kernel(FwdArgs f) {
    using S = FwdShape<DP, KG, KT, NW, WPS, DMA>;
    using Tile = typename S::Tile;
    constexpr int ROWS = S::ROWS, NS = S::NS, KEYS = S::KEYS;
    constexpr int KS = DP / 16;
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS];
    const uint32_t lds0 = lds_at(smem);
    const CoreArgs &a = f.a;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);   // uniform, so that what
                                                                 // depends on it is scalar
    const int kg = wave % KG, wr = wave / KG;
    // the arguments, read at once: the compiler loads each where it is first used, and each
    // first load is a trip to memory
    asm volatile("" ::"s"(a.q.p), "s"(a.q.sb), "s"(a.q.sh), "s"(a.q.ld), "s"(a.k.p), "s"(a.k.sb),
                 "s"(a.k.sh), "s"(a.k.ld), "s"(a.v.p), "s"(a.v.sb), "s"(a.v.sh), "s"(a.v.ld),
                 "s"(a.o.p), "s"(a.lse.p), "s"(a.len_q), "s"(a.len_k), "s"(a.batch),
                 "s"(a.kv_heads), "s"(a.group), "s"(a.sq), "s"(a.sk), "s"(a.d), "s"(a.causal),
                 "s"(a.window), "s"(a.scale), "s"(a.ws), "s"(f.tiles), "s"(f.splits), "s"(f.rows));

    // heavier (later) causal tiles first within a (sequence, head)
    int bh, t;
    deal(blockIdx.x, f.heads, f.per, &bh, &t);
    const int up = f.by_split(t), tile = f.tiles - 1 - up, split = f.by_split.rest(t, up);
    const int b = f.kv(bh), hk = f.kv.rest(bh, b);
    const SeqMask mask(a, b);

    const int row0 = tile * ROWS;
    const int row = row0 + wr * 32 + (lane & 31);
    const bool valid = row < f.rows;
    const int i = f.group(valid ? row : f.rows - 1);
    const int g = (valid ? row : f.rows - 1) - i * a.group;
    const int64_t head = (int64_t)hk * a.group + g;

    // the keys that the tile's rows see, and this split's steps of them
    const int i_first = f.group(row0);
    const int i_last = f.group(min(row0 + ROWS, f.rows) - 1);
    const int k_beg = mask.lo(i_first) & ~31;
    const int k_end = i_first < mask.lq ? mask.hi(min(i_last, mask.lq - 1)) : 0;
    const int steps = k_end > k_beg ? (k_end - k_beg + KEYS - 1) / KEYS : 0;
    // steps whose keys every row of the tile sees (rows past the sequence's end aside)
    Walk walk{steps, 0, steps};
    if (steps > 0) {
        const int all = min(mask.hi(i_first), mask.lk);
        walk.nb = all > k_beg ? min(steps, (all - k_beg) / KEYS) : 0;
        walk.na = max(0, min(walk.nb, (mask.lo(i_last) - k_beg + KEYS - 1) / KEYS));
    }
    const int per_split = f.by_split(steps + f.splits - 1);
    const int s0 = min(steps, split * per_split), s1 = min(steps, s0 + per_split);
    const int hi = mask.hi(i), lo = mask.lo(i);

    const uint16_t *K = static_cast<const uint16_t *>(a.k.p) + (int64_t)b * a.k.sb +
                        (int64_t)hk * a.k.sh;
    const uint16_t *V = static_cast<const uint16_t *>(a.v.p) + (int64_t)b * a.v.sb +
                        (int64_t)hk * a.v.sh;
    const int place_k = Tile::place(a.k.ld, a.d, wave, lane);
    const int place_v = Tile::place(a.v.ld, a.d, wave, lane);
    typename Tile::Regs rk, rv;
    Fetch to{};
    // steps past the walk's bring nothing (zeros, to a stage that is not read)
    auto fetch = [&](int x, int stage) __attribute__((always_inline)) {
        const int k0 = k_beg + walk.step(x) * KEYS;
        const int n = x < s1 ? min(KEYS, mask.lk - k0) : 0;
        if constexpr (DMA) {
            to.x = make_rsrc(K + (int64_t)k0 * a.k.ld);
            to.y = make_rsrc(V + (int64_t)k0 * a.v.ld);
            to.x[2] = __builtin_amdgcn_readfirstlane(n * (int)a.k.ld * 2);
            to.y[2] = __builtin_amdgcn_readfirstlane(n * (int)a.v.ld * 2);
            to.lds = lds0 + stage * S::STAGE;
        } else {
            Tile::load(rk, K + (int64_t)k0 * a.k.ld, a.k.ld, n, a.d, tid);
            Tile::load(rv, V + (int64_t)k0 * a.v.ld, a.v.ld, n, a.d, tid);
        }
    };
    auto fetch_part = [&](int p) {
        if constexpr (DMA) {
            if (p < Tile::NV) Tile::issue(to.x, a.k.ld, place_k, to.lds, wave, p);
            else Tile::issue(to.y, a.v.ld, place_v, to.lds + Tile::BYTES, wave, p - Tile::NV);
        }
    };
    auto arrive = [&](int stage) {   // register-staged: the loaded step goes to LDS
        if constexpr (!DMA) {
            char *lds = smem + stage * S::STAGE;
            Tile::store(rk, lds, tid);
            Tile::store(rv, lds + Tile::BYTES, tid);
        }
    };
    if constexpr (DMA) {
#pragma unroll
        for (int x = 0; x < NS - 1; ++x) {
            fetch(s0 + x, x);
#pragma unroll
            for (int p = 0; p < S::LOADS; ++p) fetch_part(p);
        }
        fetch(s1, NS - 1);   // nothing, for the parts before the first advance
    } else if (s0 < s1) {
        fetch(s0, 0);
        arrive(0);
        if (s0 + 1 < s1) fetch(s0 + 1, 1);
    }

    FwdRows<S> w(lds0 + kg * KT / Tile::RPS * Tile::SEG, lane, a.scale, lo, hi);
    // rows past a sequence's queries read nothing
    const bool live = valid && i < mask.lq;
    const uint16_t *Q = static_cast<const uint16_t *>(a.q.p) + (int64_t)b * a.q.sb +
                        head * a.q.sh + (int64_t)i * a.q.ld;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
        w.qf[ks] = row_frag<DMA>(Q, ks * 16 + 8 * half, live ? a.d : 0);
    settle(w.qf);

    // Waits for the step after x, and prepares the load of a later one.
    auto advance = [&](int x) __attribute__((always_inline)) {
        if constexpr (DMA) {
            wait_vm<(NS - 3) * S::LOADS>();
            __syncthreads();
            fetch(x + NS - 1, w.stage == 0 ? NS - 1 : w.stage - 1);
        } else {
            if (x + 1 < s1) arrive(w.stage == NS - 1 ? 0 : w.stage + 1);
            __syncthreads();
            if (x + 2 < s1) fetch(x + 2, 0);
        }
    };
    auto seen = [&](int k0) { return w.seen(k0); };
    auto first_key = [&](int x) { return k_beg + walk.step(x) * KEYS + kg * KT; };
    auto take = [&](int x, auto edge) __attribute__((always_inline)) {
        w.template take<decltype(edge)::value>(first_key(x), first_key(x + 1), x + 1 < s1, seen,
                                               [&]() __attribute__((always_inline)) { advance(x); },
                                               fetch_part);
    };
    if (s0 < s1) {
        if constexpr (DMA) wait_vm<(NS - 2) * S::LOADS>();
        __syncthreads();
        w.begin(first_key(s0), seen);
    }
    int x = s0;
    for (; x < min(s1, walk.masked()); ++x) take(x, std::true_type{});
    for (; x < s1; ++x) take(x, std::false_type{});
    wait_vm<0>();      // no load is on its way to LDS any more
    __syncthreads();

    const float mul = w.join_groups(reinterpret_cast<float *>(smem + S::PUT) + lane, wave, wr);
    const float m = w.m, l = w.l;
    // a row that sees no key: O = 0, lse = -infinity
    const bool some = live && l != 0.f;
    const float log_l = __builtin_amdgcn_logf(l);
    const bool whole = f.splits == 1;
    const int64_t d4 = (a.d + 3) & ~3;
    const int64_t at = (((int64_t)split * a.batch * a.kv_heads) + bh) * f.rows + row;
    const RowsOut out{whole ? a.o.p : a.ws, whole ? a.d : (int)d4, !whole || a.o_f32, false,
                      !whole || f.vec};
    const int64_t off = !valid ? -1
                        : whole ? (int64_t)b * a.o.sb + head * a.o.sh + (int64_t)i * a.o.ld
                                : at * d4;
    float *const put = reinterpret_cast<float *>(smem);
    stage_rows<DP>(put + wave * PUT_FLOATS<DP>, w.o, some ? mul / l : 0.f, lane);
    if (valid && half == 0 && kg == 0) {
        if (!whole)
            stats_of(f, d4)[at] = some ? f32x2{m, l} : f32x2{-INFINITY, 0.f};
        else if (a.lse.p)
            static_cast<float *>(a.lse.p)[(int64_t)b * a.lse.sb + head * a.lse.sh +
                                          (int64_t)i * a.lse.ld] =
                some ? __builtin_fmaf(m, a.scale, log_l * LN2) : -INFINITY;
    }
    __syncthreads();
    store_rows<DP, KG>(put + wr * KG * PUT_FLOATS<DP>, PUT_FLOATS<DP>, kg, out, off, lane);
}

// Joins the key splits of a row, in split order: weights l_s 2^((m_s - m) c). A thread
// owns 4 columns of a row, 16 (32 past 64 columns) a row.
__global__ __launch_bounds__(256) void attn_core_join_kernel(FwdArgs f) {
    const CoreArgs &a = f.a;
    const int lanes = a.d > 64 ? 5 : 4;
    const int64_t n = (int64_t)a.batch * a.kv_heads * f.rows, d4 = (a.d + 3) & ~3;
    const uint32_t id = blockIdx.x * 256u + threadIdx.x;
    const int at = (int)(id >> lanes), col = (int)(id & ((1u << lanes) - 1)) * 4;
    if (at >= n || col >= a.d) return;
    const f32x2 *stat = stats_of(f, d4) + at;
    const float *part = a.ws + at * d4 + col;
    const float c = a.scale * LOG2E;
    // 8 splits at a time, so that their reads are on the way together
    float top = -INFINITY, total = 0.f;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < f.splits; s += 8) {
        f32x2 w[8];
        f32x4 x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool in = s + j < f.splits;
            w[j] = in ? stat[(s + j) * n] : f32x2{-INFINITY, 0.f};
            x[j] = in ? *reinterpret_cast<const f32x4 *>(part + (s + j) * n * d4)
                      : f32x4{0.f, 0.f, 0.f, 0.f};
        }
        float high = top;
#pragma unroll
        for (int j = 0; j < 8; ++j) high = fmaxf(high, w[j][0]);
        const float base = high == -INFINITY ? 0.f : high;
        const float old = exp2_((top - base) * c);
        total *= old;
        v *= old;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float e = w[j][1] * exp2_((w[j][0] - base) * c);
            total += e;
            v += x[j] * e;
        }
        top = high;
    }
    const bool some = total != 0.f;
    const float inv = some ? 1.f / total : 0.f;
    const int bh = f.by_rows(at), row = f.by_rows.rest(at, bh);
    const int b = f.kv(bh), hk = f.kv.rest(bh, b);
    const int i = f.group(row);
    const int64_t head = (int64_t)hk * a.group + (row - i * a.group);
    store4(a.o.p, (int64_t)b * a.o.sb + head * a.o.sh + (int64_t)i * a.o.ld, col, a.d, a.o_f32,
           f.vec, [&](int e) { return v[e] * inv; });
    if (a.lse.p && col == 0)
        static_cast<float *>(a.lse.p)[(int64_t)b * a.lse.sb + head * a.lse.sh +
                                      (int64_t)i * a.lse.ld] =
            some ? __builtin_fmaf(top, a.scale, __builtin_amdgcn_logf(total) * LN2) : -INFINITY;
}

}  // namespace sbpk

namespace sbpi {

namespace {

template <int DP, int KG, int KT, int NW, int WPS>
hipError_t launch_fwd(const sbpk::FwdArgs &f, int64_t blocks, hipStream_t s) {
    char name[160];
    name[0] = 0;
    if (profiling())
        snprintf(name, sizeof(name), "attn_core_fwd_kernel<%d,%d,%d,%d,%d>", DP, KG, KT, NW,
                 (int)f.a.aligned);
    if (f.a.aligned)
        return launch_kernel(sbpk::attn_core_fwd_kernel<DP, KG, KT, NW, WPS, true>, name,
                             dim3((unsigned)blocks), dim3(64 * NW), s, f);
    return launch_kernel(sbpk::attn_core_fwd_kernel<DP, KG, KT, NW, WPS, false>, name,
                         dim3((unsigned)blocks), dim3(64 * NW), s, f);
}

// The kernel's forms: rows of a tile, keys of a step, waves, workgroups of a unit, us of a step. The
// second and third give up speed a row for smaller tiles: 16 heads over 4 of 8192 x 128,
// causal, take 256, 292 and 405 us (in a graph, like all of these); 16 heads of 1024 x 64,
// causal, 19.1, 14.3 and 16.9; one token of 16 sequences, 4 key heads with 4 rows each, 4096 x
// 64, whose keys are split, 20.4, 18.4 and 19.3 (20.0, 17.5 and 16.5 where the sequences
// have from 4096 keys down to 1200, which the host does not know).
struct Form {
    int rows, keys, waves, per_cu;
    double step;
};
constexpr Form FORMS[2][3] = {{{128, 64, 4, 2, 0.9}, {64, 64, 4, 2, 0.55}, {32, 128, 4, 1, 0.6}},
                              {{256, 64, 8, 1, 1.4}, {128, 64, 8, 1, 1.0}, {64, 64, 4, 1, 0.75}}};

// The form (returned) and key splits that the following time expects least of: an item takes
// so much a step, and `fixed` besides; the busiest unit has an even share of all items and
// half of the longest; partials are written and read once, by one more launch.
int plan_fwd(const CoreArgs &a, int64_t bhs, int cus, int64_t *splits) {
    const Form *forms = FORMS[a.d > 64];
    const int64_t packed = (int64_t)a.sq * a.group;
    const size_t d4 = (a.d + 3) & ~3;
    const double fixed = 3.5;
    double best = 1e300;
    int form = 0;
    *splits = 1;
    for (int k = 0; k < 3; ++k) {
        const Form &m = forms[k];
        const int64_t tiles = (packed + m.rows - 1) / m.rows;
        const int64_t keys = a.causal && a.window
                                 ? std::min<int64_t>(a.sk, a.window + m.rows / a.group)
                                 : a.sk;
        const int64_t steps = (keys + m.keys - 1) / m.keys;
        // a causal walk is half as long on average where it starts at nothing
        const double mean = a.causal && !a.window
                                ? steps * (1.0 - 0.5 * std::min<double>(1.0, (double)a.sq / a.sk))
                                : (double)steps;
        for (int64_t v = 1; v <= 32; v *= 2) {
            const size_t part = v > 1 ? (size_t)bhs * packed * v * (d4 + 2) : 0;
            // a launch's threads fit 32 bits (the last form's always do, with whole walks)
            if ((double)tiles * bhs * v * (64 * m.waves) > 4294967295.0) break;
            if (v > 1 && (steps / v < 2 || part > a.ws_floats ||
                          (double)bhs * packed > 134217727.0))   // the join's threads
                break;
            const double item = fixed + (double)((steps + v - 1) / v) * m.step;
            const double all = (mean * m.step + v * fixed) * tiles * bhs / (cus * m.per_cu);
            const double t = std::max(item, all + 0.5 * item) + (v > 1 ? 3.5 + part * 8 / 4e6 : 0);
            if (t < best * 0.98) {
                best = t;
                form = k;
                *splits = v;
            }
        }
    }
    return form;
}

}  // namespace

hipError_t launch_core_fwd(const CoreArgs &a, hipStream_t s) {
    sbpk::FwdArgs f;
    f.a = a;
    f.rows = a.sq * a.group;
    const int esz = a.o_f32 ? 4 : 2;
    f.vec = a.d % 4 == 0 && reinterpret_cast<uintptr_t>(a.o.p) % (4 * esz) == 0 &&
            a.o.ld % 4 == 0 && a.o.sb % 4 == 0 && a.o.sh % 4 == 0;
    const int64_t bhs = (int64_t)a.batch * a.kv_heads;
    int64_t splits;
    const int form = plan_fwd(a, bhs, device_cus(), &splits);
    const bool wide = a.d > 64;
    const int rows = FORMS[wide][form].rows;
    f.tiles = (f.rows + rows - 1) / rows;
    f.splits = (int)splits;
    f.per = sbpk::Div((int64_t)f.tiles * splits);
    f.by_split = sbpk::Div(splits);
    f.heads = sbpk::Div(bhs);
    f.kv = sbpk::Div(a.kv_heads);
    f.group = sbpk::Div(a.group);
    f.by_rows = sbpk::Div(f.rows);
    const int64_t blocks = (int64_t)f.tiles * bhs * splits;
    hipError_t e;
    if (form == 0)
        e = wide ? launch_fwd<128, 1, 64, 8, 2>(f, blocks, s) : launch_fwd<64, 1, 64, 4, 2>(f, blocks, s);
    else if (form == 1)
        e = wide ? launch_fwd<128, 2, 32, 8, 2>(f, blocks, s) : launch_fwd<64, 2, 32, 4, 2>(f, blocks, s);
    else
        e = wide ? launch_fwd<128, 2, 32, 4, 1>(f, blocks, s) : launch_fwd<64, 4, 32, 4, 1>(f, blocks, s);
    if (e != hipSuccess || splits == 1) return e;
    const int64_t items = bhs * f.rows * (wide ? 32 : 16);
    return launch_kernel(sbpk::attn_core_join_kernel, "attn_core_join_kernel",
                         dim3((unsigned)((items + 255) / 256)), dim3(256), s, f);
}

}  // namespace sbpi
