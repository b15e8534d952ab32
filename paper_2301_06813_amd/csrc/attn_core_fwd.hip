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

#include "attn_core_kernel.h"
#include "gemm.h"
#include "profile.h"

namespace sbpk {

// O rows of 4 consecutive values starting at column `col` (col < d).
template <class F>
__device__ __forceinline__ void store4(void *base, int64_t at, int col, int d, bool f32, bool vec,
                                       F value) {
    if (f32) {
        float *p = static_cast<float *>(base) + at + col;
        if (vec && col + 4 <= d) {
            f32x4 v = {value(0), value(1), value(2), value(3)};
            *reinterpret_cast<f32x4 *>(p) = v;
            return;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < d) p[e] = value(e);
    } else {
        uint16_t *p = static_cast<uint16_t *>(base) + at + col;
        if (vec && col + 4 <= d) {
            u32x2 w;
            w[0] = (uint32_t)f32_to_bf16_bits(value(0)) | (uint32_t)f32_to_bf16_bits(value(1)) << 16;
            w[1] = (uint32_t)f32_to_bf16_bits(value(2)) | (uint32_t)f32_to_bf16_bits(value(3)) << 16;
            *reinterpret_cast<u32x2 *>(p) = w;
            return;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < d) p[e] = f32_to_bf16_bits(value(e));
    }
}

// Exponents of base 2 beyond which a wave forms differences of scores first: the rounding of
// m c is at most 2^-15 below it.
constexpr float FAR = 1024.f;

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

// WPS: waves of a SIMD, of one workgroup or two.
template <int DP, int KG, int KT, int NW_, int WPS_, bool DMA>
struct FwdShape {
    static constexpr int NW = NW_, WPS = WPS_;
    static constexpr int ROWS = 32 * NW / KG, KEYS = KG * KT;
    using Tile = RowTile<DP, KEYS, NW>;
    static constexpr int STAGE = 2 * Tile::BYTES;    // K, then V
    static constexpr int LOADS = 2 * Tile::NV;
    static constexpr int ROOM = 163840 / (4 * WPS / NW);
    static constexpr int FIT = ROOM / STAGE;
    static constexpr int NS = !DMA ? 3 : FIT > 4 ? 4 : FIT;
    static constexpr int PUT = NW * PUT_FLOATS<DP> * 4;
    static constexpr int STATS = NW * 64 * 2 * 4;
    static constexpr int LDS = NS * STAGE > PUT + STATS ? NS * STAGE : PUT + STATS;
    static_assert(FIT >= NS && NS >= 3 && LDS <= ROOM, "three stages");
};

template <int DP, int KG, int KT, int NW, int WPS, bool DMA>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(WPS, WPS)))
void attn_core_fwd_kernel(FwdArgs f) {
    using S = FwdShape<DP, KG, KT, NW, WPS, DMA>;
    using Tile = typename S::Tile;
    constexpr int ROWS = S::ROWS, NS = S::NS, KEYS = S::KEYS;
    constexpr int NB = KT / 32, KS = DP / 16, DB = DP / 32;
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

    // rows past a sequence's queries read nothing
    const bool live = valid && i < mask.lq;
    const uint16_t *Q = static_cast<const uint16_t *>(a.q.p) + (int64_t)b * a.q.sb +
                        head * a.q.sh + (int64_t)i * a.q.ld;
    bf16x8 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
        qf[ks] = row_frag<DMA>(Q, ks * 16 + 8 * half, live ? a.d : 0);
    settle(qf);

    const float c = a.scale * LOG2E;
    const float grow = 8.f / c;
    float m = -INFINITY, l = 0.f;
    float mc = 0.f, limit = -INFINITY;   // what exponents add to s c; where the maximum moves
    f32x16 o[DB];
#pragma unroll
    for (int x = 0; x < DB; ++x) o[x] = splat16(0.f);

    // Two phases a block of 32 keys: the next block's scores beside this one's exponentials;
    // then this block's product with V beside the next one's maximum. The first phase has
    // priority over the other wave's second, which waits for less (16 heads over 4 of
    // 8192 x 128, causal: 273 us without, 260).
    typename Tile::Reader rd(lds0 + kg * KT / Tile::RPS * Tile::SEG, lane);
    f32x16 sp[2];                   // scores of this block and the next, in turn
    int stage = 0;                  // of the step at work
    auto scores = [&](f32x16 &s, const typename Tile::Reader &r, int r0, auto beside)
                      __attribute__((always_inline)) {
        // operands are read AHEAD products early
        constexpr int AHEAD = KS < 4 ? KS : 4;
        bf16x8 k[KS];
        s = splat16(0.f);
#pragma unroll
        for (int ks = 0; ks < AHEAD; ++ks) k[ks] = r.frag(r0, ks, 0);
        beside(0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            if (ks + AHEAD < KS) k[ks + AHEAD] = r.frag(r0, ks + AHEAD, 0);
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[ks], qf[ks], s, 0, 0, 0);
            beside(ks + 1);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto hide = [&](f32x16 &s, int k0, int r) {   // what this row does not see
        const int key = k0 + 8 * (r >> 2) + 4 * half + (r & 3);
        s[r] = key >= lo && key < hi ? s[r] : -INFINITY;
    };
    // Moves the maximum to `top`, the maximum of a lane's own scores s, where it grew by enough.
    // Where a row's is FAR, s become differences from it, and every block comes here.
    auto rise = [&](f32x16 &s, float top) __attribute__((always_inline)) {
        float t0, t1;
        halves(top, &t0, &t1);
        top = fmaxf(t0, t1);
        if (__any(top > limit)) {
            const float mn = fmaxf(m, top);
            const float x = mn == -INFINITY ? 1.f : exp2_((m - mn) * c);
            m = mn;
            limit = m + grow;
            mc = m == -INFINITY ? 0.f : -m * c;
            l *= x;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[db][r] *= x;
            if (__any(fabsf(mc) > FAR)) {
                const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] -= base;
                mc = 0.f;
                limit = -INFINITY;
            }
        }
    };
    // Waits for the step after x, and prepares the load of a later one.
    auto advance = [&](int x) __attribute__((always_inline)) {
        if constexpr (DMA) {
            wait_vm<(NS - 3) * S::LOADS>();
            __syncthreads();
            fetch(x + NS - 1, stage == 0 ? NS - 1 : stage - 1);
        } else {
            if (x + 1 < s1) arrive(stage == NS - 1 ? 0 : stage + 1);
            __syncthreads();
            if (x + 2 < s1) fetch(x + 2, 0);
        }
    };
    // EDGE: some row of the tile does not see every key of the step
    auto take = [&](int x, auto edge) __attribute__((always_inline)) {
        constexpr bool EDGE = decltype(edge)::value;
        const int kw = k_beg + walk.step(x) * KEYS + kg * KT;
        const int kn = k_beg + walk.step(x + 1) * KEYS + kg * KT;
        const bool wrap = stage == NS - 1;
        const int by = wrap ? -(NS - 1) * S::STAGE : S::STAGE;
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
            const bool last = kb == NB - 1;
            if (last) advance(x);
            typename Tile::Reader nx = rd;       // where the next block lies
            if (last) nx.move(by);
            // with an even number of blocks a step the two take turns in place
            constexpr bool TURN = NB % 2 == 0;
            constexpr int ONE = 1;
            const int now = TURN ? kb & 1 : 0;
            f32x16 &s = sp[now], &s_n = sp[ONE - now];
            bf16x8 tv[2][DB], p[2];
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
            scores(s_n, nx, last ? 0 : (kb + 1) * 32, [&](int part) __attribute__((always_inline)) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    if (!in_part(r, part, KS + 1)) continue;
                    s[r] = exp2_(__builtin_fmaf(s[r], c, mc));
                    l += s[r];
                    if (r % 8 == 7) p[r / 8] = pack8(s, r - 7);
                }
                // the first 16 keys' columns
                if (part > KS - DB)
                    tv[0][part - 1 - (KS - DB)] = rd.frag_t(part - 1 - (KS - DB), kb * 32, Tile::BYTES);
            });
            __builtin_amdgcn_s_setprio(0);
            // the loads of a step, spread over its blocks: the last one's first
            constexpr int PER = (S::LOADS + NB - 1) / NB;
            const int first = last ? 0 : (kb + 1) * PER;
            float top = -INFINITY;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tv[h][db], p[h], o[db], 0, 0, 0);
                    if (h == 0) tv[1][db] = rd.frag_t(db, kb * 32 + 16, Tile::BYTES);
                    const int k = h * DB + db;
#pragma unroll
                    for (int q = PER * k / (2 * DB); q < PER * (k + 1) / (2 * DB); ++q)
                        if (first + q < S::LOADS) fetch_part(first + q);
                    // the next scores are there one product later
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        if (k == 0 || !in_part(r, k - 1, 2 * DB - 1)) continue;
                        if constexpr (EDGE) hide(s_n, last ? kn : kw + (kb + 1) * 32, r);
                        top = fmaxf(top, s_n[r]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            if (!last || x + 1 < s1) rise(s_n, top);
            if constexpr (!TURN) sp[0] = sp[1];
        }
        rd.move(by);
        stage = wrap ? 0 : stage + 1;
    };
    if (s0 < s1) {
        if constexpr (DMA) wait_vm<(NS - 2) * S::LOADS>();
        __syncthreads();
        scores(sp[0], rd, 0, [](int) {});
        const int kw = k_beg + walk.step(s0) * KEYS + kg * KT;
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            hide(sp[0], kw, r);
            top = fmaxf(top, sp[0][r]);
        }
        rise(sp[0], top);
    }
    int x = s0;
    for (; x < min(s1, walk.masked()); ++x) take(x, std::true_type{});
    for (; x < s1; ++x) take(x, std::false_type{});
    wait_vm<0>();      // no load is on its way to LDS any more
    __syncthreads();

    float l0, l1;
    halves(l, &l0, &l1);
    l = l0 + l1;
    float mul = 1.f;         // 2^((m - the groups' maximum) c)
    if constexpr (KG > 1) {
        float *const stats = reinterpret_cast<float *>(smem + S::PUT) + lane;
        stats[wave * 128] = m;
        stats[wave * 128 + 64] = l;
        __syncthreads();
        const float *const p = stats + wr * KG * 128;
        float mn = p[0];
#pragma unroll
        for (int k = 1; k < KG; ++k) mn = fmaxf(mn, p[k * 128]);
        const float ms = mn == -INFINITY ? 0.f : mn;
        l = 0.f;
#pragma unroll
        for (int k = 0; k < KG; ++k) l += p[k * 128 + 64] * exp2_((p[k * 128] - ms) * c);
        mul = exp2_((m - ms) * c);
        m = mn;
    }
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
    stage_rows<DP>(put + wave * PUT_FLOATS<DP>, o, some ? mul / l : 0.f, lane);
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
