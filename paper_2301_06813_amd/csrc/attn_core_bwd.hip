// attn_core_bwd.hip -- softmax attention, backward: the probabilities are
// recomputed from Q, K and the forward pass's row statistics,
//   P = exp(scale Q K^T - lse),  dV = P^T dO,  dS = P (dO V^T - D),
//   dQ = scale dS K,  dK = scale dS^T Q,  D_i = sum_c dO_ic O_ic.
//
// Two launches, or three where walks are split, none with atomics, so the results do not
// depend on the order in which workgroups run:
//   * row statistics: -lse / scale and D of every query row go to the workspace;
//   * the gradients. A workgroup of dK and dV owns keys and walks over the rows that see
//     them, of every query head that shares the key head; one of dQ owns query rows (packed
//     over the query heads that share a key head, as in the forward kernel) and walks
//     over their keys. One launch holds both kinds, dK's and dV's first: they are longer,
//     and the others fill the units that they leave (16 heads of 1024 x 64, causal: 18 + 23 us
//     in two launches, 27 in one);
//   * sums of the parts of split walks.
// Scores and dO V^T are thus computed twice, seven products where five are needed;
// the alternative, one pass that adds dQ in memory, needs fp32 atomics (in
// an order that changes the result) or a partial dQ for every key tile.
//
// The statistics are the products' initial accumulators: starting S = Q K^T at
// -lse / scale and dO V^T at -D leaves one multiplication, one exponential and one
// product a score. P and dS are rounded to bf16 for the products that read them;
// every sum is fp32.
#include <math.h>

#include <algorithm>

#include "attn_core_kernel.h"
#include "gemm.h"
#include "profile.h"

namespace sbpk {

// Under a causal mask the first keys are seen by every row and the last by few, so the
// first tiles' walks are split over more workgroups. Level j: key tiles [tile[j],
// tile[j+1]), split v[j] ways (falling); its work items start at item[j], and its
// partials, where v[j] > 1, at slot[j], of one (sequence, key head).
constexpr int MAX_LEVELS = 8;
struct Levels {
    int32_t n;
    int32_t tile[MAX_LEVELS + 1], v[MAX_LEVELS], item[MAX_LEVELS], slot[MAX_LEVELS];
    int32_t items;                     // of one (sequence, key head)
    int32_t split_keys;                // keys of the tiles with v > 1
};

struct BwdArgs {
    CoreArgs a;
    int32_t tiles_q, splits_q, rows;   // dQ: row tiles, key splits; rows = sq * group
    int32_t items_kv;                  // workgroups of dK and dV; those of dQ follow
    Levels lev;
    int32_t vec_q, vec_k, vec_v;       // outputs allow 4-value stores
    const float *nl, *nd;              // row statistics: -lse / scale, -D, per (b, head, i)
    float *part_q, *part_kv;           // split partials
    Div per_q, by_split, per_kv, heads, kv, group, by_rows, by_keys;   // tiles_q x splits_q, ...
};

// Adds to or overwrites 4 consecutive values of an output row.
template <class F>
__device__ __forceinline__ void grad4(void *base, int64_t at, int col, int d, bool f32, bool acc,
                                      bool vec, F value) {
    if (f32) {
        float *p = static_cast<float *>(base) + at + col;
        if (vec && col + 4 <= d) {
            f32x4 v = {value(0), value(1), value(2), value(3)};
            if (acc) v += *reinterpret_cast<const f32x4 *>(p);
            *reinterpret_cast<f32x4 *>(p) = v;
            return;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < d) p[e] = acc ? p[e] + value(e) : value(e);
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

// Row statistics: 16 lanes a row. Rows that see no key (lse = -infinity) or lie past
// the sequence's length get -infinity and 0, which makes their P and dS zero.
__global__ __launch_bounds__(256) void attn_core_stat_kernel(CoreArgs a, Div by_sq, Div by_heads,
                                                             float *nl, float *nd) {
    const int heads = a.kv_heads * a.group;
    const int64_t n = (int64_t)a.batch * heads * a.sq;
    const int r = (int)blockIdx.x * 16 + (int)(threadIdx.x >> 4);
    const int at = (threadIdx.x & 15) * 8;
    if (r >= n) return;
    const int bh = by_sq(r), i = by_sq.rest(r, bh);
    const int64_t b = by_heads(bh), h = by_heads.rest(bh, (int)b);
    const int lq = a.len_q ? min(max(a.len_q[b], 0), a.sq) : a.sq;
    const float lse = i < lq ? static_cast<const float *>(a.lse.p)[b * a.lse.sb + h * a.lse.sh +
                                                                   i * a.lse.ld]
                             : -INFINITY;
    const bool live = lse != -INFINITY;
    float x = 0.f;
    if (live && at < a.d) {
        const bf16x8 g = row_frag<false>(static_cast<const uint16_t *>(a.dout.p) + b * a.dout.sb +
                                             h * a.dout.sh + i * a.dout.ld,
                                         at, a.d);
        const int64_t o = b * a.o.sb + h * a.o.sh + i * a.o.ld;
        if (a.o_f32) {
            const float *p = static_cast<const float *>(a.o.p) + o;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (at + e < a.d) x += (float)g[e] * p[at + e];
        } else {
            const bf16x8 y = row_frag<false>(static_cast<const uint16_t *>(a.o.p) + o, at, a.d);
#pragma unroll
            for (int e = 0; e < 8; ++e) x += (float)g[e] * (float)y[e];
        }
    }
#pragma unroll
    for (int s = 8; s > 0; s >>= 1) x += __shfl_xor(x, s, 16);
    if ((threadIdx.x & 15) == 0) {
        nl[r] = live ? -lse / a.scale : -INFINITY;
        nd[r] = live ? -x : 0.f;
    }
}

// ------------------------------------------------------------------- dQ
// Both kernels walk with 32 x 32 blocks of scores a wave, in two phases: S and dP of the
// next block, whose products alternate, beside this block's exponentials and roundings;
// then this block's products with them, whose order is kept as written (sched_barrier), the
// operands of the later ones and the loads of a step spread over them: left to itself the
// compiler read operands right before their use. (Kept in the first phase too, the
// order cost 3%: 16 heads over 4 of 8192 x 128, causal, 1020 us and 985.) With 128 columns the
// sums leave room for one wave per SIMD, which hides nothing behind another.

// S and dP of one block: S from the operand rows at `r` and `qf`, dP from the rows OFF bytes
// behind and `gf`. beside(i), i = 0 .. KS: what is written between the products.
template <int KS, int OFF, class Reader, class Beside>
__device__ __forceinline__ void block_scores(f32x16 &s, f32x16 &dp, const Reader &r, int r0,
                                             const bf16x8 *qf, const bf16x8 *gf, Beside beside) {
    // operands are read AHEAD products early: a read of LDS takes longer than two products
    constexpr int AHEAD = KS < 4 ? KS : 4;
    bf16x8 q[KS], g[KS];
#pragma unroll
    for (int ks = 0; ks < AHEAD; ++ks) {
        q[ks] = r.frag(r0, ks, 0);
        g[ks] = r.frag(r0, ks, OFF);
    }
    beside(0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        if (ks + AHEAD < KS) {
            q[ks + AHEAD] = r.frag(r0, ks + AHEAD, 0);
            g[ks + AHEAD] = r.frag(r0, ks + AHEAD, OFF);
        }
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q[ks], qf[ks], s, 0, 0, 0);
        dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(g[ks], gf[ks], dp, 0, 0, 0);
        beside(ks + 1);
    }
}

template <int DP, int KG, int KT, bool DMA>
struct DqShape {
    static constexpr int NW = 4;
    static constexpr int ROWS = 32 * NW / KG;
    using Tile = RowTile<DP, KG * KT, NW>;
    static constexpr int STAGE = 2 * Tile::BYTES;
    static constexpr int LOADS = 2 * Tile::NV;
    static constexpr int OCC = DP > 64 ? 1 : 2;
    static constexpr int FIT = 163840 / OCC / STAGE;
    static constexpr int NS = !DMA ? 3 : FIT > 4 ? 4 : FIT;
    static constexpr int PUT = NW * PUT_FLOATS<DP> * 4;
    static constexpr int LDS = NS * STAGE > PUT ? NS * STAGE : PUT;
    static_assert(FIT >= NS && NS >= 3 && LDS <= 163840 / OCC, "three stages");
};

template <int DP, int KG, int KT, bool DMA>
__device__ __forceinline__ void attn_core_dq(const BwdArgs &f, int wg, char *smem) {
    using S = DqShape<DP, KG, KT, DMA>;
    using Tile = typename S::Tile;
    constexpr int NW = S::NW, ROWS = S::ROWS, NS = S::NS;
    constexpr int NB = KT / 32, KS = DP / 16, DB = DP / 32, KEYS = KG * KT;
    const uint32_t lds0 = lds_at(smem);
    const CoreArgs &a = f.a;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);   // uniform, so that what
                                                                 // depends on it is scalar
    const int kg = wave % KG, wr = wave / KG;

    // the arguments, read at once: the compiler loads each where it is first used, and each
    // first load is a trip to memory (read one by one, a workgroup's first loads of tiles were
    // issued 0.35 us later)
    asm volatile("" ::"s"(a.q.p), "s"(a.q.sb), "s"(a.q.sh), "s"(a.q.ld), "s"(a.dout.p),
                 "s"(a.dout.sb), "s"(a.dout.sh), "s"(a.dout.ld), "s"(a.k.p), "s"(a.k.sb),
                 "s"(a.k.sh), "s"(a.k.ld), "s"(a.v.p), "s"(a.v.sb), "s"(a.v.sh), "s"(a.v.ld),
                 "s"(a.len_q), "s"(a.len_k), "s"(a.batch), "s"(a.kv_heads), "s"(a.group),
                 "s"(a.sq), "s"(a.sk), "s"(a.d), "s"(a.causal), "s"(a.window), "s"(a.scale),
                 "s"(f.tiles_q), "s"(f.splits_q), "s"(f.rows));
    // heavier (later) causal tiles first within a (sequence, head)
    int bh, t;
    deal(wg, f.heads, f.per_q, &bh, &t);
    const int up = f.by_split(t), tile = f.tiles_q - 1 - up, split = f.by_split.rest(t, up);
    const int b = f.kv(bh), hk = f.kv.rest(bh, b);
    const SeqMask mask(a, b);

    const int row0 = tile * ROWS;
    const int row = row0 + wr * 32 + (lane & 31);
    const bool valid = row < f.rows;
    const int i = f.group(valid ? row : f.rows - 1);
    const int g = (valid ? row : f.rows - 1) - i * a.group;
    const int64_t head = (int64_t)hk * a.group + g;

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
    const int per_split = f.by_split(steps + f.splits_q - 1);
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
    auto arrive = [&](int stage) {
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

    const bool live = valid && i < mask.lq;
    const uint16_t *Q = static_cast<const uint16_t *>(a.q.p) + (int64_t)b * a.q.sb +
                        head * a.q.sh + (int64_t)i * a.q.ld;
    const uint16_t *G = static_cast<const uint16_t *>(a.dout.p) + (int64_t)b * a.dout.sb +
                        head * a.dout.sh + (int64_t)i * a.dout.ld;
    bf16x8 qf[KS], gf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        qf[ks] = row_frag<DMA>(Q, ks * 16 + 8 * half, live ? a.d : 0);
        gf[ks] = row_frag<DMA>(G, ks * 16 + 8 * half, live ? a.d : 0);
    }
    const int64_t stat = ((int64_t)b * a.kv_heads * a.group + head) * a.sq + i;
    const float c = a.scale * LOG2E;
    float l2 = live ? f.nl[stat] * c : -INFINITY, d0 = live ? f.nd[stat] : 0.f;
    asm volatile("" : "+v"(l2), "+v"(d0));
    settle(qf);
    settle(gf);
    const f32x16 d_init = splat16(d0);

    f32x16 o[DB];
#pragma unroll
    for (int x = 0; x < DB; ++x) o[x] = splat16(0.f);

    typename Tile::Reader rd(lds0 + kg * KT / Tile::RPS * Tile::SEG, lane);
    f32x16 sp[2], dpp[2];           // S and dP of this block and the next, in turn
    int stage = 0;                  // of the step at work
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
            f32x16 &s = sp[now], &dp = dpp[now], &s_n = sp[ONE - now], &dp_n = dpp[ONE - now];
            bf16x8 tk[2][DB], ds[2];
            s_n = splat16(0.f);
            dp_n = d_init;
            __builtin_amdgcn_sched_barrier(0);
            block_scores<KS, Tile::BYTES>(s_n, dp_n, nx, last ? 0 : (kb + 1) * 32, qf, gf, [&](int part) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    if (!in_part(r, part, KS + 1)) continue;
                    s[r] = exp2_(__builtin_fmaf(s[r], c, l2)) * dp[r];
                    if constexpr (EDGE) {
                        const int key = kw + kb * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
                        s[r] = key >= lo && key < hi ? s[r] : 0.f;
                    }
                    if (r % 8 == 7) ds[r / 8] = pack8(s, r - 7);
                }
                // the first 16 keys' columns
                if (part > KS - DB) tk[0][part - 1 - (KS - DB)] = rd.frag_t(part - 1 - (KS - DB), kb * 32, 0);
            });
            // the loads of a step, spread over its blocks: the last one's first
            constexpr int PER = (S::LOADS + NB - 1) / NB;
            const int first = last ? 0 : (kb + 1) * PER;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tk[h][db], ds[h], o[db], 0, 0, 0);
                    if (h == 0) tk[1][db] = rd.frag_t(db, kb * 32 + 16, 0);
                    const int k = h * DB + db;
#pragma unroll
                    for (int p = PER * k / (2 * DB); p < PER * (k + 1) / (2 * DB); ++p)
                        if (first + p < S::LOADS) fetch_part(first + p);
                    __builtin_amdgcn_sched_barrier(0);
                }
            if constexpr (!TURN) {
                sp[0] = sp[1];
                dpp[0] = dpp[1];
            }
        }
        rd.move(by);
        stage = wrap ? 0 : stage + 1;
    };
    if (s0 < s1) {
        if constexpr (DMA) wait_vm<(NS - 2) * S::LOADS>();
        __syncthreads();
        sp[0] = splat16(0.f);
        dpp[0] = d_init;
        block_scores<KS, Tile::BYTES>(sp[0], dpp[0], rd, 0, qf, gf, [](int) {});
    }
    int x = s0;
    for (; x < min(s1, walk.masked()); ++x) take(x, std::true_type{});
    for (; x < s1; ++x) take(x, std::false_type{});
    wait_vm<0>();      // no load is on its way to LDS any more
    __syncthreads();
    const bool whole = f.splits_q == 1;
    const int64_t d4 = (a.d + 3) & ~3;
    const RowsOut out{whole ? a.dq.p : f.part_q, whole ? a.d : (int)d4, !whole || a.dq_f32,
                      whole && a.dq_acc, !whole || f.vec_q};
    const int64_t off = !valid ? -1
                        : whole ? (int64_t)b * a.dq.sb + head * a.dq.sh + (int64_t)i * a.dq.ld
                                : (((int64_t)split * a.batch * a.kv_heads + bh) * f.rows + row) * d4;
    float *const put = reinterpret_cast<float *>(smem);
    // rows past the sequence's length or without keys: zero, though values that are not finite
    // may have reached their sums as 0 x infinity (as the factor of a row's results, instead of
    // the scale, 985 us of 16 heads over 4 of 8192 x 128, causal; in a branch of its own 979)
    const bool some = live && lo < hi;
    if (!__all(some)) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[db][r] = some ? o[db][r] : 0.f;
    }
    stage_rows<DP>(put + wave * PUT_FLOATS<DP>, o, whole ? a.scale : 1.f, lane);
    __syncthreads();
    store_rows<DP, KG>(put + wr * KG * PUT_FLOATS<DP>, PUT_FLOATS<DP>, kg, out, off, lane);
}

// ------------------------------------------------------------ dK and dV
// One dword per lane to byte `lds` of LDS (uniform) and on (lane l at + 4 l).
__device__ __forceinline__ void dma4_at(i32x4 r, uint32_t lds, int voff) {
    const uint32_t m0 = __builtin_amdgcn_readfirstlane(lds);
    asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                 :
                 : "s"(m0), "v"(voff), "s"(r)
                 : "memory", "m0");
}

template <int DP, int KG, int QT, bool DMA>
struct DkvShape {
    static constexpr int NW = 4;
    static constexpr int KEYS = 32 * NW / KG;
    static constexpr int QROWS = KG * QT;
    using Tile = RowTile<DP, QROWS, NW>;
    static constexpr int NST = QROWS;                        // floats of one statistic a stage
    // Q, dO, -lse / scale, -D, and room for a wave's load that brings nothing
    static constexpr int STAGE = 2 * Tile::BYTES + 256 * 4;
    static constexpr int LOADS = 2 * Tile::NV + 1;           // a thread's loads of a stage
    // workgroups of a unit: one where the sums of 32 keys take 128 registers a lane
    static constexpr int OCC = DP > 64 ? 1 : 2;
    // stages: a step reads its own and the next one while later ones arrive
    static constexpr int FIT = 163840 / OCC / STAGE;
    static constexpr int NS = !DMA ? 3 : FIT > 4 ? 4 : FIT;
    static constexpr int PUT = NW * 2 * PUT_FLOATS<DP> * 4;
    static constexpr int LDS = NS * STAGE > PUT ? NS * STAGE : PUT;
    static_assert(FIT >= NS && NS >= 3 && LDS <= 163840 / OCC, "three stages");
    static_assert(NST % 64 == 0 && 2 * NST <= 256, "one statistic per thread");
};

template <int DP, int KG, int QT, bool DMA>
__device__ __forceinline__ void attn_core_dkv(const BwdArgs &f, int wg, char *smem) {
    using S = DkvShape<DP, KG, QT, DMA>;
    using Tile = typename S::Tile;
    constexpr int NW = S::NW, KEYS = S::KEYS, QROWS = S::QROWS, NST = S::NST, NS = S::NS;
    constexpr int KS = DP / 16, DB = DP / 32;
    const uint32_t lds0 = lds_at(smem);
    const CoreArgs &a = f.a;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);   // uniform, so that what
                                                                 // depends on it is scalar
    const int kg = wave % KG, wk = wave / KG;

    // the arguments, read at once: the compiler loads each where it is first used, and each
    // first load is a trip to memory (read one by one, a workgroup's first loads of tiles were
    // issued 0.35 us later)
    asm volatile("" ::"s"(a.q.p), "s"(a.q.sb), "s"(a.q.sh), "s"(a.q.ld), "s"(a.dout.p),
                 "s"(a.dout.sb), "s"(a.dout.sh), "s"(a.dout.ld), "s"(a.k.p), "s"(a.k.sb),
                 "s"(a.k.sh), "s"(a.k.ld), "s"(a.v.p), "s"(a.v.sb), "s"(a.v.sh), "s"(a.v.ld),
                 "s"(a.len_q), "s"(a.len_k), "s"(a.batch), "s"(a.kv_heads), "s"(a.group),
                 "s"(a.sq), "s"(a.sk), "s"(a.d), "s"(a.causal), "s"(a.window), "s"(a.scale),
                 "s"(f.lev.items), "s"(f.lev.n));
    // keys with more rows (earlier causal tiles) first within a (sequence, head)
    int bh, t;
    deal(wg, f.heads, f.per_kv, &bh, &t);
    int lev = 0;
    while (lev + 1 < f.lev.n && t >= f.lev.item[lev + 1]) ++lev;
    const int splits = f.lev.v[lev], in_level = t - f.lev.item[lev];
    const int up = splits == 1 ? in_level : in_level / splits;
    const int tile = f.lev.tile[lev] + up, split = in_level - up * splits;
    const int b = f.kv(bh), hk = f.kv.rest(bh, b);
    const SeqMask mask(a, b);

    const int j0 = tile * KEYS;
    const int jw = j0 + wk * 32;
    const int key = jw + (lane & 31);
    const bool live = key < mask.lk;

    // rows [i_min, i_max) of a head see some key of the tile
    int i_min = 0, i_max = 0;
    if (j0 < mask.lk) {
        i_min = mask.causal ? max(0, j0 - mask.off) : 0;
        i_max = mask.lq;
        if (mask.window)
            i_max = min(i_max, min(j0 + KEYS, mask.lk) - 1 - mask.off + mask.window);
    }
    // of a head: first the steps with rows that do not see every key of the tile
    const int nq = i_max > i_min ? (i_max - i_min + QROWS - 1) / QROWS : 0;
    Walk walk{nq, 0, nq};
    if (nq > 0) {
        if (mask.causal)
            walk.na = min(nq, max(0, j0 + KEYS - 1 - mask.off - i_min + QROWS - 1) / QROWS);
        if (mask.window)
            walk.nb = max(walk.na, min(nq, max(0, j0 - mask.off + mask.window - i_min) / QROWS));
    }
    const int ne = walk.masked(), ni = nq - ne;   // masked steps of a head, and others
    const int steps = nq * a.group, edges = ne * a.group;
    const int per_split = splits == 1 ? steps : (steps + splits - 1) / splits;
    const int s0 = min(steps, split * per_split), s1 = min(steps, s0 + per_split);

    // this lane's key is seen by rows [lo, hi)
    const int lo = mask.causal ? key - mask.off : 0;
    const int hi = mask.window ? key - mask.off + mask.window : INT32_MAX;

    const uint16_t *Q = static_cast<const uint16_t *>(a.q.p) + (int64_t)b * a.q.sb;
    const uint16_t *G = static_cast<const uint16_t *>(a.dout.p) + (int64_t)b * a.dout.sb;
    const int place_q = Tile::place(a.q.ld, a.d, wave, lane);
    const int place_g = Tile::place(a.dout.ld, a.d, wave, lane);
    typename Tile::Regs rq, rg;
    float rs = 0.f;
    // a place in the walk: the y-th step of head h among the masked ones, or the others
    struct Place {
        int h, y;
    };
    auto next = [&](Place &c, int x) {   // from step x to x + 1
        const bool edge = x < edges;
        ++c.y;
        if (c.y == (edge ? ne : nq)) {
            c.h = x + 1 == edges ? 0 : c.h + 1;
            c.y = edge && x + 1 != edges ? 0 : ne;
        }
    };
    Place load{0, 0};
    if (s0 == 0) load = Place{0, edges > 0 ? 0 : ne};
    else if (s0 < edges) load = Place{s0 / ne, s0 % ne};
    else if (s0 < s1) load = Place{(s0 - edges) / ni, ne + (s0 - edges) % ni};
    Place work = load;
    // The loads of a step, S::LOADS of a thread: fetch(x, stage) takes the next step of the
    // walk, fetch_part(i) issues load i of it. Rows past the sequence's end and steps past the
    // walk's lie outside their buffers and arrive as zeros, also as statistics: P = 1 and
    // dS = 0 then meet rows of zeros. From step to step the sources only move on; they are
    // found anew where the head changes or the walk jumps.
    Fetch to{};
    i32x4 to_s{};
    const uint16_t *at_q = Q, *at_g = G;
    const float *at_s = f.nl;
    int i0 = 0;
    constexpr int W = NST / 64;   // waves that load a statistic, 64 floats each
    auto seek = [&]() {
        const int64_t h = (int64_t)hk * a.group + min(load.h, a.group - 1);
        i0 = i_min + walk.step(load.y) * QROWS;
        at_q = Q + h * a.q.sh + (int64_t)i0 * a.q.ld;
        at_g = G + h * a.dout.sh + (int64_t)i0 * a.dout.ld;
        at_s = (wave < W ? f.nl : f.nd) + ((int64_t)b * a.kv_heads * a.group + h) * a.sq + i0;
    };
    seek();
    auto fetch = [&](int x, int stage) __attribute__((always_inline)) {
        const int n = x < s1 ? min(QROWS, mask.lq - i0) : 0;
        if constexpr (DMA) {
            to.x = make_rsrc(at_q);
            to.y = make_rsrc(at_g);
            to_s = make_rsrc(at_s);
            to.x[2] = __builtin_amdgcn_readfirstlane(n * (int)a.q.ld * 2);
            to.y[2] = __builtin_amdgcn_readfirstlane(n * (int)a.dout.ld * 2);
            to_s[2] = __builtin_amdgcn_readfirstlane(wave < 2 * W ? n * 4 : 0);
            to.lds = lds0 + stage * S::STAGE;
        } else {
            Tile::load(rq, at_q, a.q.ld, n, a.d, tid);
            Tile::load(rg, at_g, a.dout.ld, n, a.d, tid);
            if (tid < 2 * NST) {
                const int y = tid % NST;
                const float *p = at_s + (tid < NST ? f.nl - (wave < W ? f.nl : f.nd)
                                                   : f.nd - (wave < W ? f.nl : f.nd));
                rs = y < n ? p[y] : 0.f;
            }
        }
        if (x + 1 >= s1) return;
        const Place was = load;
        next(load, x);
        if (load.h == was.h && walk.step(load.y) == walk.step(was.y) + 1) {
            i0 += QROWS;
            at_q += (int64_t)QROWS * a.q.ld;
            at_g += (int64_t)QROWS * a.dout.ld;
            at_s += QROWS;
        } else {
            seek();
        }
    };
    auto fetch_part = [&](int i) {
        if constexpr (DMA) {
            constexpr int NV = Tile::NV;
            if (i < NV) Tile::issue(to.x, a.q.ld, place_q, to.lds, wave, i);
            else if (i < 2 * NV)
                Tile::issue(to.y, a.dout.ld, place_g, to.lds + Tile::BYTES, wave, i - NV);
            else
                dma4_at(to_s, to.lds + 2 * Tile::BYTES + wave * 256, (wave % W) * 256 + lane * 4);
        }
    };
    auto arrive = [&](int stage) {
        if constexpr (!DMA) {
            char *lds = smem + stage * S::STAGE;
            Tile::store(rq, lds, tid);
            Tile::store(rg, lds + Tile::BYTES, tid);
            if (tid < 2 * NST) reinterpret_cast<float *>(lds + 2 * Tile::BYTES)[tid] = rs;
        }
    };
    if constexpr (DMA) {
#pragma unroll
        for (int x = 0; x < NS - 1; ++x) {
            fetch(s0 + x, x);
#pragma unroll
            for (int i = 0; i < S::LOADS; ++i) fetch_part(i);
        }
        fetch(s1, NS - 1);   // nothing, for the parts before the first advance
    } else if (s0 < s1) {
        fetch(s0, 0);
        arrive(0);
        if (s0 + 1 < s1) fetch(s0 + 1, 1);
    }

    const int64_t krow = min(key, a.sk - 1);
    const uint16_t *K = static_cast<const uint16_t *>(a.k.p) + (int64_t)b * a.k.sb +
                        (int64_t)hk * a.k.sh + krow * a.k.ld;
    const uint16_t *V = static_cast<const uint16_t *>(a.v.p) + (int64_t)b * a.v.sb +
                        (int64_t)hk * a.v.sh + krow * a.v.ld;
    bf16x8 kf[KS], vf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        kf[ks] = row_frag<DMA>(K, ks * 16 + 8 * half, live ? a.d : 0);
        vf[ks] = row_frag<DMA>(V, ks * 16 + 8 * half, live ? a.d : 0);
    }
    settle(kf);
    settle(vf);
    const float c = a.scale * LOG2E;

    f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int x = 0; x < DB; ++x) {
        dk[x] = splat16(0.f);
        dv[x] = splat16(0.f);
    }

    constexpr int NB = QT / 32;
    typename Tile::Reader rd(lds0 + kg * QT / Tile::RPS * Tile::SEG, lane);
    const uint32_t stat0 = lds0 + 2 * Tile::BYTES + (kg * QT + 4 * half) * 4;
    f32x16 sp[2], dpp[2];           // S and dP of this block and the next, in turn
    int stage = 0;                  // of the step at work
    // The statistics of the block at st: where S and dP start.
    auto start = [&](f32x16 &s, f32x16 &dp, uint32_t st, int r0) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f32x4 x = *(SBP_LDS const f32x4 *)(st + (r0 + 8 * q) * 4);
            const f32x4 y = *(SBP_LDS const f32x4 *)(st + (NST + r0 + 8 * q) * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[4 * q + e] = x[e];
                dp[4 * q + e] = y[e];
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
    auto take = [&](int x, auto edge) __attribute__((always_inline)) {
        constexpr bool EDGE = decltype(edge)::value;
        const int iw = i_min + walk.step(work.y) * QROWS + kg * QT;
        next(work, x);
        const bool wrap = stage == NS - 1;
        const int by = wrap ? -(NS - 1) * S::STAGE : S::STAGE;
        const uint32_t stat = stat0 + stage * S::STAGE;
#pragma unroll
        for (int qb = 0; qb < NB; ++qb) {
            const bool last = qb == NB - 1;
            const int r0 = qb * 32, i0 = iw + qb * 32, n0 = last ? 0 : r0 + 32;
            if (last) advance(x);
            typename Tile::Reader nx = rd;       // where the next block lies
            if (last) nx.move(by);
            // with an even number of blocks a step the two take turns in place
            constexpr bool TURN = NB % 2 == 0;
            constexpr int ONE = 1;
            const int now = TURN ? qb & 1 : 0;
            f32x16 &s = sp[now], &dp = dpp[now], &s_n = sp[ONE - now], &dp_n = dpp[ONE - now];
            bf16x8 tg[2][DB], tq[2][DB], p[2], ds[2];
            __builtin_amdgcn_sched_barrier(0);
            start(s_n, dp_n, last ? stat + by : stat, n0);
            block_scores<KS, Tile::BYTES>(s_n, dp_n, nx, n0, kf, vf, [&](int part) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    if (!in_part(r, part, KS + 1)) continue;
                    s[r] = exp2_(s[r] * c);
                    dp[r] *= s[r];
                    if constexpr (EDGE) {
                        const int i = i0 + 8 * (r >> 2) + 4 * half + (r & 3);
                        const bool seen = i >= lo && i < hi;
                        s[r] = seen ? s[r] : 0.f;
                        dp[r] = seen ? dp[r] : 0.f;
                    }
                    if (r % 8 == 7) {
                        p[r / 8] = pack8(s, r - 7);
                        ds[r / 8] = pack8(dp, r - 7);
                    }
                }
                // the first 16 rows' columns
                if (part > KS - DB) {
                    const int db = part - 1 - (KS - DB);
                    tg[0][db] = rd.frag_t(db, r0, Tile::BYTES);
                    tq[0][db] = rd.frag_t(db, r0, 0);
                }
            });
            // the loads of a step, spread over its blocks: the last one's first
            constexpr int PER = (S::LOADS + NB - 1) / NB;
            const int first = last ? 0 : (qb + 1) * PER;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    dv[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tg[h][db], p[h], dv[db], 0, 0, 0);
                    dk[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tq[h][db], ds[h], dk[db], 0, 0, 0);
                    if (h == 0) {
                        tg[1][db] = rd.frag_t(db, r0 + 16, Tile::BYTES);
                        tq[1][db] = rd.frag_t(db, r0 + 16, 0);
                    }
                    const int k = h * DB + db;
#pragma unroll
                    for (int i = PER * k / (2 * DB); i < PER * (k + 1) / (2 * DB); ++i)
                        if (first + i < S::LOADS) fetch_part(first + i);
                    __builtin_amdgcn_sched_barrier(0);
                }
            if constexpr (!TURN) {
                sp[0] = sp[1];
                dpp[0] = dpp[1];
            }
        }
        rd.move(by);
        stage = wrap ? 0 : stage + 1;
    };
    if (s0 < s1) {
        if constexpr (DMA) wait_vm<(NS - 2) * S::LOADS>();
        __syncthreads();
        start(sp[0], dpp[0], stat0, 0);
        block_scores<KS, Tile::BYTES>(sp[0], dpp[0], rd, 0, kf, vf, [](int) {});
    }
    int x = s0;
    for (; x < min(s1, edges); ++x) take(x, std::true_type{});
    for (; x < s1; ++x) take(x, std::false_type{});
    wait_vm<0>();      // no load is on its way to LDS any more
    __syncthreads();
    // keys past the sequence's length get zeros (their lanes hold no sums of use). Partials:
    // the tile's KEYS rows of dK and dV of this (sequence, key head)
    const bool whole = splits == 1;
    const int64_t d4 = (a.d + 3) & ~3;
    const int64_t slot = (int64_t)(f.lev.slot[lev] + in_level) * a.batch * a.kv_heads + bh;
    const RowsOut out_k{whole ? a.dk.p : f.part_kv, whole ? a.d : (int)d4, !whole || a.dk_f32,
                        whole && a.dk_acc, !whole || f.vec_k};
    const RowsOut out_v{whole ? a.dv.p : f.part_kv + d4, whole ? a.d : (int)d4,
                        !whole || a.dv_f32, whole && a.dv_acc, !whole || f.vec_v};
    int64_t off_k = -1, off_v = -1;
    if (key < a.sk) {
        off_k = off_v = (slot * KEYS + wk * 32 + (lane & 31)) * 2 * d4;
        if (whole) {
            off_k = (int64_t)b * a.dk.sb + (int64_t)hk * a.dk.sh + (int64_t)key * a.dk.ld;
            off_v = (int64_t)b * a.dv.sb + (int64_t)hk * a.dv.sh + (int64_t)key * a.dv.ld;
        }
    }
    constexpr int PUT = PUT_FLOATS<DP>;
    float *const put = reinterpret_cast<float *>(smem);
    stage_rows<DP>(put + wave * 2 * PUT, dk, !live ? 0.f : whole ? a.scale : 1.f, lane);
    stage_rows<DP>(put + wave * 2 * PUT + PUT, dv, live ? 1.f : 0.f, lane);
    __syncthreads();
    store_rows<DP, KG>(put + wk * KG * 2 * PUT, 2 * PUT, kg, out_k, off_k, lane);
    store_rows<DP, KG>(put + wk * KG * 2 * PUT + PUT, 2 * PUT, kg, out_v, off_v, lane);
}

// Keys of a tile of dK and dV and rows of a step of its walk, which two wave groups share;
// KG groups share a step of dQ's.
constexpr int DKV_KG = 2, DKV_KEYS = 128 / DKV_KG, DKV_ROWS = 64;
template <int DP, int KG, bool DMA>
struct BwdShape {
    static constexpr int KT = 64 / KG;
    using Dq = DqShape<DP, KG, KT, DMA>;
    using Dkv = DkvShape<DP, DKV_KG, DKV_ROWS / DKV_KG, DMA>;
    static constexpr int LDS = Dq::LDS > Dkv::LDS ? Dq::LDS : Dkv::LDS;
    static constexpr int OCC = Dq::OCC;
    static_assert(Dq::OCC == Dkv::OCC && Dkv::KEYS == DKV_KEYS && Dkv::QROWS == DKV_ROWS, "");
};

template <int DP, int KG, bool DMA>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(BwdShape<DP, KG, DMA>::OCC, BwdShape<DP, KG, DMA>::OCC)))
void attn_core_bwd_kernel(BwdArgs f) {
    using S = BwdShape<DP, KG, DMA>;
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS];
    const int wg = blockIdx.x;
    if (wg < f.items_kv) attn_core_dkv<DP, DKV_KG, DKV_ROWS / DKV_KG, DMA>(f, wg, smem);
    else attn_core_dq<DP, KG, S::KT, DMA>(f, wg - f.items_kv, smem);
}

// Adds the splits' partials in split order. A thread owns 4 columns of a row of dQ, or of
// dK and dV (of the tiles that are split), 16 (32 past 64 columns) a row; the workgroups of
// dQ come first.
__global__ __launch_bounds__(256) void attn_core_sum_kernel(BwdArgs f, int blocks_q) {
    const CoreArgs &a = f.a;
    const bool kv = (int)blockIdx.x >= blocks_q;
    const int lanes = a.d > 64 ? 5 : 4;
    const Div &per = kv ? f.by_keys : f.by_rows;
    const int64_t d4 = (a.d + 3) & ~3, bhs = (int64_t)a.batch * a.kv_heads, n = bhs * per.d;
    const uint32_t id = (blockIdx.x - (kv ? blocks_q : 0)) * 256u + threadIdx.x;
    const int at = (int)(id >> lanes), col = (int)(id & ((1u << lanes) - 1)) * 4;
    if (at >= n || col >= a.d) return;
    const int bh = per(at), row = per.rest(at, bh);
    const int b = f.kv(bh), hk = f.kv.rest(bh, b);
    if (kv) {
        const int tile = row / DKV_KEYS;
        int lev = 0;
        while (lev + 1 < f.lev.n && tile >= f.lev.tile[lev + 1]) ++lev;
        const int v = f.lev.v[lev];
        const int64_t slot = f.lev.slot[lev] + (int64_t)(tile - f.lev.tile[lev]) * v;
        const float *p = f.part_kv + ((slot * bhs + bh) * DKV_KEYS + row % DKV_KEYS) * 2 * d4 + col;
        const int64_t step = bhs * DKV_KEYS * 2 * d4;
        f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
        for (int s = 0; s < v; ++s, p += step) {
            x += *reinterpret_cast<const f32x4 *>(p);
            y += *reinterpret_cast<const f32x4 *>(p + d4);
        }
        grad4(a.dk.p, (int64_t)b * a.dk.sb + (int64_t)hk * a.dk.sh + (int64_t)row * a.dk.ld, col,
              a.d, a.dk_f32, a.dk_acc, f.vec_k, [&](int e) { return x[e] * a.scale; });
        grad4(a.dv.p, (int64_t)b * a.dv.sb + (int64_t)hk * a.dv.sh + (int64_t)row * a.dv.ld, col,
              a.d, a.dv_f32, a.dv_acc, f.vec_v, [&](int e) { return y[e]; });
    } else {
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < f.splits_q; ++s)
            x += *reinterpret_cast<const f32x4 *>(f.part_q + ((int64_t)s * n + at) * d4 + col);
        const int i = f.group(row);
        const int64_t head = (int64_t)hk * a.group + (row - i * a.group);
        grad4(a.dq.p, (int64_t)b * a.dq.sb + head * a.dq.sh + (int64_t)i * a.dq.ld, col, a.d,
              a.dq_f32, a.dq_acc, f.vec_q, [&](int e) { return x[e] * a.scale; });
    }
}

}  // namespace sbpk

namespace sbpi {

namespace {

template <int DP, int KG>
hipError_t launch_bwd(const sbpk::BwdArgs &f, int64_t blocks, hipStream_t s) {
    char name[160];
    name[0] = 0;
    if (profiling())
        snprintf(name, sizeof(name), "attn_core_bwd_kernel<%d,%d,%d>", DP, KG, (int)f.a.aligned);
    if (f.a.aligned)
        return launch_kernel(sbpk::attn_core_bwd_kernel<DP, KG, true>, name,
                             dim3((unsigned)blocks), dim3(256), s, f);
    return launch_kernel(sbpk::attn_core_bwd_kernel<DP, KG, false>, name, dim3((unsigned)blocks),
                         dim3(256), s, f);
}

bool vec4(const CoreView &v, int d, bool f32) {
    return d % 4 == 0 && reinterpret_cast<uintptr_t>(v.p) % (f32 ? 16 : 8) == 0 &&
           v.ld % 4 == 0 && v.sb % 4 == 0 && v.sh % 4 == 0;
}

// Steps of key tile t's walk, every row and key in use.
int64_t kv_steps(const CoreArgs &a, int64_t t) {
    const int64_t off = (int64_t)a.sk - a.sq, j0 = t * sbpk::DKV_KEYS;
    int64_t n = a.sq;
    if (a.causal && a.window) n = std::min<int64_t>(n, sbpk::DKV_KEYS + a.window);
    else if (a.causal) n -= std::min<int64_t>(n, std::max<int64_t>(0, j0 - off));
    return (n + sbpk::DKV_ROWS - 1) / sbpk::DKV_ROWS * a.group;
}

// One way to split a walk: its longest item and all items, in steps, and the partials.
struct Way {
    int64_t longest, items;
    double steps, part;       // of one (sequence, key head): steps, floats of partials
};

// dK and dV with the longest walk in v parts: walks of more steps than those parts are split
// too; they get no longer from tile to tile.
Way split_kv(const CoreArgs &a, int64_t v, sbpk::Levels *lev) {
    const int64_t tiles = ((int64_t)a.sk + sbpk::DKV_KEYS - 1) / sbpk::DKV_KEYS;
    const int64_t target = std::max<int64_t>(1, (kv_steps(a, 0) + v - 1) / v);
    *lev = sbpk::Levels{};
    int64_t partials = 0, items = 0, at = 0;
    double total = 0;
    for (int64_t w = v; w >= 1 && at < tiles; --w) {
        int64_t lo = at, hi = tiles;   // the end of the tiles of w parts or more
        while (w > 1 && lo < hi) {
            const int64_t mid = (lo + hi) / 2;
            if (kv_steps(a, mid) > (w - 1) * target) lo = mid + 1;
            else hi = mid;
        }
        if (w == 1) lo = tiles;
        if (lo == at) continue;
        const int j = lev->n++;
        lev->tile[j] = (int32_t)at;
        lev->v[j] = (int32_t)w;
        lev->item[j] = (int32_t)items;
        lev->slot[j] = (int32_t)partials;
        items += (lo - at) * w;
        if (w > 1) {
            partials += (lo - at) * w;
            lev->split_keys = (int32_t)std::min<int64_t>(a.sk, lo * sbpk::DKV_KEYS);
        }
        total += (lo - at) * 0.5 * (double)(kv_steps(a, at) + kv_steps(a, lo - 1));
        at = lo;
    }
    lev->tile[lev->n] = (int32_t)tiles;
    lev->items = (int32_t)items;
    return Way{target, items, total, (double)partials * sbpk::DKV_KEYS * 2 * ((a.d + 3) & ~3)};
}

// dQ with tiles of `rows` rows, every walk in v parts.
Way split_q(const CoreArgs &a, int64_t rows, int64_t v) {
    const int64_t packed = (int64_t)a.sq * a.group, tiles = (packed + rows - 1) / rows;
    const int64_t keys = a.causal && a.window ? std::min<int64_t>(a.sk, a.window + rows / a.group)
                                              : a.sk;
    const int64_t steps = (keys + 63) / 64;
    // a causal walk is half as long on average where it starts at nothing
    const double mean = a.causal && !a.window
                            ? steps * (1.0 - 0.5 * std::min<double>(1.0, (double)a.sq / a.sk))
                            : (double)steps;
    return Way{(steps + v - 1) / v, tiles * v, mean * tiles,
               v > 1 ? (double)packed * v * ((a.d + 3) & ~3) : 0.0};
}

// Wave groups of dQ (returned) and the splits: those that the following time expects least
// of. An item takes so much a step, and `fixed` besides; the busiest unit has an even share
// of all items and a fifth of the longest; partials are written and read once, by one more
// launch. (In a graph, 16 heads over 4 of 8192 x 128, causal: 1023 us whole, with dK's and dV's
// longest walk in two parts and in three, 1075 whole with dQ in two groups; 16 heads of 1024
// x 64, causal: 25 whole with dQ in two groups, 30 in one, 34 with the longest walk in two
// parts; 4 heads of 1024 rows and 4096 keys of 64: 30 split, 46 whole.)
int plan_bwd(const CoreArgs &a, int64_t bhs, int cus, size_t room, sbpk::BwdArgs *f) {
    const bool wide = a.d > 64;
    const double slots = cus * (wide ? 1.0 : 2.0), fixed = 4.0;
    const double step_kv = wide ? 0.95 : 0.75, step_q = wide ? 0.75 : 0.6;
    constexpr int MOST = sbpk::MAX_LEVELS;
    sbpk::Levels lev[MOST];
    Way kv[MOST];
    int n = 0;
    for (; n < MOST && (n == 0 || n < kv_steps(a, 0) / 2); ++n) kv[n] = split_kv(a, n + 1, &lev[n]);
    double best = 1e300;
    int best_kg = 1, best_n = 0;     // whole walks need no room
    f->splits_q = 1;
    for (int kg = 1; kg <= 2; ++kg) {
        for (int v = 1; v <= MOST; v *= 2) {
            const Way q = split_q(a, 128 / kg, v);
            if (v > 1 && q.longest < 2) break;
            // 128 rows in one group take longer a step, by less than twice
            const double sq = step_q * (kg == 1 ? 1.7 : 1.0);
            for (int i = 0; i < n; ++i) {
                const double part = (kv[i].part + q.part) * bhs;
                // (the sums' threads, 32 a row, fit 32 bits)
                if (part > 0 && (part > (double)room ||
                                 (double)bhs * (f->rows + a.sk) > 134217727.0 ||
                                 (double)(kv[i].items + q.items) * bhs > 16777215.0))
                    continue;
                const double item = fixed + std::max(kv[i].longest * step_kv, q.longest * sq);
                const double all = (kv[i].steps * step_kv + q.steps * sq +
                                    (kv[i].items + q.items) * fixed) * bhs / slots;
                const double t = std::max(item, all + 0.2 * item) +
                                 (part > 0 ? 4.0 + part * 8 / 4e6 : 0.0);
                if (t < best * 0.98) {
                    best = t;
                    best_kg = kg;
                    best_n = i;
                    f->splits_q = v;
                }
            }
        }
    }
    f->lev = lev[best_n];
    f->items_kv = (int32_t)(bhs * f->lev.items);
    f->per_kv = sbpk::Div(f->lev.items);
    f->heads = sbpk::Div(bhs);
    f->kv = sbpk::Div(a.kv_heads);
    f->group = sbpk::Div(a.group);
    f->by_split = sbpk::Div(f->splits_q);
    f->by_rows = sbpk::Div(f->rows);
    f->by_keys = sbpk::Div(f->lev.split_keys);
    f->tiles_q = (f->rows * best_kg + 127) / 128;
    f->per_q = sbpk::Div((int64_t)f->tiles_q * f->splits_q);
    return best_kg;
}

}  // namespace

hipError_t launch_core_bwd(const CoreArgs &a, hipStream_t s) {
    sbpk::BwdArgs f;
    f.a = a;
    f.rows = a.sq * a.group;
    f.vec_q = vec4(a.dq, a.d, a.dq_f32);
    f.vec_k = vec4(a.dk, a.d, a.dk_f32);
    f.vec_v = vec4(a.dv, a.d, a.dv_f32);
    const int64_t bhs = (int64_t)a.batch * a.kv_heads;
    const int64_t qrows = bhs * f.rows;
    const size_t stat = core_bwd_stat_floats(a);
    float *const nl = a.ws, *const nd = a.ws + stat / 2;
    f.nl = nl;
    f.nd = nd;
    const int64_t d4 = (a.d + 3) & ~3;
    hipError_t e;
    if (qrows > 0) {
        e = launch_kernel(sbpk::attn_core_stat_kernel, "attn_core_stat_kernel",
                          dim3((unsigned)((qrows + 15) / 16)), dim3(256), s, a, sbpk::Div(a.sq),
                          sbpk::Div((int64_t)a.kv_heads * a.group), nl, nd);
        if (e != hipSuccess) return e;
    }
    const int kg = plan_bwd(a, bhs, device_cus(), a.ws_floats - stat, &f);
    f.part_q = a.ws + stat;
    f.part_kv = f.part_q + (f.splits_q > 1 ? qrows * f.splits_q * d4 : 0);
    const int64_t blocks = f.items_kv + bhs * f.tiles_q * f.splits_q;
    if (blocks == 0) return hipSuccess;
    if (kg == 1) e = a.d > 64 ? launch_bwd<128, 1>(f, blocks, s) : launch_bwd<64, 1>(f, blocks, s);
    else e = a.d > 64 ? launch_bwd<128, 2>(f, blocks, s) : launch_bwd<64, 2>(f, blocks, s);
    if (e != hipSuccess) return e;
    const int64_t lanes = a.d > 64 ? 32 : 16;
    const int64_t sum_q = f.splits_q > 1 ? (qrows * lanes + 255) / 256 : 0;
    const int64_t sum_kv = (bhs * f.lev.split_keys * lanes + 255) / 256;
    if (sum_q + sum_kv == 0) return hipSuccess;
    return launch_kernel(sbpk::attn_core_sum_kernel, "attn_core_sum_kernel",
                         dim3((unsigned)(sum_q + sum_kv)), dim3(256), s, f, (int)sum_q);
}

}  // namespace sbpi
