// attn_core_bwd.hip -- softmax attention, backward: the probabilities are
// recomputed from Q, K and the forward pass's row statistics,
//   P = exp(scale Q K^T - lse),  dV = P^T dO,  dS = P (dO V^T - D),
//   dQ = scale dS K,  dK = scale dS^T Q,  D_i = sum_c dO_ic O_ic.
//
// Three launches, none with atomics, so the results do not depend on the order
// in which workgroups run:
//   * row statistics: -lse / scale and D of every query row go to the workspace;
//   * dQ: a workgroup owns query rows (packed over the query heads that share a
//     key head, as in the forward kernel) and walks over their keys;
//   * dK and dV: a workgroup owns keys and walks over the rows that see them, of
//     every query head that shares the key head.
// Scores and dO V^T are thus computed twice, seven products where five are needed;
// the alternative, one pass that adds dQ in memory, needs fp32 atomics (in
// an order that changes the result) or a partial dQ for every key tile.
//
// The statistics are the products' initial accumulators: starting S = Q K^T at
// -lse / scale and dO V^T at -D leaves one multiplication, one exponential and one
// product a score. P and dS are rounded to bf16 for the products that read them;
// every sum is fp32.
#include <math.h>

#include "attn_core_kernel.h"
#include "gemm.h"
#include "profile.h"

namespace sbpk {

struct BwdArgs {
    CoreArgs a;
    int32_t tiles_q, splits_q, rows;   // dQ: row tiles, key splits; rows = sq * group
    int32_t tiles_k, splits_k;         // dK, dV: key tiles, row splits
    int32_t vec_q, vec_k, vec_v;       // outputs allow 4-value stores
    const float *nl, *nd;              // row statistics: -lse / scale, -D, per (b, head, i)
    float *part;                       // split partials
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
__global__ __launch_bounds__(256) void attn_core_stat_kernel(CoreArgs a, float *nl, float *nd) {
    const int64_t heads = (int64_t)a.kv_heads * a.group;
    const int64_t n = a.batch * heads * a.sq;
    const int64_t r = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    const int at = (threadIdx.x & 15) * 8;
    if (r >= n) return;
    const int i = (int)(r % a.sq);
    const int64_t bh = r / a.sq, b = bh / heads, h = bh % heads;
    const int lq = a.len_q ? min(max(a.len_q[b], 0), a.sq) : a.sq;
    const float lse = i < lq ? static_cast<const float *>(a.lse.p)[b * a.lse.sb + h * a.lse.sh +
                                                                   i * a.lse.ld]
                             : -INFINITY;
    const bool live = lse != -INFINITY;
    float x = 0.f;
    if (live && at < a.d) {
        const bf16x8 g = row_frag(static_cast<const uint16_t *>(a.dout.p) + b * a.dout.sb +
                                      h * a.dout.sh + i * a.dout.ld,
                                  at, a.d, false);
        const int64_t o = b * a.o.sb + h * a.o.sh + i * a.o.ld;
        if (a.o_f32) {
            const float *p = static_cast<const float *>(a.o.p) + o;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (at + e < a.d) x += (float)g[e] * p[at + e];
        } else {
            const bf16x8 y = row_frag(static_cast<const uint16_t *>(a.o.p) + o, at, a.d, false);
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
template <int DP, int KG, int KT>
struct DqShape {
    static constexpr int NW = 4;
    static constexpr int ROWS = 32 * NW / KG;
    using Tile = RowTile<DP, KG * KT, NW>;
    static constexpr int STAGE = 2 * Tile::BYTES;
    static constexpr int LDS = 2 * STAGE;
    static constexpr int OCC = LDS > 81920 ? 1 : 2;
};

template <int DP, int KG, int KT, bool DMA>
__global__ __launch_bounds__(256, (DqShape<DP, KG, KT>::OCC))
void attn_core_dq_kernel(BwdArgs f) {
    using S = DqShape<DP, KG, KT>;
    using Tile = typename S::Tile;
    constexpr int NW = S::NW, ROWS = S::ROWS, KB = KT / 32, KS = DP / 16, DB = DP / 32;
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS];
    const CoreArgs &a = f.a;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);   // uniform, so that what
                                                                 // depends on it is scalar
    const int kg = wave % KG, wr = wave / KG;

    const int per = f.tiles_q * f.splits_q;
    const int L = remap_xcd(blockIdx.x, gridDim.x);
    const int bh = L / per, t = L % per;
    const int tile = f.tiles_q - 1 - t / f.splits_q, split = t % f.splits_q;
    const int b = bh / a.kv_heads, hk = bh % a.kv_heads;
    const SeqMask mask(a, b);

    const int row0 = tile * ROWS;
    const int row = row0 + wr * 32 + (lane & 31);
    const bool valid = row < f.rows;
    const int i = (valid ? row : f.rows - 1) / a.group;
    const int g = (valid ? row : f.rows - 1) - i * a.group;
    const int64_t head = (int64_t)hk * a.group + g;

    const int i_first = row0 / a.group;
    const int i_last = (min(row0 + ROWS, f.rows) - 1) / a.group;
    const int k_beg = mask.lo(i_first) & ~31;
    const int k_end = i_first < mask.lq ? mask.hi(min(i_last, mask.lq - 1)) : 0;
    const int steps = k_end > k_beg ? (k_end - k_beg + KG * KT - 1) / (KG * KT) : 0;
    // steps whose keys every row of the tile sees (rows past the sequence's end aside)
    Walk walk{steps, 0, steps};
    if (steps > 0) {
        const int all = min(mask.hi(i_first), mask.lk);
        walk.nb = all > k_beg ? min(steps, (all - k_beg) / (KG * KT)) : 0;
        walk.na = min(walk.nb, (mask.lo(i_last) - k_beg + KG * KT - 1) / (KG * KT));
        walk.na = max(walk.na, 0);
    }
    const int per_split = (steps + f.splits_q - 1) / f.splits_q;
    const int s0 = min(steps, split * per_split), s1 = min(steps, s0 + per_split);
    const int hi = mask.hi(i), lo = mask.lo(i);

    const uint16_t *K = static_cast<const uint16_t *>(a.k.p) + (int64_t)b * a.k.sb +
                        (int64_t)hk * a.k.sh;
    const uint16_t *V = static_cast<const uint16_t *>(a.v.p) + (int64_t)b * a.v.sb +
                        (int64_t)hk * a.v.sh;
    const int place_k = Tile::place(a.k.ld, a.d, wave, lane);
    const int place_v = Tile::place(a.v.ld, a.d, wave, lane);
    typename Tile::Regs rk, rv;
    auto issue = [&](int x, int stage) {
        const int k0 = k_beg + walk.step(x) * (KG * KT);
        const int n = min(KG * KT, mask.lk - k0);
        char *lds = smem + stage * S::STAGE;
        if constexpr (DMA) {
            Tile::issue(K + (int64_t)k0 * a.k.ld, a.k.ld, n, place_k, lds, wave);
            Tile::issue(V + (int64_t)k0 * a.v.ld, a.v.ld, n, place_v, lds + Tile::BYTES, wave);
        } else {
            Tile::load(rk, K + (int64_t)k0 * a.k.ld, a.k.ld, n, a.d, tid);
            Tile::load(rv, V + (int64_t)k0 * a.v.ld, a.v.ld, n, a.d, tid);
        }
    };
    auto arrive = [&](int stage) {
        if constexpr (!DMA) {
            char *lds = smem + stage * S::STAGE;
            Tile::store(rk, lds, tid);
            Tile::store(rv, lds + Tile::BYTES, tid);
        }
    };
    if (s0 < s1) {
        issue(s0, 0);
        arrive(0);
    }

    const bool live = valid && i < mask.lq;
    const uint16_t *Q = static_cast<const uint16_t *>(a.q.p) + (int64_t)b * a.q.sb +
                        head * a.q.sh + (int64_t)i * a.q.ld;
    const uint16_t *G = static_cast<const uint16_t *>(a.dout.p) + (int64_t)b * a.dout.sb +
                        head * a.dout.sh + (int64_t)i * a.dout.ld;
    bf16x8 qf[KS], gf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        qf[ks] = row_frag(Q, ks * 16 + 8 * half, live ? a.d : 0, DMA);
        gf[ks] = row_frag(G, ks * 16 + 8 * half, live ? a.d : 0, DMA);
    }
    const int64_t stat = ((int64_t)b * a.kv_heads * a.group + head) * a.sq + i;
    const float c = a.scale * LOG2E;
    const float l2 = live ? f.nl[stat] * c : -INFINITY;
    const f32x16 d_init = splat16(live ? f.nd[stat] : 0.f);

    f32x16 o[DB];
#pragma unroll
    for (int x = 0; x < DB; ++x) o[x] = splat16(0.f);

    // a step's keys; EDGE: some row of the wave does not see all of them
    typename Tile::Reader rd(lds_at(smem) + kg * KT / Tile::RPS * Tile::SEG, lane);
    auto step = [&](int kw, auto edge) {
        constexpr bool EDGE = decltype(edge)::value;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            f32x16 s = splat16(0.f), dp = d_init;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    rd.frag(kb * 32, ks, 0), qf[ks], s, 0, 0, 0);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    rd.frag(kb * 32, ks, Tile::BYTES), gf[ks], dp, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[r] = exp2_(__builtin_fmaf(s[r], c, l2)) * dp[r];
                if constexpr (EDGE) {
                    const int key = kw + kb * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
                    s[r] = key >= lo && key < hi ? s[r] : 0.f;
                }
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const bf16x8 p = pack8(s, 8 * x);
#pragma unroll
                for (int db = 0; db < DB; ++db)
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        rd.frag_t(db, kb * 32 + 16 * x, 0), p, o[db], 0, 0, 0);
            }
        }
    };
    auto take = [&](int x, auto edge) {
        const int stage = (x - s0) & 1;
        wait_vm<0>();
        __syncthreads();
        if (x + 1 < s1) issue(x + 1, stage ^ 1);
        step(k_beg + walk.step(x) * (KG * KT) + kg * KT, edge);
        rd.move(stage ? -S::STAGE : S::STAGE);
        if (x + 1 < s1) arrive(stage ^ 1);
    };
    int x = s0;
    for (; x < min(s1, walk.masked()); ++x) take(x, std::true_type{});
    for (; x < s1; ++x) take(x, std::false_type{});

    if constexpr (KG > 1) {
        __syncthreads();
        constexpr int SLOT = DB * 16 * 64;
        static_assert((KG - 1) * (NW / KG) * SLOT * 4 <= S::LDS, "group results do not fit");
        float *const base = reinterpret_cast<float *>(smem) + lane;
        if (kg > 0) {
            float *p = base + ((kg - 1) * (NW / KG) + wr) * SLOT;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) p[(db * 16 + r) * 64] = o[db][r];
        }
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int k = 1; k < KG; ++k) {
            const float *p = base + ((k - 1) * (NW / KG) + wr) * SLOT;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[db][r] += p[(db * 16 + r) * 64];
        }
    }
    if (!valid) return;
    const int64_t d4 = (a.d + 3) & ~3;
    const int64_t at = (int64_t)b * a.dq.sb + head * a.dq.sh + (int64_t)i * a.dq.ld;
    float *const part =
        f.part + (((int64_t)split * a.batch * a.kv_heads + bh) * f.rows + row) * d4;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int col = db * 32 + 8 * q + 4 * half;
            if (col >= a.d) continue;
            if (f.splits_q > 1) {
                f32x4 v = {o[db][4 * q], o[db][4 * q + 1], o[db][4 * q + 2], o[db][4 * q + 3]};
                *reinterpret_cast<f32x4 *>(part + col) = v;
            } else {
                grad4(a.dq.p, at, col, a.d, a.dq_f32, a.dq_acc, f.vec_q,
                      [&](int e) { return o[db][4 * q + e] * a.scale; });
            }
        }
}

// ------------------------------------------------------------ dK and dV
// One dword per lane into LDS (lane l at lds + 4 l).
__device__ __forceinline__ void dma4(i32x4 r, char *lds, int voff) {
    const uint32_t m0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(SBP_LDS void *)lds);
    asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                 :
                 : "s"(m0), "v"(voff), "s"(r)
                 : "memory", "m0");
}

template <int DP, int KG, int QT>
struct DkvShape {
    static constexpr int NW = 4;
    static constexpr int KEYS = 32 * NW / KG;
    static constexpr int QROWS = KG * QT;
    using Tile = RowTile<DP, QROWS, NW>;
    static constexpr int NST = QROWS < 64 ? 64 : QROWS;      // floats of one statistic a stage
    static constexpr int STAGE = 2 * Tile::BYTES + 2 * NST * 4;
    static constexpr int LDS = 2 * STAGE;
    static constexpr int OCC = LDS > 81920 || DP > 64 ? 1 : 2;
};

template <int DP, int KG, int QT, bool DMA>
__global__ __launch_bounds__(256, (DkvShape<DP, KG, QT>::OCC))
void attn_core_dkv_kernel(BwdArgs f) {
    using S = DkvShape<DP, KG, QT>;
    using Tile = typename S::Tile;
    constexpr int NW = S::NW, KEYS = S::KEYS, QROWS = S::QROWS, NST = S::NST;
    constexpr int KS = DP / 16, DB = DP / 32;
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS];
    const CoreArgs &a = f.a;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);   // uniform, so that what
                                                                 // depends on it is scalar
    const int kg = wave % KG, wk = wave / KG;

    // keys with more rows (earlier causal tiles) first within a (sequence, head)
    const int per = f.tiles_k * f.splits_k;
    const int L = remap_xcd(blockIdx.x, gridDim.x);
    const int bh = L / per, t = L % per;
    const int tile = t / f.splits_k, split = t % f.splits_k;
    const int b = bh / a.kv_heads, hk = bh % a.kv_heads;
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
    const int per_split = (steps + f.splits_k - 1) / f.splits_k;
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
    // the next step to load: the iy-th of head ih among the masked ones, or the others
    int ih = 0, iy = 0;
    if (s0 < edges) {
        ih = s0 / ne;
        iy = s0 % ne;
    } else if (s0 < s1) {
        ih = (s0 - edges) / ni;
        iy = ne + (s0 - edges) % ni;
    }
    int ii = i_min + walk.step(iy) * QROWS;
    auto issue = [&](int x, int stage) {   // step x, the next one
        const int64_t h = (int64_t)hk * a.group + ih;
        const int i0 = ii;
        ++iy;
        if (iy == (x < edges ? ne : nq)) {
            ++ih;
            iy = x < edges ? 0 : ne;
            if (x + 1 == edges) {
                ih = 0;
                iy = ne;
            }
        }
        ii = i_min + walk.step(iy) * QROWS;
        const int n = min(QROWS, mask.lq - i0);
        const uint16_t *q = Q + h * a.q.sh + (int64_t)i0 * a.q.ld;
        const uint16_t *g = G + h * a.dout.sh + (int64_t)i0 * a.dout.ld;
        const int64_t row = ((int64_t)b * a.kv_heads * a.group + h) * a.sq + i0;
        char *lds = smem + stage * S::STAGE;
        // rows past n: zeros, also as statistics (their Q and dO are zero, so P = 1 and
        // dS = 0 meet rows of zeros)
        if constexpr (DMA) {
            Tile::issue(q, a.q.ld, n, place_q, lds, wave);
            Tile::issue(g, a.dout.ld, n, place_g, lds + Tile::BYTES, wave);
            constexpr int W = NST / 64;   // waves per statistic
            if (wave < 2 * W) {
                const int x = (wave % W) * 64 + lane;
                dma4(make_rsrc((wave < W ? f.nl : f.nd) + row),
                     lds + 2 * Tile::BYTES + wave * 256, x < n ? x * 4 : OOB);
            }
        } else {
            Tile::load(rq, q, a.q.ld, n, a.d, tid);
            Tile::load(rg, g, a.dout.ld, n, a.d, tid);
            if (tid < 2 * NST) {
                const int x = tid % NST;
                rs = x < n ? (tid < NST ? f.nl : f.nd)[row + x] : 0.f;
            }
        }
    };
    static_assert(2 * NST <= 256, "one statistic per thread");
    auto arrive = [&](int stage) {
        if constexpr (!DMA) {
            char *lds = smem + stage * S::STAGE;
            Tile::store(rq, lds, tid);
            Tile::store(rg, lds + Tile::BYTES, tid);
            if (tid < 2 * NST) reinterpret_cast<float *>(lds + 2 * Tile::BYTES)[tid] = rs;
        }
    };
    int iw = ii + kg * QT;   // this wave's rows of the step to compute
    if (s0 < s1) {
        issue(s0, 0);
        arrive(0);
    }

    const int64_t krow = min(key, a.sk - 1);
    const uint16_t *K = static_cast<const uint16_t *>(a.k.p) + (int64_t)b * a.k.sb +
                        (int64_t)hk * a.k.sh + krow * a.k.ld;
    const uint16_t *V = static_cast<const uint16_t *>(a.v.p) + (int64_t)b * a.v.sb +
                        (int64_t)hk * a.v.sh + krow * a.v.ld;
    bf16x8 kf[KS], vf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        kf[ks] = row_frag(K, ks * 16 + 8 * half, live ? a.d : 0, DMA);
        vf[ks] = row_frag(V, ks * 16 + 8 * half, live ? a.d : 0, DMA);
    }
    const float c = a.scale * LOG2E;

    f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int x = 0; x < DB; ++x) {
        dk[x] = splat16(0.f);
        dv[x] = splat16(0.f);
    }

    // a step's rows from i_wave on; EDGE: some key of the wave is not seen by all of them
    typename Tile::Reader rd(lds_at(smem) + kg * QT / Tile::RPS * Tile::SEG, lane);
    uint32_t stat = lds_at(smem) + 2 * Tile::BYTES + (kg * QT + 4 * half) * 4;
    auto step = [&](int i_wave, auto edge) {
        constexpr bool EDGE = decltype(edge)::value;
#pragma unroll
        for (int qb = 0; qb < QT / 32; ++qb) {
            const int r0 = qb * 32, i0 = i_wave + qb * 32;
            f32x16 s, dp;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 x = *(SBP_LDS const f32x4 *)(stat + (r0 + 8 * q) * 4);
                const f32x4 y = *(SBP_LDS const f32x4 *)(stat + (NST + r0 + 8 * q) * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[4 * q + e] = x[e];
                    dp[4 * q + e] = y[e];
                }
            }
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rd.frag(r0, ks, 0), kf[ks], s, 0, 0, 0);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rd.frag(r0, ks, Tile::BYTES), vf[ks], dp,
                                                             0, 0, 0);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[r] = exp2_(s[r] * c);
                dp[r] *= s[r];
                if constexpr (EDGE) {
                    const int i = i0 + 8 * (r >> 2) + 4 * half + (r & 3);
                    const bool seen = i >= lo && i < hi;
                    s[r] = seen ? s[r] : 0.f;
                    dp[r] = seen ? dp[r] : 0.f;
                }
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const bf16x8 p = pack8(s, 8 * x), ds = pack8(dp, 8 * x);
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    dv[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        rd.frag_t(db, r0 + 16 * x, Tile::BYTES), p, dv[db], 0, 0, 0);
                    dk[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        rd.frag_t(db, r0 + 16 * x, 0), ds, dk[db], 0, 0, 0);
                }
            }
        }
    };
    auto take = [&](int x, auto edge) {
        const int stage = (x - s0) & 1;
        wait_vm<0>();
        __syncthreads();
        const int next = ii + kg * QT;
        if (x + 1 < s1) issue(x + 1, stage ^ 1);
        step(iw, edge);
        iw = next;
        const int by = stage ? -S::STAGE : S::STAGE;
        rd.move(by);
        stat += by;
        if (x + 1 < s1) arrive(stage ^ 1);
    };
    int x = s0;
    for (; x < min(s1, edges); ++x) take(x, std::true_type{});
    for (; x < s1; ++x) take(x, std::false_type{});

    if constexpr (KG > 1) {
        __syncthreads();
        constexpr int SLOT = 2 * DB * 16 * 64;
        static_assert((KG - 1) * (NW / KG) * SLOT * 4 <= S::LDS, "group results do not fit");
        float *const base = reinterpret_cast<float *>(smem) + lane;
        if (kg > 0) {
            float *p = base + ((kg - 1) * (NW / KG) + wk) * SLOT;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    p[(db * 32 + r) * 64] = dk[db][r];
                    p[(db * 32 + 16 + r) * 64] = dv[db][r];
                }
        }
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int k = 1; k < KG; ++k) {
            const float *p = base + ((k - 1) * (NW / KG) + wk) * SLOT;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    dk[db][r] += p[(db * 32 + r) * 64];
                    dv[db][r] += p[(db * 32 + 16 + r) * 64];
                }
        }
    }
    if (key >= a.sk) return;
    // keys past the sequence's length get zeros (their lanes hold no sums of use)
    const int64_t d4 = (a.d + 3) & ~3;
    const int64_t n = (int64_t)a.batch * a.kv_heads * a.sk;
    float *const part = f.part + (((int64_t)split * n) + (int64_t)bh * a.sk + key) * 2 * d4;
    const int64_t atk = (int64_t)b * a.dk.sb + (int64_t)hk * a.dk.sh + (int64_t)key * a.dk.ld;
    const int64_t atv = (int64_t)b * a.dv.sb + (int64_t)hk * a.dv.sh + (int64_t)key * a.dv.ld;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int col = db * 32 + 8 * q + 4 * half;
            if (col >= a.d) continue;
            if (f.splits_k > 1) {
                f32x4 x, y;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = live ? dk[db][4 * q + e] : 0.f;
                    y[e] = live ? dv[db][4 * q + e] : 0.f;
                }
                *reinterpret_cast<f32x4 *>(part + col) = x;
                *reinterpret_cast<f32x4 *>(part + d4 + col) = y;
            } else {
                grad4(a.dk.p, atk, col, a.d, a.dk_f32, a.dk_acc, f.vec_k,
                      [&](int e) { return live ? dk[db][4 * q + e] * a.scale : 0.f; });
                grad4(a.dv.p, atv, col, a.d, a.dv_f32, a.dv_acc, f.vec_v,
                      [&](int e) { return live ? dv[db][4 * q + e] : 0.f; });
            }
        }
}

// Adds the splits' partials in split order. A thread owns 4 columns of a row of dQ
// (KV false) or of dK and dV.
template <bool KV>
__global__ __launch_bounds__(256) void attn_core_sum_kernel(BwdArgs f) {
    const CoreArgs &a = f.a;
    const int quads = (a.d + 3) >> 2;
    const int64_t d4 = quads * 4, per = KV ? a.sk : f.rows;
    const int64_t n = (int64_t)a.batch * a.kv_heads * per;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= n * quads) return;
    const int64_t at = id / quads;
    const int col = (int)(id % quads) * 4;
    const int bh = (int)(at / per), row = (int)(at % per);
    const int b = bh / a.kv_heads, hk = bh % a.kv_heads;
    if constexpr (KV) {
        f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
        for (int s = 0; s < f.splits_k; ++s) {
            const float *p = f.part + ((int64_t)s * n + at) * 2 * d4 + col;
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
            x += *reinterpret_cast<const f32x4 *>(f.part + ((int64_t)s * n + at) * d4 + col);
        const int i = row / a.group;
        const int64_t head = (int64_t)hk * a.group + (row - i * a.group);
        grad4(a.dq.p, (int64_t)b * a.dq.sb + head * a.dq.sh + (int64_t)i * a.dq.ld, col, a.d,
              a.dq_f32, a.dq_acc, f.vec_q, [&](int e) { return x[e] * a.scale; });
    }
}

}  // namespace sbpk

namespace sbpi {

namespace {

template <int DP, int KG, int KT>
hipError_t launch_dq(const sbpk::BwdArgs &f, int64_t blocks, hipStream_t s) {
    char name[160];
    name[0] = 0;
    if (profiling())
        snprintf(name, sizeof(name), "attn_core_dq_kernel<%d,%d,%d,%d>", DP, KG, KT,
                 (int)f.a.aligned);
    if (f.a.aligned)
        return launch_kernel(sbpk::attn_core_dq_kernel<DP, KG, KT, true>, name,
                             dim3((unsigned)blocks), dim3(256), s, f);
    return launch_kernel(sbpk::attn_core_dq_kernel<DP, KG, KT, false>, name,
                         dim3((unsigned)blocks), dim3(256), s, f);
}

template <int DP, int KG, int QT>
hipError_t launch_dkv(const sbpk::BwdArgs &f, int64_t blocks, hipStream_t s) {
    char name[160];
    name[0] = 0;
    if (profiling())
        snprintf(name, sizeof(name), "attn_core_dkv_kernel<%d,%d,%d,%d>", DP, KG, QT,
                 (int)f.a.aligned);
    if (f.a.aligned)
        return launch_kernel(sbpk::attn_core_dkv_kernel<DP, KG, QT, true>, name,
                             dim3((unsigned)blocks), dim3(256), s, f);
    return launch_kernel(sbpk::attn_core_dkv_kernel<DP, KG, QT, false>, name,
                         dim3((unsigned)blocks), dim3(256), s, f);
}

bool vec4(const CoreView &v, bool f32) {
    return reinterpret_cast<uintptr_t>(v.p) % (f32 ? 16 : 8) == 0 && v.ld % 4 == 0 &&
           v.sb % 4 == 0 && v.sh % 4 == 0;
}

}  // namespace

hipError_t launch_core_bwd(const CoreArgs &a, hipStream_t s) {
    sbpk::BwdArgs f;
    f.a = a;
    f.rows = a.sq * a.group;
    f.vec_q = vec4(a.dq, a.dq_f32);
    f.vec_k = vec4(a.dk, a.dk_f32);
    f.vec_v = vec4(a.dv, a.dv_f32);
    const int64_t bhs = (int64_t)a.batch * a.kv_heads;
    const int64_t qrows = bhs * f.rows;
    const size_t stat = core_bwd_stat_floats(a);
    float *const nl = a.ws, *const nd = a.ws + stat / 2;
    f.nl = nl;
    f.nd = nd;
    f.part = a.ws + stat;
    const size_t room = a.ws_floats - stat;
    const size_t d4 = (a.d + 3) & ~3;
    const int cus = device_cus();
    const bool wide = a.d > 64;
    hipError_t e;
    if (qrows > 0) {
        e = launch_kernel(sbpk::attn_core_stat_kernel, "attn_core_stat_kernel",
                          dim3((unsigned)((qrows + 15) / 16)), dim3(256), s, a, nl, nd);
        if (e != hipSuccess) return e;

        int kg = 1;
        while (kg < 4 && ((f.rows + 128 / kg - 1) / (128 / kg)) * bhs < cus) kg *= 2;
        const int rows = 128 / kg, keys = kg == 4 ? 128 : 64 * kg;
        f.tiles_q = (f.rows + rows - 1) / rows;
        const int64_t steps = ((int64_t)a.sk + keys - 1) / keys;
        int64_t splits = 1;
        while (f.tiles_q * bhs * splits * 2 <= 2 * cus && steps / (splits * 2) >= 2 &&
               (size_t)qrows * d4 * splits * 2 <= room)
            splits *= 2;
        f.splits_q = (int)splits;
        const int64_t blocks = f.tiles_q * bhs * splits;
        if (kg == 1)
            e = wide ? launch_dq<128, 1, 64>(f, blocks, s) : launch_dq<64, 1, 64>(f, blocks, s);
        else if (kg == 2)
            e = wide ? launch_dq<128, 2, 64>(f, blocks, s) : launch_dq<64, 2, 64>(f, blocks, s);
        else
            e = wide ? launch_dq<128, 4, 32>(f, blocks, s) : launch_dq<64, 4, 32>(f, blocks, s);
        if (e != hipSuccess) return e;
        if (splits > 1) {
            const int64_t items = qrows * (int64_t)(d4 / 4);
            e = launch_kernel(sbpk::attn_core_sum_kernel<false>, "attn_core_sum_kernel<0>",
                              dim3((unsigned)((items + 255) / 256)), dim3(256), s, f);
            if (e != hipSuccess) return e;
        }
    }
    const int64_t krows = bhs * a.sk;
    if (krows == 0) return hipSuccess;
    int kg = 1;
    while (kg < 4 && ((a.sk + 128 / kg - 1) / (128 / kg)) * bhs < cus) kg *= 2;
    const int keys = 128 / kg, qr = kg == 4 ? 128 : 64;
    f.tiles_k = (a.sk + keys - 1) / keys;
    const int64_t steps = (((int64_t)a.sq + qr - 1) / qr) * a.group;
    int64_t splits = 1;
    while (f.tiles_k * bhs * splits * 2 <= 2 * cus && steps / (splits * 2) >= 2 &&
           (size_t)krows * 2 * d4 * splits * 2 <= room)
        splits *= 2;
    f.splits_k = (int)splits;
    const int64_t blocks = f.tiles_k * bhs * splits;
    if (kg == 1)
        e = wide ? launch_dkv<128, 1, 64>(f, blocks, s) : launch_dkv<64, 1, 64>(f, blocks, s);
    else if (kg == 2)
        e = wide ? launch_dkv<128, 2, 32>(f, blocks, s) : launch_dkv<64, 2, 32>(f, blocks, s);
    else
        e = wide ? launch_dkv<128, 4, 32>(f, blocks, s) : launch_dkv<64, 4, 32>(f, blocks, s);
    if (e != hipSuccess || splits == 1) return e;
    const int64_t items = krows * (int64_t)(d4 / 4);
    return launch_kernel(sbpk::attn_core_sum_kernel<true>, "attn_core_sum_kernel<1>",
                         dim3((unsigned)((items + 255) / 256)), dim3(256), s, f);
}

}  // namespace sbpi
