// attn_core_walk.h -- a wave's part of a tile's walk over its keys in softmax attention
// (CDNA4 / gfx950): shared by the forward kernels over whole sequences and over a paged cache,
// which differ in where their keys come from.
#pragma once

#include "attn_core_kernel.h"

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

// WPS: waves of a SIMD, of one workgroup or two. DC: columns of the products, of the DP of a tile.
template <int DP_, int KG_, int KT_, int NW_, int WPS_, bool DMA, int DC_ = DP_>
struct FwdShape {
    static constexpr int DP = DP_, DC = DC_, KG = KG_, KT = KT_, NW = NW_, WPS = WPS_;
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

// A wave's rows (lane l has row l % 32, half of its scores, the other half-wave the rest) and
// what it holds of them: running maximum m and sum l, output O^T.
template <class S>
struct FwdRows {
    using Tile = typename S::Tile;
    static constexpr int KT = S::KT, NS = S::NS;
    static constexpr int NB = KT / 32, KS = S::DC / 16, DB = S::DC / 32;

    typename Tile::Reader rd;
    bf16x8 qf[KS];
    float c, grow;
    float m = -INFINITY, l = 0.f;
    float mc = 0.f, limit = -INFINITY;   // what exponents add to s c; where the maximum moves
    f32x16 o[DB];
    f32x16 sp[2];                   // scores of this block and the next, in turn
    int stage = 0;                  // of the step at work
    int half, lo, hi;               // the row sees keys [lo, hi)

    __device__ __forceinline__ FwdRows(uint32_t lds, int lane, float scale, int lo_, int hi_)
        : rd(lds, lane), c(scale * LOG2E), grow(8.f / c), half(lane >> 5), lo(lo_), hi(hi_) {
#pragma unroll
        for (int x = 0; x < DB; ++x) o[x] = splat16(0.f);
    }

    // Scores of 32 keys; beside(0 .. KS) are put between the products.
    template <class Beside>
    __device__ __forceinline__ void scores(f32x16 &s, const typename Tile::Reader &r, int r0,
                                           Beside beside) {
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
    }
    // The keys of the block of 32 that begins at k0 that this row sees, by its range [lo, hi): bit
    // 8 (r / 4) + r % 4 of the result for score r (half h holds keys 4 h further).
    __device__ __forceinline__ uint32_t seen(int k0) const { return range(k0) >> (4 * half); }
    __device__ __forceinline__ uint32_t range(int k0) const {
        const int x = min(max(lo - k0, 0), 32), y = min(max(hi - k0, 0), 32);
        return (uint32_t)((1ull << y) - 1) & ~(uint32_t)((1ull << x) - 1);
    }
    __device__ __forceinline__ static void hide(f32x16 &s, uint32_t seen, int r) {
        s[r] = seen & 1u << (8 * (r >> 2) + (r & 3)) ? s[r] : -INFINITY;
    }
    // Moves the maximum to `top`, the maximum of a lane's own scores s, where it grew by enough.
    // Where a row's is FAR, s become differences from it, and every block comes here.
    __device__ __forceinline__ void rise(f32x16 &s, float top) {
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
    }
    // The first block's scores, of keys from k0 on, and its maximum.
    template <class Seen>
    __device__ __forceinline__ void begin(int k0, Seen seen_) {
        scores(sp[0], rd, 0, [](int) {});
        const uint32_t bits = seen_(k0);
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            hide(sp[0], bits, r);
            top = fmaxf(top, sp[0][r]);
        }
        rise(sp[0], top);
    }
    // A step: two phases a block of 32 keys, the next block's scores beside this one's
    // exponentials; then this block's product with V beside the next one's maximum. The first
    // phase has priority over the other wave's second, which waits for less (16 heads over 4 of
    // 8192 x 128, causal: 273 us without, 260).
    // kw, kn: the wave's first key of this step and of the next; more: there is a next one.
    // EDGE: some row of the tile does not see every key of the step; seen_(k0) says which of a
    // block's, as seen() does. advance(): waits for the next
    // step and prepares the load of a later one, which part(q) issues in LOADS parts.
    template <bool EDGE, class Seen, class Advance, class Part>
    __device__ __forceinline__ void take(int kw, int kn, bool more, Seen seen_, Advance advance,
                                         Part part) {
        const bool wrap = stage == NS - 1;
        const int by = wrap ? -(NS - 1) * S::STAGE : S::STAGE;
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
            const bool last = kb == NB - 1;
            if (last) advance();
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
            scores(s_n, nx, last ? 0 : (kb + 1) * 32, [&](int part_) __attribute__((always_inline)) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    if (!in_part(r, part_, KS + 1)) continue;
                    s[r] = exp2_(__builtin_fmaf(s[r], c, mc));
                    l += s[r];
                    if (r % 8 == 7) p[r / 8] = pack8(s, r - 7);
                }
                // the first 16 keys' columns
                if (part_ > KS - DB)
                    tv[0][part_ - 1 - (KS - DB)] = rd.frag_t(part_ - 1 - (KS - DB), kb * 32, Tile::BYTES);
            });
            __builtin_amdgcn_s_setprio(0);
            // the loads of a step, spread over its blocks: the last one's first
            constexpr int PER = (S::LOADS + NB - 1) / NB;
            const int first = last ? 0 : (kb + 1) * PER;
            float top = -INFINITY;
            uint32_t bits = 0;
            if constexpr (EDGE) bits = seen_(last ? kn : kw + (kb + 1) * 32);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tv[h][db], p[h], o[db], 0, 0, 0);
                    if (h == 0) tv[1][db] = rd.frag_t(db, kb * 32 + 16, Tile::BYTES);
                    const int k = h * DB + db;
#pragma unroll
                    for (int q = PER * k / (2 * DB); q < PER * (k + 1) / (2 * DB); ++q)
                        if (first + q < S::LOADS) part(first + q);
                    // the next scores are there one product later
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        if (k == 0 || !in_part(r, k - 1, 2 * DB - 1)) continue;
                        if constexpr (EDGE) hide(s_n, bits, r);
                        top = fmaxf(top, s_n[r]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            if (!last || more) rise(s_n, top);
            if constexpr (!TURN) sp[0] = sp[1];
        }
        rd.move(by);
        stage = wrap ? 0 : stage + 1;
    }
    // The sums of both half-waves and of the KG wave groups that share the rows, whose m and l
    // become the rows'; returns 2^((m - the groups' maximum) c). A barrier lies between the
    // groups' stores to `stats` and the loads.
    __device__ __forceinline__ float join_groups(float *stats, int wave, int wr) {
        float l0, l1;
        halves(l, &l0, &l1);
        l = l0 + l1;
        float mul = 1.f;
        if constexpr (S::KG > 1) {
            stats[wave * 128] = m;
            stats[wave * 128 + 64] = l;
            __syncthreads();
            const float *const p = stats + wr * S::KG * 128;
            float mn = p[0];
#pragma unroll
            for (int k = 1; k < S::KG; ++k) mn = fmaxf(mn, p[k * 128]);
            const float ms = mn == -INFINITY ? 0.f : mn;
            l = 0.f;
#pragma unroll
            for (int k = 0; k < S::KG; ++k) l += p[k * 128 + 64] * exp2_((p[k * 128] - ms) * c);
            mul = exp2_((m - ms) * c);
            m = mn;
        }
        return mul;
    }
};

}  // namespace sbpk
