// attn_core_kernel.h -- what the softmax attention kernels share (CDNA4 /
// gfx950): row tiles in LDS, fragment reads, the mask.
//
// Every product runs on v_mfma_f32_32x32x16_bf16. Its 32 x 32 result leaves lane l
// with column l % 32 and, in register q, row 8 (q / 4) + 4 (l / 32) + q % 4. Its
// operands give lane l row (or column) l % 32 and 8 reduction indices, of which
// the two half-waves hold disjoint sets; any assignment of reduction indices to
// these slots is right as long as both operands use the same one. The kernels
// use the one that the result layout already has -- half h holds indices 4 h + 0..3
// and 8 + 4 h + 0..3 of every 16 -- so probabilities go from the product that
// made them into the product that reads them without leaving their registers.
#pragma once

#include "attn_core.h"
#include "gemm_bf16_dma.h"

namespace sbpk {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

using sbpi::CoreArgs;
using sbpi::CoreView;

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

__device__ __forceinline__ uint32_t lds_at(const void *p) {
    return (uint32_t)(uintptr_t)(SBP_LDS const void *)p;
}

// dma16 to byte `lds` of LDS (uniform).
__device__ __forceinline__ void dma16_at(i32x4 r, uint32_t lds, int voff) {
    const uint32_t m0 = __builtin_amdgcn_readfirstlane(lds);
    asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :
                 : "s"(m0), "v"(voff), "s"(r)
                 : "memory", "m0");
}

// A tile of ROWS rows of DP bf16 values in LDS. A direct-to-LDS load of a wave fills 1 KB,
// RPS whole rows in 16-byte chunks; these segments lie 1040 bytes apart, and within one
// chunk c of row b is stored as chunk c ^ swz(b). Two kinds of reads share the tile:
// 16-byte fragments (the same chunk of 16 consecutive rows) and transpose reads (4
// aligned chunks of 4 consecutive rows). Both meet every bank once: rows of a segment
// that start on the same bank differ in swz, by 4 where they are neighbours in a transpose
// read, and consecutive segments are one chunk apart. swz only changes the bits of c that
// step through the head dimension, so a lane needs 4 addresses for the fragments and one
// per 32 columns for the transposed ones; rows, stages' halves and the other reads are
// constant offsets.
template <int DP, int ROWS, int NW>
struct RowTile {
    static_assert(DP == 64 || DP == 128, "head dimension padded to 64 or 128");
    static constexpr int RB = DP * 2;          // bytes of a row
    static constexpr int CPR = DP / 8;         // its chunks
    static constexpr int RPS = 1024 / RB;      // rows of a segment
    static constexpr int SEG = 1040;
    static constexpr int SEGS = ROWS / RPS;
    static constexpr int BYTES = SEGS * SEG;
    static constexpr int NV = SEGS / NW;       // 16-byte chunks per thread
    static_assert(SEGS % NW == 0, "tile too small for the wave count");

    __host__ __device__ static constexpr int swz(int b) {   // b: row of a segment
        return DP == 128 ? (b & 3) << 2 : (((b >> 1) & 1) << 2) | (((b >> 2) & 1) << 1);
    }
    __host__ __device__ static constexpr int at(int row, int c) {
        return row / RPS * SEG + row % RPS * RB + ((c ^ swz(row % RPS)) << 4);
    }

    // Direct-to-LDS loads: base and ld 16-byte aligned, d a multiple of 8,
    // ROWS * ld * 2 < 2^31. A lane's place in the tile's first NW segments:
    __device__ __forceinline__ static int place(int64_t ld, int d, int wave, int lane) {
        const int b = lane / CPR, c = (lane % CPR) ^ swz(b);
        return c * 8 < d ? ((wave * RPS + b) * (int)ld + c * 8) * 2 : OOB;
    }
    // Load i of the NV that bring the rows of buffer `r` to byte `lds` of LDS. Rows past the
    // buffer's end and columns past d lie outside it and arrive as zeros.
    __device__ __forceinline__ static void issue(i32x4 r, int64_t ld, int place, uint32_t lds,
                                                 int wave, int i) {
        dma16_at(r, lds + (i * NW + wave) * SEG, place + i * (NW * RPS * (int)ld * 2));
    }

    // The same through registers, for rows at any element alignment and stride.
    typedef u32x4 Regs[NV];
    __device__ __forceinline__ static void load(Regs &v, const uint16_t *base, int64_t ld, int n,
                                                int d, int tid) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int q = i * 64 * NW + tid;
            const int row = q / CPR, at = q % CPR * 8;
            v[i] = u32x4{0u, 0u, 0u, 0u};
            if (row < n && at < d) {
                const uint16_t *r = base + (int64_t)row * ld;
                v[i] = at + 8 <= d ? ld16_any(r + at) : ld16_tail(r, at, d);
            }
        }
    }
    __device__ __forceinline__ static void store(const Regs &v, char *lds, int tid) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int q = i * 64 * NW + tid;
            *reinterpret_cast<u32x4 *>(lds + at(q / CPR, q % CPR)) = v[i];
        }
    }

    // A lane's read addresses in the tile at byte `base` of LDS.
    struct Reader {
        uint32_t f[4], t[DP / 32];

        __device__ __forceinline__ Reader(uint32_t base, int lane) {
            const int row = lane & 31, half = lane >> 5;
            constexpr int STEP = DP == 128 ? 4 : 2;   // chunks between addresses
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = base + at(row, STEP * j + half);
            const int g = lane >> 4, u = lane & 15;
#pragma unroll
            for (int db = 0; db < DP / 32; ++db)
                t[db] = base + at((g >> 1) * 4 + (u >> 2), db * 4 + 2 * (g & 1) + ((u & 3) >> 1)) +
                        8 * (u & 1);
        }
        __device__ __forceinline__ void move(int by) {
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] += by;
#pragma unroll
            for (int db = 0; db < DP / 32; ++db) t[db] += by;
        }
        // Rows [r0, r0 + 32), columns [16 ks, 16 ks + 16) with the columns as reduction
        // (8 h + 0..7 of them for half h). r0 and the byte offset `off` are constants.
        __device__ __forceinline__ bf16x8 frag(int r0, int ks, int off) const {
            const uint32_t p = DP == 128 ? f[ks >> 1] : f[ks];
            const int at = r0 / RPS * SEG + (DP == 128 ? (ks & 1) * 32 : 0) + off;
            return *(SBP_LDS const bf16x8 *)(p + at);
        }
        // Columns [32 db, 32 db + 32), rows [r0, r0 + 16) with the rows as reduction (rows
        // 4 h + 0..3 and 8 + 4 h + 0..3 for half h).
        __device__ __forceinline__ bf16x8 frag_t(int db, int r0, int off) const {
            const uint32_t p = t[db];
            const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (SBP_LDS s16x4 *)(p + r0 / RPS * SEG + off));
            const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (SBP_LDS s16x4 *)(p + (r0 + 8) / RPS * SEG + off));
            const s16x8 v8 = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
            return __builtin_bit_cast(bf16x8, v8);
        }
    };
};

// 8 columns of a row in memory (columns past d as zeros): ALIGNED rows have 16-byte
// blocks that lie wholly before or past d; others are read at any alignment.
template <bool ALIGNED>
__device__ __forceinline__ bf16x8 row_frag(const uint16_t *row, int at, int d) {
    u32x4 v = {0u, 0u, 0u, 0u};
    if constexpr (ALIGNED) {
        if (at < d) v = *reinterpret_cast<const u32x4 *>(row + at);
    } else {
        if (at + 8 <= d) v = ld16_any(row + at);
        else if (at < d) v = ld16_tail(row, at, d);
    }
    return __builtin_bit_cast(bf16x8, v);
}

// Waits here for the loads of x. The compiler does not see the direct-to-LDS loads; left to
// the first use inside a loop, its wait would be for every load in flight, in every pass
// (the loads of later stages among them: dK and dV of 16 heads over 4, 8192 x 128 causal,
// 625 us with those waits and 609 without).
template <int N>
__device__ __forceinline__ void settle(bf16x8 (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));
}

__device__ __forceinline__ bf16x8 pack8(const f32x16 &x, int q0) {
    bf16x8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (__bf16)x[q0 + e];
    return r;
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// Both half-waves' values of x, in every lane.
__device__ __forceinline__ void halves(float x, float *lo, float *hi) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    *lo = __builtin_bit_cast(float, (uint32_t)r[0]);
    *hi = __builtin_bit_cast(float, (uint32_t)r[1]);
}

__device__ __forceinline__ f32x16 splat16(float x) {
    f32x16 v;
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] = x;
    return v;
}

// What query i of a sequence sees: keys [lo(i), hi(i)).
struct SeqMask {
    int lq, lk, off, window;
    bool causal;
    __device__ __forceinline__ SeqMask(const CoreArgs &a, int b) {
        lq = a.len_q ? min(max(a.len_q[b], 0), a.sq) : a.sq;
        lk = a.len_k ? min(max(a.len_k[b], 0), a.sk) : a.sk;
        off = lk - lq;
        window = a.window;
        causal = a.causal != 0;
    }
    __device__ __forceinline__ int hi(int i) const {
        return causal ? max(0, min(lk, i + 1 + off)) : lk;
    }
    __device__ __forceinline__ int lo(int i) const {
        return window ? max(0, i + 1 + off - window) : 0;
    }
};

// Part i of 0 .. PARTS - 1 of a block's 16 values holds value r.
__device__ __forceinline__ constexpr bool in_part(int r, int i, int parts) {
    return r >= 16 * i / parts && r < 16 * (i + 1) / parts;
}

// A direct-to-LDS load to come: two tiles.
struct Fetch {
    i32x4 x, y;
    uint32_t lds;
};

// Where result rows go: bf16 or fp32, overwritten or added to; `vec`: d is a multiple of 4
// and the rows allow loads and stores of 4 values.
struct RowsOut {
    void *p;
    int32_t d;
    bool f32, add, vec;
};

// Results leave through LDS, so that 16 lanes store a row's 64 values side by side and the
// wave groups of a row are summed on the way (in group order), each group storing a part
// of the rows. A wave's tile is 32 x DP floats in parts of 32 x 68.
template <int DP>
constexpr int PUT_FLOATS = DP / 64 * 32 * 68;

// A wave's result (lane l holds column l % 32, here a row of the output, and in acc[db]
// register q value 32 db + 8 (q / 4) + 4 (l / 32) + q % 4 of it), times `mul` (0 where that is
// 0), to its tile.
template <int DP>
__device__ __forceinline__ void stage_rows(float *tile, const f32x16 *acc, float mul, int lane) {
    float *const row = tile + (lane & 31) * 68 + 4 * (lane >> 5);
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int q = 0; q < 16; q += 4) {
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = mul != 0.f ? acc[db][q + e] * mul : 0.f;
            *reinterpret_cast<f32x4 *>(row + db / 2 * (32 * 68) + db % 2 * 32 + 2 * q) = v;
        }
}

// Stores the rows of KG groups' tiles, `step` floats apart: group kg the kg-th part of the
// rows. off: element offset of row (lane % 32), or < 0 for none.
template <int DP, int KG>
__device__ __forceinline__ void store_rows(const float *tiles, int step, int kg, const RowsOut &o,
                                           int64_t off, int lane) {
    constexpr int N = 8 / KG;
    const int r0 = kg * (32 / KG) + (lane >> 4);
    const int lo = (int)off, hi = (int)(off >> 32);
#pragma unroll
    for (int c0 = 0; c0 < DP; c0 += 64) {
        const float *const t = tiles + c0 / 64 * (32 * 68) + r0 * 68 + (lane & 15) * 4;
        const int col = c0 + (lane & 15) * 4;
        auto value = [&](int it) {
            f32x4 v = *reinterpret_cast<const f32x4 *>(t + it * (4 * 68));
#pragma unroll
            for (int k = 1; k < KG; ++k)
                v += *reinterpret_cast<const f32x4 *>(t + k * step + it * (4 * 68));
            return v;
        };
        auto place = [&](int it) {
            const int from = 4 * (r0 + 4 * it);
            const int h = __builtin_amdgcn_ds_bpermute(from, hi);
            return (int64_t)(((uint64_t)(uint32_t)h << 32) |
                             (uint32_t)__builtin_amdgcn_ds_bpermute(from, lo));
        };
        if (o.vec && !o.f32) {
#pragma unroll
            for (int it = 0; it < N; ++it) {
                const f32x4 v = value(it);
                const int64_t at = place(it);
                bf16x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = (__bf16)v[e];
                if (at >= 0 && col < o.d)
                    *reinterpret_cast<bf16x4 *>(static_cast<uint16_t *>(o.p) + at + col) = w;
            }
        } else if (o.vec) {
#pragma unroll
            for (int it = 0; it < N; ++it) {
                f32x4 v = value(it);
                const int64_t at = place(it);
                if (at >= 0 && col < o.d) {
                    f32x4 *const p = reinterpret_cast<f32x4 *>(static_cast<float *>(o.p) + at + col);
                    if (o.add) v += *p;
                    *p = v;
                }
            }
        } else {
#pragma unroll 1
            for (int it = 0; it < N; ++it) {
                const f32x4 v = value(it);
                const int64_t at = place(it);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (at < 0 || col + e >= o.d) continue;
                    if (o.f32) {
                        float *const p = static_cast<float *>(o.p) + at + col + e;
                        *p = o.add ? *p + v[e] : v[e];
                    } else {
                        static_cast<uint16_t *>(o.p)[at + col + e] = f32_to_bf16_bits(v[e]);
                    }
                }
            }
        }
    }
}

// Division by a number that the launch knows, of n < 2^31: n m / 2^32 with m = (2^32 - 1) / d is
// at most n / d and more than n / d - n / 2^32 - 1, so off by one at most. (The compiler's
// division is a chain of 30 instructions; a workgroup does six before its first load.)
struct Div {
    uint32_t d = 1, m = ~0u;
    Div() = default;
    explicit Div(int64_t n) : d(n > 1 ? (uint32_t)n : 1u), m(~0u / d) {}
    __device__ __forceinline__ int operator()(int n) const {
        const uint32_t q = (uint32_t)((uint64_t)(uint32_t)n * m >> 32);
        return (int)(q + ((uint32_t)n - q * d >= d ? 1u : 0u));
    }
    // n % d, given q = n / d.
    __device__ __forceinline__ int rest(int n, int q) const { return n - q * (int)d; }
};

// Which (sequence, key head) and which of its `per` items, heaviest first, a workgroup takes.
// Workgroups go to the XCDs in turn. Where the heads are a multiple of 8, each XCD takes
// whole heads, one after the other, whose keys then stay in its L2; else the heads'
// items are dealt out in turn, all heaviest ones first, so that a head that is spread over
// several XCDs leaves none with its heavier half (16 query heads over 4 key heads, 8192 x 128
// causal: dQ 563 us in one
// head after the other and 412 dealt out, dK and dV 878 and 625).
__device__ __forceinline__ void deal(int wg, const Div &heads, const Div &per, int *bh, int *item) {
    const bool whole = heads.d % 8 == 0;
    const int l = whole ? remap_xcd(wg, (int)(heads.d * per.d)) : wg;
    const int q = whole ? per(l) : heads(l), r = whole ? per.rest(l, q) : heads.rest(l, q);
    *bh = whole ? q : r;
    *item = whole ? r : q;
}

// The order in which a workgroup takes the n steps of its walk: first those that need
// the mask, [0, na) and [nb, n), then the others. Two loops, so that the second holds no
// code of the first (as a branch inside one loop, the two forms' accumulators cost
// copies in every step).
struct Walk {
    int n, na, nb;
    __device__ __forceinline__ int masked() const { return na + n - nb; }
    __device__ __forceinline__ int step(int x) const {
        const int e = masked();
        return x < na ? x : x < e ? nb + (x - na) : na + (x - e);
    }
};

}  // namespace sbpk
