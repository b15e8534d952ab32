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

using sbpi::CoreArgs;
using sbpi::CoreView;

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

// A tile of ROWS rows of DP bf16 values in LDS, rows in 16-byte chunks. Chunk c of
// row r sits at r*RB + 16*(c ^ f(r)). Two kinds of reads share the tile: 16-byte
// fragments of 16 consecutive rows (the same chunk of each: f takes every value
// on rows that start on the same bank), and transpose reads of 4 consecutive rows
// and 4 aligned chunks (f moves those rows' 64 bytes to distinct quarters of the
// 64 banks, or halves where a row is half the banks long).
template <int DP, int ROWS, int NW>
struct RowTile {
    static_assert(DP == 64 || DP == 128, "head dimension padded to 64 or 128");
    static constexpr int RB = DP * 2;
    static constexpr int CPR = DP / 8;
    static constexpr int BYTES = ROWS * RB;
    static constexpr int SEGS = BYTES / 1024;
    static constexpr int NV = SEGS / NW;      // 16-byte chunks per thread
    static_assert(SEGS % NW == 0, "tile too small for the wave count");

    __device__ __forceinline__ static int swz(int r) {
        return DP == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    }

    // Rows [0, n) of the tile at `base` (uniform) go to LDS, rows past n and
    // columns past d as zeros. Direct-to-LDS loads: base and ld 16-byte aligned,
    // d a multiple of 8, ROWS * ld * 2 < 2^31.
    __device__ __forceinline__ static void issue(const uint16_t *base, int64_t ld, int n, int d,
                                                 char *lds, int wave, int lane) {
        const i32x4 r = make_rsrc(base);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int s = i * NW + wave;
            const int row = s * (1024 / RB) + lane / CPR;
            const int c = (lane % CPR) ^ swz(row);
            const bool ok = row < n && c * 8 < d;
            dma16(r, lds + s * 1024, ok ? (row * (int)ld + c * 8) * 2 : OOB);
        }
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
            const int row = q / CPR, c = q % CPR;
            *reinterpret_cast<u32x4 *>(lds + row * RB + ((c ^ swz(row)) << 4)) = v[i];
        }
    }

    // Rows [r0, r0 + 32), columns [16 ks, 16 ks + 16) with the columns as reduction
    // (8 h + 0..7 of them for half h).
    __device__ __forceinline__ static bf16x8 frag(const char *lds, int r0, int ks, int lane) {
        const int row = r0 + (lane & 31);
        const int c = ks * 2 + (lane >> 5);
        return *reinterpret_cast<const bf16x8 *>(lds + row * RB + ((c ^ swz(row)) << 4));
    }
    // Columns [c0, c0 + 32), rows [r0, r0 + 16) with the rows as reduction (rows
    // 4 h + 0..3 and 8 + 4 h + 0..3 for half h).
    __device__ __forceinline__ static bf16x8 frag_t(const char *lds, int c0, int r0, int lane) {
        const int g = lane >> 4, t = lane & 15;
        const int mn = c0 + 16 * (g & 1) + 4 * (t & 3);
        s16x4 x[2];
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            const int row = r0 + hh * 8 + (g >> 1) * 4 + (t >> 2);
            const int off = row * RB + (((mn >> 3) ^ swz(row)) << 4) + ((mn & 7) << 1);
            x[hh] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SBP_LDS s16x4 *)(lds + off));
        }
        s16x8 v8 = {x[0][0], x[0][1], x[0][2], x[0][3], x[1][0], x[1][1], x[1][2], x[1][3]};
        return __builtin_bit_cast(bf16x8, v8);
    }
};

// 8 columns of a row in memory (columns past d as zeros), at any alignment.
__device__ __forceinline__ bf16x8 row_frag(const uint16_t *row, int at, int d, bool aligned) {
    u32x4 v = {0u, 0u, 0u, 0u};
    if (at + 8 <= d)
        v = aligned ? *reinterpret_cast<const u32x4 *>(row + at) : ld16_any(row + at);
    else if (at < d)
        v = ld16_tail(row, at, d);
    return __builtin_bit_cast(bf16x8, v);
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

}  // namespace sbpk
