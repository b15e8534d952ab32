// gemm_f32.hip -- fp32-input path of the local matmul and the bf16 dispatch
// by orientation.
//
// The fp32 path serves fp32 training (the paper's P100 runs are fp32). Two
// kernels: the matrix-core kernel below for every product whose tiles fit
// 31-bit buffer offsets, and a plain FMA kernel for leading dimensions beyond
// that (2^21 elements) and for reductions so short that the stores bound the launch
// (plan.cpp f32_fma).
//
// Matrix-core kernel (gemm_f32_mfma_kernel), bound by the fp32 MFMA rate:
//   * v_mfma_f32_32x32x2_f32: fp32 products and sums, 256 flop/clk/CU -- the
//     same fp32 arithmetic as FMAs, in another order of k.
//   * Four waves (2 x 2), 128 x 128 or 64 x 64 output tile, 32-wide reduction
//     steps; two stages of both operand tiles in LDS, loaded by buffer loads
//     that write LDS directly. A 128 x 128 step is 4096 cycles of MFMA per
//     32 KB of operands, so one stage ahead and a second workgroup per CU
//     (four or five of the 64 x 64 ones) cover the memory latency, barriers
//     and epilogues. More stages (three to eight) with fewer workgroups per
//     CU, or two reduction groups of waves, were no faster; 128 x 64 tiles
//     lay between the two.
//   * The two backward products of a linear share one launch where the model
//     expects it to pay: two 256-tile products of 128 x 128 tiles 148 -> 136 us.
//   * Measured, against the FMA kernel below: 1024 x 4096 x 1024 forward
//     240 -> 75 us, 256 x 4096 x 3136 forward 660 -> 63 us, 4096^3 134
//     TFLOP/s (the library product reaches 141); the largest error against
//     64 bits over fp32 layers of those sizes 1.1e-6 -> 8.1e-7.
//   * V = 4: 16 bytes per lane, where both operands' base, ld and contiguous
//     extent are multiples of 4 floats. V = 1: 4 bytes per lane with per-element
//     bounds, for any other operand: four times the load instructions, which
//     still fit under the MFMA time of a step.
//   * k-major tiles: 128-byte rows (32 reduction values) of eight 16-byte
//     chunks, chunk c of row r at c ^ ((r / 2) % 8), so a 16-row
//     ds_read_b128 phase covers all 64 banks; lane l takes chunk 2 j + l / 32,
//     i.e. MFMA e of group j multiplies k = 8 j + e (lower half-wave) and
//     8 j + 4 + e (upper half).
//   * m/n-major tiles: rows of BM (BN) values per reduction index, read with
//     ds_read_b32 at the same k; chunks of rows with odd k / 4 are shifted by
//     8 so that the two half-waves use different banks.
//   * Split reduction as in the bf16 kernels (split_reduce.hip adds the fp32
//     partials in split order).
#include <algorithm>
#include <type_traits>

#include "gated.h"
#include "gemm.h"
#include "gemm_bf16_dma.h"
#include "profile.h"

namespace sbpk {

struct F32Args {
    const float *A;
    const float *B;
    float *C;
    int64_t lda, ldb, ldc;
    int32_t m, n, k;
    int32_t tiles_m, tiles_n;
    int32_t splits, kchunk;   // reduction elements per split (a multiple of 32)
    float *ws;                // split partials, row stride partial_ld(n)
    int32_t accumulate;       // add the product to C's contents
};

// A product that reduces over two pairs of operands in turn: k1 of each, the first
// rounded up to kp, whole steps; k = kp + k1.
struct F32ArgsTwo : F32Args {
    const float *A2, *B2;
    int64_t lda2, ldb2;
    int32_t k1, kp;
};

// A weight gradient whose operands' rows hold m_load and n_load elements that may be read.
struct F32ArgsPad : F32Args {
    int32_t m_load, n_load;
};

// One 4-byte-per-lane buffer load that writes LDS directly (see dma16).
__device__ __forceinline__ void dma4(i32x4 r, char *lds, int voff) {
    const uint32_t m0 = __builtin_amdgcn_readfirstlane(
        (uint32_t)(uintptr_t)(SBP_LDS void *)lds);
    asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                 :
                 : "s"(m0), "v"(voff), "s"(r)
                 : "memory", "m0");
}

constexpr int FK = 32;   // reduction elements per step

// Operand tile of BMN output indices x FK reduction indices (layouts above).
template <int BMN, bool KMAJ, int V>
struct F32Tile {
    static constexpr int LOADS = BMN * FK / (64 * V * 4);   // per wave (4 waves)

    __device__ __forceinline__ static int swz(int row) {
        return KMAJ ? (row >> 1) & 7 : ((row >> 2) & 1) << 3;
    }

    __device__ __forceinline__ static void issue(const float *base, int64_t ld, int mn0,
                                                 int mn_lim, int k0, int k_lim, char *lds,
                                                 int wave, int lane) {
        constexpr int ROW = KMAJ ? FK : BMN;   // floats per LDS row
        const i32x4 r = make_rsrc(KMAJ ? base + (int64_t)mn0 * ld + k0
                                       : base + (int64_t)k0 * ld + mn0);
        // rows left along the row index, elements left along the contiguous one
        const int rows = KMAJ ? mn_lim - mn0 : k_lim - k0;
        const int cols = KMAJ ? k_lim - k0 : mn_lim - mn0;
        const int ldi = (int)ld;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int seg = (i * 4 + wave) * 64 * V;
            const int pos = seg + lane * V;
            const int row = pos / ROW, in = pos % ROW;
            const int col = (((in >> 2) ^ swz(row)) << 2) + (in & 3);
            const bool ok = row < rows && col + V <= cols;
            const int voff = ok ? (row * ldi + col) * 4 : OOB;
            if constexpr (V == 4) dma16(r, lds + seg * 4, voff);
            else dma4(r, lds + seg * 4, voff);
        }
    }

    // Values k = 8 j + 4 (lane / 32) + 0..3 of output index c0 + lane % 32.
    __device__ __forceinline__ static f32x4 frag(const char *lds, int c0, int j, int lane) {
        const int mn = c0 + (lane & 31);
        if constexpr (KMAJ) {
            const int c = 2 * j + (lane >> 5);
            return *reinterpret_cast<const f32x4 *>(lds + mn * FK * 4 + ((c ^ swz(mn)) << 4));
        } else {
            const int k = 8 * j + 4 * (lane >> 5);   // rows k .. k+3 share one swizzle
            const float *p = reinterpret_cast<const float *>(lds) + k * BMN +
                             ((((mn >> 2) ^ swz(k)) << 2) | (mn & 3));
            f32x4 v = {p[0], p[BMN], p[2 * BMN], p[3 * BMN]};
            return v;
        }
    }
};

// Adds a lane's 16 elements of a 32 x 32 MFMA block (rows rbase + 8 (r / 4) + r % 4
// of the block that starts at row r0, column col) to the output `out`, row stride
// ldo, rows below m, as the bf16 kernels' direct epilogue does: all old values
// loaded before any is stored, no bounds checks kept between the two. (2000 x 1003
// over 16, 7.8 -> 5.8 us against bounds-checked loads; the FMA kernel takes 11.4.)
__device__ __forceinline__ void add_block(void *out, int64_t ldo, int rbase, int col, int r0, int m,
                                          const f32x16 v) {
    typedef __attribute__((address_space(1))) float GlobalFloat;
    float old[16];
    r0 = __builtin_amdgcn_readfirstlane(r0);
    if (r0 + 32 <= m) {
        GlobalFloat *d = (GlobalFloat *)out + ((int64_t)rbase * ldo + col);
        asm volatile("" : "+v"(d) : : "memory");
#pragma unroll
        for (int r = 0; r < 16; ++r) old[r] = d[(8 * (r >> 2) + (r & 3)) * ldo];
        asm volatile("" : "+v"(d) : : "memory");
#pragma unroll
        for (int r = 0; r < 16; ++r) d[(8 * (r >> 2) + (r & 3)) * ldo] = old[r] + v[r];
        return;
    }
    GlobalFloat *const c = (GlobalFloat *)out + col;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int row = rbase + 8 * (r >> 2) + (r & 3);
        old[r] = c[(int64_t)min(row, m - 1) * ldo];
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int row = rbase + 8 * (r >> 2) + (r & 3);
        if (row < m) c[(int64_t)row * ldo] = old[r] + v[r];
    }
}

// One work item (an output tile and a reduction split; L its logical index).
// ACCUM: as in the bf16 tile body.
template <int BM, int BN, bool A_KMAJ, bool B_KMAJ, int V, int ACCUM, class Args>
__device__ __forceinline__ void f32_tile_body(const Args &g, const int L, char *smem) {
    using TA = F32Tile<BM, A_KMAJ, V>;
    using TB = F32Tile<BN, B_KMAJ, V>;
    constexpr int A_BYTES = BM * FK * 4, STAGE = (BM + BN) * FK * 4;
    constexpr int WM = BM / 2, WN = BN / 2, MI = WM / 32, NI = WN / 32;
    const int lane = threadIdx.x & 63;
    const int wave = threadIdx.x >> 6;
    const int wm = wave >> 1, wn = wave & 1;

    const int tiles = g.tiles_m * g.tiles_n;
    const int split = L / tiles;
    const int t = L % tiles;
    constexpr int GROUP = SBP_TILE_GROUP;
    const int grp = t / (GROUP * g.tiles_n);
    const int first_m = grp * GROUP;
    const int gsize = min(g.tiles_m - first_m, GROUP);
    const int tg = t - grp * GROUP * g.tiles_n;
    const int m0 = (first_m + tg % gsize) * BM, n0 = (tg / gsize) * BN;
    const int k_begin = split * g.kchunk;
    const int k_lim = min(g.k, k_begin + g.kchunk);
    const int nkb = max(0, (k_lim - k_begin + FK - 1) / FK);

    auto issue = [&](int kb, int stage) {
        char *base = smem + stage * STAGE;
        const int k0 = k_begin + kb * FK;
        if constexpr (std::is_same<Args, F32ArgsTwo>::value) {
            const bool second = k0 >= g.kp;
            const int at = second ? k0 - g.kp : k0;
            const int lim = min(second ? k_lim - g.kp : k_lim, g.k1);
            TA::issue(second ? g.A2 : g.A, second ? g.lda2 : g.lda, m0, g.m, at, lim, base, wave,
                      lane);
            TB::issue(second ? g.B2 : g.B, second ? g.ldb2 : g.ldb, n0, g.n, at, lim,
                      base + A_BYTES, wave, lane);
        } else if constexpr (std::is_same<Args, F32ArgsPad>::value) {
            TA::issue(g.A, g.lda, m0, g.m_load, k0, k_lim, base, wave, lane);
            TB::issue(g.B, g.ldb, n0, g.n_load, k0, k_lim, base + A_BYTES, wave, lane);
        } else {
            TA::issue(g.A, g.lda, m0, g.m, k0, k_lim, base, wave, lane);
            TB::issue(g.B, g.ldb, n0, g.n, k0, k_lim, base + A_BYTES, wave, lane);
        }
    };
    f32x16 acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    if (nkb > 0) issue(0, 0);
    for (int it = 0; it < nkb; ++it) {
        // this thread's loads of step `it` are done, then everyone's; the
        // stage read last step is free to refill
        wait_vm<0>();
        __syncthreads();
        if (it + 1 < nkb) issue(it + 1, (it + 1) & 1);
        const char *cur = smem + (it & 1) * STAGE;
#pragma unroll
        for (int j = 0; j < FK / 8; ++j) {
            f32x4 a[MI], b[NI];
#pragma unroll
            for (int i = 0; i < MI; ++i) a[i] = TA::frag(cur, wm * WM + i * 32, j, lane);
#pragma unroll
            for (int i = 0; i < NI; ++i) b[i] = TB::frag(cur + A_BYTES, wn * WN + i * 32, j, lane);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int jj = 0; jj < NI; ++jj)
                        acc[i][jj] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i][e], b[jj][e],
                                                                          acc[i][jj], 0, 0, 0);
        }
    }

    // lane holds column lane % 32 of a 32 x 32 block, register r row
    // 8 (r / 4) + 4 (lane / 32) + r % 4
    const bool partial = ACCUM != ACC_ALL && g.splits > 1;
    const bool add = ACCUM == ACC_ALL || (ACCUM == ACC_SOME && g.accumulate && !partial);
    const int64_t ldo = partial ? sbpi::partial_ld(g.n) : g.ldc;
    float *const out = partial ? g.ws + (size_t)split * (size_t)g.m * (size_t)ldo : g.C;
    const __amdgpu_buffer_rsrc_t pr = part_rsrc(out);
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int col = n0 + wn * WN + j * 32 + (lane & 31);
            const int rbase = m0 + wm * WM + i * 32 + 4 * (lane >> 5);
            if (col >= g.n) continue;
            if constexpr (ACCUM != ACC_NONE) {
                if (add) {
                    // opaque: shared with the plain stores, 47 more registers hold
                    // row addresses in the pair's 64 x 64 form, four workgroups a
                    // unit for five
                    int rb = rbase;
                    asm volatile("" : "+v"(rb));
                    add_block(out, ldo, rb, col, m0 + wm * WM + i * 32, g.m, acc[i][j]);
                    continue;
                }
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = rbase + 8 * (r >> 2) + (r & 3);
                if (row >= g.m) continue;
                if (partial) st_part(pr, (int64_t)row * ldo + col, acc[i][j][r]);
                else st_nt(out + (int64_t)row * ldo + col, acc[i][j][r]);
            }
        }
}

// Two workgroups of 128 x 128 tiles per CU (64 KB of LDS each), four or five of 64 x 64 ones.
template <int BM, bool A_KMAJ, bool B_KMAJ, int V, int ACCUM>
__global__ __launch_bounds__(256, BM == 64 ? 4 : 2) void gemm_f32_mfma_kernel(F32Args g) {
    __shared__ __attribute__((aligned(1024))) char smem[4 * BM * FK * 4];
    const int total = g.tiles_m * g.tiles_n * g.splits;
    f32_tile_body<BM, BM, A_KMAJ, B_KMAJ, V, ACCUM>(g, remap_xcd(blockIdx.x, total), smem);
}

// Both backward products of one linear in one launch, the product with the
// longer work items first (as gemm_bf16_dma_bwd_kernel): a product of 256 tiles
// alone puts one workgroup on each CU, which then waits for every load.
template <int BM, int V, int ACCUM>
__global__ __launch_bounds__(256, BM == 64 ? 4 : 2) void gemm_f32_mfma_bwd_kernel(
    F32Args gd, F32Args gw, int data_first) {
    __shared__ __attribute__((aligned(1024))) char smem[4 * BM * FK * 4];
    const int wd = gd.tiles_m * gd.tiles_n * gd.splits;
    const int ww = gw.tiles_m * gw.tiles_n * gw.splits;
    const int b = blockIdx.x;
    if (data_first ? b < wd : b >= ww)
        f32_tile_body<BM, BM, true, true, V, ACCUM>(gd, remap_xcd(data_first ? b : b - ww, wd),
                                                    smem);
    else
        f32_tile_body<BM, BM, false, false, V, ACCUM>(gw, remap_xcd(data_first ? b - wd : b, ww),
                                                      smem);
}

// The three products of the gated block's backward pass (gated_bwd.hip): dX over both pairs,
// dWg and dWu, the longer items first. (513 x 1000 x 1375: two launches of a pair each, dX added
// to itself, 106 us; this one by the same 4-byte loads 94.)
template <int BM, int V, int ACCUM>
__global__ __launch_bounds__(256, BM == 64 ? 4 : 2) void gemm_f32_gated_bwd_kernel(
    F32ArgsTwo gd, F32ArgsPad gw, F32ArgsPad gu, int data_first) {
    __shared__ __attribute__((aligned(1024))) char smem[4 * BM * FK * 4];
    const int wd = gd.tiles_m * gd.tiles_n * gd.splits;
    const int ww = gw.tiles_m * gw.tiles_n * gw.splits;
    const int b = blockIdx.x;
    if (data_first ? b < wd : b >= 2 * ww) {
        f32_tile_body<BM, BM, true, true, V, ACCUM>(gd, remap_xcd(data_first ? b : b - 2 * ww, wd),
                                                    smem);
    } else {
        const int L = remap_xcd(data_first ? b - wd : b, 2 * ww);
        const bool up = L >= ww;
        F32ArgsPad g = gw;
        g.B = up ? gu.B : gw.B;
        g.ldb = up ? gu.ldb : gw.ldb;
        g.C = up ? gu.C : gw.C;
        g.ldc = up ? gu.ldc : gw.ldc;
        g.ws = up ? gu.ws : gw.ws;
        g.accumulate = up ? gu.accumulate : gw.accumulate;
        f32_tile_body<BM, BM, false, false, V, ACCUM>(g, up ? L - ww : L, smem);
    }
}

// Copies of matrices whose rows do not allow 16-byte loads into ones that do, rows padded
// with zeros to whole chunks.
struct PackArgs {
    int32_t n;
    struct {
        const float *src;
        float *dst;
        int64_t ld_src, ld_dst, first;   // first: of its row parts of 1024 columns
        int32_t cols, parts;
    } m[5];
    int64_t total;
};
__global__ __launch_bounds__(256) void gated_pack_kernel(PackArgs a) {
    for (int64_t id = blockIdx.x; id < a.total; id += gridDim.x) {
        int i = 0;
        while (i + 1 < a.n && id >= a.m[i + 1].first) ++i;
        const int64_t at = id - a.m[i].first, row = at / a.m[i].parts;
        const int col = (int)(at % a.m[i].parts) * 1024 + threadIdx.x;
        const float *const src = a.m[i].src + row * a.m[i].ld_src;
        float *const dst = a.m[i].dst + row * a.m[i].ld_dst;
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            x[e] = col + 256 * e < a.m[i].cols ? src[col + 256 * e] : 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + 256 * e < a.m[i].ld_dst) dst[col + 256 * e] = x[e];
    }
}

// Plain LDS-tiled FMA kernel (leading dimensions beyond 2^21, shortest reductions): 64 x 64
// output tile, reduction step 16, 256 threads each owning a 4 x 4 strided
// sub-block.
constexpr int F_BM = 64, F_BN = 64, F_BK = 16;

template <bool A_KMAJ, bool B_KMAJ>
__global__ __launch_bounds__(256) void gemm_f32_kernel(F32Args g) {
    __shared__ float As[F_BK][F_BM + 1];
    __shared__ float Bs[F_BK][F_BN + 1];
    const int tid = threadIdx.x;
    const int tx = tid & 15, ty = tid >> 4;
    const int tm = blockIdx.x / g.tiles_n, tn = blockIdx.x % g.tiles_n;
    const int m0 = tm * F_BM, n0 = tn * F_BN;
    float acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;

    for (int k0 = 0; k0 < g.k; k0 += F_BK) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int e = tid + 256 * q;
            int i, kk;
            if (A_KMAJ) { i = e / F_BK; kk = e % F_BK; } else { kk = e / F_BM; i = e % F_BM; }
            const int gi = m0 + i, gk = k0 + kk;
            float v = 0.f;
            if (gi < g.m && gk < g.k)
                v = A_KMAJ ? g.A[(int64_t)gi * g.lda + gk] : g.A[(int64_t)gk * g.lda + gi];
            As[kk][i] = v;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int e = tid + 256 * q;
            int j, kk;
            if (B_KMAJ) { j = e / F_BK; kk = e % F_BK; } else { kk = e / F_BN; j = e % F_BN; }
            const int gj = n0 + j, gk = k0 + kk;
            float v = 0.f;
            if (gj < g.n && gk < g.k)
                v = B_KMAJ ? g.B[(int64_t)gj * g.ldb + gk] : g.B[(int64_t)gk * g.ldb + gj];
            Bs[kk][j] = v;
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < F_BK; ++kk) {
            float a[4], b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = As[kk][ty + 16 * i];
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = Bs[kk][tx + 16 * j];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_fmaf(a[i], b[j], acc[i][j]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = m0 + ty + 16 * i;
        if (row >= g.m) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int col = n0 + tx + 16 * j;
            if (col >= g.n) continue;
            float *c = g.C + (int64_t)row * g.ldc + col;
            *c = g.accumulate ? *c + acc[i][j] : acc[i][j];
        }
    }
}

}  // namespace sbpk

namespace sbpi {

hipError_t launch_bf16_fwd(const Gemm &, const Plan &, float *, hipStream_t);
hipError_t launch_bf16_bwd_data(const Gemm &, const Plan &, float *, hipStream_t);
hipError_t launch_bf16_bwd_weight(const Gemm &, const Plan &, float *, hipStream_t);

hipError_t launch_bf16(const Gemm &g, const Plan &p, float *ws, hipStream_t s) {
    switch (g.orient) {
        case OR_FWD: return launch_bf16_fwd(g, p, ws, s);
        case OR_BWD_DATA: return launch_bf16_bwd_data(g, p, ws, s);
        case OR_BWD_WEIGHT: return launch_bf16_bwd_weight(g, p, ws, s);
    }
    return hipErrorInvalidValue;
}

static sbpk::F32Args f32_args(const Gemm &g, const Plan &p, float *ws) {
    sbpk::F32Args a;
    a.A = static_cast<const float *>(g.A);
    a.B = static_cast<const float *>(g.B);
    a.C = static_cast<float *>(g.C);
    a.lda = g.lda;
    a.ldb = g.ldb;
    a.ldc = g.ldc;
    a.m = (int32_t)g.m;
    a.n = (int32_t)g.n;
    a.k = (int32_t)g.k;
    a.tiles_m = (int32_t)((g.m + p.bm - 1) / p.bm);
    a.tiles_n = (int32_t)((g.n + p.bn - 1) / p.bn);
    a.splits = p.splits;
    a.kchunk = p.kblk_per_split * p.bk;
    a.ws = ws;
    a.accumulate = g.accumulate;
    return a;
}

template <bool AK, bool BK_>
static hipError_t launch_f32_orient(const Gemm &g, const Plan &p, float *ws, hipStream_t s) {
    const char *tf[2] = {"false", "true"};
    char name[96];
    const sbpk::F32Args a = f32_args(g, p, ws);
    const dim3 grid((unsigned)(a.tiles_m * a.tiles_n * a.splits));
    if (!p.dma) {
        if (profiling()) snprintf(name, sizeof(name), "gemm_f32_kernel<%s, %s>", tf[AK], tf[BK_]);
        return launch_kernel(sbpk::gemm_f32_kernel<AK, BK_>, name, grid, dim3(256), s, a);
    }
    const bool v4 = f32_vec4(g), add = g.accumulate && p.splits == 1;
    hipError_t e = hipErrorInvalidValue;
#define SBP_F32_TILE(BM_, V_, ACC_)                                                           \
    if (p.bm == BM_ && v4 == (V_ == 4) && add == (ACC_ == sbpk::ACC_ALL)) {                   \
        if (profiling())                                                                     \
            snprintf(name, sizeof(name), "gemm_f32_mfma_kernel<%d, %s, %s, %d, %d>", BM_,    \
                     tf[AK], tf[BK_], V_, ACC_);                                             \
        e = launch_kernel(sbpk::gemm_f32_mfma_kernel<BM_, AK, BK_, V_, ACC_>, name, grid,    \
                          dim3(256), s, a);                                                  \
    }
    SBP_F32_TILE(128, 4, sbpk::ACC_NONE)
    SBP_F32_TILE(128, 1, sbpk::ACC_NONE)
    SBP_F32_TILE(64, 4, sbpk::ACC_NONE)
    SBP_F32_TILE(64, 1, sbpk::ACC_NONE)
    SBP_F32_TILE(128, 4, sbpk::ACC_ALL)
    SBP_F32_TILE(128, 1, sbpk::ACC_ALL)
    SBP_F32_TILE(64, 4, sbpk::ACC_ALL)
    SBP_F32_TILE(64, 1, sbpk::ACC_ALL)
#undef SBP_F32_TILE
    if (e != hipSuccess || p.splits == 1) return e;
    return launch_split_reduce(g, p.splits, ws, s);
}

hipError_t launch_f32(const Gemm &g, const Plan &p, float *ws, hipStream_t s) {
    switch (g.orient) {
        case OR_FWD: return launch_f32_orient<true, false>(g, p, ws, s);
        case OR_BWD_DATA: return launch_f32_orient<true, true>(g, p, ws, s);
        case OR_BWD_WEIGHT: return launch_f32_orient<false, false>(g, p, ws, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_f32_bwd_group(const Gemm &gd, const Plan &pd, const Gemm &gw, const Plan &pw,
                                float *ws, hipStream_t s) {
    if (!pd.dma || !pw.dma || pd.bm != pw.bm) return hipErrorInvalidValue;
    char name[96];
    float *const ws_w = ws + plan_ws_floats(gd, pd);
    const sbpk::F32Args d = f32_args(gd, pd, ws), w = f32_args(gw, pw, ws_w);
    const dim3 grid((unsigned)(d.tiles_m * d.tiles_n * d.splits + w.tiles_m * w.tiles_n * w.splits));
    const int data_first = pd.kblk_per_split >= pw.kblk_per_split;
    const bool v4 = f32_vec4(gd) && f32_vec4(gw);
    const bool add = (gd.accumulate && pd.splits == 1) || (gw.accumulate && pw.splits == 1);
    hipError_t e = hipErrorInvalidValue;
#define SBP_F32_PAIR(BM_, V_, ACC_)                                                          \
    if (pd.bm == BM_ && v4 == (V_ == 4) && add == (ACC_ == sbpk::ACC_SOME)) {                \
        if (profiling())                                                                     \
            snprintf(name, sizeof(name), "gemm_f32_mfma_bwd_kernel<%d, %d, %d>", BM_, V_,    \
                     ACC_);                                                                  \
        e = launch_kernel(sbpk::gemm_f32_mfma_bwd_kernel<BM_, V_, ACC_>, name, grid,         \
                          dim3(256), s, d, w, data_first);                                   \
    }
    SBP_F32_PAIR(128, 4, sbpk::ACC_NONE)
    SBP_F32_PAIR(128, 1, sbpk::ACC_NONE)
    SBP_F32_PAIR(64, 4, sbpk::ACC_NONE)
    SBP_F32_PAIR(64, 1, sbpk::ACC_NONE)
    SBP_F32_PAIR(128, 4, sbpk::ACC_SOME)
    SBP_F32_PAIR(128, 1, sbpk::ACC_SOME)
    SBP_F32_PAIR(64, 4, sbpk::ACC_SOME)
    SBP_F32_PAIR(64, 1, sbpk::ACC_SOME)
#undef SBP_F32_PAIR
    if (e != hipSuccess) return e;
    if (pd.splits > 1 && pw.splits > 1)
        return launch_split_reduce_pair(gd, pd.splits, ws, gw, pw.splits, ws_w, s);
    if (pd.splits > 1) return launch_split_reduce(gd, pd.splits, ws, s);
    if (pw.splits > 1) return launch_split_reduce(gw, pw.splits, ws_w, s);
    return hipSuccess;
}

static Gemm gated_product(int orient, const Mat &a, const Mat &b, const Mat &c, int64_t m, int64_t n,
                          int64_t k, int acc, const Gated &g) {
    Gemm o{orient, DT_F32, DT_F32, a.p, a.ld, b.p, b.ld, c.p, c.ld, m, n, k};
    o.accumulate = acc;
    o.ws_floats = g.ws_floats;
    return o;
}

hipError_t launch_gated_products_f32(const Gated &c, hipStream_t s, bool *taken) {
    *taken = false;
    if (c.m == 0 || c.n == 0 || c.k == 0) return hipSuccess;
    const int64_t n4 = (c.n + 3) & ~int64_t(3), k4 = (c.k + 3) & ~int64_t(3);
    const int64_t kp = (c.n + 31) / 32 * 32;
    if (2 * kp + 32 > INT32_MAX || n4 + 1024 > INT32_MAX || k4 + 1024 > INT32_MAX) return hipSuccess;
    constexpr int64_t kMaxLd = int64_t(1) << 21;
    for (const Mat *x : {&c.x, &c.dg, &c.du, &c.wg, &c.wu})
        if (x->ld >= kMaxLd) return hipSuccess;
    // matrices in the way of 16-byte loads
    Gated a = c;
    const struct {
        Mat *m;
        int64_t rows, cols;
    } all[5] = {{&a.x, c.m, c.k}, {&a.wg, c.k, c.n}, {&a.wu, c.k, c.n}, {&a.dg, c.m, c.n}, {&a.du, c.m, c.n}};
    sbpk::PackArgs pack{};
    size_t packed = 0;
    for (const auto &x : all) {
        const bool rows16 = reinterpret_cast<uintptr_t>(x.m->p) % 16 == 0 && x.m->ld % 4 == 0;
        if (rows16 && x.cols % 4 == 0) continue;
        auto &p = pack.m[pack.n++];
        p.src = static_cast<const float *>(x.m->p);
        p.cols = (int32_t)x.cols;
        p.ld_src = x.m->ld;
        p.ld_dst = (x.cols + 3) & ~int64_t(3);
        p.dst = c.ws + packed;
        p.parts = (int32_t)((p.ld_dst + 1023) / 1024);
        p.first = pack.total;
        pack.total += x.rows * p.parts;
        packed += (size_t)(x.rows * p.ld_dst);
        x.m->p = p.dst;
        x.m->ld = p.ld_dst;
    }
    Gemm gd, gw;
    auto products = [&]() {
        gd = gated_product(OR_BWD_DATA, a.dg, a.wg, a.dx, a.m, a.k, 2 * kp, a.dx_acc, a);
        gw = gated_product(OR_BWD_WEIGHT, a.x, a.dg, a.dwg, a.k, a.n, a.m, a.dwg_acc, a);
    };
    // as they are by 4-byte loads, or by 16-byte loads after the copies (read and written
    // at about 4 TB/s by a launch of their own), if the workspace holds them
    Plan pd, pw;
    double time = 1e300;
    bool vec = false;
    if (packed <= c.ws_floats) {
        a.ws = c.ws + packed;
        a.ws_floats = c.ws_floats - packed;
        products();
        vec = plan_f32_gated_bwd(gd, gw, true, &pd, &pw, &time);
        if (packed) time += 4.0 + packed * 8 / 4e6;
    }
    if (pack.n) {
        const Gated copies = a;
        a = c;
        products();
        Plan qd, qw;
        double t;
        if (plan_f32_gated_bwd(gd, gw, false, &qd, &qw, &t) && (!vec || t <= time)) {
            vec = false;
            pd = qd;
            pw = qw;
        } else if (vec) {
            a = copies;
            products();
        } else {
            return hipSuccess;
        }
    } else if (!vec) {
        return hipSuccess;
    }
    hipError_t e = hipSuccess;
    if (vec && pack.n) {
        e = launch_kernel(sbpk::gated_pack_kernel, "gated_pack_kernel",
                          dim3((unsigned)std::min<int64_t>(pack.total, 1 << 20)), dim3(256), s, pack);
        if (e != hipSuccess) return e;
    }
    const bool v4 = vec;
    Gemm gu = gated_product(OR_BWD_WEIGHT, a.x, a.du, a.dwu, a.k, a.n, a.m, a.dwu_acc, a);
    const size_t part_d = plan_ws_floats(gd, pd), part_w = plan_ws_floats(gw, pw);
    float *const ws_g = a.ws + part_d, *const ws_u = ws_g + part_w;
    sbpk::F32ArgsTwo d;
    static_cast<sbpk::F32Args &>(d) = f32_args(gd, pd, a.ws);
    d.A2 = static_cast<const float *>(a.du.p);
    d.B2 = static_cast<const float *>(a.wu.p);
    d.lda2 = a.du.ld;
    d.ldb2 = a.wu.ld;
    d.k1 = (int32_t)(vec ? n4 : a.n);
    d.kp = (int32_t)kp;
    d.k = (int32_t)(kp + d.k1);
    sbpk::F32ArgsPad g, u;
    static_cast<sbpk::F32Args &>(g) = f32_args(gw, pw, ws_g);
    static_cast<sbpk::F32Args &>(u) = f32_args(gu, pw, ws_u);
    g.m_load = u.m_load = (int32_t)(vec ? k4 : a.k);
    g.n_load = u.n_load = (int32_t)(vec ? n4 : a.n);
    const dim3 grid((unsigned)(d.tiles_m * d.tiles_n * d.splits +
                               2 * g.tiles_m * g.tiles_n * g.splits));
    const int data_first = pd.kblk_per_split >= pw.kblk_per_split;
    const bool add = (a.dx_acc && pd.splits == 1) || ((a.dwg_acc || a.dwu_acc) && pw.splits == 1);
    char name[96];
    e = hipErrorInvalidValue;
#define SBP_F32_GATED(BM_, V_, ACC_)                                                         \
    if (pd.bm == BM_ && v4 == (V_ == 4) && add == (ACC_ == sbpk::ACC_SOME)) {                \
        if (profiling())                                                                     \
            snprintf(name, sizeof(name), "gemm_f32_gated_bwd_kernel<%d, %d, %d>", BM_, V_,   \
                     ACC_);                                                                  \
        e = launch_kernel(sbpk::gemm_f32_gated_bwd_kernel<BM_, V_, ACC_>, name, grid,        \
                          dim3(256), s, d, g, u, data_first);                                \
    }
    SBP_F32_GATED(128, 4, sbpk::ACC_NONE)
    SBP_F32_GATED(128, 1, sbpk::ACC_NONE)
    SBP_F32_GATED(64, 4, sbpk::ACC_NONE)
    SBP_F32_GATED(64, 1, sbpk::ACC_NONE)
    SBP_F32_GATED(128, 4, sbpk::ACC_SOME)
    SBP_F32_GATED(128, 1, sbpk::ACC_SOME)
    SBP_F32_GATED(64, 4, sbpk::ACC_SOME)
    SBP_F32_GATED(64, 1, sbpk::ACC_SOME)
#undef SBP_F32_GATED
    *taken = true;
    if (e != hipSuccess) return e;
    if (pd.splits > 1) e = launch_split_reduce(gd, pd.splits, a.ws, s);
    if (e != hipSuccess || pw.splits == 1) return e;
    return launch_split_reduce_pair(gw, pw.splits, ws_g, gu, pw.splits, ws_u, s);
}

}  // namespace sbpi
