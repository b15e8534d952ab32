// gated_fwd.hip -- H = act(X Wg) * (X Wu) in one kernel (bf16).
//
// A workgroup owns a BM x BN tile of H and computes that tile of both projections:
// every reduction step brings one tile of X and one of each weight matrix to LDS, and
// a wave holds the sums of both for the same outputs, so act and the product are
// lane-local. It is the pipelined kernel of gemm_bf16_dma.h on a BM x 2 BN
// product (same loads, LDS layouts, fragment reads and tile order), and bounded by what
// bounds that; X is read once for both projections, and neither goes to memory unless
// the caller keeps them for the backward pass. H is made of the fp32 sums; G and U are
// rounded to bf16 as they are stored.
//
// Few tiles and a long reduction: it is split, fp32 partials of both projections go to the
// workspace, and a second kernel adds them in split order and applies the gate.
#include "gated.h"
#include "gemm_bf16_dma.h"
#include "profile.h"

namespace sbpk {

struct GatedArgs {
    const uint16_t *X, *Wg, *Wu;
    uint16_t *H, *G, *U;          // G, U may be NULL
    int64_t ldx, ldg_w, ldu_w, ldh, ldg, ldu;
    int32_t m, n, k;
    int32_t tiles_m, tiles_n, splits, kchunk;
    int32_t vec_h, vec_g, vec_u;  // rows allow 16-byte stores
    float *ws;                    // splits x (gate, up) slices of m x partial_ld(n)
};

template <int BM, int BN, int NS>
struct GatedStage {
    static constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128;   // 64-wide steps
    static constexpr int BYTES = A_BYTES + 2 * B_BYTES;
    static constexpr int LDS = NS * BYTES;
};

template <int ACT, int BM, int BN, int NS, int WGM, int WGN, bool REG>
__global__ __launch_bounds__(64 * WGM * WGN, (GatedStage<BM, BN, NS>::LDS > 81920 ? 1 : 2))
void gated_fwd_kernel(GatedArgs g) {
    using St = GatedStage<BM, BN, NS>;
    constexpr int NW = WGM * WGN, NT = 64 * NW;
    constexpr int WM = BM / WGM, WN = BN / WGN, MI = WM / 32, NI = WN / 32;
    using TA = KTileDma<BM, NW, 64>;
    using TB = MNTileDma<BN, NW, 64>;
    constexpr int LOADS = TA::PER_WAVE + 2 * TB::PER_WAVE;
    __shared__ __attribute__((aligned(1024))) char smem[St::LDS];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wm = wave / WGN, wn = wave % WGN;

    const int tiles = g.tiles_m * g.tiles_n;
    const int L = remap_xcd(blockIdx.x, tiles * g.splits);
    const int split = L / tiles, t = L % tiles;
    constexpr int GROUP = SBP_TILE_GROUP;
    const int first_m = t / (GROUP * g.tiles_n) * GROUP;
    const int gsize = min(g.tiles_m - first_m, GROUP);
    const int m0 = (first_m + (t % (GROUP * g.tiles_n)) % gsize) * BM;
    const int n0 = (t % (GROUP * g.tiles_n)) / gsize * BN;
    const int k_begin = split * g.kchunk, k_lim = min(g.k, k_begin + g.kchunk);
    const int nkb = max(0, (k_lim - k_begin + 63) / 64);

    f32x16 acc[2][MI][NI];
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[w][i][j][r] = 0.f;

    // Operands are read one reduction step of 16 ahead of their products (read right before
    // them, 25 us for 8192 x 1024 -> 512); between(i): what is written before products i.
    auto compute = [&](const char *cur, auto between) {
        bf16x8 a[2][MI], b[2][2][NI];
        auto read = [&](int ks) {
#pragma unroll
            for (int i = 0; i < MI; ++i) a[ks & 1][i] = TA::frag(cur, wm * WM + i * 32, ks, lane);
#pragma unroll
            for (int w = 0; w < 2; ++w)
#pragma unroll
                for (int j = 0; j < NI; ++j)
                    b[ks & 1][w][j] = TB::frag(cur + St::A_BYTES + w * St::B_BYTES, wn * WN + j * 32, ks, lane);
        };
        read(0);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            if (ks + 1 < 4) read(ks + 1);
            between(ks);
#pragma unroll
            for (int w = 0; w < 2; ++w)
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int j = 0; j < NI; ++j)
                        acc[w][i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                            a[ks & 1][i], b[ks & 1][w][j], acc[w][i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    if constexpr (REG) {
        // operands at any alignment: through registers, the next step's loads in
        // flight while a step computes
        static_assert(!REG || NS == 2, "register staging: two stages");
        using RA = RegTile<BM, NW, true>;
        using RB = RegTile<BN, NW, false>;
        typename RA::Regs va;
        typename RB::Regs vg, vu;
        auto load = [&](int it) {
            const int k0 = k_begin + it * 64;
            RA::load_edge(va, g.X, g.ldx, m0, g.m, k0, k_lim, tid);
            RB::load_edge(vg, g.Wg, g.ldg_w, n0, g.n, k0, k_lim, tid);
            RB::load_edge(vu, g.Wu, g.ldu_w, n0, g.n, k0, k_lim, tid);
        };
        auto fill = [&](int stage) {
            char *base = smem + stage * St::BYTES;
            RA::store(va, base, tid);
            RB::store(vg, base + St::A_BYTES, tid);
            RB::store(vu, base + St::A_BYTES + St::B_BYTES, tid);
        };
        if (nkb > 0) {
            load(0);
            fill(0);
        }
        for (int it = 0; it < nkb; ++it) {
            __syncthreads();
            if (it + 1 < nkb) load(it + 1);
            compute(smem + (it & 1) * St::BYTES, [](int) {});
            if (it + 1 < nkb) fill((it + 1) & 1);
        }
    } else {
        // A large tile alone on its unit spreads a step's loads over its products (8192 x 8192
        // -> 4096: 929 -> 888 us); of two workgroups, one's loads run beside the other's
        // products anyway (8192 x 1024 -> 512: 23.6 us at once, 25.7 spread), and small tiles
        // wait for them (one row, 1024 -> 4096: 9.8 and 10.7).
        constexpr bool SPREAD = St::LDS > 81920 && BM > 64;
        // the loads of step kb: of X, Wg or Wu (part 0 .. 2), or all (-1)
        auto issue = [&](int kb, int stage, int part) {
            char *base = smem + stage * St::BYTES;
            const int k0 = k_begin + kb * 64;
            if (part <= 0)
                TA::template issue<false>(g.X, g.ldx, m0, g.m, k0, k_lim, base, wave, lane);
            if (part < 0 || part == 1)
                TB::template issue<false>(g.Wg, g.ldg_w, n0, g.n, k0, k_lim, base + St::A_BYTES,
                                          wave, lane);
            if (part < 0 || part == 2)
                TB::template issue<false>(g.Wu, g.ldu_w, n0, g.n, k0, k_lim,
                                          base + St::A_BYTES + St::B_BYTES, wave, lane);
        };
#pragma unroll
        for (int s = 0; s < NS - 1; ++s)
            if (s < nkb) issue(s, s, -1);
        for (int it = 0; it < nkb; ++it) {
            wait_stages<NS - 2, LOADS>(min(NS - 2, nkb - 1 - it));
            __syncthreads();
            const bool more = it + NS - 1 < nkb;
            if (!SPREAD && more) issue(it + NS - 1, (it + NS - 1) % NS, -1);
            compute(smem + it % NS * St::BYTES, [&](int ks) {
                if (SPREAD && more) issue(it + NS - 1, (it + NS - 1) % NS, ks);
            });
        }
    }

    if (g.splits > 1) {
        const int ldw = (int)sbpi::partial_ld(g.n);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            float *out = g.ws + ((size_t)split * 2 + w) * (size_t)g.m * ldw;
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j) {
                    const int col = n0 + wn * WN + j * 32 + (lane & 31);
                    const int row0 = m0 + wm * WM + i * 32 + 4 * (lane >> 5);
                    if (col >= g.n) continue;
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int row = row0 + 8 * (r >> 2) + (r & 3);
                        if (row < g.m)
                            st_part(part_rsrc(out), (int64_t)row * ldw + col, acc[w][i][j][r]);
                    }
                }
        }
        return;
    }

    // H, then G and U if they are kept, through LDS as 16-byte row pieces
    constexpr int LD = StageRow<BN, BM, St::LDS>::LD;
    static_assert(BM * LD * 4 <= St::LDS, "output tile does not fit the pipeline's LDS");
    float *tile = reinterpret_cast<float *>(smem);
    auto put = [&](uint16_t *out, int64_t ld, bool vec, auto value) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    tile[(wm * WM + i * 32 + 4 * (lane >> 5) + 8 * (r >> 2) + (r & 3)) * LD +
                         wn * WN + j * 32 + (lane & 31)] = value(i, j, r);
        __syncthreads();
        store_staged<BM, BN, LD, NT, false>(tile, out, ld, g.m, g.n, m0, n0, vec, tid);
    };
    if (g.G) put(g.G, g.ldg, g.vec_g, [&](int i, int j, int r) { return acc[0][i][j][r]; });
    if (g.U) put(g.U, g.ldu, g.vec_u, [&](int i, int j, int r) { return acc[1][i][j][r]; });
    put(g.H, g.ldh, g.vec_h,
        [&](int i, int j, int r) { return act_of<ACT>(acc[0][i][j][r]) * acc[1][i][j][r]; });
}

// Adds the splits of both projections in split order and applies the gate. A thread
// owns 4 columns of a row.
template <int ACT>
__global__ __launch_bounds__(256) void gated_join_kernel(GatedArgs g) {
    const int groups = (g.n + 3) / 4;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= (int64_t)g.m * groups) return;
    const int row = (int)(id / groups), col = (int)(id % groups) * 4;
    const int64_t ldw = sbpi::partial_ld(g.n);
    const size_t slice = (size_t)g.m * ldw;
    const float *p = g.ws + (size_t)row * ldw + col;
    f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
#pragma unroll 4
    for (int s = 0; s < g.splits; ++s) {
        a += *reinterpret_cast<const f32x4 *>(p + (2 * s) * slice);
        b += *reinterpret_cast<const f32x4 *>(p + (2 * s + 1) * slice);
    }
    f32x4 h;
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = act_of<ACT>(a[e]) * b[e];
    auto put = [&](uint16_t *out, int64_t ld, bool vec, const f32x4 &v) {
        uint16_t *d = out + (int64_t)row * ld + col;
        if (vec && col + 4 <= g.n) {
            u32x2 w;
            w[0] = (uint32_t)f32_to_bf16_bits(v[0]) | (uint32_t)f32_to_bf16_bits(v[1]) << 16;
            w[1] = (uint32_t)f32_to_bf16_bits(v[2]) | (uint32_t)f32_to_bf16_bits(v[3]) << 16;
            *reinterpret_cast<u32x2 *>(d) = w;
            return;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < g.n) d[e] = f32_to_bf16_bits(v[e]);
    };
    put(g.H, g.ldh, g.vec_h, h);
    if (g.G) put(g.G, g.ldg, g.vec_g, a);
    if (g.U) put(g.U, g.ldu, g.vec_u, b);
}

// H = act(G) U of matrices in memory (the fp32 path, whose projections are two
// products of their own).
template <int ACT>
__global__ __launch_bounds__(256) void gated_act_kernel(const float *G, int64_t ldg, const float *U,
                                                        int64_t ldu, float *H, int64_t ldh, int m,
                                                        int n) {
    const int groups = (n + 3) / 4;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= (int64_t)m * groups) return;
    const int64_t row = id / groups;
    const int col = (int)(id % groups) * 4;
    const float *g = G + row * ldg + col, *u = U + row * ldu + col;
    float *h = H + row * ldh + col;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (col + e < n) h[e] = act_of<ACT>(g[e]) * u[e];
}

}  // namespace sbpk

namespace sbpi {

namespace {

bool aligned16(const Mat &x) {
    return reinterpret_cast<uintptr_t>(x.p) % 16 == 0 && x.ld % 8 == 0;
}

template <int BM, int BN, int NS, int WGM, int WGN, bool REG>
hipError_t launch_fwd(int act, const sbpk::GatedArgs &g, hipStream_t s) {
    char name[160];
    name[0] = 0;
    if (profiling())
        snprintf(name, sizeof(name), "gated_fwd_kernel<%d, %d, %d, %d, %d, %d, %s>", act, BM, BN, NS,
                 WGM, WGN, REG ? "true" : "false");
    const dim3 grid((unsigned)(g.tiles_m * g.tiles_n * g.splits)), block(64 * WGM * WGN);
    switch (act) {
        case ACT_SILU:
            return launch_kernel(sbpk::gated_fwd_kernel<ACT_SILU, BM, BN, NS, WGM, WGN, REG>, name,
                                 grid, block, s, g);
        case ACT_GELU:
            return launch_kernel(sbpk::gated_fwd_kernel<ACT_GELU, BM, BN, NS, WGM, WGN, REG>, name,
                                 grid, block, s, g);
        default:
            return launch_kernel(sbpk::gated_fwd_kernel<ACT_RELU, BM, BN, NS, WGM, WGN, REG>, name,
                                 grid, block, s, g);
    }
}

hipError_t launch_join(int act, const sbpk::GatedArgs &g, hipStream_t s) {
    const int64_t items = (int64_t)g.m * ((g.n + 3) / 4);
    const dim3 grid((unsigned)((items + 255) / 256)), block(256);
    switch (act) {
        case ACT_SILU:
            return launch_kernel(sbpk::gated_join_kernel<ACT_SILU>, "gated_join_kernel<0>", grid,
                                 block, s, g);
        case ACT_GELU:
            return launch_kernel(sbpk::gated_join_kernel<ACT_GELU>, "gated_join_kernel<1>", grid,
                                 block, s, g);
        default:
            return launch_kernel(sbpk::gated_join_kernel<ACT_RELU>, "gated_join_kernel<2>", grid,
                                 block, s, g);
    }
}

}  // namespace

hipError_t launch_gated_fwd(const Gated &a, hipStream_t s) {
    sbpk::GatedArgs g;
    g.X = static_cast<const uint16_t *>(a.x.p);
    g.Wg = static_cast<const uint16_t *>(a.wg.p);
    g.Wu = static_cast<const uint16_t *>(a.wu.p);
    g.H = static_cast<uint16_t *>(a.h.p);
    g.G = static_cast<uint16_t *>(a.g.p);
    g.U = static_cast<uint16_t *>(a.u.p);
    g.ldx = a.x.ld;
    g.ldg_w = a.wg.ld;
    g.ldu_w = a.wu.ld;
    g.ldh = a.h.ld;
    g.ldg = a.g.ld;
    g.ldu = a.u.ld;
    g.m = (int32_t)a.m;
    g.n = (int32_t)a.n;
    g.k = (int32_t)a.k;
    g.vec_h = aligned16(a.h);
    g.vec_g = aligned16(a.g);
    g.vec_u = aligned16(a.u);
    g.ws = a.ws;
    const bool dma = aligned16(a.x) && aligned16(a.wg) && aligned16(a.wu) && a.k % 8 == 0 &&
                     a.n % 8 == 0 && a.x.ld <= (int64_t(1) << 21) &&
                     a.wg.ld <= (int64_t(1) << 21) && a.wu.ld <= (int64_t(1) << 21);
    // tile and splits: whole waves of the largest tile that fills the chip (1024 x 4096 over
    // 1024: 512 tiles of 128 x 64, two a unit, 22.5 us; 256 of 128 x 128, one a unit in three
    // stages, 26)
    const int cus = device_cus();
    auto tiles = [&](int bm, int bn) {
        return ((a.m + bm - 1) / bm) * ((a.n + bn - 1) / bn);
    };
    const int tile = dma && tiles(256, 128) >= cus ? 0 : tiles(128, 64) >= cus ? 1 : 2;
    const int bm = tile == 0 ? 256 : tile == 1 ? 128 : 64, bn = tile == 0 ? 128 : 64;
    g.tiles_m = (int32_t)((a.m + bm - 1) / bm);
    g.tiles_n = (int32_t)((a.n + bn - 1) / bn);
    const int64_t kb = (a.k + 63) / 64, nt = (int64_t)g.tiles_m * g.tiles_n;
    const size_t room = a.ws_floats < WS_FLOATS_PREFERRED ? a.ws_floats : WS_FLOATS_PREFERRED;
    const size_t slice = 2 * (size_t)a.m * (size_t)partial_ld(a.n);
    // Reductions of more than 1024 are split while workgroups are few (one row, 2048 -> 4096: 17.2 us
    // in two launches, 19.9 whole; 64 rows, 4096 -> 512: 13.3 and 37.4); shorter ones would
    // only gain what the second launch takes (1024 -> 4096: 11.1 us each way in a graph, 13.6
    // and 10.9 called one by one, when both were measured).
    int64_t splits = 1;
    const int slots = tile == 0 ? cus : 2 * cus;   // workgroups at a time
    while (kb > 16 && nt * splits * 2 <= slots && kb / (splits * 2) >= 2 && slice * splits * 2 <= room)
        splits *= 2;
    const int64_t per = kb ? (kb + splits - 1) / splits : 1;
    g.kchunk = (int32_t)(per * 64);
    g.splits = kb ? (int32_t)((kb + per - 1) / per) : 1;
    hipError_t e;
    if (dma)
        e = tile == 0   ? launch_fwd<256, 128, 2, 2, 4, false>(a.act, g, s)
            : tile == 1 ? launch_fwd<128, 64, 2, 2, 2, false>(a.act, g, s)
                        : launch_fwd<64, 64, 4, 2, 2, false>(a.act, g, s);
    else
        e = tile == 1 ? launch_fwd<128, 64, 2, 2, 2, true>(a.act, g, s)
                      : launch_fwd<64, 64, 2, 2, 2, true>(a.act, g, s);
    if (e != hipSuccess || g.splits == 1) return e;
    return launch_join(a.act, g, s);
}

hipError_t launch_gated_act(const Gated &a, hipStream_t s) {
    const int64_t items = a.m * ((a.n + 3) / 4);
    const dim3 grid((unsigned)((items + 255) / 256)), block(256);
    auto go = [&](auto kernel, const char *name) {
        return launch_kernel(kernel, name, grid, block, s, static_cast<const float *>(a.g.p), a.g.ld,
                             static_cast<const float *>(a.u.p), a.u.ld,
                             static_cast<float *>(a.h.p), a.h.ld, (int)a.m, (int)a.n);
    };
    switch (a.act) {
        case ACT_SILU: return go(sbpk::gated_act_kernel<ACT_SILU>, "gated_act_kernel<0>");
        case ACT_GELU: return go(sbpk::gated_act_kernel<ACT_GELU>, "gated_act_kernel<1>");
        default: return go(sbpk::gated_act_kernel<ACT_RELU>, "gated_act_kernel<2>");
    }
}

}  // namespace sbpi
