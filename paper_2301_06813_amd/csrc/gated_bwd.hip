// gated_bwd.hip -- backward pass of the gated block.
//
// First dG = dH U act'(G) and dU = dH act(G), one pass over five matrices, bound by
// memory. Then the three products dX = dG Wg^T + dU Wu^T, dWg = X^T dG and dWu = X^T dU in
// one grid of the tiles of gemm_bf16_dma.h: dX reduces over both pairs of operands in turn
// (GemmArgsTwo), so its sum is rounded once; dWg and dWu are the two items of a batch that
// shares X. The longer items are dispatched first and the others fill the units behind
// them. dG and dU are rounded to bf16 as operands of the matrix cores.
#include <algorithm>
#include <type_traits>

#include "gated.h"
#include "gated_products.h"
#include "gemm_bf16_dma.h"
#include "profile.h"

namespace sbpk {

struct GradArgs {
    const void *dH, *G, *U;
    void *dG, *dU;
    int64_t ldh, ldg, ldu, ldo_g, ldo_u;
    int32_t m, n;
};

// Rows that allow it: 8 consecutive columns of a row per thread, in 16-byte accesses. Others
// (ROWS false): 4 columns of a row, 256 apart, an element a lane and access, so that a
// wave's addresses are side by side all the same.
template <int ACT, bool F32, bool ROWS>
__global__ __launch_bounds__(256) void gated_grad_kernel(GradArgs a) {
    if constexpr (!ROWS) {
        using T = std::conditional_t<F32, float, uint16_t>;
        const int parts = (a.n + 1023) / 1024;
        auto value = [](T x) {
            if constexpr (F32) return x;
            else return __builtin_bit_cast(float, (uint32_t)x << 16);
        };
        auto rounded = [](float x) {
            if constexpr (F32) return x;
            else return f32_to_bf16_bits(x);
        };
        for (int64_t id = blockIdx.x; id < (int64_t)a.m * parts; id += gridDim.x) {
            const int64_t row = id / parts;
            const int col = (int)(id % parts) * 1024 + threadIdx.x;
            const T *dh = static_cast<const T *>(a.dH) + row * a.ldh,
                    *gp = static_cast<const T *>(a.G) + row * a.ldg,
                    *up = static_cast<const T *>(a.U) + row * a.ldu;
            T h[4], g[4], u[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int at = min(col + 256 * e, a.n - 1);
                h[e] = dh[at];
                g[e] = gp[at];
                u[e] = up[at];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int at = col + 256 * e;
                if (at >= a.n) continue;
                float y, d;
                act_grad<ACT>(value(g[e]), &y, &d);
                static_cast<T *>(a.dG)[row * a.ldo_g + at] = rounded(value(h[e]) * value(u[e]) * d);
                static_cast<T *>(a.dU)[row * a.ldo_u + at] = rounded(value(h[e]) * y);
            }
        }
    } else {
        const int groups = (a.n + 7) / 8;
        const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
        if (id >= (int64_t)a.m * groups) return;
        const int64_t row = id / groups;
        const int col = (int)(id % groups) * 8;
        const int left = a.n - col;
        float h[8], g[8], u[8];
        auto get = [&](const void *p, int64_t ld, float *x) {
            const int64_t at = row * ld + col;
            if constexpr (F32) {
                const float *q = static_cast<const float *>(p) + at;
                if (left >= 8) {
                    const f32x4 v = *reinterpret_cast<const f32x4 *>(q),
                                w = *reinterpret_cast<const f32x4 *>(q + 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[e] = v[e];
                        x[4 + e] = w[e];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = e < left ? q[e] : 0.f;
                }
            } else {
                const uint16_t *q = static_cast<const uint16_t *>(p) + at;
                const u32x4 v = left >= 8 ? *reinterpret_cast<const u32x4 *>(q)
                                          : ld16_tail(q - col, col, a.n);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[2 * e] = __builtin_bit_cast(float, v[e] << 16);
                    x[2 * e + 1] = __builtin_bit_cast(float, v[e] & 0xffff0000u);
                }
            }
        };
        get(a.dH, a.ldh, h);
        get(a.G, a.ldg, g);
        get(a.U, a.ldu, u);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float y, d;
            act_grad<ACT>(g[e], &y, &d);
            g[e] = h[e] * u[e] * d;
            u[e] = h[e] * y;
        }
        auto put = [&](void *p, int64_t ld, const float *x) {
            const int64_t at = row * ld + col;
            if constexpr (F32) {
                float *q = static_cast<float *>(p) + at;
                if (left >= 8) {
                    *reinterpret_cast<f32x4 *>(q) = f32x4{x[0], x[1], x[2], x[3]};
                    *reinterpret_cast<f32x4 *>(q + 4) = f32x4{x[4], x[5], x[6], x[7]};
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (e < left) q[e] = x[e];
                }
            } else {
                uint16_t *q = static_cast<uint16_t *>(p) + at;
                if (left >= 8) {
                    u32x4 v;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        v[e] = (uint32_t)f32_to_bf16_bits(x[2 * e]) |
                               (uint32_t)f32_to_bf16_bits(x[2 * e + 1]) << 16;
                    *reinterpret_cast<u32x4 *>(q) = v;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (e < left) q[e] = f32_to_bf16_bits(x[e]);
                }
            }
        };
        put(a.dG, a.ldo_g, g);
        put(a.dU, a.ldo_u, u);
    }
}

}  // namespace sbpk

namespace sbpi {

hipError_t launch_gated_grad(const Gated &a, hipStream_t s) {
    const bool f32 = a.dtype == DT_F32;
    sbpk::GradArgs g{a.dh.p, a.g.p,  a.u.p,  a.dg.p,       a.du.p,       a.dh.ld, a.g.ld,
                     a.u.ld, a.dg.ld, a.du.ld, (int32_t)a.m, (int32_t)a.n};
    bool rows = true;            // every row allows 16-byte accesses
    for (const Mat *x : {&a.dh, &a.g, &a.u, &a.dg, &a.du})
        if (reinterpret_cast<uintptr_t>(x->p) % 16 || x->ld % (f32 ? 4 : 8)) rows = false;
    if (a.m == 0 || a.n == 0) return hipSuccess;
    const int64_t blocks = rows ? (a.m * ((a.n + 7) / 8) + 255) / 256
                                : std::min<int64_t>(a.m * ((a.n + 1023) / 1024), 1 << 20);
    const dim3 grid((unsigned)blocks), block(256);
#define SBP_GRAD(ACT_, F32_, ROWS_)                                                             \
    if (a.act == ACT_ && f32 == F32_ && rows == ROWS_)                                          \
        return launch_kernel(sbpk::gated_grad_kernel<ACT_, F32_, ROWS_>,                        \
                             "gated_grad_kernel<" #ACT_ ", " #F32_ ", " #ROWS_ ">", grid, block, s, g);
#define SBP_GRAD4(ACT_)                                                                         \
    SBP_GRAD(ACT_, false, true) SBP_GRAD(ACT_, true, true) SBP_GRAD(ACT_, false, false)         \
    SBP_GRAD(ACT_, true, false)
    SBP_GRAD4(ACT_SILU)
    SBP_GRAD4(ACT_GELU)
    SBP_GRAD4(ACT_RELU)
#undef SBP_GRAD4
#undef SBP_GRAD
    return hipErrorInvalidValue;
}

namespace {

// Kernel arguments of m x n outputs over k, without operands.
sbpk::GemmArgsTwo product_args(const Plan &p, int64_t m, int64_t n, int64_t k, const Mat &c,
                               bool f32, int acc, float *ws) {
    sbpk::GemmArgsTwo g{};
    g.C = c.p;
    g.ldc = c.ld;
    g.m = (int32_t)m;
    g.n = (int32_t)n;
    g.k = (int32_t)k;
    g.tiles_m = (int32_t)((m + p.bm - 1) / p.bm);
    g.tiles_n = (int32_t)((n + p.bn - 1) / p.bn);
    g.splits = p.splits;
    g.kchunk = p.kblk_per_split * 64;
    g.ws = ws;
    const bool c16 = reinterpret_cast<uintptr_t>(c.p) % 16 == 0;
    g.vec_c4 = c16 && c.ld % 4 == 0;
    g.vec_c8 = c16 && c.ld % 8 == 0;
    g.accumulate = acc && f32;
    g.nbatch = 1;
    g.heads = 1;
    return g;
}

bool rows16(const Mat &x) {
    return reinterpret_cast<uintptr_t>(x.p) % 16 == 0 && x.ld % 8 == 0 &&
           x.ld <= (int64_t(1) << 21);
}

Gemm reduced(const sbpk::GemmArgsTwo &g, const Mat &c, int dtype, int acc) {
    Gemm o{OR_FWD, DT_BF16, dtype, nullptr, 0, nullptr, 0, c.p, c.ld, g.m, g.n, g.k};
    o.accumulate = acc;
    return o;
}

}  // namespace

hipError_t launch_gated_products(const Gated &a, hipStream_t s) {
    if (a.k == 0 || (a.m == 0 && a.n == 0)) return hipSuccess;
    // dX reduces over n of both pairs, each rounded up to whole 128-wide stages
    const int64_t kp = (a.n + 127) / 128 * 128;
    const bool dma = rows16(a.x) && rows16(a.wg) && rows16(a.wu) && rows16(a.dg) && rows16(a.du) &&
                     a.k % 8 == 0 && a.n % 8 == 0 && a.dg.ld == a.du.ld && a.wg.ld == a.wu.ld;
    const bool dw_acc = a.dwg_acc || a.dwu_acc;
    Gemm gd{OR_BWD_DATA, DT_BF16, a.dx_dtype, nullptr, 0, nullptr, 0, nullptr, 0, a.m, a.k, 2 * kp};
    Gemm gw{OR_BWD_WEIGHT, DT_BF16, a.dw_dtype, nullptr, 0, nullptr, 0, nullptr, 0, a.k, a.n, a.m};
    gd.accumulate = a.dx_acc;
    gw.accumulate = dw_acc;
    gw.batches = 2;
    gd.ws_floats = gw.ws_floats = a.ws_floats;
    ProductsLaunch l;
    Plan pw;
    plan_bf16_gated_bwd(gd, gw, dma, &l.p, &pw);
    const Plan &pd = l.p;
    const size_t slice_d = (size_t)a.m * (size_t)partial_ld(a.k);
    const size_t slice_w = (size_t)a.k * (size_t)partial_ld(a.n);
    float *const ws_w = a.ws + (pd.splits > 1 ? pd.splits * slice_d : 0);
    const bool d32 = a.dx_dtype == DT_F32, w32 = a.dw_dtype == DT_F32;
    l.d = product_args(pd, a.m, a.k, kp + a.n, a.dx, d32, a.dx_acc, a.ws);
    l.d.A = static_cast<const uint16_t *>(a.dg.p);
    l.d.B = static_cast<const uint16_t *>(a.wg.p);
    l.d.A2 = static_cast<const uint16_t *>(a.du.p);
    l.d.B2 = static_cast<const uint16_t *>(a.wu.p);
    l.d.lda = a.dg.ld;
    l.d.ldb = a.wg.ld;
    l.d.lda2 = a.du.ld;
    l.d.ldb2 = a.wu.ld;
    l.d.k1 = (int32_t)a.n;
    l.d.kp = (int32_t)kp;
    // dWg and dWu as a batch of two when their rows and their operands' agree (a batch
    // has one stride of each), else as two launches
    const bool batch = a.dg.ld == a.du.ld && a.dwg.ld == a.dwu.ld && a.dwg_acc == a.dwu_acc;
    l.out_w_f32 = w32 || pw.splits > 1;
    const bool out_d_f32 = d32 || pd.splits > 1;
    l.acc = (a.dx_acc && pd.splits == 1) || (dw_acc && pw.splits == 1);
    l.data_first = pd.kblk_per_split >= pw.kblk_per_split;
    hipError_t e;
    for (int w = 0; w < (batch ? 1 : 2); ++w) {
        const Mat &dy = w ? a.du : a.dg, &dw = w ? a.dwu : a.dwg;
        l.w = product_args(pw, a.k, a.n, a.m, dw, w32, w ? a.dwu_acc : a.dwg_acc,
                           ws_w + w * pw.splits * slice_w);
        l.w.A = l.w.A2 = static_cast<const uint16_t *>(a.x.p);
        l.w.B = l.w.B2 = static_cast<const uint16_t *>(dy.p);
        l.w.lda = l.w.lda2 = a.x.ld;
        l.w.ldb = l.w.ldb2 = dy.ld;
        l.w.k1 = (int32_t)a.m;
        l.w.kp = INT32_MAX;
        if (batch) {
            l.w.nbatch = 2;
            const int es = w32 ? 4 : 2;
            l.w.sb_b = static_cast<const uint16_t *>(a.du.p) - static_cast<const uint16_t *>(a.dg.p);
            const ptrdiff_t gap = static_cast<const char *>(a.dwu.p) - static_cast<const char *>(a.dwg.p);
            l.w.sc_b = gap / es;
            if (gap % 16) l.w.vec_c4 = l.w.vec_c8 = 0;
        }
        if (w == 1) l.d.tiles_m = 0;   // dX is done
        l.grid = l.d.tiles_m * l.d.tiles_n * l.d.splits +
                 l.w.tiles_m * l.w.tiles_n * l.w.splits * l.w.nbatch;
        if (l.grid > 0) {
            e = out_d_f32 ? launch_products_f32(l, s) : launch_products_bf16(l, s);
            if (e != hipSuccess) return e;
        }
    }
    if (pd.splits > 1 && a.m > 0) {
        e = launch_split_reduce(reduced(l.d, a.dx, a.dx_dtype, a.dx_acc), pd.splits, a.ws, s);
        if (e != hipSuccess) return e;
    }
    if (pw.splits > 1 && a.n > 0)
        return launch_split_reduce_pair(reduced(l.w, a.dwg, a.dw_dtype, a.dwg_acc), pw.splits, ws_w,
                                        reduced(l.w, a.dwu, a.dw_dtype, a.dwu_acc), pw.splits,
                                        ws_w + pw.splits * slice_w, s);
    return hipSuccess;
}

}  // namespace sbpi
