// gated_products.h -- the three products of the gated block's backward pass in one
// grid (see gated_bwd.hip). Included by one translation unit per output type of dX, so
// that the instances compile in parallel.
#pragma once

#include "gated.h"
#include "gemm_bf16_dma.h"
#include "profile.h"

namespace sbpk {

template <int BM, int BN, int BKD, int NS, int WGM, int WGN, int KG, int EPI, bool OUTD, bool OUTW,
          bool REG, int ACCUM>
__global__ __launch_bounds__(64 * WGM * WGN * KG,
                             (REG ? (BM * BN > 64 * 128 ? 2 : 4)
                                  : Occupancy<BM, BN, BKD, NS, WGM * WGN * KG, KG>::VALUE))
void gated_products_kernel(GemmArgsTwo gd, GemmArgsTwo gw, int data_first) {
    __shared__ __attribute__((aligned(1024))) char smem[NS * DmaStage<BM, BN, BKD, NS>::BYTES];
    const int wd = gd.tiles_m * gd.tiles_n * gd.splits;
    const int ww = gw.tiles_m * gw.tiles_n * gw.splits * gw.nbatch;
    const int b = blockIdx.x;
    if (data_first ? b < wd : b >= ww)
        dma_tile_body<BM, BN, BKD, NS, WGM, WGN, KG, EPI, true, true, OUTD, false, REG, ACCUM>(
            gd, remap_xcd(data_first ? b : b - ww, wd), smem);
    else
        dma_tile_body<BM, BN, BKD, NS, WGM, WGN, KG, EPI, false, false, OUTW, false, REG, ACCUM>(
            gw, remap_xcd(data_first ? b - wd : b, ww), smem);
}

}  // namespace sbpk

namespace sbpi {

// Pipelined instances (of SBP_MODEL_INSTANCES), and those that also exist for products
// that are added to their output; plan.cpp's kGatedCodes lists the same ones.
#define SBP_GATED_INSTANCES(X)                          \
    X(256, 256, 64, 2, 2, 4, 1, sbpk::EPI_DIRECT)       \
    X(128, 128, 128, 2, 2, 2, 2, sbpk::EPI_STAGED)      \
    X(64, 64, 128, 4, 2, 2, 2, sbpk::EPI_STAGED)        \
    SBP_GATED_ACC_INSTANCES(X)
#define SBP_GATED_ACC_INSTANCES(X)                      \
    X(128, 128, 64, 2, 2, 2, 1, sbpk::EPI_DIRECT)       \
    X(64, 64, 64, 2, 2, 2, 1, sbpk::EPI_DIRECT)

struct ProductsLaunch {
    Plan p;
    sbpk::GemmArgsTwo d, w;
    int data_first, grid;
    bool out_w_f32, acc;
};

template <bool OD, bool OW, int ACCUM>
hipError_t launch_products_tile(const ProductsLaunch &l, hipStream_t s) {
    const Plan &p = l.p;
    char name[192];
    name[0] = 0;
#define SBP_CASE(BM_, BN_, BKD_, NS_, WGM_, WGN_, KG_, EPI_, REG_)                             \
    if (p.bm == BM_ && p.bn == BN_ && (REG_ || (p.bk == BKD_ && p.kg == KG_ && p.epi == EPI_))) { \
        if (profiling())                                                                       \
            snprintf(name, sizeof(name), "gated_products_kernel<%d, %d, %d, %d, %d, %d, %d>",  \
                     BM_, BN_, BKD_, NS_, KG_, EPI_, (int)REG_);                               \
        return launch_kernel(                                                                  \
            sbpk::gated_products_kernel<BM_, BN_, BKD_, NS_, WGM_, WGN_, KG_, EPI_, OD, OW, REG_, \
                                        ACCUM>,                                                \
            name, dim3(l.grid), dim3(64 * WGM_ * WGN_ * KG_), s, l.d, l.w, l.data_first);      \
    }
#define SBP_DMA_CASE(BM_, BN_, BKD_, NS_, WGM_, WGN_, KG_, EPI_) \
    SBP_CASE(BM_, BN_, BKD_, NS_, WGM_, WGN_, KG_, EPI_, false)
    if (!p.dma) {
        SBP_CASE(128, 128, 64, 2, 2, 4, 1, sbpk::EPI_STAGED, true)
        SBP_CASE(64, 64, 64, 2, 2, 2, 2, sbpk::EPI_STAGED, true)
    } else if constexpr (ACCUM == sbpk::ACC_NONE) {
        SBP_GATED_INSTANCES(SBP_DMA_CASE)
    } else {
        SBP_GATED_ACC_INSTANCES(SBP_DMA_CASE)
    }
#undef SBP_DMA_CASE
#undef SBP_CASE
    return hipErrorInvalidValue;
}

template <bool OD>
hipError_t launch_products(const ProductsLaunch &l, hipStream_t s) {
    if (l.acc)
        return l.out_w_f32 ? launch_products_tile<OD, true, sbpk::ACC_SOME>(l, s)
               : OD        ? launch_products_tile<OD, false, OD ? sbpk::ACC_SOME : sbpk::ACC_NONE>(l, s)
                           : hipErrorInvalidValue;
    return l.out_w_f32 ? launch_products_tile<OD, true, sbpk::ACC_NONE>(l, s)
                       : launch_products_tile<OD, false, sbpk::ACC_NONE>(l, s);
}

hipError_t launch_products_f32(const ProductsLaunch &l, hipStream_t s);    // fp32 dX
hipError_t launch_products_bf16(const ProductsLaunch &l, hipStream_t s);   // bf16 dX

}  // namespace sbpi
