// gated.h -- the gated feed-forward block H = act(X Wg) * (X Wu) of a device's
// shares (include/sbp.h, "gated feed-forward block"): what the host code and the
// kernels of gated_fwd.hip and gated_bwd.hip share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gemm.h"

namespace sbpi {

enum { ACT_SILU = 0, ACT_GELU = 1, ACT_RELU = 2 };   // sbp_act_t

// A matrix in memory: elements of the call's type.
struct Mat {
    void *p = nullptr;
    int64_t ld = 0;
};

// X: m x k, Wg and Wu: k x n; H, G = X Wg, U = X Wu: m x n. The backward pass reads
// dH, G and U, writes dG and dU, and from them dX (m x k), dWg and dWu (k x n).
struct Gated {
    int dtype = DT_BF16;
    int act = ACT_SILU;
    int64_t m = 0, n = 0, k = 0;
    Mat x, wg, wu, h, g, u;          // forward: g.p, u.p may be NULL
    Mat dh, dg, du, dx, dwg, dwu;
    int dx_dtype = DT_BF16, dw_dtype = DT_BF16;
    int dx_acc = 0, dwg_acc = 0, dwu_acc = 0;
    float *ws = nullptr;
    size_t ws_floats = 0;
};

hipError_t launch_gated_fwd(const Gated &a, hipStream_t s);
// dG = dH U act'(G), dU = dH act(G).
hipError_t launch_gated_grad(const Gated &a, hipStream_t s);
// dX = dG Wg^T + dU Wu^T, dWg = X^T dG, dWu = X^T dU (bf16).
hipError_t launch_gated_products(const Gated &a, hipStream_t s);
// The same in fp32, in one launch; *taken false where its rules refuse it (an empty product,
// leading dimensions of 2^21 elements and more), with nothing launched.
hipError_t launch_gated_products_f32(const Gated &a, hipStream_t s, bool *taken);
// H = act(G) U from fp32 or bf16 matrices in memory.
hipError_t launch_gated_act(const Gated &a, hipStream_t s);

}  // namespace sbpi

#ifdef __HIP__
namespace sbpk {

__device__ __forceinline__ float sigmoid(float x) {
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * -1.4426950408889634f));
}

// tanh form of the Gaussian error linear unit: 0.5 (1 + tanh(y)) = sigmoid(2 y)
constexpr float GELU_A = 1.5957691216057308f;   // 2 sqrt(2 / pi)
constexpr float GELU_B = 0.044715f;

template <int ACT>
__device__ __forceinline__ float act_of(float x) {
    if constexpr (ACT == sbpi::ACT_RELU) return x > 0.f ? x : x != x ? x : 0.f;
    if constexpr (ACT == sbpi::ACT_SILU) return x * sigmoid(x);
    return x * sigmoid(GELU_A * x * __builtin_fmaf(GELU_B * x, x, 1.f));
}

// act(x) and its derivative.
template <int ACT>
__device__ __forceinline__ void act_grad(float x, float *a, float *d) {
    if constexpr (ACT == sbpi::ACT_RELU) {
        *a = act_of<ACT>(x);
        *d = x > 0.f ? 1.f : x != x ? x : 0.f;
    } else if constexpr (ACT == sbpi::ACT_SILU) {
        const float z = sigmoid(x);
        *a = x * z;
        *d = __builtin_fmaf(*a, 1.f - z, z);
    } else {
        const float z = sigmoid(GELU_A * x * __builtin_fmaf(GELU_B * x, x, 1.f));
        *a = x * z;
        const float t = *a * (1.f - z);   // 0 far out, where x^2 may overflow
        *d = t == 0.f ? z : __builtin_fmaf(t * GELU_A, __builtin_fmaf(3.f * GELU_B * x, x, 1.f), z);
    }
}

}  // namespace sbpk
#endif
