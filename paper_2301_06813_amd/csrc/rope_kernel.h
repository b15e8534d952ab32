// rope_kernel.h -- the rotation of a pair of columns by its row's position (CDNA4 /
// gfx950), shared by the kernels of rope.hip and paged_append.hip.
//
// A frequency is held as turns a position in 64-bit fixed point, so the fraction of a turn
// at position t is the product t turns modulo 2^64: whole turns fall out of the register, and
// a position of 10^9 has as good an angle as a near one (in fp32 the angle of position 10^6
// would be off by 2^-4). The top 32 bits, less the nearest quarter, are the angle that two
// polynomials take.
#pragma once

#include "gemm_bf16_kernel.h"
#include "rope.h"

namespace sbpk {

using sbpi::CoreView;
using sbpi::RopeArgs;
using sbpi::Rotation;

// cos and sin of a fraction of a turn (2^-32 turn), off by 1.6 2^-24 at most: the polynomials
// (least maximum error on [-pi/4, pi/4], fitted on Chebyshev points) by 2^-27 and less, the rest
// is fp32 rounding.
__device__ __forceinline__ void cos_sin(uint32_t turn, float *c, float *s) {
    const uint32_t q = (turn + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(turn - (q << 30)) * 1.4629180792671596e-9f;   // 2 pi / 2^32
    const float z = x * x;
    float p = __builtin_fmaf(-0.0001951729936990887f, z, 0.008332177996635437f);
    p = __builtin_fmaf(p, z, -0.16666655242443085f);
    const float sn = __builtin_fmaf(x * z, p, x);
    float r = __builtin_fmaf(2.4438451873720624e-5f, z, -0.001388736767694354f);
    r = __builtin_fmaf(r, z, 0.04166664555668831f);
    r = __builtin_fmaf(r, z, -0.5f);
    const float cs = __builtin_fmaf(r, z, 1.f);
    const float a = q & 1 ? sn : cs, b = q & 1 ? cs : sn;
    *c = (q + 1) & 2 ? -a : a;
    *s = q & 2 ? -b : b;
}

// mul cos and mul sin of position t's angle.
__device__ __forceinline__ void angle(uint64_t turns, int64_t t, float mul, float *c, float *s) {
    cos_sin((uint32_t)((uint64_t)t * turns >> 32), c, s);
    *c *= mul;
    *s *= mul;
}

template <typename T>
__device__ __forceinline__ float load1(const T *p) {
    if constexpr (sizeof(T) == 4) return *p;
    else return __builtin_bit_cast(float, (uint32_t)*p << 16);
}
template <typename T>
__device__ __forceinline__ void store1(T *p, float v) {
    if constexpr (sizeof(T) == 4) *p = v;
    else *p = f32_to_bf16_bits(v);
}

// Columns of pair i of a rotation.
__device__ __forceinline__ void columns(const Rotation &r, int i, int *one, int *two) {
    *one = r.pairs ? 2 * i : i;
    *two = r.pairs ? 2 * i + 1 : i + r.dim / 2;
}

}  // namespace sbpk
