// rope_kernel.h -- the rotation of a pair of columns by its row's position (CDNA4 /
// gfx950), shared by the kernels of rope.hip and paged_append.hip.
//
// A frequency is held as turns a position in 64-bit fixed point, so the fraction of a turn
// at position t is the product t turns modulo 2^64: whole turns fall out of the register, and
// a position of 10^9 has as good an angle as a near one (in fp32 the angle of position 10^6
// would be off by 2^-4). The top 32 bits, less the nearest quarter, are the angle that two
// polynomials take.
#pragma once

#include "gemm_bf16_dma.h"
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

// A head's columns are taken in units of 16: first the rotated ones, 8 pairs a unit, then the
// others. A unit is two runs of up to 8 columns.
struct Unit {
    int one, two;     // first columns of the runs
    int n, m;         // columns of the runs
    bool turn;        // the columns make pairs, else they are copied
};

__host__ __device__ inline int units_of(const Rotation &r, int d) {
    return (r.dim / 2 + 7) / 8 + (d - r.dim + 15) / 16;
}

__device__ __forceinline__ Unit unit_of(const Rotation &r, int d, int u) {
    const int half = r.dim / 2, turned = (half + 7) / 8;
    Unit x;
    x.turn = u < turned;
    if (x.turn) {
        const int k = min(8, half - 8 * u);      // pairs
        x.one = r.pairs ? 16 * u : 8 * u;
        x.two = r.pairs ? 16 * u + 8 : half + 8 * u;
        x.n = r.pairs ? min(8, 2 * k) : k;
        x.m = r.pairs ? max(0, 2 * k - 8) : k;
    } else {
        x.one = r.dim + 16 * (u - turned);
        x.two = x.one + 8;
        x.n = min(8, d - x.one);
        x.m = min(8, max(0, d - x.two));
    }
    return x;
}

// 8 values in the memory's type, which may be any element's address: whole runs move in 16-byte
// accesses (which need no alignment), others value by value.
template <typename T>
struct Run;

template <>
struct Run<uint16_t> {
    u32x4 v;
    __device__ __forceinline__ void load(const uint16_t *p, int n) {
        if (n == 8) {
            v = *reinterpret_cast<const u32x4_any *>(p);
            return;
        }
        v = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) v[e / 2] |= (uint32_t)p[e] << (16 * (e & 1));
    }
    __device__ __forceinline__ void store(uint16_t *p, int n) const {
        if (n == 8) {
            *reinterpret_cast<u32x4_any *>(p) = v;
            return;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = (uint16_t)(v[e / 2] >> (16 * (e & 1)));
    }
    __device__ __forceinline__ float get(int e) const {
        return __builtin_bit_cast(float, e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
    }
    __device__ __forceinline__ void set(const float (&x)[8]) {
#pragma unroll
        for (int e = 0; e < 8; e += 2)
            v[e / 2] = (uint32_t)f32_to_bf16_bits(x[e]) | (uint32_t)f32_to_bf16_bits(x[e + 1]) << 16;
    }
};

template <>
struct Run<float> {
    f32x4 v[2];
    __device__ __forceinline__ void load(const float *p, int n) {
        if (n == 8) {
            v[0] = *reinterpret_cast<const f32x4_any *>(p);
            v[1] = *reinterpret_cast<const f32x4_any *>(p + 4);
            return;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e / 4][e % 4] = e < n ? p[e] : 0.f;
    }
    __device__ __forceinline__ void store(float *p, int n) const {
        if (n == 8) {
            *reinterpret_cast<f32x4_any *>(p) = v[0];
            *reinterpret_cast<f32x4_any *>(p + 4) = v[1];
            return;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = v[e / 4][e % 4];
    }
    __device__ __forceinline__ float get(int e) const { return v[e / 4][e % 4]; }
    __device__ __forceinline__ void set(const float (&x)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e / 4][e % 4] = x[e];
    }
};

template <typename T>
struct Pair {
    Run<T> one, two;
    __device__ __forceinline__ void load(const T *row, const Unit &u) {
        one.load(row + u.one, u.n);
        two.load(row + u.two, u.m);
    }
};

// The angles of unit u's pairs at position t.
struct Angles {
    float c[8], s[8];
    __device__ __forceinline__ void find(const Rotation &r, int u, int64_t t, bool back) {
        const int last = r.dim / 2 - 1;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            angle(r.turns[min(8 * u + e, last)], t, r.mul, &c[e], &s[e]);
            if (back) s[e] = -s[e];
        }
    }
};

// Stores a unit, turned by its angles or as it is, to `row`. In the order of pairs a run
// holds 4 pairs whose columns are neighbours; else the runs hold 8 pairs' first and second.
template <typename TI, typename TO>
__device__ __forceinline__ void put(const Pair<TI> &x, const Angles &a, const Unit &u, bool pairs, TO *row) {
    float one[8], two[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        one[e] = x.one.get(e);
        two[e] = x.two.get(e);
    }
    if (u.turn && !pairs) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = one[e], w = two[e];
            one[e] = v * a.c[e] - w * a.s[e];
            two[e] = w * a.c[e] + v * a.s[e];
        }
    } else if (u.turn) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const float v = one[e], w = one[e + 1], y = two[e], z = two[e + 1];
            one[e] = v * a.c[e / 2] - w * a.s[e / 2];
            one[e + 1] = w * a.c[e / 2] + v * a.s[e / 2];
            two[e] = y * a.c[e / 2 + 4] - z * a.s[e / 2 + 4];
            two[e + 1] = z * a.c[e / 2 + 4] + y * a.s[e / 2 + 4];
        }
    }
    Run<TO> r;
    r.set(one);
    r.store(row + u.one, u.n);
    r.set(two);
    r.store(row + u.two, u.m);
}

}  // namespace sbpk
