// rope_kernel.h -- the rotation of a pair of columns by its row's position (CDNA4 /
// gfx950), shared by the kernels of rope.hip and paged_append.hip.
//
// A frequency is held as turns a position in 64-bit fixed point, so the fraction of a turn
// at position t is the product t turns modulo 2^64: whole turns fall out of the register, and
// a position of 10^9 has as good an angle as a near one (in fp32 the angle of position 10^6
// would be off by 2^-4). The top 32 bits, less the nearest quarter, are the angle that two
// polynomials take.
#pragma once

#include <type_traits>

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

// A head's columns are taken in units of 2 R: first the rotated ones, R pairs a unit, then the
// others. A unit is two runs of up to R columns, from the first and the second half of these, in
// either order of the pairs, so that a wave's accesses lie side by side (append of 7180 tokens of 64
// + 8 + 8 heads of 128 in the order of pairs: 66.8 us with 2 R columns a lane, 64.4).
struct Unit {
    int one, two;     // first columns of the runs
    int n, m;         // columns of the runs
    bool turn;        // the columns make pairs, else they are copied
};

// Columns of the first half of the rotated ones (whole pairs), and of the others.
__host__ __device__ inline int first_half(const Rotation &r) {
    return r.pairs ? (r.dim / 2 + 1) & ~1 : r.dim / 2;
}
template <int R>
__host__ __device__ inline int units_of(const Rotation &r, int d) {
    return (first_half(r) + R - 1) / R + (d - r.dim + 2 * R - 1) / (2 * R);
}

template <int R>
__device__ __forceinline__ Unit unit_of(const Rotation &r, int d, int u) {
    const int turned = (first_half(r) + R - 1) / R;
    Unit x;
    x.turn = u < turned;
    const int from = x.turn ? 0 : r.dim, to = x.turn ? r.dim : d, at = R * (x.turn ? u : u - turned);
    const int half = x.turn ? first_half(r) : (d - r.dim + 2 * R - 1) / (2 * R) * R;
    x.one = from + at;
    x.two = from + half + at;
    x.n = min(R, min(from + half, to) - x.one);
    x.m = min(R, max(0, to - x.two));
    return x;
}

// R values in the memory's type, 16 bytes at most, at any element's address (global accesses need
// no alignment): a whole run in one access, a shorter one in 8, 4 and 2 bytes.
template <typename T, int R>
struct Run {
    static constexpr int WORDS = R * (int)sizeof(T) / 4;
    static_assert(WORDS == 2 || WORDS == 4, "8 or 16 bytes");
    typedef uint32_t V __attribute__((ext_vector_type(WORDS)));
    typedef V V_any __attribute__((aligned(2)));
    typedef uint64_t D_any __attribute__((aligned(2)));
    typedef uint32_t W_any __attribute__((aligned(2)));
    V v;

    __device__ __forceinline__ void load(const T *from, int n) {
        if (n == R) {
            v = *reinterpret_cast<const V_any *>(from);
            return;
        }
        const char *p = reinterpret_cast<const char *>(from);
        const int bytes = n * (int)sizeof(T);
        uint64_t first = 0, rest = 0;
        if (bytes & 8) first = *reinterpret_cast<const D_any *>(p), p += 8;
        if (bytes & 4) rest = *reinterpret_cast<const W_any *>(p), p += 4;
        if (bytes & 2) rest |= (uint64_t)*reinterpret_cast<const uint16_t *>(p) << (bytes & 4 ? 32 : 0);
        const uint64_t lo = bytes & 8 ? first : rest, hi = bytes & 8 ? rest : 0;
#pragma unroll
        for (int w = 0; w < WORDS; ++w) v[w] = (uint32_t)((w < 2 ? lo : hi) >> (32 * (w & 1)));
    }
    __device__ __forceinline__ void store(T *to, int n) const {
        if (n == R) {
            *reinterpret_cast<V_any *>(to) = v;
            return;
        }
        char *p = reinterpret_cast<char *>(to);
        const int bytes = n * (int)sizeof(T);
        const uint64_t lo = v[0] | (uint64_t)v[1] << 32;
        const uint64_t hi = WORDS > 2 ? v[WORDS - 2] | (uint64_t)v[WORDS - 1] << 32 : 0;
        uint64_t rest = bytes & 8 ? hi : lo;
        if (bytes & 8) *reinterpret_cast<D_any *>(p) = lo, p += 8;
        if (bytes & 4) *reinterpret_cast<W_any *>(p) = (uint32_t)rest, p += 4, rest >>= 32;
        if (bytes & 2) *reinterpret_cast<uint16_t *>(p) = (uint16_t)rest;
    }
    __device__ __forceinline__ float get(int e) const {
        // (a copy: the cast of a vector's element itself takes the first one)
        const uint32_t w = v[e * (int)sizeof(T) / 4];
        return __builtin_bit_cast(float, sizeof(T) == 4 ? w : e & 1 ? w & 0xffff0000u : w << 16);
    }
    __device__ __forceinline__ void set(const float (&x)[R]) {
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
            if constexpr (sizeof(T) == 4) v[w] = __builtin_bit_cast(uint32_t, x[w]);
            else v[w] = (uint32_t)f32_to_bf16_bits(x[2 * w]) | (uint32_t)f32_to_bf16_bits(x[2 * w + 1]) << 16;
        }
    }
};

template <typename T, int R>
struct Pair {
    Run<T, R> one, two;
    __device__ __forceinline__ void load(const T *row, const Unit &u) {
        one.load(row + u.one, u.n);
        two.load(row + u.two, u.m);
    }
};

// The angles of unit u's pairs at position t: R pairs, or the R / 2 of either run.
template <int R>
struct Angles {
    float c[R], s[R];
    __device__ __forceinline__ void find(const Rotation &r, int u, int64_t t, bool back) {
        const int last = r.dim / 2 - 1;
        const int one = r.pairs ? R / 2 * u : R * u;
        const int two = r.pairs ? first_half(r) / 2 + one : one + R / 2;
#pragma unroll
        for (int e = 0; e < R; ++e) {
            const int i = e < R / 2 ? one + e : two + e - R / 2;
            angle(r.turns[min(i, last)], t, r.mul, &c[e], &s[e]);
            if (back) s[e] = -s[e];
        }
    }
};

// Stores a unit, turned by its angles or as it is, to `row`. In the order of pairs a run
// holds R / 2 pairs whose columns are neighbours; else the runs hold R pairs' first and second.
template <typename TI, typename TO, int R>
__device__ __forceinline__ void put(const Pair<TI, R> &x, const Angles<R> &a, const Unit &u, bool pairs,
                                    TO *row) {
    if constexpr (std::is_same<TI, TO>::value)
        if (!u.turn) {                // bit for bit
            x.one.store(row + u.one, u.n);
            x.two.store(row + u.two, u.m);
            return;
        }
    float one[R], two[R];
#pragma unroll
    for (int e = 0; e < R; ++e) {
        one[e] = x.one.get(e);
        two[e] = x.two.get(e);
    }
    if (u.turn && !pairs) {
#pragma unroll
        for (int e = 0; e < R; ++e) {
            const float v = one[e], w = two[e];
            one[e] = v * a.c[e] - w * a.s[e];
            two[e] = w * a.c[e] + v * a.s[e];
        }
    } else if (u.turn) {
#pragma unroll
        for (int e = 0; e < R; e += 2) {
            const int k = e / 2, l = (e + R) / 2;
            const float v = one[e], w = one[e + 1], y = two[e], z = two[e + 1];
            one[e] = v * a.c[k] - w * a.s[k];
            one[e + 1] = w * a.c[k] + v * a.s[k];
            two[e] = y * a.c[l] - z * a.s[l];
            two[e + 1] = z * a.c[l] + y * a.s[l];
        }
    }
    Run<TO, R> r;
    r.set(one);
    r.store(row + u.one, u.n);
    r.set(two);
    r.store(row + u.two, u.m);
}

}  // namespace sbpk
