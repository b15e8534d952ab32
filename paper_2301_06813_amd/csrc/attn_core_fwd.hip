// attn_core_fwd.hip -- softmax attention, forward.
//
// Per sequence and key head, the rows of a group of query heads that share it
// are packed as row = i * group + g (query i, head g), so K and V are read once
// for the group and a few query rows fill a tile. A workgroup owns a tile of rows
// and walks over the keys that any of them sees, 32 KG .. 64 KG at a time: scores
// as S^T = K Q^T, running maximum m and sum l of each row, O^T += V^T P^T. In these
// orientations a lane holds one query's scores (half of them, the other half-wave
// the rest), so m and l are one register each, the rows' scaling needs no
// broadcast, and P^T goes from the exponentials into the second product without
// leaving its registers.
//
//   * exp(scale (s - m)) is one multiply-add and one base-2 exponential a score.
//     The maximum is moved only when a row's grows by more than 8 in the exponent:
//     until then sums and outputs grow by up to 2^8, far inside fp32, and rescaling
//     is skipped by the whole wave.
//   * P is rounded to bf16 for the second product (the matrix cores' type, rounded
//     like the framework's other bf16 operands); the row sum adds the fp32 values.
//   * With KG wave groups, group k takes the k-th part of every step's keys; their
//     (m, l, O) are joined through LDS at the end. Few rows and many keys are also
//     split over workgroups, whose normalised partial outputs and row statistics
//     go through the workspace.
#include <math.h>

#include "attn_core_kernel.h"
#include "gemm.h"
#include "profile.h"

namespace sbpk {

// O rows of 4 consecutive values starting at column `col` (col < d).
template <class F>
__device__ __forceinline__ void store4(void *base, int64_t at, int col, int d, bool f32, bool vec,
                                       F value) {
    if (f32) {
        float *p = static_cast<float *>(base) + at + col;
        if (vec && col + 4 <= d) {
            f32x4 v = {value(0), value(1), value(2), value(3)};
            *reinterpret_cast<f32x4 *>(p) = v;
            return;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < d) p[e] = value(e);
    } else {
        uint16_t *p = static_cast<uint16_t *>(base) + at + col;
        if (vec && col + 4 <= d) {
            u32x2 w;
            w[0] = (uint32_t)f32_to_bf16_bits(value(0)) | (uint32_t)f32_to_bf16_bits(value(1)) << 16;
            w[1] = (uint32_t)f32_to_bf16_bits(value(2)) | (uint32_t)f32_to_bf16_bits(value(3)) << 16;
            *reinterpret_cast<u32x2 *>(p) = w;
            return;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < d) p[e] = f32_to_bf16_bits(value(e));
    }
}

struct FwdArgs {
    CoreArgs a;
    int32_t tiles, splits, rows;     // row tiles per (sequence, key head); rows = sq * group
    int32_t vec;                     // O allows 4-value stores
};

template <int DP, int KG, int KT>
struct FwdShape {
    static constexpr int NW = 4;
    static constexpr int ROWS = 32 * NW / KG;
    using Tile = RowTile<DP, KG * KT, NW>;
    static constexpr int STAGE = 2 * Tile::BYTES;    // K, then V
    static constexpr int LDS = 2 * STAGE;
    static constexpr int OCC = LDS > 81920 ? 1 : 2;
};

template <int DP, int KG, int KT, bool DMA>
__global__ __launch_bounds__(256, (FwdShape<DP, KG, KT>::OCC))
void attn_core_fwd_kernel(FwdArgs f) {
    using S = FwdShape<DP, KG, KT>;
    using Tile = typename S::Tile;
    constexpr int NW = S::NW, ROWS = S::ROWS, KB = KT / 32, KS = DP / 16, DB = DP / 32;
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS];
    const CoreArgs &a = f.a;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);   // uniform, so that what
                                                                 // depends on it is scalar
    const int kg = wave % KG, wr = wave / KG;

    // heavier (later) causal tiles first within a (sequence, head)
    const int per = f.tiles * f.splits;
    int bh, t;
    deal(blockIdx.x, a.batch * a.kv_heads, per, &bh, &t);
    const int tile = f.tiles - 1 - t / f.splits, split = t % f.splits;
    const int b = bh / a.kv_heads, hk = bh % a.kv_heads;
    const SeqMask mask(a, b);

    const int row0 = tile * ROWS;
    const int row = row0 + wr * 32 + (lane & 31);
    const bool valid = row < f.rows;
    const int i = (valid ? row : f.rows - 1) / a.group;
    const int g = (valid ? row : f.rows - 1) - i * a.group;
    const int64_t head = (int64_t)hk * a.group + g;

    // the keys that the tile's rows see, and this split's steps of them
    const int i_first = row0 / a.group;
    const int i_last = min(min(row0 + ROWS, f.rows) - 1, f.rows - 1) / a.group;
    const int k_beg = mask.lo(i_first) & ~31;
    const int k_end = i_first < mask.lq ? mask.hi(min(i_last, mask.lq - 1)) : 0;
    const int steps = k_end > k_beg ? (k_end - k_beg + KG * KT - 1) / (KG * KT) : 0;
    // steps whose keys every row of the tile sees (rows past the sequence's end aside)
    Walk walk{steps, 0, steps};
    if (steps > 0) {
        const int all = min(mask.hi(i_first), mask.lk);
        walk.nb = all > k_beg ? min(steps, (all - k_beg) / (KG * KT)) : 0;
        walk.na = min(walk.nb, (mask.lo(i_last) - k_beg + KG * KT - 1) / (KG * KT));
        walk.na = max(walk.na, 0);
    }
    const int per_split = (steps + f.splits - 1) / f.splits;
    const int s0 = min(steps, split * per_split), s1 = min(steps, s0 + per_split);
    const int hi = mask.hi(i), lo = mask.lo(i);

    const uint16_t *Q = static_cast<const uint16_t *>(a.q.p) + (int64_t)b * a.q.sb +
                        head * a.q.sh + (int64_t)i * a.q.ld;
    const uint16_t *K = static_cast<const uint16_t *>(a.k.p) + (int64_t)b * a.k.sb +
                        (int64_t)hk * a.k.sh;
    const uint16_t *V = static_cast<const uint16_t *>(a.v.p) + (int64_t)b * a.v.sb +
                        (int64_t)hk * a.v.sh;

    const int place_k = Tile::place(a.k.ld, a.d, wave, lane);
    const int place_v = Tile::place(a.v.ld, a.d, wave, lane);
    typename Tile::Regs rk, rv;
    auto issue = [&](int x, int stage) {
        const int k0 = k_beg + walk.step(x) * (KG * KT);
        const int n = min(KG * KT, mask.lk - k0);
        char *lds = smem + stage * S::STAGE;
        if constexpr (DMA) {
            Tile::issue(K + (int64_t)k0 * a.k.ld, a.k.ld, n, place_k, lds, wave);
            Tile::issue(V + (int64_t)k0 * a.v.ld, a.v.ld, n, place_v, lds + Tile::BYTES, wave);
        } else {
            Tile::load(rk, K + (int64_t)k0 * a.k.ld, a.k.ld, n, a.d, tid);
            Tile::load(rv, V + (int64_t)k0 * a.v.ld, a.v.ld, n, a.d, tid);
        }
    };
    auto arrive = [&](int stage) {   // register-staged: the loaded step goes to LDS
        if constexpr (!DMA) {
            char *lds = smem + stage * S::STAGE;
            Tile::store(rk, lds, tid);
            Tile::store(rv, lds + Tile::BYTES, tid);
        }
    };

    if (s0 < s1) {
        issue(s0, 0);
        arrive(0);
    }
    // rows past a sequence's queries read nothing
    const bool live = valid && i < mask.lq;
    bf16x8 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
        qf[ks] = row_frag<DMA>(Q, ks * 16 + 8 * half, live ? a.d : 0);
    settle(qf);

    const float c = a.scale * LOG2E;
    const float grow = 8.f / c;
    float m = -INFINITY, l = 0.f;
    f32x16 o[DB];
#pragma unroll
    for (int x = 0; x < DB; ++x) o[x] = splat16(0.f);

    typename Tile::Reader rd(lds_at(smem) + kg * KT / Tile::RPS * Tile::SEG, lane);
    auto step = [&](int kw, auto edge) {
        f32x16 s[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            s[kb] = splat16(0.f);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    rd.frag(kb * 32, ks, 0), qf[ks], s[kb], 0, 0, 0);
        }
        if constexpr (decltype(edge)::value) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int key = kw + kb * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
                    s[kb][r] = key >= lo && key < hi ? s[kb][r] : -INFINITY;
                }
        }
        float top = s[0][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[kb][r]);
        float t0, t1;
        halves(top, &t0, &t1);
        top = fmaxf(t0, t1);
        if (__any(top > m + grow)) {
            const float mn = fmaxf(m, top);
            const float x = mn == -INFINITY ? 1.f : exp2_((m - mn) * c);
            m = mn;
            l *= x;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[db][r] *= x;
        }
        const float mc = m == -INFINITY ? 0.f : m * c;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[kb][r] = exp2_(__builtin_fmaf(s[kb][r], c, -mc));
                l += s[kb][r];
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const bf16x8 p = pack8(s[kb], 8 * x);
#pragma unroll
                for (int db = 0; db < DB; ++db)
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        rd.frag_t(db, kb * 32 + 16 * x, Tile::BYTES), p, o[db], 0, 0, 0);
            }
        }
    };
    auto take = [&](int x, auto edge) {
        const int stage = (x - s0) & 1;
        wait_vm<0>();
        __syncthreads();
        if (x + 1 < s1) issue(x + 1, stage ^ 1);
        step(k_beg + walk.step(x) * (KG * KT) + kg * KT, edge);
        rd.move(stage ? -S::STAGE : S::STAGE);
        if (x + 1 < s1) arrive(stage ^ 1);
    };
    int x = s0;
    for (; x < min(s1, walk.masked()); ++x) take(x, std::true_type{});
    for (; x < s1; ++x) take(x, std::false_type{});

    float l0, l1;
    halves(l, &l0, &l1);
    l = l0 + l1;

    if constexpr (KG > 1) {
        // groups 1.. hand (m, l, O) to group 0 through LDS, lane by lane
        __syncthreads();
        constexpr int SLOT = (DB * 16 + 2) * 64;
        static_assert((KG - 1) * (NW / KG) * SLOT * 4 <= S::LDS, "group results do not fit");
        float *const base = reinterpret_cast<float *>(smem) + lane;
        if (kg > 0) {
            float *p = base + ((kg - 1) * (NW / KG) + wr) * SLOT;
            p[0] = m;
            p[64] = l;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) p[(2 + db * 16 + r) * 64] = o[db][r];
        }
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int k = 1; k < KG; ++k) {
            const float *p = base + ((k - 1) * (NW / KG) + wr) * SLOT;
            const float mk = p[0], mn = fmaxf(m, mk);
            const float ms = mn == -INFINITY ? 0.f : mn;
            const float x0 = exp2_((m - ms) * c), x1 = exp2_((mk - ms) * c);
            m = mn;
            l = l * x0 + p[64] * x1;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    o[db][r] = o[db][r] * x0 + p[(2 + db * 16 + r) * 64] * x1;
        }
    }

    if (!valid) return;
    // a row that sees no key: O = 0, lse = -infinity
    const bool some = live && l != 0.f;
    const float inv = some ? 1.f / l : 0.f;
    const float lse2 = some ? m * c + __builtin_amdgcn_logf(l) : -INFINITY;
    if (f.splits > 1) {
        const int64_t d4 = (a.d + 3) & ~3;
        const int64_t bhs = (int64_t)a.batch * a.kv_heads;
        const int64_t at = ((int64_t)split * bhs + bh) * f.rows + row;
        float *const part = a.ws + at * d4;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int col = db * 32 + 8 * q + 4 * half;
                if (col >= d4) continue;
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = some ? o[db][4 * q + e] * inv : 0.f;
                *reinterpret_cast<f32x4 *>(part + col) = v;
            }
        if (half == 0) a.ws[(int64_t)f.splits * bhs * f.rows * d4 + at] = lse2;
        return;
    }
    const int64_t at = (int64_t)b * a.o.sb + head * a.o.sh + (int64_t)i * a.o.ld;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int col = db * 32 + 8 * q + 4 * half;
            if (col < a.d)
                store4(a.o.p, at, col, a.d, a.o_f32, f.vec,
                       [&](int e) { return some ? o[db][4 * q + e] * inv : 0.f; });
        }
    if (a.lse.p && half == 0)
        static_cast<float *>(a.lse.p)[(int64_t)b * a.lse.sb + head * a.lse.sh +
                                      (int64_t)i * a.lse.ld] = lse2 * LN2;
}

// Joins the key splits of a row: weights 2^(lse_s - lse), in split order. A thread
// owns 4 columns of a row.
__global__ __launch_bounds__(256) void attn_core_join_kernel(FwdArgs f) {
    const CoreArgs &a = f.a;
    const int quads = (a.d + 3) >> 2;
    const int64_t bhs = (int64_t)a.batch * a.kv_heads, n = bhs * f.rows;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= n * quads) return;
    const int64_t at = id / quads;
    const int col = (int)(id % quads) * 4;
    const int64_t d4 = quads * 4;
    const float *stat = a.ws + f.splits * n * d4 + at;
    float top = -INFINITY;
    for (int s = 0; s < f.splits; ++s) top = fmaxf(top, stat[s * n]);
    const float base = top == -INFINITY ? 0.f : top;
    float total = 0.f;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < f.splits; ++s) {
        const float w = exp2_(stat[s * n] - base);
        const f32x4 x = *reinterpret_cast<const f32x4 *>(a.ws + (s * n + at) * d4 + col);
        total += w;
        v += x * w;
    }
    const bool some = total != 0.f;
    const float inv = some ? 1.f / total : 0.f;
    const int bh = (int)(at / f.rows), row = (int)(at % f.rows);
    const int b = bh / a.kv_heads, hk = bh % a.kv_heads;
    const int i = row / a.group;
    const int64_t head = (int64_t)hk * a.group + (row - i * a.group);
    store4(a.o.p, (int64_t)b * a.o.sb + head * a.o.sh + (int64_t)i * a.o.ld, col, a.d, a.o_f32,
           f.vec, [&](int e) { return v[e] * inv; });
    if (a.lse.p && col == 0)
        static_cast<float *>(a.lse.p)[(int64_t)b * a.lse.sb + head * a.lse.sh +
                                      (int64_t)i * a.lse.ld] =
            some ? (top + __builtin_amdgcn_logf(total)) * LN2 : -INFINITY;
}

}  // namespace sbpk

namespace sbpi {

namespace {

template <int DP, int KG, int KT>
hipError_t launch_fwd(const sbpk::FwdArgs &f, int64_t blocks, hipStream_t s) {
    char name[160];
    name[0] = 0;
    if (profiling())
        snprintf(name, sizeof(name), "attn_core_fwd_kernel<%d,%d,%d,%d>", DP, KG, KT,
                 (int)f.a.aligned);
    if (f.a.aligned)
        return launch_kernel(sbpk::attn_core_fwd_kernel<DP, KG, KT, true>, name,
                             dim3((unsigned)blocks), dim3(256), s, f);
    return launch_kernel(sbpk::attn_core_fwd_kernel<DP, KG, KT, false>, name,
                         dim3((unsigned)blocks), dim3(256), s, f);
}

}  // namespace

hipError_t launch_core_fwd(const CoreArgs &a, hipStream_t s) {
    sbpk::FwdArgs f;
    f.a = a;
    f.rows = a.sq * a.group;
    const int esz = a.o_f32 ? 4 : 2;
    f.vec = reinterpret_cast<uintptr_t>(a.o.p) % (4 * esz) == 0 && a.o.ld % 4 == 0 &&
            a.o.sb % 4 == 0 && a.o.sh % 4 == 0;
    const int64_t bhs = (int64_t)a.batch * a.kv_heads;
    const int cus = device_cus();
    int kg = 1;
    while (kg < 4 && ((f.rows + 128 / kg - 1) / (128 / kg)) * bhs < cus) kg *= 2;
    const int rows = 128 / kg, keys = kg == 4 ? 128 : 64 * kg;
    f.tiles = (f.rows + rows - 1) / rows;
    // split the keys while workgroups are few and each has several steps
    const int64_t steps = (a.sk + keys - 1) / keys;
    const size_t d4 = (a.d + 3) & ~3, per = (size_t)bhs * f.rows * (d4 + 1);
    int64_t splits = 1;
    while (f.tiles * bhs * splits * 2 <= 2 * cus && steps / (splits * 2) >= 2 &&
           per * splits * 2 <= a.ws_floats)
        splits *= 2;
    f.splits = (int)splits;
    const int64_t blocks = (int64_t)f.tiles * bhs * splits;
    hipError_t e;
    const bool wide = a.d > 64;
    if (kg == 1)
        e = wide ? launch_fwd<128, 1, 64>(f, blocks, s) : launch_fwd<64, 1, 64>(f, blocks, s);
    else if (kg == 2)
        e = wide ? launch_fwd<128, 2, 64>(f, blocks, s) : launch_fwd<64, 2, 64>(f, blocks, s);
    else
        e = wide ? launch_fwd<128, 4, 32>(f, blocks, s) : launch_fwd<64, 4, 32>(f, blocks, s);
    if (e != hipSuccess || splits == 1) return e;
    const int64_t items = bhs * f.rows * (int64_t)(d4 / 4);
    return launch_kernel(sbpk::attn_core_join_kernel, "attn_core_join_kernel",
                         dim3((unsigned)((items + 255) / 256)), dim3(256), s, f);
}

}  // namespace sbpi
