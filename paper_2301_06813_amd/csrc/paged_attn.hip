// paged_attn.hip -- softmax attention of new tokens over a paged cache.
//
// The walk over a tile's keys is that of whole sequences (attn_core_walk.h): rows of a group of
// query heads packed as row = i * group + g, S^T = K Q^T, running maximum and sum, O^T += V^T P^T,
// stages of keys and values on their way to LDS. What differs:
//
//   * Work. Lengths are known on the device only, and differ: a token of one sequence beside a
//     prompt of another. The items (sequence, key head, tile of rows), each as long as its steps
//     of keys and a fixed part, are laid end to end, and as many workgroups as the chip holds
//     take equal parts of that line, whatever the lengths are. Every workgroup finds its part by
//     the same sums over the sequences. An item that is cut leaves partial outputs in the
//     workspace, two at most for each workgroup, and a second kernel joins them in order.
//   * Pages. The page numbers of up to PAGES_AT_ONCE pages of a walk are brought to LDS. Rows of
//     a load of one wave (1 KB: 4 or 8) lie on one page where the page's tokens are a multiple
//     of them, so that a load is a buffer of its own, whose address is scalar arithmetic and
//     whose end is the last row that is seen; other pages, and rows that allow no 16-byte loads,
//     pass through registers.
//   * Rows that the tile does not see, and pages that do not exist, arrive as zeros; a walk with
//     such a page masks every step by the page numbers.
#include <math.h>

#include <algorithm>

#include "attn_core_walk.h"
#include "gemm.h"
#include "paged_kernel.h"
#include "profile.h"

namespace sbpk {

using sbpi::PagedArgs;

constexpr int PAGES_AT_ONCE = 1024;
constexpr int FIXED = 4;             // an item's fixed part, in steps
constexpr int SHORTEST = 2;          // steps that a cut leaves on either side
constexpr int SHARE = 8;             // units (steps and fixed parts) of a workgroup at least

// What workgroup w leaves for the join where its share begins inside an item that workgroup
// w - 1 began: the item's parts are in slot 1 of w - 1 and in slots 0 of w .. last. Else last < 0.
struct Cut {
    int32_t last, seq, head, tile;
};

struct PagedLaunch {
    PagedArgs a;
    int32_t slot_rows;               // rows of a partial output
    int32_t split;                   // items may be cut
    int32_t vec;                     // O allows 4-value stores
    int32_t groups;                  // workgroups
    Div page, group;
};

// The workspace: cuts, statistics (a row's maximum and sum), partial outputs.
typedef float f32x2 __attribute__((ext_vector_type(2)));
__host__ __device__ inline int64_t slot_floats(int64_t rows, int d) {
    return rows * (2 + ((d + 3) & ~3));
}
__device__ __forceinline__ Cut *cuts_of(const PagedLaunch &f) { return reinterpret_cast<Cut *>(f.a.ws); }
__device__ __forceinline__ f32x2 *stats_of(const PagedLaunch &f) {
    return reinterpret_cast<f32x2 *>(f.a.ws + 4 * (int64_t)f.groups);
}
__device__ __forceinline__ float *parts_of(const PagedLaunch &f) {
    return f.a.ws + 4 * (int64_t)f.groups + 4 * (int64_t)f.groups * f.slot_rows;
}

// A value that all lanes have, in a scalar register: the compiler keeps what it loads or gets from
// LDS in vector registers, and all that follows from it.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
    return (int64_t)((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x));
}

// A sequence: its rows (packed ones of the group: `rows`, of which those of n queries are in use),
// and its keys.
struct Seq {
    SeqRows at;
    int rows, lk, off;
    __device__ __forceinline__ Seq(const PagedArgs &a, int b) : Seq(a, rows_of(a.at, b)) {}
    // The sequence that a whole workgroup works on.
    __device__ __forceinline__ static Seq shared(const PagedArgs &a, int b) {
        const SeqRows r = rows_of(a.at, b);
        return Seq(a, SeqRows{a.at.row_q ? 0 : b, uniform(r.first), uniform(r.n), uniform(r.len)});
    }
    __device__ __forceinline__ Seq(const PagedArgs &a, const SeqRows &r) : at(r) {
        rows = (a.at.row_q ? at.n : a.at.rows) * a.group;
        lk = min(max(at.len, 0), a.at.width * a.at.page);
        off = lk - at.n;
    }
    __device__ __forceinline__ int hi(const PagedArgs &a, int i) const {
        return a.causal ? max(0, min(lk, i + 1 + off)) : lk;
    }
    __device__ __forceinline__ int lo(const PagedArgs &a, int i) const {
        return a.window ? max(0, i + 1 + off - a.window) : 0;
    }
};

// The keys that some row of a tile sees, [lo, end), and its steps of KEYS from beg on.
template <int ROWS, int KEYS>
struct TileKeys {
    int first, last;                 // queries of the tile
    int lo, beg, end, steps;
    __device__ __forceinline__ TileKeys(const PagedLaunch &f, const Seq &s, int tile) {
        const int row0 = tile * ROWS;
        first = f.group(row0);
        last = min(f.group(min(row0 + ROWS, s.rows) - 1), s.at.n - 1);
        lo = s.lo(f.a, first);
        beg = lo & ~31;
        end = first <= last ? s.hi(f.a, last) : 0;
        steps = end > lo ? (end - beg + KEYS - 1) / KEYS : 0;
    }
    // An item without steps counts as one: its rows are cleared.
    __device__ __forceinline__ int length() const { return max(steps, 1); }
    __device__ __forceinline__ int cost() const { return FIXED + length(); }
    // Where a cut u units into the item falls: it ends one part and begins the other.
    __device__ __forceinline__ int cut(int64_t u, bool split) const {
        if (u <= 0) return 0;
        if (u >= cost()) return length();
        const int s = (int)u - FIXED;
        if (!split) return 2 * s < length() ? 0 : length();
        return s < SHORTEST ? 0 : length() - s < SHORTEST ? length() : s;
    }
};

__device__ __forceinline__ int64_t wave_up(int64_t x, int by) {
    const uint32_t lo = __shfl_up((uint32_t)x, by), hi = __shfl_up((uint32_t)((uint64_t)x >> 32), by);
    return (int64_t)((uint64_t)hi << 32 | lo);
}

// Sum of x over this and earlier threads of the workgroup; *total: over all. `room` holds NW.
template <int NW>
__device__ __forceinline__ int64_t scan(int64_t x, int64_t *room, int64_t *total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int by = 1; by < 64; by *= 2) {
        const int64_t y = wave_up(x, by);
        if (lane >= by) x += y;
    }
    __syncthreads();
    if (lane == 63) room[wave] = x;
    __syncthreads();
    int64_t sum = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        if (w < wave) x += room[w];
        sum += room[w];
    }
    *total = sum;
    return x;
}

template <int DP, int KG, int KT, int NW, int WPS, bool DMA>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(WPS, WPS)))
void paged_attn_kernel(PagedLaunch f) {
    using S = FwdShape<DP, KG, KT, NW, WPS, DMA>;
    using Tile = typename S::Tile;
    constexpr int ROWS = S::ROWS, NS = S::NS, KEYS = S::KEYS, KS = DP / 16, NV = Tile::NV;
    using Keys = TileKeys<ROWS, KEYS>;
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS];
    __shared__ int32_t numbers[PAGES_AT_ONCE];
    __shared__ int32_t missing[NW];
    static_assert(S::LDS + 4 * PAGES_AT_ONCE + 64 <= S::ROOM, "page numbers beside the stages");
    const uint32_t lds0 = lds_at(smem);
    const PagedArgs &a = f.a;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kg = wave % KG, wr = wave / KG;
    const int64_t d4 = (a.d + 3) & ~3;
    const int wg = remap_xcd(blockIdx.x, f.groups);    // neighbours on the line share an L2

    // This workgroup's part of the line, `left` units from unit u of tile `tile` of head hk of
    // sequence b on.
    int64_t cut0, u, left, total = 0;
    int b, hk, wgs;
    {
        int64_t *const room = reinterpret_cast<int64_t *>(smem);
        int64_t one = 0, upto = 0, sum = 0;    // a sequence's units a head; sums over the threads'
        auto sums = [&](int base) {
            one = 0;
            if (base + tid < a.at.seqs) {
                const Seq s(a, base + tid);
                for (int t = 0; t * ROWS < s.rows; ++t) one += Keys(f, s, t).cost();
            }
            upto = scan<NW>(one * a.kv_heads, room, &sum);
        };
        for (int base = 0; base < a.at.seqs; base += 64 * NW) {
            sums(base);
            total += sum;
        }
        total = uniform(total);
        wgs = (int)min((int64_t)f.groups, max(total / SHARE, (int64_t)1));
        if (total == 0 || wg >= wgs) {
            if (f.split && tid == 0) cuts_of(f)[wg] = Cut{-1, 0, 0, 0};
            return;
        }
        cut0 = total * wg / wgs;
        left = total * (wg + 1) / wgs - cut0;
        int64_t before = 0;
        int base = 0;
        for (;; base += 64 * NW) {
            if (a.at.seqs > 64 * NW) sums(base);
            if (cut0 < before + sum || base + 64 * NW >= a.at.seqs) break;
            before += sum;
        }
        const int64_t in = cut0 - (before + upto - one * a.kv_heads);
        if (in >= 0 && in < one * a.kv_heads) {
            const int64_t head = (in | one) >> 32 ? in / one : (int64_t)((uint32_t)in / (uint32_t)one);
            room[NW] = base + tid;
            room[NW + 1] = head;
            room[NW + 2] = in - head * one;
        }
        __syncthreads();
        b = uniform((int)room[NW]);
        hk = uniform((int)room[NW + 1]);
        u = uniform(room[NW + 2]);
        __syncthreads();
    }
    int tile = 0;
    Seq seq = Seq::shared(a, b);
    while (u >= Keys(f, seq, tile).cost()) u -= Keys(f, seq, tile++).cost();
    if (f.split) {
        const Keys k(f, seq, tile);
        Cut cut{-1, b, hk, tile};
        const int at = k.cut(u, true);
        if (wg > 0 && at > 0 && at < k.length() && k.cut(total * (wg - 1) / wgs - cut0 + u, true) == 0) {
            // the workgroup of the item's last unit, unless its share's begin is moved to the end
            const int64_t begin = cut0 - u, end = begin + k.cost();
            int64_t w = min((int64_t)wgs - 1, (end - 1) * wgs / total);
            while (w + 1 < wgs && total * (w + 1) / wgs < end) ++w;
            while (total * w / wgs >= end) --w;
            if (k.cut(total * w / wgs - begin, true) == k.length()) --w;
            cut.last = (int)w;
        }
        if (tid == 0) cuts_of(f)[wg] = cut;
    }

    const uint16_t *const K0 = static_cast<const uint16_t *>(a.kc.p);
    const uint16_t *const V0 = static_cast<const uint16_t *>(a.vc.p);
    // a lane's place in a load's rows (DMA)
    const int row_of = lane / Tile::CPR, chunk = (lane % Tile::CPR) ^ Tile::swz(row_of);
    const int place_k = chunk * 8 < a.d ? (row_of * (int)a.kc.ld + chunk * 8) * 2 : OOB;
    const int place_v = chunk * 8 < a.d ? (row_of * (int)a.vc.ld + chunk * 8) * 2 : OOB;

    while (left > 0) {
        const Keys k(f, seq, tile);
        const int64_t until = min((int64_t)k.cost(), u + left);
        const int s0 = k.cut(u, f.split), s1 = k.cut(until, f.split);
        if (s0 < s1) {
            const bool whole = s0 == 0 && s1 == k.length();
            const int end1 = min(s1, k.steps);
            const int row0 = tile * ROWS, row = row0 + wr * 32 + (lane & 31);
            const bool valid = row < seq.rows;
            const int i = f.group(valid ? row : seq.rows - 1);
            const int g = (valid ? row : seq.rows - 1) - i * a.group;
            const int64_t head = (int64_t)hk * a.group + g;
            const int64_t at_row = seq.at.first + i;
            const bool live = valid && i < seq.at.n;      // rows past a sequence's read nothing
            FwdRows<S> w(lds0 + kg * KT / Tile::RPS * Tile::SEG, lane, a.scale, seq.lo(a, i),
                         live ? seq.hi(a, i) : 0);
            const auto reader = w.rd;
            const uint16_t *Q = static_cast<const uint16_t *>(a.q.p) + seq.at.batch * a.q.sb +
                                head * a.q.sh + at_row * a.q.ld;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                w.qf[ks] = row_frag<DMA>(Q, ks * 16 + 8 * half, live ? a.d : 0);
            settle(w.qf);
            const bool idle = !__any(live);               // a wave without rows only loads
            // steps whose keys every row of the tile sees
            const int all = min(seq.hi(a, k.first), seq.lk);
            const int nb = min(k.steps, max(0, all - k.beg) / KEYS);
            const int na = min(nb, max(0, seq.lo(a, k.last) - k.beg + KEYS - 1) / KEYS);
            const uint16_t *const K = K0 + hk * a.kc.sh, *const V = V0 + hk * a.vc.sh;

            // as many steps at a time as their pages' numbers have room
            const int some = max(1, (int)min((int64_t)(PAGES_AT_ONCE - 2) * a.at.page / KEYS, (int64_t)1 << 24));
            for (int sa = s0; sa < end1;) {
                const int sb = min(end1, sa + some), n = sb - sa;
                const int k_beg = k.beg + sa * KEYS;
                const int page0 = f.page(k_beg);
                const int count = f.page(min(k_beg + n * KEYS, k.end) - 1) - page0 + 1;
                bool bad = false;
                for (int x = tid; x < count; x += 64 * NW) {
                    int e = -1;
                    if ((page0 + x + 1) * a.at.page > k.lo) {
                        e = a.at.table[b * a.at.table_ld + page0 + x];
                        if (e < 0 || e >= a.at.pages) {
                            e = -1;
                            bad = true;
                        }
                    }
                    numbers[x] = e;
                }
                if (lane == 0) missing[wave] = 0;
                if (__any(bad) && lane == 0) missing[wave] = 1;
                wait_vm<0>();        // stores of an earlier item too: the loads below are counted
                __syncthreads();
                int holes = 0;
#pragma unroll
                for (int x = 0; x < NW; ++x) holes |= missing[x];
                holes = __builtin_amdgcn_readfirstlane(holes);
                Walk walk{n, min(max(na - sa, 0), n), min(max(nb - sa, 0), n)};
                if (holes) walk.na = walk.nb = n;     // in order
                w.rd = reader;
                w.stage = 0;

                // Loads of the step that is x-th in the walk: on DMA, the page of each load's rows
                // is read from LDS one step ahead.
                auto key0 = [&](int x) { return k_beg + walk.step(x) * KEYS; };
                int32_t next[NV];
                i32x4 to_k[NV], to_v[NV];
                int skip[NV];                // rows of a load in front of what is seen
                uint32_t to = 0;
                typename Tile::Regs rk, rv;
                auto look = [&](int x) __attribute__((always_inline)) {
#pragma unroll
                    for (int j = 0; j < NV; ++j) {
                        const int p = f.page(key0(x) + (j * NW + wave) * Tile::RPS) - page0;
                        next[j] = numbers[min(max(p, 0), PAGES_AT_ONCE - 1)];
                    }
                };
                auto fetch = [&](int x, int stage) __attribute__((always_inline)) {
                    if constexpr (DMA) {
#pragma unroll
                        for (int j = 0; j < NV; ++j) {
                            const int key = key0(x) + (j * NW + wave) * Tile::RPS;
                            const int p = __builtin_amdgcn_readfirstlane(next[j]);
                            const int at = key - f.page(key) * a.at.page;
                            const int m = x < n && p >= 0 ? min(Tile::RPS, max(0, k.end - key)) : 0;
                            to_k[j] = make_rsrc(K + p * a.kc.sb + at * a.kc.ld);
                            to_v[j] = make_rsrc(V + p * a.vc.sb + at * a.vc.ld);
                            to_k[j][2] = __builtin_amdgcn_readfirstlane(m * (int)a.kc.ld * 2);
                            to_v[j][2] = __builtin_amdgcn_readfirstlane(m * (int)a.vc.ld * 2);
                            skip[j] = k.lo - key;
                        }
                        to = lds0 + stage * S::STAGE;
                        look(x + 1);
                    } else {
                        auto load = [&](typename Tile::Regs &v, const uint16_t *base, const CoreView &c) {
#pragma unroll
                            for (int j = 0; j < NV; ++j) {
                                const int q = j * 64 * NW + tid;
                                const int key = key0(x) + q / Tile::CPR, col = q % Tile::CPR * 8;
                                v[j] = u32x4{0u, 0u, 0u, 0u};
                                if (key < k.lo || key >= k.end || col >= a.d) continue;
                                const int p = f.page(key), e = numbers[p - page0];
                                if (e < 0) continue;
                                const uint16_t *r = base + e * c.sb + (key - p * a.at.page) * c.ld;
                                v[j] = col + 8 <= a.d ? ld16_any(r + col) : ld16_tail(r, col, a.d);
                            }
                        };
                        load(rk, K, a.kc);
                        load(rv, V, a.vc);
                    }
                };
                auto part = [&](int q) __attribute__((always_inline)) {
                    if constexpr (DMA) {
                        const int j = q < NV ? q : q - NV;
                        const uint32_t lds = to + (j * NW + wave) * Tile::SEG;
                        const int out = row_of < skip[j] ? OOB : 0;
                        if (q < NV) dma16_at(to_k[j], lds, place_k | out);
                        else dma16_at(to_v[j], lds + Tile::BYTES, place_v | out);
                    }
                };
                auto arrive = [&](int stage) {
                    if constexpr (!DMA) {
                        char *lds = smem + stage * S::STAGE;
                        Tile::store(rk, lds, tid);
                        Tile::store(rv, lds + Tile::BYTES, tid);
                    }
                };
                auto after = [&]() { return w.stage == NS - 1 ? 0 : w.stage + 1; };
                auto advance = [&](int x) __attribute__((always_inline)) {
                    if constexpr (DMA) {
                        wait_vm<(NS - 3) * S::LOADS>();
                        __syncthreads();
                        fetch(x + NS - 1, w.stage == 0 ? NS - 1 : w.stage - 1);
                    } else {
                        if (x + 1 < n) arrive(after());
                        __syncthreads();
                        if (x + 2 < n) fetch(x + 2, 0);
                    }
                };
                if constexpr (DMA) {
                    look(0);
#pragma unroll
                    for (int x = 0; x < NS - 1; ++x) {
                        fetch(x, x);
#pragma unroll
                        for (int p = 0; p < S::LOADS; ++p) part(p);
                    }
                    fetch(n, NS - 1);        // nothing, for the parts before the first advance
                    look(NS - 1);
                    wait_vm<(NS - 2) * S::LOADS>();
                } else {
                    fetch(0, 0);
                    arrive(0);
                    if (1 < n) fetch(1, 1);
                }
                __syncthreads();
                // where a page is missing, the lanes look up the block's keys
                auto seen = [&](int k0) __attribute__((always_inline)) {
                    uint32_t bits = w.range(k0);
                    if (holes) {
                        const int p = f.page(min(k0 + (lane & 31), k.end - 1)) - page0;
                        bits &= (uint32_t)__ballot(numbers[min(max(p, 0), PAGES_AT_ONCE - 1)] >= 0);
                    }
                    return bits >> (4 * half);
                };
                auto mine = [&](int x) { return key0(x) + kg * KT; };
                auto take = [&](int x, auto edge) __attribute__((always_inline)) {
                    w.template take<decltype(edge)::value>(
                        mine(x), mine(x + 1), x + 1 < n, seen,
                        [&]() __attribute__((always_inline)) { advance(x); }, part);
                };
                if (idle) {
                    for (int x = 0; x < n; ++x) {
                        advance(x);
#pragma unroll
                        for (int p = 0; p < S::LOADS; ++p) part(p);
                        w.stage = after();
                    }
                } else {
                    w.begin(mine(0), seen);
                    int x = 0;
                    for (; x < min(n, walk.masked()); ++x) take(x, std::true_type{});
                    for (; x < n; ++x) take(x, std::false_type{});
                }
                wait_vm<0>();      // no load is on its way to LDS any more
                __syncthreads();
                sa = sb;
            }

            const float mul = w.join_groups(reinterpret_cast<float *>(smem + S::PUT) + lane, wave, wr);
            const float m = w.m, l = w.l;
            // a row that sees no key: O = 0, lse = -infinity
            const bool some_key = live && l != 0.f;
            const int64_t slot = (2 * (int64_t)wg + (s0 > 0 ? 0 : 1)) * f.slot_rows + (row - row0);
            const RowsOut out{whole ? a.o.p : parts_of(f), whole ? a.d : (int)d4, !whole || a.o_f32,
                              false, !whole || f.vec};
            const int64_t off = !valid ? -1
                                : whole ? seq.at.batch * a.o.sb + head * a.o.sh + at_row * a.o.ld
                                        : slot * d4;
            float *const put = reinterpret_cast<float *>(smem);
            stage_rows<DP>(put + wave * PUT_FLOATS<DP>, w.o, some_key ? mul / l : 0.f, lane);
            if (valid && half == 0 && kg == 0) {
                if (!whole)
                    stats_of(f)[slot] = some_key ? f32x2{m, l} : f32x2{-INFINITY, 0.f};
                else if (a.lse.p)
                    static_cast<float *>(a.lse.p)[seq.at.batch * a.lse.sb + head * a.lse.sh +
                                                  at_row * a.lse.ld] =
                        some_key ? __builtin_fmaf(m, a.scale, __builtin_amdgcn_logf(l) * LN2) : -INFINITY;
            }
            __syncthreads();
            store_rows<DP, KG>(put + wr * KG * PUT_FLOATS<DP>, PUT_FLOATS<DP>, kg, out, off, lane);
            __syncthreads();       // before the next item's loads
        }
        left -= until - u;
        u = 0;
        if (left <= 0) break;
        if (++tile * ROWS >= seq.rows) {
            tile = 0;
            if (++hk == a.kv_heads) {
                hk = 0;
                do {
                    if (++b >= a.at.seqs) return;
                    seq = Seq::shared(a, b);
                } while (seq.rows == 0);
            }
        }
    }
}

// Joins the parts of the items that were cut, in their order: weights l_s 2^((m_s - m) c). Workgroup
// (x, y) takes row block y of the item that workgroup x + 1 continues. A row's LANES threads own 4
// columns each, SHARES threads a column's parts in turn.
template <int LANES, int SHARES>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedLaunch f, int rows_of_tile) {
    constexpr int AT_ONCE = 256 / (LANES * SHARES);
    __shared__ float room[256][6];
    const PagedArgs &a = f.a;
    const int w = blockIdx.x + 1;
    const Cut cut = cuts_of(f)[w];
    if (cut.last < 0) return;
    const int tid = threadIdx.x, lane = tid % LANES, share = tid / LANES % SHARES;
    const int in = blockIdx.y * AT_ONCE + tid / (LANES * SHARES);
    const Seq seq(a, cut.seq);
    const int row = cut.tile * rows_of_tile + in, col = lane * 4;
    const bool valid = in < f.slot_rows && row < seq.rows && col < a.d;
    const int64_t d4 = (a.d + 3) & ~3;
    const float c = a.scale * LOG2E;
    const int n = cut.last - w + 2;
    float top = -INFINITY, sum = 0.f;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (valid)
        for (int s = share; s < n; s += 4 * SHARES) {      // 4 reads on their way together
            f32x2 z[4];
            f32x4 x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = s + j * SHARES;
                const int64_t slot = (2 * (int64_t)(w - 1 + k) + (k ? 0 : 1)) * f.slot_rows + in;
                z[j] = k < n ? stats_of(f)[slot] : f32x2{-INFINITY, 0.f};
                x[j] = k < n ? *reinterpret_cast<const f32x4 *>(parts_of(f) + slot * d4 + col)
                             : f32x4{0.f, 0.f, 0.f, 0.f};
            }
            float high = top;
#pragma unroll
            for (int j = 0; j < 4; ++j) high = fmaxf(high, z[j][0]);
            const float base = high == -INFINITY ? 0.f : high;
            const float old = exp2_((top - base) * c);
            sum *= old;
            v *= old;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float e = z[j][1] * exp2_((z[j][0] - base) * c);
                sum += e;
                v += x[j] * e;
            }
            top = high;
        }
    if constexpr (SHARES > 1) {
        room[tid][0] = top;
        room[tid][1] = sum;
#pragma unroll
        for (int e = 0; e < 4; ++e) room[tid][2 + e] = v[e];
        __syncthreads();
        if (share) return;
        float high = top;
#pragma unroll
        for (int s = 1; s < SHARES; ++s) high = fmaxf(high, room[tid + s * LANES][0]);
        const float base = high == -INFINITY ? 0.f : high;
        sum = 0.f;
        v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < SHARES; ++s) {
            const float *const p = room[tid + s * LANES];
            const float e = exp2_((p[0] - base) * c);
            sum += p[1] * e;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] += p[2 + j] * e;
        }
        top = high;
    }
    if (!valid) return;
    const bool some = sum != 0.f;
    const float inv = some ? 1.f / sum : 0.f;
    const int i = f.group(row);
    const int64_t head = (int64_t)cut.head * a.group + (row - i * a.group), at = seq.at.first + i;
    store4(a.o.p, seq.at.batch * a.o.sb + head * a.o.sh + at * a.o.ld, col, a.d, a.o_f32, f.vec,
           [&](int e) { return v[e] * inv; });
    if (a.lse.p && col == 0)
        static_cast<float *>(a.lse.p)[seq.at.batch * a.lse.sb + head * a.lse.sh + at * a.lse.ld] =
            some ? __builtin_fmaf(top, a.scale, __builtin_amdgcn_logf(sum) * LN2) : -INFINITY;
}

}  // namespace sbpk

namespace sbpi {

namespace {

template <int DP, int KG, int KT, int NW, int WPS>
hipError_t launch(const sbpk::PagedLaunch &f, bool dma, hipStream_t s) {
    char name[160];
    name[0] = 0;
    if (profiling())
        snprintf(name, sizeof(name), "paged_attn_kernel<%d,%d,%d,%d,%d>", DP, KG, KT, NW, (int)dma);
    const dim3 grid((unsigned)f.groups), block(64 * NW);
    if (dma)
        return launch_kernel(sbpk::paged_attn_kernel<DP, KG, KT, NW, WPS, true>, name, grid, block, s, f);
    return launch_kernel(sbpk::paged_attn_kernel<DP, KG, KT, NW, WPS, false>, name, grid, block, s, f);
}

// The kernel's forms: rows of a tile, keys of a step, workgroups of a unit, us of a step.
struct Form {
    int rows, keys, per_cu;
    double step;
};
constexpr Form FORMS[2][3] = {{{128, 64, 2, 0.9}, {64, 64, 2, 0.55}, {32, 128, 1, 0.6}},
                              {{256, 64, 1, 1.4}, {128, 64, 1, 1.0}, {64, 64, 1, 0.75}}};

}  // namespace

hipError_t launch_paged(const PagedArgs &a, hipStream_t s) {
    sbpk::PagedLaunch f;
    f.a = a;
    const int esz = a.o_f32 ? 4 : 2;
    f.vec = a.d % 4 == 0 && reinterpret_cast<uintptr_t>(a.o.p) % (4 * esz) == 0 &&
            a.o.ld % 4 == 0 && a.o.sb % 4 == 0 && a.o.sh % 4 == 0;
    f.page = sbpk::Div(a.at.page);
    f.group = sbpk::Div(a.group);
    const bool wide = a.d > 64;
    // tiles of a key head, at most; the form that takes the least time for a key of all of them
    const int64_t rows = (int64_t)a.at.rows * a.group;
    int form = 0;
    double best = 1e300;
    for (int k = 0; k < 3; ++k) {
        const Form &m = FORMS[wide][k];
        const double tiles = a.at.row_q ? (double)(rows / m.rows) + a.at.seqs
                                        : (double)((rows + m.rows - 1) / m.rows) * a.at.seqs;
        const double t = tiles * m.step / (m.keys * m.per_cu);
        if (t < best) best = t, form = k;
    }
    const Form &m = FORMS[wide][form];
    f.slot_rows = (int32_t)std::min<int64_t>(m.rows, rows);
    const int64_t most = (int64_t)device_cus() * m.per_cu;
    const int64_t each = 4 + 2 * sbpk::slot_floats(f.slot_rows, a.d);
    // with a workspace for half of the workgroups items may be cut
    const int64_t room = (int64_t)(a.ws_floats / (size_t)each);
    f.split = room >= most / 2;
    f.groups = (int32_t)(f.split ? std::min(room, most) : most);
    // rows of one load lie on one page
    const int per_load = wide ? 4 : 8;
    const bool dma = a.aligned && a.at.page % per_load == 0;
    hipError_t e;
    if (form == 0)
        e = wide ? launch<128, 1, 64, 8, 2>(f, dma, s) : launch<64, 1, 64, 4, 2>(f, dma, s);
    else if (form == 1)
        e = wide ? launch<128, 2, 32, 8, 2>(f, dma, s) : launch<64, 2, 32, 4, 2>(f, dma, s);
    else
        e = wide ? launch<128, 2, 32, 4, 1>(f, dma, s) : launch<64, 4, 32, 4, 1>(f, dma, s);
    if (e != hipSuccess || !f.split || f.groups < 2) return e;
    auto join = [&](auto kernel, int at_once) {
        const dim3 grid((unsigned)(f.groups - 1), (unsigned)((f.slot_rows + at_once - 1) / at_once));
        return launch_kernel(kernel, "paged_join_kernel", grid, dim3(256), s, f, m.rows);
    };
    if (form == 2)    // few rows, perhaps of many parts
        return wide ? join(sbpk::paged_join_kernel<32, 4>, 2) : join(sbpk::paged_join_kernel<16, 4>, 4);
    return wide ? join(sbpk::paged_join_kernel<32, 1>, 8) : join(sbpk::paged_join_kernel<16, 1>, 16);
}

}  // namespace sbpi
