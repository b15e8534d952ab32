// paged_attn.hip -- softmax attention of new tokens over a paged cache.
//
// The walk over a tile's keys is that of whole sequences (attn_core_walk.h): rows of a group of
// query heads packed as row = i * group + g, S^T = K Q^T, running maximum and sum, O^T += V^T P^T,
// stages of keys and values on their way to LDS. What differs:
//
//   * Work. Lengths are known on the device only, and differ: a token of one sequence beside a
//     prompt of another. The items (sequence, key head, tile of rows), each as long as its steps
//     of keys and a fixed part, are laid end to end, and as many workgroups as the chip holds
//     take equal shares of that line, whatever the lengths are (as many as the workspace has room
//     for the partial outputs of: of 64 MiB 252 of 256 with tiles of 256 rows of 128). Every wave finds
//     its share by the same sums over the sequences, a lane each, 64 at a time, which then take over 1
//     us for each 64 (2^17 keys in all, 8 heads over 1 of 128: one token of 64 sequences 20 us, of
//     256 26, of 1024 43). An item that is cut leaves partial outputs in the workspace, two at most
//     for each workgroup, and a second kernel joins them in order.
//   * Pages. The numbers of up to PAGES_AT_ONCE pages of a walk are brought to LDS. Rows of a load
//     of one wave (1 KB: 4 or 8) lie on one page where the page's tokens are a multiple of them,
//     so that a load is a buffer of its own, whose address is scalar arithmetic and whose end is
//     the last row that is seen; other pages, and rows that allow no 16-byte loads, pass through
//     registers.
//   * Rows that the tile does not see, and pages that do not exist, arrive as zeros; a walk with
//     such a page masks every step, and looks the keys' pages up.
//
// Few rows are bound by memory: one token of 32 sequences of up to 32768 keys, 64 heads over 8 of
// 128, takes 463 us, 5.9 TB/s (560 with a step's addresses made at once behind its barrier, 610
// with the arguments kept in registers through all items too). Many are bound by the step of 64 keys
// (2.0 us for 256 rows of 128): a chunk of 2048 of 16 heads over 4, 65536 keys, 1000 us, 1.08 PFLOP/s,
// with pages of 16 tokens as with one page of all (the same keys in one piece, attn_core_fwd.hip: 920).
// Rows that pass through registers are slower: chunks of 512 of 4 sequences, 16 heads over 4, up to
// 8192 x 128, 222 us with pages of 17 tokens and 136 with 16; one token of 32 sequences, 64 heads over
// 8, 4096 x 128, 234 and 106. A workgroup's second item costs it 5 to 8 us until its keys flow again.
#include <math.h>

#include <algorithm>

#include "attn_core_walk.h"
#include "gemm.h"
#include "paged_kernel.h"
#include "paged_plan.h"
#include "profile.h"

namespace sbpk {

using sbpi::has_share;
using sbpi::PagedArgs;
using sbpi::slot_of;

constexpr int PAGES_AT_ONCE = 1024;
constexpr int SHORTEST = 2;          // steps that a cut leaves on either side

// What workgroup w leaves for the join where its share begins inside an item that workgroup
// w - 1 began: the item's parts are those of w - 1 .. last (slot_of). Else last < 0.
struct Cut {
    int32_t last, head, row;         // first packed row of the tile
    int32_t batch, first, rows;      // of its sequence
    int32_t parts, spare;            // whether the line's units are parts
};
static_assert(sizeof(Cut) == 4 * sbpi::CUT_FLOATS, "a cut's place in the workspace");

struct PagedLaunch {
    PagedArgs a;
    int32_t slot_rows;               // rows of a partial output
    int32_t split;                   // items may be cut
    int32_t vec;                     // O allows 4-value stores
    int32_t runs;                    // O's rows are bf16 runs of 8 columns
    int32_t groups, slots;           // workgroups, partial outputs that the workspace holds
    int32_t fixed, scale;            // an item's fixed part in steps; a unit has 2^scale steps
    Div page, group, by_half;        // by_half: workgroups with two partial outputs each
};

// The line of items. Its units are steps (`fixed` more an item), or equal parts of items, a part a
// workgroup: an item of n steps has 1 + floor((n - 1) per). Parts are taken where they are no more
// than the workgroups though hardly longer than shares of steps: no workgroup then has a second
// item to begin, and an item's parts begin and end where its neighbours' do, so that keys that one
// workgroup reads are in the L2 for others (a chunk of 2048 of 16 heads over 4, 65536 keys: 1039 us
// in shares of steps, 1009 in two parts an item; one token of 16 sequences of 32 heads over 2, 8192
// x 64: 27.3 and 24.4 with the join).
struct Line {
    int32_t share;                   // units of a workgroup
    float per;                       // 0: units are steps
};

// A value that all lanes have, in a scalar register: the compiler keeps what it loads in vector
// registers, and all that follows from it.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// The workspace: cuts, statistics (a row's maximum and sum), partial outputs.
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ Cut *cuts_of(const PagedLaunch &f) { return reinterpret_cast<Cut *>(f.a.ws); }
__device__ __forceinline__ f32x2 *stats_of(const PagedLaunch &f) {
    return reinterpret_cast<f32x2 *>(f.a.ws + sbpi::stats_at(f.groups));
}
__device__ __forceinline__ float *parts_of(const PagedLaunch &f) {
    return f.a.ws + sbpi::parts_at(f.groups, f.slots, f.slot_rows);
}
// Workgroups that may have partial outputs.
__device__ __forceinline__ int holders_of(const PagedLaunch &f, bool parts) {
    return parts ? f.groups : (int)f.by_half.d;
}

// A sequence: its rows (packed ones of the group: `rows`, of which those of n queries are in use),
// and its keys.
struct Seq {
    SeqRows at;
    int rows, lk, off;
    __device__ __forceinline__ Seq(const PagedArgs &a, const SeqRows &r) : at(r) {
        rows = (a.at.row_q ? at.n : a.at.rows) * a.group;
        lk = min(max(at.len, 0), a.at.width * a.at.page);
        off = lk - at.n;
    }
    // The sequence that a whole workgroup works on.
    __device__ __forceinline__ static Seq shared(const PagedArgs &a, int b) {
        const SeqRows r = rows_of(a.at, b);
        return Seq(a, SeqRows{a.at.row_q ? 0 : b, uniform(r.first), uniform(r.n), uniform(r.len)});
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
        steps = end > lo ? (int)((uint32_t)(end - beg + KEYS - 1) / KEYS) : 0;
    }
    // An item without steps counts as one: its rows are cleared.
    __device__ __forceinline__ int length() const { return max(steps, 1); }
    __device__ __forceinline__ int cost(const PagedLaunch &f, const Line &line) const {
        if (line.per != 0.f) return 1 + (int)((float)(length() - 1) * line.per);
        return f.fixed + ((length() + (1 << f.scale) - 1) >> f.scale);
    }
    // Where a cut u units into the item falls: it ends one part and begins the other.
    __device__ __forceinline__ int cut(const PagedLaunch &f, const Line &line, int u) const {
        const int c = cost(f, line), n = length();
        if (u <= 0) return 0;
        if (u >= c) return n;
        if (line.per != 0.f) return (int)((float)u * ((float)n / (float)c));    // c <= n: grows with u
        const int s = (u - f.fixed) << f.scale;
        if (!f.split) return 2 * s < n ? 0 : n;
        return s < SHORTEST ? 0 : n - s < SHORTEST ? n : s;
    }
};

// Sum of x over this lane and those before it.
__device__ __forceinline__ int upto_lane(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);    // 1, 2, 4, 8 lanes up
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);    // lanes 15 and 47, then 31
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}

// Where a partial output of one wave group lies in its slot: the registers' order, quads of columns
// 8 t + 4 (lane / 32) .. + 3 of row 32 wr + lane % 32 side by side for a wave's lanes.
template <int DP>
__device__ __forceinline__ int part_place(int wr, int t, int lane) {
    return ((wr * (DP / 8) + t) * 64 + lane) * 4;
}

// Stores a wave's 32 rows (lane l has row l % 32, at element `off` of the output or < 0 for none; o as
// for stage_rows), times `mul` (0 where that is 0), as bf16 in 16 bytes a lane, through a tile of its
// own in LDS, which the wave reads in the order it wrote. (As fp32 and in 8 bytes, as the
// wave groups of a row need it, 256 rows of 128 took 3.4 us; 60 prompts of 500 rows of 16 heads over 4
// of 64 112 us and so 108.)
template <int DP, int DC>
__device__ __forceinline__ void store_runs(char *tile, const f32x16 *o, float mul, uint16_t *out, int d,
                                           int64_t off, int lane) {
    typedef u32x4 u32x4_any __attribute__((aligned(2)));
    constexpr int PITCH = DC * 2 + 16, RUNS = DP / 8;
    static_assert(31 * PITCH + DP * 2 <= PUT_FLOATS<DP> * 4, "a wave's tile");
    char *const row = tile + (lane & 31) * PITCH + 8 * (lane >> 5);
#pragma unroll
    for (int t = 0; t < DC / 8; ++t) {
        auto value = [&](int e) {
            const float v = o[t / 4][t % 4 * 4 + e];
            return (uint32_t)f32_to_bf16_bits(mul != 0.f ? v * mul : 0.f);
        };
        *reinterpret_cast<u32x2 *>(row + 16 * t) = u32x2{value(0) | value(1) << 16, value(2) | value(3) << 16};
    }
    asm volatile("" ::: "memory");
    const int run = lane % RUNS, lo = (int)off, hi = (int)(off >> 32);
#pragma unroll
    for (int it = 0; it < RUNS / 2; ++it) {
        const int r = lane / RUNS + it * (64 / RUNS);
        const u32x4 v = *reinterpret_cast<const u32x4 *>(tile + r * PITCH + run * 16);
        const int h = __builtin_amdgcn_ds_bpermute(4 * r, hi), l = __builtin_amdgcn_ds_bpermute(4 * r, lo);
        if (h >= 0 && run * 8 < d)
            *reinterpret_cast<u32x4_any *>(out + (int64_t)((uint64_t)(uint32_t)h << 32 | (uint32_t)l) +
                                           run * 8) = v;
    }
}

// The kernel's arguments, to be read again: what the compiler reads before a loop of items it keeps
// through all of them, spilled from scalar to vector registers.
__device__ __forceinline__ const PagedLaunch &again() {
    uint64_t p = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const PagedLaunch *)(const __attribute__((address_space(4))) PagedLaunch *)p;
}

template <int DP, int KG, int KT, int NW, int WPS, bool DMA, int DC>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(WPS, WPS)))
void paged_attn_kernel(PagedLaunch f0) {
    const PagedLaunch &f = f0;
    using S = FwdShape<DP, KG, KT, NW, WPS, DMA, DC>;
    using Tile = typename S::Tile;
    constexpr int ROWS = S::ROWS, NS = S::NS, KEYS = S::KEYS, KS = DC / 16, NV = Tile::NV;
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
    // the arguments' lines, read at once: each first read of one is a trip to memory
    asm volatile("" ::"s"(a.at.table), "s"(a.at.len_k), "s"(a.at.rows), "s"(a.q.sh), "s"(a.kc.p),
                 "s"(a.vc.p), "s"(a.o.p), "s"(a.lse.p), "s"(a.kv_heads), "s"(a.d), "s"(a.ws),
                 "s"(f.slot_rows), "s"(f.fixed), "s"(f.by_half.m));
    const int wg = remap_xcd(blockIdx.x, f.groups);    // neighbours on the line share an L2
    if (f.split && tid == 0) cuts_of(f)[wg].last = -1;

    // This workgroup's part of the line: `left` units from unit u of tile `tile` of head hk of
    // sequence b on. Every wave adds up the sequences by itself, a lane each. (Units fit 31 bits:
    // the launch chooses their scale.)
    int left, u, b = 0, hk, tile = 0;
    Line line{0, 0.f};
    Seq seq(a, SeqRows{0, 0, 0, 0});
    {
        constexpr int FEW = 2;
        SeqRows r{0, 0, 0, 0};
        auto one_of = [&](const SeqRows &r, int base, int l) {    // lane l's sequence
            return Seq(a, SeqRows{a.at.row_q ? 0 : base + l, __builtin_amdgcn_readlane(r.first, l),
                                  __builtin_amdgcn_readlane(r.n, l), __builtin_amdgcn_readlane(r.len, l)});
        };
        int one, upto, sum, at = 0;      // units of a head of the lane's sequence; sums
        // 64 sequences at a time: first all, for the total; then, where parts are tried, the (64 at
        // most) again; else on until the share's begin. (One loop, so that its code,
        // run cold, is fetched once.)
        enum { TOTAL, PARTS, FIND } pass = TOTAL;
        int steps_one = 0, steps_upto = 0, steps_total = 0, steps_share = 0;
        for (int total = 0;;) {
            const bool in = b + lane < a.at.seqs;
            r = SeqRows{0, 0, 0, 0};
            if (in) r = rows_of(a.at, b + lane);
            const Seq s(a, r);
            const int tiles = in ? (s.rows + ROWS - 1) / ROWS : 0;
            // a lane its own sequence's tiles, one after the other, where that is not for a few long
            // sequences' sake; the further tiles the wave, one sequence after the other, which
            // takes as long for one as a lane for 3 tiles (32 prompts of 300 rows of 16 heads over 4 of
            // 128: 64 us with only two tiles a lane, 55)
            const int longer = __builtin_popcountll(__ballot(tiles > FEW)), at_most = 3 * longer;
            const int own = 2 * __builtin_popcountll(__ballot(tiles > at_most)) <= longer
                                ? max(at_most, FEW) : FEW;
            one = 0;
            for (int t = 0; t < min(tiles, own); ++t) one += Keys(f, s, t).cost(f, line);
            for (uint64_t more = __ballot(tiles > own); more; more &= more - 1) {
                const int l = __builtin_ctzll(more);
                const Seq s = one_of(r, b, l);
                int c = 0;
                for (int t = own + lane; t * ROWS < s.rows; t += 64) c += Keys(f, s, t).cost(f, line);
                c = __builtin_amdgcn_readlane(upto_lane(c), 63);
                if (lane == l) one += c;
            }
            upto = upto_lane(one * a.kv_heads);
            sum = __builtin_amdgcn_readlane(upto, 63);
            if (pass == FIND) {
                if (at < sum || b + 64 >= a.at.seqs) break;
                at -= sum;
                b += 64;
                continue;
            }
            total += sum;
            if (b + 64 < a.at.seqs) {
                b += 64;
                continue;
            }
            if (pass == TOTAL) {
                line.share = f.by_half(max(total - 1, 0)) + 1;
                const int items = __builtin_amdgcn_readlane(upto_lane(tiles), 63) * a.kv_heads;
                // (among many items of many lengths some have just more than so many parts' steps)
                const bool alike = __all(tiles == 0 || one == __builtin_amdgcn_readfirstlane(one));
                if (b == 0 && f.split && f.scale == 0 && (alike ? items < f.groups : 8 * items <= f.groups)) {
                    // parts of 25/24 of an even share, 2 steps at least
                    line.per = min((float)f.groups * 24 / ((float)(total - f.fixed * items) * 25), 1.f / 2);
                    steps_one = one;
                    steps_upto = upto;
                    steps_total = total;
                    steps_share = line.share;
                    pass = PARTS;
                    total = 0;
                    continue;
                }
            } else if (total > f.groups) {     // too many parts: back to steps
                one = steps_one;
                upto = steps_upto;
                total = steps_total;
                line = Line{steps_share, 0.f};
            } else {
                line.share = 1;
            }
            if (!has_share(total, line.share, wg, line.per != 0.f, holders_of(f, false))) return;
            at = line.share * wg;
            left = min(line.share, total - at);
            if (b == 0) break;
            b = 0;
            pass = FIND;
        }
        const int in = at - (upto - one * a.kv_heads);
        const uint64_t here = __ballot(in >= 0 && in < one * a.kv_heads);
        if (!here) return;     // (lengths that changed under way)
        const int l = __builtin_ctzll(here);
        seq = one_of(r, b, l);
        b += l;
        one = __builtin_amdgcn_readlane(one, l);
        u = __builtin_amdgcn_readlane(in, l);
        hk = (int)((uint32_t)u / (uint32_t)one);
        u -= hk * one;
        // the tile, among 64 at a time
        while (seq.rows > ROWS) {
            const int t = tile + lane;
            const int c = t * ROWS < seq.rows ? Keys(f, seq, t).cost(f, line) : 0, up = upto_lane(c);
            const uint64_t in_tile = __ballot(u < up);
            if (in_tile) {
                const int l = __builtin_ctzll(in_tile);
                u -= __builtin_amdgcn_readlane(up - c, l);
                tile += l;
                break;
            }
            u -= __builtin_amdgcn_readlane(up, 63);
            if ((tile += 64) * ROWS >= seq.rows) return;      // (as above)
        }
    }
    // a lane's place in a load's rows (DMA)
    const int row_of = lane / Tile::CPR, chunk = (lane % Tile::CPR) ^ Tile::swz(row_of);
    const int place_k = chunk * 8 < a.d ? (row_of * (int)a.kc.ld + chunk * 8) * 2 : OOB;
    const int place_v = chunk * 8 < a.d ? (row_of * (int)a.vc.ld + chunk * 8) * 2 : OOB;

    for (bool noted = !f.split; left > 0;) {
        const PagedLaunch &f = again();
        const PagedArgs &a = f.a;
        const Keys k(f, seq, tile);
        const int until = min(k.cost(f, line), u + left);
        const int s0 = k.cut(f, line, u), s1 = k.cut(f, line, until);
        // The share's begin, for the join: noted while the first loads are on their way (and stored
        // before those to LDS, which are counted).
        auto note = [&]() {
            noted = true;
            if (s0 > 0 && s0 < k.length() && k.cut(f, line, u - line.share) == 0) {
                // the workgroup of the item's last unit, unless its share's begin is moved to the end
                int w = (int)((uint32_t)(k.cost(f, line) - u - 1) / (uint32_t)line.share);
                if (w > 0 && k.cut(f, line, u + w * line.share) == k.length()) --w;
                if (tid == 0)
                    cuts_of(f)[wg] = Cut{wg + w,       hk,       tile * ROWS,     seq.at.batch, seq.at.first,
                                         seq.rows, line.per != 0.f, 0};
            }
        };
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
            // steps whose keys every row of the tile sees
            const int all = min(seq.hi(a, k.first), seq.lk);
            const int nb = min(k.steps, max(0, all - k.beg) / KEYS);
            const int na = min(nb, max(0, seq.lo(a, k.last) - k.beg + KEYS - 1) / KEYS);
            const uint16_t *const K = static_cast<const uint16_t *>(a.kc.p) + hk * a.kc.sh;
            const uint16_t *const V = static_cast<const uint16_t *>(a.vc.p) + hk * a.vc.sh;

            // as many steps at a time as their pages' numbers have room
            const int some = max(1, (int)min((int64_t)(PAGES_AT_ONCE - 2) * a.at.page / KEYS, (int64_t)1 << 24));
            for (int sa = s0; sa < end1;) {
                const int sb = min(end1, sa + some), n = sb - sa;
                const int k_beg = k.beg + sa * KEYS;
                const int page0 = f.page(k_beg);
                const int count = f.page(min(k_beg + n * KEYS, k.end) - 1) - page0 + 1;
                bool bad = false;
                auto number = [&](int x) {       // of the x-th page; pages before the first row seen aside
                    const bool in = x < count && (page0 + x + 1) * a.at.page > k.lo;
                    return in ? a.at.table[b * a.at.table_ld + page0 + x] : 0;
                };
                int e = number(tid);
                if (!noted) note();
                for (int x = tid; x < count; x += 64 * NW, e = number(x)) {
                    if (e < 0 || e >= a.at.pages) {
                        e = -1;
                        bad = true;
                    }
                    numbers[x] = e;
                }
                if (sa == s0) settle(w.qf);
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

                // Loads of the step that is x-th in the walk. On DMA, the page of each load's rows is
                // read from LDS a step ahead, and a load's descriptor is made where it is issued,
                // beside a product: all of a step's at once after the barrier they were waited for.
                auto key0 = [&](int x) { return k_beg + walk.step(x) * KEYS; };
                int32_t next[NV];            // page of load j's rows, and their place on it
                int slot[NV], rows_left[NV], skip = 0;
                uint32_t to = 0;
                typename Tile::Regs rk, rv;
                auto look = [&](int x) __attribute__((always_inline)) {
                    const int key = key0(x) + wave * Tile::RPS;
                    skip = k.lo - key;
#pragma unroll
                    for (int j = 0; j < NV; ++j) {
                        const int at = key + j * (NW * Tile::RPS), p = f.page(at);
                        next[j] = numbers[min(p - page0, PAGES_AT_ONCE - 1)];
                        slot[j] = at - p * a.at.page;
                        rows_left[j] = x < n ? k.end - at : 0;
                    }
                };
                auto part = [&](int q) __attribute__((always_inline)) {
                    if constexpr (DMA) {
                        const int j = q < NV ? q : q - NV;
                        const CoreView &c = q < NV ? a.kc : a.vc;
                        const int e = uniform(next[j]), ld2 = (int)c.ld * 2;
                        // strides are 16-byte units below 2^32, rows of a page span less than 2^31 bytes
                        const uint64_t at = (uint64_t)(uint32_t)e * (uint32_t)(c.sb >> 3) << 4;
                        i32x4 r = make_rsrc(reinterpret_cast<const char *>(q < NV ? K : V) + at +
                                            (uint32_t)(slot[j] * ld2));
                        r[2] = uniform(e < 0 ? 0 : min(Tile::RPS, max(0, rows_left[j])) * ld2);
                        const int out = row_of < skip - j * (NW * Tile::RPS) ? OOB : 0;
                        dma16_at(r, to + (j * NW + wave) * Tile::SEG + (q < NV ? 0 : Tile::BYTES),
                                 (q < NV ? place_k : place_v) | out);
                    }
                };
                auto fetch = [&](int x, int stage) __attribute__((always_inline)) {
                    if constexpr (DMA) {
                        look(x);
                        to = lds0 + stage * S::STAGE;
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
#pragma unroll 1
                    for (int x = 0; x < NS - 1; ++x) {       // (short code: it is run cold)
                        fetch(x, x);
#pragma unroll
                        for (int p = 0; p < S::LOADS; ++p) part(p);
                    }
                    // nothing, for the parts before the first advance
#pragma unroll
                    for (int j = 0; j < NV; ++j) rows_left[j] = 0;
                    to = lds0 + (NS - 1) * S::STAGE;
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
                w.begin(mine(0), seen);
                int x = 0;
                // a wave without rows only loads (ahead of the loops, which it then passes by: as a
                // branch of theirs, or in place of them, it costs 50 registers and more)
                if (!__any(live))
                    for (; x < n; ++x) {
                        advance(x);
#pragma unroll
                        for (int p = 0; p < S::LOADS; ++p) part(p);
                        w.stage = after();
                    }
                for (; x < min(n, walk.masked()); ++x) take(x, std::true_type{});
                for (; x < n; ++x) take(x, std::false_type{});
                wait_vm<0>();      // no load is on its way to LDS any more
                __syncthreads();
                sa = sb;
            }

            const PagedLaunch &f = again();
            const PagedArgs &a = f.a;
            const float mul = w.join_groups(reinterpret_cast<float *>(smem + S::PUT) + lane, wave, wr);
            const float m = w.m, l = w.l;
            // a row that sees no key: O = 0, lse = -infinity
            const bool some_key = live && l != 0.f;
            const int64_t slot = slot_of(wg, s0 == 0, line.per != 0.f) * f.slot_rows;
            if (KG == 1 && !whole) {
                // as the registers hold it: 16 bytes a lane, 1 KB a store
                if (wr * 32 < f.slot_rows) {
                    const float by = some_key ? 1.f / l : 0.f;
                    float *const at = parts_of(f) + slot * DP + part_place<DP>(wr, 0, lane);
#pragma unroll
                    for (int t = 0; t < DC / 8; ++t) {
                        f32x4 v;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            v[e] = by != 0.f ? w.o[t / 4][t % 4 * 4 + e] * by : 0.f;
                        if (8 * t + 4 * half < a.d) *reinterpret_cast<f32x4 *>(at + t * 256) = v;
                    }
                    if (half == 0)
                        stats_of(f)[slot + wr * 32 + lane] = some_key ? f32x2{m, l}
                                                                      : f32x2{-INFINITY, 0.f};
                }
            } else {
                const RowsOut out{whole ? a.o.p : parts_of(f), whole ? a.d : (int)d4,
                                  !whole || a.o_f32, false, !whole || f.vec};
                const int64_t off = !valid ? -1
                                    : whole ? seq.at.batch * a.o.sb + head * a.o.sh + at_row * a.o.ld
                                            : (slot + row - row0) * d4;
                float *const put = reinterpret_cast<float *>(smem);
                const bool runs = KG == 1 && f.runs;
                if (!runs) stage_rows<DC>(put + wave * PUT_FLOATS<DP>, w.o, some_key ? mul / l : 0.f, lane);
                if (valid && half == 0 && kg == 0) {
                    if (!whole)
                        stats_of(f)[slot + row - row0] = some_key ? f32x2{m, l} : f32x2{-INFINITY, 0.f};
                    else if (a.lse.p)
                        static_cast<float *>(a.lse.p)[seq.at.batch * a.lse.sb + head * a.lse.sh +
                                                      at_row * a.lse.ld] =
                            some_key ? __builtin_fmaf(m, a.scale, __builtin_amdgcn_logf(l) * LN2)
                                     : -INFINITY;
                }
                if (runs) {
                    store_runs<DP, DC>(reinterpret_cast<char *>(put + wave * PUT_FLOATS<DP>), w.o,
                                       some_key ? 1.f / l : 0.f, static_cast<uint16_t *>(a.o.p), a.d, off,
                                       lane);
                } else {
                    __syncthreads();
                    store_rows<DP, KG>(put + wr * KG * PUT_FLOATS<DP>, PUT_FLOATS<DP>, kg, out, off, lane);
                }
                __syncthreads();       // before the next item's loads
            }
        }
        if (!noted) note();
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
// (x, y) takes a piece of the item that workgroup x + 1 continues. DP > 0: the parts lie in the
// registers' order, a wave takes the quads t of 32 rows; else in rows, a row's LANES threads own 4
// columns each, SHARES threads a column's parts in turn.
template <int DP, int LANES, int SHARES>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedLaunch f) {
    __shared__ float room[SHARES > 1 ? 256 : 1][6];
    const PagedArgs &a = f.a;
    const int w = blockIdx.x + 1;
    const Cut cut = cuts_of(f)[w];
    if (cut.last < 0) return;
    const int tid = threadIdx.x;
    int in, col, place = 0, share = 0;
    if constexpr (DP > 0) {
        const int unit = blockIdx.y * 4 + (tid >> 6), wr = unit / (DP / 8), t = unit % (DP / 8);
        in = wr * 32 + (tid & 31);
        col = 8 * t + (tid >> 5 & 1) * 4;
        place = part_place<DP>(wr, t, tid & 63);
    } else {
        in = blockIdx.y * (256 / (LANES * SHARES)) + tid / (LANES * SHARES);
        col = tid % LANES * 4;
        share = tid / LANES % SHARES;
    }
    const int row = cut.row + in;
    const bool valid = in < f.slot_rows && row < cut.rows && col < a.d;
    const int64_t d4 = (a.d + 3) & ~3;
    const float c = a.scale * LOG2E;
    const int n = min(cut.last, holders_of(f, cut.parts) - 1) - w + 2;
    float top = -INFINITY, sum = 0.f;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (valid)
        for (int s = share; s < n; s += 4 * SHARES) {      // 4 reads on their way together
            f32x2 z[4];
            f32x4 x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = s + j * SHARES;
                const int64_t slot = slot_of(w - 1 + k, k == 0, cut.parts) * f.slot_rows;
                const float *const part = parts_of(f) + (DP > 0 ? slot * DP + place
                                                                : (slot + in) * d4 + col);
                z[j] = k < n ? stats_of(f)[slot + in] : f32x2{-INFINITY, 0.f};
                x[j] = k < n ? *reinterpret_cast<const f32x4 *>(part) : f32x4{0.f, 0.f, 0.f, 0.f};
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
    const int64_t head = (int64_t)cut.head * a.group + (row - i * a.group), at = cut.first + i;
    store4(a.o.p, cut.batch * a.o.sb + head * a.o.sh + at * a.o.ld, col, a.d, a.o_f32, f.vec,
           [&](int e) { return v[e] * inv; });
    if (a.lse.p && col == 0)
        static_cast<float *>(a.lse.p)[cut.batch * a.lse.sb + head * a.lse.sh + at * a.lse.ld] =
            some ? __builtin_fmaf(top, a.scale, __builtin_amdgcn_logf(sum) * LN2) : -INFINITY;
}

}  // namespace sbpk

namespace sbpi {

namespace {

template <int DP, int KG, int KT, int NW, int WPS, int DC>
hipError_t launch(const sbpk::PagedLaunch &f, bool dma, hipStream_t s) {
    char name[160];
    name[0] = 0;
    if (profiling())
        snprintf(name, sizeof(name), "paged_attn_kernel<%d,%d,%d,%d,%d>", DP, KG, KT, NW, (int)dma);
    const dim3 grid((unsigned)f.groups), block(64 * NW);
    if (dma)
        return launch_kernel(sbpk::paged_attn_kernel<DP, KG, KT, NW, WPS, true, DC>, name, grid, block, s, f);
    return launch_kernel(sbpk::paged_attn_kernel<DP, KG, KT, NW, WPS, false, DC>, name, grid, block, s, f);
}
template <int DP, int DC>
hipError_t launch(int form, const sbpk::PagedLaunch &f, bool dma, hipStream_t s) {
    constexpr int NW = DP / 16;
    if (form == 0) return launch<DP, 1, 64, NW, 2, DC>(f, dma, s);
    if (form == 1) return launch<DP, 2, 32, NW, 2, DC>(f, dma, s);
    if constexpr (DP > 64) return launch<DP, 1, 32, NW / 2, 2, DC>(f, dma, s);
    return hipErrorInvalidValue;
}

// The kernel's forms: rows of a tile, workgroups of a unit, us of 64 keys, whether a tile's rows have
// one wave each (whose partial outputs lie as the registers hold them). The second gives up speed a
// row for smaller tiles: a chunk of 2048 of 16 heads over 4, 32768 keys, takes 523 and 666 us at 128
// columns, 430 and 568 at 64; chunks of 8 of 8 sequences, 64 heads over 8, 8192 x 128, 57 and 50; one
// token of 16 sequences, 16 heads over 4, up to 4096 x 64, 18 and 17.6. The third, for 128 columns,
// has two workgroups a unit, of which one works while the other begins an item: one token of 64
// sequences, 64 heads over 8, takes 55 us and with it 48 at up to 1000 keys, 91 and 96 at 2000, 292
// and 313 at 8000.
struct Form {
    int rows, per_cu;
    double step;
    bool waves;
};
constexpr Form FORMS[2][3] = {{{128, 2, 1.73, true}, {64, 2, 1.15, false}, {}},
                              {{256, 1, 2.08, true}, {128, 1, 1.34, false}, {128, 2, 2.3, true}}};
constexpr int SHORT = 1536;      // keys of an item, at most, for the third form
// An item's fixed part in steps: 3 and 5 differ where items are short and of many lengths (24 ragged
// prompts of 400, up to 1500 x 64: 138 us and 130; 16 prompts of 2000 x 128: 359 and 348; prompts among
// tokens, windows of 1000: 44.6 and 43.6), by 1 % elsewhere, to either side; 8 is no better.
constexpr int FIXED = 5;

}  // namespace

hipError_t launch_paged(const PagedArgs &a, hipStream_t s) {
    sbpk::PagedLaunch f;
    f.a = a;
    const int esz = a.o_f32 ? 4 : 2;
    f.vec = a.d % 4 == 0 && reinterpret_cast<uintptr_t>(a.o.p) % (4 * esz) == 0 &&
            a.o.ld % 4 == 0 && a.o.sb % 4 == 0 && a.o.sh % 4 == 0;
    f.runs = !a.o_f32 && a.d % 8 == 0;
    f.page = sbpk::Div(a.at.page);
    f.group = sbpk::Div(a.group);
    const bool wide = a.d > 64;
    // tiles of a key head, at most; the form that takes the least time for a key of all of them
    const int64_t rows = (int64_t)a.at.rows * a.group;
    const int64_t keys = std::min<int64_t>((int64_t)a.at.width * a.at.page,
                                           a.window && a.causal ? a.window + 256 / a.group : INT32_MAX);
    const int small = wide && keys <= SHORT ? 2 : 1;
    int form = 0;
    double best = 1e300;
    for (const int k : {0, small}) {
        const Form &m = FORMS[wide][k];
        const double tiles = a.at.row_q ? (double)(rows / m.rows) + a.at.seqs
                                        : (double)((rows + m.rows - 1) / m.rows) * a.at.seqs;
        const double t = tiles * m.step / m.per_cu;
        if (t < best) best = t, form = k;
    }
    const Form &m = FORMS[wide][form];
    // a slot holds the rows that a tile can have (whole waves' in the registers' order)
    const int padded = wide ? 128 : 64;
    f.slot_rows = (int32_t)std::min<int64_t>(m.rows, m.waves ? (rows + 31) / 32 * 32 : rows);
    // with a slot for each workgroup items may be cut; in shares of steps, where a workgroup has two,
    // fewer workgroups have one if the slots are less
    const int64_t most = (int64_t)device_cus() * m.per_cu;
    const int64_t slots = slots_in((int64_t)a.ws_floats, (int)most, f.slot_rows,
                                   m.waves ? padded : (a.d + 3) & ~3);
    f.split = slots >= most;
    f.groups = (int32_t)most;
    f.slots = (int32_t)std::min(slots, 2 * most);
    f.by_half = sbpk::Div(f.split ? f.slots / 2 : f.groups);
    // units of all items, at most: below 2^31
    const double most_tiles = a.at.row_q ? (double)(rows / m.rows) + a.at.seqs
                                         : (double)((rows + m.rows - 1) / m.rows) * a.at.seqs;
    const double steps = (double)a.at.width * a.at.page / 32 + 2;
    f.fixed = FIXED;
    f.scale = 0;
    while (most_tiles * a.kv_heads * (steps / (double)(1 << f.scale) + 1 + FIXED) > 1e9) ++f.scale;
    // rows of one load lie on one page, whose offsets fit the loads' arithmetic
    const int per_load = wide ? 4 : 8;
    const bool dma = a.aligned && a.at.page % per_load == 0 &&
                     std::max(a.kc.sb, a.vc.sb) < int64_t(1) << 35 &&
                     (double)a.at.page * std::max(a.kc.ld, a.vc.ld) < 1073741824.0;
    // up to 96 columns, tiles of 128 with products of 96 (chunks of 512 of 4 sequences, 16 heads over
    // 4, 8192 x 96: 148 us with products of 128, 132; one token of 32 sequences, 64 heads over 8, up
    // to 4096 x 80: 67 and 64)
    const hipError_t e = !wide         ? launch<64, 64>(form, f, dma, s)
                         : a.d <= 96 ? launch<128, 96>(form, f, dma, s)
                                     : launch<128, 128>(form, f, dma, s);
    if (e != hipSuccess || !f.split || f.groups < 2) return e;
    auto join = [&](auto kernel, int pieces) {
        return launch_kernel(kernel, "paged_join_kernel", dim3((unsigned)(f.groups - 1), (unsigned)pieces),
                             dim3(256), s, f);
    };
    if (m.waves) {    // 4 quads of 32 rows a workgroup
        const int pieces = f.slot_rows / 32 * padded / 32;
        return wide ? join(sbpk::paged_join_kernel<128, 1, 1>, pieces)
                    : join(sbpk::paged_join_kernel<64, 1, 1>, pieces);
    }
    auto rows_of = [&](int at_once) { return (f.slot_rows + at_once - 1) / at_once; };
    if (f.slot_rows <= 32)    // perhaps of many parts
        return wide ? join(sbpk::paged_join_kernel<0, 32, 4>, rows_of(2))
                    : join(sbpk::paged_join_kernel<0, 16, 4>, rows_of(4));
    return wide ? join(sbpk::paged_join_kernel<0, 32, 1>, rows_of(8))
                : join(sbpk::paged_join_kernel<0, 16, 1>, rows_of(16));
}

}  // namespace sbpi
