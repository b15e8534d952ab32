// paged_attn.hip -- softmax attention of new tokens over a paged cache.
//
// A wave owns a row of a query head: lane l holds columns l and l + 64, scores are summed over
// the lanes key by key, with the running maximum and sum of the softmax.
#include <math.h>

#include "attn_core_kernel.h"
#include "paged_kernel.h"
#include "profile.h"
#include "rope_kernel.h"

namespace sbpk {

using sbpi::PagedArgs;

__device__ __forceinline__ float load1(const uint16_t *p) {
    return __builtin_bit_cast(float, (uint32_t)*p << 16);
}
__device__ __forceinline__ void store1(uint16_t *p, float v) { *p = f32_to_bf16_bits(v); }

__global__ __launch_bounds__(256) void paged_attn_kernel(PagedArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int heads = a.kv_heads * a.group;
    const int h = (int)(id % heads), hk = h / a.group;
    const int i = (int)(id / heads);
    const int b = blockIdx.y;
    const SeqRows s = rows_of(a.at, b);
    const bool padded = !a.at.row_q;
    if (i >= (padded ? a.at.rows : s.n)) return;
    const int64_t row = s.first + i;
    const int lk = min(max(s.len, 0), a.at.width * a.at.page);
    const int off = lk - s.n;
    const int hi = i >= s.n ? 0 : a.causal ? min(lk, i + 1 + off) : lk;
    const int lo = a.window ? max(0, i + 1 + off - a.window) : 0;
    const bool two = lane + 64 < a.d, one = lane < a.d;
    const uint16_t *q = static_cast<uint16_t *>(a.q.p) + s.batch * a.q.sb + h * a.q.sh + row * a.q.ld;
    const float q0 = one && lo < hi ? load1(q + lane) : 0.f;
    const float q1 = two && lo < hi ? load1(q + lane + 64) : 0.f;
    const float c = a.scale * LOG2E;
    float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
    for (int j = lo; j < hi; ++j) {
        const int page = a.at.table[b * a.at.table_ld + j / a.at.page];
        if (page < 0 || page >= a.at.pages) continue;
        const int slot = j % a.at.page;
        const uint16_t *k = static_cast<uint16_t *>(a.kc.p) + page * a.kc.sb + hk * a.kc.sh +
                            slot * a.kc.ld;
        const uint16_t *v = static_cast<uint16_t *>(a.vc.p) + page * a.vc.sb + hk * a.vc.sh +
                            slot * a.vc.ld;
        float x = (one ? q0 * load1(k + lane) : 0.f) + (two ? q1 * load1(k + lane + 64) : 0.f);
        for (int w = 32; w; w >>= 1) x += __shfl_xor(x, w);
        const float mn = fmaxf(m, x);
        const float old = m == -INFINITY ? 0.f : exp2_((m - mn) * c);
        const float e = exp2_((x - mn) * c);
        l = l * old + e;
        o0 = o0 * old + (one ? e * load1(v + lane) : 0.f);
        o1 = o1 * old + (two ? e * load1(v + lane + 64) : 0.f);
        m = mn;
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    const int64_t at = s.batch * a.o.sb + h * a.o.sh + row * a.o.ld;
    auto put = [&](int col, float v) {
        if (a.o_f32) static_cast<float *>(a.o.p)[at + col] = v;
        else store1(static_cast<uint16_t *>(a.o.p) + at + col, v);
    };
    if (one) put(lane, o0 * inv);
    if (two) put(lane + 64, o1 * inv);
    if (a.lse.p && lane == 0)
        static_cast<float *>(a.lse.p)[s.batch * a.lse.sb + h * a.lse.sh + row * a.lse.ld] =
            l > 0.f ? __builtin_fmaf(m, a.scale, __builtin_amdgcn_logf(l) * LN2) : -INFINITY;
}

}  // namespace sbpk

namespace sbpi {

hipError_t launch_paged(const PagedArgs &a, hipStream_t s) {
    const int64_t waves = (int64_t)a.at.rows * a.kv_heads * a.group;
    return launch_kernel(sbpk::paged_attn_kernel, "paged_attn_kernel",
                         dim3((unsigned)((waves + 3) / 4), (unsigned)a.at.seqs), dim3(256), s, a);
}

}  // namespace sbpi
