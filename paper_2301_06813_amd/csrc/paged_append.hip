// paged_append.hip -- new tokens' keys and values to their places in a paged cache, with the
// rotation of K and Q on the way.
//
// A thread owns a pair of columns of a new token, over all heads of Q, K and V.
#include "paged_kernel.h"
#include "profile.h"
#include "rope_kernel.h"

namespace sbpk {

using sbpi::AppendArgs;

template <typename TQ>
__global__ __launch_bounds__(256) void paged_append_kernel(AppendArgs a) {
    const Rotation &r = a.rot;
    const int half = r.dim / 2, units = half + (a.d - r.dim);
    const SeqRows s = rows_of(a.at, blockIdx.y);
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int u = (int)(id % units);
    const int64_t i = id / units;
    if (i >= s.n) return;
    const int64_t t = (int64_t)s.len - s.n + i;
    int one = r.dim + (u - half), two = one;
    float c = 1.f, sn = 0.f;
    if (u < half) {
        columns(r, u, &one, &two);
        angle(r.turns[u], t, r.mul, &c, &sn);
    }
    auto turn = [&](const uint16_t *in, auto *out) {
        const float v = load1(in + one), w = load1(in + two);
        if (u < half) {
            store1(out + one, v * c - w * sn);
            store1(out + two, w * c + v * sn);
        } else {
            store1(out + one, v);
        }
    };
    auto row = [&](const CoreView &v, int h) {
        return static_cast<uint16_t *>(v.p) + s.batch * v.sb + h * v.sh + (s.first + i) * v.ld;
    };
    if (a.q.p)
        for (int h = 0; h < a.q_heads; ++h)
            turn(row(a.q, h), static_cast<TQ *>(a.qo.p) + s.batch * a.qo.sb + h * a.qo.sh +
                                  (s.first + i) * a.qo.ld);
    if (t < 0 || t >= (int64_t)a.at.width * a.at.page) return;
    const int page = a.at.table[blockIdx.y * a.at.table_ld + t / a.at.page];
    if (page < 0 || page >= a.at.pages) return;
    auto slot = [&](const CoreView &v, int h) {
        return static_cast<uint16_t *>(v.p) + page * v.sb + h * v.sh + (t % a.at.page) * v.ld;
    };
    for (int h = 0; h < a.kv_heads; ++h) {
        turn(row(a.k, h), slot(a.kc, h));
        const uint16_t *in = row(a.v, h);
        uint16_t *out = slot(a.vc, h);
        out[one] = in[one];
        out[two] = in[two];
    }
}

}  // namespace sbpk

namespace sbpi {

hipError_t launch_append(const AppendArgs &a, int qo_f32, hipStream_t s) {
    const int64_t n = (int64_t)a.at.rows * (a.rot.dim / 2 + a.d - a.rot.dim);
    const dim3 grid((unsigned)((n + 255) / 256), (unsigned)a.at.seqs), block(256);
    if (qo_f32)
        return launch_kernel(sbpk::paged_append_kernel<float>, "paged_append_kernel", grid, block, s, a);
    return launch_kernel(sbpk::paged_append_kernel<uint16_t>, "paged_append_kernel", grid, block, s, a);
}

}  // namespace sbpi
