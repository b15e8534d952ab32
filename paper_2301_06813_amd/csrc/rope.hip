// rope.hip -- rotary positions of Q and K, forward and backward.
//
// A thread owns a pair of columns of a row, over all heads of Q and K: its angle is computed
// once.
#include "profile.h"
#include "rope_kernel.h"

namespace sbpk {

template <typename TI, typename TO>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
    const Rotation &r = a.rot;
    const int half = r.dim / 2, units = half + (a.d - r.dim);
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int u = (int)(id % units);
    const int64_t row = id / units;
    if (row >= (int64_t)a.batch * a.rows) return;
    const int b = (int)(row / a.rows), i = (int)(row % a.rows);
    int one = r.dim + (u - half), two = one;
    float c = 1.f, s = 0.f;
    if (u < half) {
        columns(r, u, &one, &two);
        int64_t t = i;
        if (a.pos) t = a.pos_per_row ? a.pos[b * a.pos_ld + i] : (int64_t)a.pos[b * a.pos_ld] + i;
        angle(r.turns[u], t, r.mul, &c, &s);
        if (a.back) s = -s;
    }
    for (int x = 0; x < 2; ++x)
        for (int h = 0; h < a.heads[x]; ++h) {
            const TI *in = static_cast<const TI *>(a.in[x].p) + b * a.in[x].sb + h * a.in[x].sh +
                           i * a.in[x].ld;
            TO *out = static_cast<TO *>(a.out[x].p) + b * a.out[x].sb + h * a.out[x].sh +
                      i * a.out[x].ld;
            const float v = load1(in + one), w = load1(in + two);
            if (u < half) {
                store1(out + one, v * c - w * s);
                store1(out + two, w * c + v * s);
            } else {
                store1(out + one, v);
            }
        }
}

}  // namespace sbpk

namespace sbpi {

hipError_t launch_rope(const RopeArgs &a, int in_f32, int out_f32, hipStream_t s) {
    const int64_t n = (int64_t)a.batch * a.rows * (a.rot.dim / 2 + a.d - a.rot.dim);
    const dim3 grid((unsigned)((n + 255) / 256)), block(256);
    if (in_f32) return launch_kernel(sbpk::rope_kernel<float, float>, "rope_kernel", grid, block, s, a);
    if (out_f32)
        return launch_kernel(sbpk::rope_kernel<uint16_t, float>, "rope_kernel", grid, block, s, a);
    return launch_kernel(sbpk::rope_kernel<uint16_t, uint16_t>, "rope_kernel", grid, block, s, a);
}

}  // namespace sbpi
