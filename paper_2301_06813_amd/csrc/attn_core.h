// attn_core.h -- softmax attention of a device's heads, forward and backward
// (include/sbp.h, "softmax attention"): arguments shared by the host code and
// the kernels of attn_core_fwd.hip and attn_core_bwd.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sbpi {

// A 4-D operand of the kernels: element strides; 16 bits or fp32.
struct CoreView {
    void *p = nullptr;
    int64_t sb = 0, sh = 0, ld = 0;
};

struct CoreArgs {
    CoreView q, k, v, o, lse;            // lse.p may be NULL (forward)
    CoreView dout, dq, dk, dv;           // backward
    int32_t batch, kv_heads, group;      // local heads; query heads per kv head
    int32_t sq, sk, d;
    int32_t causal, window;              // window 0: none
    const int32_t *len_q, *len_k;        // per sequence, or NULL
    float scale;
    int32_t o_f32, dq_f32, dk_f32, dv_f32;
    int32_t dq_acc, dk_acc, dv_acc;      // add to the output's contents
    int32_t aligned;                     // 16-byte rows: the direct-to-LDS loads may read
                                         // Q, K, V (and dO)
    float *ws;                           // forward: split partials; backward: row statistics,
    size_t ws_floats;                    // then split partials
};

// Floats of workspace that the backward pass cannot do without: two per query
// row (each array padded to a multiple of 4).
inline size_t core_bwd_stat_floats(const CoreArgs &a) {
    const size_t rows = (size_t)a.batch * a.kv_heads * a.group * a.sq;
    return 2 * ((rows + 3) & ~size_t(3));
}

hipError_t launch_core_fwd(const CoreArgs &a, hipStream_t s);
hipError_t launch_core_bwd(const CoreArgs &a, hipStream_t s);

}  // namespace sbpi
