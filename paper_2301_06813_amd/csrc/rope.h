// rope.h -- rotary positions (include/sbp.h, "rotary positions"): arguments shared
// by the host code and the kernels of rope.hip.
#pragma once

#include "attn_core.h"

namespace sbpi {

struct Rotation {
    const uint64_t *turns = nullptr;     // dim / 2, of 2^-64 turn a position
    int32_t dim = 0, pairs = 0;          // pairs: the order
    float mul = 1.f;
};

struct RopeArgs {
    CoreView in[2], out[2];              // Q, K
    int32_t heads[2] = {0, 0};
    int32_t batch = 0, rows = 0, d = 0;
    Rotation rot;
    int32_t back = 0;                    // the gradient: minus the angles
    const int32_t *pos = nullptr;        // NULL: row i at i
    int64_t pos_ld = 0;
    int32_t pos_per_row = 0;
};

// Inputs and outputs fp32 (1) or bf16 (0).
hipError_t launch_rope(const RopeArgs &a, int in_f32, int out_f32, hipStream_t s);

}  // namespace sbpi
