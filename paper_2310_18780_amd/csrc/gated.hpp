// Gated linear recurrence: sizes and launchers (gated.hip, gated_grad.hip).
#pragma once

#include "lh_internal.hpp"

namespace lh {

// Sizes and inputs of a call (see include/lh.h).
struct Gated {
    const void *r, *i, *u, *z;
    int64_t ld_r, ld_i, ld_u, ld_z;
    const float *rate, *r_bias, *i_bias;
    const int* lengths;
    int64_t B, T, D;
    bool bf16_io;
};

struct GatedGrads {
    const void* dy;
    const float *marks, *dlast;
    void *dr, *di, *du, *dz;
    float *drate, *dr_bias, *di_bias, *dfirst;
};

// A prompt's blocks of steps, and how many workgroups share those of a tile of channels.
struct GatedPlan {
    int64_t blocks, shares;
    size_t ws_bytes;
};
GatedPlan gated_plan(int64_t B, int64_t T, int64_t D);

// Time chunks that the gradient's prompt is cut into (chunk: steps of one).
struct GatedGradPlan {
    int64_t chunk, chunks;
    size_t ws_bytes;
};
GatedGradPlan gated_grad_plan(int64_t B, int64_t T, int64_t D);

// Threads of the largest launch of a call.
int64_t gated_threads(int64_t B, int64_t T, int64_t D);
int64_t gated_step_threads(int64_t B, int64_t D);
int64_t gated_grad_threads(int64_t B, int64_t T, int64_t D);

hipError_t launch_gated(const Gated& g, float* state, bool resume, void* y, float* marks,
                        void* workspace, hipStream_t stream);
hipError_t launch_gated_step(const Gated& g, float* state, void* y_t, hipStream_t stream);
hipError_t launch_gated_grad(const Gated& g, const GatedGrads& d, void* workspace,
                             hipStream_t stream);

}  // namespace lh
