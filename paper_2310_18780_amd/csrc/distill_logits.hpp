// Distillation from a teacher's top logits: launchers (distill_logits.hip).
#pragma once

#include "lh_internal.hpp"

namespace lh {

struct DistillLogits {
    const void* logits;
    int64_t ld;
    const float* values;
    const int32_t* ids;
    const float* scale;
    int64_t rows, V;
    int K;
    float tau;
    bool bf16_io;
    void* dlogits;
    int64_t ld_d;
};

hipError_t launch_distill_logits(const DistillLogits& a, float* loss, float* lse, hipStream_t stream);
hipError_t launch_distill_logits_grad(const DistillLogits& a, const float* dloss, const float* lse,
                                      hipStream_t stream);

}  // namespace lh
