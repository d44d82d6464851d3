// Layer norm: launchers (norm.hip).
#pragma once

#include "lh_internal.hpp"

namespace lh {

hipError_t launch_norm(const void* x, const void* residual, const float* w, const float* b,
                       void* y, void* total, float* mean, float* rstd, bool bf16_io, int64_t rows,
                       int64_t D, float eps, hipStream_t stream);
size_t norm_grad_workspace_bytes(int64_t rows, int64_t D);
hipError_t launch_norm_grad(const void* dy, const void* x, const float* w, const float* mean,
                            const float* rstd, const void* dtotal, void* dx, float* dw, float* db,
                            bool bf16_io, int64_t rows, int64_t D, void* workspace,
                            hipStream_t stream);

}  // namespace lh
