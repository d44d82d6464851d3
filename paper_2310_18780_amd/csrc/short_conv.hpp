// The short causal convolution: launchers (short_conv.hip).
#pragma once

#include "lh_internal.hpp"

namespace lh {

// Threads of the largest launch of any of the calls, either type.
int64_t short_conv_threads(int64_t B, int64_t T, int64_t D, int64_t K);

hipError_t launch_short_conv(const void* x, int64_t ld, const float* w, const float* bias,
                             const int* lengths, void* state, bool resume, void* y, bool bf16_io,
                             bool silu, int64_t B, int64_t T, int64_t D, int64_t K,
                             hipStream_t stream);
hipError_t launch_short_conv_step(const void* x, int64_t ld, const float* w, const float* bias,
                                  void* state, void* y, bool bf16_io, bool silu, int64_t B,
                                  int64_t D, int64_t K, hipStream_t stream);
size_t short_conv_grad_workspace_bytes(int64_t B, int64_t T, int64_t D, int64_t K);
hipError_t launch_short_conv_grad(const void* dy, const void* x, int64_t ld, const float* w,
                                  const float* bias, const int* lengths, void* dx, float* dw,
                                  float* dbias, bool bf16_io, bool silu, int64_t B, int64_t T,
                                  int64_t D, int64_t K, void* workspace, hipStream_t stream);

}  // namespace lh
