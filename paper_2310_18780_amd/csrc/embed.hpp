// Token embedding: sizes and launchers (embed.hip, embed_grad.hip).
#pragma once

#include "lh_internal.hpp"

namespace lh {

hipError_t launch_embed(const void* W, const int32_t* ids, int64_t n, int64_t V, int64_t D,
                        bool bf16_table, bool bf16_io, float scale, void* y, hipStream_t stream);

// How the gradient's call is laid out in its workspace.
struct EmbedGradPlan {
    int64_t window;   // sorted tokens of a workgroup
    int64_t windows;
    int64_t tile;     // tokens of a workgroup of the sort (0: few, that one launch places)
    int64_t tiles;
    int passes, bits;  // digits of the ids, and their bits
    size_t off_keys[2], off_rows[2], off_counts, off_part;
    size_t ws_bytes;
};
EmbedGradPlan embed_grad_plan(int64_t n, int64_t V, int64_t D);
int64_t embed_grad_threads(int64_t n, int64_t V, int64_t D);
hipError_t launch_embed_grad(const void* dy, const int32_t* ids, int64_t n, int64_t V, int64_t D,
                             bool bf16_io, float scale, bool accumulate, float* dW, void* workspace,
                             hipStream_t stream);

}  // namespace lh
