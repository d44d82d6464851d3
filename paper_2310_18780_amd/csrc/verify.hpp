// Verification of drafted tokens: launchers (verify.hip).
#pragma once

#include "lh_internal.hpp"

namespace lh {

struct Verify {
    const int32_t *drafted, *lengths;
    const void *draft_p, *target_p;
    int64_t ld_draft, ld_target;
    const float *u, *u_last;
    int64_t B, K, V;
    bool bf16_io;
    int32_t *accepted, *tokens;
};

size_t verify_workspace_bytes(int64_t B, int64_t K, int64_t V);
int64_t verify_threads(int64_t B, int64_t V);
hipError_t launch_verify(const Verify& v, void* workspace, hipStream_t stream);

}  // namespace lh
