// The selective state-space scan: sizes, arguments and launchers (prompts and single
// tokens in selective.hip, gradients in selective_grad.hip).
#pragma once

#include "block_ops.hpp"

namespace lh {

constexpr int kMaxStates = 128;  // per channel

// Device pointers and sizes of a call.  Rows of dt, u, z, Bm and Cm are ld_* elements
// apart; row b T + t belongs to token t of batch row b.
struct Selective {
    const void *dt, *u, *z, *Bm, *Cm;
    int64_t ld_dt, ld_u, ld_z, ld_b, ld_c;
    const float *A, *dt_bias, *h0;
    const int* lengths;
    int64_t B, T, D;
    int N, G;
    bool bf16_io;
};

// A 64-channel tile belongs to one group, so that its input and output rows are the
// same in every lane: tiles per group x groups.
__host__ __device__ inline int64_t group_tiles(int64_t D, int G)
{
    return (D / G + kWave - 1) / kWave;
}

struct SelectivePlan {
    int ns, waves;        // states per lane, wavefronts (of other states) per tile
    int64_t chunk;        // steps per time chunk (a multiple of 16)
    int64_t nchunks;      // 1: one pass from the state
    size_t off_sums;      // workspace: step sums [B, nchunks, D] after the states
    size_t ws_bytes;      // [B, nchunks, N, D] chunk states and the sums, 0 when nchunks = 1
};
SelectivePlan selective_plan(int64_t B, int64_t T, int64_t D, int N, int G);

// Threads of the largest launch of a prompt, a step and a gradient.
int64_t selective_threads(int64_t B, int64_t T, int64_t D, int N, int G);
int64_t selective_step_threads(int64_t B, int64_t D, int N);
int64_t selective_grad_threads(int64_t B, int64_t T, int64_t D, int N, int G);

hipError_t launch_selective(const Selective& s, float* state, bool resume, void* y,
                            void* workspace, hipStream_t stream);
hipError_t launch_selective_step(const Selective& s, float* state, void* y, hipStream_t stream);

struct SelectiveGrads {
    const void* dy;
    void *ddt, *du, *dz, *dBm, *dCm;
    float *dA, *dh0, *ddt_bias;
};
size_t selective_grad_workspace_bytes(int64_t B, int64_t T, int64_t D, int N, int G);
hipError_t launch_selective_grad(const Selective& s, const SelectiveGrads& g, void* workspace,
                                 hipStream_t stream);

// The element a 32-bit byte offset from a pointer that is the same in all lanes (which
// the hardware adds by itself).
template <typename T>
__device__ __forceinline__ T& at_byte(T* p, uint32_t off)
{
    using C = std::conditional_t<std::is_const_v<T>, const char, char>;
    return *reinterpret_cast<T*>(reinterpret_cast<C*>(p) + off);
}

// Tokens of batch row b (a length outside [0, T] is taken as the nearer end).
__device__ __forceinline__ int64_t tokens_of(const int* lengths, int64_t b, int64_t T)
{
    if (!lengths) return T;
    const int64_t n = lengths[b];
    return n < 0 ? 0 : n < T ? n : T;
}

// The decay over a chunk whose steps sum to `sum`, A2 = A log2 e.  A chunk without tokens
// leaves the state alone, also where A is infinite.
__device__ __forceinline__ float chunk_decay(float A2, float sum)
{
    return exp2_fast(sum == 0.f ? 0.f : A2 * sum);
}

}  // namespace lh
