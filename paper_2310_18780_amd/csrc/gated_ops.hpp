// Device helpers shared by the gated recurrence's kernels.
#pragma once

#include "block_ops.hpp"
#include "gated.hpp"
#include "lh.h"

namespace lh {

constexpr int kRun = 8;  // steps that a wavefront takes at a time
constexpr int kTile = kWave;  // channels of a workgroup, one to a lane
constexpr int kMark = LH_GATED_MARK;  // steps between the states that the gradient takes
static_assert(kMark % kRun == 0, "marks lie before runs");

// A call's inputs in the types of its kernels.
template <typename T>
struct GatedIn {
    const T *r, *i, *u, *z;
    int64_t ld_r, ld_i, ld_u, ld_z;
    const float *rate, *r_bias, *i_bias;
    const int* lengths;
    int64_t B, T_, D, chunk, chunks, tiles, marks;
};

template <typename T>
GatedIn<T> gated_in(const Gated& g, const GatedPlan& p)
{
    GatedIn<T> a;
    a.r = static_cast<const T*>(g.r), a.i = static_cast<const T*>(g.i);
    a.u = static_cast<const T*>(g.u), a.z = static_cast<const T*>(g.z);
    a.ld_r = g.ld_r, a.ld_i = g.ld_i, a.ld_u = g.ld_u, a.ld_z = g.ld_z;
    a.rate = g.rate, a.r_bias = g.r_bias, a.i_bias = g.i_bias, a.lengths = g.lengths;
    a.B = g.B, a.T_ = g.T, a.D = g.D, a.chunk = p.chunk, a.chunks = p.chunks;
    a.tiles = (g.D + kTile - 1) / kTile;
    a.marks = (g.T + kMark - 1) / kMark;
    return a;
}

inline int64_t gated_tiles(int64_t B, int64_t D) { return B * ((D + kTile - 1) / kTile); }

__device__ __forceinline__ int64_t gated_length(const int* lengths, int64_t b, int64_t T)
{
    if (!lengths) return T;
    const int64_t n = lengths[b];
    return n < 0 ? 0 : n < T ? n : T;
}

constexpr float kMaxRate = 3.0e38f;  // (infinity times a gate of 0 would be NaN)

// Parameters of a lane's channel, the biases times -log2 e (as they enter the exponents).
struct GateParams {
    float rate2, nrb, nib;
    template <typename T>
    __device__ __forceinline__ GateParams(const GatedIn<T>& in, int64_t c)
        : rate2(in.rate[c] * kLog2e > kMaxRate ? kMaxRate : in.rate[c] * kLog2e),
          nrb(in.r_bias ? -kLog2e * in.r_bias[c] : 0.f),
          nib(in.i_bias ? -kLog2e * in.i_bias[c] : 0.f)
    {
    }
};

// (1 - 2^-x) / x for 0 <= x < kSmall, to 2^-24: the series of the exponential.
constexpr float kSmall = 0.18f;
__device__ __forceinline__ float decay_series(float x)
{
    return fmaf(x, fmaf(x, fmaf(x, fmaf(x, 1.33335581e-3f, -9.61812911e-3f), 5.55041087e-2f),
                        -0.240226507f), 0.693147181f);
}

// 1 - 2^-x for x >= 0, without cancellation; e = 2^-x.
__device__ __forceinline__ float one_minus(float x, float e)
{
    return x < kSmall ? x * decay_series(x) : 1.f - e;
}

// A state after decays of x (in log2) and inputs that alone leave h: what is lost, and not
// what is kept, multiplies the state, so that a decay near 1 is not rounded to 24 bits.
// (No decay leaves any state as it is, one that is not finite too.)
__device__ __forceinline__ float carry_on(float state, float x, float h)
{
    const float kept = fmaf(-one_minus(x, exp2_fast(-x)), state, state);
    return (x == 0.f ? state : kept) + h;
}

// A gate's sigmoid(x) from y = -x log2 e, and 1 - sigmoid(x), both without cancellation.
__device__ __forceinline__ float2 gate_pair(float y)
{
    const float e = exp2_fast(y);
    const float f = rcp_fast(1.f + e);
    return make_float2(f, fminf(e, 0x1p125f) * f);  // (infinity times 0 would be NaN)
}

}  // namespace lh
