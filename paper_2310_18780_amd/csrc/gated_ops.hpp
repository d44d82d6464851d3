// Device helpers shared by the gated recurrence's kernels.
#pragma once

#include "block_ops.hpp"
#include "gated.hpp"
#include "lh.h"

namespace lh {

constexpr int kRun = LH_GATED_MARK;  // steps that a wavefront takes at a time
constexpr int kTile = kWave;         // channels of a wavefront, one to a lane

// A call's inputs in the types of its kernels.  (The prompt and the step see all their tokens as one
// chunk.)
template <typename T>
struct GatedIn {
    const T *r, *i, *u, *z;
    int64_t ld_r, ld_i, ld_u, ld_z;
    const float *rate, *r_bias, *i_bias;
    const int* lengths;
    int64_t B, T_, D, chunk, chunks, blocks, tiles, marks;
};

template <typename T>
GatedIn<T> gated_in(const Gated& g, int64_t chunk, int64_t chunks, int64_t blocks)
{
    GatedIn<T> a;
    a.r = static_cast<const T*>(g.r), a.i = static_cast<const T*>(g.i);
    a.u = static_cast<const T*>(g.u), a.z = static_cast<const T*>(g.z);
    a.ld_r = g.ld_r, a.ld_i = g.ld_i, a.ld_u = g.ld_u, a.ld_z = g.ld_z;
    a.rate = g.rate, a.r_bias = g.r_bias, a.i_bias = g.i_bias, a.lengths = g.lengths;
    a.B = g.B, a.T_ = g.T, a.D = g.D, a.chunk = chunk, a.chunks = chunks, a.blocks = blocks;
    a.tiles = (g.D + kTile - 1) / kTile;
    a.marks = (g.T + kRun - 1) / kRun;
    return a;
}

inline int64_t gated_tiles(int64_t B, int64_t D) { return B * ((D + kTile - 1) / kTile); }

// Chunks of whole runs for about `want` of them over all tiles, each of `least` steps or more.
inline GatedGradPlan gated_chunks(int64_t B, int64_t T, int64_t D, int64_t want, int64_t least)
{
    int64_t chunks = want / gated_tiles(B, D);
    if (chunks > T / least) chunks = T / least;
    if (chunks < 1) chunks = 1;
    GatedGradPlan p{};
    const int64_t runs = (T + kRun - 1) / kRun, per = (runs + chunks - 1) / chunks;
    p.chunk = (per > 0 ? per : 1) * kRun;
    p.chunks = T > 0 ? (T + p.chunk - 1) / p.chunk : 1;
    return p;
}

__device__ __forceinline__ int64_t gated_length(const int* lengths, int64_t b, int64_t T)
{
    if (!lengths) return T;
    const int64_t n = lengths[b];
    return n < 0 ? 0 : n < T ? n : T;
}

// The 8 rows of a run in one of the call's tensors, as a buffer whose range ends with the last
// token's: what lies past it reads as zero and is not written, under no branch.  (The row is a
// scalar offset, the lane's channel a vector one: no address arithmetic in the lanes.)
template <typename T>
struct Rows {
    __amdgpu_buffer_rsrc_t buf;
    uint32_t ld;
    // p: the tile's first channel in the run's first row, `wide` channels, m <= 8 rows (<= 0: none)
    __device__ __forceinline__ Rows(const T* p, int64_t ld_, int wide, int m)
        : ld(uint32_t(ld_) * uint32_t(sizeof(T)))
    {
        const uint32_t n = (uint32_t(m - 1) * ld + uint32_t(wide) * uint32_t(sizeof(T))) & uint32_t(-(m > 0));
        buf = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(p), 0, n, 0x00027000);
    }
    __device__ __forceinline__ T load(int s, uint32_t lane_bytes) const
    {
        if constexpr (sizeof(T) == 2)
            return T{__builtin_amdgcn_raw_buffer_load_b16(buf, lane_bytes, uint32_t(s) * ld, 0)};
        else
            return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(buf, lane_bytes, uint32_t(s) * ld, 0));
    }
    __device__ __forceinline__ void store(int s, uint32_t lane_bytes, float v) const
    {
        T t;
        io_store(&t, v);
        if constexpr (sizeof(T) == 2)
            __builtin_amdgcn_raw_buffer_store_b16(t.bits, buf, lane_bytes, uint32_t(s) * ld, 0);
        else
            __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(t), buf, lane_bytes, uint32_t(s) * ld, 0);
    }
};

// Where a wavefront works: chunk k of tile c0 of row b, the tokens [t0, te), the outputs [t0, t1).
struct Place {
    int64_t b, k, c0, t0, t1, te;
    int wide;  // channels of the tile
    // the lane's channel in the tile: lanes past the last channel repeat it, and store the same
    // bits to the same place
    uint32_t lc;
    template <typename T>
    __device__ __forceinline__ Place(const GatedIn<T>& in, int64_t unit, int64_t chunks, int64_t first)
    {
        const int lane = threadIdx.x % kWave;
        // (a launch has fewer than 2^32 threads)
        const uint32_t u = uint32_t(unit), tiles = uint32_t(in.tiles), row = u / tiles;
        c0 = int64_t(u - row * tiles) * kTile;
        b = row / uint32_t(chunks);
        k = row - uint32_t(b) * uint32_t(chunks) + first;
        wide = int(in.D - c0 < kTile ? in.D - c0 : kTile);
        lc = uint32_t(lane < wide ? lane : wide - 1);
        const int64_t n = gated_length(in.lengths, b, in.T_);
        t0 = k * in.chunk;
        t1 = t0 + in.chunk < in.T_ ? t0 + in.chunk : in.T_;
        te = t1 < n ? t1 : n;
    }
    // where the chunk's last run begins (before t0: there is none)
    __device__ __forceinline__ int64_t last_run() const
    {
        return te > t0 ? t0 + (te - 1 - t0) / kRun * kRun : t0 - 1;
    }
};

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
    const float series = x * decay_series(x);
    return x < kSmall ? series : 1.f - e;
}

// A state after decays of x (in log2) and inputs that alone leave h: what is lost, and not
// what is kept, multiplies the state, so that a decay near 1 is not rounded to 24 bits.
// (No decay leaves any state as it is, one that is not finite too.)
__device__ __forceinline__ float carry_on(float state, float x, float h)
{
    const float kept = fmaf(-one_minus(x, exp2_fast(-x)), state, state);
    return (x == 0.f ? state : kept) + h;
}

// The decay of a step (l its log2, negated) and its input; a step that is not there (its r, i and
// u zeros) decays nothing and has no input.
struct GateStep {
    float l, a, v;
};
__device__ __forceinline__ GateStep gate_step(float r, float i, float u, bool there, const GateParams& par)
{
    GateStep g;
    const float f = rcp_fast(1.f + exp2_fast(fmaf(r, -kLog2e, par.nrb)));
    const float p = rcp_fast(1.f + exp2_fast(fmaf(i, -kLog2e, par.nib)));
    g.l = there ? par.rate2 * f : 0.f;
    g.a = exp2_fast(-g.l);
    g.v = __builtin_amdgcn_sqrtf(one_minus(2.f * g.l, g.a * g.a)) * p * u;
    return g;
}

// A gate's sigmoid(x) from y = -x log2 e, and 1 - sigmoid(x), both without cancellation.  From e =
// 2^126 on the reciprocal is below the smallest normal number, and is 0: so are then all gradients
// through the gate, and of e just this limit keeps infinity times 0 away.
__device__ __forceinline__ float2 gate_pair(float y)
{
    const float e = exp2_fast(y);
    const float f = rcp_fast(1.f + e);
    return make_float2(f, fminf(e, 0x1p126f) * f);
}

}  // namespace lh
