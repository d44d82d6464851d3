// Gated linear recurrence over prompts and for single tokens, per channel:
//
//   f = sigmoid(r + r_bias),  p = sigmoid(i + i_bias),  a = e^(-rate f)
//   h <- a h + sqrt(1 - a^2) p u,   y = h (times z sigmoid(z))
//
// h after any run of steps is A h_before + H, with A the product of the run's decays and
// H what its inputs alone leave.  A wavefront holds 64 channels of a row, one to a lane, and
// takes 8 steps at a time, whose loads all start together.
//
// Many rows: a workgroup of 16 wavefronts walks a prompt in blocks of 128 steps, 8 to a
// wavefront.  Each forms (A, H) of its run, they meet in LDS, each chains those before its own
// to its entry state and walks its steps again from registers: inputs are read once, outputs
// written once.  Few rows: the prompt is cut into chunks, one to a wavefront that walks it by
// itself; a first launch forms each chunk's (log2 A, H), and each chunk of the second folds those
// before it.
//
// A run's decay is carried on as the sum of its logarithms (carry_on): products of roundings
// near 1 would be off by 2^-24 a step over thousands of steps.
#include "gated_ops.hpp"

namespace lh {
namespace {

constexpr int kWaves = 16;
constexpr int kSpan = kWaves * kRun;  // steps of a block

// The inputs of a run, as they lie in memory.
template <typename T, bool GATE>
struct Run {
    T r[kRun], i[kRun], u[kRun], z[kRun];
    __device__ __forceinline__ Run(const GatedIn<T>& in, const Place& at, int64_t t, int m)
    {
        const int64_t row = at.b * in.T_ + t;
        const uint32_t lane = at.lc * uint32_t(sizeof(T));
        const Rows<T> br(in.r + row * in.ld_r + at.c0, in.ld_r, at.wide, m);
        const Rows<T> bi(in.i + row * in.ld_i + at.c0, in.ld_i, at.wide, m);
        const Rows<T> bu(in.u + row * in.ld_u + at.c0, in.ld_u, at.wide, m);
#pragma unroll
        for (int s = 0; s < kRun; ++s) {
            r[s] = br.load(s, lane);
            i[s] = bi.load(s, lane);
            u[s] = bu.load(s, lane);
        }
        if constexpr (GATE) {
            const Rows<T> bz(in.z + row * in.ld_z + at.c0, in.ld_z, at.wide, m);
#pragma unroll
            for (int s = 0; s < kRun; ++s) z[s] = bz.load(s, lane);
        }
    }
    // step s of m: steps past the last decay nothing, and their inputs are zeros
    __device__ __forceinline__ GateStep step(int s, int m, const GateParams& par) const
    {
        return gate_step(io_load(&r[s]), io_load(&i[s]), io_load(&u[s]), s < m, par);
    }
    __device__ __forceinline__ float out(int s, float h) const
    {
        if constexpr (!GATE) return h;
        const float g = io_load(&z[s]);
        return h * (g * sigmoid(g));
    }
};

template <typename T, bool GATE>
__global__ __launch_bounds__(kWaves* kWave, 8) void gated_kernel(GatedIn<T> in, float* state, int resume,
                                                              T* __restrict__ y, float* __restrict__ marks)
{
    __shared__ float2 runs[2][kWaves][kWave];
    __shared__ float logs[2][kWaves][kWave];
    const int lane = threadIdx.x % kWave;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const Place at(in, blockIdx.x, 1, 0);
    const int64_t c = at.c0 + at.lc;
    const GateParams par(in, c);
    float h = resume ? state[at.b * in.D + c] : 0.f;  // before the block
    int turn = 0;
    for (int64_t tb = 0; tb < at.te; tb += kSpan, turn ^= 1) {
        const int64_t t = tb + wave * kRun;
        const int m = int(at.te - t < kRun ? at.te - t : kRun);  // steps (<= 0: none)
        const Run<T, GATE> x(in, at, t, m);
        float a[kRun], v[kRun];
        float H = 0.f, L = 0.f;
#pragma unroll
        for (int s = 0; s < kRun; ++s) {
            const GateStep g = x.step(s, m, par);
            a[s] = g.a;
            v[s] = g.v;
            L += g.l;
            H = fmaf(a[s], H, v[s]);
        }
        runs[turn][wave][lane] = make_float2(exp2_fast(-L), H);
        logs[turn][wave][lane] = L;
        __syncthreads();
        // from zero: the states and decays before this run, and of the whole block
        float e = 0.f, le = 0.f, end = 0.f, lend = 0.f;
#pragma unroll 4
        for (int j = 0; j < kWaves; ++j) {
            if (j == wave) e = end, le = lend;
            const float2 n = runs[turn][j][lane];
            end = fmaf(n.x, end, n.y);
            lend += logs[turn][j][lane];
        }
        float o = wave == 0 ? h : fmaf(exp2_fast(-le), h, e);
        if (marks && m > 0) marks[(at.b * in.marks + t / kRun) * in.D + c] = o;
        const Rows<T> by(y + (at.b * in.T_ + t) * in.D + at.c0, in.D, at.wide, m);
#pragma unroll
        for (int s = 0; s < kRun; ++s) {
            o = fmaf(a[s], o, v[s]);
            by.store(s, at.lc * uint32_t(sizeof(T)), x.out(s, o));
        }
        h = carry_on(h, lend, end);
    }
    for (int64_t t = at.te + wave; t < in.T_; t += kWaves) io_store(y + (at.b * in.T_ + t) * in.D + c, 0.f);
    if (wave == 0) state[at.b * in.D + c] = h;
}

constexpr int kWalkWaves = 4;  // wavefronts of a workgroup, each with a chunk of its own

// ENDS: the chunks' ends only, into slots 1 .. of ends [B, chunks, D] (log2 of the decay,
// negated, and state from zero); slot 0 holds the start.
template <typename T, bool GATE, bool ENDS>
__global__ __launch_bounds__(kWalkWaves* kWave) void gated_walk_kernel(
    GatedIn<T> in, float* state, int resume, T* __restrict__ y, float* __restrict__ marks,
    float2* __restrict__ ends, int64_t units)
{
    const int64_t unit = int64_t(blockIdx.x) * kWalkWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    if (unit >= units) return;
    const Place at(in, unit, ENDS ? in.chunks - 1 : in.chunks, 0);
    const int64_t c = at.c0 + at.lc;
    const GateParams par(in, c);
    float h = 0.f, total = 0.f;  // state; log2 of the decays so far, negated
    float2* pe = ends + at.b * in.chunks * in.D + c;
    if constexpr (ENDS) {
        if (at.k == 0) pe[0] = make_float2(0.f, resume ? state[at.b * in.D + c] : 0.f);
    } else if (in.chunks == 1) {
        if (resume) h = state[at.b * in.D + c];
    } else if (at.t0 < at.te || at.k == in.chunks - 1) {
        for (int64_t j = 0; j <= at.k; ++j) {
            const float2 v = pe[j * in.D];
            h = carry_on(h, v.x, v.y);
        }
    }
    for (int64_t t = at.t0; t < at.te; t += kRun) {
        const int m = int(at.te - t < kRun ? at.te - t : kRun);
        const Run<T, GATE && !ENDS> x(in, at, t, m);
        if (!ENDS && marks) marks[(at.b * in.marks + t / kRun) * in.D + c] = h;
        float H = 0.f, L = 0.f, o = h;
        const Rows<T> by(y + (at.b * in.T_ + t) * in.D + at.c0, in.D, at.wide, m);
#pragma unroll
        for (int s = 0; s < kRun; ++s) {
            const GateStep g = x.step(s, m, par);
            L += g.l;
            H = fmaf(g.a, H, g.v);
            if constexpr (!ENDS) {
                o = fmaf(g.a, o, g.v);
                by.store(s, at.lc * uint32_t(sizeof(T)), x.out(s, o));
            }
        }
        h = carry_on(h, L, H);
        total += L;
    }
    if constexpr (ENDS) {
        pe[(at.k + 1) * in.D] = make_float2(total, h);
    } else {
        for (int64_t t = at.te > at.t0 ? at.te : at.t0; t < at.t1; ++t)
            io_store(y + (at.b * in.T_ + t) * in.D + c, 0.f);
        if (at.k == in.chunks - 1) state[at.b * in.D + c] = h;
    }
}

// One token per row.
template <typename T>
__global__ __launch_bounds__(256) void gated_step_kernel(GatedIn<T> in, float* __restrict__ state,
                                                         T* __restrict__ y)
{
    const int64_t blocks = (in.D + 255) / 256;
    const int64_t c = blockIdx.x % blocks * 256 + threadIdx.x;
    const int64_t b = blockIdx.x / blocks;
    if (c >= in.D) return;
    const GateParams par(in, c);
    const GateStep g = gate_step(io_load(in.r + b * in.ld_r + c), io_load(in.i + b * in.ld_i + c),
                                 io_load(in.u + b * in.ld_u + c), true, par);
    const float x = carry_on(state[b * in.D + c], g.l, g.v);
    state[b * in.D + c] = x;
    float o = x;
    if (in.z) {
        const float z = io_load(in.z + b * in.ld_z + c);
        o *= z * sigmoid(z);
    }
    io_store(y + b * in.D + c, o);
}

// Workgroups of 16 wavefronts from here on (half again as many as CUs).
constexpr int64_t kManyTiles = 384;

template <typename T, bool GATE>
hipError_t gated(const Gated& g, float* state, bool resume, T* y, float* marks, float2* ends,
                 hipStream_t stream)
{
    const GatedPlan p = gated_plan(g.B, g.T, g.D);
    const GatedIn<T> in = gated_in<T>(g, p);
    const int64_t tiles = gated_tiles(g.B, g.D);
    if (tiles >= kManyTiles) {
        hipLaunchKernelGGL((gated_kernel<T, GATE>), dim3(uint32_t(tiles)), dim3(kWaves * kWave), 0, stream, in,
                           state, int(resume), y, marks);
        return hipGetLastError();
    }
    const dim3 block(kWalkWaves * kWave);
    auto grid = [](int64_t units) { return dim3(uint32_t((units + kWalkWaves - 1) / kWalkWaves)); };
    if (p.chunks > 1) {
        const int64_t units = tiles * (p.chunks - 1);
        hipLaunchKernelGGL((gated_walk_kernel<T, GATE, true>), grid(units), block, 0, stream, in, state,
                           int(resume), static_cast<T*>(nullptr), static_cast<float*>(nullptr), ends, units);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    const int64_t units = tiles * p.chunks;
    hipLaunchKernelGGL((gated_walk_kernel<T, GATE, false>), grid(units), block, 0, stream, in, state, int(resume),
                       y, marks, ends, units);
    return hipGetLastError();
}

}  // namespace

GatedPlan gated_plan(int64_t B, int64_t T, int64_t D)
{
    const int64_t tiles = gated_tiles(B, D);
    if (tiles >= kManyTiles) return GatedPlan{T > 0 ? T : 1, 1, 0};
    GatedPlan p = gated_chunks(B, T, D, 4096, 64);
    p.ws_bytes = p.chunks > 1 ? sizeof(float2) * size_t(B) * p.chunks * D : 0;
    return p;
}

int64_t gated_threads(int64_t B, int64_t T, int64_t D)
{
    const int64_t tiles = gated_tiles(B, D);
    return tiles >= kManyTiles ? tiles * kWaves * kWave : (tiles * gated_plan(B, T, D).chunks + kWalkWaves) * kWave;
}

int64_t gated_step_threads(int64_t B, int64_t D) { return B * ((D + 255) / 256) * 256; }

hipError_t launch_gated(const Gated& g, float* state, bool resume, void* y, float* marks,
                        void* workspace, hipStream_t stream)
{
    float2* ends = static_cast<float2*>(workspace);
    if (g.bf16_io)
        return g.z ? gated<bf16, true>(g, state, resume, static_cast<bf16*>(y), marks, ends, stream)
                   : gated<bf16, false>(g, state, resume, static_cast<bf16*>(y), marks, ends, stream);
    return g.z ? gated<float, true>(g, state, resume, static_cast<float*>(y), marks, ends, stream)
               : gated<float, false>(g, state, resume, static_cast<float*>(y), marks, ends, stream);
}

hipError_t launch_gated_step(const Gated& g, float* state, void* y_t, hipStream_t stream)
{
    const GatedPlan p{1, 1, 0};
    const dim3 grid(uint32_t(gated_step_threads(g.B, g.D) / 256));
    if (g.bf16_io)
        hipLaunchKernelGGL((gated_step_kernel<bf16>), grid, dim3(256), 0, stream, gated_in<bf16>(g, p),
                           state, static_cast<bf16*>(y_t));
    else
        hipLaunchKernelGGL((gated_step_kernel<float>), grid, dim3(256), 0, stream, gated_in<float>(g, p),
                           state, static_cast<float*>(y_t));
    return hipGetLastError();
}

}  // namespace lh
