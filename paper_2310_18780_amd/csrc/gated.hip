// Gated linear recurrence over prompts and for single tokens, per channel:
//
//   f = sigmoid(r + r_bias),  p = sigmoid(i + i_bias),  a = e^(-rate f)
//   h <- a h + sqrt(1 - a^2) p u,   y = h (times z sigmoid(z))
//
// h after any run of steps is A h_before + H, with A the product of the run's decays and
// H what its inputs alone leave.  A workgroup of 16 wavefronts holds 64 channels of a row,
// one to a lane, and walks the time in blocks of 128 steps, 8 to a wavefront: each
// wavefront forms (A, H) of its run, they meet in LDS, each chains those before its own to
// its entry state and walks its steps again from registers.  Inputs are read once, outputs
// written once.  Where rows are few the prompt is cut into chunks; a first launch forms
// each chunk's (log2 A, H), and each chunk of the second folds those before it.
//
// A block's decay is carried on as the sum of its logarithms (carry_on): products of
// roundings near 1 would be off by 2^-24 a step over thousands of steps.
#include "gated_ops.hpp"

namespace lh {
namespace {

constexpr int kWaves = 16;
constexpr int kSpan = kWaves * kRun;  // steps of a block
static_assert(kSpan % kMark == 0, "marks lie before runs");

// ENDS: the chunks' ends only, into slots 1 .. of ends [B, chunks, D] (log2 of the decay,
// negated, and state from zero); slot 0 holds the start.
template <typename T, bool GATE, bool ENDS>
__global__ __launch_bounds__(kWaves* kWave) void gated_kernel(
    GatedIn<T> in, float* state, int resume, T* __restrict__ y, float* __restrict__ marks,
    float2* __restrict__ ends)
{
    __shared__ float2 runs[2][kWaves][kWave];
    __shared__ float logs[2][kWaves][kWave];
    const int lane = threadIdx.x % kWave;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t tile = blockIdx.x % in.tiles;
    const int64_t per = ENDS ? in.chunks - 1 : in.chunks;
    const int64_t k = blockIdx.x / in.tiles % per;
    const int64_t b = blockIdx.x / in.tiles / per;
    // Lanes past the last channel repeat it: they store the same bits to the same place.
    const int64_t c0 = tile * kTile;
    const uint32_t lc = uint32_t(c0 + lane < in.D ? lane : in.D - 1 - c0);
    const int64_t c = c0 + lc;
    const GateParams par(in, c);
    const int64_t n = gated_length(in.lengths, b, in.T_);
    const int64_t t0 = k * in.chunk;
    const int64_t t1 = t0 + in.chunk < in.T_ ? t0 + in.chunk : in.T_;
    const int64_t te = t1 < n ? t1 : n;  // the chunk's tokens end here

    float h = 0.f, total = 0.f;  // state before the block; log2 of the decays so far, negated
    if constexpr (ENDS) {
        if (k == 0 && wave == 0)
            ends[b * in.chunks * in.D + c] = make_float2(0.f, resume ? state[b * in.D + c] : 0.f);
    } else if (in.chunks == 1) {
        if (resume) h = state[b * in.D + c];
    } else {
        const float2* e = ends + b * in.chunks * in.D + c;
        for (int64_t j = 0; j <= k; ++j) {
            const float2 v = e[j * in.D];
            h = carry_on(h, v.x, v.y);
        }
    }

    // (a uniform row's address and a lane's offset)
    const T* pr = in.r + b * in.T_ * in.ld_r + c0;
    const T* pi = in.i + b * in.T_ * in.ld_i + c0;
    const T* pu = in.u + b * in.T_ * in.ld_u + c0;
    const T* pz = GATE && !ENDS ? in.z + b * in.T_ * in.ld_z + c0 : nullptr;
    T* py = ENDS ? nullptr : y + b * in.T_ * in.D + c0;

    T r[kRun], i[kRun], u[kRun], z[kRun];
    // a step past the tokens reads the last one again and takes no part
    auto load = [&](int64_t t) {
#pragma unroll
        for (int s = 0; s < kRun; ++s) {
            const int64_t row = t + s < te ? t + s : te - 1;
            r[s] = (pr + row * in.ld_r)[lc];
            i[s] = (pi + row * in.ld_i)[lc];
            u[s] = (pu + row * in.ld_u)[lc];
            if constexpr (GATE && !ENDS) z[s] = (pz + row * in.ld_z)[lc];
        }
    };
    int turn = 0;
    if (t0 < te) load(t0 + wave * kRun);
    for (int64_t tb = t0; tb < te; tb += kSpan, turn ^= 1) {
        const int64_t t = tb + wave * kRun;
        const int m = int(te - t < kRun ? te - t : kRun);  // steps of this run (<= 0: none)
        float a[kRun], v[kRun], gate[kRun];
        float H = 0.f, L = 0.f;
#pragma unroll
        for (int s = 0; s < kRun; ++s) {
            const float f = rcp_fast(1.f + exp2_fast(fmaf(io_load(&r[s]), -kLog2e, par.nrb)));
            const float p = rcp_fast(1.f + exp2_fast(fmaf(io_load(&i[s]), -kLog2e, par.nib)));
            const float l = par.rate2 * f;
            const float as = exp2_fast(-l);
            const float q = one_minus(2.f * l, as * as);
            const float vs = __builtin_amdgcn_sqrtf(q) * p * io_load(&u[s]);
            a[s] = s < m ? as : 1.f;
            v[s] = s < m ? vs : 0.f;
            L += s < m ? l : 0.f;
            H = fmaf(a[s], H, v[s]);
            if constexpr (GATE && !ENDS) {
                const float zs = io_load(&z[s]);
                gate[s] = zs * sigmoid(zs);
            }
        }
        if (tb + kSpan < te) load(t + kSpan);
        runs[turn][wave][lane] = make_float2(exp2_fast(-L), H);
        logs[turn][wave][lane] = L;
        __syncthreads();
        // from zero: the states and decays before this run, and of the whole block
        float e = 0.f, le = 0.f, end = 0.f, lend = 0.f;
#pragma unroll
        for (int j = 0; j < kWaves; ++j) {
            if (j == wave) e = end, le = lend;
            const float2 x = runs[turn][j][lane];
            end = fmaf(x.x, end, x.y);
            lend += logs[turn][j][lane];
        }
        if constexpr (!ENDS) {
            float x = fmaf(exp2_fast(-le), h, e);
            if (wave == 0) x = h;
            if (marks && t % kMark == 0 && t < te)
                marks[(b * in.marks + t / kMark) * in.D + c] = x;
#pragma unroll
            for (int s = 0; s < kRun; ++s) {
                x = fmaf(a[s], x, v[s]);
                if (s < m) io_store(py + (t + s) * in.D + lc, GATE ? x * gate[s] : x);
            }
        }
        h = carry_on(h, lend, end);
        total += lend;
    }
    if constexpr (ENDS) {
        if (wave == 0) ends[(b * in.chunks + k + 1) * in.D + c] = make_float2(total, h);
    } else {
        for (int64_t t = (te > t0 ? te : t0) + wave; t < t1; t += kWaves)
            io_store(py + t * in.D + lc, 0.f);
        if (k == in.chunks - 1 && wave == 0) state[b * in.D + c] = h;
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
    const float r = io_load(in.r + b * in.ld_r + c), i = io_load(in.i + b * in.ld_i + c);
    const float u = io_load(in.u + b * in.ld_u + c), h = state[b * in.D + c];
    const float f = rcp_fast(1.f + exp2_fast(fmaf(r, -kLog2e, par.nrb)));
    const float p = rcp_fast(1.f + exp2_fast(fmaf(i, -kLog2e, par.nib)));
    const float l = par.rate2 * f, a = exp2_fast(-l);
    const float x = carry_on(h, l, __builtin_amdgcn_sqrtf(one_minus(2.f * l, a * a)) * p * u);
    state[b * in.D + c] = x;
    float o = x;
    if (in.z) {
        const float z = io_load(in.z + b * in.ld_z + c);
        o *= z * sigmoid(z);
    }
    io_store(y + b * in.D + c, o);
}

template <typename T>
hipError_t gated(const Gated& g, float* state, bool resume, T* y, float* marks, float2* ends,
                 hipStream_t stream)
{
    const GatedPlan p = gated_plan(g.B, g.T, g.D);
    const GatedIn<T> in = gated_in<T>(g, p);
    const dim3 block(kWaves * kWave);
    if (p.chunks > 1) {
        hipLaunchKernelGGL((gated_kernel<T, false, true>), dim3(uint32_t(g.B * in.tiles * (p.chunks - 1))),
                           block, 0, stream, in, state, int(resume), static_cast<T*>(nullptr),
                           static_cast<float*>(nullptr), ends);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    const dim3 grid(uint32_t(g.B * in.tiles * p.chunks));
    if (g.z)
        hipLaunchKernelGGL((gated_kernel<T, true, false>), grid, block, 0, stream, in, state, int(resume),
                           y, marks, ends);
    else
        hipLaunchKernelGGL((gated_kernel<T, false, false>), grid, block, 0, stream, in, state, int(resume),
                           y, marks, ends);
    return hipGetLastError();
}

}  // namespace

GatedPlan gated_plan(int64_t B, int64_t T, int64_t D)
{
    // two workgroups to a CU
    const int64_t tiles = gated_tiles(B, D), spans = (T + kSpan - 1) / kSpan;
    int64_t chunks = tiles >= 384 ? 1 : (512 + tiles - 1) / tiles;
    if (chunks > spans) chunks = spans;
    if (chunks < 1) chunks = 1;
    const int64_t per = spans > 0 ? (spans + chunks - 1) / chunks : 1;
    GatedPlan p;
    p.chunk = per * kSpan;
    p.chunks = spans > 0 ? (spans + per - 1) / per : 1;
    p.ws_bytes = p.chunks > 1 ? sizeof(float2) * size_t(B) * p.chunks * D : 0;
    return p;
}

int64_t gated_threads(int64_t B, int64_t T, int64_t D)
{
    return gated_tiles(B, D) * gated_plan(B, T, D).chunks * kWaves * kWave;
}

int64_t gated_step_threads(int64_t B, int64_t D) { return B * ((D + 255) / 256) * 256; }

hipError_t launch_gated(const Gated& g, float* state, bool resume, void* y, float* marks,
                        void* workspace, hipStream_t stream)
{
    float2* ends = static_cast<float2*>(workspace);
    if (g.bf16_io) return gated(g, state, resume, static_cast<bf16*>(y), marks, ends, stream);
    return gated(g, state, resume, static_cast<float*>(y), marks, ends, stream);
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
