// Gradients of the gated linear recurrence.  With q the gradient of y (times z sigmoid(z)),
// per channel and backwards in time:
//
//   dh_t = q_t + X_t,  X_(t-1) = a_t dh_t   (X after the last token: dlast; X_-1: dfirst)
//   v = sqrt(1 - a^2) p u:  du = dh v / u,  di = dh v (1 - p)
//   L = rate f:  L dL = dh (v a^2 L / (1 - a^2) - L a h_(t-1)),
//   dr = L dL (1 - f),  drate = sum of L dL / rate
//   dz = dy h_t (the slope of z sigmoid(z))
//
// (L / (1 - a^2) -> 1 / 2 as L -> 0: nothing is divided by a small number.)  The states
// come from those that the prompt's call left before every 8th token, so that inputs
// are read once.  A wavefront holds 64 channels of a row, one to a lane, and walks a
// chunk of the time by itself, 8 steps at a time from the last to the first: forward through
// the 8 for the states and what does not need dh, then backward.  A first launch forms each
// chunk's (log2 A, G), X before it being A X after it + G; each chunk of the second folds
// those after it.  A chunk's sums over its tokens are one partial row; a last launch adds those
// in a fixed order.
//
// Bound by vector issue (0.59 of the time) beside memory: 4 x 4096 x 2048 bfloat16 with gate
// takes 45 us for the ends of the chunks and 127 for the gradients (0.64 GB: 124 at a copy's
// rate).  A first form, which formed the states again from their inputs, took 614.  At the 80
// registers of 6 wavefronts to a SIMD the gradients' kernel spills 4, and 16 to 33 scalar ones.
#include "gated_ops.hpp"

namespace lh {
namespace {

constexpr int kWaves = 4;  // wavefronts of a workgroup, each with a chunk of its own

// dy and what reaches the state of it, where there is a gate
template <bool GATE>
__device__ __forceinline__ float through_gate(float dy, float z, float* slope)
{
    if constexpr (!GATE) return dy;
    const float p = sigmoid(z);
    *slope = dy * p * fmaf(z, 1.f - p, 1.f);
    return dy * (z * p);
}

// The ends of the chunks 1 .. (slot k of ends [B, chunks, D]: log2 of the decay, negated,
// and X before the chunk from zero after it).
template <typename T, bool GATE>
__global__ __launch_bounds__(kWaves* kWave) void gated_ends_kernel(GatedIn<T> in, const T* __restrict__ dy,
                                                                   float2* __restrict__ ends, int64_t units)
{
    const int64_t unit = int64_t(blockIdx.x) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    if (unit >= units) return;
    const Place at(in, unit, in.chunks - 1, 1);
    const GateParams par(in, at.c0 + at.lc);
    const uint32_t lane = at.lc * uint32_t(sizeof(T));
    float X = 0.f, total = 0.f;
    for (int64_t t = at.last_run(); t >= at.t0; t -= kRun) {
        const int m = int(at.te - t < kRun ? at.te - t : kRun);
        const int64_t row = at.b * in.T_ + t;
        const Rows<T> br(in.r + row * in.ld_r + at.c0, in.ld_r, at.wide, m);
        const Rows<T> bd(dy + row * in.D + at.c0, in.D, at.wide, m);
        T r[kRun], d[kRun], z[kRun];
#pragma unroll
        for (int s = 0; s < kRun; ++s) {
            r[s] = br.load(s, lane);
            d[s] = bd.load(s, lane);
        }
        if constexpr (GATE) {
            const Rows<T> bz(in.z + row * in.ld_z + at.c0, in.ld_z, at.wide, m);
#pragma unroll
            for (int s = 0; s < kRun; ++s) z[s] = bz.load(s, lane);
        }
        float G = 0.f, L = 0.f;
#pragma unroll
        for (int s = kRun - 1; s >= 0; --s) {
            float l = par.rate2 * gate_pair(fmaf(io_load(&r[s]), -kLog2e, par.nrb)).x;
            l = s < m ? l : 0.f;
            float slope;
            const float q = through_gate<GATE>(io_load(&d[s]), GATE ? io_load(&z[s]) : 0.f, &slope);
            L += l;
            G = exp2_fast(-l) * (q + G);
        }
        X = carry_on(X, L, G);
        total += L;
    }
    ends[(at.b * in.chunks + at.k) * in.D + at.c0 + at.lc] = make_float2(total, X);
}

template <typename T>
struct GatedOut {
    const T* dy;
    const float *marks, *dlast;
    T *dr, *di, *du, *dz;
    float* dfirst;
    float* part;  // [B chunks, 3, D]: drate, dr_bias, di_bias of each chunk's tokens
};

template <typename T, bool GATE>
__global__ __launch_bounds__(kWaves* kWave, 6) void gated_grad_kernel(GatedIn<T> in, GatedOut<T> out,
                                                                   const float2* __restrict__ ends, int64_t units)
{
    const int64_t unit = int64_t(blockIdx.x) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    if (unit >= units) return;
    const Place at(in, unit, in.chunks, 0);
    const int64_t c = at.c0 + at.lc, rows = at.b * in.T_ * in.D;
    const uint32_t lane = at.lc * uint32_t(sizeof(T));
    const GateParams par(in, c);
    // the chunks after, each by the decays before it
    float X = 0.f, decay = 0.f;
    constexpr int kAhead = 8;
    for (int64_t j = at.k + 1; j < in.chunks; j += kAhead) {
        float2 e[kAhead];
#pragma unroll
        for (int s = 0; s < kAhead; ++s)
            e[s] = ends[(at.b * in.chunks + (j + s < in.chunks ? j + s : in.chunks - 1)) * in.D + c];
#pragma unroll
        for (int s = 0; s < kAhead; ++s) {
            const bool there = j + s < in.chunks;
            X = fmaf(exp2_fast(-decay), there ? e[s].y : 0.f, X);
            decay += there ? e[s].x : 0.f;
        }
    }
    if (out.dlast) X = fmaf(exp2_fast(-decay), out.dlast[at.b * in.D + c], X);
    float sum_rate = 0.f, sum_r = 0.f, sum_i = 0.f;
    for (int64_t t = at.last_run(); t >= at.t0; t -= kRun) {
        const int m = int(at.te - t < kRun ? at.te - t : kRun);
        const int64_t row = at.b * in.T_ + t, o = rows + t * in.D + at.c0;
        T r[kRun], i[kRun], x[kRun], d[kRun], z[kRun];
        {
            const Rows<T> br(in.r + row * in.ld_r + at.c0, in.ld_r, at.wide, m);
            const Rows<T> bi(in.i + row * in.ld_i + at.c0, in.ld_i, at.wide, m);
            const Rows<T> bu(in.u + row * in.ld_u + at.c0, in.ld_u, at.wide, m);
            const Rows<T> bd(out.dy + o, in.D, at.wide, m);
#pragma unroll
            for (int s = 0; s < kRun; ++s) {
                r[s] = br.load(s, lane);
                i[s] = bi.load(s, lane);
                x[s] = bu.load(s, lane);
                d[s] = bd.load(s, lane);
            }
            if constexpr (GATE) {
                const Rows<T> bz(in.z + row * in.ld_z + at.c0, in.ld_z, at.wide, m);
#pragma unroll
                for (int s = 0; s < kRun; ++s) z[s] = bz.load(s, lane);
            }
        }
        float h = out.marks[(at.b * in.marks + t / kRun) * in.D + c];
        const Rows<T> bdz((GATE ? out.dz : out.du) + o, in.D, at.wide, m);
        // a; w = sqrt(1 - a^2) p; u (1 - p); 1 - f; L dL / dh; the gradient that y brings
        float a[kRun], w[kRun], un[kRun], nf[kRun], dl[kRun], q[kRun];
        float L = 0.f;
#pragma unroll
        for (int s = 0; s < kRun; ++s) {
            const float2 f = gate_pair(fmaf(io_load(&r[s]), -kLog2e, par.nrb));
            const float2 p = gate_pair(fmaf(io_load(&i[s]), -kLog2e, par.nib));
            // (where it is 256, a is 0 already, and must not meet infinity below; a step that is
            // not there decays nothing, and all it reads is zeros)
            float l = par.rate2 * f.x;
            l = l > 256.f ? 256.f : l;
            l = s < m ? l : 0.f;
            const float as = exp2_fast(-l), a2 = as * as, y = 2.f * l;
            const bool small = y < kSmall;
            const float series = decay_series(y);
            const float g2 = small ? y * series : 1.f - a2;
            // a L / (1 - a^2)
            const float kq = as * ((0.5f * kLn2) * (small ? 1.f : y)) * rcp_fast(small ? series : g2);
            const float u = io_load(&x[s]);
            a[s] = as;
            nf[s] = f.y;
            w[s] = __builtin_amdgcn_sqrtf(g2) * p.x;
            un[s] = u * p.y;
            const float v = w[s] * u;
            dl[s] = as * fmaf(v, kq, -kLn2 * l * h);
            h = fmaf(as, h, v);
            float slope;
            q[s] = through_gate<GATE>(io_load(&d[s]), GATE ? io_load(&z[s]) : 0.f, &slope);
            if constexpr (GATE) bdz.store(s, lane, slope * h);
            L += l;
        }
        const Rows<T> bdu(out.du + o, in.D, at.wide, m), bdi(out.di + o, in.D, at.wide, m),
            bdr(out.dr + o, in.D, at.wide, m);
        float dx = X, G = 0.f;
#pragma unroll
        for (int s = kRun - 1; s >= 0; --s) {
            const float dh = q[s] + dx;
            const float du = dh * w[s], di = du * un[s];
            const float ldl = dh * dl[s], dr = ldl * nf[s];
            bdu.store(s, lane, du);
            bdi.store(s, lane, di);
            bdr.store(s, lane, dr);
            // (a step that is not there adds zeros, of a state or a gradient that is finite)
            sum_rate += ldl;
            sum_r += dr;
            sum_i += di;
            dx = a[s] * dh;
            G = a[s] * (q[s] + G);
        }
        X = carry_on(X, L, G);
    }
    for (int64_t t = at.te > at.t0 ? at.te : at.t0; t < at.t1; ++t) {
        const int64_t o = rows + t * in.D + c;
        io_store(out.du + o, 0.f);
        io_store(out.di + o, 0.f);
        io_store(out.dr + o, 0.f);
        if constexpr (GATE) io_store(out.dz + o, 0.f);
    }
    float* part = out.part + (at.b * in.chunks + at.k) * 3 * in.D + c;
    const float rate = in.rate[c];
    part[0] = rate == 0.f ? 0.f : sum_rate / rate;
    part[in.D] = sum_r;
    part[2 * in.D] = sum_i;
    if (at.k == 0 && out.dfirst) out.dfirst[at.b * in.D + c] = X;
}

template <typename T, bool GATE>
hipError_t gated_grad(const Gated& g, const GatedGrads& d, void* workspace, hipStream_t stream)
{
    const GatedGradPlan p = gated_grad_plan(g.B, g.T, g.D);
    const GatedIn<T> in = gated_in<T>(g, p.chunk, p.chunks, 0);
    const int64_t P = g.B * p.chunks, tiles = gated_tiles(g.B, g.D);
    float* part = static_cast<float*>(workspace);
    // (an even number of floats before it, so that pairs are aligned)
    float2* ends = reinterpret_cast<float2*>(part + (P * 3 * g.D + 1) / 2 * 2);
    GatedOut<T> out;
    out.dy = static_cast<const T*>(d.dy), out.marks = d.marks, out.dlast = d.dlast;
    out.dr = static_cast<T*>(d.dr), out.di = static_cast<T*>(d.di), out.du = static_cast<T*>(d.du);
    out.dz = static_cast<T*>(d.dz), out.dfirst = d.dfirst, out.part = part;
    const dim3 block(kWaves * kWave);
    auto grid = [](int64_t units) { return dim3(uint32_t((units + kWaves - 1) / kWaves)); };
    hipError_t e;
    if (p.chunks > 1) {
        const int64_t units = tiles * (p.chunks - 1);
        hipLaunchKernelGGL((gated_ends_kernel<T, GATE>), grid(units), block, 0, stream, in, out.dy, ends, units);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    const int64_t units = tiles * p.chunks;
    hipLaunchKernelGGL((gated_grad_kernel<T, GATE>), grid(units), block, 0, stream, in, out, ends, units);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    return launch_column_sum(part, P, g.D, d.drate, g.D, d.dr_bias, g.D, d.di_bias, stream);
}

}  // namespace

GatedGradPlan gated_grad_plan(int64_t B, int64_t T, int64_t D)
{
    // More chunks fill the GPU where channels are few, but each folds all after it: 16 steps or
    // more, and not above five chunks to a step of theirs (prompt and gradient, bfloat16 with gate:
    // 2 x 584 x 128 takes 45 us with chunks of 64 and 31 with 16; 1 x 65536 x 128 takes 150 us
    // with chunks of 120 and 337 with 24)
    // (6144: the wavefronts that the GPU holds, 6 to a SIMD)
    int64_t least = 16;
    while (least * least * 5 < T) least += kRun;
    GatedGradPlan p = gated_chunks(B, T, D, 6144, least);
    const size_t rows = size_t(B) * p.chunks * D;
    p.ws_bytes = sizeof(float) * ((rows * 3 + 1) / 2 * 2) + (p.chunks > 1 ? sizeof(float2) * rows : 0);
    return p;
}

int64_t gated_grad_threads(int64_t B, int64_t T, int64_t D)
{
    const int64_t kernel = (gated_tiles(B, D) * gated_grad_plan(B, T, D).chunks + kWaves) * kWave;
    const int64_t sums = 3 * D * 32 + 1024;
    return kernel > sums ? kernel : sums;
}

hipError_t launch_gated_grad(const Gated& g, const GatedGrads& d, void* workspace, hipStream_t stream)
{
    if (g.bf16_io)
        return g.z ? gated_grad<bf16, true>(g, d, workspace, stream)
                   : gated_grad<bf16, false>(g, d, workspace, stream);
    return g.z ? gated_grad<float, true>(g, d, workspace, stream)
               : gated_grad<float, false>(g, d, workspace, stream);
}

}  // namespace lh
