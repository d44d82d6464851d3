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
// come from those that the prompt's call left before every 64th token, so that inputs
// are read once.  A workgroup of 8 wavefronts holds 64 channels of a row and walks blocks
// of 64 steps from the last to the first, 8 steps to a wavefront; runs meet in LDS both ways,
// forward for the states, backward for X, as in the prompt.  Where rows are few
// the time is cut into chunks and a first launch forms each chunk's (log2 A, G), X before
// it being A X after it + G.  A workgroup's sums over its tokens are one partial row; a
// last launch adds those in a fixed order.
#include "gated_ops.hpp"

namespace lh {
namespace {

constexpr int kWaves = 8;
constexpr int kSpan = kWaves * kRun;  // steps of a block
static_assert(kSpan == kMark, "a block begins at a mark");

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
                                                                   float2* __restrict__ ends)
{
    __shared__ float2 runs[2][kWaves][kWave];
    __shared__ float logs[2][kWaves][kWave];
    const int lane = threadIdx.x % kWave;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t tile = blockIdx.x % in.tiles;
    const int64_t k = blockIdx.x / in.tiles % (in.chunks - 1) + 1;
    const int64_t b = blockIdx.x / in.tiles / (in.chunks - 1);
    const int64_t c0 = tile * kTile;
    const uint32_t lc = uint32_t(c0 + lane < in.D ? lane : in.D - 1 - c0);
    const int64_t c = c0 + lc;
    const GateParams par(in, c);
    const int64_t n = gated_length(in.lengths, b, in.T_);
    const int64_t t0 = k * in.chunk;
    const int64_t te = t0 + in.chunk < n ? t0 + in.chunk : n;
    const T* pr = in.r + b * in.T_ * in.ld_r + c0;
    const T* pz = GATE ? in.z + b * in.T_ * in.ld_z + c0 : nullptr;
    const T* pd = dy + b * in.T_ * in.D + c0;

    float X = 0.f, total = 0.f;
    int turn = 0;
    for (int64_t tb = te > t0 ? t0 + (te - 1 - t0) / kSpan * kSpan : t0 - 1; tb >= t0; tb -= kSpan, turn ^= 1) {
        const int64_t t = tb + wave * kRun;
        const int m = int(te - t < kRun ? te - t : kRun);
        T r[kRun], d[kRun], z[kRun];
#pragma unroll
        for (int s = 0; s < kRun; ++s) {
            const int64_t row = t + s < te ? t + s : te - 1;
            r[s] = (pr + row * in.ld_r)[lc];
            d[s] = (pd + row * in.D)[lc];
            if constexpr (GATE) z[s] = (pz + row * in.ld_z)[lc];
        }
        float G = 0.f, L = 0.f;
#pragma unroll
        for (int s = kRun - 1; s >= 0; --s) {
            const float l = par.rate2 * gate_pair(fmaf(io_load(&r[s]), -kLog2e, par.nrb)).x;
            float slope;
            const float q = through_gate<GATE>(io_load(&d[s]), GATE ? io_load(&z[s]) : 0.f, &slope);
            if (s < m) {
                L += l;
                G = exp2_fast(-l) * (q + G);
            }
        }
        runs[turn][wave][lane] = make_float2(exp2_fast(-L), G);
        logs[turn][wave][lane] = L;
        __syncthreads();
        float end = 0.f, lend = 0.f;
#pragma unroll
        for (int j = kWaves - 1; j >= 0; --j) {
            const float2 x = runs[turn][j][lane];
            end = fmaf(x.x, end, x.y);
            lend += logs[turn][j][lane];
        }
        X = carry_on(X, lend, end);
        total += lend;
    }
    if (wave == 0) ends[(b * in.chunks + k) * in.D + c] = make_float2(total, X);
}

template <typename T>
struct GatedOut {
    const T* dy;
    const float *marks, *dlast;
    T *dr, *di, *du, *dz;
    float* dfirst;
    float* part;  // [B chunks, 3, D]: drate, dr_bias, di_bias of each workgroup's tokens
};

template <typename T, bool GATE>
__global__ __launch_bounds__(kWaves* kWave, 4) void gated_grad_kernel(GatedIn<T> in, GatedOut<T> out,
                                                                      const float2* __restrict__ ends)
{
    __shared__ float4 runs[2][kWaves][kWave];  // A, H, G, log2 A negated
    __shared__ float red[3][kWaves][kWave];
    const int lane = threadIdx.x % kWave;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t tile = blockIdx.x % in.tiles;
    const int64_t k = blockIdx.x / in.tiles % in.chunks;
    const int64_t b = blockIdx.x / in.tiles / in.chunks;
    const int64_t c0 = tile * kTile;
    const uint32_t lc = uint32_t(c0 + lane < in.D ? lane : in.D - 1 - c0);
    const int64_t c = c0 + lc;
    const GateParams par(in, c);
    const int64_t n = gated_length(in.lengths, b, in.T_);
    const int64_t t0 = k * in.chunk;
    const int64_t t1 = t0 + in.chunk < in.T_ ? t0 + in.chunk : in.T_;
    const int64_t te = t1 < n ? t1 : n;

    float X = out.dlast ? out.dlast[b * in.D + c] : 0.f;
    for (int64_t j = in.chunks - 1; j > k; --j) {
        const float2 e = ends[(b * in.chunks + j) * in.D + c];
        X = carry_on(X, e.x, e.y);
    }
    const T* pr = in.r + b * in.T_ * in.ld_r + c0;
    const T* pi = in.i + b * in.T_ * in.ld_i + c0;
    const T* pu = in.u + b * in.T_ * in.ld_u + c0;
    const T* pz = GATE ? in.z + b * in.T_ * in.ld_z + c0 : nullptr;
    const int64_t rows = b * in.T_ * in.D + c0;
    const T* pd = out.dy + rows;
    const float* pm = out.marks + b * in.marks * in.D + c0;

    float sum_rate = 0.f, sum_r = 0.f, sum_i = 0.f;
    int turn = 0;
    for (int64_t tb = te > t0 ? t0 + (te - 1 - t0) / kSpan * kSpan : t0 - 1; tb >= t0; tb -= kSpan, turn ^= 1) {
        const int64_t t = tb + wave * kRun;
        const int m = int(te - t < kRun ? te - t : kRun);
        T r[kRun], i[kRun], x[kRun], d[kRun], z[kRun];
#pragma unroll
        for (int s = 0; s < kRun; ++s) {
            const int64_t row = t + s < te ? t + s : te - 1;
            r[s] = (pr + row * in.ld_r)[lc];
            i[s] = (pi + row * in.ld_i)[lc];
            x[s] = (pu + row * in.ld_u)[lc];
            d[s] = (pd + row * in.D)[lc];
            if constexpr (GATE) z[s] = (pz + row * in.ld_z)[lc];
        }
        float h = (pm + tb / kMark * in.D)[lc];
        // a; w = sqrt(1 - a^2) p; 1 - p; 1 - f; a^2 L / (1 - a^2); L a
        float a[kRun], w[kRun], np[kRun], nf[kRun], kq[kRun], la[kRun], u[kRun], q[kRun], slope[kRun];
        float H = 0.f, L = 0.f;
#pragma unroll
        for (int s = 0; s < kRun; ++s) {
            const float2 f = gate_pair(fmaf(io_load(&r[s]), -kLog2e, par.nrb));
            const float2 p = gate_pair(fmaf(io_load(&i[s]), -kLog2e, par.nib));
            float l = par.rate2 * f.x;
            l = l > 256.f ? 256.f : l;  // (a is 0, and must not meet infinity below)
            const float as = exp2_fast(-l), a2 = as * as, y = 2.f * l;
            const bool small = y < kSmall;
            const float series = decay_series(y);
            const float g2 = small ? y * series : 1.f - a2;
            kq[s] = a2 * (0.5f * kLn2) * (small ? 1.f : y) * rcp_fast(small ? series : g2);
            la[s] = kLn2 * l * as;
            nf[s] = f.y;
            np[s] = p.y;
            u[s] = io_load(&x[s]);
            q[s] = through_gate<GATE>(io_load(&d[s]), GATE ? io_load(&z[s]) : 0.f, &slope[s]);
            w[s] = __builtin_amdgcn_sqrtf(g2) * p.x;
            a[s] = as;
            if (s < m) {
                L += l;
                H = fmaf(as, H, w[s] * u[s]);
            }
        }
        float G = 0.f;
#pragma unroll
        for (int s = kRun - 1; s >= 0; --s)
            if (s < m) G = a[s] * (q[s] + G);
        runs[turn][wave][lane] = make_float4(exp2_fast(-L), H, G, L);
        __syncthreads();
        float after = 0.f, lafter = 0.f, end = 0.f, lend = 0.f;
#pragma unroll
        for (int j = kWaves - 1; j >= 0; --j) {
            if (j == wave) after = end, lafter = lend;
            const float4 v = runs[turn][j][lane];
            end = fmaf(v.x, end, v.z);
            lend += v.w;
        }
#pragma unroll
        for (int j = 0; j < kWaves - 1; ++j) {
            const float4 v = runs[turn][j][lane];
            if (j < wave) h = fmaf(v.x, h, v.y);
        }
        const int64_t o = rows + t * in.D;
        // L dL / dh, the states forward
        float dl[kRun];
#pragma unroll
        for (int s = 0; s < kRun; ++s) {
            const float v = w[s] * u[s];
            dl[s] = fmaf(v, kq[s], -la[s] * h);
            h = fmaf(a[s], h, v);
            if constexpr (GATE)
                if (s < m) io_store(out.dz + o + s * in.D + lc, slope[s] * h);
        }
        float dx = wave == kWaves - 1 ? X : fmaf(exp2_fast(-lafter), X, after);
#pragma unroll
        for (int s = kRun - 1; s >= 0; --s) {
            if (s < m) {
                const float dh = q[s] + dx;
                const float du = dh * w[s], di = du * u[s] * np[s];
                const float ldl = dh * dl[s], dr = ldl * nf[s];
                io_store(out.du + o + s * in.D + lc, du);
                io_store(out.di + o + s * in.D + lc, di);
                io_store(out.dr + o + s * in.D + lc, dr);
                sum_rate += ldl;
                sum_r += dr;
                sum_i += di;
                dx = a[s] * dh;
            }
        }
        X = carry_on(X, lend, end);
    }
    for (int64_t t = (te > t0 ? te : t0) + wave; t < t1; t += kWaves) {
        const int64_t o = rows + t * in.D + lc;
        io_store(out.du + o, 0.f);
        io_store(out.di + o, 0.f);
        io_store(out.dr + o, 0.f);
        if constexpr (GATE) io_store(out.dz + o, 0.f);
    }
    red[0][wave][lane] = sum_rate;
    red[1][wave][lane] = sum_r;
    red[2][wave][lane] = sum_i;
    __syncthreads();
    if (wave < 3) {
        float v = 0.f;
#pragma unroll
        for (int j = 0; j < kWaves; ++j) v += red[wave][j][lane];
        if (wave == 0) {
            const float rate = in.rate[c];
            v = rate == 0.f ? 0.f : v / rate;
        }
        out.part[((b * in.chunks + k) * 3 + wave) * in.D + c] = v;
    }
    if (k == 0 && wave == 0 && out.dfirst) out.dfirst[b * in.D + c] = X;
}

template <typename T, bool GATE>
hipError_t gated_grad(const Gated& g, const GatedGrads& d, void* workspace, hipStream_t stream)
{
    const GatedPlan p = gated_grad_plan(g.B, g.T, g.D);
    const GatedIn<T> in = gated_in<T>(g, p);
    const int64_t P = g.B * p.chunks;
    float* part = static_cast<float*>(workspace);
    // (an even number of floats before it, so that pairs are aligned)
    float2* ends = reinterpret_cast<float2*>(part + (P * 3 * g.D + 1) / 2 * 2);
    GatedOut<T> out;
    out.dy = static_cast<const T*>(d.dy), out.marks = d.marks, out.dlast = d.dlast;
    out.dr = static_cast<T*>(d.dr), out.di = static_cast<T*>(d.di), out.du = static_cast<T*>(d.du);
    out.dz = static_cast<T*>(d.dz), out.dfirst = d.dfirst, out.part = part;
    const dim3 block(kWaves * kWave);
    hipError_t e;
    if (p.chunks > 1) {
        hipLaunchKernelGGL((gated_ends_kernel<T, GATE>), dim3(uint32_t(g.B * in.tiles * (p.chunks - 1))),
                           block, 0, stream, in, out.dy, ends);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    hipLaunchKernelGGL((gated_grad_kernel<T, GATE>), dim3(uint32_t(g.B * in.tiles * p.chunks)), block, 0,
                       stream, in, out, ends);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    return launch_column_sum(part, P, g.D, d.drate, g.D, d.dr_bias, g.D, d.di_bias, stream);
}

}  // namespace

GatedPlan gated_grad_plan(int64_t B, int64_t T, int64_t D)
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
    const size_t rows = size_t(B) * p.chunks * D;
    p.ws_bytes = sizeof(float) * ((rows * 3 + 1) / 2 * 2) + (p.chunks > 1 ? sizeof(float2) * rows : 0);
    return p;
}

int64_t gated_grad_threads(int64_t B, int64_t T, int64_t D)
{
    const int64_t kernel = gated_tiles(B, D) * gated_grad_plan(B, T, D).chunks * kWaves * kWave;
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
