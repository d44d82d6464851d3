// Gated linear recurrence over prompts and for single tokens, per channel:
//
//   f = sigmoid(r + r_bias),  p = sigmoid(i + i_bias),  a = e^(-rate f)
//   h <- a h + sqrt(1 - a^2) p u,   y = h (times z sigmoid(z))
//
// h after any run of steps is A h_before + H, with A the product of the run's decays and
// H what its inputs alone leave.  A workgroup of 16 wavefronts holds 64 channels of a row, one
// to a lane, and takes a block of 128 steps, 8 to a wavefront.  Each wavefront forms (A, H) of its
// run, they meet in LDS, each chains those before its own to its entry state and walks its
// steps again from registers: inputs are read once, outputs written once.  Where there are
// rows enough a workgroup goes from block to block; else several take a tile's blocks in turn, and
// each leaves what its block alone does to a state as soon as it knows that, and finds the
// state before it by looking back at the blocks before.
//
// Bound by vector issue beside memory: a step of a channel is 36 vector instructions and 8
// transcendental ones, about 275 cycles of a wavefront.  16 x 4096 x 2048 bfloat16 with gate:
// 304 us (1.34 GB: 260 at a copy's rate; vector issue 0.58); 1 x 65536 x 1024 without gate, where
// 32 workgroups share each of 16 tiles: 175 us (0.54 GB: 104), 241 where a launch before formed
// the ends of chunks and so read the inputs once more.  16 x 4096 x 2048 float32: 543 us with gate
// (2.68 GB: 521), 442 without.  At the 64 registers that two workgroups to a CU leave, the form with
// gate spills 4 (20 bytes of scratch a lane), and each form 30 to 60 scalar ones into vector lanes.
//
// A block's decay is carried on as the sum of its logarithms (carry_on): products of roundings
// near 1 would be off by 2^-24 a step over thousands of steps.
#include "gated_ops.hpp"

namespace lh {
namespace {

constexpr int kWaves = 16;
constexpr int kSpan = kWaves * kRun;  // steps of a block
constexpr int64_t kGroups = 512;     // workgroups that fill the GPU
constexpr int64_t kFewTiles = 160;   // below, workgroups share them

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

// What blocks of a prompt hand on where several workgroups share a tile: a word of 64 bits for
// each channel and block, [B, blocks, D], written once and whole, so that a word that is not
// empty is all there.  Block 0 and the last of every 16 leave the state after them (low half),
// which the next blocks start from; the others the state that they alone leave and the log2 of
// their decay, negated.
constexpr int kGroup = 16;
struct Links {
    uint64_t* words;
    uint32_t* tickets;  // [B, tiles]: blocks that are taken
};
constexpr uint64_t kEmpty = ~uint64_t(0);

__device__ __forceinline__ void post(uint64_t* p, float low, float high)
{
    const uint32_t h = __float_as_uint(high);
    // (a NaN of all ones would read as empty)
    const uint64_t w = uint64_t(h == ~0u ? 0x7fc00000u : h) << 32 | __float_as_uint(low);
    __hip_atomic_store(p, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t peek(const uint64_t* p)
{
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float low_of(uint64_t w) { return __uint_as_float(uint32_t(w)); }
__device__ __forceinline__ float high_of(uint64_t w) { return __uint_as_float(uint32_t(w >> 32)); }

__global__ __launch_bounds__(256) void links_kernel(Links links, int64_t words, int64_t tiles)
{
    const int64_t step = int64_t(gridDim.x) * 256;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < words; i += step) links.words[i] = kEmpty;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < tiles; i += step) links.tickets[i] = 0;
}

// The state before block k > 0: from the nearest block before it that leaves one, and those
// between, each by the decays after it, always in the same order.  Blocks are taken in their order
// and a workgroup finishes one before it begins the next that it has taken, so the first unfinished
// block of a tile is always at work and has none to wait for: every wait ends.  (Where another
// call writes the same workspace at the same time, which no call may, it ends all the same, after
// kPatience looks of half a microsecond or more, and the state is NaN.)
constexpr int kPatience = 1 << 18;
__device__ __forceinline__ float look_back(const uint64_t* words, int64_t k, int64_t D)
{
    constexpr int kLook = 4;  // words loaded together
    const int64_t from = k < kGroup ? 0 : k / kGroup * kGroup - 1;
    float h = 0.f, decay = 0.f;
    int looks = 0;
    for (int64_t j = k - 1; j >= from;) {
        uint64_t w[kLook];
#pragma unroll
        for (int i = 0; i < kLook; ++i) w[i] = peek(words + (j - i > from ? j - i : from) * D);
        const int64_t j0 = j;
        bool wait = false;
#pragma unroll
        for (int i = 0; i < kLook; ++i) {
            wait = wait || !__all(w[i] != kEmpty);
            if (!wait && j0 - i >= from) {
                h = fmaf(exp2_fast(-decay), low_of(w[i]), h);
                decay += high_of(w[i]);
                --j;
            }
        }
        if (wait) {
            if (++looks > kPatience) return __builtin_nanf("");
            __builtin_amdgcn_s_sleep(1);
        }
    }
    return h;
}

// CHAIN: the workgroups of a tile take its blocks in turn, else one takes them all.
template <typename T, bool GATE, bool CHAIN>
__global__ __launch_bounds__(kWaves* kWave, 8) void gated_kernel(GatedIn<T> in, float* state, int resume,
                                                                 T* __restrict__ y, float* __restrict__ marks,
                                                                 Links links)
{
    __shared__ float2 runs[2][kWaves][kWave];
    __shared__ float logs[2][kWaves][kWave];
    __shared__ float before[2][kWave];
    __shared__ uint32_t taken[2];
    const int lane = threadIdx.x % kWave;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const uint32_t unit = CHAIN ? blockIdx.x % uint32_t(in.B * in.tiles) : blockIdx.x;
    uint32_t k = 0;
    if constexpr (CHAIN) {
        if (threadIdx.x == 0) taken[0] = atomicAdd(links.tickets + unit, 1u);
        __syncthreads();
        k = __builtin_amdgcn_readfirstlane(taken[0]);
    }
    const Place at(in, unit, 1, 0);
    const int64_t c = at.c0 + at.lc;
    const GateParams par(in, c);
    const uint32_t blocks = at.te > 0 ? uint32_t((at.te + kSpan - 1) / kSpan) : 1;  // with tokens
    float h = resume ? state[at.b * in.D + c] : 0.f;  // before the block
    int turn = 0;
    for (; k < blocks; turn ^= 1) {
        const int64_t tb = int64_t(k) * kSpan;
        if (CHAIN && threadIdx.x == 0) taken[turn ^ 1] = atomicAdd(links.tickets + unit, 1u);
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
        // states and decays before this run, from zero
        float e = 0.f, le = 0.f;
        auto chain = [&](int j) {
            const float2 n = runs[turn][j][lane];
            e = fmaf(n.x, e, n.y);
            le += logs[turn][j][lane];
        };
        if (wave >= 8) {
#pragma unroll
            for (int j = 0; j < 8; ++j) chain(j);
        }
        if (wave & 4) {
#pragma unroll
            for (int j = 0; j < 4; ++j) chain((wave & 8) + j);
        }
        if (wave & 2) {
            chain(wave & 12);
            chain((wave & 12) + 1);
        }
        if (wave & 1) chain(wave & 14);
        // the last wavefront knows the whole block
        const float lend = le + L, hend = fmaf(exp2_fast(-L), e, H);
        const bool last = k == blocks - 1;
        if constexpr (CHAIN) {
            if (wave == kWaves - 1) {
                uint64_t* words = links.words + at.b * in.blocks * in.D + c;
                const bool leaves = k == 0 || k % kGroup == kGroup - 1;
                if (!last && !leaves) post(words + k * in.D, hend, lend);
                if (k > 0) h = look_back(words, k, in.D);
                const float after = carry_on(h, lend, hend);
                if (last)
                    state[at.b * in.D + c] = after;
                else if (leaves)
                    post(words + k * in.D, after, 0.f);
                before[turn][lane] = h;
            }
            __syncthreads();
            h = before[turn][lane];
        } else {
            if (k > 0) h = before[turn][lane];
        }
        float o = wave == 0 ? h : fmaf(exp2_fast(-le), h, e);
        if (marks && m > 0) marks[(at.b * in.marks + t / kRun) * in.D + c] = o;
        const Rows<T> by(y + (at.b * in.T_ + t) * in.D + at.c0, in.D, at.wide, m);
#pragma unroll
        for (int s = 0; s < kRun; ++s) {
            o = fmaf(a[s], o, v[s]);
            by.store(s, at.lc * uint32_t(sizeof(T)), x.out(s, o));
        }
        if (!CHAIN && wave == kWaves - 1) {
            h = carry_on(h, lend, hend);
            if (last) state[at.b * in.D + c] = h;
            before[turn ^ 1][lane] = h;
        }
        k = CHAIN ? __builtin_amdgcn_readfirstlane(taken[turn ^ 1]) : k + 1;
    }
    const int64_t share = CHAIN ? blockIdx.x / uint32_t(in.B * in.tiles) : 0;
    const int64_t shares = CHAIN ? gridDim.x / uint32_t(in.B * in.tiles) : 1;
    for (int64_t t = at.te + share * kWaves + wave; t < in.T_; t += shares * kWaves)
        io_store(y + (at.b * in.T_ + t) * in.D + c, 0.f);
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

// Workgroups that share a tile: one where there are tiles enough, or blocks too few.  Measured with
// one and with several (prompts of 2048, bfloat16 with gate): 64 tiles 63 and 28 us, 128 tiles 70
// and 53, 192 tiles 79 and 83, 256 tiles 87 and 96, 320 tiles 130 and 129, 512 tiles 158 and 175;
// of 16 tiles two blocks 11.1 and 13.4, three 14.6 and 13.2, eight 32 and 13.
int64_t gated_shares(int64_t tiles, int64_t blocks)
{
    if (tiles >= kFewTiles || blocks < 3) return 1;
    const int64_t n = (kGroups + tiles - 1) / tiles;
    return n < blocks ? n : blocks;
}

template <typename T, bool GATE>
hipError_t gated(const Gated& g, float* state, bool resume, T* y, float* marks, void* workspace,
                 hipStream_t stream)
{
    const GatedPlan p = gated_plan(g.B, g.T, g.D);
    const GatedIn<T> in = gated_in<T>(g, g.T > 0 ? g.T : 1, 1, p.blocks);
    const int64_t tiles = g.B * in.tiles;
    const dim3 block(kWaves * kWave);
    Links links{};
    if (p.shares == 1) {
        hipLaunchKernelGGL((gated_kernel<T, GATE, false>), dim3(uint32_t(tiles)), block, 0, stream, in, state,
                           int(resume), y, marks, links);
        return hipGetLastError();
    }
    const int64_t words = g.B * p.blocks * g.D, fills = (words + 1023) / 1024;
    links.words = static_cast<uint64_t*>(workspace);
    links.tickets = reinterpret_cast<uint32_t*>(links.words + words);
    hipLaunchKernelGGL(links_kernel, dim3(uint32_t(fills < 1024 ? fills : 1024)), dim3(256), 0, stream, links, words,
                       tiles);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL((gated_kernel<T, GATE, true>), dim3(uint32_t(tiles * p.shares)), block, 0, stream, in,
                       state, int(resume), y, marks, links);
    return hipGetLastError();
}

}  // namespace

GatedPlan gated_plan(int64_t B, int64_t T, int64_t D)
{
    GatedPlan p{T > 0 ? (T + kSpan - 1) / kSpan : 1, 1, 0};
    const int64_t tiles = gated_tiles(B, D);
    p.shares = gated_shares(tiles, p.blocks);
    if (p.shares > 1)
        p.ws_bytes = (sizeof(uint64_t) * size_t(B) * p.blocks * D + sizeof(uint32_t) * size_t(tiles) + 7) / 8 * 8;
    return p;
}

int64_t gated_threads(int64_t B, int64_t T, int64_t D)
{
    return gated_tiles(B, D) * gated_plan(B, T, D).shares * kWaves * kWave;
}

int64_t gated_step_threads(int64_t B, int64_t D) { return B * ((D + 255) / 256) * 256; }

hipError_t launch_gated(const Gated& g, float* state, bool resume, void* y, float* marks,
                        void* workspace, hipStream_t stream)
{
    if (g.bf16_io)
        return g.z ? gated<bf16, true>(g, state, resume, static_cast<bf16*>(y), marks, workspace, stream)
                   : gated<bf16, false>(g, state, resume, static_cast<bf16*>(y), marks, workspace, stream);
    return g.z ? gated<float, true>(g, state, resume, static_cast<float*>(y), marks, workspace, stream)
               : gated<float, false>(g, state, resume, static_cast<float*>(y), marks, workspace, stream);
}

hipError_t launch_gated_step(const Gated& g, float* state, void* y_t, hipStream_t stream)
{
    const dim3 grid(uint32_t(gated_step_threads(g.B, g.D) / 256));
    if (g.bf16_io)
        hipLaunchKernelGGL((gated_step_kernel<bf16>), grid, dim3(256), 0, stream, gated_in<bf16>(g, 1, 1, 1),
                           state, static_cast<bf16*>(y_t));
    else
        hipLaunchKernelGGL((gated_step_kernel<float>), grid, dim3(256), 0, stream, gated_in<float>(g, 1, 1, 1),
                           state, static_cast<float*>(y_t));
    return hipGetLastError();
}

}  // namespace lh
