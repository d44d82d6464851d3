// Gradients of the selective scan from a zero state.  With o_t = C_t . x_t + h0 u_t,
// y_t = o_t silu(z_t) and the gradient d_t of o_t (d_t = dy_t silu(z_t)):
//
//   G_t[n] = C_t[n] d_t + a_(t+1)[n] G_(t+1)[n],   a_t = e^(delta_t A)
//   dC_t[n] = sum_c d_t x_t[n]         dB_t[n] = sum_c G_t[n] delta_t u_t
//   p_t = sum_n G_t[n] B_t[n]          q_t = sum_n A[n] G_t[n] a_t[n] x_(t-1)[n]
//   du_t = delta_t p_t + h0 d_t        ddt_t = (q_t + u_t p_t) sigmoid(dt_t + dt_bias)
//   dA[n] = sum_t delta_t G_t[n] a_t[n] x_(t-1)[n]
//   dz_t = dy_t o_t silu'(z_t),  dh0 = sum d_t u_t,  ddt_bias = sum ddt_t
//
// Nothing of the forward pass is kept but its inputs.  The prompt is cut into chunks
// of 64 or 32 steps.  A first pass forms, per chunk and from the inputs alone, the end
// state from zero, the gradient that its own d hands to the state before it, and the
// sum of steps; a carry turns both into what enters each chunk, from the past and from
// the future.  The main pass walks a chunk forward once, keeping the state at the
// start of each block of 8 or 4 steps, then takes the blocks from the last to
// the first: forward again with the states and decays of the block in registers, then
// backward.  As in the prompt's scan a lane is a channel and the wavefronts of a
// workgroup share out the states; p, q and o are summed over them in LDS.
//
// dB and dC are sums over channels, across lanes: the 2 NS values of a step are
// folded by halves of the wave (each fold leaves two values in one register, half the
// lanes each), about two instructions a value instead of six adds, and leave as
// partial rows per tile; a last launch adds the tiles of a group in a fixed order.
//
// Steps past a row's tokens and slots without a state are left out of a block by its guarded
// form: the block that the tokens end in, and every block of a chunk that holds a value that is
// not finite while slots or lanes are empty.  Chunks without tokens only write zeros.
//
// Bound by the VALU: per state and step 7 instructions (one an exponential) in the first
// pass and 28 in the main one (two exponentials, 5 of them folds).  4 x 4096 x 2048
// bfloat16 with 16 states: 820 us (traced 200 the first pass, 29 the carry, 562 the main pass,
// 19 and 9 the sums; vector issue 0.77 of both passes at 2.4 GHz).  With each load of a chunk
// waited for in turn it took 1425 us.
#include "selective.hpp"

namespace lh {
namespace {

// Steps of a block and of a chunk: what the registers hold of them, fewer with 8 states
// to a lane (from 33 states on).
constexpr int block_steps(int ns) { return ns < 8 ? 8 : 4; }
constexpr int chunk_steps(int ns) { return ns < 8 ? 64 : 32; }

struct GradWork {
    float* xs;    // [B, nchunks, N, D] end states, then entry states
    float* gs;    // the same of gradients, from the future
    float* sums;  // [B, nchunks, D]
    float* rows;  // [tiles, B T, 2 N] partial dB, dC
    float* part;  // [B nchunks, D N + 2 D] partial dA, dh0, ddt_bias
};

// What a lane needs to know of its place.
struct Place {
    int64_t tile, k, b, grp, c0, c, t0, t1, te;
    int lane, wave, n0, real, width;  // width: the tile's channels
    int left;     // of the chunk's steps, those that are tokens of the row
    uint32_t lc;  // the lane's channel in the tile (past the group: the last)
    bool own;
};

template <int NS>
__device__ __forceinline__ Place place_of(const Selective& s, int64_t nchunks)
{
    Place p;
    p.lane = threadIdx.x & (kWave - 1);
    p.wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t Dg = s.D / s.G, per = group_tiles(s.D, s.G), tiles = per * s.G;
    p.tile = blockIdx.x % tiles;
    const int64_t rest = blockIdx.x / tiles;
    p.k = rest % nchunks;
    p.b = rest / nchunks;
    p.grp = p.tile / per;
    p.c0 = p.grp * Dg + (p.tile % per) * kWave;
    p.width = int((p.grp + 1) * Dg - p.c0 < kWave ? (p.grp + 1) * Dg - p.c0 : kWave);
    p.own = p.lane < p.width;
    p.lc = p.own ? p.lane : p.width - 1;
    p.c = p.c0 + p.lc;
    p.n0 = p.wave * NS;
    p.real = s.N - p.n0 < NS ? s.N - p.n0 : NS;
    const int64_t len = tokens_of(s.lengths, p.b, s.T);
    constexpr int chunk = chunk_steps(NS);
    p.t0 = p.k * chunk;
    p.t1 = p.t0 + chunk < s.T ? p.t0 + chunk : s.T;
    p.te = p.t1 < len ? p.t1 : len;
    p.left = p.te > p.t0 ? int(p.te - p.t0) : 0;
    return p;
}

// A chunk's rows in LDS: steps, their inputs, d, and B, C by state.
template <int S, int NS>
struct Chunk {
    static constexpr int kChunk = chunk_steps(NS);
    float delta[kChunk][kWave], du[kChunk][kWave], d[kChunk][kWave];
    float B[kChunk][S * NS], C[kChunk][S * NS];
};

// Every load of a chunk starts before the first is used (rows past the last token are its
// copies, and become zeros in LDS).  The chunk has a token.
template <typename T, int NS, int S, bool GATE>
__device__ __forceinline__ void load_chunk(const Selective& s, const SelectiveGrads& g,
                                           const Place& p, Chunk<S, NS>& m)
{
    constexpr int kChunk = chunk_steps(NS), R = kChunk / S;
    constexpr int PER = (kChunk * NS + kWave - 1) / kWave;  // elements of B (of C) per thread
    const int left = p.left, last = left - 1;
    const int64_t row0 = p.b * s.T + p.t0;
    const uint32_t off = p.lc * sizeof(T);
    const T* pu = static_cast<const T*>(s.u) + row0 * s.ld_u + p.c0;
    const T* pdt = static_cast<const T*>(s.dt) + row0 * s.ld_dt + p.c0;
    const T* pz = GATE ? static_cast<const T*>(s.z) + row0 * s.ld_z + p.c0 : nullptr;
    const T* pg = static_cast<const T*>(g.dy) + row0 * s.D + p.c0;
    const T* pB = static_cast<const T*>(s.Bm) + row0 * s.ld_b + p.grp * s.N;
    const T* pC = static_cast<const T*>(s.Cm) + row0 * s.ld_c + p.grp * s.N;
    const float bias = s.dt_bias ? s.dt_bias[p.c] : 0.f;
    T ru[R], rd[R], rz[R], rg[R], rB[PER], rC[PER];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int64_t j = p.wave + i * S < last ? p.wave + i * S : last;
        ru[i] = at_byte(pu + j * s.ld_u, off);
        rd[i] = at_byte(pdt + j * s.ld_dt, off);
        rg[i] = at_byte(pg + j * s.D, off);
        if constexpr (GATE) rz[i] = at_byte(pz + j * s.ld_z, off);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = threadIdx.x + i * kWave * S;
        const int64_t j = e / (S * NS) < last ? e / (S * NS) : last;
        const int n = e % (S * NS) < s.N ? e % (S * NS) : s.N - 1;
        rB[i] = pB[j * s.ld_b + n];
        rC[i] = pC[j * s.ld_c + n];
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int j = p.wave + i * S;
        float delta = softplus(io_load(&rd[i]) + bias);
        float du = delta * io_load(&ru[i]), d = io_load(&rg[i]);
        if constexpr (GATE) {
            const float z = io_load(&rz[i]);
            d *= z * sigmoid(z);
        }
        if (j >= left) delta = du = d = 0.f;
        // (lanes past the group add nothing to the sums over channels)
        if (!p.own) du = d = 0.f;
        m.delta[j][p.lane] = delta;
        m.du[j][p.lane] = du;
        m.d[j][p.lane] = d;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = threadIdx.x + i * kWave * S, j = e / (S * NS), n = e % (S * NS);
        if (e < kChunk * S * NS) {
            const bool in = j < left && n < s.N;
            m.B[j][n] = in ? io_load(&rB[i]) : 0.f;
            m.C[j][n] = in ? io_load(&rC[i]) : 0.f;
        }
    }
    __syncthreads();
}

// Whether this thread's share of a chunk is finite (false, too, where its sum overflows).
template <int S, int NS>
__device__ __forceinline__ bool finite_share(const Chunk<S, NS>& m)
{
    constexpr int kSteps = Chunk<S, NS>::kChunk;
    float sum = 0.f;
    for (int e = threadIdx.x; e < kSteps * kWave; e += kWave * S)
        sum += fabsf((&m.delta[0][0])[e]) + (fabsf((&m.du[0][0])[e]) + fabsf((&m.d[0][0])[e]));
    for (int e = threadIdx.x; e < kSteps * S * NS; e += kWave * S)
        sum += fabsf((&m.B[0][0])[e]) + fabsf((&m.C[0][0])[e]);
    return sum < INFINITY;
}

template <typename T, int NS, int S, bool GATE>
__global__ __launch_bounds__(kWave* S) void grad_ends_kernel(Selective s, SelectiveGrads g,
                                                             GradWork w, int64_t nchunks)
{
    __shared__ Chunk<S, NS> m;
    const Place p = place_of<NS>(s, nchunks);
    if (p.left > 0) load_chunk<T, NS, S, GATE>(s, g, p, m);
    float A2[NS], x[NS], dec[NS], r[NS], total = 0.f;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        A2[i] = s.A[p.c * s.N + (i < p.real ? p.n0 + i : s.N - 1)];
        x[i] = r[i] = 0.f;
        dec[i] = 1.f;
    }
#pragma unroll
    for (int i = 0; i < NS; ++i) A2[i] = i < p.real ? A2[i] * kLog2e : 0.f;
    // (steps past the row's tokens are not walked: zero times an infinite state or pole is
    // not zero)
    auto walk = [&](auto steps) {
#pragma unroll 4
        for (int j = 0; j < steps; ++j) {
            const float delta = m.delta[j][p.lane], du = m.du[j][p.lane], d = m.d[j][p.lane];
            total += delta;
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                const float a = exp2_fast(delta * A2[i]);
                x[i] = fmaf(a, x[i], du * m.B[j][p.n0 + i]);
                dec[i] *= a;  // decay from the chunk's start through step j
                r[i] = fmaf(dec[i] * m.C[j][p.n0 + i], d, r[i]);
            }
        }
    };
    constexpr int kChunk = chunk_steps(NS);
    if (p.left == kChunk)
        walk(std::integral_constant<int, kChunk>());
    else
        walk(p.left);
    if (!p.own) return;
#pragma unroll
    for (int i = 0; i < NS; ++i)
        if (i < p.real) {
            const int64_t at = ((p.b * nchunks + p.k) * s.N + p.n0 + i) * s.D + p.c;
            w.xs[at] = x[i];
            w.gs[at] = r[i];
        }
    if (p.wave == 0) w.sums[(p.b * nchunks + p.k) * s.D + p.c] = total;
}

// End states to entry states, forward; gradients handed back to those that enter from
// the future, backward.
__global__ __launch_bounds__(256) void grad_carry_kernel(const float* __restrict__ A, GradWork w,
                                                         int64_t B, int64_t D, int N,
                                                         int64_t nchunks)
{
    int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x;
    const int64_t rows = B * D * N;
    if (id >= 2 * rows) return;
    const bool back = id >= rows;  // (whole wavefronts but for one)
    id -= back ? rows : 0;
    const int64_t c = id % D, n = id / D % N, b = id / (D * N);
    const float A2 = A[c * N + n] * kLog2e;
    const int64_t step = back ? -1 : 1, first = back ? nchunks - 1 : 0;
    float* px = (back ? w.gs : w.xs) + ((b * nchunks + first) * N + n) * D + c;
    const float* ps = w.sums + (b * nchunks + first) * D + c;
    const int64_t sx = step * N * D, ss = step * D;
    float x = 0.f;
    constexpr int U = 8;
    for (int64_t k = 0; k < nchunks; k += U) {
        float end[U], sum[U];
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (k + i < nchunks) {
                end[i] = px[(k + i) * sx];
                sum[i] = ps[(k + i) * ss];
            }
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (k + i < nchunks) {
                px[(k + i) * sx] = x;
                x = fmaf(chunk_decay(A2, sum[i]), x, end[i]);
            }
    }
}

// One fold of a sum across lanes: lanes whose bit BIT is 0 keep a's sum over the pair
// of lanes, the others b's.
template <int BIT>
__device__ __forceinline__ float fold(float a, float b, int lane)
{
    if constexpr (BIT == 32 || BIT == 16) {
        typedef unsigned u2 __attribute__((ext_vector_type(2)));
        u2 r;
        if constexpr (BIT == 32)
            r = __builtin_bit_cast(u2, __builtin_amdgcn_permlane32_swap(__float_as_uint(a),
                                                                       __float_as_uint(b), false, false));
        else
            r = __builtin_bit_cast(u2, __builtin_amdgcn_permlane16_swap(__float_as_uint(a),
                                                                       __float_as_uint(b), false, false));
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    } else {
        // (bound_ctrl lets the compiler take the permuted operand into the addition)
        const bool hi = lane & BIT;
        const float keep = hi ? b : a, send = hi ? a : b;
        const int v = __builtin_bit_cast(int, send);
        int q;
        if constexpr (BIT == 8)
            q = __builtin_amdgcn_mov_dpp(v, 0x128, 0xF, 0xF, true);  // row_ror:8
        else if constexpr (BIT == 4)
            // lane ^ 7 within 8: the lower bits' folds come after and sum over them anyway
            q = __builtin_amdgcn_mov_dpp(v, 0x141, 0xF, 0xF, true);
        else if constexpr (BIT == 2)
            q = __builtin_amdgcn_mov_dpp(v, 0x4E, 0xF, 0xF, true);  // quad_perm [2,3,0,1]
        else
            q = __builtin_amdgcn_mov_dpp(v, 0xB1, 0xF, 0xF, true);  // quad_perm [1,0,3,2]
        return keep + __builtin_bit_cast(float, q);
    }
}

// Folds n values from lane bit BIT on: value i ends in the lanes whose bits BIT,
// BIT / 2, .. spell i from its lowest bit; the lanes' sums are over those bits only.
template <int N, int BIT>
__device__ __forceinline__ float fold_all(const float (&v)[N], int lane)
{
    if constexpr (N == 1) {
        return v[0];
    } else {
        float h[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) h[i] = fold<BIT>(v[2 * i], v[2 * i + 1], lane);
        return fold_all<N / 2, BIT / 2>(h, lane);
    }
}
// Sums over the lane bits BIT, BIT / 2, .. 1.
template <int BIT>
__device__ __forceinline__ float sum_below(float v, int lane)
{
    if constexpr (BIT >= 1) {
        v = fold<BIT>(v, v, lane);
        return sum_below<BIT / 2>(v, lane);
    } else {
        return v;
    }
}

template <typename T, int NS, int S, bool GATE>
__global__ __launch_bounds__(kWave* S) void grad_kernel(Selective s, SelectiveGrads g, GradWork w,
                                                        int64_t nchunks)
{
    constexpr int kBlockSteps = block_steps(NS);
    __shared__ Chunk<S, NS> m;
    __shared__ float po[GATE ? S : 1][kBlockSteps][kWave], pp[S][kBlockSteps][kWave], pq[S][kBlockSteps][kWave];
    const Place p = place_of<NS>(s, nchunks);
    constexpr int kBlocks = chunk_steps(NS) / kBlockSteps;
    const uint32_t off = p.lc * sizeof(T);
    // gradients past the row's tokens are zero (of B and C: grad_rows_kernel)
    if (p.own)
        for (int64_t t = (p.te > p.t0 ? p.te : p.t0) + p.wave; t < p.t1; t += S) {
            const int64_t row = (p.b * s.T + t) * s.D + p.c0;
            io_store(&at_byte(static_cast<T*>(g.ddt) + row, off), 0.f);
            io_store(&at_byte(static_cast<T*>(g.du) + row, off), 0.f);
            if constexpr (GATE) io_store(&at_byte(static_cast<T*>(g.dz) + row, off), 0.f);
        }
    float* part = w.part + (p.b * nchunks + p.k) * (s.D * s.N + 2 * s.D);
    if (p.left == 0) {
        if (!p.own) return;
        for (int i = 0; i < p.real; ++i) part[p.c * s.N + p.n0 + i] = 0.f;
        if (p.wave == 0) part[s.D * s.N + p.c] = part[s.D * s.N + s.D + p.c] = 0.f;
        return;
    }
    load_chunk<T, NS, S, GATE>(s, g, p, m);
    // Slots past N, steps past the row's tokens and lanes past the group hold zeros and add zeros
    // to the sums, unless an input, or the state that the tokens leave, is not finite: zero times
    // infinity is not zero.  The guarded form of a block leaves them out.  A whole workgroup takes
    // the same form, since both hold barriers.
    bool guarded = false;
    if (s.N < NS * S || p.width < kWave) {
        if (p.lane == 0) pp[p.wave][0][0] = 0.f;
        if (!finite_share(m)) pp[p.wave][0][0] = 1.f;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < S; ++k) guarded |= pp[k][0][0] != 0.f;
        __syncthreads();
    }

    float A2[NS], x[NS], G[NS], dA[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        // (slots past N load the last state and become zeros, so that no load waits alone)
        const int n = i < p.real ? p.n0 + i : s.N - 1;
        A2[i] = s.A[p.c * s.N + n];
        const int64_t at = ((p.b * nchunks + p.k) * s.N + n) * s.D + p.c;
        x[i] = w.xs[at];
        G[i] = w.gs[at];
        dA[i] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        A2[i] = i < p.real ? A2[i] * kLog2e : 0.f;
        x[i] = i < p.real && p.own ? x[i] : 0.f;
        G[i] = i < p.real && p.own ? G[i] : 0.f;
    }
    const float bias = s.dt_bias ? s.dt_bias[p.c] : 0.f, h0 = s.h0 ? s.h0[p.c] : 0.f;
    float dh0 = 0.f, dbias = 0.f;
    const int64_t row0 = p.b * s.T + p.t0, last = p.left - 1;
    // the state at the start of every block
    float start[kBlocks][NS];
#pragma unroll
    for (int q = 0; q < kBlocks; ++q) {
#pragma unroll
        for (int i = 0; i < NS; ++i) start[q][i] = x[i];
        if (q < kBlocks - 1) {
#pragma unroll 4
            for (int j = q * kBlockSteps; j < (q + 1) * kBlockSteps; ++j) {
                const float delta = m.delta[j][p.lane], du = m.du[j][p.lane];
#pragma unroll
                for (int i = 0; i < NS; ++i)
                    x[i] = fmaf(exp2_fast(delta * A2[i]), x[i], du * m.B[j][p.n0 + i]);
            }
        }
    }

    // Blocks from - 1 down to `to`.
    auto walk = [&](auto plain, int from, int to) {
        constexpr bool PLAIN = decltype(plain)::value;
#pragma unroll 1
        for (int q = from - 1; q >= to; --q) {
            // registers are indexed by constants: the block's start is picked by comparison
#pragma unroll
            for (int z = 0; z < kBlocks; ++z)
                if (z == q)
#pragma unroll
                    for (int i = 0; i < NS; ++i) x[i] = start[z][i];
            float before[kBlockSteps][NS], a[kBlockSteps][NS];
            const int j0 = q * kBlockSteps;
            // what this wavefront's rows of the block need beside the sums, loaded ahead
            constexpr int kRows = (kBlockSteps + S - 1) / S;
            T ru[kRows], rd[kRows], rz[kRows], rg[kRows];
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const int64_t j = j0 + p.wave + i * S < last ? j0 + p.wave + i * S : last;
                ru[i] = at_byte(static_cast<const T*>(s.u) + (row0 + j) * s.ld_u + p.c0, off);
                rd[i] = at_byte(static_cast<const T*>(s.dt) + (row0 + j) * s.ld_dt + p.c0, off);
                if constexpr (GATE) {
                    rz[i] = at_byte(static_cast<const T*>(s.z) + (row0 + j) * s.ld_z + p.c0, off);
                    rg[i] = at_byte(static_cast<const T*>(g.dy) + (row0 + j) * s.D + p.c0, off);
                }
            }
#pragma unroll
            for (int j = 0; j < kBlockSteps; ++j) {
                const float delta = m.delta[j0 + j][p.lane], du = m.du[j0 + j][p.lane];
                float o = 0.f;
                if (!PLAIN && j0 + j > last) {
#pragma unroll
                    for (int i = 0; i < NS; ++i) a[j][i] = 1.f, before[j][i] = x[i];
                    continue;
                }
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    a[j][i] = exp2_fast(delta * A2[i]);
                    before[j][i] = x[i];
                    x[i] = fmaf(a[j][i], x[i], du * m.B[j0 + j][p.n0 + i]);
                    if (PLAIN || i < p.real) o = fmaf(m.C[j0 + j][p.n0 + i], x[i], o);
                }
                if constexpr (GATE) po[p.wave][j][p.lane] = o;
            }
            float folded[kBlockSteps];
            constexpr int kTop = 64 / (2 * NS);  // lane bits below kTop are left after a step's folds
#pragma unroll
            for (int j = kBlockSteps - 1; j >= 0; --j) {
                if (!PLAIN && j0 + j > last) {
                    folded[j] = 0.f;
                    continue;
                }
                const float delta = m.delta[j0 + j][p.lane], du = m.du[j0 + j][p.lane],
                            d = m.d[j0 + j][p.lane];
                float pv = 0.f, qv = 0.f, v[2 * NS];
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    G[i] = fmaf(m.C[j0 + j][p.n0 + i], d, G[i]);
                    const float after = j < kBlockSteps - 1 ? before[j < kBlockSteps - 1 ? j + 1 : 0][i] : x[i];
                    v[i] = PLAIN || p.own ? G[i] * du : 0.f;
                    v[NS + i] = PLAIN || p.own ? d * after : 0.f;
                    const float ag = a[j][i] * G[i], h = ag * before[j][i];
                    if (PLAIN || i < p.real) {
                        pv = fmaf(G[i], m.B[j0 + j][p.n0 + i], pv);
                        qv = fmaf(A2[i], h, qv);
                    }
                    dA[i] = fmaf(delta, h, dA[i]);
                    G[i] = ag;
                }
                pp[p.wave][j][p.lane] = pv;
                pq[p.wave][j][p.lane] = qv;
                folded[j] = fold_all<2 * NS, 32>(v, p.lane);
            }
            // fold the block's steps into the lane bits that are left
            constexpr int kHalf = kTop / 2 ? kTop / 2 : 1;
            if constexpr (kTop == kBlockSteps) {  // every lane ends with one sum
                const float r = fold_all<kBlockSteps, kHalf>(folded, p.lane);
                // lane bits from the top: log2(2 NS) of the value, 3 of the step, each lowest first
                int v = 0, j = 0;
#pragma unroll
                for (int bit = 0; (1 << bit) < 2 * NS; ++bit) v |= ((p.lane >> (5 - bit)) & 1) << bit;
#pragma unroll
                for (int bit = 0; (1 << bit) < kBlockSteps; ++bit)
                    j |= ((p.lane >> (5 - (6 - __builtin_ctz(kBlockSteps)) - bit)) & 1) << bit;
                const int i = v % NS, which = v / NS;
                if (i < p.real && j0 + j <= last)
                    w.rows[((p.tile * s.B * s.T) + row0 + j0 + j) * 2 * s.N + which * s.N + p.n0 + i] = r;
            } else {
#pragma unroll
                for (int j = 0; j < kBlockSteps; ++j) {
                    const float r = sum_below<kTop / 2>(folded[j], p.lane);
                    int v = 0;
#pragma unroll
                    for (int bit = 0; (1 << bit) < 2 * NS; ++bit) v |= ((p.lane >> (5 - bit)) & 1) << bit;
                    const int i = v % NS, which = v / NS;
                    if (p.lane % kTop == 0 && i < p.real && j0 + j <= last)
                        w.rows[((p.tile * s.B * s.T) + row0 + j0 + j) * 2 * s.N + which * s.N + p.n0 + i] = r;
                }
            }
            __syncthreads();
            // the channels' gradients of the block's steps, shared out among the wavefronts
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const int j = p.wave + i * S;
                if (j >= kBlockSteps || j0 + j > last || !p.own) continue;
                const int64_t row = (row0 + j0 + j) * s.D + p.c0;
                T& ddt_at = at_byte(static_cast<T*>(g.ddt) + row, off);
                T& du_at = at_byte(static_cast<T*>(g.du) + row, off);
                T& dz_at = GATE ? at_byte(static_cast<T*>(g.dz) + row, off) : du_at;
                float pv = 0.f, qv = 0.f;
#pragma unroll
                for (int k = 0; k < S; ++k) {
                    pv += pp[k][j][p.lane];
                    qv += pq[k][j][p.lane];
                }
                qv *= kLn2;  // (A is held times log2 e alone)
                const float u = io_load(&ru[i]), d = m.d[j0 + j][p.lane];
                const float ddt = fmaf(u, pv, qv) * sigmoid(io_load(&rd[i]) + bias);
                io_store(&ddt_at, ddt);
                io_store(&du_at, fmaf(m.delta[j0 + j][p.lane], pv, h0 * d));
                dbias += ddt;
                dh0 = fmaf(d, u, dh0);
                if constexpr (GATE) {
                    float o = h0 * u;
#pragma unroll
                    for (int k = 0; k < S; ++k) o += po[k][j][p.lane];
                    const float z = io_load(&rz[i]), sg = sigmoid(z);
                    io_store(&dz_at, io_load(&rg[i]) * o * (sg * fmaf(z, 1.f - sg, 1.f)));
                }
            }
            __syncthreads();
        }
    };
    // the guarded form for all blocks, or for the one that the tokens end in
    const int blocks = (p.left + kBlockSteps - 1) / kBlockSteps;
    const int guard = __builtin_amdgcn_readfirstlane(guarded) ? 0 : p.left / kBlockSteps;
    walk(std::false_type(), blocks, guard);
    walk(std::true_type(), guard, 0);
    // partial rows of the weights' gradients
    pp[p.wave][0][p.lane] = dh0;
    pp[p.wave][1][p.lane] = dbias;
    __syncthreads();
    if (!p.own) return;
#pragma unroll
    for (int i = 0; i < NS; ++i)
        if (i < p.real) part[p.c * s.N + p.n0 + i] = dA[i];
    if (p.wave == 0) {
        float h = 0.f, bsum = 0.f;
#pragma unroll
        for (int k = 0; k < S; ++k) {
            h += pp[k][0][p.lane];
            bsum += pp[k][1][p.lane];
        }
        part[s.D * s.N + p.c] = h;
        part[s.D * s.N + s.D + p.c] = bsum;
    }
}

// dB and dC: the tiles of each group added; zero past the row's tokens (where no partial
// rows are written).
template <typename T>
__global__ __launch_bounds__(256) void grad_rows_kernel(Selective s, const float* __restrict__ rows,
                                                        T* __restrict__ dB, T* __restrict__ dC)
{
    const int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x;
    const int N2 = 2 * s.N;
    const int64_t row = id / N2 / s.G;  // token
    if (row >= s.B * s.T) return;
    const int64_t grp = id / N2 % s.G;
    const int v = int(id % N2);
    const int64_t per = group_tiles(s.D, s.G), stride = s.B * s.T * N2;
    const float* p = rows + grp * per * stride + row * N2 + v;
    const bool token = !s.lengths || row % s.T < tokens_of(s.lengths, row / s.T, s.T);
    float acc = 0.f;
    for (int64_t i = 0; i < (token ? per : 0); ++i) acc += p[i * stride];
    const int64_t at = (row * s.G + grp) * s.N;
    if (v < s.N)
        io_store(dB + at + v, acc);
    else
        io_store(dC + at + v - s.N, acc);
}

// States per lane (a power of two) and wavefronts per tile.
void split_grad(int N, int* ns, int* waves)
{
    *ns = N <= 4 ? 1 : N <= 8 ? 2 : N <= 32 ? 4 : 8;
    *waves = N <= 16 ? 4 : N <= 64 ? 8 : 16;
}

template <typename F>
hipError_t with_grad_split(int ns, int waves, F f)
{
#define LH_SPLIT(n, w) \
    if (ns == n && waves == w) \
    return f(std::integral_constant<int, n>(), std::integral_constant<int, w>())
    LH_SPLIT(1, 4);
    LH_SPLIT(2, 4);
    LH_SPLIT(4, 4);
    LH_SPLIT(4, 8);
    LH_SPLIT(8, 8);
    LH_SPLIT(8, 16);
#undef LH_SPLIT
    return hipErrorInvalidValue;
}

size_t aligned(size_t n) { return (n + 255) / 256 * 256; }

int64_t grad_chunks(int64_t T, int N)
{
    int ns = 0, waves = 0;
    split_grad(N, &ns, &waves);
    return (T + chunk_steps(ns) - 1) / chunk_steps(ns);
}

// Regions of the workspace, in the order of GradWork; returns its size.
size_t grad_work(int64_t B, int64_t T, int64_t D, int N, int G, char* base, GradWork* w)
{
    const int64_t n = grad_chunks(T, N), tiles = group_tiles(D, G) * G;
    const size_t states = aligned(sizeof(float) * size_t(B) * n * N * D);
    const size_t sums = aligned(sizeof(float) * size_t(B) * n * D);
    const size_t rows = aligned(sizeof(float) * size_t(tiles) * B * T * 2 * N);
    const size_t part = aligned(sizeof(float) * size_t(B) * n * (size_t(D) * N + 2 * D));
    if (w) {
        w->xs = reinterpret_cast<float*>(base);
        w->gs = reinterpret_cast<float*>(base + states);
        w->sums = reinterpret_cast<float*>(base + 2 * states);
        w->rows = reinterpret_cast<float*>(base + 2 * states + sums);
        w->part = reinterpret_cast<float*>(base + 2 * states + sums + rows);
    }
    return 2 * states + sums + rows + part;
}

template <typename T>
hipError_t scan_grad(const Selective& s, const SelectiveGrads& g, void* workspace,
                     hipStream_t stream)
{
    GradWork w;
    grad_work(s.B, s.T, s.D, s.N, s.G, static_cast<char*>(workspace), &w);
    const int64_t n = grad_chunks(s.T, s.N), tiles = group_tiles(s.D, s.G) * s.G;
    hipError_t e;
    if (n > 0) {
        int ns = 0, waves = 0;
        split_grad(s.N, &ns, &waves);
        const dim3 grid(uint32_t(s.B * n * tiles));
        e = with_grad_split(ns, waves, [&](auto a, auto b) {
            constexpr int NS = decltype(a)::value, S = decltype(b)::value;
            const auto ends = s.z ? grad_ends_kernel<T, NS, S, true> : grad_ends_kernel<T, NS, S, false>;
            const auto main = s.z ? grad_kernel<T, NS, S, true> : grad_kernel<T, NS, S, false>;
            hipLaunchKernelGGL(ends, grid, dim3(kWave * S), 0, stream, s, g, w, n);
            hipError_t r = hipGetLastError();
            if (r != hipSuccess) return r;
            hipLaunchKernelGGL(grad_carry_kernel, dim3(uint32_t((2 * s.B * s.D * s.N + 255) / 256)),
                               dim3(256), 0, stream, s.A, w, s.B, s.D, s.N, n);
            if ((r = hipGetLastError()) != hipSuccess) return r;
            hipLaunchKernelGGL(main, grid, dim3(kWave * S), 0, stream, s, g, w, n);
            return hipGetLastError();
        });
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((grad_rows_kernel<T>),
                           dim3(uint32_t((s.B * s.T * s.G * 2 * s.N + 255) / 256)), dim3(256), 0,
                           stream, s, w.rows, static_cast<T*>(g.dBm), static_cast<T*>(g.dCm));
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    return launch_column_sum(w.part, s.B * n, s.D * s.N, g.dA, s.D, g.dh0, s.D, g.ddt_bias, stream);
}

}  // namespace

size_t selective_grad_workspace_bytes(int64_t B, int64_t T, int64_t D, int N, int G)
{
    return grad_work(B, T, D, N, G, nullptr, nullptr);
}

int64_t selective_grad_threads(int64_t B, int64_t T, int64_t D, int N, int G)
{
    int ns = 0, waves = 0;
    split_grad(N, &ns, &waves);
    int64_t most = 32 * D * (int64_t(N) + 2);  // column sums
    auto at_least = [&](int64_t n) { most = n > most ? n : most; };
    at_least(B * grad_chunks(T, N) * group_tiles(D, G) * G * kWave * waves);
    at_least(2 * B * D * N);      // carry
    at_least(B * T * G * 2 * N);  // rows of B and C
    return most + 1024;           // (the last workgroup)
}

hipError_t launch_selective_grad(const Selective& s, const SelectiveGrads& g, void* workspace,
                                 hipStream_t stream)
{
    return s.bf16_io ? scan_grad<bf16>(s, g, workspace, stream)
                     : scan_grad<float>(s, g, workspace, stream);
}

}  // namespace lh
