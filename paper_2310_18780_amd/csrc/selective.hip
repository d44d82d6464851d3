// The selective state-space scan, for prompts and for single tokens:
//
//   delta = softplus(dt + dt_bias)
//   x_t[n] = e^(delta A[n]) x_(t-1)[n] + delta B_t[n] u_t
//   y_t = sum_n C_t[n] x_t[n] + h0 u_t,  times silu(z_t) where there is a gate
//
// per batch row and channel, B and C shared by the channels of a group.
//
// Prompts.  A lane is a channel, so u, dt, z and y are read and written in whole
// lines, once.  The states of a 64-channel tile are split over the wavefronts of a
// workgroup, a few to a lane in registers; a tile of 16 steps passes through LDS: its
// wavefronts form the steps (delta, delta u) of some rows each, walk all 16 rows for
// their own states, and add the wavefronts' parts of y for some rows each.  The loads of
// the next tile are in flight while one is walked.
//
// Bound by the VALU: per state and step two products, two multiply-adds (4 cycles each)
// and an exponential (8 cycles), beside about 38 instructions a channel and step for
// softplus, silu, the sum of the parts and conversions.  16 x 4096 x 2048 bfloat16 with 16
// states: 565 us (1.9 TB/s; vector issue 0.84 of the time at 2.4 GHz; the clock is lower in
// the first 25 ms of load, up to 760 us).  What brought it there from 2047 us: loads not converted
// where they are issued (784), 32-bit byte offsets from a uniform row and no branch for
// the row's end inside a tile (629), twice the wavefronts with half the states (570).
// Taken back: two tiles' buffers and one barrier a tile (LDS leaves fewer workgroups,
// 1.4 times the time), values read from LDS a group of steps ahead (1.1 times), the rank-1
// update as a 4x4x1 matrix instruction (its moves cost more than the products it saves).
//
// Where batch rows and tiles leave SIMDs idle the prompt is cut into chunks: a first
// pass forms each chunk's end state from zero and its sum of steps (a chunk's decay is
// e^(A sum delta), one exponential), a carry turns end states into entry states, and
// the output pass starts every chunk from its own: 0.83 times the output pass's work
// again, for all SIMDs (1 x 65536 x 1024 float32: 477 us, the passes 195 and 262).
//
// Single tokens: four states of a (batch row, channel) to a lane, y summed over the
// row's lanes; bound by the state, read once and written once (64 x 2048, 16 states, 18
// MB: 5.5 us in a graph, and 9 us a call from the host).
#include "selective.hpp"

namespace lh {
namespace {

constexpr int kSteps = 16;  // steps of a tile
// Up to this many chunks a launch for the carry costs more than carrying in every chunk
// (1 row of 512 steps, D = 768: 18.9 us against 21.1; of 2048 steps, 64 chunks, 69.7
// against 52.5; between 16 and 64 chunks it was not measured).
constexpr int64_t kFewChunks = 16;

// f with n as a constant, 0 <= n <= MOST (n < 0 is 0).
template <int MOST, typename F>
__device__ __forceinline__ void with_count(int n, const F& f)
{
    if constexpr (MOST <= 0) {
        f(std::integral_constant<int, 0>());
    } else {
        if (n == MOST)
            f(std::integral_constant<int, MOST>());
        else
            with_count<MOST - 1>(n, f);
    }
}

template <typename T, int NS, int S, bool OUT, bool GATE>
__global__ __launch_bounds__(kWave* S) void scan_kernel(Selective s, int64_t chunk,
                                                        int64_t nchunks, bool carried,
                                                        float* xs, float* sums, float* state,
                                                        bool resume, T* y)
{
    constexpr int R = kSteps / S;    // rows per wavefront
    constexpr int W = OUT ? 2 : 1;   // B (and C)
    constexpr int E = kSteps * S * W * NS;
    constexpr int PER = (E + kWave * S - 1) / (kWave * S);
    __shared__ float2 step[kSteps][kWave];                  // delta, delta u
    __shared__ __align__(16) float rows[kSteps][S][W][NS];  // B, C
    __shared__ float part[OUT ? S : 1][kSteps][kWave];      // the wavefronts' parts of y

    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int N = s.N;
    const int64_t Dg = s.D / s.G, per = group_tiles(s.D, s.G), tiles = per * s.G;
    const int64_t tile = blockIdx.x % tiles, rest = blockIdx.x / tiles;
    // (nobody needs the last chunk's end state from zero)
    const int64_t chunks = OUT ? nchunks : nchunks - 1, k = rest % chunks, b = rest / chunks;
    const int64_t grp = tile / per, c0 = grp * Dg + (tile % per) * kWave;  // the tile's first channel
    const int width = int((grp + 1) * Dg - c0 < kWave ? (grp + 1) * Dg - c0 : kWave);
    // Lanes past the group compute its last channel and store the same bits as its own
    // lane, so that no store is under a mask.
    const bool own = lane < width;
    const uint32_t lc = own ? lane : width - 1;
    const int n0 = wave * NS, real = N - n0 < NS ? N - n0 : NS;

    const int64_t len = tokens_of(s.lengths, b, s.T);
    const int64_t t_begin = k * chunk, t_end = t_begin + chunk < s.T ? t_begin + chunk : s.T;
    const int64_t te = t_end < len ? t_end : len;

    // row 0 of this batch row and tile, the same in every lane
    const T* pu = static_cast<const T*>(s.u) + b * s.T * s.ld_u + c0;
    const T* pdt = static_cast<const T*>(s.dt) + b * s.T * s.ld_dt + c0;
    const T* pz = GATE ? static_cast<const T*>(s.z) + b * s.T * s.ld_z + c0 : nullptr;
    const T* pB = static_cast<const T*>(s.Bm) + b * s.T * s.ld_b + grp * N;
    const T* pC = static_cast<const T*>(s.Cm) + b * s.T * s.ld_c + grp * N;
    T* py = y + b * s.T * s.D + c0;
    const int64_t c = c0 + lc;
    const float bias = s.dt_bias ? s.dt_bias[c] : 0.f;
    const float h0 = OUT && s.h0 ? s.h0[c] : 0.f;

    // (slots past N load the last state and become zeros, so that no load waits alone)
    float A2[NS], x[NS];
    const int64_t lastn = N - 1;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        A2[i] = s.A[c * N + (n0 + i < N ? n0 + i : lastn)];
        x[i] = 0.f;
    }
    if (OUT && (nchunks > 1 ? carried : resume)) {
        const float* from = nchunks > 1 ? xs + (b * nchunks + k) * N * s.D + c : state + (b * s.D + c) * N;
        const int64_t stride = nchunks > 1 ? s.D : 1;
#pragma unroll
        for (int i = 0; i < NS; ++i) x[i] = from[(n0 + i < N ? n0 + i : lastn) * stride];
    }
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        A2[i] = i < real ? A2[i] * kLog2e : 0.f;
        x[i] = i < real ? x[i] : 0.f;
    }
    if (OUT && nchunks > 1 && !carried) {
        // few chunks, from zero: the end states before this chunk are carried here
        const float* end = xs + b * nchunks * N * s.D + c;
        const float* sum = sums + b * nchunks * s.D + c;
        constexpr int U = 8;
        for (int64_t j0 = 0; j0 < k; j0 += U) {
            float e[U][NS], d[U];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const int64_t at = j0 + j < k ? j0 + j : k - 1;
                d[j] = sum[at * s.D];
#pragma unroll
                for (int i = 0; i < NS; ++i)
                    e[j][i] = end[(at * N + (n0 + i < N ? n0 + i : lastn)) * s.D];
            }
#pragma unroll
            for (int j = 0; j < U; ++j)
                if (j0 + j < k) {
#pragma unroll
                    for (int i = 0; i < NS; ++i)
                        x[i] = fmaf(chunk_decay(A2[i], d[j]), x[i], e[j][i]);
                }
        }
    }
    float total = 0.f;  // sum of the steps

    // The next tile's values, in flight as they lie in memory: a conversion would wait
    // for them.  A lane's places in a tile are 32-bit byte offsets from the tile's first row,
    // the same for all tiles but the last, whose rows past the end are copies of the
    // last (so that no load is under a branch) and are not walked.
    T du[R], dd[R], dz[R], dr[PER];
    uint32_t ou[R], od[R], oz[R], oe[PER];
    bool of_c[PER];
    auto places = [&](int rows_left) {
        const int last = rows_left < kSteps ? rows_left - 1 : kSteps - 1;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint32_t j = wave * R + r < last ? wave * R + r : last;
            ou[r] = (j * uint32_t(s.ld_u) + lc) * sizeof(T);
            od[r] = (j * uint32_t(s.ld_dt) + lc) * sizeof(T);
            oz[r] = (j * uint32_t(s.ld_z) + lc) * sizeof(T);
        }
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            const int e = threadIdx.x + p * kWave * S, f = e % (S * W * NS);
            const int j = e < E ? e / (S * W * NS) : 0;  // the row
            const int n = f / (W * NS) * NS + f % NS;
            of_c[p] = f / NS % W;
            oe[p] = (uint32_t(j < last ? j : last) * uint32_t(of_c[p] ? s.ld_c : s.ld_b) +
                     (n < N ? n : N - 1)) * sizeof(T);
        }
    };
    // (the next tile's first row)
    const T* nu = pu + t_begin * s.ld_u;
    const T* nd = pdt + t_begin * s.ld_dt;
    const T* nz = GATE ? pz + t_begin * s.ld_z : nullptr;
    const T *nB = pB + t_begin * s.ld_b, *nC = pC + t_begin * s.ld_c;
    auto load = [&]() {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            du[r] = at_byte(nu, ou[r]);
            dd[r] = at_byte(nd, od[r]);
            if constexpr (GATE) dz[r] = at_byte(nz, oz[r]);
        }
#pragma unroll
        for (int p = 0; p < PER; ++p) dr[p] = at_byte(OUT && of_c[p] ? nC : nB, oe[p]);
    };
    auto advance = [&]() {
        nu += kSteps * s.ld_u;
        nd += kSteps * s.ld_dt;
        if constexpr (GATE) nz += kSteps * s.ld_z;
        nB += kSteps * s.ld_b;
        nC += kSteps * s.ld_c;
    };
    // The steps of a tile (TAIL: the first `left`) for CNT states of this wavefront.  (Slots
    // past N and steps past the row's end are not walked as zeros: zero times an infinite
    // input or pole is not zero.)
    auto walk = [&](auto count, auto tail, int left) {
        constexpr int CNT = decltype(count)::value;
        constexpr bool TAIL = decltype(tail)::value;
        // (fewer steps unrolled where their values from LDS would not fit the registers)
        constexpr int kUnroll = NS > 6 ? 2 : kSteps;
#pragma unroll kUnroll
        for (int j = 0; j < kSteps; ++j) {
            if (TAIL && j >= left) break;
            const float2 d = step[j][lane];
            float acc = 0.f;
#pragma unroll
            for (int i = 0; i < CNT; ++i) {
                x[i] = fmaf(exp2_fast(d.x * A2[i]), x[i], d.y * rows[j][wave][0][i]);
                if constexpr (OUT) acc = fmaf(rows[j][wave][W - 1][i], x[i], acc);
            }
            if constexpr (OUT)
                part[wave][j][lane] = acc;
            else
                total += d.x;
        }
    };
    // One tile: what is loaded goes to LDS, the next tile's loads start, this one is
    // walked and its outputs leave.  TAIL: rows may be missing.
    auto tile_steps = [&](int64_t t0, auto tail) {
        constexpr bool TAIL = decltype(tail)::value;
        const int left = int(te - t0 < kSteps ? te - t0 : kSteps);
        float cu[R], cz[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int j = wave * R + r;
            cu[r] = io_load(&du[r]);
            if constexpr (GATE) cz[r] = io_load(&dz[r]);
            float2 d;
            d.x = softplus(io_load(&dd[r]) + bias);
            d.y = d.x * cu[r];
            step[j][lane] = d;
        }
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            const int e = threadIdx.x + p * kWave * S;
            if (E % (kWave * S) == 0 || e < E)
                (&rows[0][0][0][0])[e] = io_load(&dr[p]);
        }
        __syncthreads();
        const int64_t after = te - t0 - kSteps;  // rows left for the next tile
        if (after > 0) {
            advance();
            if (after < kSteps) places(int(after));
        }
        load();  // (after the last tile: that tile again)
        if (real == NS)
            walk(std::integral_constant<int, NS>(), tail, left);
        else
            with_count<NS - 1>(real, [&](auto count) { walk(count, tail, left); });
        __syncthreads();
        if constexpr (OUT) {
            T* row = py + t0 * s.D;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int j = wave * R + r;
                float o = h0 * cu[r];
#pragma unroll
                for (int w = 0; w < S; ++w) o += part[w][j][lane];
                if constexpr (GATE) o *= cz[r] * sigmoid(cz[r]);
                if (!TAIL || j < left)
                    io_store(&at_byte(row, uint32_t(j) * uint32_t(s.D * sizeof(T)) + lc * uint32_t(sizeof(T))), o);
            }
        }
    };
    if (t_begin < te) {
        places(int(te - t_begin < kSteps ? te - t_begin : kSteps));
        load();
    }
    int64_t t0 = t_begin;
    for (; t0 + kSteps <= te; t0 += kSteps) tile_steps(t0, std::false_type());
    if (t0 < te) tile_steps(t0, std::true_type());
    if constexpr (OUT) {
        for (int64_t t = (te > t_begin ? te : t_begin) + wave; t < t_end; t += S)
            if (own) io_store(py + t * s.D + lc, 0.f);
        if (k == nchunks - 1 && own) {
#pragma unroll
            for (int i = 0; i < NS; ++i)
                if (i < real) state[(b * s.D + c) * N + n0 + i] = x[i];
        }
    } else if (own) {
#pragma unroll
        for (int i = 0; i < NS; ++i)
            if (i < real) xs[((b * nchunks + k) * N + n0 + i) * s.D + c] = x[i];
        if (wave == 0) sums[(b * nchunks + k) * s.D + c] = total;
    }
}

// End states from zero become entry states, in place.
__global__ __launch_bounds__(256) void carry_kernel(const float* __restrict__ A,
                                                    const float* __restrict__ sums,
                                                    float* __restrict__ xs,
                                                    const float* __restrict__ state, bool resume,
                                                    int64_t B, int64_t D, int N, int64_t nchunks)
{
    const int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x;
    const int64_t c = id % D, n = id / D % N, b = id / (D * N);
    if (b >= B) return;
    const float A2 = A[c * N + n] * kLog2e;
    float* px = xs + (b * nchunks * N + n) * D + c;
    const float* ps = sums + b * nchunks * D + c;
    float x = resume ? state[(b * D + c) * N + n] : 0.f;
    constexpr int U = 8;
    for (int64_t k = 0; k < nchunks; k += U) {
        float end[U], a[U];
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (k + i < nchunks - 1) {
                end[i] = px[(k + i) * N * D];
                a[i] = ps[(k + i) * D];
            }
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (k + i < nchunks) {
                px[(k + i) * N * D] = x;
                if (k + i < nchunks - 1) x = fmaf(chunk_decay(A2, a[i]), x, end[i]);
            }
    }
}

// V states to a lane (4, or 1 where there are fewer), LPR lanes to a (batch row,
// channel).  A lane whose states would pass the row's end takes its last V: the first
// `twice` of them are another lane's too, take no part in y, and are stored with the same
// bits.  (The row's lanes are of one wavefront, which has read them all by then.)
template <typename T, int V, int LPR>
__global__ __launch_bounds__(256) void scan_step_kernel(Selective s, float* state, T* __restrict__ y)
{
    const int sub = threadIdx.x % LPR;
    const int64_t row = (int64_t(blockIdx.x) * 256 + threadIdx.x) / LPR;
    if (row >= s.B * s.D) return;
    const int64_t b = row / s.D, c = row - b * s.D;
    const int64_t grp = c / (s.D / s.G);
    const int n = sub * V < s.N - V ? sub * V : s.N - V, twice = sub * V - n;
    float* px = state + row * s.N + n;
    const Raw<float, V> rx = load_raw<V>(px), rA = load_raw<V>(s.A + c * s.N + n);
    const Raw<T, V> rB = load_raw<V>(static_cast<const T*>(s.Bm) + b * s.ld_b + grp * s.N + n);
    const Raw<T, V> rC = load_raw<V>(static_cast<const T*>(s.Cm) + b * s.ld_c + grp * s.N + n);
    const T ru = static_cast<const T*>(s.u)[b * s.ld_u + c];
    const T rd = static_cast<const T*>(s.dt)[b * s.ld_dt + c];
    const T rz = s.z ? static_cast<const T*>(s.z)[b * s.ld_z + c] : T();
    const float bias = s.dt_bias ? s.dt_bias[c] : 0.f, h0 = s.h0 ? s.h0[c] : 0.f;
    float x[V], A[V], Bv[V], Cv[V];
    expand<V, float>(rx, x);
    expand<V, float>(rA, A);
    expand<V, T>(rB, Bv);
    expand<V, T>(rC, Cv);
    const float u = io_load(&ru), delta = softplus(io_load(&rd) + bias), du = delta * u;
    float o = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        x[i] = fmaf(exp2_fast(delta * (A[i] * kLog2e)), x[i], du * Bv[i]);
        if (i >= twice) o = fmaf(Cv[i], x[i], o);
    }
    put<V>(px, x);
#pragma unroll
    for (int off = 1; off < LPR; off *= 2) o += __shfl_xor(o, off, kWave);
    if (sub == 0) {
        o = fmaf(h0, u, o);
        if (s.z) {
            const float z = io_load(&rz);
            o *= z * sigmoid(z);
        }
        io_store(y + row, o);
    }
}

// States per lane for this many wavefronts per tile.
int states_per_lane(int N, int waves)
{
    const int n = (N + waves - 1) / waves;
    return n <= 4 ? n : n <= 6 ? 6 : 8;
}

template <typename F>
hipError_t with_split(int ns, int waves, F f)
{
#define LH_SPLIT(n, w) \
    if (ns == n && waves == w) \
    return f(std::integral_constant<int, n>(), std::integral_constant<int, w>())
    LH_SPLIT(1, 4);
    LH_SPLIT(2, 4);
    LH_SPLIT(3, 4);
    LH_SPLIT(4, 4);
    LH_SPLIT(1, 8);
    LH_SPLIT(2, 8);
    LH_SPLIT(3, 8);
    LH_SPLIT(4, 8);
    LH_SPLIT(3, 16);
    LH_SPLIT(4, 16);
    LH_SPLIT(6, 16);
    LH_SPLIT(8, 16);
#undef LH_SPLIT
    return hipErrorInvalidValue;
}

template <typename T>
hipError_t scan(const Selective& s, float* state, bool resume, T* y, void* workspace,
                hipStream_t stream)
{
    const SelectivePlan p = selective_plan(s.B, s.T, s.D, s.N, s.G);
    const int64_t blocks = s.B * p.nchunks * group_tiles(s.D, s.G) * s.G;
    float* xs = static_cast<float*>(workspace);
    float* sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.off_sums);
    return with_split(p.ns, p.waves, [&](auto ns, auto waves) {
        constexpr int NS = decltype(ns)::value, S = decltype(waves)::value;
        // (a chunk carries the end states before it by itself where they are few and nothing
        // else is written that another chunk reads)
        const bool carried = p.nchunks > kFewChunks || resume;
        if (p.nchunks > 1) {
            hipLaunchKernelGGL((scan_kernel<T, NS, S, false, false>),
                               dim3(uint32_t(blocks / p.nchunks * (p.nchunks - 1))),
                               dim3(kWave * S), 0, stream, s, p.chunk, p.nchunks, carried, xs, sums,
                               state, resume, y);
            hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            if (carried) {
                hipLaunchKernelGGL(carry_kernel, dim3(uint32_t((s.B * s.D * s.N + 255) / 256)),
                                   dim3(256), 0, stream, s.A, sums, xs, state, resume, s.B, s.D,
                                   s.N, p.nchunks);
                if ((e = hipGetLastError()) != hipSuccess) return e;
            }
        }
        const auto last = s.z ? scan_kernel<T, NS, S, true, true> : scan_kernel<T, NS, S, true, false>;
        hipLaunchKernelGGL(last, dim3(uint32_t(blocks)), dim3(kWave * S), 0, stream, s, p.chunk,
                           p.nchunks, carried, xs, sums, state, resume, y);
        return hipGetLastError();
    });
}

// States to a lane of a step, and lanes to a row (a power of two).
int step_states(int N) { return N >= 4 ? 4 : 1; }
int step_lanes(int N)
{
    int lpr = 1;
    while (lpr * step_states(N) < N) lpr *= 2;
    return lpr;
}

template <typename T>
hipError_t scan_step(const Selective& s, float* state, T* y, hipStream_t stream)
{
    const int V = step_states(s.N), lpr = step_lanes(s.N);
    const dim3 grid(uint32_t((s.B * s.D * lpr + 255) / 256));
#define LH_STEP(v, l) \
    if (V == v && lpr == l) \
    hipLaunchKernelGGL((scan_step_kernel<T, v, l>), grid, dim3(256), 0, stream, s, state, y)
    LH_STEP(1, 1);
    LH_STEP(1, 2);
    LH_STEP(1, 4);
    LH_STEP(4, 1);
    LH_STEP(4, 2);
    LH_STEP(4, 4);
    LH_STEP(4, 8);
    LH_STEP(4, 16);
    LH_STEP(4, 32);
#undef LH_STEP
    return hipGetLastError();
}

}  // namespace

SelectivePlan selective_plan(int64_t B, int64_t T, int64_t D, int N, int G)
{
    SelectivePlan p;
    const int64_t tiles = B * group_tiles(D, G) * G;
    // One pass takes about 6 us and 0.1 us a step while the tiles leave the SIMDs waiting
    // (8 wavefronts to a tile, up to 270 tiles; then in proportion), from 17 states on, where a
    // lane or a workgroup holds more of them, 50 + 2.6 N ns; chunks take 14 us for two or three
    // launches and, with the SIMDs full, 0.45 ns a step and tile at 16 states.
    // (T = 2048, D = 2048, one pass and chunks: 16 states, 4 rows 199 and 133 us, 6 rows
    // 200 and 194, 8 rows 199 and 232; 32 states, 4 rows 273 and 190, 8 rows 275 and 328; 64
    // states, 2 rows 434 and 210, 4 rows 436 and 389; 128 states, 2 rows 786 and 379, 4 rows
    // 792 and 711.  16 states: 4 rows of 128 steps 18 and 25 us, 1 row of 256 steps 30 and 22.)
    const double step = N <= 16 ? 0.1 : 0.05 + 0.0026 * N;
    const double one = 6.0 + step * T * (tiles > 270 ? tiles / 270.0 : 1.0);
    const double cut = 14.0 + 4.5e-4 * T * tiles * (N + 8) / 24;
    // Chunks fill 8192 wavefronts (8 to a SIMD) where they stay 32 steps or longer.
    const int wide = N <= 16 ? 4 : N <= 32 ? 8 : 16;
    int64_t n = cut < one ? (8192 + tiles * wide - 1) / (tiles * wide) : 1;
    if (n > T / 32) n = T / 32;
    if (n < 3) n = 1;
    // Up to 16 states, 4 wavefronts to a tile do the least work beside the states; in one
    // pass of fewer than 1024 tiles 8 wait less (16 rows 299 against 345 us, 32 rows 560
    // against 515).
    p.waves = N <= 16 && n == 1 && tiles < 1024 ? 8 : wide;
    p.ns = states_per_lane(N, p.waves);
    p.chunk = ((T + n - 1) / n + kSteps - 1) / kSteps * kSteps;
    if (p.chunk < kSteps) p.chunk = kSteps;
    p.nchunks = T > 0 ? (T + p.chunk - 1) / p.chunk : 1;
    p.off_sums = p.ws_bytes = 0;
    if (p.nchunks > 1) {
        p.off_sums = size_t(B) * p.nchunks * N * D * sizeof(float);
        p.ws_bytes = p.off_sums + size_t(B) * p.nchunks * D * sizeof(float);
    }
    return p;
}

int64_t selective_threads(int64_t B, int64_t T, int64_t D, int N, int G)
{
    const SelectivePlan p = selective_plan(B, T, D, N, G);
    const int64_t scan = B * p.nchunks * group_tiles(D, G) * G * kWave * p.waves;
    const int64_t carry = p.nchunks > 1 ? B * D * N : 0;
    return (scan > carry ? scan : carry) + 256;  // (the carry's last workgroup)
}

int64_t selective_step_threads(int64_t B, int64_t D, int N)
{
    return B * D * step_lanes(N) + 256;
}

hipError_t launch_selective(const Selective& s, float* state, bool resume, void* y,
                            void* workspace, hipStream_t stream)
{
    return s.bf16_io ? scan(s, state, resume, static_cast<bf16*>(y), workspace, stream)
                     : scan(s, state, resume, static_cast<float*>(y), workspace, stream);
}

hipError_t launch_selective_step(const Selective& s, float* state, void* y, hipStream_t stream)
{
    return s.bf16_io ? scan_step(s, state, static_cast<bf16*>(y), stream)
                     : scan_step(s, state, static_cast<float*>(y), stream);
}

}  // namespace lh
