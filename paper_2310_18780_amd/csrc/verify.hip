// Verification of drafted tokens:
//
//   token i is accepted while u_i q_i(t_i) < p_i(t_i);  m = the first that is not, or n
//   w = max(p_m - q_m, 0) where m < n, p_n where m = n
//   next token = the lowest j with w_0 + ... + w_j > u_last (w_0 + ... + w_(V-1))
//
// Which token a border falls to is decided by sums of up to 10^5 terms, so differences and sums
// are float64 (u q is exact there).  A first launch gives each tile of 2048 tokens of a row's
// target (and draft) to a workgroup: it finds m, which takes K loads, and sums its tile.  A
// second takes a row each: it adds the tiles' sums, finds the tile that the border lies in
// and walks that again.  Bound by the two launches and the loads that follow one another in
// them (tokens, their probabilities, the row); a row's probabilities are read once: 64 rows of
// 50000 float32 target and draft, 4 drafted, 7.6 and 6.4 us (25.6 MB at a copy's rate: 5), 3
// rows of 100003 bfloat16 3.8 and 4.2.  One launch would need a counter for each row that
// something has to clear first.
#include "verify.hpp"

#include "block_ops.hpp"
#include "lh.h"

namespace lh {
namespace {

constexpr int kBlock = 256;
constexpr int kEach = 8;  // values of a thread
constexpr int64_t kTileV = kBlock * kEach;

template <typename T>
struct Rows {
    const int *drafted, *lengths;
    const T *draft, *target;
    int64_t ld_draft, ld_target;
    const float *u, *u_last;
    int64_t B, K, V, tiles;
    int *accepted, *tokens;
};

template <typename T>
__device__ __forceinline__ int draft_length(const Rows<T>& a, int64_t b)
{
    if (!a.lengths) return int(a.K);
    const int n = a.lengths[b];
    return n < 0 ? 0 : n < a.K ? n : int(a.K);
}

// The number of accepted tokens, by every wavefront for itself.
template <typename T>
__device__ __forceinline__ int accepted_of(const Rows<T>& a, int64_t b, int n)
{
    const int i = threadIdx.x % kWave;
    bool taken = false;
    if (i < n) {
        const int t = a.drafted[b * a.K + i];
        if (t >= 0 && t < a.V) {
            const double p = io_load(a.target + (b * (a.K + 1) + i) * a.ld_target + t);
            const double q = a.draft ? io_load(a.draft + (b * a.K + i) * a.ld_draft + t) : 1.f;
            taken = double(a.u[b * a.K + i]) * q < p;
        }
    }
    const uint64_t refused = ~__ballot(taken);  // (lanes from n on are among them)
    return refused ? __builtin_ctzll(refused) : kWave;
}

// The weights of a thread's values from j0 on, those of the target alone in plain.
template <typename T>
__device__ __forceinline__ void weights(const Rows<T>& a, int64_t b, int m, int n, int64_t j0,
                                        double (&w)[kEach], double (&plain)[kEach])
{
    const T* p = a.target + (b * (a.K + 1) + m) * a.ld_target;
    const T* q = m < n && a.draft ? a.draft + (b * a.K + m) * a.ld_draft : nullptr;
    const int certain = m < n && !a.draft ? a.drafted[b * a.K + m] : -1;
    float pv[kEach], qv[kEach];
    if (j0 + kEach <= a.V) {
        constexpr int V = kVec<T>;
#pragma unroll
        for (int i = 0; i < kEach; i += V) {
            float x[V];
            expand<V, T>(load_raw<V>(p + j0 + i), x);
#pragma unroll
            for (int j = 0; j < V; ++j) pv[i + j] = x[j];
            if (q) expand<V, T>(load_raw<V>(q + j0 + i), x);
#pragma unroll
            for (int j = 0; j < V; ++j) qv[i + j] = q ? x[j] : 0.f;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            pv[i] = j0 + i < a.V ? io_load(p + j0 + i) : 0.f;
            qv[i] = q && j0 + i < a.V ? io_load(q + j0 + i) : 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        plain[i] = pv[i] > 0.f ? double(pv[i]) : 0.;
        const double d = double(pv[i]) - (j0 + i == certain ? 1. : double(qv[i]));
        w[i] = m < n ? (d > 0. ? d : 0.) : plain[i];
    }
}

__device__ __forceinline__ double wave_sum64(double v)
{
    for (int o = 1; o < kWave; o *= 2) v += __shfl_xor(v, o, kWave);
    return v;
}

// sums [B, tiles, 2]: a tile's weights, and the target's alone.
template <typename T>
__global__ __launch_bounds__(kBlock) void verify_sums_kernel(Rows<T> a, double2* __restrict__ sums)
{
    __shared__ double2 red[kBlock / kWave];
    const int64_t tile = blockIdx.x % a.tiles, b = blockIdx.x / a.tiles;
    const int n = draft_length(a, b), m = accepted_of(a, b, n);
    double w[kEach], plain[kEach];
    double2 s = make_double2(0., 0.);
    const int64_t j0 = tile * kTileV + threadIdx.x * kEach;
    if (j0 < a.V) {
        weights(a, b, m, n, j0, w, plain);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            s.x += w[i];
            s.y += plain[i];
        }
    }
    s.x = wave_sum64(s.x);
    s.y = wave_sum64(s.y);
    if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = make_double2(0., 0.);
        for (int i = 0; i < kBlock / kWave; ++i) {
            s.x += red[i].x;
            s.y += red[i].y;
        }
        sums[b * a.tiles + tile] = s;
        if (tile == 0) a.accepted[b] = m;
    }
}

template <typename T>
__global__ __launch_bounds__(kBlock) void verify_pick_kernel(Rows<T> a, const double2* __restrict__ sums)
{
    __shared__ double red[kBlock / kWave];
    __shared__ double2 totals;
    __shared__ int64_t found_tile;
    __shared__ double base;
    __shared__ int pick, latest;
    const int64_t b = blockIdx.x;
    // (all that does not depend on the border is asked for at once)
    const int n = draft_length(a, b), m = a.accepted[b];
    const float u_last = a.u_last[b];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int mine_drafted = threadIdx.x < a.K ? a.drafted[b * a.K + threadIdx.x] : -1;
    const double2 first = wave == 0 && lane < a.tiles ? sums[b * a.tiles + lane] : make_double2(0., 0.);
    // the first wavefront adds the tiles' sums in order, 64 at a time, twice: the total, then the
    // tile whose end is past the border (or the last one with any weight)
    if (wave == 0) {
        double2 all = first;
        for (int64_t i = lane + kWave; i < a.tiles; i += kWave) {
            const double2 s = sums[b * a.tiles + i];
            all.x += s.x;
            all.y += s.y;
        }
        all.x = wave_sum64(all.x);
        all.y = wave_sum64(all.y);
        const bool rest = all.x > 0.;
        const double border = double(u_last) * (rest ? all.x : all.y);
        double before = 0., at = 0.;
        int64_t tile = -1, some = -1;
        double some_at = 0.;
        for (int64_t i0 = 0; i0 < a.tiles && tile < 0; i0 += kWave) {
            double x = 0.;
            if (i0 + lane < a.tiles) {
                const double2 s = i0 == 0 ? first : sums[b * a.tiles + i0 + lane];
                x = rest ? s.x : s.y;
            }
            double c = x;
            for (int o = 1; o < kWave; o *= 2) {
                const double y = __shfl_up(c, o, kWave);
                if (lane >= o) c += y;
            }
            // (only a tile with weight: the lanes' sums are added in different orders, so that one without
            // may be a rounding past the sum before it, and the border lie between)
            const uint64_t past = __ballot(x > 0. && before + c > border), any = __ballot(x > 0.);
            if (any) {
                const int l = kWave - 1 - __builtin_clzll(any);
                some = i0 + l;
                some_at = before + (__shfl(c, l, kWave) - __shfl(x, l, kWave));
            }
            if (past) {
                const int l = __builtin_ctzll(past);
                tile = i0 + l;
                at = before + (l > 0 ? __shfl(c, l - 1, kWave) : 0.);
            }
            before += __shfl(c, kWave - 1, kWave);
        }
        if (tile < 0) tile = some, at = some_at;
        if (lane == 0) {
            totals = make_double2(border, rest ? 1. : 0.);
            found_tile = tile;
            base = at;
            pick = latest = -1;
        }
    }
    __syncthreads();
    const int64_t tile = found_tile;
    if (tile >= 0) {
        const double border = totals.x;
        const bool rest = totals.y != 0.;
        const int64_t j0 = tile * kTileV + threadIdx.x * kEach;
        double w[kEach] = {}, plain[kEach] = {};
        if (j0 < a.V) weights(a, b, m, n, j0, w, plain);
        double s = 0.;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if (!rest) w[i] = plain[i];
            s += w[i];
        }
        double c = s;
        for (int o = 1; o < kWave; o *= 2) {
            const double y = __shfl_up(c, o, kWave);
            if (lane >= o) c += y;
        }
        if (lane == kWave - 1) red[wave] = c;
        __syncthreads();
        double run = base;
        for (int i = 0; i < wave; ++i) run += red[i];
        run += c - s;
        int mine = -1, some = -1;  // first value past the border, last with any weight
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            run += w[i];
            if (w[i] > 0.) {
                some = int(j0) + i;
                if (mine < 0 && run > border) mine = some;
            }
        }
        // the lowest of all: of the first wavefront that has one, the lowest lane
        if (some >= 0) atomicMax(&latest, some);
        const uint64_t has = __ballot(mine >= 0);
        const int low = has ? __shfl(mine, __builtin_ctzll(has), kWave) : -1;
        if (lane == 0 && low >= 0) atomicMin(reinterpret_cast<unsigned*>(&pick), unsigned(low));
        __syncthreads();
    }
    const int next = pick >= 0 ? pick : latest;
    static_assert(LH_VERIFY_MAX_DRAFT < kBlock, "a thread for each token of a row");
    if (const int i = threadIdx.x; i <= a.K) a.tokens[b * (a.K + 1) + i] = i < m ? mine_drafted : i == m ? next : -1;
}

int64_t tiles_of(int64_t V) { return (V + kTileV - 1) / kTileV; }

template <typename T>
hipError_t verify(const Verify& v, double2* sums, hipStream_t stream)
{
    Rows<T> a;
    a.drafted = v.drafted, a.lengths = v.lengths;
    a.draft = static_cast<const T*>(v.draft_p), a.target = static_cast<const T*>(v.target_p);
    a.ld_draft = v.ld_draft, a.ld_target = v.ld_target, a.u = v.u, a.u_last = v.u_last;
    a.B = v.B, a.K = v.K, a.V = v.V, a.tiles = tiles_of(v.V);
    a.accepted = v.accepted, a.tokens = v.tokens;
    hipLaunchKernelGGL((verify_sums_kernel<T>), dim3(uint32_t(v.B * a.tiles)), dim3(kBlock), 0, stream, a, sums);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL((verify_pick_kernel<T>), dim3(uint32_t(v.B)), dim3(kBlock), 0, stream, a, sums);
    return hipGetLastError();
}

}  // namespace

size_t verify_workspace_bytes(int64_t B, int64_t, int64_t V) { return sizeof(double2) * size_t(B) * tiles_of(V); }

int64_t verify_threads(int64_t B, int64_t V) { return B * tiles_of(V) * kBlock; }

hipError_t launch_verify(const Verify& v, void* workspace, hipStream_t stream)
{
    double2* sums = static_cast<double2*>(workspace);
    return v.bf16_io ? verify<bf16>(v, sums, stream) : verify<float>(v, sums, stream);
}

}  // namespace lh
