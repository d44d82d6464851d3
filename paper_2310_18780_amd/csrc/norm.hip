// Layer norm over the last axis of [rows, D], and its gradients:
//
//   s = x (+ r),  m = mean s,  v = mean (s - m)^2,  h = (s - m) (v + eps)^(-1/2)
//   y = h w + b
//   g = dy w:  ds = (v + eps)^(-1/2) (g - mean g - h mean(g h)) (+ dtotal)
//   dw = sum over rows of dy h,  db = sum over rows of dy
//
// Bound by memory: a row is read once and written once (with the residual sum: two
// read, two written), about 8 flops per value.  A team of one wavefront, or of 4 or
// 16, holds its row in registers, so the mean is taken before the squares (no
// cancellation) without a second read.  Every load is a whole 16-byte piece at any
// alignment and under no branch; with branches for the row's end, in which each piece
// was converted and so waited for, 65536 rows of 2048 bfloat16 took 284 us, so 98 us
// (5.5 TB/s, a large copy 5.0-5.2; 13993 rows of 1001 float32: 25 us).
//
// The gradient keeps a lane's columns of dw and db in registers over all rows its
// team walks (four wavefronts to a row from 1025 columns on: 8 values a lane and five
// wavefronts per SIMD, 207 us at 65536 x 2048 bfloat16 against 290 us with 32 values
// and two); each workgroup leaves one partial row, and a second launch adds those in a
// fixed order (5 us of 219 in all).
#include "norm.hpp"

#include "block_ops.hpp"

namespace lh {
namespace {

// Values of a row that a lane holds: what the team's registers allow (the gradient
// holds five arrays of them).
constexpr int hold(int team, bool grad)
{
    return grad ? (team == 1024 ? 8 : 16) : (team == 1024 ? 16 : 32);
}
constexpr int64_t kMaxBlocks = 1 << 20;  // grid-stride beyond
constexpr int64_t kGradBlocks = 1024;  // workgroups (partial rows) of the gradient

constexpr int norm_block(int team) { return team < 256 ? 256 : team; }

// Sums of one or two values over a team; red holds a pair per wavefront.  The
// caller alternates between two halves of red, so one barrier per call is enough.
template <int TEAM>
__device__ __forceinline__ float2 team_sum(float2 v, float2* red)
{
    v.x = wave_sum(v.x);
    v.y = wave_sum(v.y);
    if constexpr (TEAM > kWave) {
        constexpr int n = TEAM / kWave;
        if ((threadIdx.x & (kWave - 1)) == 0) red[threadIdx.x / kWave] = v;
        __syncthreads();
        v = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < n; ++i) {
            v.x += red[i].x;
            v.y += red[i].y;
        }
    }
    return v;
}

// A lane's pieces of a row: ITER pieces of V values, TEAM pieces apart.  A piece that
// would pass the row's end starts V values before it instead, so that every load is a
// whole piece under no branch; its first `twice` values are another lane's as well, and
// take no part in sums.  (Both lanes store the same bits.)  FULL: no such piece.
template <int V, int TEAM, int ITER, bool FULL>
struct Pieces {
    int at[ITER], twice[ITER];
    __device__ __forceinline__ Pieces(int lane, int D)
    {
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * TEAM + lane) * V;
            at[i] = FULL || c + V <= D ? c : D - V;
            twice[i] = c - at[i];
        }
    }
    __device__ __forceinline__ bool mine(int i, int j) const { return FULL || j >= twice[i]; }
};

template <typename T, int TEAM, int ITER, bool FULL>
__global__ __launch_bounds__(norm_block(TEAM)) void norm_kernel(
    const T* x, const T* residual, const float* __restrict__ w, const float* __restrict__ b,
    T* __restrict__ y, T* total, float* __restrict__ mean, float* __restrict__ rstd, int64_t rows,
    int D, float eps)
{
    constexpr int V = kVec<T>;
    constexpr int teams = norm_block(TEAM) / TEAM;
    __shared__ float2 red[2][norm_block(TEAM) / kWave];
    const int lane = threadIdx.x % TEAM;
    const Pieces<V, TEAM, ITER, FULL> p(lane, D);
    const int64_t step = int64_t(gridDim.x) * teams;
    for (int64_t row = int64_t(blockIdx.x) * teams + threadIdx.x / TEAM; row < rows; row += step) {
        Raw<T, V> raw[ITER], res[ITER];
#pragma unroll
        for (int i = 0; i < ITER; ++i) raw[i] = load_raw<V>(x + row * D + p.at[i]);
        if (residual) {
#pragma unroll
            for (int i = 0; i < ITER; ++i) res[i] = load_raw<V>(residual + row * D + p.at[i]);
        }
        float v[ITER][V], s = 0.f;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            expand<V, T>(raw[i], v[i]);
            if (residual) {
                float r[V];
                expand<V, T>(res[i], r);
#pragma unroll
                for (int j = 0; j < V; ++j) v[i][j] += r[j];
            }
#pragma unroll
            for (int j = 0; j < V; ++j) s += p.mine(i, j) ? v[i][j] : 0.f;
        }
        const float m = team_sum<TEAM>(make_float2(s, 0.f), red[0]).x / D;
        if (total) {  // (in place of x or residual: the whole team has read them by now)
#pragma unroll
            for (int i = 0; i < ITER; ++i) put<V>(total + row * D + p.at[i], v[i]);
        }
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < ITER; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                v[i][j] -= m;
                q = fmaf(p.mine(i, j) ? v[i][j] : 0.f, v[i][j], q);
            }
        const float var = team_sum<TEAM>(make_float2(q, 0.f), red[1]).x / D;
        const float rs = 1.f / sqrtf(var + eps);
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const float *pw = w + p.at[i], *pb = b ? b + p.at[i] : nullptr;
            float o[V];
#pragma unroll
            for (int j = 0; j < V; ++j) o[j] = v[i][j] * rs * pw[j];
            if (b) {
#pragma unroll
                for (int j = 0; j < V; ++j) o[j] += pb[j];
            }
            put<V>(y + row * D + p.at[i], o);
        }
        if (lane == 0) {
            if (mean) mean[row] = m;
            if (rstd) rstd[row] = rs;
        }
    }
}

// Rows that no team holds: one workgroup of 16 wavefronts per row, read three times.
template <typename T>
__global__ __launch_bounds__(1024) void norm_wide_kernel(
    const T* x, const T* residual, const float* __restrict__ w, const float* __restrict__ b,
    T* __restrict__ y, T* total, float* __restrict__ mean, float* __restrict__ rstd, int64_t rows,
    int64_t D, float eps)
{
    constexpr int V = kVec<T>;
    __shared__ float2 red[3][16];
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T* px = x + row * D;
        const T* pr = residual ? residual + row * D : nullptr;
        auto load = [&](int64_t c, float(&v)[V]) {
            const int n = int(D - c < V ? D - c : V);
            load_some<V>(px + c, n, v);
            if (pr) {
                float r[V];
                load_some<V>(pr + c, n, r);
                for (int j = 0; j < V; ++j) v[j] += r[j];
            }
            return n;
        };
        float s = 0.f;
        for (int64_t c = threadIdx.x * V; c < D; c += 1024 * V) {
            float v[V];
            load(c, v);
            for (int j = 0; j < V; ++j) s += v[j];
        }
        const float m = team_sum<1024>(make_float2(s, 0.f), red[0]).x / D;
        float q = 0.f;
        for (int64_t c = threadIdx.x * V; c < D; c += 1024 * V) {
            float v[V];
            const int n = load(c, v);
            for (int j = 0; j < V; ++j)
                if (j < n) q = fmaf(v[j] - m, v[j] - m, q);
        }
        const float var = team_sum<1024>(make_float2(q, 0.f), red[1]).x / D;
        const float rs = 1.f / sqrtf(var + eps);
        for (int64_t c = threadIdx.x * V; c < D; c += 1024 * V) {
            float v[V];
            const int n = load(c, v);
            if (total) store_some<V>(total + row * D + c, n, v);
            for (int j = 0; j < V; ++j)
                if (j < n) v[j] = fmaf((v[j] - m) * rs, w[c + j], b ? b[c + j] : 0.f);
            store_some<V>(y + row * D + c, n, v);
        }
        if (threadIdx.x == 0) {
            if (mean) mean[row] = m;
            if (rstd) rstd[row] = rs;
        }
    }
}

template <typename T, int TEAM, int ITER, bool FULL>
__global__ __launch_bounds__(norm_block(TEAM)) void norm_grad_kernel(
    const T* __restrict__ dy, const T* __restrict__ x, const float* __restrict__ w,
    const float* __restrict__ mean, const float* __restrict__ rstd, const T* dtotal, T* dx,
    float* __restrict__ part, int64_t rows, int D)
{
    constexpr int V = kVec<T>;
    constexpr int teams = norm_block(TEAM) / TEAM;
    __shared__ float2 red[2][norm_block(TEAM) / kWave];
    const int lane = threadIdx.x % TEAM;
    const Pieces<V, TEAM, ITER, FULL> p(lane, D);
    const float inv = 1.f / D;
    float wv[ITER][V], aw[ITER][V], ab[ITER][V];
#pragma unroll
    for (int i = 0; i < ITER; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            wv[i][j] = w[p.at[i] + j];
            aw[i][j] = ab[i][j] = 0.f;
        }
    const int64_t step = int64_t(gridDim.x) * teams;
    int turn = 0;
    for (int64_t row = int64_t(blockIdx.x) * teams + threadIdx.x / TEAM; row < rows; row += step) {
        Raw<T, V> rx[ITER], rg[ITER], rt[ITER];
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            rx[i] = load_raw<V>(x + row * D + p.at[i]);
            rg[i] = load_raw<V>(dy + row * D + p.at[i]);
        }
        if (dtotal) {  // (read before the team's sum: dx may be its buffer)
#pragma unroll
            for (int i = 0; i < ITER; ++i) rt[i] = load_raw<V>(dtotal + row * D + p.at[i]);
        }
        const float m = mean[row], rs = rstd[row];
        float h[ITER][V], g[ITER][V];
        float2 s = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            expand<V, T>(rx[i], h[i]);
            expand<V, T>(rg[i], g[i]);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                h[i][j] = (h[i][j] - m) * rs;
                aw[i][j] = fmaf(g[i][j], h[i][j], aw[i][j]);
                ab[i][j] += g[i][j];
                g[i][j] *= wv[i][j];
                const float own = p.mine(i, j) ? g[i][j] : 0.f;
                s.x += own;
                s.y = fmaf(own, h[i][j], s.y);
            }
        }
        s = team_sum<TEAM>(s, red[turn]);
        turn ^= 1;
        const float mg = s.x * inv, mgh = s.y * inv;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            float t[V];
            if (dtotal) expand<V, T>(rt[i], t);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = rs * (g[i][j] - fmaf(h[i][j], mgh, mg));
                h[i][j] = dtotal ? d + t[j] : d;
            }
            put<V>(dx + row * D + p.at[i], h[i]);
        }
    }
    // one partial row [2, D] per workgroup
    float* out = part + int64_t(blockIdx.x) * 2 * D;
    if constexpr (teams == 1) {
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (p.mine(i, j)) {
                    out[p.at[i] + j] = aw[i][j];
                    out[D + p.at[i] + j] = ab[i][j];
                }
        }
    } else {
        // the teams' sums of a lane's columns, added (TEAM is a wavefront)
        __shared__ float sum[teams][2][V][kWave];
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < V; ++j) {
                sum[threadIdx.x / TEAM][0][j][lane] = aw[i][j];
                sum[threadIdx.x / TEAM][1][j][lane] = ab[i][j];
            }
            __syncthreads();
            for (int k = threadIdx.x / TEAM; k < 2 * V; k += teams) {
                const int which = k / V, j = k % V;
                float a = 0.f;
#pragma unroll
                for (int t = 0; t < teams; ++t) a += sum[t][which][j][lane];
                if (p.mine(i, j)) out[int64_t(which) * D + p.at[i] + j] = a;
            }
        }
    }
}

// Rows that no team holds: the rows' gradient, read twice; the columns' sums apart.
template <typename T>
__global__ __launch_bounds__(1024) void norm_grad_wide_kernel(
    const T* __restrict__ dy, const T* __restrict__ x, const float* __restrict__ w,
    const float* __restrict__ mean, const float* __restrict__ rstd, const T* dtotal, T* dx,
    int64_t rows, int64_t D)
{
    __shared__ float2 red[2][16];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const float m = mean[row], rs = rstd[row];
        const T *px = x + row * D, *pg = dy + row * D;
        float2 s = make_float2(0.f, 0.f);
        for (int64_t c = threadIdx.x; c < D; c += 1024) {
            const float g = io_load(pg + c) * w[c];
            s.x += g;
            s.y = fmaf(g, (io_load(px + c) - m) * rs, s.y);
        }
        s = team_sum<1024>(s, red[turn]);
        turn ^= 1;
        const float mg = s.x / D, mgh = s.y / D;
        for (int64_t c = threadIdx.x; c < D; c += 1024) {
            const float g = io_load(pg + c) * w[c], h = (io_load(px + c) - m) * rs;
            const float d = rs * (g - fmaf(h, mgh, mg));
            io_store(dx + row * D + c, dtotal ? d + io_load(dtotal + row * D + c) : d);
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void norm_columns_kernel(
    const T* __restrict__ dy, const T* __restrict__ x, const float* __restrict__ mean,
    const float* __restrict__ rstd, float* __restrict__ part, int64_t rows, int64_t D)
{
    const int64_t c = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (c >= D) return;
    float aw = 0.f, ab = 0.f;
    for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
        const float g = io_load(dy + row * D + c);
        aw = fmaf(g, (io_load(x + row * D + c) - mean[row]) * rstd[row], aw);
        ab += g;
    }
    part[int64_t(blockIdx.y) * 2 * D + c] = aw;
    part[int64_t(blockIdx.y) * 2 * D + D + c] = ab;
}

// Threads per row (0: the wide kernels): a wavefront where it holds the row and there are
// rows enough to fill the GPU (two wavefronts per SIMD), else more, so that few rows
// finish sooner (64 rows of 2048: 3 us).
template <typename T>
int norm_team(int64_t rows, int64_t D, bool grad)
{
    if (D < kVec<T>) return 0;
    if (D <= 64 * hold(64, grad) && (rows >= 2048 || D <= 64 * kVec<T>)) return 64;
    if (D <= 256 * hold(256, grad) && (rows >= 512 || D <= 256 * kVec<T>)) return 256;
    return D <= 1024 * hold(1024, grad) ? 1024 : 0;
}

// ITER for a team: the pieces of a row that a lane holds.
template <typename T, bool GRAD, typename F>
hipError_t with_shape(int team, int64_t D, F f)
{
    const int64_t pieces = (D + int64_t(team) * kVec<T> - 1) / (int64_t(team) * kVec<T>);
    auto iters = [&](auto t) {
        constexpr int most = hold(decltype(t)::value, GRAD) / kVec<T>;
        auto full = [&](auto it) {
            if (D == int64_t(team) * kVec<T> * decltype(it)::value) return f(t, it, std::true_type());
            return f(t, it, std::false_type());
        };
        if constexpr (most > 1)
            if (pieces <= 1) return full(std::integral_constant<int, 1>());
        if constexpr (most > 2)
            if (pieces <= 2) return full(std::integral_constant<int, 2>());
        if constexpr (most > 4)
            if (pieces <= 4) return full(std::integral_constant<int, 4>());
        return full(std::integral_constant<int, most>());
    };
    if (team == 64) return iters(std::integral_constant<int, 64>());
    if (team == 256) return iters(std::integral_constant<int, 256>());
    return iters(std::integral_constant<int, 1024>());
}

int64_t blocks_for(int team, int64_t rows, int64_t cap)
{
    const int64_t teams = norm_block(team) / team;
    const int64_t n = (rows + teams - 1) / teams;
    return n < cap ? n : cap;
}

template <typename T>
hipError_t norm(const T* x, const T* residual, const float* w, const float* b, T* y, T* total,
                float* mean, float* rstd, int64_t rows, int64_t D, float eps, hipStream_t stream)
{
    const int team = norm_team<T>(rows, D, false);
    if (team == 0) {
        hipLaunchKernelGGL((norm_wide_kernel<T>), dim3(uint32_t(rows < kMaxBlocks ? rows : kMaxBlocks)),
                           dim3(1024), 0, stream, x, residual, w, b, y, total, mean, rstd, rows, D,
                           eps);
        return hipGetLastError();
    }
    return with_shape<T, false>(team, D, [&](auto t, auto it, auto whole) {
        constexpr int TEAM = decltype(t)::value, ITER = decltype(it)::value;
        constexpr bool FULL = decltype(whole)::value;
        hipLaunchKernelGGL((norm_kernel<T, TEAM, ITER, FULL>),
                           dim3(uint32_t(blocks_for(TEAM, rows, kMaxBlocks))),
                           dim3(norm_block(TEAM)), 0, stream, x, residual, w, b, y, total, mean,
                           rstd, rows, int(D), eps);
        return hipGetLastError();
    });
}

template <typename T>
hipError_t norm_grad(const T* dy, const T* x, const float* w, const float* mean, const float* rstd,
                     const T* dtotal, T* dx, float* dw, float* db, int64_t rows, int64_t D,
                     float* part, hipStream_t stream)
{
    const int team = norm_team<T>(rows, D, true);
    if (rows == 0) return launch_column_sum(part, 0, D, dw, D, db, 0, nullptr, stream);
    int64_t P;
    hipError_t e;
    if (team == 0) {
        P = 2048 / ((D + 255) / 256);  // eight workgroups to a CU
        P = P < 16 ? 16 : P > kGradBlocks ? kGradBlocks : P;
        P = P < rows ? P : rows;
        hipLaunchKernelGGL((norm_grad_wide_kernel<T>),
                           dim3(uint32_t(rows < kMaxBlocks ? rows : kMaxBlocks)), dim3(1024), 0,
                           stream, dy, x, w, mean, rstd, dtotal, dx, rows, D);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        hipLaunchKernelGGL((norm_columns_kernel<T>),
                           dim3(uint32_t((D + 255) / 256), uint32_t(P)), dim3(256), 0, stream, dy,
                           x, mean, rstd, part, rows, D);
        e = hipGetLastError();
    } else {
        // Eight rows to a team, since a partial row costs about as much as two (4096 rows of
        // 2048 bfloat16: 21 us, with four 26), where that leaves a workgroup to a CU.
        P = blocks_for(team, (rows + 7) / 8, kGradBlocks);
        if (P < 256) P = blocks_for(team, rows, 256);
        e = with_shape<T, true>(team, D, [&](auto t, auto it, auto whole) {
            constexpr int TEAM = decltype(t)::value, ITER = decltype(it)::value;
        constexpr bool FULL = decltype(whole)::value;
            hipLaunchKernelGGL((norm_grad_kernel<T, TEAM, ITER, FULL>), dim3(uint32_t(P)),
                               dim3(norm_block(TEAM)), 0, stream, dy, x, w, mean, rstd, dtotal, dx,
                               part, rows, int(D));
            return hipGetLastError();
        });
    }
    if (e != hipSuccess) return e;
    return launch_column_sum(part, P, D, dw, D, db, 0, nullptr, stream);
}

}  // namespace

size_t norm_grad_workspace_bytes(int64_t rows, int64_t D)
{
    return sizeof(float) * 2 * D * (rows < kGradBlocks ? rows : kGradBlocks);
}

hipError_t launch_norm(const void* x, const void* residual, const float* w, const float* b,
                       void* y, void* total, float* mean, float* rstd, bool bf16_io, int64_t rows,
                       int64_t D, float eps, hipStream_t stream)
{
    if (bf16_io)
        return norm(static_cast<const bf16*>(x), static_cast<const bf16*>(residual), w, b,
                    static_cast<bf16*>(y), static_cast<bf16*>(total), mean, rstd, rows, D, eps,
                    stream);
    return norm(static_cast<const float*>(x), static_cast<const float*>(residual), w, b,
                static_cast<float*>(y), static_cast<float*>(total), mean, rstd, rows, D, eps,
                stream);
}

hipError_t launch_norm_grad(const void* dy, const void* x, const float* w, const float* mean,
                            const float* rstd, const void* dtotal, void* dx, float* dw, float* db,
                            bool bf16_io, int64_t rows, int64_t D, void* workspace,
                            hipStream_t stream)
{
    float* part = static_cast<float*>(workspace);
    if (bf16_io)
        return norm_grad(static_cast<const bf16*>(dy), static_cast<const bf16*>(x), w, mean, rstd,
                         static_cast<const bf16*>(dtotal), static_cast<bf16*>(dx), dw, db, rows, D,
                         part, stream);
    return norm_grad(static_cast<const float*>(dy), static_cast<const float*>(x), w, mean, rstd,
                     static_cast<const float*>(dtotal), static_cast<float*>(dx), dw, db, rows, D,
                     part, stream);
}

}  // namespace lh
