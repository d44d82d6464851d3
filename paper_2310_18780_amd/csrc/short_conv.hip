// The short causal convolution before a scan or a long convolution, one filter of K
// taps per channel, for prompts, single tokens and gradients:
//
//   o_t = bias + sum_k w[k] x_(t - K + 1 + k),   y_t = o_t or o_t sigmoid(o_t)
//   state = the last K - 1 inputs, oldest first
//   g_t = dy_t (times the slope of silu at o_t),  dx_t = sum_k w[k] g_(t + K - 1 - k)
//   dw[k] = sum_t g_t x_(t - K + 1 + k),  dbias = sum_t g_t
//
// Bound by memory: x is read and y written once; 2 K flops (and 4 for silu) a value.
// A thread holds 16 bytes of channels and walks a run of time steps with the K - 1
// inputs before it in registers, so each input is loaded once, but for the K - 1 at
// the start of a run, which the run before it has just loaded.  Runs are as long as
// leaves the GPU enough threads.
//
// The gradient walks the same way: o_t and g_t at the front, dx K - 1 steps behind.
// A run's sums for dw and dbias stay in registers; the workgroup's runs over the
// same channels are added in LDS, and a second launch adds the workgroups' rows in a
// fixed order.
#include "short_conv.hpp"

#include "block_ops.hpp"

namespace lh {
namespace {

constexpr int kBlock = 256;
constexpr int64_t kThreads = 1 << 18;  // threads that fill the GPU: 4 wavefronts per SIMD

// Channels per thread: 16 bytes, half of that for long filters (registers).
template <typename T, int K>
constexpr int kChan = K <= 4 ? kVec<T> : kVec<T> / 2;

__device__ __forceinline__ int64_t length_of(const int* lengths, int64_t b, int64_t T)
{
    if (!lengths) return T;
    const int64_t n = lengths[b];
    return n < 0 ? 0 : n < T ? n : T;
}

template <typename T, int K, bool SILU>
__global__ __launch_bounds__(kBlock) void conv_kernel(
    const T* __restrict__ x, int64_t ld, const float* __restrict__ w,
    const float* __restrict__ bias, const int* __restrict__ lengths, T* __restrict__ state,
    bool resume, T* __restrict__ y, int64_t B, int64_t T_, int64_t D, int64_t run, int64_t runs)
{
    constexpr int V = kChan<T, K>;
    const int64_t cols = (D + V - 1) / V;
    const int64_t id = int64_t(blockIdx.x) * kBlock + threadIdx.x;
    const int64_t row = id / cols;
    if (row >= B * runs) return;
    const int64_t c = (id - row * cols) * V, b = row / runs, r = row - b * runs;
    const int n = int(D - c < V ? D - c : V);
    const int64_t len = length_of(lengths, b, T_);
    const int64_t t0 = r * run, t1 = t0 + run < T_ ? t0 + run : T_;
    const T* px = x + b * T_ * ld + c;
    T* py = y + b * T_ * D + c;
    T* ps = state + b * (K - 1) * D + c;

    float win[K][V];  // win[k] = x_(t - K + 1 + k)
#pragma unroll
    for (int k = 0; k < K - 1; ++k) {
        const int64_t t = t0 - (K - 1) + k;
        if (t >= 0 && t < len)
            load_some<V>(px + t * ld, n, win[k]);
        else if (t < 0 && resume)
            load_some<V>(ps + (t + K - 1) * D, n, win[k]);
        else
#pragma unroll
            for (int j = 0; j < V; ++j) win[k][j] = 0.f;
    }
    if (r == 0) {
        // The state after the row's last token.  Only this thread reads the old one
        // (above, and here where the row is shorter than the state), so it may write.
        float tail[K][V];
#pragma unroll
        for (int k = 0; k < K - 1; ++k) {
            const int64_t t = len - (K - 1) + k;
            if (t >= 0)
                load_some<V>(px + t * ld, n, tail[k]);
            else if (resume)
                load_some<V>(ps + (t + K - 1) * D, n, tail[k]);
            else
#pragma unroll
                for (int j = 0; j < V; ++j) tail[k][j] = 0.f;
        }
#pragma unroll
        for (int k = 0; k < K - 1; ++k) store_some<V>(ps + k * D, n, tail[k]);
    }
    float wv[K][V], bv[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int64_t cj = c + (j < n ? j : 0);
        bv[j] = bias ? bias[cj] : 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) wv[k][j] = w[cj * K + k];
    }
    const int64_t te = t1 < len ? t1 : len;
    int64_t t = t0;
    for (; t < te; ++t) {
        load_some<V>(px + t * ld, n, win[K - 1]);
        float o[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            o[j] = bv[j];
#pragma unroll
            for (int k = 0; k < K; ++k) o[j] = fmaf(wv[k][j], win[k][j], o[j]);
            if constexpr (SILU) o[j] *= sigmoid(o[j]);
        }
        store_some<V>(py + t * D, n, o);
#pragma unroll
        for (int k = 0; k < K - 1; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) win[k][j] = win[k + 1][j];
    }
    const float zero[V] = {};
    for (; t < t1; ++t) store_some<V>(py + t * D, n, zero);
}

template <typename T, int K, bool SILU>
__global__ __launch_bounds__(kBlock) void conv_step_kernel(
    const T* __restrict__ x, int64_t ld, const float* __restrict__ w,
    const float* __restrict__ bias, T* __restrict__ state, T* __restrict__ y, int64_t B, int64_t D)
{
    const int64_t id = int64_t(blockIdx.x) * kBlock + threadIdx.x;
    const int64_t b = id / D, c = id - b * D;
    if (b >= B) return;
    T* ps = state + b * (K - 1) * D + c;
    float win[K];
#pragma unroll
    for (int k = 0; k < K - 1; ++k) win[k] = io_load(ps + k * D);
    win[K - 1] = io_load(x + b * ld + c);
    float o = bias ? bias[c] : 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) o = fmaf(w[c * K + k], win[k], o);
    if constexpr (SILU) o *= sigmoid(o);
    io_store(y + b * D + c, o);
#pragma unroll
    for (int k = 0; k < K - 1; ++k) io_store(ps + k * D, win[k + 1]);
}

// A workgroup: 64 pieces of channels x 4 runs, whose sums are added in LDS.
template <typename T, int K, bool SILU>
__global__ __launch_bounds__(kBlock) void conv_grad_kernel(
    const T* __restrict__ dy, const T* __restrict__ x, int64_t ld, const float* __restrict__ w,
    const float* __restrict__ bias, const int* __restrict__ lengths, T* __restrict__ dx,
    float* __restrict__ part, int64_t B, int64_t T_, int64_t D, int64_t run, int64_t runs)
{
    constexpr int V = kChan<T, K>;
    constexpr int kRuns = kBlock / kWave;
    __shared__ float sums[kRuns][V][kWave];
    const int64_t tiles = ((D + V - 1) / V + kWave - 1) / kWave;
    const int lane = threadIdx.x & (kWave - 1), sub = threadIdx.x / kWave;
    const int64_t tile = blockIdx.x % tiles, group = blockIdx.x / tiles;
    const int64_t row = group * kRuns + sub;
    const int64_t c = (tile * kWave + lane) * V;
    float aw[K][V], ab[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        ab[j] = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) aw[k][j] = 0.f;
    }
    if (row < B * runs && c < D) {
        const int n = int(D - c < V ? D - c : V);
        const int64_t b = row / runs, t0 = (row - b * runs) * run;
        const int64_t len = length_of(lengths, b, T_);
        const int64_t t1 = t0 + run < T_ ? t0 + run : T_;
        const T* px = x + b * T_ * ld + c;
        const T* pg = dy + b * T_ * D + c;
        T* pd = dx + b * T_ * D + c;
        float wv[K][V], bv[V], win[K][V], g[K][V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int64_t cj = c + (j < n ? j : 0);
            bv[j] = bias ? bias[cj] : 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                wv[k][j] = w[cj * K + k];
                win[k][j] = g[k][j] = 0.f;
            }
        }
#pragma unroll
        for (int k = 0; k < K - 1; ++k) {
            const int64_t t = t0 - (K - 1) + k;
            if (t >= 0 && t < len) load_some<V>(px + t * ld, n, win[k]);
        }
        // g[k] = g_(t - K + 1 + k); dx_(t - K + 1) leaves at step t.  The run's own steps
        // feed dw and dbias, the K - 1 after it only its last dx.
        const int64_t te = t1 < len ? t1 : len;
        for (int64_t t = t0; t < te + K - 1; ++t) {
            if (t < len) {
                load_some<V>(px + t * ld, n, win[K - 1]);
                load_some<V>(pg + t * D, n, g[K - 1]);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    if constexpr (SILU) {
                        float o = bv[j];
#pragma unroll
                        for (int k = 0; k < K; ++k) o = fmaf(wv[k][j], win[k][j], o);
                        const float p = sigmoid(o);
                        g[K - 1][j] *= p * fmaf(o, 1.f - p, 1.f);
                    }
                    if (t < te) {
                        ab[j] += g[K - 1][j];
#pragma unroll
                        for (int k = 0; k < K; ++k)
                            aw[k][j] = fmaf(g[K - 1][j], win[k][j], aw[k][j]);
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) g[K - 1][j] = 0.f;
            }
            if (t - (K - 1) >= t0) {
                // w[K - 1] meets the output of its own step, w[0] the one K - 1 later
                float d[V];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    d[j] = 0.f;
#pragma unroll
                    for (int k = 0; k < K; ++k) d[j] = fmaf(wv[K - 1 - k][j], g[k][j], d[j]);
                }
                store_some<V>(pd + (t - (K - 1)) * D, n, d);
            }
#pragma unroll
            for (int k = 0; k < K - 1; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    win[k][j] = win[k + 1][j];
                    g[k][j] = g[k + 1][j];
                }
        }
        const float zero[V] = {};
        for (int64_t t = te > t0 ? te : t0; t < t1; ++t) store_some<V>(pd + t * D, n, zero);
    }
    // partial row [D K | D] of this workgroup
    float* out = part + group * (K + 1) * D;
#pragma unroll
    for (int k = 0; k <= K; ++k) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < V; ++j) sums[sub][j][lane] = k < K ? aw[k < K ? k : 0][j] : ab[j];
        __syncthreads();
        for (int i = threadIdx.x; i < V * kWave; i += kBlock) {
            const int j = i / kWave, l = i % kWave;
            const int64_t cj = (tile * kWave + l) * V + j;
            float s = 0.f;
#pragma unroll
            for (int q = 0; q < kRuns; ++q) s += sums[q][j][l];
            if (cj < D) out[k < K ? cj * K + k : D * K + cj] = s;
        }
    }
}

// Time steps per run: as many as leave kThreads threads, 4 to 64.
int64_t run_length(int64_t B, int64_t T, int64_t cols)
{
    int64_t run = 64;
    while (run > 4 && B * ((T + run - 1) / run) * cols < kThreads) run /= 2;
    return run;
}

struct GradShape {
    int64_t run, runs, groups, tiles;
};
GradShape grad_shape(int64_t B, int64_t T, int64_t D, int V)
{
    GradShape s;
    const int64_t cols = (D + V - 1) / V;
    s.run = run_length(B, T, cols);
    s.runs = (T + s.run - 1) / s.run;
    s.groups = (B * s.runs + 3) / 4;
    s.tiles = (cols + kWave - 1) / kWave;
    return s;
}

template <typename F>
hipError_t with_taps(int64_t K, F f)
{
    switch (K) {
        case 1: return f(std::integral_constant<int, 1>());
        case 2: return f(std::integral_constant<int, 2>());
        case 3: return f(std::integral_constant<int, 3>());
        case 4: return f(std::integral_constant<int, 4>());
        case 5: return f(std::integral_constant<int, 5>());
        case 6: return f(std::integral_constant<int, 6>());
        case 7: return f(std::integral_constant<int, 7>());
        default: return f(std::integral_constant<int, 8>());
    }
}

template <typename F>
hipError_t with_type(bool bf16_io, bool silu, F f)
{
    if (bf16_io) return silu ? f(bf16(), std::true_type()) : f(bf16(), std::false_type());
    return silu ? f(float(), std::true_type()) : f(float(), std::false_type());
}

}  // namespace

int64_t short_conv_threads(int64_t B, int64_t T, int64_t D, int64_t K)
{
    int64_t most = B * D;  // a step
    most = 16 * D * (K + 1) > most ? 16 * D * (K + 1) : most;  // column sums
    for (int V : {2, 4, 8}) {
        const int64_t cols = (D + V - 1) / V, run = run_length(B, T, cols);
        const int64_t n = B * (T > 0 ? (T + run - 1) / run : 1) * cols + kBlock;
        most = n > most ? n : most;
        const GradShape s = grad_shape(B, T, D, V);
        const int64_t m = s.groups * s.tiles * kBlock;
        most = m > most ? m : most;
    }
    return most + kBlock;
}

hipError_t launch_short_conv(const void* x, int64_t ld, const float* w, const float* bias,
                             const int* lengths, void* state, bool resume, void* y, bool bf16_io,
                             bool silu, int64_t B, int64_t T, int64_t D, int64_t K,
                             hipStream_t stream)
{
    return with_type(bf16_io, silu, [&](auto type, auto act) {
        using E = decltype(type);
        constexpr bool S = decltype(act)::value;
        return with_taps(K, [&](auto taps) {
            constexpr int KK = decltype(taps)::value;
            constexpr int V = kChan<E, KK>;
            const int64_t cols = (D + V - 1) / V;
            const int64_t run = run_length(B, T, cols);
            const int64_t runs = T > 0 ? (T + run - 1) / run : 1;
            const int64_t blocks = (B * runs * cols + kBlock - 1) / kBlock;
            hipLaunchKernelGGL((conv_kernel<E, KK, S>), dim3(uint32_t(blocks)), dim3(kBlock), 0,
                               stream, static_cast<const E*>(x), ld, w, bias, lengths,
                               static_cast<E*>(state), resume, static_cast<E*>(y), B, T, D, run,
                               runs);
            return hipGetLastError();
        });
    });
}

hipError_t launch_short_conv_step(const void* x, int64_t ld, const float* w, const float* bias,
                                  void* state, void* y, bool bf16_io, bool silu, int64_t B,
                                  int64_t D, int64_t K, hipStream_t stream)
{
    return with_type(bf16_io, silu, [&](auto type, auto act) {
        using E = decltype(type);
        constexpr bool S = decltype(act)::value;
        return with_taps(K, [&](auto taps) {
            constexpr int KK = decltype(taps)::value;
            hipLaunchKernelGGL((conv_step_kernel<E, KK, S>),
                               dim3(uint32_t((B * D + kBlock - 1) / kBlock)), dim3(kBlock), 0,
                               stream, static_cast<const E*>(x), ld, w, bias,
                               static_cast<E*>(state), static_cast<E*>(y), B, D);
            return hipGetLastError();
        });
    });
}

size_t short_conv_grad_workspace_bytes(int64_t B, int64_t T, int64_t D, int64_t K)
{
    // the wider of the two types' partial rows (pieces of 2 to 8 channels)
    int64_t groups = 0;
    for (int V : {2, 4, 8}) {
        const GradShape s = grad_shape(B, T, D, V);
        groups = s.groups > groups ? s.groups : groups;
    }
    return sizeof(float) * size_t(groups) * (K + 1) * D;
}

hipError_t launch_short_conv_grad(const void* dy, const void* x, int64_t ld, const float* w,
                                  const float* bias, const int* lengths, void* dx, float* dw,
                                  float* dbias, bool bf16_io, bool silu, int64_t B, int64_t T,
                                  int64_t D, int64_t K, void* workspace, hipStream_t stream)
{
    float* part = static_cast<float*>(workspace);
    int64_t groups = 0;
    const hipError_t e = with_type(bf16_io, silu, [&](auto type, auto act) {
        using E = decltype(type);
        constexpr bool S = decltype(act)::value;
        return with_taps(K, [&](auto taps) {
            constexpr int KK = decltype(taps)::value;
            const GradShape s = grad_shape(B, T, D, kChan<E, KK>);
            groups = s.groups;
            if (s.groups == 0) return hipSuccess;
            hipLaunchKernelGGL((conv_grad_kernel<E, KK, S>), dim3(uint32_t(s.groups * s.tiles)),
                               dim3(kBlock), 0, stream, static_cast<const E*>(dy),
                               static_cast<const E*>(x), ld, w, bias, lengths,
                               static_cast<E*>(dx), part, B, T, D, s.run, s.runs);
            return hipGetLastError();
        });
    });
    if (e != hipSuccess) return e;
    return launch_column_sum(part, groups, D * K, dw, D, dbias, 0, nullptr, stream);
}

}  // namespace lh
