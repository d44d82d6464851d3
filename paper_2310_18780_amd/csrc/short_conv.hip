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
// leaves the GPU a wavefront per SIMD, and the inputs of the next four steps are in
// flight while four are computed: 64 x 4096 x 2048 bfloat16 in 426 us (5.0 TB/s, the
// rate of a copy; 463 us with each step's input waited for).
//
// The gradient walks the same way: o_t and g_t at the front, dx K - 1 steps behind.
// A run's sums for dw and dbias stay in registers; the workgroup's runs over the
// same channels are added in LDS, and a second launch adds the workgroups' rows in a
// fixed order (16 x 2048 x 768 float32, rows 2 x 768 apart: 71 us for 302 MB, 84 us
// without the inputs ahead; 57 us where the call before read the same inputs, part of which
// then lie in the 256 MB cache; 64 x 2048 x 2048 bfloat16 361 us, 4.5 TB/s, against 554).
#include "short_conv.hpp"

#include "block_ops.hpp"

namespace lh {
namespace {

constexpr int kBlock = 256;
constexpr int64_t kThreads = 1 << 16;  // one wavefront per SIMD

constexpr int kAhead = 4;  // steps whose inputs are in flight while as many are computed

// Channels per thread: 16 bytes, half of that for long filters (registers); one where
// the width is less.
template <typename T, int K>
constexpr int kChan = K <= 4 ? kVec<T> : kVec<T> / 2;

__device__ __forceinline__ int64_t length_of(const int* lengths, int64_t b, int64_t T)
{
    if (!lengths) return T;
    const int64_t n = lengths[b];
    return n < 0 ? 0 : n < T ? n : T;
}

// The values of a piece but the first `twice`.
template <int V, typename T>
__device__ __forceinline__ void put_from(T* p, const float (&v)[V], int twice)
{
    if (twice == 0) {
        put<V>(p, v);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j >= twice) io_store(p + j, v[j]);
    }
}

// The filter of V channels from c: w[k], K taps, and the bias.
template <int V, int K>
__device__ __forceinline__ void load_filter(const float* w, const float* bias, int64_t c,
                                            float (&wv)[K][V], float (&bv)[V])
{
#pragma unroll
    for (int j = 0; j < V; ++j) {
        bv[j] = bias ? bias[c + j] : 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) wv[k][j] = w[(c + j) * K + k];
    }
}

// The input of step t of a row, or of the state where t < 0 (zero without one): where it
// lies, and whether it is there.  No load is under a branch; one that is not there reads
// another place and is replaced by zero.
template <typename T, int K>
__device__ __forceinline__ const T* place_of(int64_t t, const T* px, int64_t ld, const T* ps,
                                             int64_t D, bool resume, bool* there)
{
    *there = t >= 0 || resume;
    return t >= 0 ? px + t * ld : ps + (resume ? t + K - 1 : 0) * D;
}

template <typename T, int K, int V, bool SILU>
__global__ __launch_bounds__(kBlock) void conv_kernel(
    const T* __restrict__ x, int64_t ld, const float* __restrict__ w,
    const float* __restrict__ bias, const int* __restrict__ lengths, T* state, bool resume,
    T* __restrict__ y, int64_t B, int64_t T_, int64_t D, int64_t run, int64_t runs)
{
    const int64_t cols = (D + V - 1) / V;
    const int64_t id = int64_t(blockIdx.x) * kBlock + threadIdx.x;
    const int64_t row = id / cols;
    if (row >= B * runs) return;
    // The last piece ends with the row.  The channels it shares with the one before are
    // that one's to store (whose thread may have written their new state already).
    const int64_t at = (id - row * cols) * V, c = at < D - V ? at : D - V;
    const int twice = int(at - c);
    const int64_t b = row / runs, r = row - b * runs;
    const int64_t len = length_of(lengths, b, T_);
    const int64_t t0 = r * run, t1 = t0 + run < T_ ? t0 + run : T_, te = t1 < len ? t1 : len;
    const T* px = x + b * T_ * ld + c;
    T* py = y + b * T_ * D + c;
    T* ps = state + b * (K - 1) * D + c;

    Raw<T, V> head[K], tail[K], next[kAhead];
    bool in_head[K], in_tail[K];
    if (t0 < te) {
#pragma unroll
        for (int k = 0; k < K - 1; ++k)
            head[k] = load_raw<V>(place_of<T, K>(t0 - (K - 1) + k, px, ld, ps, D, resume, &in_head[k]));
#pragma unroll
        for (int i = 0; i < kAhead; ++i) next[i] = load_raw<V>(px + (t0 + i < te ? t0 + i : te - 1) * ld);
    }
    float wv[K][V], bv[V];
    load_filter<V, K>(w, bias, c, wv, bv);
    if (K > 1 && r == 0) {
        // The state after the row's last token.  Only the first runs of a row read the old
        // one, above and here where the row is shorter than the state.
#pragma unroll
        for (int k = 0; k < K - 1; ++k)
            tail[k] = load_raw<V>(place_of<T, K>(len - (K - 1) + k, px, ld, ps, D, resume, &in_tail[k]));
    }
    float win[K][V];  // win[k] = x_(t - K + 1 + k)
    if (t0 < te) {
#pragma unroll
        for (int k = 0; k < K - 1; ++k) {
            expand<V, T>(head[k], win[k]);
#pragma unroll
            for (int j = 0; j < V; ++j) win[k][j] = in_head[k] ? win[k][j] : 0.f;
        }
    }
    if (K > 1 && r == 0) {
#pragma unroll
        for (int k = 0; k < K - 1; ++k) {
            float v[V];
            expand<V, T>(tail[k], v);
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = in_tail[k] ? v[j] : 0.f;
            put_from<V>(ps + k * D, v, twice);
        }
    }
    // kAhead steps at a time, the next ones in flight
    for (int64_t t = t0; t < te; t += kAhead) {
        Raw<T, V> now[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            now[i] = next[i];
            const int64_t ahead = t + kAhead + i;
            next[i] = load_raw<V>(px + (ahead < te ? ahead : te - 1) * ld);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            expand<V, T>(now[i], win[K - 1]);
            float o[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                o[j] = bv[j];
#pragma unroll
                for (int k = 0; k < K; ++k) o[j] = fmaf(wv[k][j], win[k][j], o[j]);
                if constexpr (SILU) o[j] *= sigmoid(o[j]);
            }
            if (t + i < te) put_from<V>(py + (t + i) * D, o, twice);
#pragma unroll
            for (int k = 0; k < K - 1; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) win[k][j] = win[k + 1][j];
        }
    }
    const float zero[V] = {};
    for (int64_t t = te > t0 ? te : t0; t < t1; ++t) put<V>(py + t * D, zero);
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
template <typename T, int K, int V, bool SILU>
__global__ __launch_bounds__(kBlock) void conv_grad_kernel(
    const T* __restrict__ dy, const T* __restrict__ x, int64_t ld, const float* __restrict__ w,
    const float* __restrict__ bias, const int* __restrict__ lengths, T* __restrict__ dx,
    float* __restrict__ part, int64_t B, int64_t T_, int64_t D, int64_t run, int64_t runs)
{
    constexpr int kRuns = kBlock / kWave;
    __shared__ float sums[kRuns][V][kWave];
    const int64_t tiles = ((D + V - 1) / V + kWave - 1) / kWave;
    const int lane = threadIdx.x & (kWave - 1), sub = threadIdx.x / kWave;
    const int64_t tile = blockIdx.x % tiles, group = blockIdx.x / tiles;
    const int64_t row = group * kRuns + sub;
    // (the last piece ends with the row: the channels it shares with the one before count
    // there)
    const int64_t at = (tile * kWave + lane) * V, c = at < D - V ? at : D - V;
    const int twice = int(at - c < V ? at - c : V);
    float aw[K][V], ab[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        ab[j] = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) aw[k][j] = 0.f;
    }
    if (row < B * runs && at < D) {
        const int64_t b = row / runs, t0 = (row - b * runs) * run;
        const int64_t len = length_of(lengths, b, T_);
        const int64_t t1 = t0 + run < T_ ? t0 + run : T_, te = t1 < len ? t1 : len;
        const T* px = x + b * T_ * ld + c;
        const T* pg = dy + b * T_ * D + c;
        T* pd = dx + b * T_ * D + c;
        if (t0 < te) {
            Raw<T, V> head[K], nx[kAhead], ng[kAhead];
#pragma unroll
            for (int k = 0; k < K - 1; ++k) {
                const int64_t t = t0 - (K - 1) + k;
                head[k] = load_raw<V>(px + (t > 0 ? t : 0) * ld);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int64_t t = t0 + i < len ? t0 + i : len - 1;
                nx[i] = load_raw<V>(px + t * ld);
                ng[i] = load_raw<V>(pg + t * D);
            }
            float wv[K][V], bv[V], win[K][V], g[K][V];
            load_filter<V, K>(w, bias, c, wv, bv);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (k < K - 1) expand<V, T>(head[k], win[k]);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    if (k < K - 1) win[k][j] = t0 - (K - 1) + k >= 0 ? win[k][j] : 0.f;
                    g[k][j] = 0.f;
                }
            }
            // g[k] = g_(t - K + 1 + k); dx_(t - K + 1) leaves at step t.  The run's own
            // steps feed dw and dbias, the K - 1 after it only its last dx.
            for (int64_t t = t0; t < te + K - 1; t += kAhead) {
                Raw<T, V> rx[kAhead], rg[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    rx[i] = nx[i];
                    rg[i] = ng[i];
                    const int64_t ahead = t + kAhead + i < len ? t + kAhead + i : len - 1;
                    nx[i] = load_raw<V>(px + ahead * ld);
                    ng[i] = load_raw<V>(pg + ahead * D);
                }
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const int64_t now = t + i;
                    expand<V, T>(rx[i], win[K - 1]);
                    expand<V, T>(rg[i], g[K - 1]);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        if constexpr (SILU) {
                            float o = bv[j];
#pragma unroll
                            for (int k = 0; k < K; ++k) o = fmaf(wv[k][j], win[k][j], o);
                            const float p = sigmoid(o);
                            g[K - 1][j] *= p * fmaf(o, 1.f - p, 1.f);
                        }
                        g[K - 1][j] = now < len ? g[K - 1][j] : 0.f;
                    }
                    if (now < te) {
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            ab[j] += g[K - 1][j];
#pragma unroll
                            for (int k = 0; k < K; ++k)
                                aw[k][j] = fmaf(g[K - 1][j], win[k][j], aw[k][j]);
                        }
                    }
                    if (now - (K - 1) >= t0 && now - (K - 1) < te) {
                        // w[K - 1] meets the output of its own step, w[0] the one K - 1 later
                        float d[V];
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            d[j] = 0.f;
#pragma unroll
                            for (int k = 0; k < K; ++k) d[j] = fmaf(wv[K - 1 - k][j], g[k][j], d[j]);
                        }
                        put<V>(pd + (now - (K - 1)) * D, d);
                    }
#pragma unroll
                    for (int k = 0; k < K - 1; ++k)
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            win[k][j] = win[k + 1][j];
                            g[k][j] = g[k + 1][j];
                        }
                }
            }
        }
        const float zero[V] = {};
        for (int64_t t = te > t0 ? te : t0; t < t1; ++t) put<V>(pd + t * D, zero);
    }
    // partial row [D K | D] of this workgroup
    float* out = part + group * (K + 1) * D;
#pragma unroll
    for (int k = 0; k <= K; ++k) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < V; ++j) sums[sub][j][lane] = k < K ? aw[k < K ? k : 0][j] : ab[j];
        __syncthreads();
        for (int j = sub; j < V; j += kRuns) {  // (this thread's lane: the same piece)
            float s = 0.f;
#pragma unroll
            for (int q = 0; q < kRuns; ++q) s += sums[q][j][lane];
            if (at < D && j >= twice) out[k < K ? (c + j) * K + k : D * K + c + j] = s;
        }
    }
}

// Time steps per run: as many as leave kThreads threads, 4 to 64, and not fewer than the
// inputs before a run: only the first run of a row may reach back to the state, which its
// thread replaces.
int64_t run_length(int64_t B, int64_t T, int64_t cols, int64_t K)
{
    const int64_t least = K <= 5 ? 4 : 8;
    int64_t run = 64;
    while (run > least && B * ((T + run - 1) / run) * cols < kThreads) run /= 2;
    return run;
}

struct GradShape {
    int64_t run, runs, groups, tiles;
};
GradShape grad_shape(int64_t B, int64_t T, int64_t D, int64_t K, int V)
{
    // Runs of up to 64 steps: 64 where that leaves three workgroups to a CU, else the
    // longest up to 32 that leaves one (on the inputs of the call before, 16 x 2048 x 768:
    // float32 runs of 32 and 64 steps 58 and 60 us; 2 x 2048 x 2048 bfloat16 runs of 16 and 8
    // steps 24 and 27 us).
    const int64_t cols = (D + V - 1) / V, least = K <= 5 ? 4 : 8;
    GradShape s;
    s.tiles = (cols + kWave - 1) / kWave;
    for (s.run = 64;; s.run /= 2) {
        s.runs = (T + s.run - 1) / s.run;
        s.groups = (B * s.runs + 3) / 4;
        if (s.run <= least || s.groups * s.tiles >= (s.run == 64 ? 768 : 256)) break;
    }
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
    most = 32 * D * (K + 1) > most ? 32 * D * (K + 1) : most;  // column sums
    for (int V : {1, 2, 4, 8}) {
        const int64_t cols = (D + V - 1) / V, run = run_length(B, T, cols, K);
        const int64_t n = B * (T > 0 ? (T + run - 1) / run : 1) * cols + kBlock;
        most = n > most ? n : most;
        const GradShape s = grad_shape(B, T, D, K, V);
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
            const bool whole = D >= V;
            const int64_t cols = whole ? (D + V - 1) / V : D;
            const int64_t run = run_length(B, T, cols, K);
            const int64_t runs = T > 0 ? (T + run - 1) / run : 1;
            const int64_t blocks = (B * runs * cols + kBlock - 1) / kBlock;
            const auto kernel = whole ? conv_kernel<E, KK, V, S> : conv_kernel<E, KK, 1, S>;
            hipLaunchKernelGGL(kernel, dim3(uint32_t(blocks)), dim3(kBlock), 0, stream,
                               static_cast<const E*>(x), ld, w, bias, lengths,
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
    // the wider of the two types' partial rows (pieces of 1 to 8 channels)
    int64_t groups = 0;
    for (int V : {1, 2, 4, 8}) {
        const GradShape s = grad_shape(B, T, D, K, V);
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
            constexpr int V = kChan<E, KK>;
            const GradShape s = grad_shape(B, T, D, K, D >= V ? V : 1);
            groups = s.groups;
            if (s.groups == 0) return hipSuccess;
            const auto kernel = D >= V ? conv_grad_kernel<E, KK, V, S> : conv_grad_kernel<E, KK, 1, S>;
            hipLaunchKernelGGL(kernel, dim3(uint32_t(s.groups * s.tiles)), dim3(kBlock), 0, stream,
                               static_cast<const E*>(dy),
                               static_cast<const E*>(x), ld, w, bias, lengths,
                               static_cast<E*>(dx), part, B, T, D, s.run, s.runs);
            return hipGetLastError();
        });
    });
    if (e != hipSuccess) return e;
    return launch_column_sum(part, groups, D * K, dw, D, dbias, 0, nullptr, stream);
}

}  // namespace lh
