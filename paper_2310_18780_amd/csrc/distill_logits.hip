// Distillation from a teacher's top logits, loss and gradient:
//
//   p = softmax(values / tau) over the row's slots,  q = softmax(logits / tau)
//   loss = scale tau^2 sum_k p_k (log p_k - log q[id_k])
//   dlogits[j] = scale tau (q[j] - sum of p_k with id_k = j)
//
// Bound by memory: a row of logits is read once, and written once for the gradient, beside one
// exponential a value for each.  A workgroup of 4 or 16 wavefronts holds its row in registers
// as it lies in memory, so that the largest value is known before the exponentials and they are
// formed again for the gradient without a second read; rows that no workgroup holds are
// read once more for each.
//
// The slots lie in LDS.  The dense gradient is stored first; then each slot's thread stores its
// own value over it, all slots of that id subtracted in their order (an id given twice has the
// same bits from both).
#include "distill_logits.hpp"

#include "block_ops.hpp"
#include "lh.h"

namespace lh {
namespace {

constexpr int64_t kMaxBlocks = 1 << 20;  // grid-stride beyond
constexpr int kHold = 16;  // pieces of a row that a thread holds

constexpr float kNone = -__builtin_inff();

__device__ __forceinline__ float wave_max(float v)
{
    for (int o = 1; o < kWave; o *= 2) v = fmaxf(v, __shfl_xor(v, o, kWave));
    return v;
}

template <typename T>
struct Args {
    const T* logits;
    int64_t ld;
    const float* values;
    const int* ids;
    const float* scale;
    int64_t rows, V;
    int K;
    float tau, to2;  // to2 = log2(e) / tau
    float *loss, *lse_out;
    const float *dloss, *lse_in;
    T* dlogits;
    int64_t ld_d;
};

// A row's pieces: the whole ones of a thread from registers (ITER > 0) or memory.
// MODE 0: loss; 1: loss and gradient; 2: gradient from lse.
template <typename T, int BLOCK, int ITER, int MODE>
__global__ __launch_bounds__(BLOCK) void distill_kernel(Args<T> a)
{
    constexpr int V = kVec<T>;
    constexpr int waves = BLOCK / kWave;
    __shared__ float2 red[2][waves];
    __shared__ float reds[waves];
    __shared__ float2 slots[LH_DISTILL_MAX_TOP];  // id (bits), p
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int64_t pieces = a.V / V, tail = a.V % V;  // whole pieces, then single values
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* x = a.logits + row * a.ld;
        T* out = MODE ? a.dlogits + row * a.ld_d : nullptr;
        const float scale = a.scale ? a.scale[row] : 1.f;
        // the teacher's side: one slot to a thread (K <= 1024, four to a thread of 256)
        constexpr int S = LH_DISTILL_MAX_TOP / BLOCK;
        float t[S];
        int id[S];
        float top_t = kNone;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const int k = threadIdx.x + i * BLOCK;
            t[i] = kNone;
            id[i] = -1;
            if (k < a.K) {
                id[i] = a.ids[row * a.K + k];
                const float v = a.values[row * a.K + k];
                // (NaN as infinity, which the maximum does not drop: the row is NaN)
                if (id[i] >= 0 && id[i] < a.V) t[i] = v != v ? -kNone : v;
            }
            top_t = fmaxf(top_t, t[i]);
        }
        // the student's: pieces and values past the last whole piece
        Raw<T, V> raw[ITER > 0 ? ITER : 1];
        float last = kNone, top = kNone;
        auto each = [&](auto f) {
            if constexpr (ITER > 0) {
#pragma unroll
                for (int i = 0; i < ITER; ++i) {
                    const int64_t p = i * BLOCK + threadIdx.x;
                    if (p < pieces) f(raw[i], p);
                }
            } else {
                for (int64_t p = threadIdx.x; p < pieces; p += BLOCK) f(load_raw<V>(x + p * V), p);
            }
        };
        if (scale != 0.f) {
            if constexpr (ITER > 0) {
#pragma unroll
                for (int i = 0; i < ITER; ++i) {
                    const int64_t p = i * BLOCK + threadIdx.x;
                    if (p < pieces) raw[i] = load_raw<V>(x + p * V);
                }
            }
            if (threadIdx.x < tail) last = io_load(x + pieces * V + threadIdx.x);
            if constexpr (MODE < 2) {
                top = last;
                each([&](const Raw<T, V>& r, int64_t) {
                    float v[V];
                    expand<V, T>(r, v);
#pragma unroll
                    for (int j = 0; j < V; ++j) top = fmaxf(top, v[j]);
                });
            }
        }
        top = wave_max(top);
        top_t = wave_max(top_t);
        __syncthreads();  // (the row before has been read from LDS)
        if (lane == 0) red[0][wave] = make_float2(top, top_t);
        __syncthreads();
#pragma unroll
        for (int w = 0; w < waves; ++w) {
            const float2 v = red[0][w];
            top = fmaxf(top, v.x);
            top_t = fmaxf(top_t, v.y);
        }
        const bool none = scale == 0.f || top_t == kNone;
        if (none) {  // no slots, or a row that takes no part
            if (threadIdx.x == 0) {
                if (MODE < 2) a.loss[row] = 0.f;
                if (MODE < 2 && a.lse_out) a.lse_out[row] = 0.f;
            }
            if constexpr (MODE > 0)
                for (int64_t j = threadIdx.x; j < a.V; j += BLOCK) io_store(out + j, 0.f);
            continue;
        }
        // exponents in base 2: less the row's largest (a difference first: the rounding of a
        // product of a large offset would not cancel), or less lse
        float off = MODE == 2 ? a.lse_in[row] * kLog2e : top;
        if (off == kNone) off = 0.f;
        auto power = [&](float v) { return MODE == 2 ? fmaf(v, a.to2, -off) : (v - off) * a.to2; };
        float2 sum = make_float2(0.f, 0.f);  // of the student's exponentials, of the teacher's
        float cross = 0.f, e[S], own[S];
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const float d = (t[i] - top_t) * a.to2;
            e[i] = t[i] == kNone ? 0.f : exp2_fast(d);
            own[i] = e[i] != 0.f ? power(io_load(x + id[i])) : 0.f;
            sum.y += e[i];
            cross += e[i] != 0.f ? e[i] * (d - own[i]) : 0.f;
        }
        if constexpr (MODE < 2) {
            if (threadIdx.x < tail) sum.x = exp2_fast(power(last));
            each([&](const Raw<T, V>& r, int64_t) {
                float v[V];
                expand<V, T>(r, v);
#pragma unroll
                for (int j = 0; j < V; ++j) sum.x += exp2_fast(power(v[j]));
            });
            cross = wave_sum(cross);
            sum.x = wave_sum(sum.x);
        }
        sum.y = wave_sum(sum.y);
        if (lane == 0) {
            red[1][wave] = sum;
            reds[wave] = cross;
        }
        __syncthreads();
        sum = make_float2(0.f, 0.f);
        cross = 0.f;
#pragma unroll
        for (int w = 0; w < waves; ++w) {
            sum.x += red[1][w].x;
            sum.y += red[1][w].y;
            cross += reds[w];
        }
        if (MODE < 2 && threadIdx.x == 0) {
            const float l2 = __builtin_amdgcn_logf(sum.x);
            // (no finite logit: the student's probabilities are 0)
            const float nats = sum.x == 0.f ? __builtin_inff()
                                            : kLn2 * (cross / sum.y + (l2 - __builtin_amdgcn_logf(sum.y)));
            a.loss[row] = scale * a.tau * a.tau * nats;
            if (a.lse_out) a.lse_out[row] = fmaf(kLn2, l2, top == kNone ? kNone : top / a.tau);
        }
        if constexpr (MODE > 0) {
            float c = scale * a.tau;
            if (MODE == 2) c *= a.dloss[row];
            const float cq = MODE == 2 ? c : sum.x == 0.f ? 0.f : c / sum.x;
            const float rp = 1.f / sum.y;
#pragma unroll
            for (int i = 0; i < S; ++i) {
                const int k = threadIdx.x + i * BLOCK;
                if (k < a.K) slots[k] = make_float2(__int_as_float(t[i] == kNone ? -1 : id[i]), e[i] * rp);
            }
            each([&](const Raw<T, V>& r, int64_t p) {
                float v[V];
                expand<V, T>(r, v);
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = exp2_fast(power(v[j])) * cq;
                put<V>(out + p * V, v);
            });
            if (threadIdx.x < tail)
                io_store(out + pieces * V + threadIdx.x, exp2_fast(power(last)) * cq);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < S; ++i) {
                if (e[i] == 0.f) continue;
                float p = 0.f;
                for (int k = 0; k < a.K; ++k) {
                    const float2 s = slots[k];
                    p += __float_as_int(s.x) == id[i] ? s.y : 0.f;
                }
                io_store(out + id[i], fmaf(exp2_fast(own[i]), cq, -c * p));
            }
        }
    }
}

// Threads to a row and pieces of a thread (0: read again from memory).
template <int MODE, typename T, typename F>
hipError_t with_shape(int64_t V, F f)
{
    const int64_t pieces = V / kVec<T>;
    auto iters = [&](auto block) {
        constexpr int B = decltype(block)::value;
        const int64_t n = (pieces + B - 1) / B;
        if (n <= 1) return f(block, std::integral_constant<int, 1>());
        if (n <= 2) return f(block, std::integral_constant<int, 2>());
        if (n <= 4) return f(block, std::integral_constant<int, 4>());
        if (n <= 8) return f(block, std::integral_constant<int, 8>());
        if constexpr (B == 1024)
            if (n <= kHold) return f(block, std::integral_constant<int, kHold>());
        return f(block, std::integral_constant<int, 0>());
    };
    if (pieces <= 4 * 256) return iters(std::integral_constant<int, 256>());
    return iters(std::integral_constant<int, 1024>());
}

template <typename T, int MODE>
hipError_t distill(const DistillLogits& d, float* loss, float* lse, const float* dloss, hipStream_t stream)
{
    if (d.rows == 0) return hipSuccess;
    Args<T> a;
    a.logits = static_cast<const T*>(d.logits), a.ld = d.ld, a.values = d.values, a.ids = d.ids;
    a.scale = d.scale, a.rows = d.rows, a.V = d.V, a.K = d.K, a.tau = d.tau, a.to2 = kLog2e / d.tau;
    a.loss = loss, a.lse_out = lse, a.dloss = dloss, a.lse_in = lse;
    a.dlogits = static_cast<T*>(d.dlogits), a.ld_d = d.ld_d;
    return with_shape<MODE, T>(d.V, [&](auto block, auto iter) {
        constexpr int B = decltype(block)::value, ITER = decltype(iter)::value;
        hipLaunchKernelGGL((distill_kernel<T, B, ITER, MODE>),
                           dim3(uint32_t(d.rows < kMaxBlocks ? d.rows : kMaxBlocks)), dim3(B), 0, stream, a);
        return hipGetLastError();
    });
}

}  // namespace

size_t distill_logits_workspace_bytes(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_distill_logits(const DistillLogits& a, float* loss, float* lse, void*, hipStream_t stream)
{
    if (a.bf16_io)
        return a.dlogits ? distill<bf16, 1>(a, loss, lse, nullptr, stream) : distill<bf16, 0>(a, loss, lse, nullptr, stream);
    return a.dlogits ? distill<float, 1>(a, loss, lse, nullptr, stream) : distill<float, 0>(a, loss, lse, nullptr, stream);
}

hipError_t launch_distill_logits_grad(const DistillLogits& a, const float* dloss, const float* lse, hipStream_t stream)
{
    float* l = const_cast<float*>(lse);
    if (a.bf16_io) return distill<bf16, 2>(a, nullptr, l, dloss, stream);
    return distill<float, 2>(a, nullptr, l, dloss, stream);
}

}  // namespace lh
