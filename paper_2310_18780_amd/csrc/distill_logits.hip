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
// read once more for each.  8192 rows of 50000 bfloat16 with 64 slots, loss and gradient, 15% of
// them without a loss: 292 us, 1.51 GB at a copy's rate (vector issue 0.58 of the time beside it).
// With values expanded in registers, a row to a CU, it took 604.  517 x 32003 float32: loss 17 us,
// gradient 20 (66 and 132 MB, the second read from the cache in part).
//
// The slots lie in LDS.  The dense gradient is stored first; then each slot's thread stores its
// own value over it, all slots of that id subtracted in their order (an id given twice has the
// same bits from both).
//
// A float32 lse is off by up to 2^-24 of its size, and so is every exponent that it is subtracted
// from.  The gradient from lse takes it as it is up to kNear, where that is no more than the
// exponentials' own rounding; where it lies farther out (logits with a large offset) the row's
// largest value and its sum are formed again, as for the loss (q was off by 7e-4 at logits of 10^4).
// 517 x 32003 float32: 27.8 us near and 30.4 far, 1789 x 80479, read again for each, 244 and 342.
#include "distill_logits.hpp"

#include "block_ops.hpp"
#include "lh.h"

namespace lh {
namespace {

constexpr int kHold = 16;  // pieces of a row that a thread holds

constexpr float kNone = -__builtin_inff();
constexpr float kNear = 16.f;  // |lse| that is taken as it is (its rounding: 2^-21)

__device__ __forceinline__ float wave_max(float v)
{
    for (int o = 1; o < kWave; o *= 2) v = fmaxf(v, __shfl_xor(v, o, kWave));
    return v;
}

// A row's pieces stay as they lie in memory from one pass to the next: the values that they
// expand to, and exponentials of those, would take four times the registers.
template <typename R>
__device__ __forceinline__ void forget(R& r)
{
    if constexpr (sizeof(R) == 16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t x = r[i];
            asm("" : "+v"(x));
            r[i] = x;
        }
    }
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

// One row: MODE 0: loss; 1: loss and gradient; 2: gradient from lse.  A thread has ITER pieces of
// the row in registers, or reads them again (ITER = 0), and at most one slot (K <= BLOCK).
template <typename T, int BLOCK, int ITER, int MODE>
__global__ __launch_bounds__(BLOCK, ITER <= 8 ? 8 : 4) void distill_kernel(Args<T> a)
{
    constexpr int V = kVec<T>;
    constexpr int waves = BLOCK / kWave;
    __shared__ float2 tops[waves];
    __shared__ float4 sums[waves];
    __shared__ float2 slots[BLOCK];  // id (bits), e
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int pieces = int(a.V / V), tail = int(a.V % V);  // whole pieces, then single values
    const int64_t row = blockIdx.x;
    const T* x = a.logits + row * a.ld;
    T* out = MODE ? a.dlogits + row * a.ld_d : nullptr;
    const float scale = a.scale ? a.scale[row] : 1.f;
    const float lse = MODE == 2 ? a.lse_in[row] : 0.f;
    const bool forms = MODE < 2 || !(fabsf(lse) <= kNear);  // the row's largest value and sum

    // the teacher's side: a slot to a thread
    const bool has = int(threadIdx.x) < a.K;
    int id = -1;
    float t = kNone;
    if (has) {
        id = a.ids[row * a.K + threadIdx.x];
        const float v = a.values[row * a.K + threadIdx.x];
        // (NaN as infinity, which the maximum does not drop: the row is NaN)
        if (id >= 0 && id < a.V) t = v != v ? -kNone : v;
    }
    // the student's: pieces and values past the last whole piece
    Raw<T, V> raw[ITER > 0 ? ITER : 1];
    float last = kNone, own = 0.f, top = kNone;
    auto each = [&](auto f) __attribute__((always_inline)) {
        if constexpr (ITER > 0) {
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                const int p = i * BLOCK + int(threadIdx.x);
                if (p < pieces) f(raw[i], p);
                forget(raw[i]);
            }
        } else {
            constexpr int kAhead = 4;  // pieces in flight
            for (int p0 = threadIdx.x; p0 < pieces; p0 += kAhead * BLOCK) {
                Raw<T, V> r[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i)
                    if (p0 + i * BLOCK < pieces) r[i] = load_raw<V>(x + int64_t(p0 + i * BLOCK) * V);
#pragma unroll
                for (int i = 0; i < kAhead; ++i)
                    if (p0 + i * BLOCK < pieces) f(r[i], p0 + i * BLOCK);
            }
        }
    };
    if (scale != 0.f) {
        if constexpr (ITER > 0) {
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                const int p = i * BLOCK + int(threadIdx.x);
                if (p < pieces) raw[i] = load_raw<V>(x + int64_t(p) * V);
            }
        }
        if (int(threadIdx.x) < tail) last = io_load(x + int64_t(pieces) * V + threadIdx.x);
        if (t != kNone) own = io_load(x + id);
        if (forms) {
            top = last;
            each([&](const Raw<T, V>& r, int) {
                float v[V];
                expand<V, T>(r, v);
#pragma unroll
                for (int j = 0; j < V; j += 2) top = fmaxf(fmaxf(v[j], v[j + 1]), top);
            });
        }
    }
    const float2 most = make_float2(forms ? wave_max(top) : kNone, wave_max(t));
    if (lane == 0) tops[wave] = most;
    __syncthreads();
    const float2 of_wave = tops[lane % waves];
    top = of_wave.x;
    float top_t = of_wave.y;
#pragma unroll
    for (int o = 1; o < waves; o *= 2) {
        if (forms) top = fmaxf(top, __shfl_xor(top, o, kWave));
        top_t = fmaxf(top_t, __shfl_xor(top_t, o, kWave));
    }
    if (scale == 0.f || top_t == kNone) {  // a row that takes no part, or without slots
        if (MODE < 2 && threadIdx.x == 0) {
            a.loss[row] = 0.f;
            if (a.lse_out) a.lse_out[row] = 0.f;
        }
        if constexpr (MODE > 0) {
            const float zeros[V] = {};
            for (int p = threadIdx.x; p < pieces; p += BLOCK) put<V>(out + int64_t(p) * V, zeros);
            if (int(threadIdx.x) < tail) io_store(out + int64_t(pieces) * V + threadIdx.x, 0.f);
        }
        return;
    }
    // exponents in base 2: less the row's largest (a difference first: the rounding of a product of
    // a large offset would not cancel), or less lse
    const float off = !forms || top == kNone ? 0.f : top, off2 = forms ? 0.f : lse * kLog2e;
    auto power = [&](float v) { return MODE == 2 ? fmaf(v - off, a.to2, -off2) : (v - off) * a.to2; };
    const float d = (t - top_t) * a.to2;
    const float e = t == kNone ? 0.f : exp2_fast(d);
    own = power(own);
    if (MODE > 0 && has) slots[threadIdx.x] = make_float2(__int_as_float(id), e);
    // of the student's exponentials, of the teacher's, and of those times both exponents' distance
    float4 sum = make_float4(0.f, e, e != 0.f ? e * (d - own) : 0.f, 0.f);
    if (forms) {
        if (int(threadIdx.x) < tail) sum.x = exp2_fast(power(last));
        each([&](const Raw<T, V>& r, int) {
            float v[V];
            expand<V, T>(r, v);
#pragma unroll
            for (int j = 0; j < V; ++j) sum.x += exp2_fast(power(v[j]));
        });
        sum.x = wave_sum(sum.x);
    }
    if constexpr (MODE < 2) sum.z = wave_sum(sum.z);
    sum.y = wave_sum(sum.y);
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    sum = sums[lane % waves];
#pragma unroll
    for (int o = 1; o < waves; o *= 2) {
        if (forms) sum.x += __shfl_xor(sum.x, o, kWave);
        sum.y += __shfl_xor(sum.y, o, kWave);
        sum.z += __shfl_xor(sum.z, o, kWave);
    }
    if (MODE < 2 && threadIdx.x == 0) {
        const float l2 = __builtin_amdgcn_logf(sum.x);
        // (no finite logit: the student's probabilities are 0)
        const float nats = sum.x == 0.f ? __builtin_inff()
                                        : kLn2 * (sum.z / sum.y + (l2 - __builtin_amdgcn_logf(sum.y)));
        a.loss[row] = scale * a.tau * a.tau * nats;
        if (a.lse_out) a.lse_out[row] = fmaf(kLn2, l2, top == kNone ? kNone : top / a.tau);
    }
    if constexpr (MODE > 0) {
        float c = scale * a.tau;
        if (MODE == 2) c *= a.dloss[row];
        const float cq = !forms ? c : sum.x == 0.f ? 0.f : c / sum.x;
        each([&](const Raw<T, V>& r, int p) {
            float v[V];
            expand<V, T>(r, v);
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = exp2_fast(power(v[j])) * cq;
            put<V>(out + int64_t(p) * V, v);
        });
        if (int(threadIdx.x) < tail)
            io_store(out + int64_t(pieces) * V + threadIdx.x, exp2_fast(power(last)) * cq);
        // a slot's own value: the exponentials of all slots of its id, in their order
        float of_id = 0.f;
        if (e != 0.f) {
#pragma unroll 8
            for (int k = 0; k < a.K; ++k) {
                const float2 s = slots[k];
                of_id += __float_as_int(s.x) == id ? s.y : 0.f;
            }
        }
        __syncthreads();
        if (e != 0.f) io_store(out + id, fmaf(exp2_fast(own), cq, -c * (of_id / sum.y)));
    }
}

// Threads to a row and pieces of a thread (0: read again from memory).
template <int MODE, typename T, typename F>
hipError_t with_shape(int64_t V, int K, F f)
{
    const int64_t pieces = V / kVec<T>;
    auto iters = [&](auto block) {
        constexpr int B = decltype(block)::value;
        const int64_t n = (pieces + B - 1) / B;
        if (n <= 1) return f(block, std::integral_constant<int, 1>());
        if (n <= 2) return f(block, std::integral_constant<int, 2>());
        if constexpr (B < 1024) {  // (four at most)
            return f(block, std::integral_constant<int, 4>());
        } else {
            if (n <= 4) return f(block, std::integral_constant<int, 4>());
            if (n <= 6) return f(block, std::integral_constant<int, 6>());
            if (n <= 8) return f(block, std::integral_constant<int, 8>());
            if (n <= kHold) return f(block, std::integral_constant<int, kHold>());
            return f(block, std::integral_constant<int, 0>());
        }
    };
    if (pieces <= 4 * 256 && K <= 256) return iters(std::integral_constant<int, 256>());
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
    return with_shape<MODE, T>(d.V, d.K, [&](auto block, auto iter) {
        constexpr int B = decltype(block)::value, ITER = decltype(iter)::value;
        hipLaunchKernelGGL((distill_kernel<T, B, ITER, MODE>),
                           dim3(uint32_t(d.rows)), dim3(B), 0, stream, a);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_distill_logits(const DistillLogits& a, float* loss, float* lse, hipStream_t stream)
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
