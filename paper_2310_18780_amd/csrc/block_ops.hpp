// Device helpers shared by the selective block's kernels (layer norm, short
// convolution, selective scan): rows of any alignment, wave sums, and the
// elementary functions of the gate and of the time step.
#pragma once

#include "lh_internal.hpp"

namespace lh {

constexpr int kWave = 64;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// Elements of a 16-byte piece.
template <typename T>
constexpr int kVec = 16 / sizeof(T);

// Rows begin where the caller's slices do: 2- (4-) byte aligned.  The hardware
// serves 16-byte pieces at any such address; the type only says so.
typedef uint32_t piece4 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t piece2 __attribute__((ext_vector_type(2), aligned(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    const bf16x2 v = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
    return __builtin_bit_cast(uint32_t, v);
}

// A piece of V values as it lies in memory (16 or 8 bytes, or one value), and its
// values.  (A piece that is converted where it is loaded is waited for there.)
template <typename T, int V>
struct RawOf {
    using type = std::conditional_t<V * sizeof(T) == 16, piece4, piece2>;
};
template <typename T>
struct RawOf<T, 1> {
    using type = T;
};
template <typename T, int V>
using Raw = typename RawOf<T, V>::type;

template <int V, typename T>
__device__ __forceinline__ Raw<T, V> load_raw(const T* p)
{
    return *reinterpret_cast<const Raw<T, V>*>(p);
}
template <int V, typename T>
__device__ __forceinline__ void expand(const Raw<T, V>& r, float (&v)[V])
{
    if constexpr (V == 1) {
        v[0] = io_load(&r);
    } else if constexpr (sizeof(T) == 4) {
        for (int i = 0; i < V; ++i) v[i] = __uint_as_float(r[i]);
    } else {
        for (int i = 0; i < V / 2; ++i) {
            v[2 * i] = __uint_as_float(r[i] << 16);
            v[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
        }
    }
}
template <int V, typename T>
__device__ __forceinline__ void put(T* p, const float (&v)[V])
{
    if constexpr (V == 1) {
        io_store(p, v[0]);
    } else if constexpr (sizeof(T) == 4) {
        Raw<T, V> r;
        for (int i = 0; i < V; ++i) r[i] = __float_as_uint(v[i]);
        *reinterpret_cast<Raw<T, V>*>(p) = r;
    } else {
        Raw<T, V> r;
        for (int i = 0; i < V / 2; ++i) r[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
        *reinterpret_cast<Raw<T, V>*>(p) = r;
    }
}

// The first n of V elements (n <= 0: none); the others read as zero.
template <int V, typename T>
__device__ __forceinline__ void load_some(const T* p, int n, float (&v)[V])
{
    if (n >= V) {
        expand<V, T>(load_raw<V>(p), v);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = i < n ? io_load(p + i) : 0.f;
    }
}
template <int V, typename T>
__device__ __forceinline__ void store_some(T* p, int n, const float (&v)[V])
{
    if (n >= V) {
        put<V>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) io_store(p + i, v[i]);
    }
}

// Sum over the wave's 64 lanes, in every lane: butterflies within 16 lanes by
// DPP, then rows and halves of the wave exchanged.
__device__ __forceinline__ float dpp_add(float v, int perm_of_v)
{
    return v + __builtin_bit_cast(float, perm_of_v);
}
__device__ __forceinline__ float wave_sum(float v)
{
    v = dpp_add(v, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0xB1, 0xF, 0xF, true));
    v = dpp_add(v, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x4E, 0xF, 0xF, true));
    v = dpp_add(v, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x141, 0xF, 0xF, true));
    v = dpp_add(v, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x140, 0xF, 0xF, true));
    v += __shfl_xor(v, 16, kWave);
    v += __shfl_xor(v, 32, kWave);
    return v;
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float rcp_fast(float x) { return __builtin_amdgcn_rcpf(x); }

// 1 / (1 + e^-x): exactly 0 once e^-x overflows (x below about -88).
__device__ __forceinline__ float sigmoid(float x)
{
    return rcp_fast(1.f + exp2_fast(-kLog2e * x));
}

// log(1 + e^x) = max(x, 0) + log(1 + e), e = e^-|x|.  w = 1 + e is rounded; the
// rounding e - (w - 1) is added back to log w, so that nothing of e is lost where it is
// far below 1 (there w = 1 and the term is e).  What is left is e's own error: its exponent
// -|x| log2 e is rounded, so the relative error grows with |x|, to at most about
// (7 + 1.25 |x|) 2^-24 for x < 0 and 7 x 2^-24 above.
__device__ __forceinline__ float softplus(float x)
{
    const float e = exp2_fast(-kLog2e * fabsf(x));
    const float w = 1.f + e;
    const float l = __builtin_amdgcn_logf(w);  // log2
    // (NaN stays NaN through e)
    return fmaxf(x, 0.f) + fmaf(kLn2, l, e - (w - 1.f));
}

// The block launchers.  Outputs that may be NULL are said so in include/lh.h.

// Column sums of the rows of part [P, Q], Q = n0 + n1 + n2: out0 gets the first n0
// columns, out1 the next n1, out2 the last n2 (NULL: not written).  Sums run in a
// fixed order.
hipError_t launch_column_sum(const float* part, int64_t P, int64_t n0, float* out0, int64_t n1,
                             float* out1, int64_t n2, float* out2, hipStream_t stream);

}  // namespace lh
