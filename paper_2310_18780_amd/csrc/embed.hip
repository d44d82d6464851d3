// Embedding lookup: y[k] = scale W[ids[k]] (zeros where the id is outside the table).
//
// Bound by memory: a row of the table is read and a row of y written for each token.  A
// team of one wavefront, or of four where rows are few, takes a token; its id is one scalar
// load, and its pieces of 16 bytes of y are all in flight together.  A piece that would pass
// the row's end starts before it instead, so that every access is a whole piece at any
// alignment (two lanes then store the same bits).  65536 tokens x 2048 from a float32 table to
// bfloat16 take 93 us (268 MB written, 360 MB read, the 16600 rows met more than twice on average: 6.7
// TB/s); 64 tokens from a bfloat16 table 2.3 us.
#include "embed.hpp"

#include "block_ops.hpp"

namespace lh {
namespace {

constexpr int64_t kMaxBlocks = 1 << 20;  // grid-stride beyond

// V values of a row from p.
template <int V, typename T>
__device__ __forceinline__ void load_values(const T* p, float (&v)[V])
{
    constexpr int n = V < kVec<T> ? V : kVec<T>;
#pragma unroll
    for (int i = 0; i < V / n; ++i) {
        float part[n];
        expand<n, T>(load_raw<n>(p + i * n), part);
#pragma unroll
        for (int j = 0; j < n; ++j) v[i * n + j] = part[j];
    }
}

template <typename W, typename T, int V, int TEAM>
__global__ __launch_bounds__(256) void embed_kernel(const W* __restrict__ table,
                                                    const int* __restrict__ ids, int64_t n,
                                                    uint32_t rows, int64_t D, float scale,
                                                    T* __restrict__ y)
{
    constexpr int teams = 256 / TEAM;
    const int lane = threadIdx.x % TEAM;
    const int team = teams == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / TEAM);
    const int64_t step = int64_t(gridDim.x) * teams;
    for (int64_t k = int64_t(blockIdx.x) * teams + team; k < n; k += step) {
        const uint32_t id = uint32_t(ids[k]);
        T* out = y + k * D;
        if (id < rows) {
            const W* in = table + int64_t(id) * D;
#pragma unroll 4
            for (int64_t c = int64_t(lane) * V; c < D; c += TEAM * V) {
                const int64_t at = c + V <= D ? c : D - V;
                float v[V];
                load_values<V>(in + at, v);
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] *= scale;
                put<V>(out + at, v);
            }
        } else {
            float v[V] = {};
            for (int64_t c = int64_t(lane) * V; c < D; c += TEAM * V)
                put<V>(out + (c + V <= D ? c : D - V), v);
        }
    }
}

template <typename T>
int embed_team(int64_t n, int64_t D)
{
    return n >= 2048 || D <= 64 * kVec<T> ? 64 : 256;
}

int64_t embed_blocks(int team, int64_t n)
{
    const int64_t b = (n + 256 / team - 1) / (256 / team);
    return b < kMaxBlocks ? b : kMaxBlocks;
}

template <typename W, typename T>
hipError_t embed(const W* table, const int32_t* ids, int64_t n, int64_t V, int64_t D, float scale,
                 T* y, hipStream_t stream)
{
    const int team = embed_team<T>(n, D);
    const dim3 grid(uint32_t(embed_blocks(team, n)));
    const uint32_t rows = uint32_t(V);
    if (D < kVec<T>)
        hipLaunchKernelGGL((embed_kernel<W, T, 1, 64>), dim3(uint32_t(embed_blocks(64, n))), dim3(256), 0,
                           stream, table, ids, n, rows, D, scale, y);
    else if (team == 64)
        hipLaunchKernelGGL((embed_kernel<W, T, kVec<T>, 64>), grid, dim3(256), 0, stream, table, ids, n,
                           rows, D, scale, y);
    else
        hipLaunchKernelGGL((embed_kernel<W, T, kVec<T>, 256>), grid, dim3(256), 0, stream, table, ids, n,
                           rows, D, scale, y);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embed(const void* W, const int32_t* ids, int64_t n, int64_t V, int64_t D,
                        bool bf16_table, bool bf16_io, float scale, void* y, hipStream_t stream)
{
    if (bf16_table)
        return bf16_io ? embed(static_cast<const bf16*>(W), ids, n, V, D, scale, static_cast<bf16*>(y), stream)
                       : embed(static_cast<const bf16*>(W), ids, n, V, D, scale, static_cast<float*>(y), stream);
    return bf16_io ? embed(static_cast<const float*>(W), ids, n, V, D, scale, static_cast<bf16*>(y), stream)
                   : embed(static_cast<const float*>(W), ids, n, V, D, scale, static_cast<float*>(y), stream);
}

}  // namespace lh
