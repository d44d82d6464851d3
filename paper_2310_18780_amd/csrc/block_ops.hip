// Column sums of partial results: the last step of every weight gradient of the
// selective block (layer norm, short convolution, selective scan).
#include "block_ops.hpp"

namespace lh {
namespace {

constexpr int kSlices = 16;  // rows are summed in 16 interleaved slices, then across them

__global__ __launch_bounds__(kWave* kSlices) void column_sum_kernel(
    const float* __restrict__ part, int64_t P, int64_t n0, float* out0, int64_t n1, float* out1,
    int64_t n2, float* out2)
{
    __shared__ float red[kSlices][kWave];
    const int lane = threadIdx.x & (kWave - 1);
    const int slice = threadIdx.x / kWave;
    const int64_t Q = n0 + n1 + n2;
    const int64_t q = int64_t(blockIdx.x) * kWave + lane;
    float acc = 0.f;
    if (q < Q) {
        const float* p = part + q;
        int64_t r = slice;
        for (; r + 3 * kSlices < P; r += 4 * kSlices) {
            const float a = p[r * Q], b = p[(r + kSlices) * Q], c = p[(r + 2 * kSlices) * Q],
                        d = p[(r + 3 * kSlices) * Q];
            acc += (a + b) + (c + d);
        }
        for (; r < P; r += kSlices) acc += p[r * Q];
    }
    red[slice][lane] = acc;
    __syncthreads();
    if (slice == 0 && q < Q) {
        float s = 0.f;
        for (int i = 0; i < kSlices; ++i) s += red[i][lane];
        if (q < n0) {
            if (out0) out0[q] = s;
        } else if (q < n0 + n1) {
            if (out1) out1[q - n0] = s;
        } else if (out2) {
            out2[q - n0 - n1] = s;
        }
    }
}

}  // namespace

hipError_t launch_column_sum(const float* part, int64_t P, int64_t n0, float* out0, int64_t n1,
                             float* out1, int64_t n2, float* out2, hipStream_t stream)
{
    const int64_t blocks = (n0 + n1 + n2 + kWave - 1) / kWave;
    hipLaunchKernelGGL(column_sum_kernel, dim3(uint32_t(blocks)), dim3(kWave * kSlices), 0, stream,
                       part, P, n0, out0, n1, out1, n2, out2);
    return hipGetLastError();
}

}  // namespace lh
