// Column sums of partial results: the last step of every weight gradient of the
// selective block (layer norm, short convolution, selective scan).
#include "block_ops.hpp"

namespace lh {
namespace {

// A workgroup sums 32 columns (a line of a row), the rows in 32 interleaved slices, then
// across those.  (64 columns in 16 slices leave half the workgroups: 1024 rows of 4096
// columns 7 us.)
constexpr int kCols = 32, kSlices = 32;

__global__ __launch_bounds__(kCols* kSlices) void column_sum_kernel(
    const float* __restrict__ part, int64_t P, int64_t n0, float* out0, int64_t n1, float* out1,
    int64_t n2, float* out2)
{
    __shared__ float red[kSlices][kCols];
    const int lane = threadIdx.x % kCols;
    const int slice = threadIdx.x / kCols;
    const int64_t Q = n0 + n1 + n2;
    const int64_t q = int64_t(blockIdx.x) * kCols + lane;
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
    const int64_t blocks = (n0 + n1 + n2 + kCols - 1) / kCols;
    hipLaunchKernelGGL(column_sum_kernel, dim3(uint32_t(blocks)), dim3(kCols * kSlices), 0, stream,
                       part, P, n0, out0, n1, out1, n2, out2);
    return hipGetLastError();
}

}  // namespace lh
