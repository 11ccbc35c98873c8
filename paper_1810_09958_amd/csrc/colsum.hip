// Sums over rows of fp32 partial sums, in a fixed order: the last step of the
// gradients of biases, gates and norm weights, whose workgroups each leave one
// row of partial sums.
#include "kernels.hpp"
#include "rowio.hpp"

namespace isam {

namespace {

// 64 columns and 16 row groups per workgroup; group g adds rows g, g + 16, ...,
// then the sixteen sums are added in order.
template <int ES>
__global__ __launch_bounds__(1024) void colsum_kernel(const float* part, int64_t rows, int64_t cols, void* out) {
    __shared__ float sums[16][64];
    const int cl = threadIdx.x & 63, g = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + cl, z = blockIdx.y;
    float s = 0.0f;
    if (c < cols) {
        const float* p = part + z * rows * cols + c;
#pragma unroll 8
        for (int64_t r = g; r < rows; r += 16) s += p[r * cols];
    }
    sums[g][cl] = s;
    __syncthreads();
    if (g != 0 || c >= cols) return;
    for (int i = 1; i < 16; ++i) s += sums[i][cl];
    Row16<ES>::put(out, z * cols + c, s);
}

}  // namespace

hipError_t launch_colsum(const float* part, int64_t rows, int64_t cols, int64_t groups, int out_type, void* out, hipStream_t s) {
    if (cols <= 0 || groups <= 0) return hipSuccess;
    if ((cols + 63) / 64 > INT32_MAX || groups > 65535) return hipErrorInvalidValue;
    hipLaunchKernelGGL((out_type == kBF16 ? colsum_kernel<2> : colsum_kernel<4>), dim3((unsigned)((cols + 63) / 64), (unsigned)groups),
                       dim3(1024), 0, s, part, rows, cols, out);
    return hipGetLastError();
}

}  // namespace isam
