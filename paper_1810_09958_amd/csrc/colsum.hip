// Sums over rows of fp32 partial sums, in a fixed order: the last step of the
// gradients of biases, gates and norm weights, whose workgroups each leave one
// row of partial sums.
#include "kernels.hpp"
#include "rowio.hpp"

namespace isam {

namespace {

struct ColSums {
    ColSum s[3];
};

// 32 columns and 32 row groups per workgroup; group g adds rows g, g + 32, ..., then
// the groups are added in pairs.
__global__ __launch_bounds__(1024) void colsum_kernel(ColSums all) {
    __shared__ float sums[32][33];
    const ColSum& c = all.s[blockIdx.z];
    const int cl = threadIdx.x & 31, g = threadIdx.x >> 5;
    const int64_t col = (int64_t)blockIdx.x * 32 + cl;
    if ((int64_t)blockIdx.x * 32 >= c.cols) return;
    for (int64_t z = blockIdx.y; z < c.groups; z += gridDim.y) {
        float s = 0.0f;
        if (col < c.cols) {
            const float* const p = c.part + z * c.rows * c.cols + col;
#pragma unroll 16
            for (int64_t r = g; r < c.rows; r += 32) s += p[r * c.cols];
        }
        sums[g][cl] = s;
        __syncthreads();
        // row cl of the transposed sums, 32 lanes at a time
        float v = sums[cl][g];
        static_for<5>([&](auto k) { v += __shfl_xor(v, 1 << decltype(k)::value); });
        const int64_t out = (int64_t)blockIdx.x * 32 + g;
        if (cl == 0 && out < c.cols) {
            if (c.type == kBF16) Row16<2>::put(c.out, z * c.cols + out, v);
            else Row16<4>::put(c.out, z * c.cols + out, v);
        }
        __syncthreads();
    }
}

}  // namespace

hipError_t launch_colsum(const ColSum* sums, int count, hipStream_t s) {
    ColSums all{};
    int64_t cols = 0, groups = 0;
    for (int i = 0; i < count; ++i) {
        all.s[i] = sums[i];
        cols = sums[i].cols > cols ? sums[i].cols : cols;
        groups = sums[i].groups > groups ? sums[i].groups : groups;
    }
    if (cols <= 0 || groups <= 0) return hipSuccess;
    if (count > 3 || (cols + 31) / 32 > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL(colsum_kernel, dim3((unsigned)((cols + 31) / 32), (unsigned)(groups < 4096 ? groups : 4096), (unsigned)count),
                       dim3(1024), 0, s, all);
    return hipGetLastError();
}

}  // namespace isam
