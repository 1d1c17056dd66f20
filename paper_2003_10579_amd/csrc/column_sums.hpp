// Sums over the rows of a matrix of partial sums, each of which a workgroup has left.
#pragma once
#include "ops.hpp"

namespace ssgd {
namespace {

// Sums of 16 columns: the 64 quarter waves of a workgroup take every 64th partial sum, eight loads in flight (a load that is left out would
// wait for those before: past the end the last sum is read again), and add in fp64 (768 sums of 4096 columns: 6.0 us, 512 of 1537 4.3 us; with 64 columns
// and whole cache lines to a workgroup no faster).
__global__ __launch_bounds__(1024) void column_sums_kernel(const float* partial, int64_t groups, int32_t d, float* sums) {
    __shared__ double part[64][17];
    const int c = threadIdx.x & 15, group = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
    double sum = 0.0;
    if (col < d) {
        for (int64_t t = group; t < groups; t += 64 * 8) {
            float x[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) x[q] = partial[(t + 64 * q < groups ? t + 64 * q : groups - 1) * d + col];
#pragma unroll
            for (int q = 0; q < 8; ++q) sum += t + 64 * q < groups ? (double)x[q] : 0.0;
        }
    }
    part[group][c] = sum;
    __syncthreads();
    if (threadIdx.x < 64) {
        // sixteen sums a lane, then the four lanes of a column
        sum = 0.0;
#pragma unroll
        for (int q = 0; q < 16; ++q) sum += part[q * 4 + group][c];
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (group == 0 && col < d) sums[col] = (float)sum;
    }
}

// d < 2^25: 16 columns to a workgroup of 1024, and a launch ends at 2^32 threads.
void launch_column_sums(const float* partial, int64_t groups, int64_t d, float* sums, hipStream_t s) {
    hipLaunchKernelGGL(column_sums_kernel, dim3((unsigned)((d + 15) / 16)), dim3(1024), 0, s, partial, groups, (int32_t)d, sums);
}

}  // namespace
}  // namespace ssgd
