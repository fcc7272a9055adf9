// The last step of every sum over rows: partial sums of the workgroups, added in their order.
#include "rows.h"

namespace {
// 16 columns a workgroup, 64 shares of the parts each: a share's loads are independent and its sum is in order, as is the sum of the shares.
// With 64 columns and 16 shares, 1024 parts of 1024 columns took 11 us.
constexpr int SHARES = 64, COLS = 16;
__global__ __launch_bounds__(COLS * SHARES) void column_sums_kernel(const float* __restrict__ part, int parts, int C, ColumnSums o) {
    __shared__ float sums[SHARES][COLS];
    const int col = threadIdx.x % COLS, share = threadIdx.x / COLS, c = blockIdx.x * COLS + col, v = blockIdx.y;
    float* const out = o.out[v];
    if (!out) return;
    const int64_t stride = (int64_t)gridDim.y * C;
    float sum = 0.f;
    if (c < C) {
        const float* p = part + (int64_t)v * C + c;
#pragma unroll 8
        for (int i = share; i < parts; i += SHARES) sum += p[i * stride];
    }
    sums[share][col] = sum;
    __syncthreads();
    if (share == 0 && c < C) {
#pragma unroll 8
        for (int s = 1; s < SHARES; ++s) sum += sums[s][col];
        out[c] = sum;
    }
}

__global__ __launch_bounds__(256) void zero_kernel(uint16_t* p, size_t n) {
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) p[i] = 0;
}
}  // namespace

// A kernel, not a memset: the call may be captured into a graph.
hipError_t launch_zero(void* p, size_t bytes, hipStream_t s) {
    const size_t blocks = (bytes / 2 + 255) / 256;
    if (!p || !blocks) return hipSuccess;
    hipLaunchKernelGGL(zero_kernel, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, s, (uint16_t*)p, bytes / 2);
    return hipGetLastError();
}

hipError_t launch_column_sums(const float* part, int parts, int vectors, int C, const ColumnSums& o, hipStream_t s) {
    hipLaunchKernelGGL(column_sums_kernel, dim3((C + COLS - 1) / COLS, vectors), dim3(COLS * SHARES), 0, s, part, parts, C, o);
    return hipGetLastError();
}
