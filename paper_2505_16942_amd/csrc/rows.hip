// The last step of every sum over rows: partial sums of the workgroups, added in their order.
#include "rows.h"

namespace {
// 64 columns a workgroup, 16 shares of the parts each: the loads of a share are independent, its sum is in order.
constexpr int SHARES = 16;
__global__ __launch_bounds__(64 * SHARES) void column_sums_kernel(const float* __restrict__ part, int parts, int C, ColumnSums o) {
    __shared__ float sums[SHARES][64];
    const int lane = threadIdx.x & 63, share = threadIdx.x >> 6, c = blockIdx.x * 64 + lane, v = blockIdx.y;
    float* const out = o.out[v];
    if (!out) return;
    const int64_t stride = (int64_t)gridDim.y * C;
    float sum = 0.f;
    if (c < C) {
        const float* p = part + (int64_t)v * C + c;
#pragma unroll 8
        for (int i = share; i < parts; i += SHARES) sum += p[i * stride];
    }
    sums[share][lane] = sum;
    __syncthreads();
    if (share == 0 && c < C) {
        for (int s = 1; s < SHARES; ++s) sum += sums[s][lane];
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
    hipLaunchKernelGGL(column_sums_kernel, dim3((C + 63) / 64, vectors), dim3(64 * SHARES), 0, s, part, parts, C, o);
    return hipGetLastError();
}
