// Norm over the channels of a group and all pixels of an item, with an activation, channels last, and its gradient.
#include "matrix.h"
#include "group_norm.h"

namespace {

constexpr int THREADS = 256;
inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// A thread has V neighbouring channels (16 bytes of them) and every rt-th row of its workgroup's share; ct threads stand beside each other.
template <int V> struct Columns {
    int ct, rt, c, r0, left;
    __device__ __forceinline__ Columns(int C, int ct_) : ct(ct_), rt(THREADS / ct_) {
        c = (blockIdx.x * ct + threadIdx.x % ct) * V;
        r0 = threadIdx.x / ct;
        left = C - c;
    }
};
template <int V> int threads_across(int C) {
    int ct = 1;
    while (ct < THREADS && ct * V < C) ct *= 2;
    return ct;
}

// n values with mean and sum of squares about it, and m more: Chan, Golub and LeVeque's rule, which cancels nothing however large the mean is
__device__ __forceinline__ void merge(float n, float& mean, float& square, float m, float mean2, float square2) {
    if (m == 0.f) return;
    const float d = mean2 - mean, f = m / (n + m);
    mean = fmaf(d, f, mean);
    square += square2 + d * (n * f) * d;
}

// Means and squares of every channel over the workgroup's rows, U rows at a time from registers.
template <class T, int V>
__global__ __launch_bounds__(THREADS) void stats_kernel(GroupNormArgs a, int ct) {
    constexpr int U = 8;
    __shared__ float means[THREADS][V], squares[THREADS][V];
    const Columns<V> at(a.C, ct);
    const int64_t lo = blockIdx.y * a.share, hi = min(a.P, lo + a.share), item = blockIdx.z * a.P;
    const T* const x = (const T*)a.x + at.c;
    float mean[V] = {}, square[V] = {}, n = 0.f;
    if (at.left > 0) {
        int64_t r = lo + at.r0;
        for (; r + (U - 1) * at.rt < hi; r += U * at.rt) {
            float v[U][V];
#pragma unroll
            for (int u = 0; u < U; ++u) load_some<T, V>(x + (item + r + u * at.rt) * a.x_stride, v[u], at.left);
            const float f = (float)U / (n + U), nf = n * f;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float s = 0.f, q = 0.f;
#pragma unroll
                for (int u = 0; u < U; ++u) s += v[u][e];
                s *= 1.f / U;
#pragma unroll
                for (int u = 0; u < U; ++u) { const float d = v[u][e] - s; q = fmaf(d, d, q); }
                const float d = s - mean[e];
                mean[e] = fmaf(d, f, mean[e]);
                square[e] += fmaf(d * nf, d, q);
            }
            n += U;
        }
        for (; r < hi; r += at.rt) {
            float v[V];
            load_some<T, V>(x + (item + r) * a.x_stride, v, at.left);
#pragma unroll
            for (int e = 0; e < V; ++e) merge(n, mean[e], square[e], 1.f, v[e], 0.f);
            n += 1.f;
        }
    }
    // threads r0 and r0 + half meet; both counts follow from the rows
    auto count = [&](int r0, int64_t step) { return hi - lo > r0 ? (float)((hi - lo - r0 + step - 1) / step) : 0.f; };
#pragma unroll
    for (int e = 0; e < V; ++e) { means[threadIdx.x][e] = mean[e]; squares[threadIdx.x][e] = square[e]; }
    for (int half = at.rt / 2; half; half /= 2) {
        __syncthreads();
        if (at.r0 < half) {
            const float m = count(at.r0 + half, 2 * half);
            const int other = threadIdx.x + half * ct;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                merge(n, mean[e], square[e], m, means[other][e], squares[other][e]);
                means[threadIdx.x][e] = mean[e];
                squares[threadIdx.x][e] = square[e];
            }
            n = count(at.r0, half);
        }
    }
    if (at.r0 == 0)
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e < at.left) {
                float* const p = a.part + 2 * ((int64_t)(blockIdx.z * a.parts + blockIdx.y) * a.C + at.c + e);
                p[0] = mean[e];
                p[1] = square[e];
            }
}

// A group's parts: mean and 1 / spread.  One workgroup a group and item.
__global__ __launch_bounds__(THREADS) void finish_stats_kernel(GroupNormArgs a) {
    __shared__ float means[THREADS], squares[THREADS], counts[THREADS];
    const int g = blockIdx.x % a.G, b = blockIdx.x / a.G, width = a.C / a.G, tid = threadIdx.x;
    const int64_t all = (int64_t)a.parts * width;
    float mean = 0.f, square = 0.f, n = 0.f;
    for (int64_t i = tid; i < all; i += THREADS) {
        const int64_t p = i / width;
        const float* const q = a.part + 2 * (((int64_t)b * a.parts + p) * a.C + g * width + (i - p * width));
        const float m = (float)min(a.share, a.P - p * a.share);
        merge(n, mean, square, m, q[0], q[1]);
        n += m;
    }
    means[tid] = mean; squares[tid] = square; counts[tid] = n;
    for (int half = THREADS / 2; half; half /= 2) {
        __syncthreads();
        if (tid < half) {
            merge(n, mean, square, counts[tid + half], means[tid + half], squares[tid + half]);
            n += counts[tid + half];
            means[tid] = mean; squares[tid] = square; counts[tid] = n;
        }
    }
    if (tid == 0) {
        a.stats[2 * blockIdx.x] = mean;
        a.stats[2 * blockIdx.x + 1] = 1.f / sqrtf(square / n + a.eps);
    }
}

// mean, 1 / spread, weight and bias of a thread's channels
template <int V> struct Channels { float mean[V], rho[V], w[V], b[V]; };
template <int V>
__device__ __forceinline__ void load_channels(const GroupNormArgs& a, int item, int c, Channels<V>& k) {
    const int width = a.C / a.G;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int ch = min(c + e, a.C - 1);
        const float* const s = a.stats + 2 * (item * a.G + ch / width);
        k.mean[e] = s[0];
        k.rho[e] = s[1];
        k.w[e] = a.weight ? a.weight[ch] : 1.f;
        k.b[e] = a.bias ? a.bias[ch] : 0.f;
    }
}

template <class T, int V>
__global__ __launch_bounds__(THREADS) void apply_kernel(GroupNormArgs a, int ct) {
    constexpr int U = 4;
    const Columns<V> at(a.C, ct);
    if (at.left <= 0) return;
    const int64_t lo = blockIdx.y * a.share, hi = min(a.P, lo + a.share), item = blockIdx.z * a.P;
    Channels<V> k;
    load_channels(a, blockIdx.z, at.c, k);
#pragma unroll
    for (int e = 0; e < V; ++e) k.w[e] *= k.rho[e];
    const T* const x = (const T*)a.x + at.c;
    T* const y = (T*)a.y + at.c;
    for (int64_t r = lo + at.r0; r < hi; r += U * at.rt) {
        float v[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (r + u * at.rt < hi) load_some<T, V>(x + (item + r + u * at.rt) * a.x_stride, v[u], at.left);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (r + u * at.rt >= hi) break;
#pragma unroll
            for (int e = 0; e < V; ++e) v[u][e] = fmaf(v[u][e] - k.mean[e], k.w[e], k.b[e]);
            row_act_all(a.act, v[u]);
            store_some<T, V>(y + (item + r + u * at.rt) * a.C, v[u], at.left);
        }
    }
}

// ---- gradient.  hat = (x - mean) rho, z = hat w + b, dz = d_y act'(z).
template <class T, int V>
__device__ __forceinline__ void slopes(const GroupNormArgs& a, const Channels<V>& k, float (&x)[V], float (&g)[V]) {
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = (x[e] - k.mean[e]) * k.rho[e];
    if (a.act != CORR_ACT_NONE) {
        float z[V];
#pragma unroll
        for (int e = 0; e < V; ++e) z[e] = fmaf(x[e], k.w[e], k.b[e]);
        row_slope_all(a.act, z);
#pragma unroll
        for (int e = 0; e < V; ++e) g[e] *= z[e];
    }
}
// Sums over the workgroup's rows of dz hat and dz, channel by channel.
template <class T, int V>
__global__ __launch_bounds__(THREADS) void sums_kernel(GroupNormArgs a, int ct) {
    constexpr int U = 4;
    __shared__ float first[THREADS][V], second[THREADS][V];
    const Columns<V> at(a.C, ct);
    const int64_t lo = blockIdx.y * a.share, hi = min(a.P, lo + a.share), item = blockIdx.z * a.P;
    float hats[V] = {}, ones[V] = {};
    if (at.left > 0) {
        Channels<V> k;
        load_channels(a, blockIdx.z, at.c, k);
        const T* const x = (const T*)a.x + at.c;
        const T* const d = (const T*)a.d_y + at.c;
        for (int64_t r = lo + at.r0; r < hi; r += U * at.rt) {
            float v[U][V], g[U][V];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (r + u * at.rt < hi) {
                    load_some<T, V>(x + (item + r + u * at.rt) * a.x_stride, v[u], at.left);
                    load_some<T, V>(d + (item + r + u * at.rt) * a.d_y_stride, g[u], at.left);
                }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (r + u * at.rt >= hi) break;
                slopes<T>(a, k, v[u], g[u]);
#pragma unroll
                for (int e = 0; e < V; ++e) { hats[e] = fmaf(g[u][e], v[u][e], hats[e]); ones[e] += g[u][e]; }
            }
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) { first[threadIdx.x][e] = hats[e]; second[threadIdx.x][e] = ones[e]; }
    for (int half = at.rt / 2; half; half /= 2) {
        __syncthreads();
        if (at.r0 < half)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                first[threadIdx.x][e] = hats[e] += first[threadIdx.x + half * ct][e];
                second[threadIdx.x][e] = ones[e] += second[threadIdx.x + half * ct][e];
            }
    }
    if (at.r0 == 0 && at.left > 0) {
        float* const p = a.part + (int64_t)(blockIdx.z * a.parts + blockIdx.y) * 2 * a.C + at.c;
        store_some<float, V>(p, hats, at.left);
        store_some<float, V>(p + a.C, ones, at.left);
    }
}
// The parts of an item added in order: 16 channels a workgroup, 16 shares of the parts.
__global__ __launch_bounds__(THREADS) void join_kernel(GroupNormArgs a) {
    __shared__ float sums[16][16];
    const int col = threadIdx.x & 15, share = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
    const float* const p = a.part + ((int64_t)blockIdx.z * a.parts * 2 + blockIdx.y) * a.C + c;
    float sum = 0.f;
    if (c < a.C)
#pragma unroll 4
        for (int i = share; i < a.parts; i += 16) sum += p[(int64_t)i * 2 * a.C];
    sums[share][col] = sum;
    __syncthreads();
    if (share || c >= a.C) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) sum += sums[i][col];
    a.sums[((int64_t)blockIdx.z * 2 + blockIdx.y) * a.C + c] = sum;
    if (a.B == 1) {
        float* const out = blockIdx.y ? a.d_bias : a.d_weight;
        if (out) out[c] = sum;
    }
}
// d_x = rho (w dz - S1 / n - hat S2 / n), S1 and S2 the group's sums of w dz and w dz hat.  Each thread adds up its channels' groups by itself.
template <class T, int V>
__global__ __launch_bounds__(THREADS) void dx_kernel(GroupNormArgs a, int ct) {
    constexpr int U = 4;
    __shared__ float s1[THREADS * V], s2[THREADS * V];       // of the channels from the first column's group on: groups of this workgroup's columns
    const Columns<V> at(a.C, ct);
    const int width = a.C / a.G, c0 = blockIdx.x * ct * V, c1 = min(a.C, c0 + ct * V), g0 = c0 / width, groups = (c1 - 1) / width - g0 + 1;
    const float* const sums = a.sums + (int64_t)blockIdx.z * 2 * a.C;
    const float by = 1.f / ((float)a.P * (float)width);
    // 2^k neighbouring threads a group, as many as there are
    int team = 64;
    while (team > 1 && (team > width || groups * team > THREADS)) team /= 2;
    for (int g = threadIdx.x / team; g < (groups + THREADS / team - 1) / (THREADS / team) * (THREADS / team); g += THREADS / team) {
        float x = 0.f, y = 0.f;
        if (g < groups)
            for (int c = (g0 + g) * width + threadIdx.x % team; c < (g0 + g + 1) * width; c += team) {
                const float w = a.weight ? a.weight[c] : 1.f;
                x = fmaf(w, sums[a.C + c], x);
                y = fmaf(w, sums[c], y);
            }
        for (int s = 1; s < team; s *= 2) { x += __shfl_xor(x, s); y += __shfl_xor(y, s); }
        if (g < groups && threadIdx.x % team == 0) { s1[g] = x * by; s2[g] = y * by; }
    }
    __syncthreads();
    if (at.left <= 0) return;
    const int64_t lo = blockIdx.y * a.share, hi = min(a.P, lo + a.share), item = blockIdx.z * a.P;
    Channels<V> k;
    load_channels(a, blockIdx.z, at.c, k);
    float m1[V], m2[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int g = min(at.c + e, a.C - 1) / width - g0;
        m1[e] = s1[g];
        m2[e] = s2[g];
    }
    const T* const x = (const T*)a.x + at.c;
    const T* const d = (const T*)a.d_y + at.c;
    T* const out = (T*)a.d_x + at.c;
    for (int64_t r = lo + at.r0; r < hi; r += U * at.rt) {
        float v[U][V], g[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (r + u * at.rt < hi) {
                load_some<T, V>(x + (item + r + u * at.rt) * a.x_stride, v[u], at.left);
                load_some<T, V>(d + (item + r + u * at.rt) * a.d_y_stride, g[u], at.left);
            }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (r + u * at.rt >= hi) break;
            slopes<T>(a, k, v[u], g[u]);
#pragma unroll
            for (int e = 0; e < V; ++e) g[u][e] = k.rho[e] * (fmaf(k.w[e], g[u][e], -m1[e]) - v[u][e] * m2[e]);
            store_some<T, V>(out + (item + r + u * at.rt) * a.C, g[u], at.left);
        }
    }
}

template <class T, int V>
void forward(const GroupNormArgs& a, hipStream_t s) {
    const int ct = threads_across<V>(a.C);
    const dim3 grid((unsigned)cdiv(a.C, ct * V), a.parts, a.B);
    hipLaunchKernelGGL((stats_kernel<T, V>), grid, dim3(THREADS), 0, s, a, ct);
    hipLaunchKernelGGL(finish_stats_kernel, dim3(a.B * a.G), dim3(THREADS), 0, s, a);
    hipLaunchKernelGGL((apply_kernel<T, V>), grid, dim3(THREADS), 0, s, a, ct);
}
template <class T, int V>
void backward(const GroupNormArgs& a, hipStream_t s) {
    const int ct = threads_across<V>(a.C);
    const dim3 grid((unsigned)cdiv(a.C, ct * V), a.parts, a.B);
    hipLaunchKernelGGL((sums_kernel<T, V>), grid, dim3(THREADS), 0, s, a, ct);
    hipLaunchKernelGGL(join_kernel, dim3((a.C + 15) / 16, 2, a.B), dim3(THREADS), 0, s, a);
    if (a.d_x) hipLaunchKernelGGL((dx_kernel<T, V>), grid, dim3(THREADS), 0, s, a, ct);
}

}  // namespace

// Shares for eight workgroups on every compute unit, of 32 rows a thread at least (forward; four where there are few).
void group_norm_plan(GroupNormArgs& a, bool gradient) {
    const int V = a.type == CORR_TYPE_F32 ? 4 : 8, ct = V == 4 ? threads_across<4>(a.C) : threads_across<8>(a.C), rt = THREADS / ct;
    const int64_t across = cdiv(a.C, ct * V) * a.B, want = cdiv(2048, across), most = cdiv(a.P, 8 * rt);
    int64_t parts = want < most ? want : most;
    if (parts < 1) parts = 1;
    a.share = cdiv(a.P, parts);
    a.parts = (int)cdiv(a.P, a.share);
    (void)gradient;
}
hipError_t launch_group_norm(const GroupNormArgs& a, hipStream_t s) {
    if (a.type == CORR_TYPE_F32) forward<float, 4>(a, s);
    else if (a.type == CORR_TYPE_BF16) forward<__bf16, 8>(a, s);
    else forward<_Float16, 8>(a, s);
    return hipGetLastError();
}
hipError_t launch_group_norm_backward(const GroupNormArgs& a, hipStream_t s) {
    if (a.type == CORR_TYPE_F32) backward<float, 4>(a, s);
    else if (a.type == CORR_TYPE_BF16) backward<__bf16, 8>(a, s);
    else backward<_Float16, 8>(a, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.B == 1 || (!a.d_weight && !a.d_bias)) return e;
    const ColumnSums o = {{a.d_weight, a.d_bias, nullptr, nullptr, nullptr}};
    return launch_column_sums(a.sums, a.B, 2, a.C, o, s);
}
