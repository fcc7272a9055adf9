// Norms before and after a block, with the block's gate, its scale and the residual, and their gradient:
//   p = norm1(y) w1 + b1,   t = alpha h + s act(g) p   (h_out),   n = norm2(t) w2 + b2.
// A row's elements stay in the registers of G threads from its only load to its only store; sums over a row go through the
// lanes of a wave and, for rows that need more than a wave, LDS.  Means and squares in fp32; the layer norm subtracts the mean
// before it squares.  The gradient makes the forward pass's row again from the forward pass's inputs (as many bytes as
// reading saved ones) and keeps the sums over rows of its columns in registers from row to row.
#include "rows_internal.h"

namespace {

enum { V_SCALE, V_W1, V_B1, V_W2, V_B2, VECTORS };

// Sums over the G threads of a row.  Waves of one row add up in LDS (two buffers in turn: a wave may be one sum ahead of
// another, never two).
template <int G>
struct RowSum {
    float2* lds;
    int turn;
    __device__ __forceinline__ float2 operator()(float x, float y) {
        constexpr int WIDTH = G < 64 ? G : 64;
#pragma unroll
        for (int d = WIDTH / 2; d > 0; d >>= 1) {
            x += __shfl_xor(x, d);
            y += __shfl_xor(y, d);
        }
        if constexpr (G > 64) {
            constexpr int WAVES = G / 64;
            float2* const b = lds + (turn ^= 1) * WAVES;
            if ((threadIdx.x & 63) == 0) b[threadIdx.x >> 6] = make_float2(x, y);
            __syncthreads();
            x = y = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) { x += b[w].x; y += b[w].y; }
        }
        return make_float2(x, y);
    }
};

// E elements of a row per thread, in pieces of V: element e of thread j is column ((e / V) * G + j) * V + e % V.
template <int G, int E, int V>
struct Cols {
    int j, C;
    __device__ __forceinline__ int at(int piece) const { return (piece * G + j) * V; }
    template <class T> __device__ __forceinline__ void load(const T* row, float (&v)[E]) const {
#pragma unroll
        for (int q = 0; q < E / V; ++q) {
            float x[V] = {};
            if (at(q) < C) row_load<T, V>(row + at(q), x);
#pragma unroll
            for (int e = 0; e < V; ++e) v[q * V + e] = x[e];
        }
    }
    template <class T> __device__ __forceinline__ void store(T* row, const float (&v)[E]) const {
#pragma unroll
        for (int q = 0; q < E / V; ++q) {
            float x[V];
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = v[q * V + e];
            if (at(q) < C) row_store<T, V>(row + at(q), x);
        }
    }
    // a vector of parameters; `none` where there is none
    __device__ __forceinline__ void vector(const float* p, float none, float (&v)[E]) const {
        if (p) load<float>(p, v);
        else
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = none;
    }
    __device__ __forceinline__ bool in(int e) const { return at(e / V) < C; }
};

// v becomes the normalised row; returns 1 / its spread (1 for CORR_NORM_NONE).  Elements past the row's end stay zero.
template <int G, int E, int V>
__device__ __forceinline__ float normalise(int kind, float (&v)[E], const Cols<G, E, V>& c, float inv, float eps, RowSum<G>& sum) {
    if (kind == CORR_NORM_NONE) return 1.f;
    if (kind == CORR_NORM_LAYER) {
        float m = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) m += v[e];
        const float mean = sum(m, 0.f).x * inv;
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = c.in(e) ? v[e] - mean : 0.f;
    }
    float q = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) q = fmaf(v[e], v[e], q);
    const float rho = 1.f / sqrtf(sum(q, 0.f).x * inv + eps);
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] *= rho;
    return rho;
}
// q, the gradient of the normalised row `hat`, becomes the gradient of the row.
template <int G, int E, int V>
__device__ __forceinline__ void normalise_back(int kind, float (&q)[E], const float (&hat)[E], float rho, const Cols<G, E, V>& c, float inv,
                                               RowSum<G>& sum) {
    if (kind == CORR_NORM_NONE) return;
    float a = 0.f, b = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) { a = fmaf(q[e], hat[e], a); b += q[e]; }
    const float2 s = sum(a, b);
    const float along = s.x * inv, mean = kind == CORR_NORM_LAYER ? s.y * inv : 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) q[e] = c.in(e) ? rho * (q[e] - mean - hat[e] * along) : 0.f;
}

template <class S, class T, int G, int E, int V>
__global__ __launch_bounds__(G < 256 ? 256 : G) void residual_norm_kernel(NormArgs n) {
    constexpr int THREADS = G < 256 ? 256 : G, GROUPS = THREADS / G;
    constexpr bool KEEP = E <= 8;                        // vectors stay in registers from row to row
    __shared__ float2 lds[G > 64 ? 2 * (G / 64) : 1];
    const corr_residual_norm_args& a = n.a;
    const Cols<G, E, V> c = {(int)threadIdx.x % G, (int)a.cols};
    const float inv = 1.f / (float)a.cols;
    RowSum<G> sum = {lds, 0};
    float s[E], w1[E], b1[E], w2[E], b2[E];
    if (KEEP) {
        c.vector(a.scale, 1.f, s);
        c.vector(a.post_weight, 1.f, w1); c.vector(a.post_bias, 0.f, b1);
        c.vector(a.pre_weight, 1.f, w2); c.vector(a.pre_bias, 0.f, b2);
    }
    for (int64_t r = (int64_t)blockIdx.x * GROUPS + threadIdx.x / G; r < a.rows; r += (int64_t)gridDim.x * GROUPS) {
        float t[E];
        c.load((const S*)a.h + r * a.h_stride, t);
        if (a.y) {
            float p[E];
            c.load((const T*)a.y + r * a.y_stride, p);
            float g[E];
            if (a.gate) c.load((const T*)a.gate + r * a.gate_stride, g);
            normalise(a.post, p, c, inv, a.eps, sum);
            if (!KEEP) { c.vector(a.post_weight, 1.f, w1); c.vector(a.post_bias, 0.f, b1); c.vector(a.scale, 1.f, s); }
#pragma unroll
            for (int e = 0; e < E; ++e) p[e] = fmaf(p[e], w1[e], b1[e]) * s[e];
            if (a.gate) {
                row_act_all(a.gate_act, g);
#pragma unroll
                for (int e = 0; e < E; ++e) p[e] *= g[e];
            }
#pragma unroll
            for (int e = 0; e < E; ++e) t[e] = c.in(e) ? fmaf(a.h_scale, t[e], p[e]) : 0.f;
            if (n.h_out) c.store((S*)n.h_out + r * a.cols, t);
        }
        if (a.pre != CORR_NORM_NONE) {
            normalise(a.pre, t, c, inv, a.eps, sum);
            if (!KEEP) { c.vector(a.pre_weight, 1.f, w2); c.vector(a.pre_bias, 0.f, b2); }
#pragma unroll
            for (int e = 0; e < E; ++e) t[e] = fmaf(t[e], w2[e], b2[e]);
            c.store((T*)n.n_out + r * a.cols, t);
        }
    }
}

// Rows past 8192 columns leave no registers for the columns' sums: they are added up in the workgroup's own part, in memory.
template <class S, class T, int G, int E, int V>
__global__ __launch_bounds__(G < 256 ? 256 : G) void residual_norm_backward_kernel(NormArgs n) {
    constexpr int THREADS = G < 256 ? 256 : G, GROUPS = THREADS / G;
    constexpr bool KEEP = E <= 4, IN_MEMORY = E > 8 && G >= 1024;
    __shared__ float2 lds[G > 64 ? 2 * (G / 64) : 1];
    __shared__ float join[GROUPS > 1 ? (GROUPS - 1) * G * E : 1];
    const corr_residual_norm_args& a = n.a;
    const Cols<G, E, V> c = {(int)threadIdx.x % G, (int)a.cols};
    const int group = threadIdx.x / G;
    const float inv = 1.f / (float)a.cols;
    RowSum<G> sum = {lds, 0};
    float s[E], w1[E], b1[E], w2[E];
    if (KEEP) {
        c.vector(a.scale, 1.f, s);
        c.vector(a.post_weight, 1.f, w1); c.vector(a.post_bias, 0.f, b1);
        c.vector(a.pre_weight, 1.f, w2);
    }
    float* const part = n.part ? n.part + (int64_t)blockIdx.x * VECTORS * a.cols : nullptr;
    float acc[IN_MEMORY ? 1 : VECTORS][E] = {};
    bool first = true;
    auto add = [&](int v, auto value) {                  // value(e), summed over rows
        if constexpr (IN_MEMORY) {
            if (!part) return;
            float x[E] = {};
            float* const row = part + (int64_t)v * a.cols;
            if (!first) c.load(row, x);
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] += value(e);
            c.store(row, x);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) acc[v][e] += value(e);
        }
    };
    for (int64_t r = (int64_t)blockIdx.x * GROUPS + group; r < a.rows; r += (int64_t)gridDim.x * GROUPS) {
        float t[E], p[E], g[E], D[E];
        c.load((const S*)a.h + r * a.h_stride, t);
        float rho1 = 1.f;
        if (a.y) {
            c.load((const T*)a.y + r * a.y_stride, p);
            if (a.gate) c.load((const T*)a.gate + r * a.gate_stride, g);
        }
        if (n.d_n_out) c.load((const T*)n.d_n_out + r * a.cols, D);
        if (a.y) {
            rho1 = normalise(a.post, p, c, inv, a.eps, sum);
            if (!KEEP) { c.vector(a.post_weight, 1.f, w1); c.vector(a.post_bias, 0.f, b1); c.vector(a.scale, 1.f, s); }
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float u = fmaf(p[e], w1[e], b1[e]) * s[e] * (a.gate ? row_act(a.gate_act, g[e]) : 1.f);
                t[e] = c.in(e) ? fmaf(a.h_scale, t[e], u) : 0.f;
            }
        }
        if (n.d_n_out) {
            const float rho2 = normalise(a.pre, t, c, inv, a.eps, sum);
            if (a.pre_weight) add(V_W2, [&](int e) { return D[e] * t[e]; });
            if (a.pre_bias) add(V_B2, [&](int e) { return D[e]; });
            if (!KEEP) c.vector(a.pre_weight, 1.f, w2);
#pragma unroll
            for (int e = 0; e < E; ++e) D[e] *= w2[e];
            normalise_back(a.pre, D, t, rho2, c, inv, sum);
            if (n.d_h_out) {
                float x[E];
                c.load((const S*)n.d_h_out + r * a.cols, x);
#pragma unroll
                for (int e = 0; e < E; ++e) D[e] += x[e];
            }
        } else {
            c.load((const S*)n.d_h_out + r * a.cols, D);
            if (IN_MEMORY && first) {                    // nothing reaches these: zeros
                add(V_W2, [](int) { return 0.f; });
                add(V_B2, [](int) { return 0.f; });
            }
        }
        const float alpha = a.y ? a.h_scale : 1.f;
        if (n.d_h) {
            float x[E];
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = alpha * D[e];
            c.store((S*)n.d_h + r * a.cols, x);
        }
        if (a.y) {
            // from here on t holds act(g), D the gradient of s act(g) p
            if (a.gate) {
#pragma unroll
                for (int e = 0; e < E; ++e) t[e] = row_act(a.gate_act, g[e]);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) t[e] = 1.f;
            }
            if (a.scale) {
                add(V_SCALE, [&](int e) { return D[e] * t[e] * fmaf(p[e], w1[e], b1[e]); });
#pragma unroll
                for (int e = 0; e < E; ++e) D[e] *= s[e];
            }
            if (n.d_gate) {
                float x[E];
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] = D[e] * fmaf(p[e], w1[e], b1[e]) * row_act_slope(a.gate_act, g[e]);
                c.store((T*)n.d_gate + r * a.cols, x);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) D[e] *= t[e];
            if (a.post_weight) add(V_W1, [&](int e) { return D[e] * p[e]; });
            if (a.post_bias) add(V_B1, [&](int e) { return D[e]; });
#pragma unroll
            for (int e = 0; e < E; ++e) D[e] *= w1[e];
            normalise_back(a.post, D, p, rho1, c, inv, sum);
            if (n.d_y) c.store((T*)n.d_y + r * a.cols, D);
        }
        first = false;
    }
    if (!part) return;
    if constexpr (!IN_MEMORY) {
#pragma unroll
        for (int v = 0; v < VECTORS; ++v) {
            if constexpr (GROUPS > 1) {
                __syncthreads();
                if (group) {
#pragma unroll
                    for (int e = 0; e < E; ++e) join[((group - 1) * E + e) * G + c.j] = acc[v][e];
                }
                __syncthreads();
                if (!group)
                    for (int o = 0; o < GROUPS - 1; ++o)
#pragma unroll
                        for (int e = 0; e < E; ++e) acc[v][e] += join[(o * E + e) * G + c.j];
            }
            if (!group) c.store(part + (int64_t)v * a.cols, acc[v]);
        }
    }
}

// Rows of up to `cols` columns in pieces of V.
template <class S, class T, bool BACK, int G, int E, int V>
void run(const NormArgs& n, hipStream_t s) {
    constexpr int THREADS = G < 256 ? 256 : G, GROUPS = THREADS / G;
    const int64_t need = (n.a.rows + GROUPS - 1) / GROUPS;
    if (BACK) hipLaunchKernelGGL((residual_norm_backward_kernel<S, T, G, E, V>), dim3(n.parts), dim3(THREADS), 0, s, n);
    else {
        const int64_t most = 2048 * 256 / THREADS;
        hipLaunchKernelGGL((residual_norm_kernel<S, T, G, E, V>), dim3((unsigned)(need < most ? need : most)), dim3(THREADS), 0, s, n);
    }
}
template <class S, class T, bool BACK>
void run(const NormArgs& n, bool wide, hipStream_t s) {
    const int64_t C = n.a.cols;
    if (wide) {
        if (C <= 64) run<S, T, BACK, 16, 4, 4>(n, s);
        else if (C <= 256) run<S, T, BACK, 64, 4, 4>(n, s);
        else if (C <= 512) run<S, T, BACK, 64, 8, 8>(n, s);
        else if (C <= 1024) run<S, T, BACK, 256, 4, 4>(n, s);
        else if (C <= 2048) run<S, T, BACK, 256, 8, 8>(n, s);
        else if (C <= 4096) run<S, T, BACK, 512, 8, 8>(n, s);
        else if (C <= 8192) run<S, T, BACK, 1024, 8, 8>(n, s);
        else run<S, T, BACK, 1024, 16, 8>(n, s);
    } else {
        if (C <= 256) run<S, T, BACK, 64, 4, 1>(n, s);
        else if (C <= 1024) run<S, T, BACK, 256, 4, 1>(n, s);
        else if (C <= 8192) run<S, T, BACK, 1024, 8, 1>(n, s);
        else run<S, T, BACK, 1024, 16, 1>(n, s);
    }
}
template <bool BACK>
hipError_t launch(const NormArgs& n, hipStream_t s) {
    const corr_residual_norm_args& a = n.a;
    // eight elements at once: rows of whole pieces that start on the border of every access (16 bytes, the widest)
    const uintptr_t all = (uintptr_t)a.h | (uintptr_t)a.y | (uintptr_t)a.gate | (uintptr_t)a.scale | (uintptr_t)a.post_weight |
                          (uintptr_t)a.post_bias | (uintptr_t)a.pre_weight | (uintptr_t)a.pre_bias | (uintptr_t)n.h_out | (uintptr_t)n.n_out |
                          (uintptr_t)n.d_h_out | (uintptr_t)n.d_n_out | (uintptr_t)n.d_h | (uintptr_t)n.d_y | (uintptr_t)n.d_gate;
    const bool wide = (all & 15) == 0 && ((a.cols | a.h_stride | a.y_stride | a.gate_stride) & 7) == 0;
    if (a.stream_type == CORR_TYPE_F32) {
        if (a.type == CORR_TYPE_F32) run<float, float, BACK>(n, wide, s);
        else if (a.type == CORR_TYPE_BF16) run<float, __bf16, BACK>(n, wide, s);
        else run<float, _Float16, BACK>(n, wide, s);
    } else if (a.type == CORR_TYPE_BF16) run<__bf16, __bf16, BACK>(n, wide, s);
    else run<_Float16, _Float16, BACK>(n, wide, s);
    return hipGetLastError();
}

}  // namespace

int norm_backward_parts(int64_t rows, int64_t cols) {
    const int64_t per = cols <= 64 ? 16 : cols <= 512 ? 4 : 1;      // rows a workgroup has at a time (a lower bound)
    const int64_t most = cols <= 1024 ? 1024 : 512, need = (rows + per - 1) / per;
    return (int)(need < most ? need : most);
}
hipError_t launch_residual_norm(const NormArgs& n, hipStream_t s) { return launch<false>(n, s); }
hipError_t launch_residual_norm_backward(const NormArgs& n, hipStream_t s) { return launch<true>(n, s); }
