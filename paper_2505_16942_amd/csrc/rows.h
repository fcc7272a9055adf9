// What the row operators (linear.hip, residual_norm.hip) share: element types, activations and their slopes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "corr.h"

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

static inline int corr_elem_bytes(corr_dtype t) { return t == CORR_TYPE_F32 ? 4 : 2; }

#ifdef __HIPCC__
// Activations in fp32.  e^x is v_exp_f32 of x log2 e (off by |x| 2^-24 relative, where the products that e^x meets are small), 1 / x
// v_rcp_f32 (1 ulp).  Where e^-z overflows, 1 / (1 + e^-z) is 0, as it should be.  A comparison keeps a NaN where fmaxf would drop it.
__device__ __forceinline__ float row_exp(float x) { return __builtin_amdgcn_exp2f(1.4426950408889634f * x); }
__device__ __forceinline__ float row_sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + row_exp(-z)); }
// e^-z / (1 + e^-z)^2 is even: from |z| no digits cancel (1 - sigmoid(z) has none left at z = 17, where the slope is 4e-8).
__device__ __forceinline__ float row_sigmoid_slope(float z) {
    const float e = row_exp(-fabsf(z)), r = __builtin_amdgcn_rcpf(1.f + e);
    return e * r * r;
}
// u of 0.5 z (1 + tanh u) = z sigmoid(2 u), times two
__device__ __forceinline__ float row_gelu_2u(float z) { return 1.5957691216057308f * fmaf(0.044715f * z * z, z, z); }
// The normal distribution's integral up to z, and `tail` = e^(-z^2/2).  The integral from |z| on is tail t P(t), t = 1 / (1 + 0.35 |z|): P, of
// degree eight, has the least relative error over t (3e-8, fitted on Chebyshev points), so that gelu keeps its digits where it dies away:
// off by (1.5 z^2 + 32) 2^-24 at most, relative, most of it from the exponent.  A polynomial that is good to 1.5e-7
// absolute (Abramowitz and Stegun 7.1.26) is 5e-5 off at z = -3, 1.6e-3 at -5.  The library's erff has two branches, and a wave takes
// both: 32400 x 1024 outputs took 122 us with it.
__device__ __forceinline__ float row_normal(float z, float& tail) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.35f, fabsf(z), 1.f));
    tail = __builtin_amdgcn_exp2f(-0.72134752044448170f * (z * z));
    float q = fmaf(t, -0.02914595525f, 0.1439718181f);
    q = fmaf(t, q, -0.2557145002f);
    q = fmaf(t, q, 0.1591744381f);
    q = fmaf(t, q, -0.02311002419f);
    q = fmaf(t, q, 0.1055080832f);
    q = fmaf(t, q, 0.1198328478f);
    q = fmaf(t, q, 0.1398618724f);
    q = fmaf(t, q, 0.1396214041f) * t * tail;
    return z < 0.f ? q : 1.f - q;
}
__device__ __forceinline__ float row_act(int act, float z) {
    switch (act) {
        case CORR_ACT_RELU: return z < 0.f ? 0.f : z;
        case CORR_ACT_GELU: { float tail; return z * row_normal(z, tail); }
        case CORR_ACT_GELU_TANH: return z * row_sigmoid(row_gelu_2u(z));
        case CORR_ACT_SILU: return z * row_sigmoid(z);
        case CORR_ACT_SIGMOID: return row_sigmoid(z);
    }
    return z;
}
__device__ __forceinline__ float row_act_slope(int act, float z) {
    switch (act) {
        case CORR_ACT_RELU: return z > 0.f ? 1.f : 0.f;
        case CORR_ACT_GELU: {
            float tail;
            const float p = row_normal(z, tail);
            return fmaf(z * tail, 0.39894228040143268f, p);
        }
        case CORR_ACT_GELU_TANH: {
            // where z^2 overflows s (1 - s) is zero, and has to stay it: a finite factor (a NaN is in s too)
            const float s = row_sigmoid(row_gelu_2u(z)), d2u = fminf(1.5957691216057308f * fmaf(0.134145f * z, z, 1.f), 3e38f);
            return fmaf(z * (s * (1.f - s)), d2u, s);
        }
        case CORR_ACT_SILU: { const float s = row_sigmoid(z); return s * fmaf(z, 1.f - s, 1.f); }
        case CORR_ACT_SIGMOID: return row_sigmoid_slope(z);
    }
    return 1.f;
}
// V values at once: the choice is made once, and their chains of dependent instructions overlap.
template <int V, class F> __device__ __forceinline__ void row_each(float (&v)[V], F f) {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = f(v[e]);
}
template <int V> __device__ __forceinline__ void row_act_all(int act, float (&v)[V]) {
    switch (act) {
        case CORR_ACT_RELU: row_each(v, [](float z) { return row_act(CORR_ACT_RELU, z); }); break;
        case CORR_ACT_GELU: row_each(v, [](float z) { return row_act(CORR_ACT_GELU, z); }); break;
        case CORR_ACT_GELU_TANH: row_each(v, [](float z) { return row_act(CORR_ACT_GELU_TANH, z); }); break;
        case CORR_ACT_SILU: row_each(v, [](float z) { return row_act(CORR_ACT_SILU, z); }); break;
        case CORR_ACT_SIGMOID: row_each(v, [](float z) { return row_act(CORR_ACT_SIGMOID, z); }); break;
    }
}
template <int V> __device__ __forceinline__ void row_slope_all(int act, float (&v)[V]) {
    switch (act) {
        case CORR_ACT_RELU: row_each(v, [](float z) { return row_act_slope(CORR_ACT_RELU, z); }); break;
        case CORR_ACT_GELU: row_each(v, [](float z) { return row_act_slope(CORR_ACT_GELU, z); }); break;
        case CORR_ACT_GELU_TANH: row_each(v, [](float z) { return row_act_slope(CORR_ACT_GELU_TANH, z); }); break;
        case CORR_ACT_SILU: row_each(v, [](float z) { return row_act_slope(CORR_ACT_SILU, z); }); break;
        case CORR_ACT_SIGMOID: row_each(v, [](float z) { return row_act_slope(CORR_ACT_SIGMOID, z); }); break;
        default: row_each(v, [](float) { return 1.f; });
    }
}

// V consecutive elements of type T as fp32 and back (rounded to nearest even), as one access of V * sizeof(T) bytes.
template <class T, int V> struct RowVec {
    typedef T value __attribute__((ext_vector_type(V)));
    typedef value type __attribute__((aligned(V * sizeof(T) < 16 ? V * sizeof(T) : 16)));   // two accesses of 16 bytes ask for no more
};
template <class T> struct RowVec<T, 1> { typedef T type; };
template <class T, int V>
__device__ __forceinline__ void row_load(const T* p, float (&v)[V]) {
    if constexpr (V == 1) v[0] = (float)*p;
    else {
        const typename RowVec<T, V>::type x = *reinterpret_cast<const typename RowVec<T, V>::type*>(p);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (float)x[i];
    }
}
template <class T, int V>
__device__ __forceinline__ void row_store(T* p, const float (&v)[V]) {
    if constexpr (V == 1) *p = (T)v[0];
    else {
        typename RowVec<T, V>::type x;
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (T)v[i];
        *reinterpret_cast<typename RowVec<T, V>::type*>(p) = x;
    }
}
#endif

// out[v][c] = sum over p of part[p][v][c] (rows.hip): the last step of every column sum.  out[v] may be null.
struct ColumnSums { float* out[5]; };
hipError_t launch_column_sums(const float* part, int parts, int vectors, int C, const ColumnSums& o, hipStream_t s);
// zeros of a multiple of two bytes
hipError_t launch_zero(void* p, size_t bytes, hipStream_t s);
