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
// Activations in fp32.  1 / (1 + e^-z) by v_rcp_f32 (1 ulp); where e^-z overflows the quotient is 0, as it should be.
// A comparison keeps a NaN where fmaxf would drop it.
__device__ __forceinline__ float row_sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + expf(-z)); }
// u of 0.5 z (1 + tanh u) = z sigmoid(2 u), times two
__device__ __forceinline__ float row_gelu_2u(float z) { return 1.5957691216057308f * fmaf(0.044715f * z * z, z, z); }
__device__ __forceinline__ float row_act(int act, float z) {
    switch (act) {
        case CORR_ACT_RELU: return z < 0.f ? 0.f : z;
        case CORR_ACT_GELU: return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
        case CORR_ACT_GELU_TANH: return z * row_sigmoid(row_gelu_2u(z));
        case CORR_ACT_SILU: return z * row_sigmoid(z);
        case CORR_ACT_SIGMOID: return row_sigmoid(z);
    }
    return z;
}
__device__ __forceinline__ float row_act_slope(int act, float z) {
    switch (act) {
        case CORR_ACT_RELU: return z > 0.f ? 1.f : 0.f;
        case CORR_ACT_GELU:
            return fmaf(z * expf(-0.5f * z * z), 0.39894228040143268f, 0.5f * (1.f + erff(z * 0.70710678118654752f)));
        case CORR_ACT_GELU_TANH: {
            const float s = row_sigmoid(row_gelu_2u(z));
            return fmaf(z * s * (1.f - s), 1.5957691216057308f * fmaf(0.134145f * z, z, 1.f), s);
        }
        case CORR_ACT_SILU: { const float s = row_sigmoid(z); return s * fmaf(z, 1.f - s, 1.f); }
        case CORR_ACT_SIGMOID: { const float s = row_sigmoid(z); return s * (1.f - s); }
    }
    return 1.f;
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
