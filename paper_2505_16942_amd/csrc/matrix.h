// What the kernels on the matrix cores (linear.hip, attention.hip) share: fragments, loads that land in LDS, pieces of rows.
#pragma once
#include "rows.h"

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) unsigned char lds_byte;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
template <class T> struct Frag;
template <> struct Frag<__bf16> { typedef bf16x8 type; };
template <> struct Frag<_Float16> { typedef f16x8 type; };

// 16 bytes per lane from a buffer straight into LDS at lds + lane * 16.  A lane whose offset lies beyond the resource's size
// writes zeros.
__device__ __forceinline__ void dma16(i32x4 rsrc, unsigned lds, unsigned voff) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :: "s"(lds), "v"(voff), "s"(rsrc) : "memory");
}
// Everything this wave has asked for has arrived, then everything every wave has: the next tile can be read, and the
// reads of the last one are over.
__device__ __forceinline__ void arrive_all() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// V elements of a row at a time, as far as they go, wherever the row begins (vector accesses need no border).
template <class T, int V> struct Some { typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T)))); };
// `past`: past the caches
template <class T, int V>
__device__ __forceinline__ void store_some(T* p, const float (&v)[V], int left, bool past = false) {
    if (left >= V) {
        typename Some<T, V>::type x;
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = (T)v[e];
        if (past) __builtin_nontemporal_store(x, reinterpret_cast<typename Some<T, V>::type*>(p));
        else *reinterpret_cast<typename Some<T, V>::type*>(p) = x;
    } else
#pragma unroll
        for (int e = 0; e < V; ++e) if (e < left) p[e] = (T)v[e];
}
template <class T, int V>
__device__ __forceinline__ void load_some(const T* p, float (&v)[V], int left) {
    if (left >= V) {
        const typename Some<T, V>::type x = *reinterpret_cast<const typename Some<T, V>::type*>(p);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = (float)x[e];
    } else
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = e < left ? (float)p[e] : 0.f;
}

}  // namespace
