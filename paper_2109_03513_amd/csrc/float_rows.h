// Rows of 16- and 32-bit floats in the decoder operators: element types, and loads and stores of
// eight consecutive elements at any element's alignment.
#pragma once

#include "esb_internal.h"

namespace esb {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

template <typename T> struct Vec8;
template <> struct Vec8<float> { typedef f32x8 type; };
template <> struct Vec8<__bf16> { typedef bf16x8 type; };
template <> struct Vec8<_Float16> { typedef f16x8 type; };

// The hardware reads and writes wide words at any address; the type says that the compiler may
// not assume more than the element's alignment (rows of odd length or pitch).
template <typename V, typename T> struct __attribute__((packed, aligned(alignof(T)))) Loose {
    V v;
};

// Elements p[0 .. n-1], zeros after them (n >= 8: all eight).
template <typename T>
__device__ __forceinline__ typename Vec8<T>::type load8(const T* p, int n) {
    typedef typename Vec8<T>::type V;
    if (n >= 8) return ((const Loose<V, T>*)p)->v;
    V r = {};
#pragma unroll
    for (int i = 0; i < 8; i++)
        if (i < n) r[i] = p[i];
    return r;
}

template <typename T>
__device__ __forceinline__ void store8(T* p, typename Vec8<T>::type v, int n) {
    typedef typename Vec8<T>::type V;
    if (n >= 8) {
        ((Loose<V, T>*)p)->v = v;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; i++)
        if (i < n) p[i] = v[i];
}

// Eight fp32 values to eight E4M3 bytes, rounded to nearest even (values of at most 448).
__device__ __forceinline__ uint2 to_e4m3(f32x8 v) {
    uint2 r;
    r.x = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
    r.x = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], r.x, true);
    r.y = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], 0, false);
    r.y = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], r.y, true);
    return r;
}

}  // namespace esb
