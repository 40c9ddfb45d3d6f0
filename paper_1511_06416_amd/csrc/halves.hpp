// Numbers as the sum of two fp16, for the kernels of orthogonalised updates.
#pragma once

#include <hip/hip_runtime.h>

namespace same {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// a, b to the nearest fp16 and what remains of them: two conversions of a pair
// and two multiply-adds that take fp16 as they are.
__device__ __forceinline__ void split(float a, float b, f16x2 &hi, f16x2 &lo) {
    hi = __builtin_convertvector(f32x2{a, b}, f16x2);
    lo = __builtin_convertvector(
        f32x2{__builtin_fmaf((float)hi[0], -1.0f, a), __builtin_fmaf((float)hi[1], -1.0f, b)}, f16x2);
}

// X in planes, sx G / (|G| + eps), of one number of G.  The factor lies between
// 2^-132 and 2^138 and passes 32 bits at both ends: its power of two comes first,
// exact where X is not below 2^-126 by then, so that one rounding is left.
struct PlaneFactor {
    float part;
    int power;
    __device__ __forceinline__ PlaneFactor() : part(0.0f), power(0) {}
    __device__ __forceinline__ PlaneFactor(float sx, double squares, float eps) {
        const double f = (double)sx / (__builtin_sqrt(squares) + (double)eps);
        part = (float)__builtin_amdgcn_frexp_mant(f);   // 0 stays 0, NaN NaN
        power = __builtin_amdgcn_frexp_exp(f);
    }
    __device__ __forceinline__ float operator()(float g) const { return __builtin_amdgcn_ldexpf(g, power) * part; }
};

// N numbers v(0), v(1), ...
template <int N, typename V, typename H>
__device__ __forceinline__ void split_all(V v, H &hi, H &lo) {
#pragma unroll
    for (int e = 0; e < N; e += 2) {
        f16x2 h, l;
        split(v(e), v(e + 1), h, l);
        hi[e] = h[0];
        hi[e + 1] = h[1];
        lo[e] = l[0];
        lo[e + 1] = l[1];
    }
}

}  // namespace same
