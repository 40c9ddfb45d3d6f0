// Exchanges within a wave and unaligned vectors, for the operators of a
// training step.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

namespace same {
namespace wave {

template <int CTRL, typename V>
__device__ __forceinline__ V moved(V v) {
    return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}

// An operation with the same lane of the other 16 of 32 lanes, or the other 32
// of 64: a swap of a value with its copy leaves both in every lane, in either
// order.  The copy must not share the value's register, or nothing is swapped.
template <int ROW, typename V, typename Op>
__device__ __forceinline__ V across(V v, Op op) {
    const uint32_t a = __builtin_bit_cast(uint32_t, v);
    uint32_t b = a;
    asm volatile("" : "+v"(b));
    const auto r = ROW == 16 ? __builtin_amdgcn_permlane16_swap(a, b, false, false)
                             : __builtin_amdgcn_permlane32_swap(a, b, false, false);
    return op(__builtin_bit_cast(V, (uint32_t)r[0]), __builtin_bit_cast(V, (uint32_t)r[1]));
}

// A commutative operation over the lanes of a group (a power of two of them),
// its result in every lane, bit for bit the same: exchanges of neighbours, of
// pairs, mirrored halves and rows of sixteen, then across rows.
template <typename V, typename Op>
__device__ __forceinline__ V reduce(V v, int lanes, Op op) {
    if (lanes > 1) v = op(v, moved<0xB1>(v));    // quad_perm 1,0,3,2
    if (lanes > 2) v = op(v, moved<0x4E>(v));    // quad_perm 2,3,0,1
    if (lanes > 4) v = op(v, moved<0x141>(v));   // row_half_mirror
    if (lanes > 8) v = op(v, moved<0x140>(v));   // row_mirror
    if (lanes > 16) v = across<16>(v, op);
    if (lanes > 32) v = across<32>(v, op);
    return v;
}
struct Add {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
struct Max {
    __device__ __forceinline__ float operator()(float a, float b) const { return __builtin_fmaxf(a, b); }
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};
struct Min {
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return a < b ? a : b; }
};

// Orders a wave's own LDS traffic, for the compiler too.
__device__ __forceinline__ void sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// N elements at any address: one access of the hardware all the same.
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Loose {
    T v[N];
};

}  // namespace wave
}  // namespace same
