// What blocks of orthogonalised updates share that hold columns of X in
// registers and small products in LDS.
#pragma once

#include "halves.hpp"
#include "wave.hpp"

namespace same {

__device__ __forceinline__ f32x16 mfma(f16x8 l, f16x8 r, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(l, r, c, 0, 0, 0);
}

__device__ __forceinline__ f32x16 zero16() {
    f32x16 z;
#pragma unroll
    for (int e = 0; e < 16; ++e) z[e] = 0.0f;
    return z;
}

// Four rows of a column go to LDS, lane i's column beside lane i ^ 1's: the two
// exchange halves, and each writes two rows of both columns.  `to`: row 2 (i & 1)
// of the four, the even column.
__device__ __forceinline__ void write_rows(_Float16 *to, int pitch, f16x2 first, f16x2 last) {
    const bool odd = threadIdx.x & 1;
    const uint32_t a = __builtin_bit_cast(uint32_t, first), b = __builtin_bit_cast(uint32_t, last);
    const uint32_t other = wave::moved<0xB1>(odd ? a : b), own = odd ? b : a;
    *(uint32_t *)to = __builtin_amdgcn_perm(other, own, odd ? 0x01000504 : 0x05040100);
    *(uint32_t *)(to + pitch) = __builtin_amdgcn_perm(other, own, odd ? 0x03020706 : 0x07060302);
}

// A 32 x 32 product leaves a lane with the rows 8 q + 4 (lane / 32) + e of a
// column.  Two of the fours, q even and q + 1, become the eight rows from
// 8 (q + lane / 32) on, or such eight become two fours again.
__device__ __forceinline__ void exchange(f16x4 &even, f16x4 &odd) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    u32x2 a = __builtin_bit_cast(u32x2, even), b = __builtin_bit_cast(u32x2, odd);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        uint32_t to = a[w], from = b[w];
        asm volatile("" : "+v"(to), "+v"(from));   // registers of their own
        const auto r = __builtin_amdgcn_permlane32_swap(to, from, false, false);
        a[w] = r[0];
        b[w] = r[1];
    }
    even = __builtin_bit_cast(f16x4, a);
    odd = __builtin_bit_cast(f16x4, b);
}
union Eight {
    f16x4 h[2];
    f16x8 v;
};
// Sixteen numbers v(0), v(1), ... of a product's column to LDS, 16 bytes at a time: as a
// row; or a lane's own eight together, fours q and q + STEP, the order that B X takes.
// All pointers stand at 8 (lane / 32) of the row.
template <typename V>
__device__ __forceinline__ void write_row(_Float16 *hi, _Float16 *lo, V v) {
#pragma unroll
    for (int q = 0; q < 4; q += 2) {
        Eight h, l;
        split_all<4>([&](int e) { return v(4 * q + e); }, h.h[0], l.h[0]);
        split_all<4>([&](int e) { return v(4 * q + 4 + e); }, h.h[1], l.h[1]);
        exchange(h.h[0], h.h[1]);
        exchange(l.h[0], l.h[1]);
        *(f16x8 *)(hi + 8 * q) = h.v;
        *(f16x8 *)(lo + 8 * q) = l.v;
    }
}
template <int STEP, typename V>
__device__ __forceinline__ void write_own(_Float16 *hi, _Float16 *lo, V v) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int q = STEP == 1 ? 2 * r : r;
        Eight h, l;
        split_all<4>([&](int e) { return v(4 * q + e); }, h.h[0], l.h[0]);
        split_all<4>([&](int e) { return v(4 * (q + STEP) + e); }, h.h[1], l.h[1]);
        *(f16x8 *)(hi + 16 * r) = h.v;
        *(f16x8 *)(lo + 16 * r) = l.v;
    }
}
// v = take v + keep (hi + lo), of what write_row wrote.
template <typename V>
__device__ __forceinline__ void add_row(const _Float16 *hi, const _Float16 *lo, float take, float keep, V &v) {
#pragma unroll
    for (int q = 0; q < 4; q += 2) {
        Eight h, l;
        h.v = *(const f16x8 *)(hi + 8 * q);
        l.v = *(const f16x8 *)(lo + 8 * q);
        exchange(h.h[0], h.h[1]);
        exchange(l.h[0], l.h[1]);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[4 * q + e] = __builtin_fmaf(take, v[4 * q + e], keep * ((float)h.v[e] + (float)l.v[e]));
    }
}

// acc += C[a][b], a = a0 + GROUPS t, of three products over `depth` columns
// (a multiple of 32) of rows of `pitch` numbers: 32 x 32 a tile.
template <int NT, int GROUPS, int MINE>
__device__ __forceinline__ void add_products(f32x16 (&acc)[MINE], const _Float16 *hi, const _Float16 *lo, int pitch,
                                             int depth, int a0, int b) {
    const int row = threadIdx.x & 31, half = (threadIdx.x >> 5) & 1;
    struct Operands {
        f16x8 r_hi, r_lo, l_hi[MINE], l_lo[MINE];
    } now, then;
    auto load = [&](Operands &o, int k) {
        const int at_b = (32 * b + row) * pitch + 8 * half + k;
        o.r_hi = *(const f16x8 *)&hi[at_b];
        o.r_lo = *(const f16x8 *)&lo[at_b];
#pragma unroll
        for (int t = 0; t < MINE; ++t) {
            const int at = (32 * min(a0 + t * GROUPS, NT - 1) + row) * pitch + 8 * half + k;
            o.l_hi[t] = *(const f16x8 *)&hi[at];
            o.l_lo[t] = *(const f16x8 *)&lo[at];
        }
        __builtin_amdgcn_sched_barrier(0);   // before the products of the other
    };
    auto multiply = [&](const Operands &o) {   // products of one sum apart from each other
#pragma unroll
        for (int t = 0; t < MINE; ++t) acc[t] = mfma(o.l_lo[t], o.r_hi, acc[t]);
#pragma unroll
        for (int t = 0; t < MINE; ++t) acc[t] = mfma(o.l_hi[t], o.r_lo, acc[t]);
#pragma unroll
        for (int t = 0; t < MINE; ++t) acc[t] = mfma(o.l_hi[t], o.r_hi, acc[t]);
        __builtin_amdgcn_sched_barrier(0);
    };
    load(now, 0);
    for (int k = 0; k < depth; k += 32) {
        load(then, k + 16);
        multiply(now);
        if (k + 32 < depth) load(now, k + 32);
        multiply(then);
    }
}

// x <- keep x + B x / sb for 16 columns a wave, x in 16 x 16 tiles; B's columns
// in LDS in the order of write_own<2>.
template <int NT>
__device__ __forceinline__ void update_strip(f32x4 (&x)[2 * NT], const _Float16 *hi, const _Float16 *lo, int pitch,
                                             float keep, float take) {
    const int col = threadIdx.x & 15, quarter = (threadIdx.x >> 4) & 3;
    // x's halves are formed here, not kept since they went to LDS
#pragma unroll
    for (int t = 0; t < 2 * NT; ++t) asm volatile("" : "+v"(x[t]));
    f32x4 sum[2 * NT];
#pragma unroll
    for (int t = 0; t < 2 * NT; ++t) sum[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < NT; ++k) {
        f16x8 x_hi, x_lo;
        split_all<8>([&](int e) { return x[2 * k + (e >> 2)][e & 3]; }, x_hi, x_lo);
        f16x8 l_hi[2 * NT], l_lo[2 * NT];
#pragma unroll
        for (int t = 0; t < 2 * NT; ++t) {
            const int at = (16 * t + col) * pitch + 32 * k + 8 * quarter;
            l_hi[t] = *(const f16x8 *)&hi[at];
            l_lo[t] = *(const f16x8 *)&lo[at];
        }
#pragma unroll
        for (int t = 0; t < 2 * NT; ++t) sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(l_lo[t], x_hi, sum[t], 0, 0, 0);
#pragma unroll
        for (int t = 0; t < 2 * NT; ++t) sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(l_hi[t], x_lo, sum[t], 0, 0, 0);
#pragma unroll
        for (int t = 0; t < 2 * NT; ++t) sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(l_hi[t], x_hi, sum[t], 0, 0, 0);
    }
#pragma unroll
    for (int t = 0; t < 2 * NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[t][e] = __builtin_fmaf(sum[t][e], take, keep * x[t][e]);
}

// x to LDS, row by row: to column 16 wave + lane % 16 of rows of `pitch` numbers.
template <int NT>
__device__ __forceinline__ void write_strip(const f32x4 (&x)[2 * NT], _Float16 *hi, _Float16 *lo, int pitch) {
    const int lane = threadIdx.x & 63, column = 16 * (threadIdx.x >> 6) + (lane & 15);
    const int first = (4 * (lane >> 4) + 2 * (lane & 1)) * pitch + (column & ~1);
#pragma unroll
    for (int t = 0; t < 2 * NT; ++t) {
        f16x2 h[2], l[2];
        split(x[t][0], x[t][1], h[0], l[0]);
        split(x[t][2], x[t][3], h[1], l[1]);
        write_rows(hi + 16 * t * pitch + first, pitch, h[0], h[1]);
        write_rows(lo + 16 * t * pitch + first, pitch, l[0], l[1]);
    }
}

}  // namespace same
