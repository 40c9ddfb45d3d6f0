// Orthogonalised updates that one block holds, for gfx950: smaller sides of 33
// to 96 with larger ones up to 256, and up to 128 x 128.  The products and their two fp16
// a number are those of orthogonalise.hip, all three for every type, without a
// launch or a trip to memory between.
//
// A wave owns 32 of X's columns, in 32 bits in registers, in the layout that a
// 32 x 32 product leaves: column lane % 32, rows 8 q + 4 (lane / 32) + e.  As
// the right operand of B X these are the rows of 16 that a step contracts, in
// another order, which the left operand, read from LDS, takes as well.  For
// X X^T, which contracts columns, X goes to LDS, row by row.
#include <algorithm>

#include "halves.hpp"
#include "step.hpp"
#include "wave.hpp"

namespace same {
namespace {

__device__ __forceinline__ f32x16 mfma(f16x8 l, f16x8 r, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(l, r, c, 0, 0, 0);
}

__device__ __forceinline__ f32x16 zero16() {
    f32x16 z;
#pragma unroll
    for (int e = 0; e < 16; ++e) z[e] = 0.0f;
    return z;
}

// NT tiles of 32 rows, up to MT waves.  Rows in LDS are padded by 16 bytes: an odd
// number of 16-byte pieces, so that 16 of them lie in banks of their own.
template <typename T, int NT, int MT>
__global__ __launch_bounds__(MT * 64) void ortho_whole_kernel(OrthoParams p) {
    static_assert(MT >= NT, "B fits where X was");
    constexpr int kRowX = 32 * MT + 8, kRowA = 32 * NT + 8;
    __shared__ _Float16 xs[2][32 * NT * kRowX], as[2][32 * NT * kRowA];
    __shared__ double sums[MT];
    const int lane = threadIdx.x & 63, own = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = p.parts;
    const int col = lane & 31, half = lane >> 5;
    const int64_t mat = blockIdx.x;
    const T *g = (const T *)p.g + mat * p.g_mat;
    T *out = (T *)p.out + mat * p.out_mat;
    const int64_t down = p.tall ? 1 : p.g_row, across = p.tall ? p.g_row : 1;
    const int64_t out_down = p.tall ? 1 : p.out_row, out_across = p.tall ? p.out_row : 1;
    const int j = 32 * own + col;
    f32x16 x[NT];
    double total = 0.0;
    const T *const mine = g + min(j, p.m - 1) * across;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int i = 32 * t + 8 * (e >> 2) + 4 * half + (e & 3);
            const float v = (float)mine[min(i, p.n - 1) * down];
            x[t][e] = i < p.n && j < p.m ? v : 0.0f;
            total = __builtin_fma((double)x[t][e], (double)x[t][e], total);
        }
        if (NT < 4) __builtin_amdgcn_sched_barrier(0);   // no further addresses at the same time
    }
    for (int o = 32; o; o >>= 1) total += __shfl_xor(total, o);
    if (lane == 0) sums[own] = total;
    __syncthreads();
    total = 0.0;
    for (int w = 0; w < waves; ++w) total += sums[w];
    const float factor = (float)((double)p.sx / (__builtin_sqrt(total) + (double)p.eps));
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) x[t][e] *= factor;

    // Of the small products a wave takes tiles (a, b) of one column b, every
    // groups-th; both halves of a symmetric matrix are formed, which costs less
    // than turning one of them.
    const int groups = waves / NT, b = own % NT, a0 = own / NT;
    const bool squares = a0 < groups && a0 < NT;
    for (int step = 0; step < p.steps; ++step) {
        const float ca = p.coef[step][0], cb = p.coef[step][1], cc = p.coef[step][2];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                f16x2 h, l;
                split(x[t][e], x[t][e + 1], h, l);
                const int at = (32 * t + 8 * (e >> 2) + 4 * half + (e & 3)) * kRowX + j;
                xs[0][at] = h[0];
                xs[0][at + kRowX] = h[1];
                xs[1][at] = l[0];
                xs[1][at + kRowX] = l[1];
            }
        __syncthreads();
        // C[a][b] over `depth` columns of rows of `row` numbers
        f32x16 acc[NT];
        auto product = [&](const _Float16 *hi, const _Float16 *lo, int row, int depth) {
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[t] = zero16();
            const int at_b = (32 * b + col) * row + 8 * half;
            struct Operands {
                f16x8 r_hi, r_lo, l_hi[NT], l_lo[NT];
            } now, then;
            auto load = [&](Operands &o, int k) {
                o.r_hi = *(const f16x8 *)&hi[at_b + k];
                o.r_lo = *(const f16x8 *)&lo[at_b + k];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const int at = (32 * min(a0 + t * groups, NT - 1) + col) * row + 8 * half + k;
                    o.l_hi[t] = *(const f16x8 *)&hi[at];
                    o.l_lo[t] = *(const f16x8 *)&lo[at];
                }
                __builtin_amdgcn_sched_barrier(0);   // before the products of the other
            };
            auto multiply = [&](const Operands &o) {   // products of one sum apart from each other
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[t] = mfma(o.l_lo[t], o.r_hi, acc[t]);
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[t] = mfma(o.l_hi[t], o.r_lo, acc[t]);
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[t] = mfma(o.l_hi[t], o.r_hi, acc[t]);
                __builtin_amdgcn_sched_barrier(0);
            };
            load(now, 0);
            for (int k = 0; k < depth; k += 32) {
                load(then, k + 16);
                multiply(now);
                if (k + 32 < depth) load(now, k + 32);
                multiply(then);
            }
        };
        // rows b of the result, columns a: the matrix is symmetric
        auto put = [&](_Float16 *to_hi, _Float16 *to_lo, int a, const f32x16 &v) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                f16x4 hi, lo;
                split_all<4>([&](int e) { return v[4 * q + e]; }, hi, lo);
                const int at = (32 * b + col) * kRowA + 32 * a + 8 * q + 4 * half;
                *(f16x4 *)&to_hi[at] = hi;
                *(f16x4 *)&to_lo[at] = lo;
            }
        };
        // A = X X^T
        if (squares) {
            product(xs[0], xs[1], kRowX, 32 * waves);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if (a0 + t * groups >= NT) continue;
                const float s = p.sa / (p.sx * p.sx);
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[t][e] *= s;
                put(as[0], as[1], a0 + t * groups, acc[t]);
            }
        }
        __syncthreads();
        // B = b A + c A A, where X was
        if (squares) {
            product(as[0], as[1], kRowA, 32 * NT);
            const float keep = cb * (p.sb / p.sa), take = cc * (p.sb / (p.sa * p.sa));
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if (a0 + t * groups >= NT) continue;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int at = (32 * b + col) * kRowA + 32 * (a0 + t * groups) + 8 * q + 4 * half;
                    const f16x4 hi = *(const f16x4 *)&as[0][at], lo = *(const f16x4 *)&as[1][at];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        acc[t][4 * q + e] =
                            __builtin_fmaf(take, acc[t][4 * q + e], keep * ((float)hi[e] + (float)lo[e]));
                }
                put(xs[0], xs[1], a0 + t * groups, acc[t]);
            }
        }
        __syncthreads();
        // X <- a X + B X; X's halves are formed again, not kept since they went to LDS
#pragma unroll
        for (int t = 0; t < NT; ++t) asm volatile("" : "+v"(x[t]));
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[t] = zero16();
#pragma unroll
        for (int k = 0; k < 2 * NT; ++k) {
            f16x8 hi, lo;
            split_all<8>([&](int e) { return x[k >> 1][8 * (k & 1) + e]; }, hi, lo);
            union Eight {
                f16x4 h[2];
                f16x8 v;
            } l_hi[NT], l_lo[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int at = (32 * t + col) * kRowA + 16 * k + 4 * half;
                l_hi[t].h[0] = *(const f16x4 *)&xs[0][at];
                l_hi[t].h[1] = *(const f16x4 *)&xs[0][at + 8];
                l_lo[t].h[0] = *(const f16x4 *)&xs[1][at];
                l_lo[t].h[1] = *(const f16x4 *)&xs[1][at + 8];
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[t] = mfma(l_lo[t].v, hi, acc[t]);
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[t] = mfma(l_hi[t].v, lo, acc[t]);
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[t] = mfma(l_hi[t].v, hi, acc[t]);
            if (NT == 2 || (NT == 3 && (k & 1))) __builtin_amdgcn_sched_barrier(0);  // further operands would not fit
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) x[t][e] = __builtin_fmaf(acc[t][e], 1.0f / p.sb, ca * x[t][e]);
        __syncthreads();
    }
    const float scale = p.out_scale / p.sx;
    T *const to = out + 4 * half * out_down + j * out_across;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int above = 32 * t + 8 * (e >> 2) + (e & 3);
            if (above + 4 * half < p.n && j < p.m) to[above * out_down] = (T)(x[t][e] * scale);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

template <typename T>
hipError_t run_typed(const OrthoParams &all, hipStream_t s) {
    OrthoParams p = all;
    const int waves = p.parts = (p.m + 31) / 32;
    const uint32_t mats = (uint32_t)p.n_mats;
    if (p.n <= 64)
        ortho_whole_kernel<T, 2, 8><<<mats, 64 * waves, 0, s>>>(p);
    else if (p.n <= 96)
        ortho_whole_kernel<T, 3, 8><<<mats, 64 * waves, 0, s>>>(p);
    else
        ortho_whole_kernel<T, 4, 4><<<mats, 64 * waves, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_ortho_whole(const OrthoParams &p, int dtype, hipStream_t s) {
    if (dtype == 2) return run_typed<__bf16>(p, s);
    if (dtype == 1) return run_typed<_Float16>(p, s);
    return run_typed<float>(p, s);
}

}  // namespace same
