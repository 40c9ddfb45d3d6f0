// Orthogonalised updates that one block holds, for gfx950: smaller sides of 33
// to 96 with larger ones up to 256, and up to 128 x 128.  The products and their
// two fp16 a number are those of orthogonalise.hip, all three for every type,
// without a launch or a trip to memory between.
//
// A wave owns some of X's columns, in 32 bits in registers, in the layout that a
// product leaves: a lane has rows of one column.  As the right operand of B X
// these are the rows that a step contracts, in another order, which the left
// operand takes as well: B is written to LDS in that order.  For X X^T, which
// contracts columns, X goes to LDS, row by row.
//
// What bounds it is the chain on one compute unit: a step of 128 x 128 takes 7 us,
// of which the matrix units work 3.9 (both halves of the symmetric products,
// which costs less than turning one of them), vector units, between barriers,
// most of the rest.  Five steps take 44 us, in launches of their own on many
// compute units 74; 256 matrices take 60.
#include <algorithm>

#include "ortho_block.hpp"
#include "step.hpp"

namespace same {
namespace {

// More than 128 columns: a wave owns 32, NT tiles of 32 rows, up to MT waves
// (64 x 256 31 us).  Rows in LDS are padded by 16 bytes: an odd
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
    const int j = 32 * own + col, at_x = (4 * half + 2 * (lane & 1)) * kRowX + (j & ~1);
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
        __builtin_amdgcn_sched_barrier(0);   // no further addresses at the same time
    }
    for (int o = 32; o; o >>= 1) total += __shfl_xor(total, o);
    if (lane == 0) sums[own] = total;
    __syncthreads();
    total = 0.0;
    for (int w = 0; w < waves; ++w) total += sums[w];
    const PlaneFactor of_g(p.sx, total, p.eps);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) x[t][e] = of_g(x[t][e]);

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
            for (int q = 0; q < 4; ++q) {
                f16x2 h[2], l[2];
                split(x[t][4 * q], x[t][4 * q + 1], h[0], l[0]);
                split(x[t][4 * q + 2], x[t][4 * q + 3], h[1], l[1]);
                const int at = (32 * t + 8 * q) * kRowX + at_x;
                write_rows(&xs[0][at], kRowX, h[0], h[1]);
                write_rows(&xs[1][at], kRowX, l[0], l[1]);
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
        // A = X X^T, rows b and columns a: the matrix is symmetric
        const int at_b = (32 * b + col) * kRowA + 8 * half;
        if (squares) {
            product(xs[0], xs[1], kRowX, 32 * waves);
            const float s = p.sa / (p.sx * p.sx);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int at = at_b + 32 * (a0 + t * groups);
                if (a0 + t * groups < NT) write_row(&as[0][at], &as[1][at], [&](int e) { return acc[t][e] * s; });
            }
        }
        __syncthreads();
        // B = b A + c A A, where X was
        if (squares) {
            product(as[0], as[1], kRowA, 32 * NT);
            const float keep = cb * (p.sb / p.sa), take = cc * (p.sb / (p.sa * p.sa));
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int at = at_b + 32 * (a0 + t * groups);
                if (a0 + t * groups >= NT) continue;
                add_row(&as[0][at], &as[1][at], take, keep, acc[t]);
                write_own<1>(&xs[0][at], &xs[1][at], [&](int e) { return acc[t][e]; });
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
            f16x8 l_hi[NT], l_lo[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int at = (32 * t + col) * kRowA + 16 * k + 8 * half;
                l_hi[t] = *(const f16x8 *)&xs[0][at];
                l_lo[t] = *(const f16x8 *)&xs[1][at];
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[t] = mfma(l_lo[t], hi, acc[t]);
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[t] = mfma(l_hi[t], lo, acc[t]);
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[t] = mfma(l_hi[t], hi, acc[t]);
            if (NT == 2 || (k & 1)) __builtin_amdgcn_sched_barrier(0);  // further operands would not fit
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

// Up to 128 columns: eight waves, two a SIMD, a wave owns 16 columns (128 x 128
// with four waves of 32 63 us, with eight 44; 64 x 64 16).  The small
// products are formed in tiles of 32 x 32 as above; B X in tiles of 16 x 16, whose
// contraction of 32 takes rows 16 u + 4 (lane / 16) + e as its place
// 8 (lane / 16) + 4 u + e: B's columns are written in that order.
template <typename T, int NT>
__global__ __launch_bounds__(512) void ortho_strips_kernel(OrthoParams p) {
    constexpr int kWaves = 8, kRowX = 16 * kWaves + 8, kRowA = 32 * NT + 8;
    constexpr int kGroups = kWaves / NT, kMine = (NT + kGroups - 1) / kGroups;
    __shared__ _Float16 xs[2][32 * NT * kRowX], as[2][32 * NT * kRowA];
    __shared__ double sums[kWaves];
    const int lane = threadIdx.x & 63, own = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quarter = lane >> 4, row = lane & 31, half = lane >> 5;
    const int64_t mat = blockIdx.x;
    const T *g = (const T *)p.g + mat * p.g_mat;
    T *out = (T *)p.out + mat * p.out_mat;
    const int64_t down = p.tall ? 1 : p.g_row, across = p.tall ? p.g_row : 1;
    const int64_t out_down = p.tall ? 1 : p.out_row, out_across = p.tall ? p.out_row : 1;
    const int j = 16 * own + col, depth = (p.m + 31) / 32 * 32;
    f32x4 x[2 * NT];
    double total = 0.0;
    const T *const mine = g + min(j, p.m - 1) * across;
#pragma unroll
    for (int t = 0; t < 2 * NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = 16 * t + 4 * quarter + e;
            const float v = (float)mine[min(i, p.n - 1) * down];
            x[t][e] = i < p.n && j < p.m ? v : 0.0f;
        }
#pragma unroll
    for (int t = 0; t < 2 * NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) total = __builtin_fma((double)x[t][e], (double)x[t][e], total);
    for (int o = 32; o; o >>= 1) total += __shfl_xor(total, o);
    if (lane == 0) sums[own] = total;
    __syncthreads();
    total = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) total += sums[w];
    const PlaneFactor of_g(p.sx, total, p.eps);
#pragma unroll
    for (int t = 0; t < 2 * NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[t][e] = of_g(x[t][e]);

    // of the small products a wave takes tiles (a0 + groups i, b)
    const int b = own % NT, a0 = own / NT;
    const bool squares = a0 < kGroups && a0 < NT;
    const int at_b = (32 * b + row) * kRowA + 8 * half;
    f32x16 acc[kMine], old[kMine];
    auto product = [&](const _Float16 *hi, const _Float16 *lo, int pitch, int depth) {
#pragma unroll
        for (int t = 0; t < kMine; ++t) acc[t] = zero16();
        add_products<NT, kGroups>(acc, hi, lo, pitch, depth, a0, b);
    };
    for (int step = 0; step < p.steps; ++step) {
        const float ca = p.coef[step][0], cb = p.coef[step][1], cc = p.coef[step][2];
        write_strip<NT>(x, xs[0], xs[1], kRowX);
        __syncthreads();
        // A = X X^T, rows b and columns a: the matrix is symmetric
        if (squares) {
            product(xs[0], xs[1], kRowX, depth);
            const float s = p.sa / (p.sx * p.sx);
#pragma unroll
            for (int t = 0; t < kMine; ++t) {
                const int at = at_b + 32 * (a0 + t * kGroups);
                if (a0 + t * kGroups >= NT) continue;
#pragma unroll
                for (int e = 0; e < 16; ++e) old[t][e] = acc[t][e] * s;
                write_row(&as[0][at], &as[1][at], [&](int e) { return old[t][e]; });
            }
        }
        __syncthreads();
        // B = b A + c A A, where X was
        if (squares) {
            product(as[0], as[1], kRowA, 32 * NT);
            const float keep = cb * (p.sb / p.sa), take = cc * (p.sb / (p.sa * p.sa));
#pragma unroll
            for (int t = 0; t < kMine; ++t) {
                const int at = at_b + 32 * (a0 + t * kGroups);
                if (a0 + t * kGroups >= NT) continue;
                write_own<2>(&xs[0][at], &xs[1][at],
                             [&](int e) { return __builtin_fmaf(take, acc[t][e], keep * old[t][e]); });
            }
        }
        __syncthreads();
        update_strip<NT>(x, xs[0], xs[1], kRowA, ca, 1.0f / p.sb);
        __syncthreads();
    }
    const float scale = p.out_scale / p.sx;
    T *const to = out + 4 * quarter * out_down + j * out_across;
#pragma unroll
    for (int t = 0; t < 2 * NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (16 * t + 4 * quarter + e < p.n && j < p.m) to[(16 * t + e) * out_down] = (T)(x[t][e] * scale);
}

template <typename T>
hipError_t run_typed(const OrthoParams &all, hipStream_t s) {
    OrthoParams p = all;
    const int waves = p.parts = (p.m + 31) / 32;
    const uint32_t mats = (uint32_t)p.n_mats;
    if (p.m <= 128) {
        if (p.n <= 64)
            ortho_strips_kernel<T, 2><<<mats, 512, 0, s>>>(p);
        else if (p.n <= 96)
            ortho_strips_kernel<T, 3><<<mats, 512, 0, s>>>(p);
        else
            ortho_strips_kernel<T, 4><<<mats, 512, 0, s>>>(p);
    } else if (p.n <= 64)
        ortho_whole_kernel<T, 2, 8><<<mats, 64 * waves, 0, s>>>(p);
    else
        ortho_whole_kernel<T, 3, 8><<<mats, 64 * waves, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_ortho_whole(const OrthoParams &p, int dtype, hipStream_t s) {
    if (dtype == 2) return run_typed<__bf16>(p, s);
    if (dtype == 1) return run_typed<_Float16>(p, s);
    return run_typed<float>(p, s);
}

}  // namespace same
