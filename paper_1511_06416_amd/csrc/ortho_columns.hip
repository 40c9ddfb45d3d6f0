// Orthogonalised updates with a smaller side of 33 to 128 and more columns than one
// block holds, up to 8,192 of them, for gfx950.  A block holds 128 columns of X at a time
// in registers, as the one-block kernels do, and a step is one pass over X:
//   B = b A + c A A from A, X <- a X + B X, and at once the columns' part of the
//   next A = X X^T; a second launch sums the parts, in order.
// Every block forms B anew: that is less than waiting for a launch.  X stays in 32
// bits between steps, products take two fp16 a number, all three for every type.
//
// A step costs 8 bytes a number of X and two launches, where tiled products take
// three or four launches and every layout of X in halves.  Few matrices are bound
// by the launches and a block's chain (128 x 1,000: 12 us a pass and 4 a join, 85
// in all), many by the bytes of X (750 of 905 x 33: 70 us a pass, 20 a join).
#include <algorithm>

#include "ortho_block.hpp"
#include "step.hpp"

namespace same {
namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves, kStrip = 16 * kWaves;
enum Pass { kFirst, kMiddle, kLast };

// NT tiles of 32 rows.
template <typename T, int NT, int PASS>
__global__ __launch_bounds__(kThreads) void ortho_columns_kernel(OrthoParams p, int step, int square_parts) {
    constexpr int kRowX = kStrip + 8, kRowA = 32 * NT + 8;
    constexpr int kGroups = kWaves / NT, kMine = (NT + kGroups - 1) / kGroups;
    __shared__ _Float16 xs[2][32 * NT * kRowX], as[2][32 * NT * kRowA];
    __shared__ double sums[kWaves];
    const int lane = threadIdx.x & 63, own = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quarter = lane >> 4, row = lane & 31, half = lane >> 5;
    const int64_t mat = blockIdx.x / p.parts;
    const int part = (int)(blockIdx.x - mat * p.parts);
    const int strips = (p.m + kStrip - 1) / kStrip, each = p.part_cols / kStrip;
    const int beg = part * each, end = min(strips, beg + each);
    const int b = own % NT, a0 = own / NT;
    const bool squares = a0 < kGroups && a0 < NT;
    f32x16 acc[kMine];
    PlaneFactor of_g;
    if (PASS == kFirst) {
        double total = 0.0;
        for (int i = threadIdx.x; i < square_parts; i += kThreads) total += p.squares[mat * kNormParts + i];
        for (int o = 32; o; o >>= 1) total += __shfl_xor(total, o);
        if (lane == 0) sums[own] = total;
        __syncthreads();
        total = 0.0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) total += sums[w];
        of_g = PlaneFactor(p.sx, total, p.eps);
    } else {
        // B = b A + c A A, where A was
        constexpr int kChunks = 4 * NT;   // of 16 bytes a row
        const _Float16 *a_hi = p.a.hi + mat * (32 * NT) * (32 * NT), *a_lo = p.a.lo + mat * (32 * NT) * (32 * NT);
        for (int e = threadIdx.x; e < 32 * NT * kChunks; e += kThreads) {
            const int i = e / kChunks, to = i * kRowA + 8 * (e - i * kChunks);
            *(f16x8 *)&as[0][to] = *(const f16x8 *)(a_hi + 8 * e);
            *(f16x8 *)&as[1][to] = *(const f16x8 *)(a_lo + 8 * e);
        }
        __syncthreads();
        const int at_b = (32 * b + row) * kRowA + 8 * half;
        if (squares) {
            const float keep = p.coef[step][1] * (p.sb / p.sa), take = p.coef[step][2] * (p.sb / (p.sa * p.sa));
#pragma unroll
            for (int t = 0; t < kMine; ++t) acc[t] = zero16();
            add_products<NT, kGroups>(acc, as[0], as[1], kRowA, 32 * NT, a0, b);
#pragma unroll
            for (int t = 0; t < kMine; ++t)
                if (a0 + t * kGroups < NT) {
                    const int at = at_b + 32 * (a0 + t * kGroups);
                    add_row(&as[0][at], &as[1][at], take, keep, acc[t]);
                }
        }
        __syncthreads();
        if (squares) {
#pragma unroll
            for (int t = 0; t < kMine; ++t)
                if (a0 + t * kGroups < NT) {
                    const int at = at_b + 32 * (a0 + t * kGroups);
                    write_own<2>(&as[0][at], &as[1][at], [&](int e) { return acc[t][e]; });
                }
        }
        __syncthreads();
    }
#pragma unroll
    for (int t = 0; t < kMine; ++t) acc[t] = zero16();
    const int64_t down = p.tall ? 1 : p.g_row, across = p.tall ? p.g_row : 1;
    const int64_t out_down = p.tall ? 1 : p.out_row, out_across = p.tall ? p.out_row : 1;
    for (int strip = beg; strip < end; ++strip) {
        const int j = kStrip * strip + 16 * own + col;
        f32x4 x[2 * NT];
        // 16 rows and columns of zeros stay zeros and are not kept
        const auto kept_rows = [&](int t) { return 16 * t < p.n && kStrip * strip + 16 * own < p.m; };
        f32x4 *const kept = (f32x4 *)p.x32 + ((mat * strips + strip) * kWaves + own) * (2 * NT * 64) + lane;
        if (PASS == kFirst) {
            const T *const mine = (const T *)p.g + mat * p.g_mat + min(j, p.m - 1) * across;
#pragma unroll
            for (int t = 0; t < 2 * NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 16 * t + 4 * quarter + e;
                    const float v = (float)mine[min(i, p.n - 1) * down];
                    x[t][e] = i < p.n && j < p.m ? of_g(v) : 0.0f;
                }
        } else {
#pragma unroll
            for (int t = 0; t < 2 * NT; ++t) x[t] = kept_rows(t) ? kept[64 * t] : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            update_strip<NT>(x, as[0], as[1], kRowA, p.coef[step][0], 1.0f / p.sb);
        }
        if (PASS == kLast) {
            const float scale = p.out_scale / p.sx;
            T *const to = (T *)p.out + mat * p.out_mat + 4 * quarter * out_down + j * out_across;
#pragma unroll
            for (int t = 0; t < 2 * NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (16 * t + 4 * quarter + e < p.n && j < p.m) to[(16 * t + e) * out_down] = (T)(x[t][e] * scale);
        } else {
#pragma unroll
            for (int t = 0; t < 2 * NT; ++t)
                if (kept_rows(t)) kept[64 * t] = x[t];
            write_strip<NT>(x, xs[0], xs[1], kRowX);
            __syncthreads();
            if (squares) add_products<NT, kGroups>(acc, xs[0], xs[1], kRowX, kStrip, a0, b);
            __syncthreads();
        }
    }
    if (PASS != kLast && squares) {
#pragma unroll
        for (int t = 0; t < kMine; ++t)
            if (a0 + t * kGroups < NT) {
                const int tile = b * NT + a0 + t * kGroups;
                f32x4 *const to = (f32x4 *)p.gram_parts + ((mat * p.parts + part) * (NT * NT) + tile) * 256 + lane;
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    to[64 * q] = f32x4{acc[t][4 * q], acc[t][4 * q + 1], acc[t][4 * q + 2], acc[t][4 * q + 3]};
            }
    }
}

// A from its parts: a wave takes a tile, its rows b.
template <int NT>
__global__ __launch_bounds__(64) void ortho_columns_join_kernel(OrthoParams p) {
    const int lane = threadIdx.x, tile = blockIdx.x, b = tile / NT, a = tile - b * NT;
    const int64_t mat = blockIdx.y;
    const f32x4 *from = (const f32x4 *)p.gram_parts + (mat * p.parts * (NT * NT) + tile) * 256 + lane;
    f32x4 v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int i = 0; i < p.parts; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] += from[i * (NT * NT * 256) + 64 * q];
    const float s = p.sa / (p.sx * p.sx);
    const int64_t at = (mat * (32 * NT) + 32 * b + (lane & 31)) * (32 * NT) + 32 * a + 8 * (lane >> 5);
    write_row(p.a.hi + at, p.a.lo + at, [&](int e) { return v[e >> 2][e & 3] * s; });
}

template <typename T, int NT>
hipError_t run_side(const OrthoParams &p, int square_parts, hipStream_t s) {
    const uint32_t mats = (uint32_t)p.n_mats, blocks = mats * (uint32_t)p.parts;
    ortho_columns_kernel<T, NT, kFirst><<<blocks, kThreads, 0, s>>>(p, 0, square_parts);
    for (int step = 0; step < p.steps; ++step) {
        ortho_columns_join_kernel<NT><<<dim3(NT * NT, mats), 64, 0, s>>>(p);
        if (step + 1 < p.steps)
            ortho_columns_kernel<float, NT, kMiddle><<<blocks, kThreads, 0, s>>>(p, step, 0);
        else
            ortho_columns_kernel<T, NT, kLast><<<blocks, kThreads, 0, s>>>(p, step, 0);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
hipError_t run_typed(const OrthoParams &p, int square_parts, hipStream_t s) {
    return p.n <= 64   ? run_side<T, 2>(p, square_parts, s)
           : p.n <= 96 ? run_side<T, 3>(p, square_parts, s)
                       : run_side<T, 4>(p, square_parts, s);
}

}  // namespace

// A block's columns, by the matrix's size alone: one strip of 128 up to 16 of
// them, then as many as keep parts few.
void ortho_columns_layout(int64_t n, int64_t m, int32_t *parts, int32_t *part_cols, size_t *x_bytes,
                          size_t *part_bytes, size_t *plane_bytes) {
    const int64_t tiles = (n + 31) / 32, strips = (m + kStrip - 1) / kStrip;
    const int64_t each = (strips + 15) / 16;
    *part_cols = (int32_t)(each * kStrip);
    *parts = (int32_t)((strips + each - 1) / each);
    *x_bytes = (size_t)(strips * kStrip * 32 * tiles * 4);
    *part_bytes = (size_t)(*parts * tiles * tiles * 4096);
    *plane_bytes = (size_t)(tiles * tiles * 2048);
}

hipError_t launch_ortho_columns(const OrthoParams &p, int dtype, hipStream_t s) {
    int square_parts = 0;
    const hipError_t e = launch_ortho_squares(p, dtype, s, &square_parts);
    if (e != hipSuccess) return e;
    if (dtype == 2) return run_typed<__bf16>(p, square_parts, s);
    if (dtype == 1) return run_typed<_Float16>(p, square_parts, s);
    return run_typed<float>(p, square_parts, s);
}

}  // namespace same
