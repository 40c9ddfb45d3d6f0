// Orthogonalising an update by Newton-Schulz products, for gfx950:
//   X = G / (|G| + eps), |G| the root of the sum of squares, then per step
//   A = X X^T,  B = b A + c A A,  X <- a X + B X
// with X's rows along the smaller side of G, so that A is small.
//
// Products run on the fp16 matrix units.  A number is held as the sum of two
// fp16, hi + lo, times a power of two that keeps both in the type's normal
// range: 22 bits.  Of a product of two such, hi hi + hi lo + lo hi are formed
// (what is left out is 2^-22 of it), summed in fp32, for every type: off by as much
// as a form in fp32 or less (1,024 x 1,024 of noise 2.1e-6 of the result's size for
// 3.1e-6, 64 x 8,193 1.4e-6 for 1.35e-6).  hi hi alone was tried for bf16: 4,096 x
// 4,096 took 1,690 us, but noise of 64 x 8,193 was off by 3.8e-3 and of 200 x 300 by
// 2.6e-3, where rounding out leaves 1.66e-3.
// A and B are symmetric: tiles on and above the diagonal are formed and written
// to both places.
//
// Measured: 4,096 x 4,096 in bf16, five steps, 4,060 us (fp32 4,080): 1,015 TFLOP/s of
// the three products that have to be computed, where a large library product of fp16
// reaches 1,117; a step is 215 us for A, 224 for B, 344 to 366 for X, matrix units 50
// to 67 % busy.  In fp32 four of 1,024 x 1,024 take 540 us, where a form in fp32
// products takes 1,450.
#include <algorithm>

#include "halves.hpp"
#include "step.hpp"
#include "wave.hpp"

namespace same {
namespace {

constexpr int kThreads = 256;
constexpr int kStage = 32;  // columns of a stage
constexpr int kTurn = 36;   // floats of a row of a tile that is turned

// Sums over a block, in every thread.
__device__ __forceinline__ double block_sum(double t) {
    __shared__ double sums[kThreads / 64];
    for (int o = 32; o; o >>= 1) t += __shfl_xor(t, o);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = t;
    __syncthreads();
    t = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) t += sums[w];
    return t;
}

// Parts of the sums of squares, in 64 bits: no update is too large or small.
// A block takes stretches of rows, eight elements a thread, `row_threads` (a power
// of two) a row: 750 of 905 x 33 with all threads on one row 358 us.
template <typename T>
__global__ __launch_bounds__(kThreads) void ortho_squares_kernel(OrthoParams p, int parts, int items, int across,
                                                                 int row_threads) {
    const int64_t mat = blockIdx.x / parts;
    const int part = (int)(blockIdx.x - mat * parts), at_once = kThreads / row_threads;
    const int row = threadIdx.x / row_threads, piece = threadIdx.x & (row_threads - 1);
    double t = 0.0;
    for (int item = part; item < items; item += parts) {
        const int up = item / across, i = up * at_once + row, j = ((item - up * across) * row_threads + piece) * 8;
        if (i >= p.rows) continue;
        const T *src = (const T *)p.g + mat * p.g_mat + i * p.g_row + j;
        if (j + 8 <= p.cols) {
            const wave::Loose<T, 8> v = *(const wave::Loose<T, 8> *)src;
#pragma unroll
            for (int e = 0; e < 8; ++e) t = __builtin_fma((double)(float)v.v[e], (double)(float)v.v[e], t);
        } else {
            for (int e = 0; j + e < p.cols; ++e) t = __builtin_fma((double)(float)src[e], (double)(float)src[e], t);
        }
    }
    t = block_sum(t);
    if (threadIdx.x == 0) p.squares[mat * kNormParts + part] = t;
}

// X in planes, both ways, zeros around it: a block takes 64 x 64.
template <typename T>
__global__ __launch_bounds__(kThreads) void ortho_split_kernel(OrthoParams p, int parts, int tiles_i, int tiles_j) {
    __shared__ float tile[64][65];
    const int tiles = tiles_i * tiles_j;
    const int64_t mat = blockIdx.x / tiles;
    const int at = (int)(blockIdx.x - mat * tiles);
    double total = 0.0;
    for (int i = threadIdx.x; i < parts; i += kThreads) total += p.squares[mat * kNormParts + i];
    total = block_sum(total);
    const PlaneFactor of_g(p.sx, total, p.eps);
    const int i0 = at % tiles_i * 64, j0 = at / tiles_i * 64;
    const T *g = (const T *)p.g + mat * p.g_mat;
    const int c = 8 * (threadIdx.x & 7);
#pragma unroll
    for (int r = threadIdx.x >> 3; r < 64; r += kThreads / 8) {
        // along g's rows
        const int i = p.tall ? j0 + r : i0 + r, j = (p.tall ? i0 : j0) + c;
        const T *src = g + i * p.g_row + j;
        float v[8];
        if (i < p.rows && j + 8 <= p.cols) {
            const wave::Loose<T, 8> l = *(const wave::Loose<T, 8> *)src;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = of_g((float)l.v[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = i < p.rows && j + e < p.cols ? of_g((float)src[e]) : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (p.tall)
                tile[c + e][r] = v[e];
            else
                tile[r][c + e] = v[e];
        }
    }
    __syncthreads();
    const int64_t x0 = mat * p.np * p.mp;
#pragma unroll
    for (int r = threadIdx.x >> 3; r < 64; r += kThreads / 8) {
        f16x8 hi, lo;
        if (i0 + r < p.np && j0 + c < p.mp) {
            split_all<8>([&](int e) { return tile[r][c + e]; }, hi, lo);
            const int64_t to = x0 + (int64_t)(i0 + r) * p.mp + j0 + c;
            *(f16x8 *)(p.x.hi + to) = hi;
            *(f16x8 *)(p.x.lo + to) = lo;
        }
        if (j0 + r < p.mp && i0 + c < p.np) {
            split_all<8>([&](int e) { return tile[c + e][r]; }, hi, lo);
            const int64_t to = x0 + (int64_t)(j0 + r) * p.np + i0 + c;
            *(f16x8 *)(p.xt[0].hi + to) = hi;
            *(f16x8 *)(p.xt[0].lo + to) = lo;
        }
    }
}

// Eight numbers of a row of out.
template <typename T>
__device__ __forceinline__ void write_out(const OrthoParams &p, int64_t mat, int row, int rows, int col, int cols,
                                          const f32x4 (&v)[2]) {
    if (row >= rows) return;
    T *dst = (T *)p.out + mat * p.out_mat + row * p.out_row + col;
    const float scale = p.out_scale / p.sx;
    wave::Loose<T, 8> o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o.v[e] = (T)(v[e >> 2][e & 3] * scale);
    if (col + 8 <= cols) {
        *(wave::Loose<T, 8> *)dst = o;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (col + e < cols) dst[e] = o.v[e];
    }
}

enum Kind { kGram, kSquare, kUpdate, kLast };

// What a product becomes, from a tile of 32 x 32 that a wave holds in LDS, column
// by column: both of its places are read and written 16 bytes a lane, 64 bytes of
// a row.
template <typename T, int KIND>
__device__ __forceinline__ void leave(const OrthoParams &p, int64_t mat, int step, int i0, int j0,
                                      float (*turn)[kTurn]) {
    constexpr bool symmetric = KIND == kGram || KIND == kSquare;
    const int lane = threadIdx.x & 63;
    const float keep = KIND == kGram ? 0.0f : KIND == kSquare ? p.coef[step][1] * (p.sb / p.sa) : p.coef[step][0];
    const float take = KIND == kGram     ? p.sa / (p.sx * p.sx)
                       : KIND == kSquare ? p.coef[step][2] * (p.sb / (p.sa * p.sa))
                                         : 1.0f / p.sb;
    const Planes old = KIND == kSquare ? p.a : p.xt[step & 1];
    const Planes to_t = KIND == kGram ? p.a : KIND == kSquare ? p.b : p.xt[(step & 1) ^ 1];
    const Planes to_d = KIND == kGram ? p.a : KIND == kSquare ? p.b : p.x;
    const int64_t t0 = mat * p.np * (symmetric ? p.np : p.mp);
    const int ld_d = symmetric ? p.np : p.mp;
    const bool diagonal = symmetric && i0 == j0;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int j = 16 * r + (lane >> 2), i = 8 * (lane & 3);
        const int64_t at = t0 + (int64_t)(j0 + j) * p.np + i0 + i;
        f32x4 *const here = (f32x4 *)&turn[j][i];
        f32x4 v[2] = {here[0], here[1]};
        if (diagonal) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (i + e > j) v[e >> 2][e & 3] = turn[i + e][j];
        }
        f16x8 hi, lo;
        if (KIND != kGram) {
            hi = *(const f16x8 *)(old.hi + at);
            lo = *(const f16x8 *)(old.lo + at);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float x = take * v[e >> 2][e & 3];
            if (KIND != kGram) x = __builtin_fmaf(keep, (float)hi[e] + (float)lo[e], x);
            v[e >> 2][e & 3] = x;
        }
        split_all<8>([&](int e) { return v[e >> 2][e & 3]; }, hi, lo);
        if (!diagonal) {
            here[0] = v[0];
            here[1] = v[1];
        }
        if (KIND == kLast) {
            if (p.tall) write_out<T>(p, mat, j0 + j, p.m, i0 + i, p.n, v);
        } else {
            *(f16x8 *)(to_t.hi + at) = hi;
            *(f16x8 *)(to_t.lo + at) = lo;
        }
    }
    wave::sync();
    if (KIND == kLast ? p.tall : diagonal) return;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int i = 16 * r + (lane & 15), j = 8 * (lane >> 4);
        f32x4 v[2];
        f16x8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e >> 2][e & 3] = turn[j + e][i];
        if (KIND == kLast) {
            write_out<T>(p, mat, i0 + i, p.n, j0 + j, p.m, v);
        } else {
            split_all<8>([&](int e) { return v[e >> 2][e & 3]; }, hi, lo);
            const int64_t at = t0 + (int64_t)(i0 + i) * ld_d + j0 + j;
            *(f16x8 *)(to_d.hi + at) = hi;
            *(f16x8 *)(to_d.lo + at) = lo;
        }
    }
}

// Tile `tile` on and above the diagonal, by columns.
__device__ __forceinline__ void triangle(int tile, int &ti, int &tj) {
    tj = (int)((__builtin_sqrtf(8.0f * (float)tile + 1.0f) - 1.0f) * 0.5f);
    while ((tj + 1) * (tj + 2) / 2 <= tile) ++tj;
    while (tj * (tj + 1) / 2 > tile) --tj;
    ti = tile - tj * (tj + 1) / 2;
}

// Waits until at most N of the wave's loads are under way, then for the other
// waves.  A barrier alone does not wait for loads into LDS.
template <int N>
__device__ __forceinline__ void arrive() {
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0) as the compiler counts: later waits are for later reads alone
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// C[i][j] = sum_k P[i][k] Q[j][k] over a TM x TN tile by WM x WN waves.
// Operands come straight into LDS by buffer loads, whose stage is a scalar offset
// (addresses of 64 bits a lane cost 6 %), STAGES stages of 32 columns in turn, all
// but one under way; rows of 64 bytes, whose 16-byte chunks are turned by the row
// so that a read of 32 rows meets no bank twice.  Rows past the matrix repeat
// its last one and are not written.
template <typename T, int TM, int TN, int WM, int WN, int STAGES, int KIND>
__global__ __launch_bounds__(WM * WN * 64) void ortho_product_kernel(OrthoParams p, int step, int tiles_i, int tiles_j) {
    constexpr int THREADS = WM * WN * 64, MT = TM / WM / 32, NT = TN / WN / 32, PL = 2;   // planes
    constexpr int kLoadsP = TM * 4 / THREADS, kLoadsQ = TN * 4 / THREADS;   // 16-byte loads a lane, per plane
    constexpr int kLoads = PL * (kLoadsP + kLoadsQ), kRows = PL * (TM + TN);
    static_assert(kLoadsP * THREADS == TM * 4 && kLoadsQ * THREADS == TN * 4, "every lane stages the same");
    static_assert(MT * WM * 32 == TM && NT * WN * 32 == TN, "whole tiles a wave");
    static_assert(WM * WN * 32 * kTurn * 4 <= STAGES * kRows * kStage * 2, "tiles are turned where operands were");
    __shared__ _Float16 stage[STAGES][kRows * kStage];
    const int lane = threadIdx.x & 63, own = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Neighbouring blocks go to different XCDs: each gets a stretch of tiles, which
    // share operands in its L2.
    const int tiles = gridDim.x, each = tiles / 8, rest = tiles % 8, xcd = blockIdx.x % 8;
    const int tile = xcd * each + min(xcd, rest) + blockIdx.x / 8;
    int ti, tj;
    if (KIND == kGram || KIND == kSquare) {
        triangle(tile, ti, tj);
    } else {
        // bands of four rows, by columns
        const int band = tile / (4 * tiles_j), height = min(4, tiles_i - 4 * band), at = tile - band * 4 * tiles_j;
        ti = 4 * band + at % height;
        tj = at / height;
    }
    const int64_t mat = blockIdx.y;
    const int64_t x0 = mat * p.np * p.mp, a0 = mat * p.np * p.np;
    const int ld = KIND == kGram ? p.mp : p.np;
    const int rows_j = KIND == kGram || KIND == kSquare ? p.np : p.mp;
    const Planes left = KIND == kGram ? p.x : KIND == kSquare ? p.a : p.b;
    const Planes right = KIND == kGram ? p.x : KIND == kSquare ? p.a : p.xt[step & 1];
    // a part of a long sum, in stages
    const int all = ld / kStage, share = KIND == kGram ? (all + p.splits - 1) / p.splits : all;
    const int first = KIND == kGram ? min((int)blockIdx.z * share, all) : 0, stages = min(share, all - first);
    const int64_t l0 = KIND == kGram ? x0 : a0, r0 = KIND == kSquare ? a0 : x0;
    // what this lane stages: its chunks, in bytes from the first row
    uint32_t off_p[kLoadsP], off_q[kLoadsQ];
#pragma unroll
    for (int l = 0; l < kLoadsP; ++l) {
        const int slot = (own * kLoadsP + l) * 64 + lane, row = slot >> 2;
        off_p[l] = 2u * (uint32_t)(min(ti * TM + row, p.np - 1) * ld + ((slot & 3) ^ ((row >> 2) & 3)) * 8);
    }
#pragma unroll
    for (int l = 0; l < kLoadsQ; ++l) {
        const int slot = (own * kLoadsQ + l) * 64 + lane, row = slot >> 2;
        off_q[l] = 2u * (uint32_t)(min(tj * TN + row, rows_j - 1) * ld + ((slot & 3) ^ ((row >> 2) & 3)) * 8);
    }
    // planes of this matrix as buffers of their size
    const auto plane = [&](const _Float16 *at, int rows) {
        return __builtin_amdgcn_make_buffer_rsrc((void *)at, (short)0, (int)(2u * (uint32_t)rows * (uint32_t)ld), 0x00020000);
    };
    const __amdgpu_buffer_rsrc_t left_hi = plane(left.hi + l0, p.np), left_lo = plane(left.lo + l0, p.np);
    const __amdgpu_buffer_rsrc_t right_hi = plane(right.hi + r0, rows_j), right_lo = plane(right.lo + r0, rows_j);
    auto load = [&](__amdgpu_buffer_rsrc_t src, uint32_t off, int k, _Float16 *dst) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (__attribute__((address_space(3))) void *)dst, 16, off, 2 * k, 0, 0);
    };
    auto fetch = [&](int buffer, int s) {
        const int k = (first + s) * kStage;
        _Float16 *to_p = &stage[buffer][own * kLoadsP * 512], *to_q = &stage[buffer][PL * TM * kStage + own * kLoadsQ * 512];
#pragma unroll
        for (int l = 0; l < kLoadsP; ++l) {
            load(left_hi, off_p[l], k, to_p + l * 512);
            load(left_lo, off_p[l], k, to_p + TM * kStage + l * 512);
        }
#pragma unroll
        for (int l = 0; l < kLoadsQ; ++l) {
            load(right_hi, off_q[l], k, to_q + l * 512);
            load(right_lo, off_q[l], k, to_q + TN * kStage + l * 512);
        }
    };
    f32x16 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    const int wi = (own % WM) * (TM / WM), wj = (own / WM) * (TN / WN);
    struct Operands {
        f16x8 l[PL][MT], r[PL][NT];
    };
    // where this lane's chunks of a stage's first 16 columns are; the others' are one bit apart
    const int turned = ((lane >> 5) ^ ((lane >> 2) & 3)) << 3;
    const int off_l = (wi + (lane & 31)) * kStage + turned, off_r = PL * TM * kStage + (wj + (lane & 31)) * kStage + turned;
    auto fill = [&](int buffer, int t, Operands &o) {
        const _Float16 *at_l = &stage[buffer][off_l ^ (t << 4)], *at_r = &stage[buffer][off_r ^ (t << 4)];
#pragma unroll
        for (int h = 0; h < PL; ++h) {
#pragma unroll
            for (int i = 0; i < MT; ++i) o.l[h][i] = *(const f16x8 *)(at_l + (h * TM + 32 * i) * kStage);
#pragma unroll
            for (int j = 0; j < NT; ++j) o.r[h][j] = *(const f16x8 *)(at_r + (h * TN + 32 * j) * kStage);
        }
    };
    auto multiply = [&](const Operands &o) {
        __builtin_amdgcn_sched_barrier(0);   // reads under way stay before the products
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(o.l[1][i], o.r[0][j], acc[i][j], 0, 0, 0);
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(o.l[0][i], o.r[1][j], acc[i][j], 0, 0, 0);
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(o.l[0][i], o.r[0][j], acc[i][j], 0, 0, 0);
            }
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
    };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s)
        if (s < stages) fetch(s, s);
    // A wave reads half a stage ahead of its products.  When it arrives at a
    // stage, that is there, and everyone has left the one before it, whose place
    // the next fetch takes.
    auto reach = [&](int s) {
        if (s + STAGES - 2 < stages)
            arrive<kLoads * (STAGES - 2)>();
        else
            arrive<0>();
    };
    Operands now, then;
    reach(0);
    fill(0, 0, now);
    for (int s = 0, buffer = 0, next = STAGES - 1; s < stages; ++s) {
        if (s + STAGES - 1 < stages) fetch(next, s + STAGES - 1);
        fill(buffer, 1, then);
        multiply(now);
        buffer = buffer + 1 == STAGES ? 0 : buffer + 1;
        next = next + 1 == STAGES ? 0 : next + 1;
        reach(s + 1);
        fill(buffer, 0, now);   // behind the last stage for nothing
        multiply(then);
    }
    // The way out, a tile of 32 x 32 at a time
    arrive<0>();
    float(*turn)[kTurn] = (float(*)[kTurn])((float *)&stage[0][0] + own * 32 * kTurn);
#pragma unroll
    for (int it = 0; it < MT; ++it)
#pragma unroll
        for (int jt = 0; jt < NT; ++jt) {
            const int i0 = ti * TM + wi + 32 * it, j0 = tj * TN + wj + 32 * jt;
            if (i0 >= p.np || j0 >= rows_j) continue;  // whole tiles: both are multiples of 32
            // Of a symmetric matrix, what lies on and above the diagonal is taken and
            // written to both places: the other half is summed in another order.
            if ((KIND == kGram || KIND == kSquare) && i0 > j0) continue;
            // a lane holds column j and, in fours, rows i
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(f32x4 *)&turn[lane & 31][8 * q + 4 * (lane >> 5)] =
                    f32x4{acc[it][jt][4 * q], acc[it][jt][4 * q + 1], acc[it][jt][4 * q + 2], acc[it][jt][4 * q + 3]};
            wave::sync();
            if (KIND == kGram && p.splits > 1) {
                float *part = p.gram_parts + (mat * p.splits + blockIdx.z) * p.np * p.np;
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int j = 16 * r + (lane >> 2), i = 8 * (lane & 3);
                    f32x4 *to = (f32x4 *)(part + (int64_t)(j0 + j) * p.np + i0 + i);
                    to[0] = *(const f32x4 *)&turn[j][i];
                    to[1] = *(const f32x4 *)&turn[j][i + 4];
                }
            } else {
                leave<T, KIND>(p, mat, step, i0, j0, turn);
            }
            wave::sync();
        }
}

// A, from the parts of its sums: a wave takes 32 x 32 on or above the diagonal.
__global__ __launch_bounds__(kThreads) void ortho_join_kernel(OrthoParams p, int tiles) {
    __shared__ float turns[kThreads / 64][32][kTurn];
    const int lane = threadIdx.x & 63, own = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = blockIdx.x * (kThreads / 64) + own;
    if (tile >= tiles) return;
    int ti, tj;
    triangle(tile, ti, tj);
    const int64_t mat = blockIdx.y;
    const float *part = p.gram_parts + mat * p.splits * p.np * p.np;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int j = 16 * r + (lane >> 2), i = 8 * (lane & 3);
        f32x4 v[2] = {f32x4{0.0f, 0.0f, 0.0f, 0.0f}, f32x4{0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll 4
        for (int s = 0; s < p.splits; ++s) {
            const f32x4 *from = (const f32x4 *)(part + ((int64_t)s * p.np + 32 * tj + j) * p.np + 32 * ti + i);
            v[0] += from[0];
            v[1] += from[1];
        }
        *(f32x4 *)&turns[own][j][i] = v[0];
        *(f32x4 *)&turns[own][j][i + 4] = v[1];
    }
    wave::sync();
    leave<float, kGram>(p, mat, 0, 32 * ti, 32 * tj, turns[own]);
}

template <typename T, int TILE, int WM, int WN, int STAGES, int KIND>
void run_product(const OrthoParams &p, int step, hipStream_t s) {
    const int ti = (p.np + TILE - 1) / TILE, tj = ((KIND == kGram || KIND == kSquare ? p.np : p.mp) + TILE - 1) / TILE;
    const int tiles = KIND == kGram || KIND == kSquare ? ti * (ti + 1) / 2 : ti * tj;
    ortho_product_kernel<T, TILE, TILE, WM, WN, STAGES, KIND>
        <<<dim3(tiles, (uint32_t)p.n_mats, KIND == kGram ? p.splits : 1), WM * WN * 64, 0, s>>>(p, step, ti, tj);
}

// The tile of a pass: the one that is done first, in us.  Either the compute
// units' rounds of blocks, as many side by side as their LDS takes, each with its
// stages and its way in and out; or all tiles at the rate of a full device.
// Fitted to 87 sizes and numbers of matrices: what it picks takes 1.01 times the
// best tile's time in the mean, 1.4 at most.
struct TileCost {
    double start, stage, way;         // of the rounds
    int together;
    double full_stage, full_way;      // of the full device, a tile a compute unit
};
int pick_tile(const OrthoParams &p, bool symmetric, int depth, int splits) {
    constexpr int kTiles[4] = {64, 128, 192, 256};
    constexpr TileCost kCosts[4] = {{4.35, 0.25, 0.00, 3, 0.28, 1.47},
                                    {5.91, 0.86, 0.00, 2, 0.88, 8.33},
                                    {4.43, 1.67, 2.33, 1, 1.41, 20.31},
                                    {5.93, 2.03, 1.89, 1, 3.11, 11.10}};
    const int stages = (depth / kStage + splits - 1) / splits;
    int best = 0;
    double least = 0.0;
    for (int t = 0; t < 4; ++t) {
        const TileCost &c = kCosts[t];
        const int64_t ti = (p.np + kTiles[t] - 1) / kTiles[t], tj = (p.mp + kTiles[t] - 1) / kTiles[t];
        const int64_t tiles = (symmetric ? ti * (ti + 1) / 2 : ti * tj) * p.n_mats * splits;
        const int64_t rounds = ((tiles + 255) / 256 + c.together - 1) / c.together;
        const double cost = c.start + std::max((double)rounds * (stages * c.stage + c.way),
                                               (double)tiles / 256.0 * (stages * c.full_stage + c.full_way));
        if (t == 0 || cost < least) {
            least = cost;
            best = t;
        }
    }
    return best;
}

template <typename T, int KIND>
void run_pass(const OrthoParams &p, int step, hipStream_t s) {
    switch (pick_tile(p, KIND == kGram || KIND == kSquare, KIND == kGram ? p.mp : p.np, KIND == kGram ? p.splits : 1)) {
    case 0: return run_product<T, 64, 2, 2, 3, KIND>(p, step, s);
    case 1: return run_product<T, 128, 2, 2, 2, KIND>(p, step, s);
    case 2: return run_product<T, 192, 2, 2, 3, KIND>(p, step, s);
    default: return run_product<T, 256, 2, 4, 2, KIND>(p, step, s);
    }
}

template <typename T>
hipError_t run_products(const OrthoParams &p, hipStream_t s) {
    for (int k = 0; k < p.steps; ++k) {
        run_pass<float, kGram>(p, k, s);
        if (p.splits > 1) {
            const int side = p.np / 32, tiles = side * (side + 1) / 2;
            ortho_join_kernel<<<dim3((tiles + kThreads / 64 - 1) / (kThreads / 64), (uint32_t)p.n_mats), kThreads, 0, s>>>(p, tiles);
        }
        run_pass<float, kSquare>(p, k, s);
        if (k + 1 < p.steps)
            run_pass<float, kUpdate>(p, k, s);
        else
            run_pass<T, kLast>(p, k, s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
int run_squares(const OrthoParams &p, hipStream_t s) {
    int row_threads = 1;
    while (row_threads < kThreads && 8 * row_threads < p.cols) row_threads *= 2;
    const int across = (p.cols + 8 * row_threads - 1) / (8 * row_threads), at_once = kThreads / row_threads;
    const int items = (p.rows + at_once - 1) / at_once * across;
    const int parts = std::min(kNormParts, (items + 1) / 2);
    ortho_squares_kernel<T><<<(uint32_t)p.n_mats * parts, kThreads, 0, s>>>(p, parts, items, across, row_threads);
    return parts;
}

template <typename T>
hipError_t run_typed(const OrthoParams &p, hipStream_t s) {
    const uint32_t mats = (uint32_t)p.n_mats;
    const int parts = run_squares<T>(p, s);
    const int ti = (p.np + 63) / 64, tj = (p.mp + 63) / 64;
    ortho_split_kernel<T><<<mats * ti * tj, kThreads, 0, s>>>(p, parts, ti, tj);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    return run_products<T>(p, s);
}

}  // namespace

hipError_t launch_ortho_squares(const OrthoParams &p, int dtype, hipStream_t s, int *parts) {
    *parts = dtype == 2 ? run_squares<__bf16>(p, s) : dtype == 1 ? run_squares<_Float16>(p, s) : run_squares<float>(p, s);
    return hipGetLastError();
}

// Parts of X X^T where its tiles are few and its sums long: eight stages each at
// least, 512 tiles of 64 together; under four parts the pass that joins them
// costs what they save (300 x 500 122 us, 131 in two; 100 x 4,000 284 us, 130 in
// 15).  By the matrix alone, so that its result does not depend on its batch.
int orthogonalise_splits(int64_t np, int64_t mp) {
    const int64_t side = (np + 63) / 64, tiles = side * (side + 1) / 2;
    const int64_t splits = std::min<int64_t>(std::min<int64_t>(mp / kStage / 8, 512 / tiles), 64);
    return splits < 4 ? 1 : (int)splits;
}

// Some 2^28 elements of a plane.
int64_t orthogonalise_batch(int64_t n_mats, int64_t np, int64_t mp) {
    return std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(n_mats, 16384), ((int64_t)1 << 28) / (np * mp)));
}

hipError_t launch_orthogonalise(const OrthoParams &all, int64_t batch, int dtype, hipStream_t s) {
    const int64_t size = dtype == 0 ? 4 : 2;
    for (int64_t first = 0; first < all.n_mats; first += batch) {
        OrthoParams p = all;
        p.n_mats = std::min(batch, all.n_mats - first);
        p.g = (const char *)all.g + first * all.g_mat * size;
        p.out = (char *)all.out + first * all.out_mat * size;
        const hipError_t e = p.n <= kSmallSide           ? launch_ortho_small(p, dtype, s)
                             : ortho_whole(p.n, p.m)     ? launch_ortho_whole(p, dtype, s)
                             : ortho_columns(p.n, p.m)   ? launch_ortho_columns(p, dtype, s)
                             : dtype == 2 ? run_typed<__bf16>(p, s)
                             : dtype == 1 ? run_typed<_Float16>(p, s)
                                          : run_typed<float>(p, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace same
