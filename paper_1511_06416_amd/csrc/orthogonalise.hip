// Orthogonalising an update by Newton-Schulz products, for gfx950:
//   X = G / (|G| + eps), |G| the root of the sum of squares, then per step
//   A = X X^T,  B = b A + c A A,  X <- a X + B X
// with X's rows along the smaller side of G, so that A is small.
//
// Products run on the fp16 matrix units.  A number is held as the sum of two
// fp16, hi + lo, times a power of two that keeps both in the type's normal
// range: 22 bits.  Of a product of two such, hi hi + hi lo + lo hi are formed
// (what is left out is 2^-22 of it), summed in fp32.  fp32 and fp16 updates
// take all three: 4e-7 of the result's size against 64 bits, where a form in
// fp32 has 1.5e-6.  bf16 ones take hi hi alone, with a X and b A in full: 2e-3,
// as much as rounding the result to bf16 (1.7e-3).
// A and B are symmetric: tiles on and above the diagonal are formed and written
// to both places.
#include <algorithm>

#include "step.hpp"
#include "wave.hpp"

namespace same {
namespace {

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256;
constexpr int kStage = 32;  // columns of a stage

__device__ __forceinline__ void split(float v, _Float16 &hi, _Float16 &lo) {
    hi = (_Float16)v;
    lo = (_Float16)(v - (float)hi);
}

template <typename T>
__device__ __forceinline__ float read(const OrthoParams &p, int64_t mat, int i, int j) {  // X's element
    return (float)((const T *)p.g)[mat * p.g_mat + (p.tall ? j * p.g_row + i : i * p.g_row + j)];
}

// Parts of the sums of squares, in 64 bits: no update is too large or small.
template <typename T>
__global__ __launch_bounds__(kThreads) void ortho_squares_kernel(OrthoParams p) {
    __shared__ double sums[kThreads / 64];
    const int64_t mat = blockIdx.y, n = (int64_t)p.rows * p.cols;
    double t = 0.0;
    for (int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x; e < n; e += (int64_t)gridDim.x * kThreads) {
        const int64_t i = e / p.cols, j = e - i * p.cols;
        const double v = (double)(float)((const T *)p.g)[mat * p.g_mat + i * p.g_row + j];
        t = __builtin_fma(v, v, t);
    }
    for (int o = 32; o; o >>= 1) t += __shfl_xor(t, o);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = t;
    __syncthreads();
    if (threadIdx.x == 0) {
        t = 0.0;
        for (int w = 0; w < kThreads / 64; ++w) t += sums[w];
        p.squares[mat * kNormParts + blockIdx.x] = t;
    }
}

// X in planes, both ways, zeros around it: a block takes 64 x 64.
template <typename T>
__global__ __launch_bounds__(kThreads) void ortho_split_kernel(OrthoParams p, int parts) {
    __shared__ float tile[64][65];
    const int64_t mat = blockIdx.z;
    double total = 0.0;
    for (int i = 0; i < parts; ++i) total += p.squares[mat * kNormParts + i];
    const float factor = (float)((double)p.sx / (__builtin_sqrt(total) + (double)p.eps));
    const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;
    const int c = threadIdx.x & 63;
    for (int r = threadIdx.x >> 6; r < 64; r += kThreads / 64) {
        // along g's rows
        const int i = p.tall ? i0 + c : i0 + r, j = p.tall ? j0 + r : j0 + c;
        const float v = i < p.n && j < p.m ? read<T>(p, mat, i, j) * factor : 0.0f;
        tile[p.tall ? c : r][p.tall ? r : c] = v;
    }
    __syncthreads();
    const int64_t x0 = mat * p.np * p.mp;
    for (int r = threadIdx.x >> 6; r < 64; r += kThreads / 64) {
        _Float16 hi, lo;
        split(tile[r][c], hi, lo);
        const int64_t at = x0 + (int64_t)(i0 + r) * p.mp + j0 + c;
        p.x.hi[at] = hi;
        p.x.lo[at] = lo;
        split(tile[c][r], hi, lo);
        const int64_t back = x0 + (int64_t)(j0 + r) * p.np + i0 + c;
        p.xt[0].hi[back] = hi;
        p.xt[0].lo[back] = lo;
    }
}

enum Kind { kGram, kSquare, kUpdate, kLast };

// C[i][j] = sum_k P[i][k] Q[j][k] over a square tile, WM x WN waves, operands
// staged in LDS: rows of 64 bytes, whose 16-byte chunks are turned by the row
// so that a read of 32 rows meets no bank twice.
template <typename T, int TILE, int WM, int WN, int PROD, int KIND>
__global__ __launch_bounds__(WM * WN * 64) void ortho_product_kernel(OrthoParams p, int step, int tiles_i, int tiles_j) {
    constexpr int MT = TILE / WM / 32, NT = TILE / WN / 32, PL = PROD == 1 ? 1 : 2;
    constexpr int kPlane = TILE * kStage;                 // elements of a staged plane
    constexpr int kLoads = TILE * 4 / (WM * WN * 64);     // 16-byte loads a lane, per plane
    static_assert(kLoads >= 1 && kLoads * WM * WN * 64 == TILE * 4, "every lane stages the same");
    __shared__ _Float16 stage[2][2 * PL][kPlane];
    const int lane = threadIdx.x & 63, own = threadIdx.x >> 6;
    int ti, tj;
    if (KIND == kGram || KIND == kSquare) {
        // on and above the diagonal, by columns
        tj = (int)((__builtin_sqrtf(8.0f * (float)blockIdx.x + 1.0f) - 1.0f) * 0.5f);
        while ((tj + 1) * (tj + 2) / 2 <= (int)blockIdx.x) ++tj;
        while (tj * (tj + 1) / 2 > (int)blockIdx.x) --tj;
        ti = blockIdx.x - tj * (tj + 1) / 2;
    } else {
        ti = blockIdx.x % tiles_i;
        tj = blockIdx.x / tiles_i;
    }
    const int64_t mat = blockIdx.y;
    const int64_t x0 = mat * p.np * p.mp, a0 = mat * p.np * p.np;
    const int ld = KIND == kGram ? p.mp : p.np, depth = ld;
    const Planes from = p.xt[step & 1], to = p.xt[(step & 1) ^ 1];
    const Planes left = KIND == kGram ? p.x : KIND == kSquare ? p.a : p.b;
    const Planes right = KIND == kGram ? p.x : KIND == kSquare ? p.a : from;
    const int64_t l0 = (KIND == kGram ? x0 : a0) + (int64_t)ti * TILE * ld;
    const int64_t r0 = (KIND == kSquare ? a0 : x0) + (int64_t)tj * TILE * ld;
    const _Float16 *src[2 * PL];
    src[0] = left.hi + l0;
    src[PL] = right.hi + r0;
    if (PL == 2) {
        src[1] = left.lo + l0;
        src[PL + 1] = right.lo + r0;
    }
    auto fetch = [&](int buffer, int k) {
#pragma unroll
        for (int s = 0; s < 2 * PL; ++s)
#pragma unroll
            for (int l = 0; l < kLoads; ++l) {
                const int slot = (own * kLoads + l) * 64 + lane, row = slot >> 2;
                const int chunk = (slot & 3) ^ ((row >> 1) & 3);
                __builtin_amdgcn_global_load_lds(
                    (const __attribute__((address_space(1))) void *)(src[s] + (int64_t)row * ld + k + chunk * 8),
                    (__attribute__((address_space(3))) void *)&stage[buffer][s][(own * kLoads + l) * 512], 16, 0, 0);
            }
    };
    f32x16 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    const int wi = (own % WM) * (TILE / WM), wj = (own / WM) * (TILE / WN);
    auto operand = [&](int buffer, int s, int row, int t) {
        return *(const f16x8 *)&stage[buffer][s][row * kStage + (((2 * t + (lane >> 5)) ^ ((row >> 1) & 3)) << 3)];
    };
    // a barrier alone does not wait for loads into LDS
    auto arrive = [&]() {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    fetch(0, 0);
    arrive();
    for (int k = 0, buffer = 0; k < depth; k += kStage, buffer ^= 1) {
        if (k + kStage < depth) fetch(buffer ^ 1, k + kStage);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f16x8 l[PL][MT], r[PL][NT];
#pragma unroll
            for (int s = 0; s < PL; ++s) {
#pragma unroll
                for (int i = 0; i < MT; ++i) l[s][i] = operand(buffer, s, wi + 32 * i + (lane & 31), t);
#pragma unroll
                for (int j = 0; j < NT; ++j) r[s][j] = operand(buffer, PL + s, wj + 32 * j + (lane & 31), t);
            }
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    if (PL == 2) {
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[PL - 1][i], r[0][j], acc[i][j], 0, 0, 0);
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[0][i], r[PL - 1][j], acc[i][j], 0, 0, 0);
                    }
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[0][i], r[0][j], acc[i][j], 0, 0, 0);
                }
        }
        arrive();
    }
    // a lane holds column j and, in fours, rows i
    const float ca = p.coef[step][0], cb = p.coef[step][1], cc = p.coef[step][2];
#pragma unroll
    for (int it = 0; it < MT; ++it)
#pragma unroll
        for (int jt = 0; jt < NT; ++jt) {
            const int j = tj * TILE + wj + 32 * jt + (lane & 31);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int i = ti * TILE + wi + 32 * it + 8 * q + 4 * (lane >> 5);
                float v[4];
                if (KIND == kGram) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = acc[it][jt][4 * q + e] * (p.sa / (p.sx * p.sx));
                } else {
                    // what stays of the old: A[j][i..] (symmetric), or X^T
                    const int64_t at = (KIND == kSquare ? a0 : x0) + (int64_t)j * p.np + i;
                    const Planes old = KIND == kSquare ? p.a : from;
                    const f16x4 hi = *(const f16x4 *)(old.hi + at), lo = *(const f16x4 *)(old.lo + at);
                    const float keep = KIND == kSquare ? cb * (p.sb / p.sa) : ca;
                    const float take = KIND == kSquare ? cc * (p.sb / (p.sa * p.sa)) : 1.0f / p.sb;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        v[e] = __builtin_fmaf(take, acc[it][jt][4 * q + e], keep * ((float)hi[e] + (float)lo[e]));
                }
                if (KIND == kLast) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (i + e < p.n && j < p.m)
                            ((T *)p.out)[mat * p.out_mat + (p.tall ? j * p.out_row + i + e : (i + e) * p.out_row + j)] =
                                (T)(v[e] * (p.out_scale / p.sx));
                    continue;
                }
                f16x4 hi, lo;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    _Float16 h, l;
                    split(v[e], h, l);
                    hi[e] = h;
                    lo[e] = l;
                }
                const Planes d = KIND == kGram ? p.a : p.b;
                if (KIND == kUpdate) {
                    const int64_t at = x0 + (int64_t)j * p.np + i;
                    *(f16x4 *)(to.hi + at) = hi;
                    *(f16x4 *)(to.lo + at) = lo;
                } else if (ti != tj) {  // a tile on the diagonal holds both, rounded apart: one of them is taken
                    const int64_t at = a0 + (int64_t)j * p.np + i;
                    *(f16x4 *)(d.hi + at) = hi;
                    *(f16x4 *)(d.lo + at) = lo;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int64_t at = KIND == kUpdate ? x0 + (int64_t)(i + e) * p.mp + j : a0 + (int64_t)(i + e) * p.np + j;
                    const Planes w = KIND == kUpdate ? p.x : d;
                    w.hi[at] = hi[e];
                    w.lo[at] = lo[e];
                }
            }
        }
}

template <typename T, int TILE, int WM, int WN, int PROD>
hipError_t run_products(const OrthoParams &p, hipStream_t s) {
    const int ti = p.np / TILE, tj = p.mp / TILE, tri = ti * (ti + 1) / 2;
    constexpr int threads = WM * WN * 64;
    const dim3 small(tri, (uint32_t)p.n_mats), whole(ti * tj, (uint32_t)p.n_mats);
    for (int k = 0; k < p.steps; ++k) {
        ortho_product_kernel<float, TILE, WM, WN, PROD, kGram><<<small, threads, 0, s>>>(p, k, ti, tj);
        ortho_product_kernel<float, TILE, WM, WN, PROD, kSquare><<<small, threads, 0, s>>>(p, k, ti, tj);
        if (k + 1 < p.steps)
            ortho_product_kernel<float, TILE, WM, WN, PROD, kUpdate><<<whole, threads, 0, s>>>(p, k, ti, tj);
        else
            ortho_product_kernel<T, TILE, WM, WN, PROD, kLast><<<whole, threads, 0, s>>>(p, k, ti, tj);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T, int PROD>
hipError_t run_typed(const OrthoParams &p, hipStream_t s) {
    const int64_t n = (int64_t)p.rows * p.cols;
    const int parts = (int)std::min<int64_t>(kNormParts, (n + 4 * kThreads - 1) / (4 * kThreads));
    ortho_squares_kernel<T><<<dim3(parts, (uint32_t)p.n_mats), kThreads, 0, s>>>(p);
    ortho_split_kernel<T><<<dim3(p.mp / 64, p.np / 64, (uint32_t)p.n_mats), kThreads, 0, s>>>(p, parts);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (p.np % 128 == 0 && p.mp % 128 == 0) return run_products<T, 128, 2, 2, PROD>(p, s);
    return run_products<T, 64, 2, 2, PROD>(p, s);
}

}  // namespace

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
        const hipError_t e = p.n <= kSmallSide ? launch_ortho_small(p, dtype, s)
                             : dtype == 2 ? run_typed<__bf16, 1>(p, s)
                             : dtype == 1 ? run_typed<_Float16, 3>(p, s)
                                          : run_typed<float, 3>(p, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace same
