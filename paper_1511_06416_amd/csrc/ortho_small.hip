// Orthogonalised updates whose smaller side is at most 32, for gfx950.  Every
// step's factor is a polynomial in A = X X^T, so all of them commute and the
// steps run on that small matrix alone:
//   P = a + b A + c A^2,  A <- P A P,  T <- P T,   and out = T G at the end:
// the update is read for A and once more for out.  A holds the squares of the
// singular values and T's large entries cancel in the strong directions: in 32
// bits that would lose digits that the steps on X keep, so all of it is in 64,
// on the matrix units (16 x 16 x 4).
//
// A product's output leaves a lane with the elements (4 i + lane / 16,
// lane % 16) of a 16 x 16 tile; the operand of the next product needs the row
// lane % 16 and the columns 4 t + lane / 16: of a symmetric matrix the same
// numbers, so the chain needs no exchange within a tile.
//
// Measured: 1,000 of 8 x 128 8.8 us (12.6 with the factors through LDS and all 16
// columns contracted), 1,000 of 30 x 40 33, mostly the steps' chain of dependent
// 64-bit products; one launch where a block holds a matrix's columns.
#include <algorithm>

#include "step.hpp"
#include "wave.hpp"

namespace same {
namespace {

typedef double f64x4 __attribute__((ext_vector_type(4)));
using wave::Loose;

constexpr int kThreads = 256, kWaves = 4;

// FOURS of the operands' columns, four each; zeros behind them would add nothing.
template <int FOURS>
__device__ __forceinline__ f64x4 product(f64x4 p, f64x4 q, f64x4 c) {
#pragma unroll
    for (int t = 0; t < FOURS; ++t) c = __builtin_amdgcn_mfma_f64_16x16x4f64(p[t], q[t], c, 0, 0, 0);
    return c;
}
__device__ __forceinline__ f64x4 zero4() { return f64x4{0.0, 0.0, 0.0, 0.0}; }

// SIDE tiles of 16 rows.  Tile (i, j) of a symmetric matrix, as an operand.
template <int SIDE>
struct Tiles {
    f64x4 v[SIDE][SIDE][64];
};

// Adds X X^T over the columns [beg, end) that this wave takes: four columns a
// lane and step, the same numbers for both operands.
template <typename T, int SIDE>
__device__ __forceinline__ void gram(const OrthoParams &p, int64_t mat, int beg, int end, f64x4 (&acc)[SIDE][SIDE]) {
    const int lane = threadIdx.x & 63, own = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const T *base = (const T *)p.g + mat * p.g_mat;
    for (int j0 = beg + own * 16; j0 < end; j0 += kWaves * 16) {
        const int j = j0 + 4 * g;
        f64x4 x[SIDE];
#pragma unroll
        for (int s = 0; s < SIDE; ++s) {
            const int row = 16 * s + r, at = min(row, p.n - 1);
            float v[4];
            if (p.tall) {
#pragma unroll
                for (int t = 0; t < 4; ++t) v[t] = (float)base[min(j + t, p.m - 1) * p.g_row + at];
            } else if (j + 4 <= p.m) {
                const Loose<T, 4> l = *(const Loose<T, 4> *)(base + at * p.g_row + j);
#pragma unroll
                for (int t = 0; t < 4; ++t) v[t] = (float)l.v[t];
            } else {
#pragma unroll
                for (int t = 0; t < 4; ++t) v[t] = (float)base[at * p.g_row + min(j + t, p.m - 1)];
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) x[s][t] = row < p.n && j + t < end ? (double)v[t] : 0.0;
        }
#pragma unroll
        for (int a = 0; a < SIDE; ++a)
#pragma unroll
            for (int b = 0; b < SIDE; ++b) acc[a][b] = product<4>(x[a], x[b], acc[a][b]);
    }
}

// The waves' sums, as operands in tiles.v; every wave gets there.
template <int SIDE>
__device__ __forceinline__ void gather(f64x4 (&acc)[SIDE][SIDE], Tiles<SIDE> (&part)[kWaves], Tiles<SIDE> &sum) {
    const int lane = threadIdx.x & 63, own = threadIdx.x >> 6;
#pragma unroll
    for (int a = 0; a < SIDE; ++a)
#pragma unroll
        for (int b = 0; b < SIDE; ++b) part[own].v[b][a][lane] = acc[a][b];
    __syncthreads();
    for (int e = threadIdx.x; e < SIDE * SIDE * 64; e += kThreads) {
        f64x4 t = zero4();
        for (int w = 0; w < kWaves; ++w) t += part[w].v[0][0][e];
        sum.v[0][0][e] = t;
    }
    __syncthreads();
}

// From A = G G^T in `a` to T in `t`, by one wave a tile.
template <int SIDE, int FOURS>
__device__ __forceinline__ void iterate(const OrthoParams &p, Tiles<SIDE> &a, Tiles<SIDE> &t, Tiles<SIDE> &u) {
    const int lane = threadIdx.x & 63, own = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    // the trace of G G^T is the sum of squares
    double trace = 0.0;
#pragma unroll
    for (int s = 0; s < SIDE; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) trace += 4 * e + g == r ? a.v[s][s][lane][e] : 0.0;
    for (int o = 32; o; o >>= 1) trace += __shfl_xor(trace, o);
    const double f = 1.0 / (__builtin_sqrt(trace) + (double)p.eps);
    if constexpr (SIDE == 1) {
        // one wave, whose numbers already are the next operands
        if (own == 0) {
            f64x4 x = a.v[0][0][lane] * f * f, one = zero4();   // f^2 may pass 64 bits where A is 0
#pragma unroll
            for (int e = 0; e < 4; ++e) one[e] = 4 * e + g == r ? 1.0 : 0.0;
            f64x4 y = one;
            // without a branch between products and what reads them: the compiler
            // has left too few wait states there
            auto factor = [&](int step) {
                const double ca = p.coef[step][0], cb = p.coef[step][1], cc = p.coef[step][2];
                f64x4 s = product<FOURS>(x, x, zero4());
#pragma unroll
                for (int e = 0; e < 4; ++e) s[e] = cc * s[e] + cb * x[e] + ca * one[e];
                return s;
            };
            for (int step = 0; step + 1 < p.steps; ++step) {
                const f64x4 s = factor(step);
                x = product<FOURS>(s, x, zero4());
                y = product<FOURS>(s, y, zero4());
                x = product<FOURS>(s, x, zero4());
            }
            y = product<FOURS>(factor(p.steps - 1), y, zero4());
            t.v[0][0][lane] = y * (f * (double)p.out_scale);
        }
        __syncthreads();
        return;
    }
    __syncthreads();   // every wave has the trace: the tiles that it comes from are scaled in place
    static_assert(SIDE == 1 || SIDE * SIDE == kWaves, "a wave takes a tile");
    const int i = own / SIDE % SIDE, j = own % SIDE;   // the output tile of this wave
    // P Q of two matrices that commute: tile (i, j), which is operand (j, i)
    auto times = [&](const Tiles<SIDE> &l, const Tiles<SIDE> &q) {
        f64x4 c = zero4();
#pragma unroll
        for (int k = 0; k < SIDE; ++k) c = product<FOURS>(l.v[i][k][lane], q.v[j][k][lane], c);
        return c;
    };
    // one of f's factors at a time: f^2 may pass 64 bits where A is 0
    a.v[j][i][lane] = a.v[j][i][lane] * f * f;
    f64x4 one = zero4();
#pragma unroll
    for (int e = 0; e < 4; ++e) one[e] = i == j && 4 * e + g == r ? 1.0 : 0.0;
    t.v[j][i][lane] = one;
    __syncthreads();
    // straight-line code between products and what reads them, as above
    auto factor = [&](int step) {
        const double ca = p.coef[step][0], cb = p.coef[step][1], cc = p.coef[step][2];
        f64x4 s = times(a, a);
        const f64x4 old = a.v[j][i][lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = cc * s[e] + cb * old[e] + (i == j && 4 * e + g == r ? ca : 0.0);
        u.v[j][i][lane] = s;
        __syncthreads();
    };
    for (int step = 0; step + 1 < p.steps; ++step) {
        factor(step);
        const f64x4 next = times(u, t), half = times(u, a);
        __syncthreads();
        t.v[j][i][lane] = next;
        a.v[j][i][lane] = half;
        __syncthreads();
        const f64x4 whole = times(u, a);
        __syncthreads();
        a.v[j][i][lane] = whole;
        __syncthreads();
    }
    factor(p.steps - 1);
    const f64x4 last = times(u, t);
    __syncthreads();
    t.v[j][i][lane] = last * (f * (double)p.out_scale);
    __syncthreads();
}

// out = T G over the columns [beg, end): a wave takes 16 at a time.
template <typename T, int SIDE, int FOURS>
__device__ __forceinline__ void apply(const OrthoParams &p, int64_t mat, int beg, int end, const Tiles<SIDE> &t) {
    const int lane = threadIdx.x & 63, own = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
    const T *base = (const T *)p.g + mat * p.g_mat;
    T *out = (T *)p.out + mat * p.out_mat;
    const int64_t down = p.tall ? 1 : p.g_row, across = p.tall ? p.g_row : 1;
    const int64_t out_down = p.tall ? 1 : p.out_row, out_across = p.tall ? p.out_row : 1;
    for (int j0 = beg + own * 16; j0 < end; j0 += kWaves * 16) {
        const int j = j0 + c;
        f64x4 x[SIDE];
#pragma unroll
        for (int s = 0; s < SIDE; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int row = 16 * s + 4 * e + g;
                float v = 0.0f;
                if (e < FOURS) v = (float)base[min(row, p.n - 1) * down + min(j, p.m - 1) * across];
                x[s][e] = row < p.n && j < end ? (double)v : 0.0;
            }
#pragma unroll
        for (int a = 0; a < SIDE; ++a) {
            f64x4 y = zero4();
#pragma unroll
            for (int k = 0; k < SIDE; ++k) y = product<FOURS>(t.v[a][k][lane], x[k], y);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int row = 16 * a + 4 * e + g;
                if (row < p.n && j < end) out[row * out_down + j * out_across] = (T)(float)y[e];
            }
        }
    }
}

template <typename T, int SIDE, int FOURS>
__global__ __launch_bounds__(kThreads) void ortho_small_kernel(OrthoParams p) {
    __shared__ Tiles<SIDE> part[kWaves], a;
    const int64_t mat = blockIdx.x;
    f64x4 acc[SIDE][SIDE];
#pragma unroll
    for (int i = 0; i < SIDE; ++i)
#pragma unroll
        for (int j = 0; j < SIDE; ++j) acc[i][j] = zero4();
    gram<T, SIDE>(p, mat, 0, p.m, acc);
    gather<SIDE>(acc, part, a);
    iterate<SIDE, FOURS>(p, a, part[0], part[1]);
    // out may be g: it is written where this block alone has read
    apply<T, SIDE, FOURS>(p, mat, 0, p.m, part[0]);
}

// Long rows: parts of A, the steps, parts of out.
template <typename T, int SIDE>
__global__ __launch_bounds__(kThreads) void ortho_gram_kernel(OrthoParams p) {
    __shared__ Tiles<SIDE> part[kWaves], a;
    const int64_t mat = blockIdx.x / p.parts;
    const int beg = (int)(blockIdx.x - mat * p.parts) * p.part_cols;
    f64x4 acc[SIDE][SIDE];
#pragma unroll
    for (int i = 0; i < SIDE; ++i)
#pragma unroll
        for (int j = 0; j < SIDE; ++j) acc[i][j] = zero4();
    gram<T, SIDE>(p, mat, beg, min(p.m, beg + p.part_cols), acc);
    gather<SIDE>(acc, part, a);
    Tiles<SIDE> *to = (Tiles<SIDE> *)p.small_parts + blockIdx.x;
    for (int e = threadIdx.x; e < SIDE * SIDE * 64; e += kThreads) to->v[0][0][e] = a.v[0][0][e];
}

template <int SIDE, int FOURS>
__global__ __launch_bounds__(kThreads) void ortho_steps_kernel(OrthoParams p) {
    __shared__ Tiles<SIDE> part[kWaves], a;
    const int64_t mat = blockIdx.x;
    const int lane = threadIdx.x & 63, own = threadIdx.x >> 6;
    const Tiles<SIDE> *from = (const Tiles<SIDE> *)p.small_parts + mat * p.parts;
    f64x4 acc[SIDE][SIDE];
#pragma unroll
    for (int i = 0; i < SIDE; ++i)
#pragma unroll
        for (int j = 0; j < SIDE; ++j) {
            acc[i][j] = zero4();
            for (int k = own; k < p.parts; k += kWaves) acc[i][j] += from[k].v[j][i][lane];
        }
    gather<SIDE>(acc, part, a);
    iterate<SIDE, FOURS>(p, a, part[0], part[1]);
    Tiles<SIDE> *to = (Tiles<SIDE> *)p.small_factors + mat;
    for (int e = threadIdx.x; e < SIDE * SIDE * 64; e += kThreads) to->v[0][0][e] = part[0].v[0][0][e];
}

template <typename T, int SIDE, int FOURS>
__global__ __launch_bounds__(kThreads) void ortho_apply_kernel(OrthoParams p) {
    __shared__ Tiles<SIDE> t;
    const int64_t mat = blockIdx.x / p.parts;
    const int beg = (int)(blockIdx.x - mat * p.parts) * p.part_cols;
    const Tiles<SIDE> *from = (const Tiles<SIDE> *)p.small_factors + mat;
    for (int e = threadIdx.x; e < SIDE * SIDE * 64; e += kThreads) t.v[0][0][e] = from->v[0][0][e];
    __syncthreads();
    apply<T, SIDE, FOURS>(p, mat, beg, min(p.m, beg + p.part_cols), t);
}

template <typename T, int SIDE, int FOURS>
hipError_t run_side(const OrthoParams &p, hipStream_t s) {
    const uint32_t mats = (uint32_t)p.n_mats, parts = mats * (uint32_t)p.parts;
    if (p.parts == 1) {
        ortho_small_kernel<T, SIDE, FOURS><<<mats, kThreads, 0, s>>>(p);
    } else {
        ortho_gram_kernel<T, SIDE><<<parts, kThreads, 0, s>>>(p);
        ortho_steps_kernel<SIDE, FOURS><<<mats, kThreads, 0, s>>>(p);
        ortho_apply_kernel<T, SIDE, FOURS><<<parts, kThreads, 0, s>>>(p);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t run_typed(const OrthoParams &p, hipStream_t s) {
    // contracted rows, in fours: a count at run time costs more than it saves
    if (p.n <= 4) return run_side<T, 1, 1>(p, s);
    if (p.n <= 8) return run_side<T, 1, 2>(p, s);
    return p.n <= 16 ? run_side<T, 1, 4>(p, s) : run_side<T, 2, 4>(p, s);
}

}  // namespace

// Columns are cut into parts of 512 at least, three launches (30 x 4,096 73 us in
// two parts, 33 in eight; 4 x 3,000 42 us in one block, 19 in five), whatever the
// number of matrices, so that a matrix's result does not depend on its batch.
void ortho_small_parts(int64_t n, int64_t m, int32_t *parts, int32_t *part_cols, size_t *tile_bytes) {
    *parts = (int32_t)std::max<int64_t>(1, std::min<int64_t>(256, m / 512));
    *part_cols = (int32_t)((m + *parts - 1) / *parts + 63) / 64 * 64;
    *parts = (int32_t)std::max<int64_t>(1, (m + *part_cols - 1) / std::max(1, *part_cols));
    *tile_bytes = (n <= 16 ? sizeof(Tiles<1>) : sizeof(Tiles<2>));
}

hipError_t launch_ortho_small(const OrthoParams &p, int dtype, hipStream_t s) {
    if (dtype == 2) return run_typed<__bf16>(p, s);
    if (dtype == 1) return run_typed<_Float16>(p, s);
    return run_typed<float>(p, s);
}

}  // namespace same
