// Norms of query and key heads with the rotation by position, for gfx950:
//   r = (mean x^2 + eps)^-1/2, z = w x r, and for the pairs (i, i + h), i < h:
//   y_i = z_i cos a_i - z_{i+h} sin a_i, y_{i+h} = z_{i+h} cos a_i + z_i sin a_i
// with a_i = position x angle_i.  Gradient, with dz the inverse rotation of dy
// and xhat = x r: dx = r (w dz - xhat mean(w dz xhat)), dw = sum dz xhat.
//
// Bytes bound it.  A lane takes W elements at one place and the W that turn
// with them, so that a rotation stays in the lane; a row (a head's vector) is a
// group of lanes, whose sums are exchanges within the wave.  A wave takes a
// token, whose sines serve all of its heads; they are made for as many of its
// tokens at a time as there are lanes, a pair a lane (21,120 tokens of 8 + 8
// heads of 64, 16 pairs: gradient 33 -> 29 us against a token at a time, 25 ->
// 24 without).
//
// Measured: 65,536 tokens of 16 + 4 heads of 128 in bf16 124 us, 5.4 TB/s, the
// copy's rate.  The 21,120 tokens stay in the last-level cache: 23 us (3.8 TB/s,
// vector units two thirds busy) and, with the gradient, 28 (4.6 TB/s, loads under
// way: more blocks make more parts of the weights' gradients, 32 us with 1,536
// blocks for 1,024).
#include <algorithm>
#include <type_traits>

#include "step.hpp"
#include "wave.hpp"

namespace same {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

template <typename T, int N>
struct alignas(N * sizeof(T) < 16 ? N * sizeof(T) : 16) Chunk {
    T v[N];
};

__device__ __forceinline__ float group_sum(float v, int lanes) { return wave::reduce(v, lanes, wave::Add()); }

// cos and sin of 2 pi t for |t| <= 1/8: Taylor's series, whose next terms are
// below 2^-31.
__device__ __forceinline__ float2 turn_eighth(float t) {
    const float x = t * 6.283185307179586f, x2 = x * x;
    float s = __builtin_fmaf(x2, 2.7557319224e-6f, -1.9841269841e-4f);
    s = __builtin_fmaf(x2, s, 8.3333333333e-3f);
    s = __builtin_fmaf(x2, s, -1.6666666667e-1f);
    s = __builtin_fmaf(x * x2, s, x);
    float c = __builtin_fmaf(x2, -2.7557319224e-7f, 2.4801587302e-5f);
    c = __builtin_fmaf(x2, c, -1.3888888889e-3f);
    c = __builtin_fmaf(x2, c, 4.1666666667e-2f);
    c = __builtin_fmaf(x2, c, -0.5f);
    c = __builtin_fmaf(x2, c, 1.0f);
    return make_float2(c, s);
}

// cos and sin of a position's angle: the turns in two 64-bit parts, less the
// whole ones, then the eighth around the nearest quarter in 32 bits.
__device__ __forceinline__ float2 turn_of(const NormParams &p, int32_t position, int pair) {
    const double at = (double)position, hi = p.turn[pair];
    const double whole = at * hi;
    double t = whole - __builtin_rint(whole);
    t += __builtin_fma(at, hi, -whole) + at * p.turn_low[pair];
    const double quarter = __builtin_rint(4.0 * t);
    const float2 e = turn_eighth((float)__builtin_fma(quarter, -0.25, t));
    const int q = (int)quarter & 3;
    const float c = (q & 1) ? -e.y : e.x, s = (q & 1) ? e.x : e.y;
    return make_float2((q & 2) ? -c : c, (q & 2) ? -s : s);
}

// What a lane reads of a row, as it is: W elements at either place.
template <typename T, int W>
struct Raw {
    Chunk<T, W> lo, hi;
    __device__ __forceinline__ void load(const T *row, int a, int b) {
        lo = *(const Chunk<T, W> *)(row + a);
        hi = *(const Chunk<T, W> *)(row + b);
    }
    __device__ __forceinline__ void widen(float (&v)[2 * W]) const {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            v[i] = (float)lo.v[i];
            v[W + i] = (float)hi.v[i];
        }
    }
};

template <typename T, int W>
__device__ __forceinline__ void store(T *row, int a, int b, const float (&v)[2 * W]) {
    Chunk<T, W> lo, hi;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        lo.v[i] = (T)v[i];
        hi.v[i] = (T)v[W + i];
    }
    *(Chunk<T, W> *)(row + a) = lo;
    *(Chunk<T, W> *)(row + b) = hi;
}

// (mean x^2 + eps)^-1/2 of a row.  Where the squares pass 32 bits, the row becomes
// x 2^-72 and the result is that row's: 128 squares of the type's largest number
// stay below 2^119.  `up` is what x was scaled by.
template <int W>
__device__ __forceinline__ float inverse_norm(const NormParams &p, float (&x)[2 * W], int lanes, float &up) {
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < 2 * W; ++i) ss = __builtin_fmaf(x[i], x[i], ss);
    ss = group_sum(ss, lanes);
    float mean = __builtin_fmaf(ss, p.inv_dim, p.eps);
    up = 1.0f;
    if (__builtin_isinf(mean)) {
        up = 0x1p-72f;
        ss = 0.0f;
#pragma unroll
        for (int i = 0; i < 2 * W; ++i) {
            x[i] *= up;
            ss = __builtin_fmaf(x[i], x[i], ss);
        }
        mean = __builtin_fmaf(group_sum(ss, lanes), p.inv_dim, p.eps * up * up);
    }
    // the hardware's root is off by an ulp: one step of Newton's method
    float r = __builtin_amdgcn_rsqf(mean);
    const float e = __builtin_fmaf(-mean * r, r, 1.0f);
    if (__builtin_fabsf(e) < 0.5f) r = __builtin_fmaf(0.5f * r, e, r);
    return r;
}

// Tokens that a wave's groups of lanes take at once where they have few heads
// (53,073 + 43,339 tokens of one head of 40 with gradient 31 us, 79 with one).
int pack_of(const NormSide &s, int lanes) {
    const int groups = 64 / lanes;
    return s.heads < groups && s.tokens >= groups ? groups / s.heads : 1;
}

// Rows of which a lane sums the weights' gradients in 32 bits before they go to a
// sum in 64, so that the error does not grow with the tokens (in 32 bits alone it was
// 10^-5 of a sum of 2^24 equal terms; the times are the same).
constexpr int kRun = 16;

// A row's loads are under way while the one before it is worked on.  With LANES
// a row fills that many lanes, known to the compiler (21,120 tokens of 8 + 8 heads
// of 64 23 us, 24 without); LANES = 0 takes any width.  PACK: a side's tokens are
// packed (the scalar work for it cost 2 to 8 % where none are).
template <typename T, int W, bool GRAD, int LANES, bool PACK>
__global__ __launch_bounds__(kThreads) void qk_norm_kernel(NormParams p, int any_lanes) {
    const int lanes = LANES ? LANES : any_lanes;
    __shared__ float2 turns[kWaves][PACK ? 64 * W : 64];
    __shared__ double sums[GRAD ? kWaves : 1][GRAD ? kMaxHeadDim : 1];
    const int lane = threadIdx.x & 63, own = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool keys = (int)blockIdx.x >= p.side[1].first_block;
    const NormSide &s = p.side[keys];
    const int groups = 64 / lanes, group = lane / lanes, unit = lane & (lanes - 1);
    const int turning = p.half / W;
    const bool used = LANES || unit < p.dim / (2 * W);
    const int dim = LANES ? LANES * 2 * W : p.dim;
    // a lane without a place of its own reads and computes another's, and writes nothing
    const int place = used ? unit : 0;
    const bool turned = place < turning;
    const int a = turned ? place * W : 2 * p.half + (place - turning) * 2 * W;
    const int b = turned ? a + p.half : a + W;
    float w[2 * W], dw[2 * W];
#pragma unroll
    for (int i = 0; i < W; ++i) {
        w[i] = s.weight ? s.weight[a + i] : 1.0f;
        w[W + i] = s.weight ? s.weight[b + i] : 1.0f;
    }
    double dws[2 * W];
    int run = 0;
    if (GRAD) {
#pragma unroll
        for (int i = 0; i < 2 * W; ++i) {
            dw[i] = 0.0f;
            dws[i] = 0.0;
        }
    }
    // items: a token, one of the shares of its heads, or `pack` tokens of few heads
    const int pack = PACK ? s.pack : 1, cut = s.shares.cut, part = s.shares.part;
    const int64_t items = (s.tokens + pack - 1) / pack * cut, step = (int64_t)s.blocks * kWaves;
    struct Spot {   // where a wave is: its groups' rows are first, first + 1, ...
        int64_t item, token;
        int first, last;
    } at, next;
    auto enter = [&](Spot &o, int64_t item) {
        o.item = item;
        o.token = cut == 1 ? item * pack : item / cut;
        o.first = cut == 1 ? 0 : (int)(item - o.token * cut) * part;
        o.last = pack == 1 ? min(o.first + part, s.heads) : (int)min((int64_t)pack, s.tokens - o.token) * s.heads;
    };
    Raw<T, W> x, y, next_x, next_y;
    const T *from_x = (const T *)s.x, *from_y = (const T *)s.dout;
    T *to = (T *)s.out;
    asm("" : "+s"(from_x), "+s"(from_y), "+s"(to));   // in registers: else they are read again for each row
    // scalar addresses of the wave's first row; this lane's is ahead of it
    const int up = pack == 1 ? 0 : min(group / s.heads, pack - 1), head = group - up * s.heads;
    const int64_t x_ahead = up * s.x_row + head * s.x_head, y_ahead = up * s.dout_row + head * s.dout_head;
    const int out_ahead = group * dim;
    auto load = [&](const Spot &o, Raw<T, W> &rx, Raw<T, W> &ry) {
        const bool there = o.first + group < o.last;   // rows that are not there repeat the first
        rx.load(from_x + o.token * s.x_row + o.first * s.x_head + (there ? x_ahead : 0), a, b);
        if (GRAD) ry.load(from_y + o.token * s.dout_row + o.first * s.dout_head + (there ? y_ahead : 0), a, b);
    };
    float c[W], sn[W];
#pragma unroll
    for (int i = 0; i < W; ++i) {
        c[i] = 1.0f;
        sn[i] = 0.0f;
    }
    // sines of an item, or of as many as the wave has lanes; divisions of numbers below 256
    const int half = max(p.half, 1), pairs = pack * half, ahead = max(1, 64 / pairs);
    const int by_pairs = (65535 + pairs) / pairs, by_half = (65535 + half) / half;
    const int turn_item = lane / half, turn_pair = lane - turn_item * half;
    int made = ahead;
    enter(at, (int64_t)((int)blockIdx.x - s.first_block) * kWaves + own);
    bool entered = true;
    if (at.item < items) load(at, x, y);
    while (at.item < items) {
        next = at;
        next.first += groups;
        const bool leaves = next.first >= next.last;
        if (leaves) enter(next, at.item + step);
        if (next.item < items) load(next, next_x, next_y);
        if (entered && p.half) {
            if (made == ahead) {
                made = 0;
                wave::sync();
                if (PACK) {
                    for (int e = lane; e < ahead * pairs; e += 64) {
                        const int later = e * by_pairs >> 16, rest = e - later * pairs;
                        const int over = rest * by_half >> 16, pair = rest - over * half;
                        const int64_t item = min(at.item + later * step, items - 1);
                        const int64_t token = cut == 1 ? min(item * pack + over, s.tokens - 1) : item / cut;
                        turns[own][e] = turn_of(p, s.positions[token], pair);
                    }
                } else {
                    const int64_t item = min(at.item + turn_item * step, items - 1);
                    if (turn_item < ahead) turns[own][lane] = turn_of(p, s.positions[cut == 1 ? item : item / cut], turn_pair);
                }
                wave::sync();
            }
            if (turned) {
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const float2 t = turns[own][made * pairs + up * half + a + i];
                    c[i] = t.x;
                    sn[i] = t.y;
                }
            }
            ++made;
        }
        const int h = at.first + group;
        const bool here = used && h < at.last;
        float v[2 * W], u[2 * W];
        x.widen(v);
        if (!used) {   // nothing to the sums
#pragma unroll
            for (int i = 0; i < 2 * W; ++i) v[i] = 0.0f;
        }
        float scaled;
        const float norm = inverse_norm<W>(p, v, lanes, scaled);
#pragma unroll
        for (int i = 0; i < 2 * W; ++i) v[i] *= norm;  // xhat
        if (!GRAD) {
            // where nothing turns, cos is 1 and sin 0
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float lo = v[i] * w[i], hi = v[W + i] * w[W + i];
                u[i] = lo * c[i] - hi * sn[i];
                u[W + i] = hi * c[i] + lo * sn[i];
            }
        } else {
            y.widen(u);
            if (!here) {
#pragma unroll
                for (int i = 0; i < 2 * W; ++i) u[i] = 0.0f;
            }
            float t = 0.0f;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float lo = u[i] * c[i] + u[W + i] * sn[i], hi = u[W + i] * c[i] - u[i] * sn[i];
                dw[i] = __builtin_fmaf(lo, v[i], dw[i]);
                dw[W + i] = __builtin_fmaf(hi, v[W + i], dw[W + i]);
                u[i] = lo * w[i];
                u[W + i] = hi * w[W + i];
                t = __builtin_fmaf(u[i], v[i], t);
                t = __builtin_fmaf(u[W + i], v[W + i], t);
            }
            t = group_sum(t, lanes) * p.inv_dim;
            const float of_x = norm * scaled;
#pragma unroll
            for (int i = 0; i < 2 * W; ++i) u[i] = of_x * __builtin_fmaf(-v[i], t, u[i]);
        }
        if (here) store<T, W>(to + (at.token * s.heads + at.first) * dim, out_ahead + a, out_ahead + b, u);
        entered = leaves;
        at = next;
        x = next_x;
        if (GRAD) y = next_y;
        if (GRAD && ++run == kRun) {
            run = 0;
#pragma unroll
            for (int i = 0; i < 2 * W; ++i) {
                dws[i] += (double)dw[i];
                dw[i] = 0.0f;
            }
        }
    }
    if (GRAD && s.dweight) {
#pragma unroll
        for (int i = 0; i < 2 * W; ++i) {
            dws[i] += (double)dw[i];
            for (int o = lanes; o < 64; o <<= 1) dws[i] += __shfl_xor(dws[i], o);
        }
        if (used && group == 0) {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                sums[own][a + i] = dws[i];
                sums[own][b + i] = dws[W + i];
            }
        }
        __syncthreads();
        for (int e = threadIdx.x; e < p.dim; e += kThreads) {
            double t = 0.0;
#pragma unroll
            for (int v = 0; v < kWaves; ++v) t += sums[v][e];
            p.part[(int64_t)blockIdx.x * p.dim + e] = (float)t;
        }
    }
}

// The weights' gradients of the blocks' parts, summed in a fixed order: a
// block takes 32 elements of a side.
__global__ __launch_bounds__(1024) void qk_norm_join_kernel(NormParams p) {
    __shared__ double sums[32][33];
    const NormSide &s = p.side[blockIdx.y];
    if (!s.dweight) return;
    const int e = blockIdx.x * 32 + (threadIdx.x & 31), row = threadIdx.x >> 5;
    double t = 0.0;
    if (e < p.dim)
#pragma unroll 8
        for (int b = row; b < s.blocks; b += 32) t += (double)p.part[(int64_t)(s.first_block + b) * p.dim + e];
    sums[row][threadIdx.x & 31] = t;
    __syncthreads();
    if (row == 0 && e < p.dim) {
        t = 0.0;
#pragma unroll
        for (int i = 0; i < 32; ++i) t += sums[i][threadIdx.x & 31];
        s.dweight[e] = (float)t;
    }
}

template <typename T, int W>
hipError_t launch(NormParams &p, bool grad, hipStream_t s) {
    int lanes = 1;
    while (lanes * 2 * W < p.dim) lanes *= 2;
    for (NormSide &side : p.side) side.pack = pack_of(side, lanes);
    const bool packed = p.side[0].pack > 1 || p.side[1].pack > 1;
    // few tokens: their heads over several waves
    int split = 1;
    if (!grad) {
        const int64_t tokens = std::max<int64_t>(1, p.side[0].tokens + p.side[1].tokens);
        const int rounds = (std::max(p.side[0].heads, p.side[1].heads) * lanes + 63) / 64;
        split = (int)std::min<int64_t>(rounds, std::max<int64_t>(1, 4096 / tokens));
    }
    for (NormSide &side : p.side) side.shares = norm_shares(side.heads, side.pack > 1 ? 1 : split);
    if (!grad) {
        int64_t all[2], first = 0;
        for (int i = 0; i < 2; ++i) {
            const int pack = p.side[i].pack;
            const int64_t items = (p.side[i].tokens + pack - 1) / pack * p.side[i].shares.cut;
            all[i] = (items + kWaves - 1) / kWaves;
        }
        // blocks go on to further tokens: about three each, of 4,096 to 8,192
        // (65,536 tokens of 16 + 4 heads 126 us with 8,192, 135 with half of
        // them, 143 with one token a wave; 21,120 of 8 + 8 heads of 64, 29, 25.5
        // and 31)
        const int64_t total = all[0] + all[1];
        const int64_t want = std::min<int64_t>(total, std::min<int64_t>(8192, std::max<int64_t>(4096, total / 3)));
        for (int i = 0; i < 2; ++i) {
            p.side[i].first_block = (int)first;
            p.side[i].blocks = (int)std::min<int64_t>(all[i], (want * all[i] + total - 1) / std::max<int64_t>(1, total));
            first += p.side[i].blocks;
        }
    }
    const int blocks = p.side[1].first_block + p.side[1].blocks;
    if (blocks == 0) {
        // no token: the weights' gradients alone are written
    } else {
        // rows of a power of two of places
        const int known = W == 4 && lanes >= 4 && lanes * 2 * W == p.dim ? lanes : 0;
        const auto run_packed = [&](auto l, auto pack) {
            if (grad)
                qk_norm_kernel<T, W, true, decltype(l)::value, decltype(pack)::value><<<blocks, kThreads, 0, s>>>(p, lanes);
            else
                qk_norm_kernel<T, W, false, decltype(l)::value, decltype(pack)::value><<<blocks, kThreads, 0, s>>>(p, lanes);
        };
        const auto run = [&](auto l) { packed ? run_packed(l, std::true_type()) : run_packed(l, std::false_type()); };
        if constexpr (W == 4) {
            if (known == 4) run(std::integral_constant<int, 4>());
            if (known == 8) run(std::integral_constant<int, 8>());
            if (known == 16) run(std::integral_constant<int, 16>());
        }
        if (!known) run(std::integral_constant<int, 0>());
    }
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && grad && (p.side[0].dweight || p.side[1].dweight)) {
        qk_norm_join_kernel<<<dim3((p.dim + 31) / 32, 2), 1024, 0, s>>>(p);
        e = hipGetLastError();
    }
    return e;
}

template <typename T>
hipError_t launch_typed(NormParams &p, bool grad, hipStream_t s) {
    if (p.half % 4 == 0) return launch<T, 4>(p, grad, s);
    if (p.half % 2 == 0) return launch<T, 2>(p, grad, s);
    return launch<T, 1>(p, grad, s);
}

}  // namespace

// A gradient's blocks, of both sides and of the queries: as many as its rows'
// bytes keep busy, at most kNormBlocks, shared by their rows.
int qk_norm_grad_blocks(int64_t rows_q, int64_t rows_k, int32_t dim, int32_t *blocks_q) {
    const double rows = (double)rows_q + (double)rows_k;
    const double want = std::min((double)kNormBlocks, std::max(2.0, rows * dim / 4096.0));
    int q = rows_q ? std::max(1, (int)(want * ((double)rows_q / rows))) : 0;
    int k = rows_k ? std::max(1, (int)(want * ((double)rows_k / rows))) : 0;
    *blocks_q = q;
    return q + k;
}

hipError_t launch_qk_norm(NormParams &p, int dtype, bool grad, hipStream_t s) {
    if (dtype == 2) return launch_typed<__bf16>(p, grad, s);
    if (dtype == 1) return launch_typed<_Float16>(p, grad, s);
    return launch_typed<float>(p, grad, s);
}

}  // namespace same
