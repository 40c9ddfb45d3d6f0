// Log probabilities of given states with entropy and the most likely
// alternatives, for gfx950.  For a row's first n logits x, with m the largest
// of them and s = sum e^(x_j - m):
//   l_j = x_j - m - log s,   H = log s - sum (x_j - m) e^(x_j - m) / s
// m and log s are kept apart: their sum in 32 bits would lose l's digits where
// m is large.  Each logit is read once and stays in registers.
//
// Alternatives are ordered by one 64-bit key: the value's bits in the order of
// their values, then the complement of the index, so that keys differ and ties
// go to the lowest index.  NaN ranks with -inf.
#include <algorithm>

#include "step.hpp"
#include "wave.hpp"

namespace same {
namespace {

using wave::Loose;

constexpr int kThreads = 256;
constexpr int64_t kMaxBlocks = 1 << 21;  // of up to 1024 threads: 2^32 and more run short, without an error
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_huge_valf();
constexpr int kCandidates = 512;

__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }
__device__ __forceinline__ float log_of(float s) { return __builtin_amdgcn_logf(s) * kLn2; }

// Bits in the order of values: both zeros alike, NaN as -inf; never 0.
__device__ __forceinline__ uint32_t ordered(float x) {
    x = x == x ? x + 0.0f : -kInf;
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    return (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
    return __builtin_bit_cast(float, (o >> 31) ? o & 0x7FFFFFFFu : ~o);
}
__device__ __forceinline__ uint64_t key_of(uint32_t o, uint32_t index) { return (uint64_t)o << 32 | (uint32_t)~index; }

// A sum of exponents and of their weighted distances, relative to max.
__device__ __forceinline__ void add_logit(float x, float max, float &sum, float &weighted) {
    const float d = x - max, e = exp_of(d);
    sum += e;
    weighted = __builtin_fmaf(e, __builtin_fmaxf(d, -200.0f), weighted);  // -inf: 0 of it; NaN is in the sum
}

// One part's sums relative to a larger maximum.
__device__ __forceinline__ void rescale(RowStats &r, float max) {
    if (r.max == max || r.max == -kInf) {  // nothing there, or nothing to change
        r.max = max;
        return;
    }
    const float d = r.max - max, e = exp_of(d);
    r.weighted = e * (r.weighted + d * r.sum);
    if (e == 0.0f && r.sum == r.sum) r.weighted = 0.0f;
    r.sum *= e;
    r.max = max;
}

// What a row's statistics say, written by one thread.
__device__ __forceinline__ void finish(const LogProbsParams &p, int64_t row, int n, const RowStats &r, float asked,
                                       int target, float log_sum) {
    const bool none = r.max == -kInf && r.sum == 0.0f;  // no state is possible
    if (p.sums) p.sums[row] = make_float2(r.max, none ? 0.0f : log_sum);
    if (p.entropy) p.entropy[row] = none ? 0.0f : log_sum - r.weighted / r.sum;
    if (p.log_probs)
        p.log_probs[row] = target < 0 ? 0.0f : none || target >= n ? -kInf : (asked - r.max) - log_sum;
}

__device__ __forceinline__ int count_of(const int32_t *counts, int64_t row, int cols) {
    if (!counts) return cols;
    const int n = counts[row];
    return n < 0 ? 0 : n < cols ? n : cols;
}

// ---------------------------------------------------------------- short rows
// Up to 64 columns: a lane takes E neighbouring logits, a group of lanes a row.

template <typename T, int E>
__global__ __launch_bounds__(kThreads) void log_probs_short_kernel(LogProbsParams p, int lanes) {
    const int lane = threadIdx.x & (lanes - 1);
    const int64_t step = (int64_t)gridDim.x * (kThreads / lanes);
    for (int64_t row = (int64_t)blockIdx.x * (kThreads / lanes) + threadIdx.x / lanes; row < p.rows; row += step) {
        const int n = count_of(p.counts, row, p.cols), first = lane * E;
        const int target = p.targets ? p.targets[row] : -1;
        const T *src = (const T *)p.x + row * p.x_row + first;
        float x[E];
        if (first + E <= p.cols) {
            const Loose<T, E> v = *(const Loose<T, E> *)src;
#pragma unroll
            for (int i = 0; i < E; ++i) x[i] = (float)v.v[i];
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) x[i] = first + i < p.cols ? (float)src[i] : -kInf;
        }
        RowStats r{-kInf, 0.0f, 0.0f, 0.0f};
        float asked = -kInf;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if (first + i >= n) x[i] = -kInf;
            r.max = __builtin_fmaxf(r.max, x[i]);
        }
        r.max = wave::reduce(r.max, lanes, wave::Max());
        const float base = r.max == -kInf ? 0.0f : r.max;
#pragma unroll
        for (int i = 0; i < E; ++i) add_logit(x[i], base, r.sum, r.weighted);
        r.sum = wave::reduce(r.sum, lanes, wave::Add());
        r.weighted = wave::reduce(r.weighted, lanes, wave::Add());
        const float log_sum = log_of(r.sum);
        // the lane that holds the target writes
        const int owner = target >= 0 && target < n ? target / E : 0;
        if (lane == owner) {
#pragma unroll
            for (int i = 0; i < E; ++i) asked = first + i == target ? x[i] : asked;
            finish(p, row, n, r, asked, target, log_sum);
        }
        uint32_t left[E];
        if (p.n_top) {
#pragma unroll
            for (int i = 0; i < E; ++i) left[i] = first + i < n ? ordered(x[i]) : 0;
        }
        for (int k = 0; k < p.n_top; ++k) {
            uint32_t best = 0;
#pragma unroll
            for (int i = 0; i < E; ++i) best = left[i] > best ? left[i] : best;
            best = wave::reduce(best, lanes, wave::Max());
            uint32_t at = 0xFFFFFFFFu;
#pragma unroll
            for (int i = E - 1; i >= 0; --i) at = left[i] == best ? (uint32_t)(first + i) : at;
            at = wave::reduce(at, lanes, wave::Min());
#pragma unroll
            for (int i = 0; i < E; ++i)
                if ((uint32_t)(first + i) == at) left[i] = 0;
            if (lane == 0) {
                p.top_ids[row * p.n_top + k] = best ? (int)at : -1;
                p.top_log_probs[row * p.n_top + k] =
                    best ? (r.max == -kInf && r.sum == 0.0f ? -kInf : (value_of(best) - r.max) - log_sum) : -kInf;
            }
        }
    }
}

// ----------------------------------------------------------------- long rows
// WAVES waves take a row, or a part of one, with VECS vectors of 16 bytes a
// lane.  Candidates for the alternatives: the n_top-th largest of the 64 lanes'
// maxima (over the row's waves) bounds the n_top-th largest logit from below,
// and about as many logits reach it as are wanted; they are collected in LDS
// and ranked by counting.  Where more than kCandidates reach it (many alike),
// the alternatives are found one after another.

template <typename T, int WAVES, int VECS, bool TOP>
struct RowShared {
    RowStats stats[WAVES];
    uint32_t largest[WAVES][64];
    uint64_t keys[TOP ? kCandidates : 1];
    uint64_t best[WAVES];
    int count;
};

template <int WAVES>
__device__ __forceinline__ void row_sync() {
    if (WAVES == 1)
        wave::sync();
    else
        __syncthreads();
}

// The largest T such that `want` lanes at least hold o >= T.
__device__ __forceinline__ uint32_t kth_largest(uint32_t o, int want) {
    uint32_t t = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t trial = t | (1u << bit);
        const int c = __builtin_popcountll(__ballot(o >= trial));
        if (c >= want) {
            t = trial;
            if (c == want) break;
        }
    }
    return t;
}

template <typename T, int WAVES, int VECS, bool TOP>
__global__ __launch_bounds__(WAVES == 1 ? kThreads : WAVES * 64) void log_probs_kernel(LogProbsParams p) {
    constexpr int N = 16 / sizeof(T), ROWS = WAVES == 1 ? kThreads / 64 : 1;
    __shared__ RowShared<T, WAVES, VECS, TOP> shared[ROWS];
    const int lane = threadIdx.x & 63, own = WAVES == 1 ? 0 : threadIdx.x >> 6;
    RowShared<T, WAVES, VECS, TOP> &sh = shared[WAVES == 1 ? threadIdx.x >> 6 : 0];
    const int64_t items = p.rows * p.parts, step = (int64_t)gridDim.x * ROWS;
    for (int64_t item = (int64_t)blockIdx.x * ROWS + (WAVES == 1 ? threadIdx.x >> 6 : 0); item < items; item += step) {
        const int64_t row = p.parts == 1 ? item : item / p.parts;
        const int part = p.parts == 1 ? 0 : (int)(item - row * p.parts);
        const int n = count_of(p.counts, row, p.cols);
        const int beg = part * p.part_cols, end = min(n, beg + p.part_cols);
        const T *src = (const T *)p.x + row * p.x_row;
        const int target = p.targets && p.parts == 1 ? p.targets[row] : -1;
        const bool writer = own == 0 && lane == 0;
        float asked = -kInf;
        if (writer && target >= 0 && target < n) asked = (float)src[target];
        Loose<T, N> v[VECS];
        const int at0 = beg + (own * 64 + lane) * N;
#pragma unroll
        for (int i = 0; i < VECS; ++i) {
            const int at = at0 + i * WAVES * 64 * N;
            if (at <= end - N) {
                v[i] = *(const Loose<T, N> *)(src + at);
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) v[i].v[e] = at + e < end ? src[at + e] : (T)-kInf;
            }
        }
        float most = -kInf;
#pragma unroll
        for (int i = 0; i < VECS; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) most = __builtin_fmaxf(most, (float)v[i].v[e]);
        RowStats r{wave::reduce(most, 64, wave::Max()), 0.0f, 0.0f, 0.0f};
        const float base = r.max == -kInf ? 0.0f : r.max;
#pragma unroll
        for (int i = 0; i < VECS; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) add_logit((float)v[i].v[e], base, r.sum, r.weighted);
        r.sum = wave::reduce(r.sum, 64, wave::Add());
        r.weighted = wave::reduce(r.weighted, 64, wave::Add());
        if (WAVES > 1 || TOP) {
            if (WAVES > 1 && lane == 0) sh.stats[own] = r;
            if (TOP) sh.largest[own][lane] = at0 < end ? ordered(most) : 0;
            if (writer) sh.count = 0;
            row_sync<WAVES>();
        }
        if (WAVES > 1) {
            float max = -kInf;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) max = __builtin_fmaxf(max, sh.stats[w].max);
            r.max = max;
            r.sum = r.weighted = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                RowStats o = sh.stats[w];
                rescale(o, max);
                r.sum += o.sum;
                r.weighted += o.weighted;
            }
        }
        const float log_sum = log_of(r.sum);
        if (writer) {
            if (p.parts == 1)
                finish(p, row, n, r, asked, target, log_sum);
            else
                p.part_stats[item] = r;
        }
        if (TOP) {
            uint32_t o = sh.largest[0][lane];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) o = max(o, sh.largest[w][lane]);
            const uint32_t bound = kth_largest(o, p.n_top);
            const float low = bound ? value_of(bound) : -kInf;
#pragma unroll
            for (int i = 0; i < VECS; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float x = (float)v[i].v[e];
                    const int at = at0 + i * WAVES * 64 * N + e;
                    if (!(x < low) && at < end) {
                        const uint32_t u = ordered(x);
                        if (u >= bound) {
                            const int slot = atomicAdd(&sh.count, 1);
                            if (slot < kCandidates) sh.keys[slot] = key_of(u, (uint32_t)at);
                        }
                    }
                }
            row_sync<WAVES>();
            const int found = sh.count;
            const bool none = r.max == -kInf && r.sum == 0.0f;
            const int64_t out = item * p.n_top;
            auto put = [&](int k, uint64_t key) {
                if (p.parts > 1) {
                    p.part_keys[out + k] = key;
                } else {
                    p.top_ids[out + k] = key ? (int)~(uint32_t)key : -1;
                    p.top_log_probs[out + k] =
                        key && !none ? (value_of((uint32_t)(key >> 32)) - r.max) - log_sum : -kInf;
                }
            };
            const int me = own * 64 + lane;
            if (found <= kCandidates) {
                for (int c = me; c < found; c += WAVES * 64) {
                    const uint64_t key = sh.keys[c];
                    int rank = 0;
                    for (int j = 0; j < found; ++j) rank += sh.keys[j] > key;
                    if (rank < p.n_top) put(rank, key);
                }
                for (int k = found + me; k < p.n_top; k += WAVES * 64) put(k, 0);
            } else {
                uint64_t last = ~0ull;
                for (int k = 0; k < p.n_top; ++k) {
                    uint64_t best = 0;
#pragma unroll
                    for (int i = 0; i < VECS; ++i)
#pragma unroll
                        for (int e = 0; e < N; ++e) {
                            const int at = at0 + i * WAVES * 64 * N + e;
                            const uint64_t key = at < end ? key_of(ordered((float)v[i].v[e]), (uint32_t)at) : 0;
                            if (key < last && key > best) best = key;
                        }
                    for (int o = 32; o; o >>= 1) {
                        const uint64_t other = __shfl_xor(best, o);
                        best = other > best ? other : best;
                    }
                    if (WAVES > 1) {
                        if (lane == 0) sh.best[own] = best;
                        __syncthreads();
#pragma unroll
                        for (int w = 0; w < WAVES; ++w) best = sh.best[w] > best ? sh.best[w] : best;
                        __syncthreads();
                    }
                    if (writer) put(k, best);
                    last = best;
                }
            }
        }
        if (WAVES > 1 || TOP) row_sync<WAVES>();  // the next item writes what this one reads
    }
}

// A long row's parts: a wave a row, a lane a part.
__global__ __launch_bounds__(kThreads) void log_probs_join_kernel(LogProbsParams p, int dtype) {
    const int lane = threadIdx.x & 63;
    const int64_t step = (int64_t)gridDim.x * (kThreads / 64);
    for (int64_t row = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6); row < p.rows; row += step) {
        const int n = count_of(p.counts, row, p.cols);
        RowStats r{-kInf, 0.0f, 0.0f, 0.0f};
        if (lane < p.parts) r = p.part_stats[row * p.parts + lane];
        const float max = wave::reduce(r.max, 64, wave::Max());
        rescale(r, max);
        r.sum = wave::reduce(r.sum, 64, wave::Add());
        r.weighted = wave::reduce(r.weighted, 64, wave::Add());
        const float log_sum = log_of(r.sum);
        if (lane == 0) {
            const int target = p.targets ? p.targets[row] : -1;
            float asked = -kInf;
            if (target >= 0 && target < n) {
                const int64_t at = row * p.x_row + target;
                asked = dtype == 0   ? ((const float *)p.x)[at]
                        : dtype == 1 ? (float)((const _Float16 *)p.x)[at]
                                     : (float)((const __bf16 *)p.x)[at];
            }
            finish(p, row, n, r, asked, target, log_sum);
        }
        const uint64_t *keys = p.part_keys + (row * p.parts + lane) * p.n_top;
        int next = 0;
        const bool none = r.max == -kInf && r.sum == 0.0f;
        for (int k = 0; k < p.n_top; ++k) {
            const uint64_t mine = lane < p.parts && next < p.n_top ? keys[next] : 0;
            uint64_t best = mine;
            for (int o = 32; o; o >>= 1) {
                const uint64_t other = __shfl_xor(best, o);
                best = other > best ? other : best;
            }
            if (mine == best) ++next;
            if (lane == 0) {
                p.top_ids[row * p.n_top + k] = best ? (int)~(uint32_t)best : -1;
                p.top_log_probs[row * p.n_top + k] =
                    best && !none ? (value_of((uint32_t)(best >> 32)) - r.max) - log_sum : -kInf;
            }
        }
    }
}

// ------------------------------------------------------------------ gradient
//   dx_j = dl (1[j = t] - p_j) - dH p_j (l_j + H),  0 from the count on.

struct RowGrad {
    float max, log_sum, entropy, dl, dh;
    int n, target;
};

__device__ __forceinline__ RowGrad row_grad(const LogProbsGradParams &p, int64_t row) {
    RowGrad g;
    const float2 s = p.sums[row];
    g.max = s.x;
    g.log_sum = s.y;
    g.n = s.x == -kInf && s.y == 0.0f ? 0 : count_of(p.counts, row, p.cols);  // no state is possible: no gradient
    g.target = p.targets ? p.targets[row] : -1;
    g.dl = p.dlog_probs && g.target >= 0 ? p.dlog_probs[row] : 0.0f;
    g.dh = p.dentropy ? p.dentropy[row] : 0.0f;
    g.entropy = p.dentropy ? p.entropy[row] : 0.0f;
    return g;
}

__device__ __forceinline__ float logit_grad(const RowGrad &g, float x, int at) {
    const float l = (x - g.max) - g.log_sum, prob = exp_of(l);
    const float v = -prob * __builtin_fmaf(g.dh, __builtin_fmaxf(l, -200.0f) + g.entropy, g.dl);
    return at < g.n ? v + (at == g.target ? g.dl : 0.0f) : 0.0f;
}

template <typename T, int E>
__device__ __forceinline__ void grad_vector(const LogProbsGradParams &p, const RowGrad &g, int64_t row, int at) {
    const T *src = (const T *)p.x + row * p.x_row + at;
    T *dst = (T *)p.dx + row * p.dx_row + at;
    if (at + E <= p.cols) {
        Loose<T, E> v = *(const Loose<T, E> *)src;
#pragma unroll
        for (int i = 0; i < E; ++i) v.v[i] = (T)logit_grad(g, (float)v.v[i], at + i);
        *(Loose<T, E> *)dst = v;
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (at + i < p.cols) dst[i] = (T)logit_grad(g, (float)src[i], at + i);
    }
}

template <typename T, int E>
__global__ __launch_bounds__(kThreads) void log_probs_grad_short_kernel(LogProbsGradParams p, int lanes) {
    const int first = (threadIdx.x & (lanes - 1)) * E;
    const int64_t step = (int64_t)gridDim.x * (kThreads / lanes);
    for (int64_t row = (int64_t)blockIdx.x * (kThreads / lanes) + threadIdx.x / lanes; row < p.rows; row += step)
        if (first < p.cols) grad_vector<T, E>(p, row_grad(p, row), row, first);
}

// A wave takes VECS vectors a lane of a row.
constexpr int kGradVecs = 4;

template <typename T>
__global__ __launch_bounds__(kThreads) void log_probs_grad_kernel(LogProbsGradParams p, int parts) {
    constexpr int N = 16 / sizeof(T);
    const int lane = threadIdx.x & 63;
    const int64_t items = p.rows * parts, step = (int64_t)gridDim.x * (kThreads / 64);
    for (int64_t item = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6); item < items; item += step) {
        const int64_t row = item / parts;
        const int beg = (int)(item - row * parts) * (64 * N * kGradVecs);
        const RowGrad g = row_grad(p, row);
#pragma unroll
        for (int i = 0; i < kGradVecs; ++i) {
            const int at = beg + (i * 64 + lane) * N;
            if (at < p.cols) grad_vector<T, N>(p, g, row, at);
        }
    }
}

// ------------------------------------------------------------------ launches

inline uint32_t blocks_for(int64_t items, int64_t per_block) {
    return (uint32_t)std::min<int64_t>(kMaxBlocks, (items + per_block - 1) / per_block);
}

inline int lanes_for(int cols, int each) {
    int lanes = 1;
    while (lanes * each < cols) lanes *= 2;
    return lanes;
}

constexpr int kShort = 64;

template <typename T, int WAVES, int VECS>
hipError_t launch_rows(const LogProbsParams &p, hipStream_t s) {
    const int64_t items = p.rows * p.parts;
    const uint32_t blocks = blocks_for(items, WAVES == 1 ? kThreads / 64 : 1);
    const int threads = WAVES == 1 ? kThreads : WAVES * 64;
    if (p.n_top)
        log_probs_kernel<T, WAVES, VECS, true><<<blocks, threads, 0, s>>>(p);
    else
        log_probs_kernel<T, WAVES, VECS, false><<<blocks, threads, 0, s>>>(p);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_typed(const LogProbsParams &p, int dtype, hipStream_t s) {
    constexpr int N = 16 / sizeof(T);
    if (p.cols <= kShort) {
        if (p.cols <= 2) {
            log_probs_short_kernel<T, 2><<<blocks_for(p.rows, kThreads), kThreads, 0, s>>>(p, 1);
        } else {
            const int lanes = lanes_for(p.cols, 4);
            log_probs_short_kernel<T, 4><<<blocks_for(p.rows, kThreads / lanes), kThreads, 0, s>>>(p, lanes);
        }
        return hipGetLastError();
    }
    const int64_t vecs = (p.part_cols + 64 * N - 1) / (64 * N);
    hipError_t e;
    if (vecs <= 1)
        e = launch_rows<T, 1, 1>(p, s);
    else if (vecs <= 4)
        e = launch_rows<T, 1, 4>(p, s);
    else if (vecs <= 16)
        e = launch_rows<T, 4, 4>(p, s);
    else if (sizeof(T) == 2 || vecs <= 64)
        e = launch_rows<T, 16, 4>(p, s);
    else
        e = launch_rows<T, 16, sizeof(T) == 2 ? 4 : 8>(p, s);
    if (e == hipSuccess && p.parts > 1) {
        log_probs_join_kernel<<<blocks_for(p.rows, kThreads / 64), kThreads, 0, s>>>(p, dtype);
        e = hipGetLastError();
    }
    return e;
}

template <typename T>
hipError_t launch_grad_typed(const LogProbsGradParams &p, hipStream_t s) {
    if (p.cols <= 2) {
        log_probs_grad_short_kernel<T, 2><<<blocks_for(p.rows, kThreads), kThreads, 0, s>>>(p, 1);
    } else if (p.cols <= kShort) {
        const int lanes = lanes_for(p.cols, 4);
        log_probs_grad_short_kernel<T, 4><<<blocks_for(p.rows, kThreads / lanes), kThreads, 0, s>>>(p, lanes);
    } else {
        const int each = 64 * (16 / (int)sizeof(T)) * kGradVecs, parts = (p.cols + each - 1) / each;
        log_probs_grad_kernel<T><<<blocks_for(p.rows * parts, kThreads / 64), kThreads, 0, s>>>(p, parts);
    }
    return hipGetLastError();
}

}  // namespace

// Rows of up to 32,768 columns are whole; longer ones have parts of that.
void log_probs_parts(int64_t rows, int64_t cols, int32_t *parts, int32_t *part_cols) {
    (void)rows;
    *parts = (int32_t)std::max<int64_t>(1, (cols + 32767) / 32768);
    *part_cols = (int32_t)((cols + *parts - 1) / *parts + 7) / 8 * 8;
}

hipError_t launch_log_probs(const LogProbsParams &p, int dtype, hipStream_t s) {
    if (dtype == 2) return launch_typed<__bf16>(p, dtype, s);
    if (dtype == 1) return launch_typed<_Float16>(p, dtype, s);
    return launch_typed<float>(p, dtype, s);
}

hipError_t launch_log_probs_grad(const LogProbsGradParams &p, int dtype, hipStream_t s) {
    if (dtype == 2) return launch_grad_typed<__bf16>(p, s);
    if (dtype == 1) return launch_grad_typed<_Float16>(p, s);
    return launch_grad_typed<float>(p, s);
}

}  // namespace same
