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
//
// Measured: 4,099 rows of 32,768 in bf16 66 us (4.1 TB/s, vector units 69 % busy
// with an exponential and three more operations an element), gradient 77 (7 TB/s
// with what the last-level cache still holds); 1.2 million rows of 8 in fp32 14 and
// 20 us; one row of 32,767 with 20 alternatives 7.7 us, the chain of one block.
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

__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

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

// Sums are formed in powers of two.  With base = max log2 e, rounded, a logit's
// place is t = x log2 e - base, one multiply-add; e = 2^t goes to the sum and
// t e to the weighted one.  The base's rounding shifts every t alike: it is
// known to the last bit from a multiply-add, belongs to the logarithm of the
// sum, and cancels from the entropy.  It is half of the base's last place: 2^-8
// up to kFar, all of fp16; beyond, it would reach whole powers of two, and from
// 2^31 on leave the exponents' range, so that distances are formed first.
constexpr float kFar = 65536.0f;

struct Place {
    float max, base;
    bool far;   // distances are formed first: t has no shift
    __device__ __forceinline__ explicit Place(float m) {
#pragma clang fp contract(off)
        max = m == -kInf ? 0.0f : m;   // nothing is there, or NaN alone
        base = max * kLog2e;
        far = __builtin_fabsf(max) > kFar;
    }
    // What t's of this place lack, the base's rounding.
    __device__ __forceinline__ float shift() const { return far ? 0.0f : __builtin_fmaf(-max, kLog2e, base); }
};

template <bool FAR>
__device__ __forceinline__ void add_logit(float x, const Place &at, float &sum, float &weighted) {
    const float t = FAR ? (x - at.max) * kLog2e : __builtin_fmaf(x, kLog2e, -at.base);
    const float e = __builtin_amdgcn_exp2f(t);
    sum += e;
    weighted = __builtin_fmaf(e, __builtin_fmaxf(t, -300.0f), weighted);  // -inf: 0 of it; NaN is in the sum
}

// One part's sums relative to a larger maximum.
__device__ __forceinline__ void rescale(RowStats &r, float max) {
#pragma clang fp contract(off)  // the bases' difference, each rounded
    if (r.max == max || r.max == -kInf) {  // nothing to change, or nothing there
        r.max = max;
        return;
    }
    const Place from(r.max), to(max);
    const float d =
        from.far || to.far ? (r.max - max) * kLog2e + (from.shift() - to.shift()) : from.base - to.base;
    const float e = __builtin_amdgcn_exp2f(d);
    r.weighted = e == 0.0f && r.sum == r.sum ? 0.0f : e * __builtin_fmaf(d, r.sum, r.weighted);
    r.sum *= e;
    r.max = max;
}

// A row's values.
struct RowValues {
    float max, log_sum, entropy;
    bool none;   // no state is possible
    // shifted: by the base's rounding
    __device__ __forceinline__ explicit RowValues(const RowStats &r, bool shifted = true) {
        const Place at(r.max);
        const float bits = __builtin_amdgcn_logf(r.sum);
        const float off = shifted ? at.shift() : 0.0f;
        none = r.max == -kInf && r.sum == 0.0f;
        max = r.max;
        log_sum = none ? 0.0f : (bits + off) * kLn2;
        entropy = none ? 0.0f : (bits - r.weighted / r.sum) * kLn2;
    }
};

// A row's outputs, written by one thread.
__device__ __forceinline__ void finish(const LogProbsParams &p, int64_t row, int n, const RowValues &r, float asked,
                                       int target) {
    if (p.sums) p.sums[row] = make_float2(r.max, r.log_sum);
    if (p.entropy) p.entropy[row] = r.entropy;
    if (p.log_probs)
        p.log_probs[row] = target < 0 ? 0.0f : r.none || target >= n ? -kInf : (asked - r.max) - r.log_sum;
}

// An alternative, key 0 where there is none.
__device__ __forceinline__ void put_top(const LogProbsParams &p, int64_t at, uint64_t key, const RowValues &r) {
    p.top_ids[at] = key ? (int)~(uint32_t)key : -1;
    p.top_log_probs[at] = key && !r.none ? (value_of((uint32_t)(key >> 32)) - r.max) - r.log_sum : -kInf;
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
        RowStats r{-kInf, 0.0f, 0.0f};
        float asked = -kInf;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if (first + i >= n) x[i] = -kInf;
            r.max = __builtin_fmaxf(r.max, x[i]);
        }
        r.max = wave::reduce(r.max, lanes, wave::Max());
        const Place at(r.max);
#pragma unroll
        for (int i = 0; i < E; ++i) add_logit<true>(x[i], at, r.sum, r.weighted);
        r.sum = wave::reduce(r.sum, lanes, wave::Add());
        r.weighted = wave::reduce(r.weighted, lanes, wave::Add());
        const RowValues values(r, false);
        // the lane that holds the target writes
        const int owner = target >= 0 && target < n ? target / E : 0;
        if (lane == owner) {
#pragma unroll
            for (int i = 0; i < E; ++i) asked = first + i == target ? x[i] : asked;
            finish(p, row, n, values, asked, target);
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
            if (lane == 0) put_top(p, row * p.n_top + k, best ? key_of(best, at) : 0, values);
        }
    }
}

// ----------------------------------------------------------------- long rows
// WAVES waves take a row, or a part of one, with VECS vectors of 16 bytes a
// lane.  Candidates for the alternatives: the n_top-th largest of the 64 lanes'
// maxima (over the row's waves) bounds the n_top-th largest logit from below,
// and about as many logits reach it as are wanted; they are collected in LDS
// and ranked by counting.  Where more than kept reach it (many alike),
// the alternatives are found one after another.

template <int WAVES, bool TOP>
struct RowShared {
    static constexpr int kKept = WAVES == 1 ? 512 : WAVES == 4 ? 256 : 128;   // candidates of a wave
    RowStats stats[WAVES];
    uint32_t largest[TOP ? WAVES : 1][64];
    uint64_t keys[TOP ? WAVES : 1][TOP ? kKept : 1];
    int count[WAVES];
    uint64_t best[WAVES];
    RowStats all;
    uint32_t bound;
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

// Keeps a vector as it was read: the compiler would hold its elements widened
// to fp32, twice the registers and half the waves.
template <typename V>
__device__ __forceinline__ void keep_packed(V &v) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    u32x4 w = __builtin_bit_cast(u32x4, v);
    asm volatile("" : "+v"(w));
    v = __builtin_bit_cast(V, w);
}

// N neighbouring logits of a row from `at` on, -inf from `end` on, for rows of N
// columns at least: behind the row's last vector that one is read (vector_at),
// and moved down (settle).  Reads come first, all of them: a branch between
// would wait for each.
template <typename T, int N>
__device__ __forceinline__ Loose<T, N> vector_at(const T *row, int at, int cols) {
    return *(const Loose<T, N> *)(row + min(at, cols - N));
}
template <typename T, int N>
__device__ __forceinline__ void settle(Loose<T, N> &v, int at, int end, int cols) {
    if (at <= end - N) return;
    struct Pair {
        uint64_t lo, hi;
    };
    Pair w = __builtin_bit_cast(Pair, v);
    int bits = min(at - min(at, cols - N), N) * (int)sizeof(T) * 8;
    if (bits >= 64) {
        w.lo = w.hi;
        w.hi = 0;
        bits -= 64;
    }
    if (bits > 0) {
        w.lo = bits < 64 ? w.lo >> bits | w.hi << (64 - bits) : w.hi;
        w.hi = bits < 64 ? w.hi >> bits : 0;
    }
    v = __builtin_bit_cast(Loose<T, N>, w);
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (at + e >= end) v.v[e] = (T)-kInf;
}

// Sums of a row's parts, a lane each: merged relative to the largest.
__device__ __forceinline__ RowStats merge(RowStats r, int lanes) {
    rescale(r, wave::reduce(r.max, lanes, wave::Max()));
    r.sum = wave::reduce(r.sum, lanes, wave::Add());
    r.weighted = wave::reduce(r.weighted, lanes, wave::Add());
    return r;
}

__device__ __forceinline__ uint64_t largest_key(uint64_t k) {
    for (int o = 32; o; o >>= 1) {
        const uint64_t other = __shfl_xor(k, o);
        k = other > k ? other : k;
    }
    return k;
}

template <typename T, int WAVES, int VECS, bool TOP>
__global__ __launch_bounds__(WAVES == 1 ? kThreads : WAVES * 64) void log_probs_kernel(LogProbsParams p) {
    constexpr int N = 16 / sizeof(T), ROWS = WAVES == 1 ? kThreads / 64 : 1;
    __shared__ RowShared<WAVES, TOP> shared[ROWS];
    const int lane = threadIdx.x & 63, wave_id = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int own = WAVES == 1 ? 0 : wave_id, which = WAVES == 1 ? wave_id : 0;
    RowShared<WAVES, TOP> &sh = shared[which];
    const int64_t items = p.rows * p.parts, step = (int64_t)gridDim.x * ROWS;
    for (int64_t item = (int64_t)blockIdx.x * ROWS + which; item < items; item += step) {
        const int64_t row = p.parts == 1 ? item : item / p.parts;
        const int part = p.parts == 1 ? 0 : (int)(item - row * p.parts);
        const int n = count_of(p.counts, row, p.cols);
        const int beg = part * p.part_cols, end = min(n, beg + p.part_cols);
        const T *src = (const T *)p.x + row * p.x_row;
        const int target = p.targets && p.parts == 1 ? p.targets[row] : -1;
        Loose<T, N> v[VECS];
        const int limit = max(end, N);   // nothing behind the states is read
        const int at0 = beg + (own * 64 + lane) * N;
#pragma unroll
        for (int i = 0; i < VECS; ++i) v[i] = vector_at<T, N>(src, at0 + i * WAVES * 64 * N, limit);
#pragma unroll
        for (int i = 0; i < VECS; ++i) settle<T, N>(v[i], at0 + i * WAVES * 64 * N, end, limit);
        float asked = -kInf;
        if (own == 0 && lane == 0 && target >= 0 && target < n) asked = (float)src[target];
        float most = -kInf;
#pragma unroll
        for (int i = 0; i < VECS; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) most = __builtin_fmaxf(most, (float)v[i].v[e]);
        RowStats r{wave::reduce(most, 64, wave::Max()), 0.0f, 0.0f};
        if (TOP) sh.largest[own][lane] = at0 < end ? ordered(most) : 0;
        const Place place(r.max);
        if (place.far) {
#pragma unroll
            for (int i = 0; i < VECS; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) add_logit<true>((float)v[i].v[e], place, r.sum, r.weighted);
        } else {
#pragma unroll
            for (int i = 0; i < VECS; ++i) {
                if (sizeof(T) == 2) keep_packed(v[i]);
#pragma unroll
                for (int e = 0; e < N; ++e) add_logit<false>((float)v[i].v[e], place, r.sum, r.weighted);
            }
        }
        r.sum = wave::reduce(r.sum, 64, wave::Add());
        r.weighted = wave::reduce(r.weighted, 64, wave::Add());
        if (WAVES > 1 && lane == 0) sh.stats[own] = r;
        if (WAVES > 1 || TOP) row_sync<WAVES>();
        if (own == 0) {
            if (WAVES > 1) r = merge(sh.stats[lane & (WAVES - 1)], WAVES);
            if (lane == 0) {
                if (p.parts == 1)
                    finish(p, row, n, RowValues(r), asked, target);
                else
                    p.part_stats[item] = r;
            }
            if (TOP) {
                uint32_t o = sh.largest[0][lane];
#pragma unroll
                for (int w = 1; w < WAVES; ++w) o = max(o, sh.largest[w][lane]);
                const uint32_t bound = kth_largest(o, p.n_top);
                if (lane == 0) {
                    sh.bound = bound;
                    sh.all = r;
                }
            }
        }
        if (TOP) {
            row_sync<WAVES>();
            const uint32_t bound = sh.bound;
            const float low = bound ? value_of(bound) : -kInf;
            int mine = 0;
            if (__ballot(!(most < low))) {
#pragma unroll
                for (int i = 0; i < VECS; ++i) {
                    if (sizeof(T) == 2) keep_packed(v[i]);
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const float x = (float)v[i].v[e];
                        if (__ballot(!(x < low))) {
                            const int at = at0 + i * WAVES * 64 * N + e;
                            const uint32_t u = ordered(x);
                            const bool in = u >= bound && at < end;
                            const uint64_t who = __ballot(in);
                            const int slot = mine + __builtin_amdgcn_mbcnt_hi(
                                                        (uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
                            if (in && slot < sh.kKept) sh.keys[own][slot] = key_of(u, (uint32_t)at);
                            mine += __builtin_popcountll(who);
                        }
                    }
                }
            }
            if (lane == 0) sh.count[own] = mine;
            row_sync<WAVES>();
            int found = 0;
            bool kept = true;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                found += sh.count[w];
                kept = kept && sh.count[w] <= sh.kKept;
            }
            const RowValues all(sh.all);
            const int64_t out = item * p.n_top;
            auto put = [&](int k, uint64_t key) {
                if (p.parts > 1)
                    p.part_keys[out + k] = key;
                else
                    put_top(p, out + k, key, all);
            };
            // candidate c of the waves' lists, one after another
            auto candidate = [&](int c) {
                uint64_t key = 0;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    const int n_w = sh.count[w];
                    if (c >= 0 && c < n_w) key = sh.keys[w][c];
                    c -= n_w;
                }
                return key;
            };
            if (kept) {
                // a wave takes 64 candidates; the others pass by in registers
                for (int c0 = own * 64; c0 < found; c0 += WAVES * 64) {
                    const uint64_t key = candidate(c0 + lane);
                    int rank = 0;
                    for (int j0 = 0; j0 < found; j0 += 64) {
                        const uint64_t others = j0 == c0 ? key : candidate(j0 + lane);
                        const int n_others = min(64, found - j0);
                        for (int j = 0; j < n_others; ++j) {
                            const uint64_t other =
                                (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(others >> 32), j) << 32 |
                                (uint32_t)__builtin_amdgcn_readlane((int)others, j);
                            rank += other > key;
                        }
                    }
                    if (key && rank < p.n_top) put(rank, key);
                }
                for (int k = found + own * 64 + lane; k < p.n_top; k += WAVES * 64) put(k, 0);
            } else {
                uint64_t last = ~0ull;
                for (int k = 0; k < p.n_top; ++k) {
                    uint64_t best = 0;
                    // read again, a logit at a time: it happens seldom, and registers are short
#pragma unroll 1
                    for (int i = 0; i < VECS; ++i)
#pragma unroll 1
                        for (int e = 0; e < N; ++e) {
                            const int at = at0 + i * WAVES * 64 * N + e;
                            const uint64_t key = at < end ? key_of(ordered((float)src[at]), (uint32_t)at) : 0;
                            if (key < last && key > best) best = key;
                        }
                    best = largest_key(best);
                    if (WAVES > 1) {
                        if (lane == 0) sh.best[own] = best;
                        __syncthreads();
#pragma unroll
                        for (int w = 0; w < WAVES; ++w) best = sh.best[w] > best ? sh.best[w] : best;
                        __syncthreads();
                    }
                    if (own == 0 && lane == 0) put(k, best);
                    last = best;
                }
            }
        }
        if (WAVES > 1 || TOP) row_sync<WAVES>();  // the next item writes what this one reads
    }
}

// A long row's parts: a block a row, a lane a part.  The parts' alternatives are
// in falling order: with t of each as many as are wanted, the smallest of the
// t-th ones bounds the wanted ones from below; what reaches it is ranked by
// counting.
__global__ __launch_bounds__(kThreads) void log_probs_join_kernel(LogProbsParams p, int dtype) {
    __shared__ uint64_t keys[kMaxRowParts * kMaxTop], nth[kMaxRowParts];
    __shared__ int found;
    const int lane = threadIdx.x & 63, k = p.n_top, all = p.parts * k, t = (k + p.parts - 1) / p.parts;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const int n = count_of(p.counts, row, p.cols);
        const uint64_t *src = p.part_keys + row * all;
        RowStats r{-kInf, 0.0f, 0.0f};
        if (lane < p.parts) r = p.part_stats[row * p.parts + lane];
        if (k && threadIdx.x < p.parts) nth[threadIdx.x] = src[threadIdx.x * k + t - 1];
        if (threadIdx.x == 0) found = 0;
        const RowValues values(merge(r, 64));
        if (threadIdx.x == 0) {
            const int target = p.targets ? p.targets[row] : -1;
            float asked = -kInf;
            if (target >= 0 && target < n) {
                const int64_t at = row * p.x_row + target;
                asked = dtype == 0   ? ((const float *)p.x)[at]
                        : dtype == 1 ? (float)((const _Float16 *)p.x)[at]
                                     : (float)((const __bf16 *)p.x)[at];
            }
            finish(p, row, n, values, asked, target);
        }
        if (k) {
            __syncthreads();
            uint64_t bound = lane < p.parts ? nth[lane] : ~0ull;
            for (int o = 32; o; o >>= 1) {
                const uint64_t other = __shfl_xor(bound, o);
                bound = other < bound ? other : bound;
            }
            for (int c = threadIdx.x; c < all; c += kThreads) {
                const uint64_t key = src[c];
                if (key && key >= bound) keys[atomicAdd(&found, 1)] = key;
            }
            __syncthreads();
            for (int c = threadIdx.x; c < found; c += kThreads) {
                const uint64_t key = keys[c];
                int rank = 0;
#pragma unroll 8
                for (int j = 0; j < found; ++j) rank += keys[j] > key;
                if (rank < k) put_top(p, row * k + rank, key, values);
            }
            // fewer than wanted: then all of them were found
            for (int c = found + threadIdx.x; c < k; c += kThreads) put_top(p, row * k + c, 0, values);
            __syncthreads();
        }
    }
}

// ------------------------------------------------------------------ gradient
//   dx_j = dl (1[j = t] - p_j) - dH p_j (l_j + H),  0 from the count on.

struct RowGrad {
    float max, log_sum, slope, rest, dl;   // -(dl + dH H), -dH
    int n, target;
};

__device__ __forceinline__ RowGrad row_grad(const LogProbsGradParams &p, int64_t row) {
    RowGrad g;
    // all loads first: none waits for another
    const float2 s = p.sums[row];
    const int n = count_of(p.counts, row, p.cols), target = p.targets ? p.targets[row] : -1;
    const float dl = p.dlog_probs ? p.dlog_probs[row] : 0.0f, dh = p.dentropy ? p.dentropy[row] : 0.0f;
    const float entropy = p.dentropy ? p.entropy[row] : 0.0f;
    g.max = s.x;
    g.log_sum = s.y;
    g.n = s.x == -kInf && s.y == 0.0f ? 0 : n;  // no state is possible: no gradient
    g.target = target;
    g.dl = target >= 0 ? dl : 0.0f;
    g.slope = -dh;
    g.rest = p.dentropy ? -__builtin_fmaf(dh, entropy, g.dl) : -g.dl;
    return g;
}

__device__ __forceinline__ float logit_grad(const RowGrad &g, float x) {
    const float l = (x - g.max) - g.log_sum;
    return exp_of(l) * __builtin_fmaf(g.slope, __builtin_fmaxf(l, -200.0f), g.rest);
}

template <typename T, int E>
__device__ __forceinline__ Loose<T, E> vector_grad(const RowGrad &g, Loose<T, E> v, int at) {
    if (at + E <= g.n && (uint32_t)(g.target - at) >= (uint32_t)E) {
#pragma unroll
        for (int i = 0; i < E; ++i) v.v[i] = (T)logit_grad(g, (float)v.v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float d = logit_grad(g, (float)v.v[i]) + (at + i == g.target ? g.dl : 0.0f);
            v.v[i] = (T)(at + i < g.n ? d : 0.0f);
        }
    }
    return v;
}

// The last logits of a row, fewer than a vector.
template <typename T>
__device__ __forceinline__ void grad_rest(const RowGrad &g, const T *src, T *dst, int at, int cols) {
    for (; at < cols; ++at) {
        const float d = logit_grad(g, (float)src[at]) + (at == g.target ? g.dl : 0.0f);
        dst[at] = (T)(at < g.n ? d : 0.0f);
    }
}

template <typename T, int E>
__global__ __launch_bounds__(kThreads) void log_probs_grad_short_kernel(LogProbsGradParams p, int lanes) {
    const int at = (threadIdx.x & (lanes - 1)) * E;
    const int64_t step = (int64_t)gridDim.x * (kThreads / lanes);
    for (int64_t row = (int64_t)blockIdx.x * (kThreads / lanes) + threadIdx.x / lanes; row < p.rows; row += step) {
        const T *src = (const T *)p.x + row * p.x_row;
        T *dst = (T *)p.dx + row * p.dx_row;
        if (at + E <= p.cols) {
            const Loose<T, E> v = *(const Loose<T, E> *)(src + at);
            *(Loose<T, E> *)(dst + at) = vector_grad<T, E>(row_grad(p, row), v, at);
        } else if (at < p.cols) {
            grad_rest<T>(row_grad(p, row), src, dst, at, p.cols);
        }
    }
}

// A wave takes kGradVecs vectors a lane of a row, one after another: 4,099 x
// 32,768 bf16 77 us; with all four loads before the first store 95, with one vector
// 130 (81 then).
constexpr int kGradVecs = 4;

template <typename T>
__global__ __launch_bounds__(kThreads) void log_probs_grad_kernel(LogProbsGradParams p, int parts) {
    constexpr int N = 16 / sizeof(T);
    const int lane = threadIdx.x & 63;
    const int64_t items = p.rows * parts, step = (int64_t)gridDim.x * (kThreads / 64);
    for (int64_t item = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6); item < items; item += step) {
        const int64_t row = item / parts;
        const int at0 = (int)(item - row * parts) * (64 * N * kGradVecs) + lane * N;
        const T *src = (const T *)p.x + row * p.x_row;
        T *dst = (T *)p.dx + row * p.dx_row;
        const RowGrad g = row_grad(p, row);
#pragma unroll
        for (int i = 0; i < kGradVecs; ++i) {
            const int at = at0 + i * 64 * N;
            if (at + N <= p.cols) {
                const Loose<T, N> v = *(const Loose<T, N> *)(src + at);
                *(Loose<T, N> *)(dst + at) = vector_grad<T, N>(g, v, at);
            } else if (at < p.cols) {
                grad_rest<T>(g, src, dst, at, p.cols);
            }
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
        } else if (p.cols % 8 == 0) {
            const int lanes = lanes_for(p.cols, 8);
            log_probs_short_kernel<T, 8><<<blocks_for(p.rows, kThreads / lanes), kThreads, 0, s>>>(p, lanes);
        } else {
            const int lanes = lanes_for(p.cols, 4);
            log_probs_short_kernel<T, 4><<<blocks_for(p.rows, kThreads / lanes), kThreads, 0, s>>>(p, lanes);
        }
        return hipGetLastError();
    }
    const int64_t vecs = (p.part_cols + 64 * N - 1) / (64 * N);
    hipError_t e;
    // Few waves a row, so that other rows' loads run beside its chain, and vectors
    // that fit: 4,095 rows of 15,406 fp16 with 20 alternatives 42 us by four waves of
    // eight, 128 by 16 of four; of 30,000 80 by eight of eight, 128 by 16 of four.
    // A lone row, or sums alone, take more waves (32,767 columns 7.7 us for 8.1).
    if (vecs <= 1)
        e = launch_rows<T, 1, 1>(p, s);
    else if (vecs <= 2)
        e = launch_rows<T, 1, 2>(p, s);
    else if (vecs <= 4)
        e = launch_rows<T, 1, 4>(p, s);
    else if (vecs <= 8)
        e = launch_rows<T, 4, 2>(p, s);
    else if (vecs <= 12)
        e = launch_rows<T, 4, 3>(p, s);
    else if (vecs <= 16)
        e = launch_rows<T, 4, 4>(p, s);
    else if (vecs <= 24)
        e = launch_rows<T, 4, 6>(p, s);
    else if (vecs <= 32)
        e = launch_rows<T, 4, 8>(p, s);
    else if (vecs <= 64 && (p.rows <= 256 || (sizeof(T) == 2 && !p.n_top)))
        e = launch_rows<T, 16, 4>(p, s);
    else if (vecs <= 48)
        e = launch_rows<T, 8, 6>(p, s);
    else if (sizeof(T) == 2 || vecs <= 64)
        e = launch_rows<T, 8, 8>(p, s);
    else
        e = launch_rows<T, 16, sizeof(T) == 2 ? 4 : 8>(p, s);
    if (e == hipSuccess && p.parts > 1) {
        log_probs_join_kernel<<<blocks_for(p.rows, 1), kThreads, 0, s>>>(p, dtype);
        e = hipGetLastError();
    }
    return e;
}

template <typename T>
hipError_t launch_grad_typed(const LogProbsGradParams &p, hipStream_t s) {
    if (p.cols <= 2) {
        log_probs_grad_short_kernel<T, 2><<<blocks_for(p.rows, kThreads), kThreads, 0, s>>>(p, 1);
    } else if (p.cols <= kShort && p.cols % 8 == 0) {
        const int lanes = lanes_for(p.cols, 8);
        log_probs_grad_short_kernel<T, 8><<<blocks_for(p.rows, kThreads / lanes), kThreads, 0, s>>>(p, lanes);
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

// Rows of up to 32,768 columns are whole; longer ones have parts of a quarter
// of that, 64 at most.
void log_probs_parts(int64_t rows, int64_t cols, int32_t *parts, int32_t *part_cols) {
    (void)rows;
    const int64_t part = std::max<int64_t>(8192, (cols + kMaxRowParts - 1) / kMaxRowParts);
    *part_cols = (int32_t)(cols <= 32768 ? std::max<int64_t>(cols, 1) : (part + 7) / 8 * 8);
    *parts = (int32_t)std::max<int64_t>(1, (cols + *part_cols - 1) / *part_cols);
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
