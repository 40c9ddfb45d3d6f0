// Dropout with the residual sum, for gfx950: y = residual + x * keep * gain.
// The mask is never stored: element e of the matrix (row * cols + column)
// takes 16 bits, number e % 8 of the Philox block at counter
// {e / 8, high word, 4 << 24, call}, so any later pass makes it again.
// Memory bounds it: 65,536 x 1,024 bf16 with a residual 68 us (5.9 TB/s, 402
// MB), 20,003 x 1,000 fp32 in rows of 1,024 31 us (5.2 TB/s); a copy of 1 GiB
// runs at 5.1.  The generator hides behind that: with two blocks for eight
// elements instead of one the times are the same.
#include <algorithm>

#include "cross.hpp"
#include "philox.hpp"

namespace same {
namespace {

constexpr int kThreads = 256;
// Groups of one launch: the device takes fewer than 2^32 threads and runs the
// rest of a larger grid without an error, short.
constexpr int64_t kLaunchGroups = (int64_t)1 << 31;
// Outputs larger than the L2s together are stored past them: 62 against 68 us
// for two passes over the fp32 matrix above.  (Two groups a thread instead of
// one: 69 and 74 us.)
constexpr int64_t kPastL2 = 32 << 20;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename T>
struct alignas(16) Group {
    T v[8];
};

__device__ __forceinline__ dev::Philox4 group_bits(const DropoutParams &p, int64_t g) {
    return dev::philox4x32_10((uint32_t)g, (uint32_t)((uint64_t)g >> 32), 4u << 24, p.call_id, p.seed_lo, p.seed_hi);
}

__device__ __forceinline__ float dropped(const DropoutParams &p, const dev::Philox4 &w, int e, float x, float base) {
    const uint32_t h = (w.w[e >> 1] >> (16 * (e & 1))) & 0xFFFFu;
    return h >= p.drop_below ? __builtin_fmaf(x, p.keep_gain, base) : base;
}

template <typename T, bool PAST>
__device__ __forceinline__ void store(T *dst, const Group<T> &g) {
    if (!PAST) {
        *(Group<T> *)dst = g;
        return;
    }
    union {
        Group<T> g;
        u32x4 w[sizeof(Group<T>) / 16];
    } u;
    u.g = g;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(Group<T>) / 16); ++i) __builtin_nontemporal_store(u.w[i], (u32x4 *)dst + i);
}

// Groups of eight that lie whole in a row (or in a contiguous matrix), one a
// thread, 16-byte accesses; per_row groups a row, the last n % 8 elements of a
// contiguous matrix by the first thread.  The launch begins at group `first`.
template <typename T, bool RES, bool DROP, bool PAST>
__global__ __launch_bounds__(kThreads) void dropout_kernel(DropoutParams p, int64_t first, int64_t n_groups,
                                                           int64_t per_row, int tail) {
    const int64_t g = first + (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (g < n_groups) {
        const int64_t row = per_row == n_groups          ? 0
                            : n_groups <= 0xFFFFFFFFll   ? (uint32_t)g / (uint32_t)per_row
                                                         : g / per_row;
        const int64_t off = (g - row * per_row) * 8;
        const Group<T> x = *(const Group<T> *)((const T *)p.x + row * p.x_row + off);
        Group<T> r, y;
        if (RES) r = *(const Group<T> *)((const T *)p.residual + row * p.r_row + off);
        dev::Philox4 w;
        if (DROP) w = group_bits(p, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float base = RES ? (float)r.v[e] : 0.0f;
            y.v[e] = (T)(DROP ? dropped(p, w, e, (float)x.v[e], base) : (float)x.v[e] + base);
        }
        store<T, PAST>((T *)p.y + row * p.y_row + off, y);
    }
    if (tail && g == 0) {
        dev::Philox4 w;
        if (DROP) w = group_bits(p, n_groups);
        for (int e = 0; e < tail; ++e) {
            const int64_t at = n_groups * 8 + e;
            const float v = (float)((const T *)p.x)[at], base = RES ? (float)((const T *)p.residual)[at] : 0.0f;
            ((T *)p.y)[at] = (T)(DROP ? dropped(p, w, e, v, base) : v + base);
        }
    }
}

// Any strides and alignment: a thread takes a group of eight, element by
// element.  65,536 x 330 bf16 in rows of 344 with a residual 58 us, where 336
// of 344 take 21 by 16 bytes: eight loads and stores a thread, 16 bytes apart
// between lanes, are what it waits for.
template <typename T, bool RES, bool DROP>
__global__ __launch_bounds__(kThreads) void dropout_any_kernel(DropoutParams p, int64_t first, int64_t n) {
    const int64_t g = first + (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (g * 8 >= n) return;
    dev::Philox4 w;
    if (DROP) w = group_bits(p, g);
    int64_t row = g * 8 / p.cols, col = g * 8 - row * p.cols;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (g * 8 + e < n) {
            const float v = (float)((const T *)p.x)[row * p.x_row + col];
            const float base = RES ? (float)((const T *)p.residual)[row * p.r_row + col] : 0.0f;
            ((T *)p.y)[row * p.y_row + col] = (T)(DROP ? dropped(p, w, e, v, base) : v + base);
            if (++col == p.cols) {
                col = 0;
                ++row;
            }
        }
    }
}

template <typename T, bool RES, bool DROP>
hipError_t launch(const DropoutParams &p, hipStream_t s) {
    const int64_t n = p.rows * p.cols;
    const bool whole = p.x_row == p.cols && p.y_row == p.cols && (!RES || p.r_row == p.cols);
    const uintptr_t mix = (uintptr_t)p.x | (uintptr_t)p.y | (RES ? (uintptr_t)p.residual : 0);
    const int64_t steps = p.x_row | p.y_row | (RES ? p.r_row : 0) | p.cols;
    const bool wide = mix % 16 == 0 && (whole || steps % 8 == 0);
    const int64_t groups = wide ? n / 8 : (n + 7) / 8, per_row = whole ? groups : p.cols / 8;
    const int tail = wide && whole ? (int)(n % 8) : 0;
    for (int64_t first = 0; first < groups || first == 0; first += kLaunchGroups) {
        const int64_t count = std::max<int64_t>(1, std::min(groups - first, kLaunchGroups));  // 1: a tail alone
        const dim3 grid((uint32_t)((count + kThreads - 1) / kThreads));
        if (!wide)
            dropout_any_kernel<T, RES, DROP><<<grid, kThreads, 0, s>>>(p, first, n);
        else if (n * (int64_t)sizeof(T) > kPastL2)
            dropout_kernel<T, RES, DROP, true><<<grid, kThreads, 0, s>>>(p, first, groups, per_row, tail);
        else
            dropout_kernel<T, RES, DROP, false><<<grid, kThreads, 0, s>>>(p, first, groups, per_row, tail);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
hipError_t launch_typed(const DropoutParams &p, hipStream_t s) {
    if (p.drop_below)
        return p.residual ? launch<T, true, true>(p, s) : launch<T, false, true>(p, s);
    return p.residual ? launch<T, true, false>(p, s) : launch<T, false, false>(p, s);
}

}  // namespace

hipError_t launch_dropout(const DropoutParams &p, int dtype, hipStream_t s) {
    if (dtype == kCrossBf16) return launch_typed<__bf16>(p, s);
    if (dtype == kCrossF16) return launch_typed<_Float16>(p, s);
    return launch_typed<float>(p, s);
}

}  // namespace same
