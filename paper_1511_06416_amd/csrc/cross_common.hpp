// Device code that the passes of cross attention share: LDS tiles, operand
// reads, staging, the counter-based keep flags, epilogues and the launch by
// type, width and geometry.
#pragma once

#include "cross.hpp"
#include "philox.hpp"

namespace same {
namespace cross {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename T>
struct Vec {
    typedef T x4 __attribute__((ext_vector_type(4)));
    typedef T x8 __attribute__((ext_vector_type(8)));
};

__device__ __forceinline__ f32x16 mfma(Vec<__bf16>::x8 a, Vec<__bf16>::x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma(Vec<_Float16>::x8 a, Vec<_Float16>::x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_huge_valf();

// LDS tiles hold rows of kPitch 16-byte chunks.  Chunk c of row r sits at
// c ^ turn(r), so that both reads are free of bank conflicts: a chunk of 16
// consecutive rows (matrix operand, 16 bytes a lane) and 64 bytes of four
// consecutive rows (transposed operand).
template <int NS>
struct Tile {
    static constexpr int kChunks = 2 * NS;
    static constexpr int kPitch = NS <= 2 ? 4 : NS <= 4 ? 8 : 16;
    static constexpr int kRowBytes = kPitch * 16;
    __device__ static __forceinline__ int turn(int r) {
        if (kPitch == 16) return ((r & 3) << 2) | ((r >> 2) & 3);
        if (kPitch == 8) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
        return (r >> 2) & 3;
    }
    __device__ static __forceinline__ int at(int r, int c) { return r * kRowBytes + ((c ^ turn(r)) << 4); }
};

// Matrix operand: chunk c of row r.
template <typename T, int NS>
__device__ __forceinline__ typename Vec<T>::x8 read_rows(const char *tile, int r, int c) {
    return *(const typename Vec<T>::x8 *)(tile + Tile<NS>::at(r, c));
}

// Transposed operand of 16 rows from row0 on (a multiple of 16) and columns
// 32 dt .. 32 dt + 31: lane l gets column 32 dt + l % 32 of rows
// row0 + 4 (l / 32) + {0..3} and the same eight rows further: the rows that
// the accumulator layout of a 32x32 product gives a lane.
template <typename T, int NS>
__device__ __forceinline__ typename Vec<T>::x8 read_columns(const char *tile, int row0, int dt, int lane) {
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const int t = lane & 15;
    const int c = 4 * dt + 2 * ((lane >> 4) & 1) + ((t & 3) >> 1);
    const int r = row0 + 4 * (lane >> 5) + (t >> 2);
    union {
        s16x4 h[2];
        typename Vec<T>::x8 v;
    } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + Tile<NS>::at(r, c) + (t & 1) * 8));
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + Tile<NS>::at(r + 8, c) + (t & 1) * 8));
    return u.v;
}

// Logical block of a launch: `chunk` consecutive ones run on one XCD (blocks
// are dealt to the eight XCDs in turn), so that tiles which read the same
// keys share an L2.
__device__ __forceinline__ int64_t logical_block(int chunk) {
    const int64_t b = blockIdx.x;
    const int64_t slot = b >> 3;
    return ((slot / chunk) * 8 + (b & 7)) * chunk + slot % chunk;
}

// A query row of a segment: its tensors' element offset.
__device__ __forceinline__ int64_t row_at(const CrossTensor &t, int64_t q0, int r, int group, int hk) {
    const int i = r / group;
    return (q0 + i) * t.row + (int64_t)(hk * group + r - i * group) * t.head;
}
__device__ __forceinline__ int64_t row_id(const CrossParams &p, int64_t q0, int r, int hk) {
    const int i = r / p.group;
    return (q0 + i) * p.heads_q + hk * p.group + r - i * p.group;
}

// Keep flags of query row `row` and the 16 keys a lane holds of the 32-key
// block kb, bit e = accumulator element e.
__device__ __forceinline__ uint32_t keep_bits(const CrossParams &p, int64_t row, int kb, int half) {
    const dev::Philox4 w = dev::philox4x32_10((uint32_t)(2 * kb + half), (uint32_t)row,
                                              (3u << 24) | (uint32_t)((uint64_t)row >> 32), p.call_id,
                                              p.seed_lo, p.seed_hi);
    uint32_t bits = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e)
        bits |= (((w.w[e >> 2] >> (8 * (e & 3))) & 255u) >= p.drop_below ? 1u : 0u) << e;
    return bits;
}

template <typename T>
__device__ __forceinline__ typename Vec<T>::x8 zero8() {
    typename Vec<T>::x8 z;
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = (T)0.0f;
    return z;
}

// ROWS rows of two tensors on their way from global memory to LDS, 16 bytes a
// lane: a thread takes the same chunk of every kStep-th row, so that one
// address per tensor and a uniform step serve all of them.
template <typename T, int NS, int ROWS, int NT>
struct Stage {
    static constexpr int kSlots = Tile<NS>::kPitch;  // lanes per row (three in four work for NS = 6)
    static constexpr int kStep = NT / kSlots;
    static constexpr int kN = (ROWS + kStep - 1) / kStep;
    static_assert(NT % kSlots == 0 && (ROWS % kStep == 0 || kN == 1), "whole rows per thread");
    typename Vec<T>::x8 a[kN], b[kN];
    __device__ static __forceinline__ int row() { return threadIdx.x / kSlots; }
    __device__ static __forceinline__ int slot() { return threadIdx.x % kSlots; }
    // lanes without a chunk of the tile, or past the width
    __device__ static __forceinline__ bool idle() { return slot() >= 2 * NS || row() >= ROWS; }

    __device__ __forceinline__ void store(char *ta, char *tb) const {
        const int r = row(), c = slot();
        if (idle()) return;
#pragma unroll
        for (int n = 0; n < kN; ++n) {
            *(typename Vec<T>::x8 *)(ta + Tile<NS>::at(r + n * kStep, c)) = a[n];
            *(typename Vec<T>::x8 *)(tb + Tile<NS>::at(r + n * kStep, c)) = b[n];
        }
    }
};

// Tiles of keys and values.  Rows past `end`, hidden keys and chunks past the
// head's width become zeros, so that nothing a hidden key holds (infinities,
// NaN) reaches a product.
template <typename T, int NS, int ROWS, int NT>
struct KeyStage : Stage<T, NS, ROWS, NT> {
    typedef Stage<T, NS, ROWS, NT> Base;
    const T *kp, *vp;
    const uint8_t *mp;
    int left;   // rows from this thread's first one to the end; 0 for idle lanes
    __device__ __forceinline__ KeyStage(const CrossParams &p, const CrossItem &it, int hk) {
        const int64_t tok = it.k0 + it.beg + Base::row();
        kp = (const T *)p.k.p + tok * p.k.row + (int64_t)hk * p.k.head + Base::slot() * 8;
        vp = (const T *)p.v.p + tok * p.v.row + (int64_t)hk * p.v.head + Base::slot() * 8;
        mp = p.key_mask ? p.key_mask + tok : nullptr;
        left = Base::slot() * 8 < p.dim && !Base::idle() ? it.end - it.beg - Base::row() : 0;
    }
    __device__ __forceinline__ void load(const CrossParams &p) {
#pragma unroll
        for (int n = 0; n < Base::kN; ++n) {
            bool in = n * Base::kStep < left;
            if (in && p.key_mask) in = mp[n * Base::kStep] != 0;
            this->a[n] = in ? *(const typename Vec<T>::x8 *)(kp + n * Base::kStep * p.k.row) : zero8<T>();
            this->b[n] = in ? *(const typename Vec<T>::x8 *)(vp + n * Base::kStep * p.v.row) : zero8<T>();
        }
        kp += ROWS * p.k.row;
        vp += ROWS * p.v.row;
        mp += ROWS;
        left -= ROWS;
    }
};

// Tiles of query rows of q and dout.
template <typename T, int NS, int ROWS, int NT>
struct QueryStage : Stage<T, NS, ROWS, NT> {
    typedef Stage<T, NS, ROWS, NT> Base;
    int64_t q0;
    int hk, r, end;
    __device__ __forceinline__ QueryStage(const CrossParams &p, const CrossItem &it, int head) {
        q0 = it.q0;
        hk = head;
        r = it.beg + Base::row();
        end = Base::slot() * 8 < p.dim && !Base::idle() ? it.end : 0;
    }
    __device__ __forceinline__ void load(const CrossParams &p) {
#pragma unroll
        for (int n = 0; n < Base::kN; ++n) {
            const int rr = r + n * Base::kStep;
            const bool in = rr < end;
            this->a[n] = in ? *(const typename Vec<T>::x8 *)((const T *)p.q.p + row_at(p.q, q0, rr, p.group, hk) +
                                                             Base::slot() * 8)
                            : zero8<T>();
            this->b[n] = in ? *(const typename Vec<T>::x8 *)((const T *)p.dout.p +
                                                             row_at(p.dout, q0, rr, p.group, hk) + Base::slot() * 8)
                            : zero8<T>();
        }
        r += ROWS;
    }
};

// Operand fragments of a lane's own row: chunks 2 s + half.
template <typename T, int NS>
__device__ __forceinline__ void load_own(typename Vec<T>::x8 (&f)[NS], const T *row, bool in, int half, int dim) {
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const int c = 2 * s + half;
        f[s] = in && c * 8 < dim ? *(const typename Vec<T>::x8 *)(row + c * 8) : zero8<T>();
    }
}

__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32, 64); }

// Accumulator element e of a lane is row 8 (e / 4) + 4 half + e % 4.
__device__ __forceinline__ int acc_row(int e, int half) { return 8 * (e >> 2) + 4 * half + (e & 3); }

template <typename T>
__device__ __forceinline__ typename Vec<T>::x8 round8(const f32x16 &a, int first) {
    typename Vec<T>::x8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (T)a[first + i];
    return r;
}

// Writes the columns of one owner that a lane holds: o[dt][e] is column
// 32 dt + acc_row(e).
template <typename T, int ND>
__device__ __forceinline__ void write_owner(T *dst, const f32x16 (&o)[ND], float gain, int half, int dim) {
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * dt + 8 * g + 4 * half;
            if (d >= dim) continue;
            typename Vec<T>::x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = (T)(o[dt][4 * g + i] * gain);
            *(typename Vec<T>::x4 *)(dst + d) = w;
        }
}

template <int ND>
__device__ __forceinline__ void write_part(float *dst, const f32x16 (&o)[ND], int half, int dim) {
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * dt + 8 * g + 4 * half;
            if (d >= dim) continue;
            f32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = o[dt][4 * g + i];
            *(f32x4 *)(dst + d) = w;
        }
}

// Adds the accumulators of the waves that share a tile of owners into those
// of the first (in a fixed order); f scales a wave's own before the sum.
template <int ND, int OW, int CW>
__device__ __forceinline__ void join_waves(f32x16 (&o)[ND], char *lds, int ow, int cw, int lane) {
    if (CW == 1) return;
    float *buf = (float *)lds;
#pragma unroll
    for (int step = 1; step < CW; ++step) {
        __syncthreads();
        if (cw == step)
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int e = 0; e < 16; ++e) buf[((ow * ND + dt) * 16 + e) * 64 + lane] = o[dt][e];
        __syncthreads();
        if (cw == 0)
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[dt][e] += buf[((ow * ND + dt) * 16 + e) * 64 + lane];
    }
}

constexpr int max_of(int a, int b) { return a > b ? a : b; }

inline uint32_t grid_of(const CrossParams &p) {
    const int64_t n = (int64_t)p.n_items * p.heads_kv, unit = 8 * (int64_t)p.chunk;
    return (uint32_t)((n + unit - 1) / unit * unit);
}

// One launch of Pass::run<T, NS, OW, CW, DROP>, then the join of its parts.
template <typename Pass, typename T, int NS>
void launch_shape(const CrossParams &p, const CrossPass &w, hipStream_t s) {
    const bool drop = p.drop_below != 0;
    if (w.own_waves == 4)
        drop ? Pass::template run<T, NS, 4, 1, true>(p, s) : Pass::template run<T, NS, 4, 1, false>(p, s);
    else if (w.cut_waves == 4)
        drop ? Pass::template run<T, NS, 1, 4, true>(p, s) : Pass::template run<T, NS, 1, 4, false>(p, s);
    else
        drop ? Pass::template run<T, NS, 1, 1, true>(p, s) : Pass::template run<T, NS, 1, 1, false>(p, s);
}

template <typename Pass, typename T>
hipError_t launch_typed(CrossParams p, const CrossPass &w, hipStream_t s) {
    if (w.n_items == 0) return hipSuccess;
    p.items = w.items;
    p.n_items = w.n_items;
    p.chunk = 4;
    if (p.dim <= 32)
        launch_shape<Pass, T, 2>(p, w, s);
    else if (p.dim <= 64)
        launch_shape<Pass, T, 4>(p, w, s);
    else if (p.dim <= 96)
        launch_shape<Pass, T, 6>(p, w, s);
    else
        launch_shape<Pass, T, 8>(p, w, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || w.n_joins == 0) return e;
    Pass::template join<T>(p, w, dim3((uint32_t)w.n_joins * p.heads_kv), s);
    return hipGetLastError();
}

template <typename Pass>
hipError_t launch_pass(const CrossParams &p, const CrossPass &w, int dtype, hipStream_t s) {
    return dtype == kCrossBf16 ? launch_typed<Pass, __bf16>(p, w, s) : launch_typed<Pass, _Float16>(p, w, s);
}

}  // namespace cross
}  // namespace same
