// Device code that the passes of cross attention share: LDS tiles, operand
// reads, staging, the counter-based keep flags, epilogues and the launch by
// type, width and geometry.
#pragma once

#include <algorithm>

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

// Powers of two that probabilities carry while they are rounded, and their
// inverse: fp16's normal numbers end at 2^-14, where a key that hardly counts,
// or each of 2^14 alike, would be rounded to a fixed step instead of its own
// digits.  A normalised one (at most 1) takes kUp and has normal numbers down
// to 2^-28.  dS has no bound of its own, takes none, and follows dout.
template <typename T>
constexpr int kUpBits = __is_same(T, _Float16) ? 14 : 0;
template <typename T>
constexpr float kUp = (float)(1 << kUpBits<T>);
template <typename T>
constexpr float kDown = 1.0f / kUp<T>;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_huge_valf();

// Rows of a head's width in LDS, 16-byte chunks, so that a read meets no bank
// twice.  Two reads occur: "rows", a chunk of 16 consecutive rows (matrix
// operand, 16 bytes a lane), and "columns", 64 bytes of each of four
// consecutive rows (transposed operand, 8 bytes a lane).  A tile that is read
// in one way only is padded (addresses are one register and constants); one
// that is read in both has its chunks turned by the row number instead.
constexpr int lanes_per_row(int ns) { return ns <= 2 ? 4 : ns <= 4 ? 8 : 16; }

template <int NS>
struct RowTile {
    static constexpr int kRowBytes = 32 * NS + 16;
    __device__ static __forceinline__ int at(int r, int c) { return r * kRowBytes + c * 16; }
};
template <int NS>
struct ColumnTile {
    // four consecutive rows 64 bytes apart modulo 256
    static constexpr int kRowBytes = NS == 4 || NS == 8 ? 32 * NS + 64 : 32 * NS;
    __device__ static __forceinline__ int at(int r, int c) { return r * kRowBytes + c * 16; }
};
template <int NS>
struct BothTile {
    static constexpr int kRowBytes = lanes_per_row(NS) * 16;
    __device__ static __forceinline__ int turn(int r) {
        if (NS > 4) return ((r & 3) << 2) | ((r >> 2) & 3);
        if (NS > 2) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
        return (r >> 2) & 3;
    }
    __device__ static __forceinline__ int at(int r, int c) { return r * kRowBytes + ((c ^ turn(r)) << 4); }
};

// Reads of BothTile tiles by one lane.  A turned chunk number is a fixed one
// exclusive-or a constant of the read, so a lane needs two addresses; renew()
// keeps the compiler from holding every combination in a register.
template <typename T, int NS>
struct BothReader {
    typedef BothTile<NS> Tile;
    typedef __attribute__((address_space(3))) const typename Vec<T>::x8 lds_x8;
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    uint32_t rows, columns;
    __device__ __forceinline__ BothReader(const char *lds, int lane) {
        const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)lds;
        const int t = lane & 15, r = 4 * (lane >> 5) + (t >> 2);
        rows = base + (uint32_t)Tile::at(lane & 31, lane >> 5);
        columns = base + (uint32_t)Tile::at(r, 2 * ((lane >> 4) & 1) + ((t & 3) >> 1)) + (t & 1) * 8;
    }
    __device__ __forceinline__ void renew() {
        asm volatile("" : "+v"(rows), "+v"(columns));
    }
    // to another buffer, whole tiles away
    __device__ __forceinline__ void move(int bytes) {
        rows += bytes;
        columns += bytes;
    }
    // chunk 2 t + lane / 32 of row lane % 32, `at` bytes (whole tiles) on
    __device__ __forceinline__ typename Vec<T>::x8 row(uint32_t at, int t) const {
        return *(lds_x8 *)(uintptr_t)((rows ^ (uint32_t)(t << 5)) + at);
    }
    // as read_columns, rows 16 half .. 16 half + 15
    __device__ __forceinline__ typename Vec<T>::x8 column(uint32_t at, int half, int dt) const {
        constexpr uint32_t kEight = 2 << 4;  // turn(r + 8) = turn(r) ^ 2
        const uint32_t a = (columns ^ (uint32_t)(dt << 6)) + at + half * 16 * Tile::kRowBytes;
        const uint32_t b = (columns ^ (uint32_t)(dt << 6) ^ kEight) + at + (half * 16 + 8) * Tile::kRowBytes;
        union {
            s16x4 h[2];
            typename Vec<T>::x8 v;
        } u;
        u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)a);
        u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)b);
        return u.v;
    }
};

// Matrix operand: chunk c of row r.
template <typename T, typename Tile>
__device__ __forceinline__ typename Vec<T>::x8 read_rows(const char *tile, int r, int c) {
    return *(const typename Vec<T>::x8 *)(tile + Tile::at(r, c));
}

// Transposed operand of 16 rows from row0 on (a multiple of 16) and columns
// 32 dt .. 32 dt + 31: lane l gets column 32 dt + l % 32 of rows
// row0 + 4 (l / 32) + {0..3} and the same eight rows further: the rows that
// the accumulator layout of a 32x32 product gives a lane.
template <typename T, typename Tile>
__device__ __forceinline__ typename Vec<T>::x8 read_columns(const char *tile, int row0, int dt, int lane) {
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const int t = lane & 15;
    const int c = 4 * dt + 2 * ((lane >> 4) & 1) + ((t & 3) >> 1);
    const int r = row0 + 4 * (lane >> 5) + (t >> 2);
    union {
        s16x4 h[2];
        typename Vec<T>::x8 v;
    } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + Tile::at(r, c) + (t & 1) * 8));
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + Tile::at(r + 8, c) + (t & 1) * 8));
    return u.v;
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

// The 16 numbers of query row `row` and the keys a lane holds of the 32-key
// block kb: byte e % 4 of word e / 4 belongs to accumulator element e.
__device__ __forceinline__ dev::Philox4 keep_words(const CrossParams &p, int64_t row, int kb, int half) {
    return dev::philox4x32_10((uint32_t)(2 * kb + half), (uint32_t)row, (3u << 24) | (uint32_t)((uint64_t)row >> 32),
                              p.call_id, p.seed_lo, p.seed_hi);
}
__device__ __forceinline__ bool kept(const dev::Philox4 &w, int e, uint32_t below) {
    return ((w.w[e >> 2] >> (8 * (e & 3))) & 255u) >= below;
}

// The same for probabilities already rounded and packed in pairs: masks of
// the four numbers of one word, of elements (0, 1) and (2, 3).  Each byte's
// comparison with the threshold comes out in its top bit: that of the low
// seven bits by a subtraction that cannot borrow, then the top bits' own.
__device__ __forceinline__ void keep_pairs(uint32_t w, uint32_t below, uint32_t (&m)[2]) {
    const uint32_t t = below * 0x01010101u, tops = 0x80808080u;
    const uint32_t low = (w | tops) - (t & ~tops);
    // top bit of w above that of t, or equal and the rest no less: (w & low) | ((w | low) & ~t)
    const uint32_t ge = __builtin_amdgcn_bitop3_b32(w, low, t, 0xD4);
    const uint32_t up = ge << 8;
    // the top bits of bytes 1 and 3 of (up, ge), spread over 16 bits each
    m[0] = __builtin_amdgcn_perm(up, ge, 0x08080A0Au);
    m[1] = __builtin_amdgcn_perm(up, ge, 0x09090B0Bu);
}

template <typename T>
__device__ __forceinline__ typename Vec<T>::x8 zero8() {
    typename Vec<T>::x8 z;
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = (T)0.0f;
    return z;
}

// Orders a wave's own LDS traffic, for the compiler too.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// A 32 x 32 tile of 16-bit numbers that lanes write by rows and read by
// columns, each in accumulator order: element e of a lane is column (row)
// 8 (e / 4) + 4 half + e % 4 of its row (column).  The eight-byte pieces of a
// row are turned by the row number, so that neither way meets a bank twice.
struct TurnTile {
    static constexpr int kBytes = 2048;
    __device__ static __forceinline__ int at(int row, int piece) {
        return row * 64 + ((piece ^ ((row >> 2) & 7)) << 3);
    }
    // elements 4 g .. 4 g + 3 of a lane's row
    __device__ static __forceinline__ uint64_t *row_piece(char *tile, int lane, int g) {
        return (uint64_t *)(tile + at(lane & 31, 2 * g + (lane >> 5)));
    }
    // elements 4 g .. 4 g + 3 of a lane's column
    __device__ static __forceinline__ s16x4 column_piece(const char *tile, int lane, int g) {
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const int t = lane & 15;
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4 *)(tile + at(8 * g + 4 * (lane >> 5) + (t >> 2), 4 * ((lane >> 4) & 1) + (t & 3))));
    }
};

// ROWS rows on their way from global memory to LDS, 16 bytes a lane: a thread
// takes the same chunk of every kStep-th row.
template <typename T, int NS, int ROWS, int NT>
struct Lanes {
    static constexpr int kSlots = lanes_per_row(NS);  // three in four work for NS = 6
    static constexpr int kStep = (NT >= 512 ? 512 : NT >= 256 ? 256 : NT >= 128 ? 128 : 64) / kSlots;
    static constexpr int kN = (ROWS + kStep - 1) / kStep;
    static_assert(ROWS % kStep == 0 || kN == 1, "whole rows per thread");
    __device__ static __forceinline__ int row() { return (int)threadIdx.x / kSlots; }
    __device__ static __forceinline__ int slot() { return (int)threadIdx.x % kSlots; }
    // lanes without a chunk of the tile, or past the width
    __device__ static __forceinline__ bool idle() { return slot() >= 2 * NS || row() >= (kN == 1 ? ROWS : kStep); }
    template <typename Tile>
    __device__ static __forceinline__ void store(char *tile, const typename Vec<T>::x8 (&a)[kN]) {
        if (idle()) return;
#pragma unroll
        for (int n = 0; n < kN; ++n) *(typename Vec<T>::x8 *)(tile + Tile::at(row() + n * kStep, slot())) = a[n];
    }
};

// A resource over `bytes` from a uniform address on (almost 4 GiB unless
// said); a load past it, as at kOutside, returns zeros.
constexpr uint32_t kRange = 0xFFFFFF00u, kOutside = 0xFFFFFFF0u;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t resource(const void *base, uint32_t bytes = kRange) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), (short)0, (int)bytes, 0x00020000);
}
template <typename T>
__device__ __forceinline__ typename Vec<T>::x8 load8(__amdgpu_buffer_rsrc_t r, uint32_t at) {
    union {
        u32x4 w;
        typename Vec<T>::x8 v;
    } u;
    u.w = __builtin_amdgcn_raw_buffer_load_b128(r, (int)at, 0, 0);
    return u.v;
}

// Tiles of one of k and v.  The tile's base is uniform and a lane's part of
// the address 32 bits (64 rows of less than 2^25 elements).  Rows past the
// end, hidden keys and chunks past the head's width become zeros, so that
// nothing a hidden key holds (infinities, NaN) reaches a product.  The mask
// travels with the rows and is applied on the way into LDS, so that no load
// waits for it.
template <typename T, int NS, int ROWS, int NT>
struct KeyStage {
    typedef Lanes<T, NS, ROWS, NT> L;
    static_assert(L::kStep <= 64, "a lane's row is below 64");
    typename Vec<T>::x8 a[L::kN];
    uint32_t m[L::kN];
    const char *base;
    const uint8_t *mask;
    int64_t step;      // bytes of a row
    uint32_t lane_at;  // bytes
    int left;          // rows from the tile's first one to the end (uniform)
    __device__ __forceinline__ KeyStage(const CrossTensor &t, const CrossParams &p, const CrossItem &it, int hk) {
        const int64_t tok = it.k0 + it.beg;
        step = 2 * t.row;
        base = (const char *)t.p + tok * step + 2 * (int64_t)hk * t.head;
        mask = p.key_mask ? p.key_mask + tok : nullptr;
        lane_at = L::slot() * 8 < p.dim && !L::idle() ? (uint32_t)L::row() * (uint32_t)step + (uint32_t)L::slot() * 16
                                                      : kOutside;
        left = it.end - it.beg;
    }
    // MASK: with the mask, which k and v of the same rows share
    template <bool MASK>
    __device__ __forceinline__ void load() {
#pragma unroll
        for (int n = 0; n < L::kN; ++n) {
            uint32_t at = lane_at;
            if (left < ROWS) at = L::row() + n * L::kStep < left ? lane_at : kOutside;
            a[n] = load8<T>(resource(base + n * L::kStep * step), at);
            // rows past the end read as hidden
            if (MASK && mask)
                m[n] = __builtin_amdgcn_raw_buffer_load_b8(resource(mask, (uint32_t)max(left, 0)),
                                                           L::row() + n * L::kStep, 0, 0);
        }
        base += ROWS * step;
        if (MASK && mask) mask += ROWS;
        left -= ROWS;
    }
    template <typename Tile>
    __device__ __forceinline__ void store(char *tile, const KeyStage &masked) {
        if (masked.mask)
#pragma unroll
            for (int n = 0; n < L::kN; ++n)
                if (!masked.m[n]) a[n] = zero8<T>();
        L::template store<Tile>(tile, a);
    }
};

// What the scores of a tile's keys begin at: 0, or -inf for keys that are past
// the end or hidden, as the accumulator of the first product of a score.
// `any` (may be null) tells whether an item has a visible key at all.
template <int KT>
struct SeenStage {
    const uint8_t *mask;  // of the tile (uniform)
    int left;             // keys from the tile's first one to the end (uniform)
    uint32_t m;
    __device__ __forceinline__ SeenStage(const CrossParams &p, const CrossItem &it) {
        mask = p.key_mask ? p.key_mask + it.k0 + it.beg : nullptr;
        left = it.end - it.beg;
    }
    __device__ __forceinline__ void load() {
        if (mask) {
            m = __builtin_amdgcn_raw_buffer_load_b8(resource(mask, (uint32_t)max(left, 0)), threadIdx.x, 0, 0);
            mask += KT;
        }
        left -= KT;
    }
    __device__ __forceinline__ void store(float *start, uint32_t *any) const {
        if ((int)threadIdx.x < KT) {
            bool in = (int)threadIdx.x < left + KT;
            if (mask) {
                uint32_t v = m;
                asm volatile("" : "+v"(v));  // the comparison, and the wait for the load, stay here
                in = v != 0;
            }
            start[threadIdx.x] = in ? 0.0f : -kInf;
            if (any && in) *any = 1;
        }
    }
};

// The accumulator that a lane's 16 scores of 32 keys begin with.
__device__ __forceinline__ f32x16 start_of(const float *start, int half) {
    f32x16 s;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const f32x4 v = *(const f32x4 *)(start + 8 * g + 4 * half);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[4 * g + i] = v[i];
    }
    return s;
}

// Accumulator elements whose bit is not set become `hidden`.
__device__ __forceinline__ void hide(f32x16 &s, uint32_t bits, int half, float hidden) {
    const uint32_t mine = bits >> (4 * half);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe((int)mine, 8 * (e >> 2) + (e & 3), 1);
        s[e] = __uint_as_float((__float_as_uint(s[e]) & keep) | (__float_as_uint(hidden) & ~keep));
    }
}

// Tiles of query rows: q and dout, and the softmax sums and deltas of the
// rows.  Row numbers run over tokens and the heads of a group; the addresses
// step by whole tiles, so that no division is left in the loop.
template <typename T, int NS, int ROWS, int NT>
struct QueryStage {
    typedef Lanes<T, NS, ROWS, NT> L;
    typename Vec<T>::x8 a[L::kN], b[L::kN];
    const T *pq[L::kN], *pg[L::kN];
    int g[L::kN];
    int left;                          // rows from this thread's first one to the end; 0 for idle lanes
    int64_t step_q, wrap_q, step_g, wrap_g;
    int step, group;
    int64_t id, step_id, loaded_id;    // this thread's row of the statistics
    int id_g, id_left, heads;
    float lse, delta;
    __device__ __forceinline__ QueryStage(const CrossParams &p, const CrossItem &it, int hk) {
        group = p.group;
        heads = p.heads_q;
        const int tokens = ROWS / group;
        step = ROWS - tokens * group;
        step_q = tokens * p.q.row + step * p.q.head;
        wrap_q = p.q.row - group * p.q.head;
        step_g = tokens * p.dout.row + step * p.dout.head;
        wrap_g = p.dout.row - group * p.dout.head;
        step_id = (int64_t)tokens * heads + step;
#pragma unroll
        for (int n = 0; n < L::kN; ++n) {
            const int r = it.beg + L::row() + n * L::kStep;
            g[n] = r % group;
            a[n] = b[n] = zero8<T>();
            pq[n] = (const T *)p.q.p + row_at(p.q, it.q0, r, group, hk) + L::slot() * 8;
            pg[n] = (const T *)p.dout.p + row_at(p.dout, it.q0, r, group, hk) + L::slot() * 8;
        }
        left = L::slot() * 8 < p.dim && !L::idle() ? it.end - it.beg - L::row() : 0;
        const int r = it.beg + (int)threadIdx.x;
        id = row_id(p, it.q0, r, hk);
        id_g = r % group;
        id_left = (int)threadIdx.x < ROWS ? it.end - r : 0;
    }
    __device__ __forceinline__ void load(const CrossParams &p) {
#pragma unroll
        for (int n = 0; n < L::kN; ++n) {
            // rows past the end keep what an earlier tile had there (or zeros):
            // their probabilities are zero
            if (n * L::kStep < left) {
                a[n] = *(const typename Vec<T>::x8 *)pq[n];
                b[n] = *(const typename Vec<T>::x8 *)pg[n];
            }
            g[n] += step;
            const bool over = g[n] >= group;
            g[n] -= over ? group : 0;
            pq[n] += step_q + (over ? wrap_q : 0);
            pg[n] += step_g + (over ? wrap_g : 0);
        }
        left -= ROWS;
        lse = -kInf;
        delta = 0.0f;
        loaded_id = id;
        if (id_left > 0) {
            lse = p.lse[id];
            delta = p.delta[id];
        }
        id_g += step;
        const bool over = id_g >= group;
        id_g -= over ? group : 0;
        id += step_id + (over ? heads - group : 0);
        id_left -= ROWS;
    }
    // A row without a visible key, or past the end, gets exponent -inf.  Its
    // number is that of the tile just loaded.
    template <typename Tile>
    __device__ __forceinline__ void store(char *tq, char *tg, float *stat_lse, float *stat_delta,
                                          int64_t *stat_id) const {
        L::template store<Tile>(tq, a);
        L::template store<Tile>(tg, b);
        if ((int)threadIdx.x < ROWS) {
            stat_lse[(int)threadIdx.x] = lse == -kInf ? kInf : lse * kLog2e;
            stat_delta[(int)threadIdx.x] = -delta;
            if (stat_id) stat_id[(int)threadIdx.x] = loaded_id;
        }
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

// A lane's value and that of the lane 32 away.
__device__ __forceinline__ float both_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float both_sum(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Accumulator element e of a lane is row 8 (e / 4) + 4 half + e % 4.
__device__ __forceinline__ int acc_row(int e, int half) { return 8 * (e >> 2) + 4 * half + (e & 3); }

template <typename T>
__device__ __forceinline__ typename Vec<T>::x8 round8(const f32x16 &a, int first, float up = 1.0f) {
    typename Vec<T>::x8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (T)(a[first + i] * up);
    return r;
}

// Writes the columns of one owner: a lane holds o[dt][e] = column
// 32 dt + acc_row(e), four and four; the two lanes of an owner exchange them
// to eight in a row.  Both lanes of an owner call it.
template <typename T, int ND>
__device__ __forceinline__ void write_owner(T *dst, const f32x16 (&o)[ND], float gain, int half, int dim) {
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            union {
                typename Vec<T>::x4 v[2];
                uint32_t w[4];
            } x;
#pragma unroll
            for (int i = 0; i < 8; ++i) x.v[i >> 2][i & 3] = (T)(o[dt][8 * g + i] * gain);
            u32x4 y;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const auto r = __builtin_amdgcn_permlane32_swap(x.w[i], x.w[2 + i], false, false);
                y[i] = r[0];
                y[2 + i] = r[1];
            }
            const int d = 32 * dt + 16 * g + 8 * half;
            if (d < dim) *(u32x4 *)(dst + d) = y;
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

// The second choice of owner waves beside 4 (see build_pass).
template <bool FORWARD, int NS>
constexpr int kWide = FORWARD ? (NS > 4 ? 8 : 4) : (NS > 4 ? 4 : 2);

inline uint32_t grid_of(const CrossParams &p) { return (uint32_t)p.n_items * (uint32_t)p.heads_kv; }

template <typename Pass, typename T, int NS, int OW, int CW>
void launch_drop(const CrossParams &p, hipStream_t s) {
    if (p.drop_below)
        Pass::template run<T, NS, OW, CW, true>(p, s);
    else
        Pass::template run<T, NS, OW, CW, false>(p, s);
}

// The geometries that a plan may choose for a pass and a width.
template <typename Pass, typename T, int NS>
void launch_shape(const CrossParams &p, const CrossPass &w, hipStream_t s) {
    if (w.own_waves == kWide<Pass::kForward, NS>)
        launch_drop<Pass, T, NS, kWide<Pass::kForward, NS>, 1>(p, s);
    else if (w.own_waves == 4)
        launch_drop<Pass, T, NS, 4, 1>(p, s);
    else
        launch_drop<Pass, T, NS, 1, 4>(p, s);
}

template <typename Pass, typename T>
hipError_t launch_typed(CrossParams p, const CrossPass &w, hipStream_t s) {
    if (w.n_items == 0) return hipSuccess;
    const int32_t per = items_per_launch(p.heads_kv);
    for (int64_t first = 0; first < w.n_items; first += per) {
        p.items = w.items + first;
        p.n_items = (int32_t)std::min<int64_t>(per, w.n_items - first);
        if (p.dim <= 32)
            launch_shape<Pass, T, 2>(p, w, s);
        else if (p.dim <= 64)
            launch_shape<Pass, T, 4>(p, w, s);
        else if (p.dim <= 96)
            launch_shape<Pass, T, 6>(p, w, s);
        else
            launch_shape<Pass, T, 8>(p, w, s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (w.n_joins == 0) return hipSuccess;
    Pass::template join<T>(p, w, dim3((uint32_t)w.n_joins, p.heads_kv, 32 * w.own_waves / kJoinOwners), s);
    return hipGetLastError();
}

template <typename Pass>
hipError_t launch_pass(const CrossParams &p, const CrossPass &w, int dtype, hipStream_t s) {
    return dtype == kCrossBf16 ? launch_typed<Pass, __bf16>(p, w, s) : launch_typed<Pass, _Float16>(p, w, s);
}

}  // namespace cross
}  // namespace same
