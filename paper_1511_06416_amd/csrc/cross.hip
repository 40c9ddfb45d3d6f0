// Cross attention over ragged segments and its gradients, for gfx950.
#include "cross.hpp"
#include "philox.hpp"

namespace same {
namespace {

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

// Rows of keys (or of queries) on their way from global memory to LDS.
template <typename T, int NS, int ROWS, int NT>
struct Stage {
    static constexpr int kN = (ROWS * 2 * NS + NT - 1) / NT;
    typename Vec<T>::x8 a[kN], b[kN];
};

template <typename T>
__device__ __forceinline__ typename Vec<T>::x8 zero8() {
    typename Vec<T>::x8 z;
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = (T)0.0f;
    return z;
}

// Keys [key, key + ROWS) of k and v; rows past `end`, hidden keys and chunks
// past the head's width become zeros, so that nothing a hidden key holds
// (infinities, NaN) reaches a product.
template <typename T, int NS, int ROWS, int NT>
__device__ __forceinline__ void load_keys(Stage<T, NS, ROWS, NT> &st, const CrossParams &p, int64_t k0, int key,
                                          int end, int hk) {
    const T *kp = (const T *)p.k.p + (int64_t)hk * p.k.head;
    const T *vp = (const T *)p.v.p + (int64_t)hk * p.v.head;
#pragma unroll
    for (int n = 0; n < st.kN; ++n) {
        const int idx = threadIdx.x + n * NT;
        const int r = idx / (2 * NS), c = idx % (2 * NS);
        const int64_t tok = k0 + key + r;
        bool in = r < ROWS && key + r < end && c * 8 < p.dim;
        if (in && p.key_mask) in = p.key_mask[tok] != 0;
        st.a[n] = in ? *(const typename Vec<T>::x8 *)(kp + tok * p.k.row + c * 8) : zero8<T>();
        st.b[n] = in ? *(const typename Vec<T>::x8 *)(vp + tok * p.v.row + c * 8) : zero8<T>();
    }
}

// Query rows [row, row + ROWS) of q and dout.
template <typename T, int NS, int ROWS, int NT>
__device__ __forceinline__ void load_queries(Stage<T, NS, ROWS, NT> &st, const CrossParams &p, int64_t q0, int row,
                                             int end, int hk) {
#pragma unroll
    for (int n = 0; n < st.kN; ++n) {
        const int idx = threadIdx.x + n * NT;
        const int r = idx / (2 * NS), c = idx % (2 * NS);
        const bool in = r < ROWS && row + r < end && c * 8 < p.dim;
        st.a[n] = in ? *(const typename Vec<T>::x8 *)((const T *)p.q.p + row_at(p.q, q0, row + r, p.group, hk) + c * 8)
                     : zero8<T>();
        st.b[n] = in ? *(const typename Vec<T>::x8 *)((const T *)p.dout.p +
                                                      row_at(p.dout, q0, row + r, p.group, hk) + c * 8)
                     : zero8<T>();
    }
}

template <typename T, int NS, int ROWS, int NT>
__device__ __forceinline__ void store_stage(const Stage<T, NS, ROWS, NT> &st, char *ta, char *tb) {
#pragma unroll
    for (int n = 0; n < st.kN; ++n) {
        const int idx = threadIdx.x + n * NT;
        const int r = idx / (2 * NS), c = idx % (2 * NS);
        if (ROWS * 2 * NS % NT && r >= ROWS) continue;
        *(typename Vec<T>::x8 *)(ta + Tile<NS>::at(r, c)) = st.a[n];
        *(typename Vec<T>::x8 *)(tb + Tile<NS>::at(r, c)) = st.b[n];
    }
}

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

// ---------------------------------------------------------------- forward
//
// A wave owns 32 query rows and keeps, per row (= per lane, both halves), the
// running maximum and sum of the softmax over the keys seen so far and the
// weighted sum of values O^T [width x rows] in accumulators.  Per 32 keys:
// S^T = K Q^T (keys x rows), so that a lane holds 16 scores of its own row;
// those, rounded to 16 bits, are already the B operand of O^T += V^T P^T with
// the keys in accumulator order, and V^T is read transposed from LDS in the
// same order.
template <typename T, int NS, int OW, int CW, int KS, bool DROP>
__global__ __launch_bounds__(64 * OW * CW, 1) void cross_forward_kernel(CrossParams p) {
    constexpr int NT = 64 * OW * CW, KT = 32 * KS * CW, ND = (NS + 1) / 2;
    constexpr int kTile = KT * Tile<NS>::kRowBytes;
    constexpr int kBufs = CW > 1 ? 1 : 2;
    constexpr int kLds = max_of(2 * kTile * kBufs, CW > 1 ? OW * ND * 4096 : 0);
    __shared__ __attribute__((aligned(16))) char lds[kLds];
    __shared__ uint32_t seen[kBufs][KT / 4];
    __shared__ float stat[2][OW * CW * 32];
    const int64_t lb = logical_block(p.chunk);
    if (lb >= (int64_t)p.n_items * p.heads_kv) return;
    const int hk = (int)(lb / p.n_items);
    const CrossItem it = p.items[lb - (int64_t)hk * p.n_items];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, col = lane & 31;
    const int ow = wave % OW, cw = wave / OW;
    const int own = ow * 32 + col;
    const bool valid = own < it.n_own;
    const int r = valid ? it.own0 + own : it.own0;
    const int64_t row = row_id(p, it.q0, r, hk);
    typename Vec<T>::x8 qf[NS];
    load_own<T, NS>(qf, (const T *)p.q.p + row_at(p.q, it.q0, r, p.group, hk), valid, half, p.dim);
    f32x16 o[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) o[dt] = 0.0f;
    float top = -kInf, sum = 0.0f;
    const float c = p.scale * kLog2e;

    Stage<T, NS, KT, NT> st;
    auto flags = [&](int buf, int key) {
        for (int i = threadIdx.x; i < KT; i += NT) {
            bool in = key + i < it.end;
            if (in && p.key_mask) in = p.key_mask[it.k0 + key + i] != 0;
            ((uint8_t *)seen[buf])[i] = in;
        }
    };
    if (it.beg < it.end) {
        load_keys(st, p, it.k0, it.beg, it.end, hk);
        store_stage(st, lds, lds + kTile);
        flags(0, it.beg);
    }
    __syncthreads();
    int buf = 0;
    for (int key = it.beg; key < it.end; key += KT) {
        const bool more = key + KT < it.end;
        if (more) load_keys(st, p, it.k0, key + KT, it.end, hk);
        const char *tk = lds + buf * 2 * kTile, *tv = tk + kTile;
        f32x16 s[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            s[ks] = 0.0f;
            const int base = (cw * KS + ks) * 32;
#pragma unroll
            for (int t = 0; t < NS; ++t) s[ks] = mfma(read_rows<T, NS>(tk, base + col, 2 * t + half), qf[t], s[ks]);
        }
        if (p.key_mask || key + KT > it.end) {
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const uint32_t f = seen[buf][((cw * KS + ks) * 32 + 8 * g + 4 * half) >> 2];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!((f >> (8 * i)) & 1)) s[ks][4 * g + i] = -kInf;
                }
        }
        float mx = top;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[ks][e]);
        mx = fmaxf(mx, other_half(mx));
        if (__any(mx > top)) {
            // a row whose keys are all hidden so far keeps -inf; 0 stands in for it below
            const float from = top == -kInf ? 0.0f : top, to = mx == -kInf ? 0.0f : mx;
            const float f = __builtin_amdgcn_exp2f((from - to) * c);
            const float g = top == -kInf ? 0.0f : f;
            sum *= g;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) o[dt] *= g;
            top = mx;
        }
        const float base2 = (top == -kInf ? 0.0f : top) * c;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[ks][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[ks][e], c, -base2));
                sum += s[ks][e];
            }
            if (DROP) {
                const uint32_t keep = keep_bits(p, row, ((key + (cw * KS + ks) * 32)) >> 5, half);
#pragma unroll
                for (int e = 0; e < 16; ++e) s[ks][e] = (keep >> e) & 1 ? s[ks][e] : 0.0f;
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const typename Vec<T>::x8 pf = round8<T>(s[ks], 8 * t);
#pragma unroll
                for (int dt = 0; dt < ND; ++dt)
                    o[dt] = mfma(read_columns<T, NS>(tv, (cw * KS + ks) * 32 + 16 * t, dt, lane), pf, o[dt]);
            }
        }
        if (kBufs == 1) __syncthreads();
        if (more) {
            const int nb = kBufs == 1 ? 0 : buf ^ 1;
            store_stage(st, lds + nb * 2 * kTile, lds + nb * 2 * kTile + kTile);
            flags(nb, key + KT);
            buf = nb;
        }
        __syncthreads();
    }
    sum += other_half(sum);
    if (CW > 1) {
        // the waves that share these rows bring their sums to the common maximum
        if (half == 0) {
            stat[0][(ow * CW + cw) * 32 + col] = top;
            stat[1][(ow * CW + cw) * 32 + col] = sum;
        }
        __syncthreads();
        float mx = -kInf;
#pragma unroll
        for (int w = 0; w < CW; ++w) mx = fmaxf(mx, stat[0][(ow * CW + w) * 32 + col]);
        const float to = mx == -kInf ? 0.0f : mx;
        float total = 0.0f;
#pragma unroll
        for (int w = 0; w < CW; ++w)
            total += stat[1][(ow * CW + w) * 32 + col] * __builtin_amdgcn_exp2f((stat[0][(ow * CW + w) * 32 + col] - to) * c);
        const float f = __builtin_amdgcn_exp2f((top - to) * c);
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) o[dt] *= f;
        join_waves<ND, OW, CW>(o, lds, ow, cw, lane);
        top = mx;
        sum = total;
        if (cw != 0) return;
    }
    if (!valid) return;
    if (it.slot >= 0) {
        const int64_t at = ((int64_t)it.slot * p.heads_kv + hk) * (32 * OW) + own;
        write_part<ND>(p.part + at * p.dim, o, half, p.dim);
        if (half == 0) {
            p.part_ml[2 * at] = top;
            p.part_ml[2 * at + 1] = sum;
        }
        return;
    }
    write_owner<T, ND>((T *)p.out + row * p.dim, o, sum > 0.0f ? (DROP ? p.keep_gain : 1.0f) / sum : (sum == 0.0f ? 0.0f : sum), half,
                       p.dim);
    if (p.lse && half == 0)
        p.lse[row] = sum == 0.0f ? -kInf : top * p.scale + __builtin_amdgcn_logf(sum) * kLn2;
}

// Joins the parts of split rows: one block per tile of rows and key head.
template <typename T>
__global__ __launch_bounds__(256) void cross_join_forward_kernel(CrossParams p, const CrossJoin *joins, int32_t n_joins,
                                                                 int tile) {
    const int hk = blockIdx.x / n_joins;
    const CrossJoin j = joins[blockIdx.x - hk * n_joins];
    const float c = p.scale * kLog2e;
    const int quads = p.dim / 4;
    for (int idx = threadIdx.x; idx < j.n_own * quads; idx += blockDim.x) {
        const int own = idx / quads, d = (idx % quads) * 4;
        float mx = -kInf;
        for (int s = 0; s < j.n_parts; ++s)
            mx = fmaxf(mx, p.part_ml[2 * (((int64_t)(j.slot + s) * p.heads_kv + hk) * tile + own)]);
        const float to = mx == -kInf ? 0.0f : mx;
        float total = 0.0f;
        f32x4 acc = 0.0f;
        for (int s = 0; s < j.n_parts; ++s) {
            const int64_t at = ((int64_t)(j.slot + s) * p.heads_kv + hk) * tile + own;
            const float f = __builtin_amdgcn_exp2f((p.part_ml[2 * at] - to) * c);
            total += f * p.part_ml[2 * at + 1];
            acc += *(const f32x4 *)(p.part + at * p.dim + d) * f;
        }
        const int64_t row = row_id(p, j.q0, j.own0 + own, hk);
        const float gain = total > 0.0f ? p.keep_gain / total : (total == 0.0f ? 0.0f : total);
        typename Vec<T>::x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (T)(acc[i] * gain);
        *(typename Vec<T>::x4 *)((T *)p.out + row * p.dim + d) = w;
        if (p.lse && d == 0) p.lse[row] = total == 0.0f ? -kInf : mx * p.scale + __builtin_amdgcn_logf(total) * kLn2;
    }
}

// ------------------------------------------------------------- gradient: dQ
//
// A wave owns 32 query rows and walks the keys as the forward does:
// P = exp(S - lse), dP^T = V dO^T, dS = P (D dP - delta),
// dQ^T += K^T dS^T; delta = sum over the width of dO * O, kept for dK, dV.
template <typename T, int NS, int OW, int CW, bool DROP>
__global__ __launch_bounds__(64 * OW * CW, 1) void cross_dq_kernel(CrossParams p) {
    constexpr int NT = 64 * OW * CW, KT = 32 * CW, ND = (NS + 1) / 2;
    constexpr int kTile = KT * Tile<NS>::kRowBytes;
    constexpr int kBufs = CW > 1 ? 1 : 2;
    constexpr int kLds = max_of(2 * kTile * kBufs, CW > 1 ? OW * ND * 4096 : 0);
    __shared__ __attribute__((aligned(16))) char lds[kLds];
    __shared__ uint32_t seen[kBufs][KT / 4];
    const int64_t lb = logical_block(p.chunk);
    if (lb >= (int64_t)p.n_items * p.heads_kv) return;
    const int hk = (int)(lb / p.n_items);
    const CrossItem it = p.items[lb - (int64_t)hk * p.n_items];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, col = lane & 31;
    const int ow = wave % OW, cw = wave / OW;
    const int own = ow * 32 + col;
    const bool valid = own < it.n_own;
    const int r = valid ? it.own0 + own : it.own0;
    const int64_t row = row_id(p, it.q0, r, hk);
    typename Vec<T>::x8 qf[NS], gf[NS];
    load_own<T, NS>(qf, (const T *)p.q.p + row_at(p.q, it.q0, r, p.group, hk), valid, half, p.dim);
    load_own<T, NS>(gf, (const T *)p.dout.p + row_at(p.dout, it.q0, r, p.group, hk), valid, half, p.dim);
    float delta = 0.0f;
    {
        typename Vec<T>::x8 of[NS];
        load_own<T, NS>(of, (const T *)p.out_in + row * p.dim, valid, half, p.dim);
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int i = 0; i < 8; ++i) delta = __builtin_fmaf((float)of[s][i], (float)gf[s][i], delta);
        delta += other_half(delta);
    }
    if (valid && half == 0 && cw == 0 && it.beg == 0) p.delta[row] = delta;
    f32x16 o[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) o[dt] = 0.0f;
    const float c = p.scale * kLog2e;
    const float lse = valid ? p.lse[row] : -kInf;
    const float base2 = lse == -kInf ? kInf : lse * kLog2e;
    const float gain = DROP ? p.keep_gain : 1.0f;

    Stage<T, NS, KT, NT> st;
    auto flags = [&](int buf, int key) {
        for (int i = threadIdx.x; i < KT; i += NT) {
            bool in = key + i < it.end;
            if (in && p.key_mask) in = p.key_mask[it.k0 + key + i] != 0;
            ((uint8_t *)seen[buf])[i] = in;
        }
    };
    if (it.beg < it.end) {
        load_keys(st, p, it.k0, it.beg, it.end, hk);
        store_stage(st, lds, lds + kTile);
        flags(0, it.beg);
    }
    __syncthreads();
    int buf = 0;
    for (int key = it.beg; key < it.end; key += KT) {
        const bool more = key + KT < it.end;
        if (more) load_keys(st, p, it.k0, key + KT, it.end, hk);
        const char *tk = lds + buf * 2 * kTile, *tv = tk + kTile;
        const int base = cw * 32;
        f32x16 s = 0.0f, dp = 0.0f;
#pragma unroll
        for (int t = 0; t < NS; ++t) {
            s = mfma(read_rows<T, NS>(tk, base + col, 2 * t + half), qf[t], s);
            dp = mfma(read_rows<T, NS>(tv, base + col, 2 * t + half), gf[t], dp);
        }
        uint32_t keep = 0xFFFF;
        if (DROP) keep = keep_bits(p, row, (key + base) >> 5, half);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, -base2));
            const float d = DROP ? ((keep >> e) & 1 ? dp[e] * gain : 0.0f) : dp[e];
            s[e] = w * (d - delta);
        }
        if (p.key_mask || key + KT > it.end) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const uint32_t f = seen[buf][(base + 8 * g + 4 * half) >> 2];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!((f >> (8 * i)) & 1)) s[4 * g + i] = 0.0f;
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const typename Vec<T>::x8 df = round8<T>(s, 8 * t);
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) o[dt] = mfma(read_columns<T, NS>(tk, base + 16 * t, dt, lane), df, o[dt]);
        }
        if (kBufs == 1) __syncthreads();
        if (more) {
            const int nb = kBufs == 1 ? 0 : buf ^ 1;
            store_stage(st, lds + nb * 2 * kTile, lds + nb * 2 * kTile + kTile);
            flags(nb, key + KT);
            buf = nb;
        }
        __syncthreads();
    }
    if (CW > 1) {
        join_waves<ND, OW, CW>(o, lds, ow, cw, lane);
        if (cw != 0) return;
    }
    if (!valid) return;
    if (it.slot >= 0) {
        const int64_t at = ((int64_t)it.slot * p.heads_kv + hk) * (32 * OW) + own;
        write_part<ND>(p.part + at * p.dim, o, half, p.dim);
        return;
    }
    write_owner<T, ND>((T *)p.dq + row * p.dim, o, p.scale, half, p.dim);
}

// -------------------------------------------------------- gradient: dK and dV
//
// The mirror image: a wave owns 32 keys of a key head (a lane one key) and
// walks the query rows of every head that shares it, so that the sum over
// those heads stays in its accumulators.  S = Q K^T (rows x keys),
// dV^T += dO^T (D P), dK^T += Q^T dS.
template <typename T, int NS, int OW, int CW, bool DROP>
__global__ __launch_bounds__(64 * OW * CW, 1) void cross_dkv_kernel(CrossParams p) {
    constexpr int NT = 64 * OW * CW, QT = 32 * CW, ND = (NS + 1) / 2;
    constexpr int kTile = QT * Tile<NS>::kRowBytes;
    constexpr int kBufs = CW > 1 ? 1 : 2;
    constexpr int kLds = max_of(2 * kTile * kBufs, CW > 1 ? OW * ND * 4096 : 0);
    __shared__ __attribute__((aligned(16))) char lds[kLds];
    __shared__ f32x4 stat[kBufs][2][QT / 4];
    const int64_t lb = logical_block(p.chunk);
    if (lb >= (int64_t)p.n_items * p.heads_kv) return;
    const int hk = (int)(lb / p.n_items);
    const CrossItem it = p.items[lb - (int64_t)hk * p.n_items];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, col = lane & 31;
    const int ow = wave % OW, cw = wave / OW;
    const int own = ow * 32 + col;
    const bool valid = own < it.n_own;
    const int64_t tok = it.k0 + it.own0 + (valid ? own : 0);
    const bool visible = valid && (!p.key_mask || p.key_mask[tok] != 0);
    typename Vec<T>::x8 kf[NS], vf[NS];
    load_own<T, NS>(kf, (const T *)p.k.p + tok * p.k.row + (int64_t)hk * p.k.head, visible, half, p.dim);
    load_own<T, NS>(vf, (const T *)p.v.p + tok * p.v.row + (int64_t)hk * p.v.head, visible, half, p.dim);
    f32x16 ok[ND], ov[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) ok[dt] = ov[dt] = 0.0f;
    const float c = p.scale * kLog2e;
    const float gain = DROP ? p.keep_gain : 1.0f;

    Stage<T, NS, QT, NT> st;
    auto stats = [&](int buf, int row) {
        for (int i = threadIdx.x; i < QT; i += NT) {
            float l = kInf, d = 0.0f;
            if (row + i < it.end) {
                const int64_t id = row_id(p, it.q0, row + i, hk);
                l = p.lse[id];
                l = l == -kInf ? kInf : l * kLog2e;
                d = p.delta[id];
            }
            ((float *)stat[buf][0])[i] = l;
            ((float *)stat[buf][1])[i] = d;
        }
    };
    if (it.beg < it.end) {
        load_queries(st, p, it.q0, it.beg, it.end, hk);
        store_stage(st, lds, lds + kTile);
        stats(0, it.beg);
    }
    __syncthreads();
    int buf = 0;
    for (int row = it.beg; row < it.end; row += QT) {
        const bool more = row + QT < it.end;
        if (more) load_queries(st, p, it.q0, row + QT, it.end, hk);
        const char *tq = lds + buf * 2 * kTile, *tg = tq + kTile;
        const int base = cw * 32;
        f32x16 s = 0.0f, dp = 0.0f;
#pragma unroll
        for (int t = 0; t < NS; ++t) {
            s = mfma(read_rows<T, NS>(tq, base + col, 2 * t + half), kf[t], s);
            dp = mfma(read_rows<T, NS>(tg, base + col, 2 * t + half), vf[t], dp);
        }
        uint32_t keep = 0xFFFFFFFF;  // bit i: the block's row i keeps this lane's key
        if (DROP) {
            // the flags are made row by row, as in the other passes (a lane a
            // row, 16 keys); a ballot per element turns them into one word of
            // 32 rows per key, and lane l takes the word of key l % 32
            const int rr = row + base + col;
            const int64_t id = row_id(p, it.q0, rr < it.end ? rr : it.end - 1, hk);
            const uint32_t mine = keep_bits(p, id, (it.own0 + ow * 32) >> 5, half);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint64_t b = __ballot((mine >> e) & 1);
                if (col == acc_row(e, 0)) keep = (uint32_t)b;
                if (col == acc_row(e, 1)) keep = (uint32_t)(b >> 32);
            }
        }
        f32x16 w;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 l4 = stat[buf][0][(base + 8 * g + 4 * half) >> 2];
            const f32x4 d4 = stat[buf][1][(base + 8 * g + 4 * half) >> 2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = 4 * g + i;
                float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, -l4[i]));
                x = visible ? x : 0.0f;
                float d = dp[e];
                w[e] = x;
                if (DROP) {
                    const bool kept = (keep >> acc_row(e, half)) & 1;
                    d = kept ? d * gain : 0.0f;
                    w[e] = kept ? x : 0.0f;
                }
                s[e] = x * (d - d4[i]);
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const typename Vec<T>::x8 wf = round8<T>(w, 8 * t), df = round8<T>(s, 8 * t);
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) {
                ov[dt] = mfma(read_columns<T, NS>(tg, base + 16 * t, dt, lane), wf, ov[dt]);
                ok[dt] = mfma(read_columns<T, NS>(tq, base + 16 * t, dt, lane), df, ok[dt]);
            }
        }
        if (kBufs == 1) __syncthreads();
        if (more) {
            const int nb = kBufs == 1 ? 0 : buf ^ 1;
            store_stage(st, lds + nb * 2 * kTile, lds + nb * 2 * kTile + kTile);
            stats(nb, row + QT);
            buf = nb;
        }
        __syncthreads();
    }
    if (CW > 1) {
        join_waves<ND, OW, CW>(ok, lds, ow, cw, lane);
        join_waves<ND, OW, CW>(ov, lds, ow, cw, lane);
        if (cw != 0) return;
    }
    if (!valid) return;
    if (!visible)  // whatever the queries hold, a hidden key's gradients are zero
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) ok[dt] = ov[dt] = 0.0f;
    if (it.slot >= 0) {
        const int64_t at = ((int64_t)it.slot * p.heads_kv + hk) * (32 * OW) + own;
        write_part<ND>(p.part + 2 * at * p.dim, ok, half, p.dim);
        write_part<ND>(p.part + (2 * at + 1) * p.dim, ov, half, p.dim);
        return;
    }
    const int64_t at = (tok * p.heads_kv + hk) * p.dim;
    write_owner<T, ND>((T *)p.dk + at, ok, p.scale, half, p.dim);
    write_owner<T, ND>((T *)p.dv + at, ov, gain, half, p.dim);
}

// Sums the parts of dQ (SIDES = 1) or of dK and dV (SIDES = 2), in order.
template <typename T, int SIDES>
__global__ __launch_bounds__(256) void cross_join_grad_kernel(CrossParams p, const CrossJoin *joins, int32_t n_joins,
                                                              int tile) {
    const int hk = blockIdx.x / n_joins;
    const CrossJoin j = joins[blockIdx.x - hk * n_joins];
    const int quads = p.dim / 4;
    for (int idx = threadIdx.x; idx < j.n_own * quads * SIDES; idx += blockDim.x) {
        const int own = idx / (quads * SIDES), side = (idx / quads) % SIDES, d = (idx % quads) * 4;
        f32x4 acc = 0.0f;
        for (int s = 0; s < j.n_parts; ++s) {
            const int64_t at = ((int64_t)(j.slot + s) * p.heads_kv + hk) * tile + own;
            acc += *(const f32x4 *)(p.part + (SIDES * at + side) * p.dim + d);
        }
        T *dst;
        float gain = p.scale;
        if (SIDES == 1) {
            dst = (T *)p.dq + row_id(p, j.q0, j.own0 + own, hk) * p.dim;
        } else {
            dst = (T *)(side ? p.dv : p.dk) + ((j.k0 + j.own0 + own) * p.heads_kv + hk) * p.dim;
            gain = side ? p.keep_gain : p.scale;
        }
        typename Vec<T>::x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (T)(acc[i] * gain);
        *(typename Vec<T>::x4 *)(dst + d) = w;
    }
}

inline uint32_t grid_of(const CrossParams &p) {
    const int64_t n = (int64_t)p.n_items * p.heads_kv, unit = 8 * (int64_t)p.chunk;
    return (uint32_t)((n + unit - 1) / unit * unit);
}

enum Pass { kForward, kDq, kDkv };

template <Pass PASS, typename T, int NS, int OW, int CW, bool DROP>
void launch_one(const CrossParams &p, hipStream_t s) {
    const dim3 grid(grid_of(p)), block(64 * OW * CW);
    if constexpr (PASS == kForward)
        cross_forward_kernel<T, NS, OW, CW, (OW > 1 ? 2 : 1), DROP><<<grid, block, 0, s>>>(p);
    else if constexpr (PASS == kDq)
        cross_dq_kernel<T, NS, OW, CW, DROP><<<grid, block, 0, s>>>(p);
    else
        cross_dkv_kernel<T, NS, OW, CW, DROP><<<grid, block, 0, s>>>(p);
}

template <Pass PASS, typename T, int NS>
void launch_shape(const CrossParams &p, const CrossPass &w, hipStream_t s) {
    const bool drop = p.drop_below != 0;
    if (w.own_waves == 4)
        drop ? launch_one<PASS, T, NS, 4, 1, true>(p, s) : launch_one<PASS, T, NS, 4, 1, false>(p, s);
    else if (w.cut_waves == 4)
        drop ? launch_one<PASS, T, NS, 1, 4, true>(p, s) : launch_one<PASS, T, NS, 1, 4, false>(p, s);
    else
        drop ? launch_one<PASS, T, NS, 1, 1, true>(p, s) : launch_one<PASS, T, NS, 1, 1, false>(p, s);
}

template <Pass PASS, typename T>
hipError_t launch_pass(CrossParams p, const CrossPass &w, hipStream_t s) {
    if (w.n_items == 0) return hipSuccess;
    p.items = w.items;
    p.n_items = w.n_items;
    p.chunk = 4;
    if (p.dim <= 32)
        launch_shape<PASS, T, 2>(p, w, s);
    else if (p.dim <= 64)
        launch_shape<PASS, T, 4>(p, w, s);
    else if (p.dim <= 96)
        launch_shape<PASS, T, 6>(p, w, s);
    else
        launch_shape<PASS, T, 8>(p, w, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || w.n_joins == 0) return e;
    const dim3 grid((uint32_t)w.n_joins * p.heads_kv);
    const int tile = 32 * w.own_waves;
    if constexpr (PASS == kForward)
        cross_join_forward_kernel<T><<<grid, 256, 0, s>>>(p, w.joins, w.n_joins, tile);
    else
        cross_join_grad_kernel<T, (PASS == kDq ? 1 : 2)><<<grid, 256, 0, s>>>(p, w.joins, w.n_joins, tile);
    return hipGetLastError();
}

template <Pass PASS>
hipError_t launch_typed(const CrossParams &p, const CrossPass &w, int dtype, hipStream_t s) {
    return dtype == kCrossBf16 ? launch_pass<PASS, __bf16>(p, w, s) : launch_pass<PASS, _Float16>(p, w, s);
}

}  // namespace

hipError_t launch_cross_forward(const CrossParams &p, const CrossPass &w, int dtype, hipStream_t s) {
    return launch_typed<kForward>(p, w, dtype, s);
}
hipError_t launch_cross_dq(const CrossParams &p, const CrossPass &w, int dtype, hipStream_t s) {
    return launch_typed<kDq>(p, w, dtype, s);
}
hipError_t launch_cross_dkv(const CrossParams &p, const CrossPass &w, int dtype, hipStream_t s) {
    return launch_typed<kDkv>(p, w, dtype, s);
}

}  // namespace same
