// Cross attention over ragged segments, forward pass (gfx950).
#include "cross_common.hpp"

namespace same {
namespace {

using namespace cross;

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
__global__ __launch_bounds__(64 * OW * CW, 2) void cross_forward_kernel(CrossParams p) {
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

    KeyStage<T, NS, KT, NT> st(p, it, hk);
    auto flags = [&](int buf, int key) {
        for (int i = threadIdx.x; i < KT; i += NT) {
            bool in = key + i < it.end;
            if (in && p.key_mask) in = p.key_mask[it.k0 + key + i] != 0;
            ((uint8_t *)seen[buf])[i] = in;
        }
    };
    if (it.beg < it.end) {
        st.load(p);
        st.store(lds, lds + kTile);
        flags(0, it.beg);
    }
    __syncthreads();
    int buf = 0;
    for (int key = it.beg; key < it.end; key += KT) {
        const bool more = key + KT < it.end;
        if (more) st.load(p);
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
            st.store(lds + nb * 2 * kTile, lds + nb * 2 * kTile + kTile);
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

struct Pass {
    template <typename T, int NS, int OW, int CW, bool DROP>
    static void run(const CrossParams &p, hipStream_t s) {
        cross_forward_kernel<T, NS, OW, CW, (OW > 1 ? 2 : 1), DROP><<<dim3(grid_of(p)), 64 * OW * CW, 0, s>>>(p);
    }
    template <typename T>
    static void join(const CrossParams &p, const CrossPass &w, dim3 grid, hipStream_t s) {
        cross_join_forward_kernel<T><<<grid, 256, 0, s>>>(p, w.joins, w.n_joins, 32 * w.own_waves);
    }
};

}  // namespace

hipError_t launch_cross_forward(const CrossParams &p, const CrossPass &w, int dtype, hipStream_t s) {
    return cross::launch_pass<Pass>(p, w, dtype, s);
}

}  // namespace same
