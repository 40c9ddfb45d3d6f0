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
// same order.  A row's largest probability is rounded as a number from 1 to 2^8
// (fp16: 2^7 to 2^15, so that keys down to 2^-21 of the largest, and not 2^-14,
// are normal numbers), each with the type's digits; sums, statistics and O stay
// in fp32.
//
// What bounds it: at 128 wide the matrix units and the exponents beside them
// (busy 45 and 41 % of the time: a wave's products wait for its softmax, which
// the second wave of the SIMD hides in part), 2 x 4,099 rows on 7,951 keys, 16
// heads on 4, 522 us, 1020 TFLOP/s.  At 64 wide with dropout the vector units
// (77 % busy), 64 columns of 1000 nodes 118 us; the whole call takes 102 us
// without dropout, 125 with it and 137 with twice the generator's work, which
// 16 bits instead of 8 a probability would need.  Columns of 330 nodes (about
// 165 rows on 149 visible keys) spend most of their 49 us on the way in and
// out, 13 % on products.  One query in each of 16 columns of up to 20,011 keys
// reads k and v at 5.4 TB/s in 168 us.
//
// One buffer: the next tiles come to registers during the products, and the
// other waves of the SIMD (four up to 64 wide, two above) fill the wait for
// them to reach LDS.  Scores formed 32 keys ahead, in two buffers, took 71
// against 62 us for 256 columns of 330 nodes, and the same time at 128 wide.
// Above 64 wide a tile has 64 keys: 545 against 557 us with 32, 611 with 128.
template <typename T, int NS, int OW, int CW, int KS, bool DROP>
__global__ __launch_bounds__(64 * OW * CW, NS <= 4 && OW > 1 ? 4 : 2) void cross_forward_kernel(CrossParams p) {
    constexpr int NT = 64 * OW * CW, KT = 32 * KS * CW, ND = (NS + 1) / 2;
    typedef RowTile<NS> KTile;
    typedef ColumnTile<NS> VTile;
    constexpr int kTileK = KT * KTile::kRowBytes, kTileV = KT * VTile::kRowBytes;
    constexpr int kLds = max_of(kTileK + kTileV, CW > 1 ? OW * ND * 4096 : 0);
    __shared__ __attribute__((aligned(16))) char lds[kLds];
    __shared__ __attribute__((aligned(16))) float start[KT];
    __shared__ uint32_t any;
    __shared__ float stat[2][OW * CW * 32];
    char *const lds_v = lds + kTileK;
    const int hk = (int)(blockIdx.x % (uint32_t)p.heads_kv);
    const CrossItem it = p.items[blockIdx.x / (uint32_t)p.heads_kv];
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int ow = wave % OW, cw = wave / OW;
    const int own = ow * 32 + col;
    const bool valid = own < it.n_own;
    const int r = valid ? it.own0 + own : it.own0;
    const int64_t row = row_id(p, it.q0, r, hk);
    KeyStage<T, NS, KT, NT> sk(p.k, p, it, hk), sv(p.v, p, it, hk);
    SeenStage<KT> ss(p, it);
    if (threadIdx.x == 0) any = 0;
    sk.template load<true>();
    sv.template load<false>();
    ss.load();
    typename Vec<T>::x8 qf[NS];
    load_own<T, NS>(qf, (const T *)p.q.p + row_at(p.q, it.q0, r, p.group, hk), valid, half, p.dim);
    const bool works = ow * 32 < it.n_own;  // waves without rows only help to load
    f32x16 o[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) o[dt] = 0.0f;
    // exponents are taken from `from` (in powers of two); a row that has seen
    // nothing yet has limit -inf
    float from = 0.0f, limit = -kInf, sum = 0.0f;
    const float c = p.scale * kLog2e;

    auto scores = [&](int ks, bool partial) {
        f32x16 s;
        const int base = (cw * KS + ks) * 32;
        const typename Vec<T>::x8 k0 = read_rows<T, KTile>(lds, base + col, half);
        if (partial)
            s = mfma(k0, qf[0], start_of(start + base, half));
        else
            s = mfma(k0, qf[0], f32x16(0.0f));
#pragma unroll
        for (int t = 1; t < NS; ++t) s = mfma(read_rows<T, KTile>(lds, base + col, 2 * t + half), qf[t], s);
        return s;
    };
    // Scores to exponents.  What they are taken from follows the running
    // maximum only when that has grown by more than 2^8: until then the
    // probabilities stay within 2^8 of kStart's power, in range for either
    // type, and the accumulators need no rescaling.
    constexpr float kStart = kUpBits<T> / 2, kLimit = 8.0f + kStart;
    auto exponents = [&](f32x16 &s) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = __builtin_fmaf(s[e], c, -from);
        float mx = s[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
        mx = both_max(mx);
        if (__any(mx > limit)) {
            const bool up = mx > limit;
            const float by = up ? mx - kStart : 0.0f;
            const float f = limit == kLimit ? __builtin_amdgcn_exp2f(-by) : 1.0f;  // before: sums are zero
            sum *= f;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) o[dt] *= f;
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] -= by;
            from += by;
            limit = up ? kLimit : limit;
        }
    };
    auto weigh = [&](f32x16 &s, int key, int ks) {
        float part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            s[e] = __builtin_amdgcn_exp2f(s[e]);
            part[e & 3] += s[e];
        }
        sum += (part[0] + part[1]) + (part[2] + part[3]);
        dev::Philox4 w;
        if (DROP) w = keep_words(p, row, (key + (cw * KS + ks) * 32) >> 5, half);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            union {
                typename Vec<T>::x8 v;
                uint32_t w[4];
            } pf;
            pf.v = round8<T>(s, 8 * t);
            if (DROP)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t m[2];
                    keep_pairs(w.w[2 * t + i], p.drop_below, m);
                    pf.w[2 * i] &= m[0];
                    pf.w[2 * i + 1] &= m[1];
                }
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
                o[dt] = mfma(read_columns<T, VTile>(lds_v, (cw * KS + ks) * 32 + 16 * t, dt, lane), pf.v, o[dt]);
        }
    };
    if (it.beg < it.end) {
        __syncthreads();
        sk.template store<KTile>(lds, sk);
        sv.template store<VTile>(lds_v, sk);
        ss.store(start, &any);
        __syncthreads();
        for (int key = it.beg; key < it.end; key += KT) {
            sk.template load<true>();
            sv.template load<false>();
            ss.load();
            const bool partial = p.key_mask || key + KT > it.end;
            if (works)
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    f32x16 s = scores(ks, partial);
                    exponents(s);
                    weigh(s, key, ks);
                }
            __syncthreads();
            sk.template store<KTile>(lds, sk);
            sv.template store<VTile>(lds_v, sk);
            ss.store(start, &any);
            __syncthreads();
        }
        if (!any) {  // whatever the queries hold, nothing was seen
            limit = -kInf;
            sum = 0.0f;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) o[dt] = 0.0f;
        }
    }
    sum = both_sum(sum);
    float top = limit == kLimit ? from : -kInf;
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
            total += stat[1][(ow * CW + w) * 32 + col] * __builtin_amdgcn_exp2f(stat[0][(ow * CW + w) * 32 + col] - to);
        const float f = __builtin_amdgcn_exp2f(top - to);
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
        p.lse[row] = sum == 0.0f ? -kInf : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

// Joins the parts of split rows: a block per tile, key head and kJoinOwners
// rows.  The parts' weights are formed once per row, then the loads of several
// parts are in flight together.
template <typename T>
__global__ __launch_bounds__(256) void cross_join_forward_kernel(CrossParams p, const CrossJoin *joins) {
    __shared__ float weight[kJoinOwners][kMaxParts], gain[kJoinOwners];
    const CrossJoin j = joins[blockIdx.x];
    const int hk = blockIdx.y, tile = kJoinOwners * gridDim.z, first = kJoinOwners * blockIdx.z;
    const int rows = min(kJoinOwners, j.n_own - first);
    {
        const int own = threadIdx.x / 32, l = threadIdx.x % 32;
        float top[kMaxParts / 32], sum[kMaxParts / 32], mx = -kInf;
#pragma unroll
        for (int k = 0; k < kMaxParts / 32; ++k) {
            const int s = l + 32 * k;
            top[k] = -kInf;
            sum[k] = 0.0f;
            if (own < rows && s < j.n_parts) {
                const int64_t at = ((int64_t)(j.slot + s) * p.heads_kv + hk) * tile + first + own;
                top[k] = p.part_ml[2 * at];
                sum[k] = p.part_ml[2 * at + 1];
            }
            mx = fmaxf(mx, top[k]);
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d, 32));
        const float to = mx == -kInf ? 0.0f : mx;
        float total = 0.0f;
#pragma unroll
        for (int k = 0; k < kMaxParts / 32; ++k) {
            const float f = __builtin_amdgcn_exp2f(top[k] - to);
            if (own < kJoinOwners && l + 32 * k < j.n_parts) weight[own][l + 32 * k] = f;
            total += f * sum[k];
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) total += __shfl_xor(total, d, 32);
        if (own < rows && l == 0) {
            gain[own] = total > 0.0f ? p.keep_gain / total : (total == 0.0f ? 0.0f : total);
            if (p.lse)
                p.lse[row_id(p, j.q0, j.own0 + first + own, hk)] =
                    total == 0.0f ? -kInf : (mx + __builtin_amdgcn_logf(total)) * kLn2;
        }
    }
    __syncthreads();
    const int quads = p.dim / 4;
    for (int idx = threadIdx.x; idx < rows * quads; idx += blockDim.x) {
        const int own = idx / quads, d = (idx - own * quads) * 4;
        const int64_t step = (int64_t)p.heads_kv * tile * p.dim;
        const float *src = p.part + (((int64_t)j.slot * p.heads_kv + hk) * tile + first + own) * p.dim + d;
        f32x4 acc = 0.0f;
#pragma unroll 8
        for (int s = 0; s < j.n_parts; ++s) acc += *(const f32x4 *)(src + s * step) * weight[own][s];
        typename Vec<T>::x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (T)(acc[i] * gain[own]);
        *(typename Vec<T>::x4 *)((T *)p.out + row_id(p, j.q0, j.own0 + first + own, hk) * p.dim + d) = w;
    }
}

struct Pass {
    static constexpr bool kForward = true;
    template <typename T, int NS, int OW, int CW, bool DROP>
    static void run(const CrossParams &p, hipStream_t s) {
        cross_forward_kernel<T, NS, OW, CW, (OW >= 4 && NS > 4 ? 2 : 1), DROP><<<dim3(grid_of(p)), 64 * OW * CW, 0, s>>>(p);
    }
    template <typename T>
    static void join(const CrossParams &p, const CrossPass &w, dim3 grid, hipStream_t s) {
        cross_join_forward_kernel<T><<<grid, 256, 0, s>>>(p, w.joins);
    }
};

}  // namespace

hipError_t launch_cross_forward(const CrossParams &p, const CrossPass &w, int dtype, hipStream_t s) {
    return cross::launch_pass<Pass>(p, w, dtype, s);
}

}  // namespace same
