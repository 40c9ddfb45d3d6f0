// Cross attention: the gradient of the queries (gfx950).
#include "cross_join.hpp"

namespace same {
namespace {

using namespace cross;

// ------------------------------------------------------------- gradient: dQ
//
// A wave owns 32 query rows and walks the keys as the forward does:
// P = exp(S - lse), dP^T = V dO^T, dS = P (D dP - delta),
// dQ^T += K^T dS^T; delta = sum over the width of dO * O, kept for dK, dV
// divided by D's value, which every gradient takes at its end.  S and dP are
// formed again from the operands rather than kept: 4 products of width a pair
// against 2 x 4 bytes written and read.  dS is rounded to 16 bits as an
// operand; everything else is fp32.
//
// A row's q, dout and accumulators fill the registers of two waves a SIMD (one
// for four waves that share 32 wide rows, which would spill at two), so the
// tiles of k and v have two buffers and the loads of the next ones fly during
// the products.  4,099 rows on 4,095 keys, 16 heads on 4 of 128: 204 us, the
// matrix units busy 44 % of it, the vector units 35; 128 columns of 330 nodes, 8 heads
// of 64 with dropout: 38 us, of which most is the way in and out.
template <typename T, int NS, int OW, int CW, bool DROP>
__global__ __launch_bounds__(64 * OW * CW, CW > 1 && NS > 4 ? 1 : NS == 2 ? 3 : 2) void cross_dq_kernel(
    CrossParams p) {
    constexpr int NT = 64 * OW * CW, KT = 32 * CW, ND = (NS + 1) / 2;
    typedef BothTile<NS> KTile;
    typedef RowTile<NS> VTile;
    constexpr int kTileK = KT * KTile::kRowBytes, kTileV = KT * VTile::kRowBytes;
    constexpr int kBufs = CW > 1 ? 1 : 2;
    constexpr int kLds = max_of((kTileK + kTileV) * kBufs, CW > 1 ? OW * ND * 4096 : 0);
    __shared__ __attribute__((aligned(256))) char lds[kLds];
    __shared__ __attribute__((aligned(16))) float start[kBufs][KT];
    char *const lds_v = lds + kBufs * kTileK;
    const int hk = (int)(blockIdx.x % (uint32_t)p.heads_kv);
    const CrossItem it = p.items[blockIdx.x / (uint32_t)p.heads_kv];
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int ow = wave % OW, cw = wave / OW;
    const int own = ow * 32 + col;
    const bool valid = own < it.n_own;
    const int r = valid ? it.own0 + own : it.own0;
    const int64_t row = row_id(p, it.q0, r, hk);
    // every load of the prologue is under way before the first is waited for
    KeyStage<T, NS, KT, NT> sk(p.k, p, it, hk), sv(p.v, p, it, hk);
    SeenStage<KT> ss(p, it);
    if (it.beg < it.end) {
        sk.template load<true>();
        sv.template load<false>();
        ss.load();
    }
    typename Vec<T>::x8 qf[NS], gf[NS], of[NS];
    load_own<T, NS>(gf, (const T *)p.dout.p + row_at(p.dout, it.q0, r, p.group, hk), valid, half, p.dim);
    load_own<T, NS>(of, (const T *)p.out_in + row * p.dim, valid, half, p.dim);
    load_own<T, NS>(qf, (const T *)p.q.p + row_at(p.q, it.q0, r, p.group, hk), valid, half, p.dim);
    const float lse = valid ? p.lse[row] : -kInf;
    if (it.beg < it.end) {
        sk.template store<KTile>(lds, sk);
        sv.template store<VTile>(lds_v, sk);
        ss.store(start[0], nullptr);
    }
    float delta = 0.0f;
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) delta = __builtin_fmaf((float)of[s][i], (float)gf[s][i], delta);
    float rest = -both_sum(delta) * (DROP ? p.keep_part : 1.0f);
    // Up to 32 keys lie in one wave, which then forms delta from P and dP in fp32:
    // with so few keys out's rounding would cost dS a good part of its digits.
    const bool short_row = it.slot < 0 && it.end - it.beg <= 32;
    f32x16 o[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) o[dt] = 0.0f;
    const float c = p.scale * kLog2e;
    const float base2 = lse == -kInf ? kInf : lse * kLog2e;
    const float gain = DROP ? p.keep_gain : 1.0f;

    __syncthreads();
    BothReader<T, NS> rk(lds + cw * 32 * KTile::kRowBytes, lane);
    int buf = 0;
    for (int key = it.beg; key < it.end; key += KT) {
        sk.template load<true>();
        sv.template load<false>();
        ss.load();
        if (ow * 32 < it.n_own) {  // waves without rows only help to load
        const int base = cw * 32;
        constexpr uint32_t at_k = 0;
        const char *tv = lds_v + buf * kTileV;
        rk.renew();
        f32x16 s, dp = 0.0f;
        if (p.key_mask || key + KT > it.end)
            s = mfma(rk.row(at_k, 0), qf[0], start_of(start[buf] + base, half));
        else
            s = mfma(rk.row(at_k, 0), qf[0], f32x16(0.0f));
        dp = mfma(read_rows<T, VTile>(tv, base + col, half), gf[0], dp);
#pragma unroll
        for (int t = 1; t < NS; ++t) {
            s = mfma(rk.row(at_k, t), qf[t], s);
            dp = mfma(read_rows<T, VTile>(tv, base + col, 2 * t + half), gf[t], dp);
        }
        dev::Philox4 bits;
        if (DROP) bits = keep_words(p, row, (key + base) >> 5, half);
        // dS / gain = (keep P) dP - P delta / gain
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, -base2));
        f32x16 w = s;
        if (DROP)
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = kept(bits, e, p.drop_below) ? s[e] : 0.0f;
        if (short_row) {
            float d = 0.0f;
#pragma unroll
            for (int e = 0; e < 16; ++e) d = __builtin_fmaf(w[e], dp[e], d);
            rest = -both_sum(d);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = DROP ? __builtin_fmaf(s[e], rest, w[e] * dp[e]) : s[e] * (dp[e] + rest);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const typename Vec<T>::x8 df = round8<T>(s, 8 * t);
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) o[dt] = mfma(rk.column(at_k, t, dt), df, o[dt]);
        }
        }
        if (kBufs == 1)
            __syncthreads();
        else {
            buf ^= 1;
            rk.move(buf ? kTileK : -kTileK);
        }
        sk.template store<KTile>(lds + buf * kTileK, sk);
        sv.template store<VTile>(lds_v + buf * kTileV, sk);
        ss.store(start[buf], nullptr);
        __syncthreads();
    }
    if (valid && half == 0 && cw == 0 && it.beg == 0) p.delta[row] = -rest;
    if (CW > 1) {
        join_waves<ND, OW, CW>(o, lds, ow, cw, lane);
        if (cw != 0) return;
    }
    if (lse == -kInf)  // a row that sees nothing, whatever it holds
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) o[dt] = 0.0f;
    if (!valid) return;
    if (it.slot >= 0) {
        const int64_t at = ((int64_t)it.slot * p.heads_kv + hk) * (32 * OW) + own;
        write_part<ND>(p.part + at * p.dim, o, half, p.dim);
        return;
    }
    write_owner<T, ND>((T *)p.dq + row * p.dim, o, p.scale * gain, half, p.dim);
}

struct Pass {
    static constexpr bool kForward = false;
    template <typename T, int NS, int OW, int CW, bool DROP>
    static void run(const CrossParams &p, hipStream_t s) {
        cross_dq_kernel<T, NS, OW, CW, DROP><<<dim3(grid_of(p)), 64 * OW * CW, 0, s>>>(p);
    }
    template <typename T>
    static void join(const CrossParams &p, const CrossPass &w, dim3 grid, hipStream_t s) {
        cross_join_grad_kernel<T, 1><<<grid, 256, 0, s>>>(p, w.joins);
    }
};

}  // namespace

hipError_t launch_cross_dq(const CrossParams &p, const CrossPass &w, int dtype, hipStream_t s) {
    return cross::launch_pass<Pass>(p, w, dtype, s);
}

}  // namespace same
