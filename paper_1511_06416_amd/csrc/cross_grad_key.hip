// Cross attention: the gradients of keys and values (gfx950).
#include "cross_join.hpp"

namespace same {
namespace {

using namespace cross;

// Waves a SIMD: as many as leave every value a register, for spilled ones cost
// more than the waves bring.
constexpr int key_waves(int ns, int cw, bool drop) {
    if (ns > 4 && cw > 1) return 1;
    return ns == 2 ? 3 : ns == 8 && drop ? 1 : 2;
}

// -------------------------------------------------------- gradient: dK and dV
//
// The mirror image: a wave owns 32 keys of a key head (a lane one key) and
// walks the query rows of every head that shares it, so that the sum over
// those heads stays in its accumulators.  S = Q K^T (rows x keys),
// dV^T += dO^T (D P), dK^T += Q^T dS.  D P (in fp16 times 2^14) and dS are
// rounded to 16 bits as operands, the sums are fp32 and in a fixed order: no
// atomics.
//
// Two accumulators of the head's width a wave leave room for two waves a SIMD
// (LDS for one where four waves share 32 wide keys).  4,099 rows on 4,095 keys,
// 16 heads on 4 of 128: 284 us, the matrix units busy 40 % of it, LDS 35, the vector
// units 31 (with dropout, one wave a SIMD, some 600 us); 128 columns of 330 nodes, 8 heads
// of 64 with dropout: 49 us, of
// some 38,000 cycles of a wave 9,000 before its first product, 3,500 after its
// last and 3,300 to 4,600 for each 32 rows.
template <typename T, int NS, int OW, int CW, bool DROP>
__global__ __launch_bounds__(64 * OW * CW, key_waves(NS, CW, DROP)) void cross_dkv_kernel(CrossParams p) {
    constexpr int NT = 64 * OW * CW, QT = 32 * CW, ND = (NS + 1) / 2;
    typedef BothTile<NS> Tile;
    constexpr int kTile = QT * Tile::kRowBytes;
    constexpr int kBufs = CW > 1 ? 1 : 2;
    // Wide heads: a wave's own rows of v stay in LDS, for the registers that
    // its two accumulators and its rows of k leave do not hold them.
    constexpr bool kOwnLds = NS > 4;
    typedef RowTile<NS> OwnTile;
    constexpr int kOwn = kOwnLds ? 32 * OW * CW * OwnTile::kRowBytes : 0;
    constexpr int kLds = max_of(2 * kTile * kBufs + kOwn, CW > 1 ? OW * ND * 4096 : 0);
    __shared__ __attribute__((aligned(256))) char lds[kLds];
    __shared__ f32x4 stat[kBufs][2][QT / 4];
    __shared__ int64_t stat_id[kBufs][DROP ? QT : 1];
    __shared__ __attribute__((aligned(256))) char turn_all[DROP ? OW * CW : 1][TurnTile::kBytes];
    const int hk = (int)(blockIdx.x % (uint32_t)p.heads_kv);
    const CrossItem it = p.items[blockIdx.x / (uint32_t)p.heads_kv];
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    char *const turn = turn_all[DROP ? wave : 0];
    const int ow = wave % OW, cw = wave / OW;
    const int own = ow * 32 + col;
    const bool valid = own < it.n_own;
    const int64_t tok = it.k0 + it.own0 + (valid ? own : 0);
    // every load of the prologue is under way before the first is waited for
    typename Vec<T>::x8 kf[NS], vf[NS];
    load_own<T, NS>(kf, (const T *)p.k.p + tok * p.k.row + (int64_t)hk * p.k.head, valid, half, p.dim);
    load_own<T, NS>(vf, (const T *)p.v.p + tok * p.v.row + (int64_t)hk * p.v.head, valid, half, p.dim);
    uint32_t byte = 1;
    if (p.key_mask) byte = p.key_mask[tok];
    QueryStage<T, NS, QT, NT> sq(p, it, hk);
    if (it.beg < it.end) sq.load(p);
    const bool visible = valid && byte != 0;
    if (p.key_mask)
#pragma unroll
        for (int t = 0; t < NS; ++t) {
            kf[t] = visible ? kf[t] : zero8<T>();
            vf[t] = visible ? vf[t] : zero8<T>();
        }
    char *const own_v = lds + 2 * kTile * kBufs + wave * 32 * OwnTile::kRowBytes;
    if (kOwnLds)
#pragma unroll
        for (int t = 0; t < NS; ++t) *(typename Vec<T>::x8 *)(own_v + OwnTile::at(col, 2 * t + half)) = vf[t];
    if (it.beg < it.end)
        sq.template store<Tile>(lds, lds + kTile, (float *)stat[0][0], (float *)stat[0][1],
                                DROP ? stat_id[0] : nullptr);
    f32x16 ok[ND], ov[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) ok[dt] = ov[dt] = 0.0f;
    const float c = p.scale * kLog2e;
    const float gain = DROP ? p.keep_gain : 1.0f;
    __syncthreads();
    BothReader<T, NS> rd(lds + cw * 32 * Tile::kRowBytes, lane);
    int buf = 0;
    for (int row = it.beg; row < it.end; row += QT) {
        sq.load(p);
        if (ow * 32 < it.n_own) {  // waves without keys only help to load
        const int base = cw * 32;
        constexpr uint32_t at_q = 0, at_g = kTile;
        rd.renew();
        f32x16 s = 0.0f, dp = 0.0f;
#pragma unroll
        for (int t = 0; t < NS; ++t) {
            s = mfma(rd.row(at_q, t), kf[t], s);
            dp = mfma(rd.row(at_g, t), kOwnLds ? read_rows<T, OwnTile>(own_v, col, 2 * t + half) : vf[t], dp);
        }
        // The keep numbers are made as in the other passes, a lane a row and 16
        // keys of it; as 16-bit masks they are turned in LDS like an operand,
        // so that a lane gets those of its key and accumulator rows.
        uint32_t mask[8];
        if (DROP) {
            const dev::Philox4 bits = keep_words(p, stat_id[buf][base + col], (it.own0 + ow * 32) >> 5, half);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                uint32_t m[2];
                keep_pairs(bits.w[g], p.drop_below, m);
                *TurnTile::row_piece(turn, lane, g) = m[0] | (uint64_t)m[1] << 32;
            }
            wave_sync();
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                union {
                    s16x4 h;
                    uint32_t w[2];
                } u;
                u.h = TurnTile::column_piece(turn, lane, g);
                mask[2 * g] = u.w[0];
                mask[2 * g + 1] = u.w[1];
            }
            wave_sync();
        }
        f32x16 w;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 l4 = stat[buf][0][(base + 8 * g + 4 * half) >> 2];
            const f32x4 d4 = stat[buf][1][(base + 8 * g + 4 * half) >> 2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = 4 * g + i;
                const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, -l4[i]));
                w[e] = x;
                if (DROP) {
                    const uint32_t m = (uint32_t)__builtin_amdgcn_sbfe((int)mask[e >> 1], 16 * (e & 1), 16);
                    w[e] = __uint_as_float(__float_as_uint(x) & m);
                    s[e] = __builtin_fmaf(w[e], dp[e], x * d4[i]);   // dS / gain
                } else {
                    s[e] = x * (dp[e] + d4[i]);
                }
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const typename Vec<T>::x8 wf = round8<T>(w, 8 * t, kUp<T>), df = round8<T>(s, 8 * t);
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) {
                ov[dt] = mfma(rd.column(at_g, t, dt), wf, ov[dt]);
                ok[dt] = mfma(rd.column(at_q, t, dt), df, ok[dt]);
            }
        }
        }
        if (kBufs == 1)
            __syncthreads();
        else {
            buf ^= 1;
            rd.move(buf ? 2 * kTile : -2 * kTile);
        }
        sq.template store<Tile>(lds + buf * 2 * kTile, lds + buf * 2 * kTile + kTile, (float *)stat[buf][0],
                                (float *)stat[buf][1], DROP ? stat_id[buf] : nullptr);
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
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) ov[dt] *= kDown<T>;
    if (it.slot >= 0) {
        const int64_t at = ((int64_t)it.slot * p.heads_kv + hk) * (32 * OW) + own;
        write_part<ND>(p.part + 2 * at * p.dim, ok, half, p.dim);
        write_part<ND>(p.part + (2 * at + 1) * p.dim, ov, half, p.dim);
        return;
    }
    const int64_t at = (tok * p.heads_kv + hk) * p.dim;
    write_owner<T, ND>((T *)p.dk + at, ok, p.scale * gain, half, p.dim);
    write_owner<T, ND>((T *)p.dv + at, ov, gain, half, p.dim);
}

struct Pass {
    static constexpr bool kForward = false;
    template <typename T, int NS, int OW, int CW, bool DROP>
    static void run(const CrossParams &p, hipStream_t s) {
        cross_dkv_kernel<T, NS, OW, CW, DROP><<<dim3(grid_of(p)), 64 * OW * CW, 0, s>>>(p);
    }
    template <typename T>
    static void join(const CrossParams &p, const CrossPass &w, dim3 grid, hipStream_t s) {
        cross_join_grad_kernel<T, 2><<<grid, 256, 0, s>>>(p, w.joins);
    }
};

}  // namespace

hipError_t launch_cross_dkv(const CrossParams &p, const CrossPass &w, int dtype, hipStream_t s) {
    return cross::launch_pass<Pass>(p, w, dtype, s);
}

}  // namespace same
