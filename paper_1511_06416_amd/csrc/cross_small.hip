// Cross attention over columns of a few entries (gfx950): a wave takes as many
// neighbouring segments as fit 32 query rows and 32 keys.
#include "cross_common.hpp"

namespace same {
namespace {

using namespace cross;

// One 32 x 32 product of query rows and keys holds several segments as blocks
// on its diagonal: their tokens are neighbours in q and in k, and a row sees
// the keys [lo, hi) of its own segment only.  Nothing is left to loop over, so
// a row's statistics are complete at once, and the gradient needs one launch
// that forms P, dP and dS once and delta from them in fp32.  What bounds it is
// a wave's chain of loads, products and stores and the number of waves, which
// packing cuts: 2,000 columns of the five-node network, 4 heads of 32, from
// 7,700 waves to 710, the forward pass from 8.5 to 4.5 us and the gradients,
// in one launch instead of two, from 26 to 7 us.
constexpr int units(int ns) { return ns <= 4 ? 4 : 2; }  // waves of a block, each with an item of its own

template <int NS>
struct SmallLds {
    typedef ColumnTile<NS> Tile;
    static constexpr int kTile = 32 * Tile::kRowBytes;
    static constexpr int kTurn = TurnTile::kBytes;
};

struct SmallUnit {
    CrossSmallItem it;
    int hk, lane, half, col;
    bool row_in, key_in, key_seen;
    int64_t row, key;      // this lane's query row number and key token
    int lo, hi;            // keys of the row's segment
    uint32_t sees;         // those that are visible, one bit each
};

__device__ __forceinline__ bool small_unit(const CrossParams &p, int per_block, SmallUnit &u) {
    const uint32_t index = blockIdx.x * per_block + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (index >= (uint32_t)p.n_items * (uint32_t)p.heads_kv) return false;
    u.hk = (int)(index % (uint32_t)p.heads_kv);
    const CrossSmallItem *src = p.small + index / (uint32_t)p.heads_kv;
    u.it.q0 = src->q0;
    u.it.k0 = src->k0;
    u.it.n_rows = src->n_rows;
    u.it.n_keys = src->n_keys;
    u.lane = threadIdx.x & 63;
    u.half = u.lane >> 5;
    u.col = u.lane & 31;
    const uint32_t range = src->range[u.col];
    u.row_in = u.col < u.it.n_rows;
    u.key_in = u.key_seen = u.col < u.it.n_keys;
    u.row = row_id(p, u.it.q0, u.row_in ? u.col : 0, u.hk);
    u.key = u.it.k0 + (u.key_in ? u.col : 0);
    u.lo = (int)(range & 255u);
    u.hi = (int)(range >> 8);
    u.sees = (uint32_t)((1ull << u.hi) - (1ull << u.lo));
    return true;
}

// Rows (or keys) of the unit, a lane one row, chunks 2 t + half.
template <typename T, int NS>
__device__ __forceinline__ void load_rows(typename Vec<T>::x8 (&f)[NS], const CrossParams &p, const CrossTensor &t,
                                          const SmallUnit &u) {
    load_own<T, NS>(f, (const T *)t.p + row_at(t, u.it.q0, u.row_in ? u.col : 0, p.group, u.hk), u.row_in, u.half,
                    p.dim);
}
template <typename T, int NS>
__device__ __forceinline__ void load_key_rows(typename Vec<T>::x8 (&f)[NS], const CrossParams &p,
                                              const CrossTensor &t, const SmallUnit &u) {
    load_own<T, NS>(f, (const T *)t.p + u.key * t.row + (int64_t)u.hk * t.head, u.key_in, u.half, p.dim);
}
template <typename T, int NS>
__device__ __forceinline__ void to_tile(char *tile, const typename Vec<T>::x8 (&f)[NS], const SmallUnit &u) {
#pragma unroll
    for (int t = 0; t < NS; ++t) *(typename Vec<T>::x8 *)(tile + ColumnTile<NS>::at(u.col, 2 * t + u.half)) = f[t];
}

// Hidden keys become zeros and leave every row's view.
template <typename T, int NS>
__device__ __forceinline__ void hide_keys(const CrossParams &p, uint32_t byte, typename Vec<T>::x8 (&kf)[NS],
                                          typename Vec<T>::x8 (&vf)[NS], SmallUnit &u) {
    if (!p.key_mask) return;
    u.key_seen = u.key_in && byte != 0;
    u.sees &= (uint32_t)__ballot(u.key_seen);
#pragma unroll
    for (int t = 0; t < NS; ++t) {
        kf[t] = u.key_seen ? kf[t] : zero8<T>();
        vf[t] = u.key_seen ? vf[t] : zero8<T>();
    }
}

// Keep flags of the row's keys at their places in the tile, one bit each.  A
// half of the row's lanes makes the flags of half of its 32 keys.
__device__ __forceinline__ uint32_t keep_of(const CrossParams &p, const SmallUnit &u) {
    const dev::Philox4 w = keep_words(p, u.row, 0, u.half);
    const uint32_t t = p.drop_below * 0x01010101u, tops = 0x80808080u;
    uint32_t bits = 0;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const uint32_t low = (w.w[g] | tops) - (t & ~tops);
        const uint32_t ge = __builtin_amdgcn_bitop3_b32(w.w[g], low, t, 0xD4) >> 7 & 0x01010101u;
        bits |= (ge * 0x01020408u >> 24 & 15u) << (8 * g);  // the four flags side by side
    }
    bits <<= 4 * u.half;
    const auto both = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);
    return (both[0] | both[1]) << (u.lo & 31);
}

template <typename T, int NS>
__device__ __forceinline__ f32x16 product(const typename Vec<T>::x8 (&a)[NS], const typename Vec<T>::x8 (&b)[NS]) {
    f32x16 s = 0.0f;
#pragma unroll
    for (int t = 0; t < NS; ++t) s = mfma(a[t], b[t], s);
    return s;
}

// o[columns of the tile x lanes] = tile^T b, b in accumulator order.
template <typename T, int NS, int ND>
__device__ __forceinline__ void times_columns(f32x16 (&o)[ND], const char *tile,
                                              const typename Vec<T>::x8 (&b)[2], int lane) {
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) {
        o[dt] = 0.0f;
#pragma unroll
        for (int t = 0; t < 2; ++t) o[dt] = mfma(read_columns<T, ColumnTile<NS>>(tile, 16 * t, dt, lane), b[t], o[dt]);
    }
}

// Infinities or NaN among a wave's rows.
template <typename T, int NS>
__device__ __forceinline__ bool any_infinite(const typename Vec<T>::x8 (&f)[NS]) {
    // all exponent bits set: one more carries into the sign's place
    constexpr bool kBf16 = __is_same(T, __bf16);
    constexpr uint32_t kExp = kBf16 ? 0x7F807F80u : 0x7C007C00u, kOne = kBf16 ? 0x00800080u : 0x04000400u;
    uint32_t found = 0;
#pragma unroll
    for (int t = 0; t < NS; ++t) {
        union {
            typename Vec<T>::x8 v;
            uint32_t w[4];
        } x;
        x.v = f[t];
#pragma unroll
        for (int i = 0; i < 4; ++i) found |= (x.w[i] & kExp) + kOne;
    }
    return __any((found & 0x80008000u) != 0);
}

// The same with the rows f, which become the tile; KEYS: they are keys and the
// lanes query rows, else the other way round.  The weights of other segments
// are zero, but zero times an infinity is not: rows that hold one are
// multiplied segment by segment.
template <typename T, int NS, int ND, bool KEYS>
__device__ __forceinline__ void times_rows(f32x16 (&o)[ND], char *tile, const typename Vec<T>::x8 (&f)[NS],
                                           const typename Vec<T>::x8 (&b)[2], const SmallUnit &u) {
    if (!any_infinite<T, NS>(f)) {
        to_tile<T, NS>(tile, f, u);
        wave_sync();
        times_columns<T, NS, ND>(o, tile, b, u.lane);
        wave_sync();
        return;
    }
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) o[dt] = 0.0f;
    uint32_t rows = (uint32_t)__ballot(u.row_in && u.hi > u.lo);
    while (rows) {
        const int r = __builtin_ctz(rows);
        const int lo = __builtin_amdgcn_readlane(u.lo, r), hi = __builtin_amdgcn_readlane(u.hi, r);
        const uint32_t own_rows = (uint32_t)__ballot(u.row_in && u.lo == lo && u.hi == hi);
        const uint32_t own_keys = (uint32_t)((1ull << hi) - (1ull << lo));
        const bool tile_in = ((KEYS ? own_keys : own_rows) >> u.col) & 1;
        const bool lane_in = ((KEYS ? own_rows : own_keys) >> u.col) & 1;
        typename Vec<T>::x8 g[NS];
#pragma unroll
        for (int t = 0; t < NS; ++t) g[t] = tile_in ? f[t] : zero8<T>();
        to_tile<T, NS>(tile, g, u);
        wave_sync();
        f32x16 part[ND];
        times_columns<T, NS, ND>(part, tile, b, u.lane);
        wave_sync();
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[dt][e] = lane_in ? part[dt][e] : o[dt][e];
        rows &= ~own_rows;
    }
}

// A tile of numbers, times `up` and rounded, from lanes that hold rows to
// lanes that hold keys.
template <typename T>
__device__ __forceinline__ void turn(char *tile, const f32x16 &s, float up, typename Vec<T>::x8 (&out)[2],
                                     const SmallUnit &u) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        union {
            typename Vec<T>::x4 v;
            uint64_t w;
        } x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x.v[i] = (T)(s[4 * g + i] * up);
        *TurnTile::row_piece(tile, u.lane, g) = x.w;
    }
    wave_sync();
    union {
        s16x4 h[4];
        typename Vec<T>::x8 v[2];
    } r;
#pragma unroll
    for (int g = 0; g < 4; ++g) r.h[g] = TurnTile::column_piece(tile, u.lane, g);
    out[0] = r.v[0];
    out[1] = r.v[1];
    wave_sync();
}

template <typename T, int NS, bool DROP>
__global__ __launch_bounds__(64 * units(NS), NS <= 4 ? 4 : 2) void cross_small_forward_kernel(CrossParams p) {
    constexpr int ND = (NS + 1) / 2;
    typedef SmallLds<NS> L;
    __shared__ __attribute__((aligned(16))) char lds_all[units(NS)][L::kTile];
    SmallUnit u;
    if (!small_unit(p, units(NS), u)) return;
    char *const lds = lds_all[threadIdx.x >> 6];
    typename Vec<T>::x8 qf[NS], kf[NS], vf[NS];
    load_key_rows<T, NS>(kf, p, p.k, u);
    load_key_rows<T, NS>(vf, p, p.v, u);
    load_rows<T, NS>(qf, p, p.q, u);
    uint32_t byte = 1;
    if (p.key_mask) byte = u.key_in ? p.key_mask[u.key] : 0;
    hide_keys<T, NS>(p, byte, kf, vf, u);
    f32x16 s = product<T, NS>(kf, qf);
    hide(s, u.sees, u.half, -kInf);
    float top = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(top, s[e]);
    top = both_max(top);
    // exponents are at most kUpBits, and that exactly for the largest score
    // however large it is: the sum carries kUp too
    const float c = p.scale * kLog2e, from = top == -kInf ? 0.0f : top;
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        s[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e] - from, c, (float)kUpBits<T>));
        sum += s[e];
    }
    sum = both_sum(sum);
    if (DROP) hide(s, keep_of(p, u), u.half, 0.0f);
    const typename Vec<T>::x8 pf[2] = {round8<T>(s, 0), round8<T>(s, 8)};
    f32x16 o[ND];
    times_rows<T, NS, ND, true>(o, lds, vf, pf, u);
    if (!u.row_in) return;
    write_owner<T, ND>((T *)p.out + u.row * p.dim, o,
                       sum > 0.0f ? (DROP ? p.keep_gain : 1.0f) / sum : (sum == 0.0f ? 0.0f : sum), u.half, p.dim);
    if (p.lse && u.half == 0) p.lse[u.row] = sum == 0.0f ? -kInf : top * p.scale + __builtin_amdgcn_logf(sum * kDown<T>) * kLn2;
}

template <int ND>
__device__ __forceinline__ void zero_unless(bool keep, f32x16 (&o)[ND]) {
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[dt][e] = keep ? o[dt][e] : 0.0f;
}

template <typename T, int NS, bool DROP>
__global__ __launch_bounds__(64 * units(NS), NS < 8 ? 2 : 1) void cross_small_grad_kernel(CrossParams p) {
    constexpr int ND = (NS + 1) / 2;
    typedef SmallLds<NS> L;
    __shared__ __attribute__((aligned(16))) char lds_all[units(NS)][L::kTile + L::kTurn];
    SmallUnit u;
    if (!small_unit(p, units(NS), u)) return;
    char *const lds = lds_all[threadIdx.x >> 6], *const lds_turn = lds + L::kTile;
    typename Vec<T>::x8 qf[NS], gf[NS], kf[NS], vf[NS];
    load_key_rows<T, NS>(kf, p, p.k, u);
    load_key_rows<T, NS>(vf, p, p.v, u);
    load_rows<T, NS>(qf, p, p.q, u);
    load_rows<T, NS>(gf, p, p.dout, u);
    const float lse = u.row_in ? p.lse[u.row] : -kInf;
    uint32_t byte = 1;
    if (p.key_mask) byte = u.key_in ? p.key_mask[u.key] : 0;
    hide_keys<T, NS>(p, byte, kf, vf, u);
    f32x16 s = product<T, NS>(kf, qf), dp = product<T, NS>(vf, gf);
    hide(s, u.sees, u.half, -kInf);
    // what a row's gradient holds against keys that it does not see stays out of every sum
    hide(dp, u.sees, u.half, 0.0f);
    const float c = p.scale * kLog2e, base2 = lse == -kInf ? kInf : lse * kLog2e;
    const float gain = DROP ? p.keep_gain : 1.0f;
    f32x16 w;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, -base2));
    hide(s, u.sees, u.half, 0.0f);
    w = s;
    if (DROP) hide(w, keep_of(p, u), u.half, 0.0f);
    // divided by D's value, as in the passes over long axes
    float delta = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) delta = __builtin_fmaf(w[e], dp[e], delta);
    const float rest = -both_sum(delta);
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = __builtin_fmaf(s[e], rest, w[e] * dp[e]);
    hide(s, u.sees, u.half, 0.0f);
    f32x16 o[ND];
    {
        const typename Vec<T>::x8 df[2] = {round8<T>(s, 0), round8<T>(s, 8)};
        times_rows<T, NS, ND, true>(o, lds, kf, df, u);
        if (u.row_in) write_owner<T, ND>((T *)p.dq + u.row * p.dim, o, p.scale * gain, u.half, p.dim);
    }
    typename Vec<T>::x8 f[2];
    const int64_t at = (u.key * p.heads_kv + u.hk) * p.dim;
    turn<T>(lds_turn, w, kUp<T>, f, u);
    times_rows<T, NS, ND, false>(o, lds, gf, f, u);
    // whatever the queries hold, a hidden key's gradients are zero
    zero_unless<ND>(u.key_seen, o);
    if (u.key_in) write_owner<T, ND>((T *)p.dv + at, o, gain * kDown<T>, u.half, p.dim);
    turn<T>(lds_turn, s, 1.0f, f, u);
    times_rows<T, NS, ND, false>(o, lds, qf, f, u);
    zero_unless<ND>(u.key_seen, o);
    if (u.key_in) write_owner<T, ND>((T *)p.dk + at, o, p.scale * gain, u.half, p.dim);
}

template <typename T, int NS, bool GRAD>
void launch(const CrossParams &p, hipStream_t s) {
    const uint32_t n = (uint32_t)p.n_items * (uint32_t)p.heads_kv;
    const dim3 grid((n + units(NS) - 1) / units(NS)), block(64 * units(NS));
    if (GRAD)
        p.drop_below ? cross_small_grad_kernel<T, NS, true><<<grid, block, 0, s>>>(p)
                     : cross_small_grad_kernel<T, NS, false><<<grid, block, 0, s>>>(p);
    else
        p.drop_below ? cross_small_forward_kernel<T, NS, true><<<grid, block, 0, s>>>(p)
                     : cross_small_forward_kernel<T, NS, false><<<grid, block, 0, s>>>(p);
}

template <typename T, bool GRAD>
void launch_width(const CrossParams &p, hipStream_t s) {
    if (p.dim <= 32)
        launch<T, 2, GRAD>(p, s);
    else if (p.dim <= 64)
        launch<T, 4, GRAD>(p, s);
    else if (p.dim <= 96)
        launch<T, 6, GRAD>(p, s);
    else
        launch<T, 8, GRAD>(p, s);
}

}  // namespace

hipError_t launch_cross_small(const CrossParams &all, bool grad, int dtype, hipStream_t s) {
    const int32_t per = items_per_launch(all.heads_kv);
    for (int64_t first = 0; first < all.n_items; first += per) {
        CrossParams p = all;
        p.small = all.small + first;
        p.n_items = (int32_t)std::min<int64_t>(per, all.n_items - first);
        if (dtype == kCrossBf16)
            grad ? launch_width<__bf16, true>(p, s) : launch_width<__bf16, false>(p, s);
        else
            grad ? launch_width<_Float16, true>(p, s) : launch_width<_Float16, false>(p, s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace same
