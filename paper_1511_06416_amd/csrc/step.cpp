// C ABI of a training step's operators (declared in include/same.h): norms of
// queries and keys with the position rotation, log probabilities of given
// states, and orthogonalised updates.  Argument checks, workspaces and the
// launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <exception>
#include <limits>
#include <new>

#include "checks.hpp"
#include "step.hpp"

namespace {

using same::align_up;
using same::aligned;
using same::check_apart;
using same::check_hip;
using same::extent;
using same::Extent;
using same::kAlign;
using same::overlap;
using same::record_error;

int check_dtype(int32_t dtype, int64_t *size) {
    if (dtype != SAME_F32 && dtype != SAME_F16 && dtype != SAME_BF16)
        return record_error(SAME_EINVAL, "dtype must be SAME_F32, SAME_F16 or SAME_BF16");
    *size = dtype == SAME_F32 ? 4 : 2;
    return SAME_OK;
}

// Runs an entry's body; nothing may leave a C entry.
template <typename F>
int guarded(F body) {
    try {
        return body();
    } catch (const std::bad_alloc &) {
        return record_error(SAME_ENOMEM, "out of host memory");
    } catch (const std::exception &e) {
        return record_error(SAME_EINVAL, e.what());
    }
}

// ---- norms of queries and keys

struct Heads {
    const char *name;
    const void *x;
    int64_t row, head, tokens;
    int32_t heads;
    const float *weight;
    const int32_t *positions;
};

constexpr double kMaxAngle = (double)((int64_t)1 << 40);

// An angle in turns, less the whole ones, which no whole position notices: of what is
// left a position of 2^31 asks for all 64 bits.  2 pi is taken off in three parts, of
// which the first two have 23 bits, so that their products with up to 2^38 turns are
// exact.
long double turn_of_angle(double angle) {
    const long double turns = 1.0L / 6.283185307179586476925286766559L;
    if (std::fabs(angle) <= 3.0) return (long double)angle * turns;   // none whole
    const long double whole = std::rint((long double)angle * turns);
    const long double rest =
        (((long double)angle - whole * 0x6.487EDp0L) - whole * 0x5.110B4p-24L) - whole * 0x6.11A62633145C06E0Ep-48L;
    return rest * turns;
}

int check_heads(const std::string &name, const void *p, int64_t row, int64_t head, int64_t tokens, int64_t heads,
                int64_t dim, int64_t size, std::vector<Extent> &reads) {
    if (tokens == 0) return SAME_OK;
    if (!p) return record_error(SAME_EINVAL, name + " is null");
    if (row < 0 || head < 0) return record_error(SAME_EINVAL, name + ": strides must not be negative");
    if (!aligned(p, 16) || row % 8 != 0 || head % 8 != 0)
        return record_error(SAME_EALIGN, name + " must be 16-byte aligned, with strides that are multiples of 8");
    const double last = (double)(tokens - 1) * (double)row + (double)(heads - 1) * (double)head + (double)dim;
    if (last >= 1e18) return record_error(SAME_ESIZE, name + ": strides pass 10^18 elements");
    reads.push_back(extent(p, size * ((tokens - 1) * row + (heads - 1) * head + dim)));
    return SAME_OK;
}

// What both directions share.
int check_norm(int32_t dtype, int32_t dim, const Heads &q, const Heads &k, double eps, int32_t rot_dim,
               const double *angles, same::NormParams &p, int64_t *size, std::vector<Extent> &reads) {
    int rc = check_dtype(dtype, size);
    if (rc) return rc;
    if (dim < 8 || dim > same::kMaxHeadDim || dim % 8 != 0)
        return record_error(SAME_EINVAL, "head_dim must be a multiple of 8 in [8, 128]");
    if (!((float)eps >= std::numeric_limits<float>::min()) || !std::isfinite((float)eps))
        return record_error(SAME_EINVAL, "eps must be a positive normal number in 32 bits");
    if (rot_dim < 0 || rot_dim > dim || rot_dim % 2 != 0)
        return record_error(SAME_EINVAL, "rot_dim must be even, in [0, head_dim]");
    if (rot_dim && !angles) return record_error(SAME_EINVAL, "angles is null");
    std::memset((void *)&p, 0, sizeof(p));
    for (int i = 0; i < rot_dim / 2; ++i) {
        if (!(std::fabs(angles[i]) <= kMaxAngle)) return record_error(SAME_EINVAL, "angles must lie within 2^40");
        const long double t = turn_of_angle(angles[i]);
        p.turn[i] = (double)t;
        p.turn_low[i] = (double)(t - (long double)p.turn[i]);
    }
    p.dim = dim;
    p.half = rot_dim / 2;
    p.eps = (float)eps;
    p.inv_dim = 1.0f / (float)dim;
    const Heads *sides[2] = {&q, &k};
    for (int i = 0; i < 2; ++i) {
        const Heads &h = *sides[i];
        const std::string name = h.name;
        if (h.tokens < 0) return record_error(SAME_EINVAL, name + ": tokens must not be negative");
        if (h.heads < 1) return record_error(SAME_EINVAL, name + ": heads must be positive");
        if (h.heads > 65536) return record_error(SAME_ESIZE, name + ": heads must be at most 65536");
        if (h.tokens >= (int64_t)1 << 40) return record_error(SAME_ESIZE, name + ": tokens must stay below 2^40");
        rc = check_heads(name, h.x, h.row, h.head, h.tokens, h.heads, dim, *size, reads);
        if (rc) return rc;
        if (!aligned(h.weight, 4) || !aligned(h.positions, 4))
            return record_error(SAME_EALIGN, name + "'s weight and positions must be 4-byte aligned");
        if (rot_dim && h.tokens && !h.positions) return record_error(SAME_EINVAL, name + "'s positions are null");
        if (h.weight) reads.push_back(extent(h.weight, 4 * (int64_t)dim));
        if (rot_dim && h.tokens) reads.push_back(extent(h.positions, 4 * h.tokens));
        same::NormSide &s = p.side[i];
        s.x = h.x;
        s.x_row = h.row;
        s.x_head = h.head;
        s.weight = h.weight;
        s.positions = h.positions;
        s.tokens = h.tokens;
        s.heads = h.heads;
    }
    return SAME_OK;
}

// A contiguous output, which may be the (contiguous) input `in` itself.
int check_result(const std::string &name, const void *out, const Heads &h, int64_t dim, int64_t size, const void *in,
                 int64_t row, int64_t head, std::vector<Extent> &writes, std::vector<Extent> &reads) {
    if (h.tokens == 0) return SAME_OK;
    if (!out) return record_error(SAME_EINVAL, name + " is null");
    if (!aligned(out, 16)) return record_error(SAME_EALIGN, name + " must be 16-byte aligned");
    const Extent e = extent(out, size * h.tokens * h.heads * dim);
    writes.push_back(e);
    if (out == in && (h.tokens == 1 || row == h.heads * dim) && (h.heads == 1 || head == dim))
        for (Extent &r : reads)
            if (r.lo == e.lo && r.hi == e.hi) {
                r = Extent();  // each row is read before it is written
                break;
            }
    return SAME_OK;
}

// ---- log probabilities

int check_logits(int32_t dtype, const char *name, const void *p, int64_t row, int64_t rows, int64_t cols, int64_t *size,
                 Extent *e) {
    int rc = check_dtype(dtype, size);
    if (rc) return rc;
    if (rows < 0 || cols < 0) return record_error(SAME_EINVAL, "rows and cols must not be negative");
    if (cols > (int64_t)1 << 21) return record_error(SAME_ESIZE, "cols must be at most 2^21");
    if (rows >= (int64_t)1 << 40) return record_error(SAME_ESIZE, "rows must stay below 2^40");
    if (rows == 0 || cols == 0) return SAME_OK;
    if (!p) return record_error(SAME_EINVAL, std::string(name) + " is null");
    if (!aligned(p, *size)) return record_error(SAME_EALIGN, std::string(name) + " must be aligned to its elements");
    if (row < 0) return record_error(SAME_EINVAL, "row strides must not be negative");
    if ((double)(rows - 1) * (double)row >= 1e18) return record_error(SAME_ESIZE, "row strides pass 10^18 elements");
    *e = extent(p, *size * ((rows - 1) * row + cols));
    return SAME_OK;
}

// Values a row (null: not there).
int add_rows(const char *name, const void *p, int64_t rows, int64_t bytes, size_t align, std::vector<Extent> &list) {
    if (!p || rows == 0) return SAME_OK;
    if (!aligned(p, align))
        return record_error(SAME_EALIGN, std::string(name) + " must be " + std::to_string(align) + "-byte aligned");
    list.push_back(extent(p, rows * bytes));
    return SAME_OK;
}

void log_probs_layout(int64_t rows, int64_t cols, int32_t n_top, int32_t *parts, int32_t *part_cols, size_t *stats,
                      size_t *bytes) {
    same::log_probs_parts(rows, cols, parts, part_cols);
    *stats = *bytes = 0;
    if (*parts > 1) {
        *stats = align_up((size_t)rows * *parts * sizeof(same::RowStats));
        *bytes = *stats + align_up((size_t)rows * *parts * n_top * sizeof(uint64_t));
    }
}

// ---- orthogonalised updates

struct OrthoLayout {
    int64_t n, m, np, mp, batch;
    size_t squares, wide, square, total;  // bytes of the sums and of one plane of each shape
    int32_t parts, part_cols;             // small updates: tiles of their parts, and of their factors
    size_t small_parts, small_factors;
    int32_t splits;                       // of the sums of X X^T, and their parts
    size_t gram_parts, x32;
};

int ortho_layout(int32_t dtype, int64_t n_mats, int64_t rows, int64_t cols, OrthoLayout &l) {
    int64_t size;
    int rc = check_dtype(dtype, &size);
    if (rc) return rc;
    if (n_mats < 0 || rows < 0 || cols < 0)
        return record_error(SAME_EINVAL, "n_mats, rows and cols must not be negative");
    l.n = std::min(rows, cols);
    l.m = std::max(rows, cols);
    if (l.n > 1 << 15 || l.m > 1 << 24 || (double)rows * (double)cols > 1.1e9)
        return record_error(SAME_ESIZE, "a matrix has at most 2^15 by 2^24 and 1.1 10^9 elements");
    if (n_mats >= (int64_t)1 << 40 || (double)n_mats * (double)rows * (double)cols >= 1e15)
        return record_error(SAME_ESIZE, "the matrices pass 10^15 elements");
    if (l.n <= same::kSmallSide) {
        size_t tiles = 0;
        same::ortho_small_parts(l.n, l.m, &l.parts, &l.part_cols, &tiles);
        l.batch = l.n ? std::min<int64_t>(n_mats, ((int64_t)1 << (l.parts > 1 ? 15 : 22)) / l.parts) : 0;
        l.small_parts = l.parts > 1 ? align_up((size_t)l.batch * l.parts * tiles) : 0;
        l.small_factors = l.parts > 1 ? align_up((size_t)l.batch * tiles) : 0;
        l.total = l.small_parts + l.small_factors;
        return SAME_OK;
    }
    if (same::ortho_whole(l.n, l.m)) {  // nothing is kept outside the block
        l.batch = std::min<int64_t>(n_mats, (int64_t)1 << 21);
        l.total = 0;
        return SAME_OK;
    }
    if (same::ortho_columns(l.n, l.m)) {
        size_t x, part, plane;
        same::ortho_columns_layout(l.n, l.m, &l.parts, &l.part_cols, &x, &part, &plane);
        // some 2^30 bytes of X
        l.batch = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(n_mats, 16384), ((int64_t)1 << 30) / (int64_t)x));
        if (n_mats == 0) l.batch = 0;
        l.squares = align_up((size_t)l.batch * same::kNormParts * sizeof(double));
        l.x32 = align_up((size_t)l.batch * x);
        l.gram_parts = align_up((size_t)l.batch * part);
        l.square = align_up((size_t)l.batch * plane);
        l.total = l.squares + l.x32 + l.gram_parts + 2 * l.square;
        return SAME_OK;
    }
    const int64_t pad = 32;  // a stage of the products
    l.np = (l.n + pad - 1) / pad * pad;
    l.mp = (l.m + pad - 1) / pad * pad;
    l.batch = l.n && n_mats ? same::orthogonalise_batch(n_mats, l.np, l.mp) : 0;
    l.squares = align_up((size_t)l.batch * same::kNormParts * sizeof(double));
    l.wide = align_up((size_t)l.batch * l.np * l.mp * 2);
    l.square = align_up((size_t)l.batch * l.np * l.np * 2);
    l.splits = same::orthogonalise_splits(l.np, l.mp);
    l.gram_parts = l.splits > 1 ? align_up((size_t)l.batch * l.splits * l.np * l.np * 4) : 0;
    l.total = l.squares + 6 * l.wide + 4 * l.square + l.gram_parts;
    return SAME_OK;
}

// The largest |x (a + b x^2 + c x^4)| of |x| <= bound.
double largest_of(const double *k, double bound) {
    const auto value = [&](double x) { return std::fabs(x * (k[0] + x * x * (k[1] + x * x * k[2]))); };
    double most = value(bound);
    const double A = 5.0 * k[2], B = 3.0 * k[1], C = k[0];  // the derivative in x^2
    double roots[2] = {-1.0, -1.0};
    if (A != 0.0) {
        const double d = B * B - 4.0 * A * C;
        if (d >= 0.0) {
            roots[0] = (-B + std::sqrt(d)) / (2.0 * A);
            roots[1] = (-B - std::sqrt(d)) / (2.0 * A);
        }
    } else if (B != 0.0) {
        roots[0] = -C / B;
    }
    for (double u : roots)
        if (u > 0.0 && u < bound * bound) most = std::max(most, value(std::sqrt(u)));
    return most;
}

// The largest power of two by which numbers up to `bound` stay in half of
// fp16's range, at most 2^most.
float plane_scale(double bound, int most) {
    return std::ldexp(1.0f, std::min(most, (int)std::floor(std::log2(32768.0 / bound))));
}

}  // namespace

extern "C" {

int same_qk_norm_workspace_size(int32_t head_dim, int64_t q_tokens, int32_t heads_q, int64_t k_tokens, int32_t heads_kv,
                                size_t *bytes) {
    if (!bytes) return record_error(SAME_EINVAL, "bytes is null");
    if (head_dim < 8 || head_dim > same::kMaxHeadDim || head_dim % 8 != 0)
        return record_error(SAME_EINVAL, "head_dim must be a multiple of 8 in [8, 128]");
    if (q_tokens < 0 || k_tokens < 0 || heads_q < 1 || heads_kv < 1)
        return record_error(SAME_EINVAL, "tokens must not be negative, heads must be positive");
    if (q_tokens >= (int64_t)1 << 40 || k_tokens >= (int64_t)1 << 40 || heads_q > 65536 || heads_kv > 65536)
        return record_error(SAME_ESIZE, "tokens must stay below 2^40, heads be at most 65536");
    int32_t of_q;
    *bytes = sizeof(float) * (size_t)head_dim *
             (size_t)same::qk_norm_grad_blocks(q_tokens * heads_q, k_tokens * heads_kv, head_dim, &of_q);
    return SAME_OK;
}

int same_qk_norm(int32_t dtype, int32_t head_dim, const void *q, int64_t q_row, int64_t q_head, int64_t q_tokens,
                 int32_t heads_q, const float *q_weight, const int32_t *q_positions, const void *k, int64_t k_row,
                 int64_t k_head, int64_t k_tokens, int32_t heads_kv, const float *k_weight, const int32_t *k_positions,
                 double eps, int32_t rot_dim, const double *angles, void *q_out, void *k_out, void *stream) {
    return guarded([&]() -> int {
        const Heads hq{"q", q, q_row, q_head, q_tokens, heads_q, q_weight, q_positions};
        const Heads hk{"k", k, k_row, k_head, k_tokens, heads_kv, k_weight, k_positions};
        same::NormParams p;
        std::vector<Extent> reads, writes;
        int64_t size;
        int rc = check_norm(dtype, head_dim, hq, hk, eps, rot_dim, angles, p, &size, reads);
        if (!rc) rc = check_result("q_out", q_out, hq, head_dim, size, q, q_row, q_head, writes, reads);
        if (!rc) rc = check_result("k_out", k_out, hk, head_dim, size, k, k_row, k_head, writes, reads);
        if (!rc) rc = check_apart(writes, reads);
        if (rc || q_tokens + k_tokens == 0) return rc;
        p.side[0].out = q_out;
        p.side[1].out = k_out;
        return check_hip(same::launch_qk_norm(p, dtype, false, (hipStream_t)stream), "norm launch");
    });
}

int same_qk_norm_backward(int32_t dtype, int32_t head_dim, const void *q, int64_t q_row, int64_t q_head,
                          int64_t q_tokens, int32_t heads_q, const float *q_weight, const int32_t *q_positions,
                          const void *k, int64_t k_row, int64_t k_head, int64_t k_tokens, int32_t heads_kv,
                          const float *k_weight, const int32_t *k_positions, double eps, int32_t rot_dim,
                          const double *angles, const void *dq_out, int64_t dq_out_row, int64_t dq_out_head,
                          const void *dk_out, int64_t dk_out_row, int64_t dk_out_head, void *dq, void *dk,
                          float *dq_weight, float *dk_weight, void *workspace, void *stream) {
    return guarded([&]() -> int {
        const Heads hq{"q", q, q_row, q_head, q_tokens, heads_q, q_weight, q_positions};
        const Heads hk{"k", k, k_row, k_head, k_tokens, heads_kv, k_weight, k_positions};
        same::NormParams p;
        std::vector<Extent> reads, writes;
        int64_t size;
        int rc = check_norm(dtype, head_dim, hq, hk, eps, rot_dim, angles, p, &size, reads);
        if (!rc) rc = check_heads("dq_out", dq_out, dq_out_row, dq_out_head, q_tokens, heads_q, head_dim, size, reads);
        if (!rc) rc = check_heads("dk_out", dk_out, dk_out_row, dk_out_head, k_tokens, heads_kv, head_dim, size, reads);
        if (!rc) rc = check_result("dq", dq, hq, head_dim, size, dq_out, dq_out_row, dq_out_head, writes, reads);
        if (!rc) rc = check_result("dk", dk, hk, head_dim, size, dk_out, dk_out_row, dk_out_head, writes, reads);
        if (rc) return rc;
        if (!aligned(dq_weight, 4) || !aligned(dk_weight, 4))
            return record_error(SAME_EALIGN, "dq_weight and dk_weight must be 4-byte aligned");
        if (dq_weight) writes.push_back(extent(dq_weight, 4 * (int64_t)head_dim));
        if (dk_weight) writes.push_back(extent(dk_weight, 4 * (int64_t)head_dim));
        int32_t of_q = 0;
        const int blocks = same::qk_norm_grad_blocks(q_tokens * heads_q, k_tokens * heads_kv, head_dim, &of_q);
        if (dq_weight || dk_weight) {
            if (blocks && !workspace) return record_error(SAME_EINVAL, "workspace is null");
            if (!aligned(workspace, kAlign)) return record_error(SAME_EALIGN, "workspace must be 256-byte aligned");
            writes.push_back(extent(workspace, 4 * (int64_t)head_dim * blocks));
        }
        rc = check_apart(writes, reads);
        if (rc) return rc;
        if (blocks == 0 && !dq_weight && !dk_weight) return SAME_OK;
        p.side[0].out = dq;
        p.side[1].out = dk;
        p.side[0].dout = dq_out;
        p.side[0].dout_row = dq_out_row;
        p.side[0].dout_head = dq_out_head;
        p.side[0].dweight = dq_weight;
        p.side[1].dout = dk_out;
        p.side[1].dout_row = dk_out_row;
        p.side[1].dout_head = dk_out_head;
        p.side[1].dweight = dk_weight;
        p.side[0].blocks = p.side[1].first_block = of_q;
        p.side[1].blocks = blocks - of_q;
        p.part = (float *)workspace;
        return check_hip(same::launch_qk_norm(p, dtype, true, (hipStream_t)stream), "norm gradient launch");
    });
}

int same_log_probs_workspace_size(int64_t rows, int64_t cols, int32_t n_top, size_t *bytes) {
    if (!bytes) return record_error(SAME_EINVAL, "bytes is null");
    if (rows < 0 || cols < 0) return record_error(SAME_EINVAL, "rows and cols must not be negative");
    if (n_top < 0 || n_top > same::kMaxTop) return record_error(SAME_EINVAL, "n_top must lie in [0, 64]");
    if (cols > (int64_t)1 << 21) return record_error(SAME_ESIZE, "cols must be at most 2^21");
    if (rows >= (int64_t)1 << 40) return record_error(SAME_ESIZE, "rows must stay below 2^40");
    int32_t parts, part_cols;
    size_t stats;
    log_probs_layout(rows, cols, n_top, &parts, &part_cols, &stats, bytes);
    return SAME_OK;
}

int same_log_probs(int32_t dtype, const void *logits, int64_t row_stride, int64_t rows, int64_t cols,
                   const int32_t *counts, const int32_t *targets, float *log_probs, float *sums, float *entropy,
                   int32_t n_top, int32_t *top_ids, float *top_log_probs, void *workspace, void *stream) {
    return guarded([&]() -> int {
        std::vector<Extent> reads(1), writes;
        int64_t size;
        int rc = check_logits(dtype, "logits", logits, row_stride, rows, cols, &size, &reads[0]);
        if (rc) return rc;
        if (n_top < 0 || n_top > same::kMaxTop) return record_error(SAME_EINVAL, "n_top must lie in [0, 64]");
        if (rows && log_probs && !targets) return record_error(SAME_EINVAL, "log_probs needs targets");
        if (rows && n_top && (!top_ids || !top_log_probs))
            return record_error(SAME_EINVAL, "top_ids and top_log_probs must be non-null");
        same::LogProbsParams p;
        std::memset((void *)&p, 0, sizeof(p));
        size_t stats, need;
        log_probs_layout(rows, cols, n_top, &p.parts, &p.part_cols, &stats, &need);
        if (!rc) rc = add_rows("counts", counts, rows, 4, 4, reads);
        if (!rc) rc = add_rows("targets", targets, rows, 4, 4, reads);
        if (!rc) rc = add_rows("log_probs", log_probs, rows, 4, 4, writes);
        if (!rc) rc = add_rows("sums", sums, rows, 8, 8, writes);
        if (!rc) rc = add_rows("entropy", entropy, rows, 4, 4, writes);
        if (!rc && n_top) rc = add_rows("top_ids", top_ids, rows, 4 * n_top, 4, writes);
        if (!rc && n_top) rc = add_rows("top_log_probs", top_log_probs, rows, 4 * n_top, 4, writes);
        if (!rc && need) {
            if (!workspace) return record_error(SAME_EINVAL, "workspace is null");
            rc = add_rows("workspace", workspace, 1, (int64_t)need, kAlign, writes);
        }
        if (!rc) rc = check_apart(writes, reads);
        if (rc || rows == 0) return rc;
        p.x = logits;
        p.x_row = rows > 1 ? row_stride : 0;
        p.rows = rows;
        p.cols = (int32_t)cols;
        p.counts = counts;
        p.targets = targets;
        p.log_probs = log_probs;
        p.sums = (float2 *)sums;
        p.entropy = entropy;
        p.n_top = n_top;
        p.top_ids = top_ids;
        p.top_log_probs = top_log_probs;
        p.part_stats = (same::RowStats *)workspace;
        p.part_keys = (uint64_t *)((char *)workspace + stats);
        return check_hip(same::launch_log_probs(p, dtype, (hipStream_t)stream), "log probabilities launch");
    });
}

int same_log_probs_backward(int32_t dtype, const void *logits, int64_t row_stride, int64_t rows, int64_t cols,
                            const int32_t *counts, const int32_t *targets, const float *sums, const float *entropy,
                            const float *dlog_probs, const float *dentropy, void *dlogits, int64_t dlogits_row,
                            void *stream) {
    return guarded([&]() -> int {
        std::vector<Extent> reads(1), writes(1);
        int64_t size;
        int rc = check_logits(dtype, "logits", logits, row_stride, rows, cols, &size, &reads[0]);
        if (!rc) rc = check_logits(dtype, "dlogits", dlogits, dlogits_row, rows, cols, &size, &writes[0]);
        if (rc || rows == 0 || cols == 0) return rc;
        if (rows > 1 && dlogits_row < cols) return record_error(SAME_EINVAL, "dlogits_row must be at least cols");
        if (!sums) return record_error(SAME_EINVAL, "sums is null");
        if (dlog_probs && !targets) return record_error(SAME_EINVAL, "dlog_probs needs targets");
        if (dentropy && !entropy) return record_error(SAME_EINVAL, "dentropy needs entropy");
        if (logits == dlogits && (rows == 1 || row_stride == dlogits_row)) reads[0] = Extent();  // each logit is read first
        if (!rc) rc = add_rows("counts", counts, rows, 4, 4, reads);
        if (!rc) rc = add_rows("targets", targets, rows, 4, 4, reads);
        if (!rc) rc = add_rows("sums", sums, rows, 8, 8, reads);
        if (!rc) rc = add_rows("entropy", entropy, rows, 4, 4, reads);
        if (!rc) rc = add_rows("dlog_probs", dlog_probs, rows, 4, 4, reads);
        if (!rc) rc = add_rows("dentropy", dentropy, rows, 4, 4, reads);
        if (!rc) rc = check_apart(writes, reads);
        if (rc) return rc;
        same::LogProbsGradParams p;
        std::memset((void *)&p, 0, sizeof(p));
        p.x = logits;
        p.dx = dlogits;
        p.x_row = rows > 1 ? row_stride : 0;
        p.dx_row = rows > 1 ? dlogits_row : 0;
        p.rows = rows;
        p.cols = (int32_t)cols;
        p.counts = counts;
        p.targets = targets;
        p.sums = (const float2 *)sums;
        p.entropy = entropy;
        p.dlog_probs = dlog_probs;
        p.dentropy = dentropy;
        return check_hip(same::launch_log_probs_grad(p, dtype, (hipStream_t)stream), "log probabilities' gradient launch");
    });
}

int same_orthogonalise_workspace_size(int32_t dtype, int64_t n_mats, int64_t rows, int64_t cols, size_t *bytes) {
    if (!bytes) return record_error(SAME_EINVAL, "bytes is null");
    OrthoLayout l{};
    const int rc = ortho_layout(dtype, n_mats, rows, cols, l);
    if (rc) return rc;
    *bytes = l.batch ? l.total : 0;
    return SAME_OK;
}

int same_orthogonalise(int32_t dtype, const void *g, int64_t g_mat, int64_t g_row, int64_t n_mats, int64_t rows,
                       int64_t cols, const double *coefs, int32_t steps, double eps, double scale, void *out,
                       int64_t out_mat, int64_t out_row, void *workspace, void *stream) {
    return guarded([&]() -> int {
        OrthoLayout l{};
        int rc = ortho_layout(dtype, n_mats, rows, cols, l);
        if (rc) return rc;
        if (!coefs) return record_error(SAME_EINVAL, "coefs is null");
        if (steps < 1 || steps > same::kMaxSteps) return record_error(SAME_EINVAL, "steps must lie in [1, 32]");
        if (!((float)eps >= std::numeric_limits<float>::min()) || !std::isfinite((float)eps))
            return record_error(SAME_EINVAL, "eps must be a positive normal number in 32 bits");
        if (!std::isfinite((float)scale)) return record_error(SAME_EINVAL, "scale must be finite in 32 bits");
        same::OrthoParams p;
        std::memset((void *)&p, 0, sizeof(p));
        // X's singular values lie in [0, 1] before the first step
        double bound = 1.0, most = 1.0, product = 1.0;
        for (int t = 0; t < steps; ++t) {
            for (int i = 0; i < 3; ++i) {
                if (!std::isfinite((float)coefs[3 * t + i]))
                    return record_error(SAME_EINVAL, "coefs must be finite in 32 bits");
                p.coef[t][i] = (float)coefs[3 * t + i];
            }
            const double b2 = bound * bound;
            product = std::max(product, std::fabs(coefs[3 * t + 1]) * b2 + std::fabs(coefs[3 * t + 2]) * b2 * b2);
            // a little over, for the steps' own roundings
            bound = 1.001 * largest_of(coefs + 3 * t, bound);
            most = std::max(most, bound);
            if (!(most <= 16.0) || !(product <= 4096.0))
                return record_error(SAME_EINVAL, "coefs let singular values of 1 or less grow beyond 16");
        }
        if (l.batch == 0) return SAME_OK;
        if (!g || !out) return record_error(SAME_EINVAL, "g and out must be non-null");
        const int64_t size = dtype == SAME_F32 ? 4 : 2;
        if (!aligned(g, size) || !aligned(out, size))
            return record_error(SAME_EALIGN, "g and out must be aligned to their elements");
        if (rows == 1) g_row = out_row = cols;
        if (n_mats == 1) g_mat = out_mat = 0;
        if (g_row < 0 || g_mat < 0 || out_row < 0 || out_mat < 0)
            return record_error(SAME_EINVAL, "strides must not be negative");
        const double far = (double)(n_mats - 1) * (double)std::max(g_mat, out_mat) +
                           (double)(rows - 1) * (double)std::max(g_row, out_row);
        if (far >= 1e18) return record_error(SAME_ESIZE, "strides pass 10^18 elements");
        if (out_row < cols || (n_mats > 1 && out_mat < (rows - 1) * out_row + cols))
            return record_error(SAME_EINVAL, "out's rows and matrices must not overlap");
        if (l.total && !workspace) return record_error(SAME_EINVAL, "workspace is null");
        if (!aligned(workspace, kAlign)) return record_error(SAME_EALIGN, "workspace must be 256-byte aligned");
        const Extent eg = extent(g, size * ((n_mats - 1) * g_mat + (rows - 1) * g_row + cols));
        const Extent eo = extent(out, size * ((n_mats - 1) * out_mat + (rows - 1) * out_row + cols));
        const bool itself = g == out && g_mat == out_mat && g_row == out_row;
        const std::vector<Extent> writes = {eo, extent(workspace, (int64_t)l.total)};
        std::vector<Extent> reads;
        if (!itself) reads.push_back(eg);  // g is read whole before out is written
        rc = check_apart(writes, reads);
        if (!rc && itself && overlap(eg, writes[1])) rc = record_error(SAME_EINVAL, "workspace overlaps g");
        if (rc) return rc;
        p.g = g;
        p.out = out;
        p.g_mat = g_mat;
        p.g_row = g_row;
        p.out_mat = out_mat;
        p.out_row = out_row;
        p.n_mats = n_mats;
        p.rows = (int32_t)rows;
        p.cols = (int32_t)cols;
        p.n = (int32_t)l.n;
        p.m = (int32_t)l.m;
        p.np = (int32_t)l.np;
        p.mp = (int32_t)l.mp;
        p.tall = rows > cols;
        p.eps = (float)eps;
        p.out_scale = (float)scale;
        p.sx = plane_scale(most, 12);
        p.sa = plane_scale(most * most, 13);
        p.sb = plane_scale(product, 10);
        p.steps = steps;
        p.parts = l.parts;
        p.part_cols = l.part_cols;
        p.small_parts = workspace;
        p.small_factors = (char *)workspace + l.small_parts;
        char *at = (char *)workspace;
        const auto take = [&](size_t bytes) {
            char *here = at;
            at += bytes;
            return here;
        };
        p.splits = l.splits;
        p.squares = (double *)take(l.squares);
        p.gram_parts = (float *)take(l.gram_parts);
        p.x32 = (float *)take(l.x32);
        for (same::Planes *w : {&p.x, &p.xt[0], &p.xt[1]}) {
            w->hi = (_Float16 *)take(l.wide);
            w->lo = (_Float16 *)take(l.wide);
        }
        for (same::Planes *w : {&p.a, &p.b}) {
            w->hi = (_Float16 *)take(l.square);
            w->lo = (_Float16 *)take(l.square);
        }
        return check_hip(same::launch_orthogonalise(p, l.batch, dtype, (hipStream_t)stream), "orthogonalise launch");
    });
}

}  // extern "C"
