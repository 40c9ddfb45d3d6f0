// Internal interface between the entry points of a training step's operators
// (step.cpp) and their gfx950 kernels (qk_norm.hip, log_probs*.hip,
// orthogonalise*.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

#include "norm_shares.hpp"

namespace same {

// ---- norms of queries and keys with the position rotation

constexpr int kMaxHeadDim = 128;
constexpr int kNormBlocks = 1024;  // of a gradient: each leaves a part of the weights' gradient

// Queries or keys.
struct NormSide {
    const void *x, *dout;
    int64_t x_row, x_head, dout_row, dout_head;  // strides in elements
    const float *weight;                         // null: ones
    const int32_t *positions;
    void *out;                                   // contiguous: the result, or dx
    float *dweight;                              // null: not wanted
    int64_t tokens;
    int32_t heads;
    int32_t pack;                                // tokens that a wave takes at once
    NormShares shares;                           // of a token's heads
    int32_t first_block, blocks;                 // of the launch
};

struct NormParams {
    NormSide side[2];
    float *part;          // [blocks][head_dim]
    int32_t dim, half;    // half: pairs that turn
    float eps, inv_dim;
    // turns a position of every pair, in two parts: far positions need more than 53 bits
    double turn[kMaxHeadDim / 2], turn_low[kMaxHeadDim / 2];
};

hipError_t launch_qk_norm(NormParams &p, int dtype, bool grad, hipStream_t s);
int qk_norm_grad_blocks(int64_t rows_q, int64_t rows_k, int32_t dim, int32_t *blocks_q);

// ---- log probabilities of given states, with entropy and alternatives

constexpr int kMaxTop = 64;
constexpr int kMaxRowParts = 64;

// A part of a row: its largest logit, and the sums of e = 2^t and of t e, t the
// distance from that in powers of two.
struct RowStats {
    float max, sum, weighted;
};

struct LogProbsParams {
    const void *x;
    int64_t x_row, rows;
    int32_t cols;
    const int32_t *counts, *targets;   // null: cols; none asked for
    float *log_probs;
    float2 *sums;                      // largest logit, logarithm of the sum relative to it
    float *entropy;
    int32_t n_top;
    int32_t *top_ids;
    float *top_log_probs;
    int32_t parts, part_cols;          // of a long row
    RowStats *part_stats;              // [rows][parts]
    uint64_t *part_keys;               // [rows][parts][n_top]
};

struct LogProbsGradParams {
    const void *x;
    void *dx;
    int64_t x_row, dx_row, rows;
    int32_t cols;
    const int32_t *counts, *targets;
    const float2 *sums;
    const float *entropy, *dlog_probs, *dentropy;  // either gradient may be null
};

// Parts of a row, and the columns of each.
void log_probs_parts(int64_t rows, int64_t cols, int32_t *parts, int32_t *part_cols);
hipError_t launch_log_probs(const LogProbsParams &p, int dtype, hipStream_t s);
hipError_t launch_log_probs_grad(const LogProbsGradParams &p, int dtype, hipStream_t s);

// ---- orthogonalising an update by Newton-Schulz products

constexpr int kMaxSteps = 32;

// A plane pair holds numbers as the sum of two fp16, times a power of two.
struct Planes {
    _Float16 *hi, *lo;
};

struct OrthoParams {
    const void *g;
    void *out;
    int64_t g_mat, g_row, out_mat, out_row, n_mats;
    int32_t rows, cols;       // of g
    int32_t n, m;             // the smaller and the larger of them
    int32_t np, mp;           // padded
    bool tall;                // rows > cols: X is g's transpose
    float eps, out_scale;
    float sx, sa, sb;         // the planes' powers of two
    double *squares;          // [n_mats][kNormParts]
    Planes x, xt[2], a, b;    // [n_mats] of [np][mp], [mp][np], [np][np], [np][np]
    int32_t splits;           // of the sums of X X^T
    float *gram_parts;        // [n_mats][splits][np][np], or of columns
    float *x32;               // X between steps, of columns
    int32_t parts, part_cols; // of a small update's columns
    void *small_parts, *small_factors;  // [n_mats][parts] and [n_mats] sets of tiles
    int32_t steps;
    float coef[kMaxSteps][3];
};

constexpr int kNormParts = 1024;  // of a sum of squares

constexpr int kSmallSide = 32;  // of updates that take the small kernels

void ortho_small_parts(int64_t n, int64_t m, int32_t *parts, int32_t *part_cols, size_t *tile_bytes);
hipError_t launch_ortho_small(const OrthoParams &p, int dtype, hipStream_t s);

int orthogonalise_splits(int64_t np, int64_t mp);
// Updates that one block holds.
inline bool ortho_whole(int64_t n, int64_t m) {
    return n <= 96 ? m <= 256 : n <= 128 && m <= 128;
}
hipError_t launch_ortho_whole(const OrthoParams &p, int dtype, hipStream_t s);

// Updates of which each block holds some columns, at most 16 parts of four strips
// of 128 (us, here and in the tiled form: 60 x 1,000 52 and 91; 750 of 905 x 33 613
// and 1,012; 128 x 1,000 85 and 102; 30 of 100 x 1,500 191 and 216).
inline bool ortho_columns(int64_t n, int64_t m) {
    return n <= 64 ? m <= 8192 : n <= 128 && m <= 4096;
}
void ortho_columns_layout(int64_t n, int64_t m, int32_t *parts, int32_t *part_cols, size_t *x_bytes,
                          size_t *part_bytes, size_t *plane_bytes);
hipError_t launch_ortho_columns(const OrthoParams &p, int dtype, hipStream_t s);

// Sums of squares of all matrices, in `parts` parts each.
hipError_t launch_ortho_squares(const OrthoParams &p, int dtype, hipStream_t s, int *parts);

// Matrices that share the planes (or tiles) of the workspace, in turn.
int64_t orthogonalise_batch(int64_t n_mats, int64_t np, int64_t mp);
hipError_t launch_orthogonalise(const OrthoParams &p, int64_t batch, int dtype, hipStream_t s);

}  // namespace same
