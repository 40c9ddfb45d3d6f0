// Internal interface between the cross-attention and dropout entry points
// (operators.cpp) and their gfx950 kernels (cross_*.hip, dropout.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

namespace same {

// One block's work: 32 * (owner waves) owners of a segment (query rows in the
// forward and dQ passes, keys in the dK/dV pass) against [beg, end) of the
// other axis.  slot >= 0: a part of a split axis, joined afterwards.
// A segment's query rows of one key head are numbered i * group + g.
struct CrossItem {
    int64_t q0, k0;      // the segment's first query token and first key
    int32_t own0, n_own;
    int32_t beg, end;
    int32_t slot, pad;
};

// Parts [slot, slot + n_parts) of one tile of owners, at most kMaxParts.
struct CrossJoin {
    int64_t q0, k0;
    int32_t own0, n_own;
    int32_t slot, n_parts;
};

// One wave's work where segments are small: neighbouring segments with at most
// 32 query rows (of one key head) and 32 keys together.
struct CrossSmallItem {
    int64_t q0, k0;           // first query token and first key
    int32_t n_rows, n_keys;
    uint16_t range[32];       // a row's keys in the tile: first | (last + 1) << 8
};

struct CrossPass {
    const CrossItem *items;
    const CrossJoin *joins;
    int32_t n_items, n_joins;
    int32_t own_waves;  // waves of a block that own tiles; one shares the other axis with three more
};

struct CrossTensor {
    const void *p;
    int64_t row, head;   // strides in elements
};

struct CrossParams {
    CrossTensor q, k, v, dout;
    const uint8_t *key_mask;
    const void *out_in;        // gradient: the forward's output
    void *out, *dq, *dk, *dv;  // contiguous [tokens][heads][head_dim]
    float *lse, *delta;        // [tokens][heads]
    float *part, *part_ml;     // parts: [slot][key head][owner][head_dim], (max, sum)
    const CrossItem *items;
    const CrossSmallItem *small;
    int32_t n_items;
    int32_t heads_q, heads_kv, group, dim;
    float scale;
    uint32_t drop_below;       // bytes below this are dropped (0: no dropout)
    float keep_gain;           // 256 / (256 - drop_below)
    float keep_part;           // its inverse
    uint32_t seed_lo, seed_hi, call_id;
};

constexpr int kCrossF16 = 1, kCrossBf16 = 2;
constexpr int kJoinOwners = 8;  // owners that a join's block takes
constexpr int kMaxParts = 64;   // of one tile
// Blocks (of up to 512 threads) of one launch: the device takes fewer than
// 2^32 threads and runs the rest of a larger grid without an error, short.
// More items go into further launches.
constexpr int32_t kLaunchBlocks = 1 << 22;
inline int32_t items_per_launch(int32_t heads_kv) { return kLaunchBlocks / heads_kv; }

hipError_t launch_cross_forward(const CrossParams &p, const CrossPass &w, int dtype, hipStream_t s);
hipError_t launch_cross_small(const CrossParams &p, bool grad, int dtype, hipStream_t s);
hipError_t launch_cross_dq(const CrossParams &p, const CrossPass &w, int dtype, hipStream_t s);
hipError_t launch_cross_dkv(const CrossParams &p, const CrossPass &w, int dtype, hipStream_t s);

struct DropoutParams {
    const void *x, *residual;
    void *y;
    int64_t rows, cols, x_row, r_row, y_row;
    uint32_t drop_below;  // 16-bit numbers below this are dropped
    float keep_gain;
    uint32_t seed_lo, seed_hi, call_id;
};

hipError_t launch_dropout(const DropoutParams &p, int dtype, hipStream_t s);

}  // namespace same
