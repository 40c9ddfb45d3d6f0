// The join of a gradient's parts.
#pragma once

#include "cross_common.hpp"

namespace same {
namespace cross {

// Sums the parts of dQ (SIDES = 1) or of dK and dV (SIDES = 2), in order.
// Latency bounds it: 5 us where there is little to add, 16 us for dK and dV of
// 4,095 keys, 4 key heads of 128, in parts of 33 MB.
template <typename T, int SIDES>
__global__ __launch_bounds__(256) void cross_join_grad_kernel(CrossParams p, const CrossJoin *joins) {
    const CrossJoin j = joins[blockIdx.x];
    const int hk = blockIdx.y, tile = kJoinOwners * gridDim.z, first = kJoinOwners * blockIdx.z;
    const int quads = p.dim / 4, owners = min(kJoinOwners, j.n_own - first);
    for (int idx = threadIdx.x; idx < owners * quads * SIDES; idx += blockDim.x) {
        const int line = idx / quads, d = (idx - line * quads) * 4;
        const int own = first + line / SIDES, side = line % SIDES;
        const int64_t step = (int64_t)p.heads_kv * tile * SIDES * p.dim;
        const float *src = p.part + ((((int64_t)j.slot * p.heads_kv + hk) * tile + own) * SIDES + side) * p.dim + d;
        f32x4 acc = 0.0f;
#pragma unroll 8
        for (int s = 0; s < j.n_parts; ++s) acc += *(const f32x4 *)(src + s * step);
        T *dst;
        float gain = p.scale * p.keep_gain;
        if (SIDES == 1) {
            dst = (T *)p.dq + row_id(p, j.q0, j.own0 + own, hk) * p.dim;
        } else {
            dst = (T *)(side ? p.dv : p.dk) + ((j.k0 + j.own0 + own) * p.heads_kv + hk) * p.dim;
            if (side) gain = p.keep_gain;
        }
        typename Vec<T>::x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (T)(acc[i] * gain);
        *(typename Vec<T>::x4 *)(dst + d) = w;
    }
}

}  // namespace cross
}  // namespace same
