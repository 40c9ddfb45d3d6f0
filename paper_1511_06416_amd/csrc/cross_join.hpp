// The join of a gradient's parts.
#pragma once

#include "cross_common.hpp"

namespace same {
namespace cross {

// Sums the parts of dQ (SIDES = 1) or of dK and dV (SIDES = 2), in order.
template <typename T, int SIDES>
__global__ __launch_bounds__(256) void cross_join_grad_kernel(CrossParams p, const CrossJoin *joins) {
    const int hk = blockIdx.y, tile = 32 * gridDim.z;
    const CrossJoin j = joins[blockIdx.x];
    const int quads = p.dim / 4;
    const int owners = min(32, j.n_own - 32 * (int)blockIdx.z);
    for (int idx = threadIdx.x; idx < owners * quads * SIDES; idx += blockDim.x) {
        const int own = 32 * blockIdx.z + idx / (quads * SIDES), side = (idx / quads) % SIDES, d = (idx % quads) * 4;
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

}  // namespace cross
}  // namespace same
