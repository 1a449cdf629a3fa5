// Rotary positions over several axes.
//
//   (a, b) -> (a cos t - b sin t, a sin t + b cos t),  t = +- positions[axis(p)] freqs[p]
#pragma once
#include "tile.hpp"

namespace nsl {

struct RotaryArgs {
    View in[2], out[2];      // q and k
    int heads[2];
    const void* positions;
    int64_t pos_axis, pos_batch;
    const float* freqs;
    int64_t rows, tokens;    // tokens = batch * rows
    int pos_type, dim, pairs, ends[4];   // ends[x]: first pair past axis x
    int chunks, each;        // work items of a head; heads an item takes
    bool interleaved, inverse;
};

// cos and sin of +-position * freq. The product and its reduction to turns
// are in 64 bits (a 32-bit product of a position near 10^5 is off by 10^-2
// rad). Sine and cosine are taken of the reduced angle in 32 bits, which is
// off by up to 2^-26 of a turn; what that rounding left enters to first order.
__device__ inline void turn_of(const RotaryArgs& a, int64_t at, int p, float& cs, float& sn) {
    const int axis = (p >= a.ends[0]) + (p >= a.ends[1]) + (p >= a.ends[2]);
    const int64_t i = axis * a.pos_axis + at;
    double x;
    if (a.pos_type == 0)
        x = static_cast<const float*>(a.positions)[i];
    else if (a.pos_type == 1)
        x = static_cast<const double*>(a.positions)[i];
    else
        x = static_cast<double>(static_cast<const int64_t*>(a.positions)[i]);
    double turns = x * static_cast<double>(a.freqs[p]) * 0.15915494309189535;
    turns -= rint(turns);
    const float near = static_cast<float>(turns);
    const float left = static_cast<float>(turns - static_cast<double>(near)) * 6.2831853f;
    float s0, c0;
    sincospif(2.f * near, &s0, &c0);
    sn = fmaf(c0, left, s0);
    cs = fmaf(-s0, left, c0);
    if (a.inverse) sn = -sn;
}

// One item: V pairs (or V values past the pairs, which are copied) of one
// token, for `each` heads: the angles are formed once and serve them all.
// Rows need no more alignment than their element's. Bound by memory:
// 446,932 tokens of 8 + 2 heads of 64, bfloat16: 250 us (4.6 TB/s, 232 at the
// rate of a large copy); 88,835 of 6 + 3 heads of 80 with 30 pairs, float32
// (V = 2): 136 us (3.8 TB/s, 104).
template <class T, int V>
__global__ __launch_bounds__(256) void k_rotary(RotaryArgs a) {
    const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, token = id / a.chunks;
    if (token >= a.tokens) return;
    const int chunk = static_cast<int>(id - token * a.chunks);
    const int64_t b = token / a.rows, row = token - b * a.rows;
    const int turned = a.pairs / V, h0 = blockIdx.y * a.each, h1 = min(h0 + a.each, a.heads[0] + a.heads[1]);
    float cs[V], sn[V];
    int d0, d1;   // where the item's values lie (interleaved pairs: 2 V from d0 on)
    const bool pairs = chunk < turned;
    if (pairs) {
        const int64_t at = b * a.pos_batch + row;
#pragma unroll
        for (int j = 0; j < V; ++j) turn_of(a, at, chunk * V + j, cs[j], sn[j]);
        d0 = a.interleaved ? 2 * V * chunk : V * chunk;
        d1 = a.pairs + d0;
    } else {
        d0 = 2 * a.pairs + V * (chunk - turned);
        d1 = d0;
    }
    for (int hh = h0; hh < h1; ++hh) {
        const int which = hh >= a.heads[0], head = which ? hh - a.heads[0] : hh;
        const View &in = a.in[which], &out = a.out[which];
        const T* x = reinterpret_cast<const T*>(in.data) + b * in.batch + row * in.row + head * in.head;
        T* y = reinterpret_cast<T*>(out.data) + b * out.batch + row * out.row + head * out.head;
        T u[2 * V];
        if (!pairs) {
            __builtin_memcpy(u, x + d0, V * sizeof(T));
            __builtin_memcpy(y + d0, u, V * sizeof(T));
            continue;
        }
        if (a.interleaved) {
            __builtin_memcpy(u, x + d0, 2 * V * sizeof(T));
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float m = static_cast<float>(u[2 * j]), n = static_cast<float>(u[2 * j + 1]);
                u[2 * j] = static_cast<T>(fmaf(m, cs[j], -n * sn[j]));
                u[2 * j + 1] = static_cast<T>(fmaf(m, sn[j], n * cs[j]));
            }
            __builtin_memcpy(y + d0, u, 2 * V * sizeof(T));
        } else {
            __builtin_memcpy(u, x + d0, V * sizeof(T));
            __builtin_memcpy(u + V, x + d1, V * sizeof(T));
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float m = static_cast<float>(u[j]), n = static_cast<float>(u[V + j]);
                u[j] = static_cast<T>(fmaf(m, cs[j], -n * sn[j]));
                u[V + j] = static_cast<T>(fmaf(m, sn[j], n * cs[j]));
            }
            __builtin_memcpy(y + d0, u, V * sizeof(T));
            __builtin_memcpy(y + d1, u + V, V * sizeof(T));
        }
    }
}

}  // namespace nsl
