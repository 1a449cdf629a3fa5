// Attention of one new token a stream over its ring cache, and the cache's fill.
//
// The cache's valid slots are a prefix (the window's order does not matter to
// a softmax), so a step reads slots 0 .. min(pos + 1, sinks + window) - 1.
#pragma once
#include "attention.hpp"

namespace nsl {

struct StepArgs {
    View q, k, v, o;           // batch stride: from stream to stream
    void *k_cache, *v_cache;   // [streams][kv_heads][slots][dim]
    const int64_t* pos;
    float* part;               // [streams][heads][splits][dim + 2]: sum p v, base, sum p
    int64_t streams;
    int heads, kv_heads, dim, group, head_blocks, splits;
    int slots, sinks, window;
    AttnScale by;
};

__device__ inline int ring_slot(int64_t t, int sinks, int window) {
    return static_cast<int>(t < sinks ? t : sinks + (t - sinks) % window);
}

// What a part whose base is `base` weighs beside one of base `all`, the largest (-inf: nothing was seen).
__device__ inline float weight_of(float base, float all) { return base == -INFINITY ? 0.f : exp2_(base - all); }

// A workgroup takes one stream, one kv head with up to 32 of its query heads
// (the columns of S^T = K Q^T), and one of `splits` stretches of the slots;
// its waves take every fourth tile of 32 slots. K goes from memory to
// fragments; V goes through a stretch of LDS of the wave's own to be turned.
// In 16 bits p enters its product as two numbers, as in k_attention.
// Bound by reading the cache: 3,536 streams of 260 slots, 8 heads of 64 over 2,
// bfloat16: 103 us (4.3 TB/s, 90 at the rate of a large copy); 4 streams of
// 131,076 slots of 128, float16: 100 us and 6.5 for the join (5.1 TB/s, 109).
// WIDE: every view and the caches take 16-byte accesses (one kernel for both
// spilled at heads above 64: 142 us on the long streams).
template <class T, int DP, bool WIDE>
__global__ __launch_bounds__(256, 2) void k_step(StepArgs a) {
    constexpr int RB = row_bytes<T, DP>(), kEach = 32 * DP / 8 / 64;
    __shared__ __align__(128) char vt[4][32 * RB];
    __shared__ float tops[4][32], sums[4][32];
    __shared__ float joined[DP][33];
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), m = lane & 31, h = lane >> 5;
    const unsigned id = die_order(blockIdx.x, gridDim.x), rest = id / a.splits;
    const int split = id - rest * a.splits;
    const int hb = static_cast<int>(rest % a.head_blocks);
    const unsigned sk = rest / a.head_blocks;
    const int64_t stream = sk / a.kv_heads;
    const int kv = static_cast<int>(sk % a.kv_heads);
    const int h_first = 32 * hb, h_count = min(32, a.group - h_first);

    const int64_t pos = a.pos[stream];
    const int n = pos < 0 ? 0 : pos < a.slots ? static_cast<int>(pos) + 1 : a.slots;
    const int fresh = pos < 0 ? -1 : ring_slot(pos, a.sinks, a.window);
    const T* kn = reinterpret_cast<T*>(a.k.data) + stream * a.k.batch + kv * a.k.head;
    const T* vn = reinterpret_cast<T*>(a.v.data) + stream * a.v.batch + kv * a.v.head;
    T* kc = static_cast<T*>(a.k_cache) + static_cast<int64_t>(sk) * a.slots * a.dim;
    T* vc = static_cast<T*>(a.v_cache) + static_cast<int64_t>(sk) * a.slots * a.dim;
    const int tiles = (n + 31) / 32;
    const int t0 = static_cast<int>(static_cast<int64_t>(tiles) * split / a.splits);
    const int t1 = static_cast<int>(static_cast<int64_t>(tiles) * (split + 1) / a.splits);

    // the new token's row is taken from the arguments, by every workgroup
    // that needs it; only one of them writes it to the cache
    if (hb == 0 && fresh >= 32 * t0 && fresh < 32 * t1) {
        for (int d = tid; d < a.dim; d += 256) {
            kc[static_cast<int64_t>(fresh) * a.dim + d] = kn[d];
            vc[static_cast<int64_t>(fresh) * a.dim + d] = vn[d];
        }
    }
    const bool mine = m < h_count;
    const T* qp = reinterpret_cast<T*>(a.q.data) + stream * a.q.batch +
                  static_cast<int64_t>(kv * a.group + h_first + (mine ? m : 0)) * a.q.head;
    frag<T> qf[DP / 16], kf[DP / 16], vr[kEach];
    load_rows<T, DP>(qf, qp, mine && n > 0, a.dim, WIDE, lane);
    acc16 o[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) o[d] = zero16();
    float sum = 0.f;
    Base<T, 0> base;

    auto fetch = [&](int t) {
        const int key = 32 * t + m;
        const T* kr = key == fresh ? kn : kc + static_cast<int64_t>(key) * a.dim;
#pragma unroll
        for (int s = 0; s < DP / 16; ++s)
            kf[s] = load8<T, WIDE>(kr + 16 * s + 8 * h, key < n ? a.dim - 16 * s - 8 * h : 0, s + h > 0);
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int c = lane + 64 * e, slot = 32 * t + c / (DP / 8), d = c % (DP / 8) * 8;
            vr[e] = load8<T, WIDE>((slot == fresh ? vn : vc + static_cast<int64_t>(slot) * a.dim) + d,
                                   slot < n ? a.dim - d : 0, d > 0);
        }
    };
    if (t0 + wave < t1) fetch(t0 + wave);
    for (int t = t0 + wave; t < t1; t += 4) {
        acc16 s = zero16();
#pragma unroll
        for (int x = 0; x < DP / 16; ++x) s = mma(kf[x], qf[x], s);
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int c = lane + 64 * e;
            write8<T, RB>(vt[wave], c / (DP / 8), c % (DP / 8), vr[e]);
        }
        if (t + 4 < t1) fetch(t + 4);
        if (32 * t + 32 > n) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = 32 * t + 8 * (r >> 2) + 4 * h + (r & 3) < n ? s[r] : -INFINITY;
        }
        float mx = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
        float factor;
        if (base.move(half_max(mx), a.by, factor)) {
            sum *= factor;
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) o[d] *= factor;
        }
        const float zero = base.of(a.by);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = exp2_(fmaf(s[r], a.by.c, -zero));
            sum += s[r];
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const frag<T> p = narrow<T>(s, x), low = rest_of<T>(s, x, p);
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) {
                const frag<T> vd = read_turned<T, RB>(vt[wave], 16 * x, 32 * d, lane);
                o[d] = mma(vd, p, o[d]);
                if constexpr (sizeof(T) == 2) o[d] = mma(vd, low, o[d]);
            }
        }
    }
    // the four waves' results, in the waves' order
    sum = half_sum(sum);
    if (h == 0) {
        tops[wave][m] = base.top == -INFINITY ? -INFINITY : base.of(a.by);
        sums[wave][m] = sum;
    }
    __syncthreads();
    // weights are differences of the bases as the exponentials took them
    const float all = fmaxf(fmaxf(tops[0][m], tops[1][m]), fmaxf(tops[2][m], tops[3][m]));
    const float share = weight_of(tops[wave][m], all);
    for (int v = 0; v < 4; ++v) {
        if (wave == v) {
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int row = 32 * d + 8 * (r >> 2) + 4 * h + (r & 3);
                    joined[row][m] = (v ? joined[row][m] : 0.f) + o[d][r] * share;
                }
        }
        __syncthreads();
    }
    for (int x = tid; x < h_count * a.dim; x += 256) {
        const int hd = x / a.dim, d = x - hd * a.dim;
        const int head = kv * a.group + h_first + hd;
        const float am = fmaxf(fmaxf(tops[0][hd], tops[1][hd]), fmaxf(tops[2][hd], tops[3][hd]));
        float total = 0.f;
#pragma unroll
        for (int v = 0; v < 4; ++v) total += sums[v][hd] * weight_of(tops[v][hd], am);
        const float val = joined[d][hd];
        if (a.splits == 1) {
            reinterpret_cast<T*>(a.o.data)[stream * a.o.batch + head * a.o.head + d] =
                static_cast<T>(total == 0.f ? 0.f : val / total);
        } else {
            float* p = a.part + ((stream * a.heads + head) * a.splits + split) * (a.dim + 2);
            p[d] = val;
            if (d == 0) {
                p[a.dim] = am;
                p[a.dim + 1] = total;
            }
        }
    }
}

// Joins the stretches (at most 256) of one head of one stream: their weights
// first, then each wave adds up every fourth stretch and the four sums are added.
template <class T>
__global__ __launch_bounds__(256) void k_step_join(StepArgs a) {
    __shared__ float tops[4], totals[4], weight[256], sums[4][128];
    const int64_t stream = blockIdx.x / a.heads, stride = a.dim + 2;
    const int head = blockIdx.x % a.heads, tid = threadIdx.x, lane = tid & 63, wave = wave_number();
    const float* p = a.part + static_cast<int64_t>(blockIdx.x) * a.splits * stride;
    const bool there = tid < a.splits;
    const float mine = there ? p[tid * stride + a.dim] : -INFINITY;
    float top = mine;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x));
    if (lane == 0) tops[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    const float w = weight_of(mine, top);
    weight[tid] = w;
    float total = there ? p[tid * stride + a.dim + 1] * w : 0.f;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) total += __shfl_xor(total, x);
    if (lane == 0) totals[wave] = total;
    __syncthreads();
    total = totals[0] + totals[1] + totals[2] + totals[3];
    float x0 = 0.f, x1 = 0.f;
#pragma unroll 8
    for (int s = wave; s < a.splits; s += 4) {
        const float* q = p + s * stride;
        x0 = fmaf(lane < a.dim ? q[lane] : 0.f, weight[s], x0);
        x1 = fmaf(lane + 64 < a.dim ? q[lane + 64] : 0.f, weight[s], x1);
    }
    sums[wave][lane] = x0;
    sums[wave][lane + 64] = x1;
    __syncthreads();
    if (tid < a.dim) {
        const float val = sums[0][tid] + sums[1][tid] + sums[2][tid] + sums[3][tid];
        reinterpret_cast<T*>(a.o.data)[stream * a.o.batch + head * a.o.head + tid] =
            static_cast<T>(total == 0.f ? 0.f : val / total);
    }
}

struct FillArgs {
    View k, v;
    void *k_cache, *v_cache;
    const int64_t* off;
    int rows, n_bands, kv_heads, dim, slots, sinks, window;
};

// One thread copies V values of a slot's row (8 where the width is a
// multiple of 8), which also share the index arithmetic: 3,536 streams of 260
// slots of 2 x 64, bfloat16, 120 us; value by value 344.
template <class T, int V>
__global__ __launch_bounds__(256) void k_fill(FillArgs a) {
    const int64_t stream = blockIdx.y;
    const int64_t b = stream / a.n_bands;
    const int band = static_cast<int>(stream % a.n_bands);
    const int start = band_bound(a.off, a.n_bands, a.rows, band + 1);
    const int last = band_bound(a.off, a.n_bands, a.rows, band + 2) - start - 1;
    const unsigned parts = a.dim / V;
    const int64_t rows = static_cast<int64_t>(a.kv_heads) * a.slots, first = stream * rows * a.dim;
    for (int64_t e = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; e < rows * parts; e += 256 * gridDim.x) {
        const int64_t row = e / parts;
        const int kv = static_cast<int>(row / a.slots), slot = static_cast<int>(row - static_cast<int64_t>(kv) * a.slots);
        const int d = static_cast<int>(e - row * parts) * V;
        int t = slot;
        if (slot >= a.sinks) {   // the last token that went to this slot
            const int since = last - slot;
            t = since < 0 ? -1 : slot + since / a.window * a.window;
        }
        if (t >= 0 && t <= last) {
            std::conditional_t<V == 8, frag<T>, T> x, y;
            __builtin_memcpy(&x, row_of<T>(a.k, b, start + t, kv) + d, sizeof(x));
            __builtin_memcpy(&y, row_of<T>(a.v, b, start + t, kv) + d, sizeof(y));
            __builtin_memcpy(static_cast<T*>(a.k_cache) + first + row * a.dim + d, &x, sizeof(x));
            __builtin_memcpy(static_cast<T*>(a.v_cache) + first + row * a.dim + d, &y, sizeof(y));
        }
    }
}

}  // namespace nsl
