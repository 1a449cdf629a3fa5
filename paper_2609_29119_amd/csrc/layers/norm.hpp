// Group norm with an activation on ragged rows, channels last.
//
// A group's statistics go over its cg channels and all tokens of one band of one signal:
//   xh = (x - mean) rstd   z = w xh + b   y = act(z)        (w, b: of the band and the channel)
//   dz = dy act'(z)   d = w dz   dx = rstd (d - mean(d) - xh mean(d xh))
//   db = sum dz   dw = sum dz xh     over the band's tokens of all signals
//
// A workgroup takes a chunk of a band's tokens, all channels; a thread 8
// channels of every n-th token, held in registers from the load to the store.
// So a band of one chunk is read once; longer ones leave their chunks'
// statistics in slots, which a second kernel joins and a third applies.
// Statistics are means and sums of squared differences from them, never
// differences of large sums, and are held in 64 bits.
#pragma once
#include "act.hpp"

namespace nsl {

constexpr int kNormThreads = 512, kNormChannels = 8 * kNormThreads, kNormGroups = 1024;
// Octets of x that a thread holds (half as many where dy is held beside it).
template <class T> constexpr int norm_held() { return sizeof(T) == 4 ? 4 : 8; }

struct NormArgs {
    View x, y, dy;                // (the gradient's result dx is y)
    const void *w, *b;            // [n_bands][channels] or NULL
    int64_t w_band, b_band;       // their strides from band to band
    void *dw, *db;
    double2* stats;               // [batch][n_bands][groups]: mean, rstd
    double2* part;                // [batch][slots][groups]: of a chunk (mean, sum of squares) or (sum d, sum d xh)
    float* sums;                  // weights' gradient: [items][2][channels]
    const int64_t* off;
    int rows, n_bands, batch, channels, groups, cg;
    int octets, together;         // octets of a token's channels, tokens that a workgroup takes at once
    int shift, weight_shift;      // of a chunk's tokens; of the weights' gradient's rows
    unsigned items;               // work items of a signal
    int64_t first_block;          // of a launch of a kernel whose blocks may pass a grid's limit
    int act;
    double eps;
};

template <class T> __device__ inline T* norm_row(const View& v, int64_t b, int64_t row) {
    return reinterpret_cast<T*>(v.data) + b * v.batch + row * v.row;
}

// A thread's 8 channels: what is applied to them.
struct NormOctet {
    float high[8], low[8], rstd[8], w[8], b[8];   // the mean as two numbers
    template <class T> __device__ void load_affine(const NormArgs& a, int band, int col) {
        const T* wp = static_cast<const T*>(a.w) + band * a.w_band;
        const T* bp = static_cast<const T*>(a.b) + band * a.b_band;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool there = col + i < a.channels;
            w[i] = a.w && there ? static_cast<float>(wp[col + i]) : 1.f;
            b[i] = a.b && there ? static_cast<float>(bp[col + i]) : 0.f;
        }
    }
    __device__ void set(int i, double mean, double r) {
        high[i] = static_cast<float>(mean);
        low[i] = static_cast<float>(mean - static_cast<double>(high[i]));
        rstd[i] = static_cast<float>(r);
    }
    __device__ void load_stats(const NormArgs& a, const double2* st, int col) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double2 v = st[min(col + i, a.channels - 1) / a.cg];
            set(i, v.x, v.y);
        }
    }
    __device__ float hat(float x, int i) const { return ((x - high[i]) - low[i]) * rstd[i]; }
};

template <class T> __device__ inline void store8(T* p, const float (&v)[8], int n, bool wide) {
    frag<T> f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = static_cast<T>(v[i]);
    if (wide) {
        *reinterpret_cast<frag<T>*>(p) = f;
    } else if (n >= 8) {
        __builtin_memcpy(p, &f, sizeof(f));
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < n) p[i] = f[i];
    }
}

// Sums over a workgroup's tokens and a group's channels, in a fixed order.
// `cells` holds a value of each of the tokens taken at once and each channel.
__device__ inline void norm_put(const NormArgs& a, double* cells, int tr, int col, const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) cells[tr * a.octets * 8 + col + i] = v[i];
}
__device__ inline void norm_put(const NormArgs& a, double* cells, int tr, int col, const double (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) cells[tr * a.octets * 8 + col + i] = v[i];
}
// result: [groups], in LDS. All threads; begins and ends with a barrier.
__device__ inline void norm_add_up(const NormArgs& a, double* cells, double* result, int tid) {
    const int width = a.octets * 8;
    __syncthreads();
    if (a.together > 1) {
        for (int c = tid; c < a.channels; c += kNormThreads) {
            double s = cells[c];
            for (int r = 1; r < a.together; ++r) s += cells[r * width + c];
            cells[c] = s;
        }
        __syncthreads();
    }
    if (a.cg <= 32) {
        for (int g = tid; g < a.groups; g += kNormThreads) {
            double s = 0.0;
            for (int c = g * a.cg; c < (g + 1) * a.cg; ++c) s += cells[c];
            result[g] = s;
        }
    } else {
        const int lane = tid & 63;
        for (int g = wave_number(); g < a.groups; g += kNormThreads / 64) {
            double s = 0.0;
            for (int c = lane; c < a.cg; c += 64) s += cells[g * a.cg + c];
#pragma unroll
            for (int x = 1; x < 64; x <<= 1) s += __shfl_xor(s, x);
            if (lane == 0) result[g] = s;
        }
    }
    __syncthreads();
}

// What a workgroup works on, and where this thread's part of it lies: channels
// col .. col + 7 of every together-th token from tr on, those below n.
struct NormPlace {
    int64_t b;
    Tile<int> t;
    int all, n, tr, col;   // all: the chunk's tokens
    bool outside, several;
    __device__ explicit NormPlace(const NormArgs& a) {
        const unsigned id = die_order(blockIdx.x, gridDim.x);
        const int tid = threadIdx.x;
        b = id / a.items;
        t = find_tile<int>(a.off, a.n_bands, a.rows, 1, a.shift, static_cast<int>(id % a.items), tid & 63);
        all = min(t.len - t.first, 1 << a.shift);
        outside = t.band < 0 || t.band >= a.n_bands;
        several = t.len > 1 << a.shift;
        tr = tid / a.octets;
        col = 8 * (tid - tr * a.octets);
        n = works(a) ? all : 0;
    }
    __device__ bool works(const NormArgs& a) const { return tr < a.together; }
    __device__ double2* stats(const NormArgs& a) const { return a.stats + (b * a.n_bands + t.band) * a.groups; }
    __device__ double2* part(const NormArgs& a) const {
        return a.part + (b * slot_count(a.rows, a.shift) + slot_of(t.start, t.first >> a.shift, a.shift)) * a.groups;
    }
    template <class T> __device__ T* at(const View& v, int token) const {
        return norm_row<T>(v, b, t.start + t.first + token) + col;
    }
    template <class T, int N, bool WIDE> __device__ void load(const NormArgs& a, const View& v, frag<T> (&f)[N]) const {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int token = tr + a.together * k;
            f[k] = load8<T, WIDE>(at<T>(v, token < n ? token : 0), token < n ? a.channels - col : 0, col > 0);
        }
    }
};

// f(k, token) for the thread's tokens that exist
template <int N, class F> __device__ __attribute__((always_inline)) inline void norm_tokens(const NormArgs& a, const NormPlace& p, F f) {
    each<N>([&](auto k) __attribute__((always_inline)) {
        const int token = p.tr + a.together * k.value;
        if (token < p.n) f(k.value, token);
    });
}

template <class T, bool WIDE> __device__ inline void norm_zero(const NormArgs& a, const NormPlace& p) {
    const float zero[8] = {};
    for (int token = p.tr; token < p.n; token += a.together) store8<T>(p.at<T>(a.y, token), zero, a.channels - p.col, WIDE);
}

// y of bands of one chunk; else the chunk's statistics.
template <class T, bool WIDE>
__global__ __launch_bounds__(kNormThreads, 2) void k_norm(NormArgs a) {
    constexpr int N = norm_held<T>();
    extern __shared__ __align__(16) double norm_lds[];
    __shared__ double mean[kNormGroups], squares[kNormGroups];
    const int tid = threadIdx.x;
    const NormPlace p(a);
    if (!p.t.live) return;
    if (p.outside) return norm_zero<T, WIDE>(a, p);
    frag<T> x[N];
    p.load<T, N, WIDE>(a, a.x, x);
    const double count = static_cast<double>(p.all) * a.cg;
    double s[8] = {};
    norm_tokens<N>(a, p, [&](int k, int) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] += static_cast<double>(static_cast<float>(x[k][i]));
    });
    if (p.works(a)) norm_put(a, norm_lds, p.tr, p.col, s);
    norm_add_up(a, norm_lds, mean, tid);
    NormOctet o;
    float q[8] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) o.set(i, mean[min(p.col + i, a.channels - 1) / a.cg] / count, 1.0);
    norm_tokens<N>(a, p, [&](int k, int) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = o.hat(static_cast<float>(x[k][i]), i);
            q[i] = fmaf(d, d, q[i]);
        }
    });
    if (p.works(a)) norm_put(a, norm_lds, p.tr, p.col, q);
    norm_add_up(a, norm_lds, squares, tid);
    double2* st = p.several ? p.part(a) : p.stats(a);
    for (int g = tid; g < a.groups; g += kNormThreads)
        st[g] = double2{mean[g] / count, p.several ? squares[g] : 1.0 / sqrt(squares[g] / count + a.eps)};
    if (p.several || !p.works(a)) return;
    o.load_affine<T>(a, p.t.band, p.col);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int g = min(p.col + i, a.channels - 1) / a.cg;
        o.set(i, mean[g] / count, 1.0 / sqrt(squares[g] / count + a.eps));
    }
    by_act(a.act, [&](auto act) __attribute__((always_inline)) {
        norm_tokens<N>(a, p, [&](int k, int token) __attribute__((always_inline)) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] = act_of<act.value>(fmaf(o.hat(static_cast<float>(x[k][i]), i), o.w[i], o.b[i]));
            store8<T>(p.at<T>(a.y, token), v, a.channels - p.col, WIDE);
        });
    });
}

// Statistics of bands of several chunks: a thread joins one group's, in order.
// GRAD: the sums of d and d xh, into the first chunk's slot.
template <bool GRAD> __global__ __launch_bounds__(256) void k_norm_join(NormArgs a) {
    const int64_t id = (a.first_block + blockIdx.x) * 256 + threadIdx.x, place = id / a.groups;
    const int g = static_cast<int>(id % a.groups), band = static_cast<int>(place % a.n_bands);
    const int64_t b = place / a.n_bands;
    if (b >= a.batch) return;
    const int start = band_bound(a.off, a.n_bands, a.rows, band + 1), len = band_bound(a.off, a.n_bands, a.rows, band + 2) - start;
    if (len <= 1 << a.shift) return;
    double2* part = a.part + (b * slot_count(a.rows, a.shift) + slot_of(start, 0, a.shift)) * a.groups + g;
    double2 all = part[0];
    double n = static_cast<double>(1 << a.shift) * a.cg;
    for (int c = 1; c << a.shift < len; ++c) {
        const double2 v = part[static_cast<int64_t>(c) * a.groups];
        if (GRAD) {
            all.x += v.x;
            all.y += v.y;
        } else {   // the mean and the squares of both together
            const double m = static_cast<double>(min(len - (c << a.shift), 1 << a.shift)) * a.cg, d = v.x - all.x;
            all.x += d * (m / (n + m));
            all.y += v.y + d * d * (n * m / (n + m));
            n += m;
        }
    }
    if (GRAD)
        part[0] = all;
    else
        a.stats[place * a.groups + g] = double2{all.x, 1.0 / sqrt(all.y / n + a.eps)};
}

// y of bands of several chunks.
template <class T, bool WIDE>
__global__ __launch_bounds__(kNormThreads) void k_norm_apply(NormArgs a) {
    constexpr int N = norm_held<T>();
    const NormPlace p(a);
    if (!p.t.live || p.outside || !p.several || !p.works(a)) return;
    frag<T> x[N];
    p.load<T, N, WIDE>(a, a.x, x);
    NormOctet o;
    o.load_affine<T>(a, p.t.band, p.col);
    o.load_stats(a, p.stats(a), p.col);
    by_act(a.act, [&](auto act) __attribute__((always_inline)) {
        norm_tokens<N>(a, p, [&](int k, int token) __attribute__((always_inline)) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] = act_of<act.value>(fmaf(o.hat(static_cast<float>(x[k][i]), i), o.w[i], o.b[i]));
            store8<T>(p.at<T>(a.y, token), v, a.channels - p.col, WIDE);
        });
    });
}

// d and xh of 8 values
template <int ACT, class T>
__device__ inline void norm_slope(const NormOctet& o, const frag<T>& x, const frag<T>& dy, float (&hat)[8], float (&dz)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        hat[i] = o.hat(static_cast<float>(x[i]), i);
        float slope;
        act_of<ACT>(fmaf(hat[i], o.w[i], o.b[i]), slope);
        dz[i] = static_cast<float>(dy[i]) * slope;
    }
}

// dx of bands of one chunk; else the chunk's sums of d and d xh. JOINED: dx of
// bands of several chunks, whose sums are in the first one's slot.
template <class T, bool WIDE, bool JOINED>
__global__ __launch_bounds__(kNormThreads, 2) void k_norm_grad(NormArgs a) {
    constexpr int N = norm_held<T>() / 2;
    extern __shared__ __align__(16) double norm_lds[];
    __shared__ double first[JOINED ? 1 : kNormGroups], second[JOINED ? 1 : kNormGroups];
    const int tid = threadIdx.x;
    const NormPlace p(a);
    if (!p.t.live || (JOINED && (p.outside || !p.several))) return;
    if (p.outside) return norm_zero<T, WIDE>(a, p);
    frag<T> x[N], dy[N];
    p.load<T, N, WIDE>(a, a.x, x);
    p.load<T, N, WIDE>(a, a.dy, dy);
    NormOctet o;
    if (p.works(a)) {
        o.load_affine<T>(a, p.t.band, p.col);
        o.load_stats(a, p.stats(a), p.col);
    }
    if constexpr (!JOINED) {
        float s1[8] = {}, s2[8] = {};
        by_act(a.act, [&](auto act) __attribute__((always_inline)) {
            norm_tokens<N>(a, p, [&](int k, int) __attribute__((always_inline)) {
                float hat[8], dz[8];
                norm_slope<act.value, T>(o, x[k], dy[k], hat, dz);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    s1[i] = fmaf(dz[i], o.w[i], s1[i]);
                    s2[i] = fmaf(dz[i] * o.w[i], hat[i], s2[i]);
                }
            });
        });
        if (p.works(a)) norm_put(a, norm_lds, p.tr, p.col, s1);
        norm_add_up(a, norm_lds, first, tid);
        if (p.works(a)) norm_put(a, norm_lds, p.tr, p.col, s2);
        norm_add_up(a, norm_lds, second, tid);
        if (p.several) {
            double2* to = p.part(a);
            for (int g = tid; g < a.groups; g += kNormThreads) to[g] = double2{first[g], second[g]};
            return;
        }
    }
    const double2* sums = JOINED ? p.part(a) - static_cast<int64_t>(p.t.first >> a.shift) * a.groups : nullptr;
    const double share = 1.0 / (static_cast<double>(p.t.len) * a.cg);
    float m1[8], m2[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int g = min(p.col + i, a.channels - 1) / a.cg;
        m1[i] = static_cast<float>((JOINED ? sums[g].x : first[g]) * share);
        m2[i] = static_cast<float>((JOINED ? sums[g].y : second[g]) * share);
    }
    by_act(a.act, [&](auto act) __attribute__((always_inline)) {
        norm_tokens<N>(a, p, [&](int k, int token) __attribute__((always_inline)) {
            float hat[8], dz[8], v[8];
            norm_slope<act.value, T>(o, x[k], dy[k], hat, dz);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = o.rstd[i] * (fmaf(dz[i], o.w[i], -m1[i]) - hat[i] * m2[i]);
            store8<T>(p.at<T>(a.y, token), v, a.channels - p.col, WIDE);
        });
    });
}

// dw and db: sums over 2^weight_shift rows of a band, token r % len of signal
// r / len, into the item's place.
template <class T, bool WIDE>
__global__ __launch_bounds__(kNormThreads) void k_norm_weight(NormArgs a) {
    extern __shared__ __align__(16) float norm_sums[];   // [together][2][8 octets]
    const int tid = threadIdx.x, lane = tid & 63;
    const unsigned id = die_order(blockIdx.x, gridDim.x);
    const Tile<int64_t> t = find_tile<int64_t>(a.off, a.n_bands, a.rows, a.batch, a.weight_shift, id, lane);
    if (!t.live || t.band < 0 || t.band >= a.n_bands) return;
    const int64_t end = min(t.first + (int64_t(1) << a.weight_shift), static_cast<int64_t>(t.len) * a.batch);
    const int tr = tid / a.octets, col = 8 * (tid - tr * a.octets), width = 8 * a.octets;
    if (tr < a.together) {
        NormOctet o;
        o.load_affine<T>(a, t.band, col);
        float s1[8] = {}, s2[8] = {};
        int64_t signal = -1;
        by_act(a.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll 2
            for (int64_t r = t.first + tr; r < end; r += a.together) {
                const int64_t b = r / t.len, row = t.start + (r - b * t.len);
                const frag<T> x = load8<T, WIDE>(norm_row<T>(a.x, b, row) + col, a.channels - col, col > 0);
                const frag<T> dy = load8<T, WIDE>(norm_row<T>(a.dy, b, row) + col, a.channels - col, col > 0);
                if (b != signal) o.load_stats(a, a.stats + (b * a.n_bands + t.band) * a.groups, col);
                signal = b;
                float hat[8], dz[8];
                norm_slope<act.value, T>(o, x, dy, hat, dz);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    s1[i] = fmaf(dz[i], hat[i], s1[i]);
                    s2[i] += dz[i];
                }
            }
        });
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            norm_sums[2 * tr * width + col + i] = s1[i];
            norm_sums[(2 * tr + 1) * width + col + i] = s2[i];
        }
    }
    __syncthreads();
    float* to = a.sums + static_cast<int64_t>(id) * 2 * a.channels;
    for (int e = tid; e < 2 * a.channels; e += kNormThreads) {
        const int which = e >= a.channels, c = e - which * a.channels;
        float s = norm_sums[which * width + c];
        for (int r = 1; r < a.together; ++r) s += norm_sums[(2 * r + which) * width + c];
        to[e] = s;
    }
}

// Adds up the items of each band, in order.
template <class T> __global__ __launch_bounds__(256) void k_norm_weight_join(NormArgs a) {
    const int64_t id = (a.first_block + blockIdx.x) * 256 + threadIdx.x;
    const int c = static_cast<int>(id % a.channels), band = static_cast<int>(id / a.channels);
    if (id >= static_cast<int64_t>(a.n_bands) * a.channels) return;
    const int64_t b0 = band_bound(a.off, a.n_bands, a.rows, band + 1), b1 = band_bound(a.off, a.n_bands, a.rows, band + 2);
    const int64_t n = b1 > b0 ? (b1 - b0) * a.batch : 0;
    const int64_t count = (n + (int64_t(1) << a.weight_shift) - 1) >> a.weight_shift;
    const float* s = a.sums + (((b0 * a.batch) >> a.weight_shift) + band + 1) * 2 * a.channels + c;
    float dw = 0.f, db = 0.f;
#pragma unroll 4
    for (int64_t i = 0; i < count; ++i) {
        dw += s[i * 2 * a.channels];
        db += s[(2 * i + 1) * a.channels];
    }
    if (a.dw) static_cast<T*>(a.dw)[id] = static_cast<T>(dw);
    if (a.db) static_cast<T*>(a.db)[id] = static_cast<T>(db);
}

}  // namespace nsl
