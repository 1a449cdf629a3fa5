// Group norm with an activation on ragged rows, channels last.
//
// A group's statistics go over its cg channels and all tokens of one band of one signal:
//   xh = (x - mean) rstd   z = w xh + b   y = act(z)        (w, b: of the band and the channel)
//   dz = dy act'(z)   d = w dz   dx = rstd (d - mean(d) - xh mean(d xh))
//   db = sum dz   dw = sum dz xh     over the band's tokens of all signals
//
// A workgroup takes a chunk of a band's tokens, all channels; a thread 8
// channels of every n-th token. What a chunk holds stays in registers from the
// load to the store: bands of one chunk are read once. Longer bands are read
// twice: first in parts of several chunks for their sums, which a small kernel
// joins, then chunk by chunk. Statistics are summed in 64 bits, of differences
// from a value of the group itself, so that a level far above them does not hide
// the variance; d's sums are those that db and dw are made of, times w.
#pragma once
#include "act.hpp"

namespace nsl {

constexpr int kNormThreads = 512, kNormChannels = 8 * kNormThreads, kNormGroups = 1024;   // the most of each
// Octets of x that a thread holds (half as many where dy is held beside it).
template <class T> constexpr int norm_held() { return sizeof(T) == 4 ? 4 : 8; }

struct NormArgs {
    View x, y, dy;                // (the gradient's result dx is y)
    const void *w, *b;            // [n_bands][channels] or NULL
    int64_t w_band, b_band;       // their strides from band to band
    void *dw, *db;
    double2* stats;               // [batch][n_bands][groups]: mean, rstd
    double2* part;                // [batch][parts][groups]: a part's (sum v, sum v^2), v = x - norm_pivot, or (sum d, sum d xh)
    float* sums;                  // dw and db before they are joined, [2][channels] each (NULL: not wanted):
                                  // [batch][n_bands] of bands of one chunk, then [batch][parts]; or of k_norm_weight's items
    const int64_t* off;
    int rows, n_bands, batch, channels, groups, cg;
    int threads;                  // of a workgroup
    int octets, together;         // octets of a token's channels, tokens that a workgroup takes at once
    int shift, part_shift;        // of a chunk's tokens; of a part's
    int weight_shift;             // of the rows of an item of k_norm_weight
    unsigned parts;               // of a signal, the empty ones among them
    int zeros;                    // workgroups of a signal for the tokens that no band holds
    int64_t first_block, first_signal;   // of a launch, where a call takes several
    int act;
    bool octet_groups;            // a group is whole octets of channels
    double eps;
};

template <class T> __device__ inline T* norm_row(const View& v, int64_t b, int64_t row) {
    return reinterpret_cast<T*>(v.data) + b * v.batch + row * v.row;
}

// A thread's 8 channels: their groups, and what is applied to them. Values are
// taken from the mean before they are scaled, and the mean's rest in 32 bits
// after that: equal values give 0 at any level, also where eps alone is the scale.
template <class T> struct NormOctet {
    static constexpr bool kExact = sizeof(T) == 4;
    int group[8];
    float high[8], low[8], rstd[8], w[8], b[8];   // (low: of the mean's rest, times -rstd)
    __device__ NormOctet(const NormArgs& a, int col) {
        int g = col / a.cg, r = col - g * a.cg;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            group[i] = min(g, a.groups - 1);
            if (++r == a.cg) {
                r = 0;
                ++g;
            }
        }
    }
    __device__ void load_affine(const NormArgs& a, int band, int col) {
        const T* wp = static_cast<const T*>(a.w) + band * a.w_band + col;
        const T* bp = static_cast<const T*>(a.b) + band * a.b_band + col;
        const frag<T> fw = load8<T, false>(wp, a.w ? a.channels - col : 0), fb = load8<T, false>(bp, a.b ? a.channels - col : 0);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w[i] = a.w ? static_cast<float>(fw[i]) : 1.f;
            b[i] = static_cast<float>(fb[i]);
        }
    }
    // f(group) gives its (mean, rstd)
    template <class F> __device__ __attribute__((always_inline)) void set(const NormArgs& a, F f) {
        auto put = [&](int i, double2 v) __attribute__((always_inline)) {
            rstd[i] = static_cast<float>(v.y);
            high[i] = static_cast<float>(v.x);
            low[i] = static_cast<float>((static_cast<double>(high[i]) - v.x) * v.y);
        };
        if (a.octet_groups) {
            const double2 v = f(group[0]);
            each<8>([&](auto i) __attribute__((always_inline)) { put(i.value, v); });
        } else {
            each<8>([&](auto i) __attribute__((always_inline)) { put(i.value, f(group[i.value])); });
        }
    }
    __device__ float hat(T x, int i) const { return fmaf(static_cast<float>(x) - high[i], rstd[i], low[i]); }
    // For `out` alone: the mean's rest goes into b, so that it takes no registers.
    __device__ void fold() {
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = fmaf(low[i], w[i], b[i]);
    }
    template <int ACT> __device__ frag<T> out(frag<T> x) const {
        frag<T> y;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            y[i] = static_cast<T>(act_of<ACT, kExact>(fmaf((static_cast<float>(x[i]) - high[i]) * rstd[i], w[i], b[i])));
        return y;
    }
    // xh and dz
    template <int ACT> __device__ void slope(frag<T> x, frag<T> dy, float (&xh)[8], float (&dz)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            xh[i] = hat(x[i], i);
            float d;
            act_of<ACT, kExact>(fmaf(xh[i], w[i], b[i]), d);
            dz[i] = static_cast<float>(dy[i]) * d;
        }
    }
};

template <class T> __device__ inline void store8(T* p, frag<T> f, int n, bool wide) {
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

// Sums over a workgroup's tokens and channels, in a fixed order. `cells` holds
// a row of 8 octets values for each of the tokens taken at once, channel c at
// norm_cell(c) of it, which spreads a wave's writes over the banks. norm_columns
// leaves the sum of a channel in parts, [part * width + cell]: a thread adds
// every parts-th row into its own first one. All threads; ends with a barrier.
__device__ inline int norm_cell(const NormArgs& a, int c) { return (c & 7) * a.octets + (c >> 3); }
__device__ inline int norm_parts(const NormArgs& a) { return min(a.together, max(1, a.threads / (8 * a.octets))); }
template <class V> __device__ inline void norm_columns(const NormArgs& a, V* cells, bool works, int tr, int col, const V (&v)[8], int tid) {
    const int width = 8 * a.octets, parts = norm_parts(a);
    if (works) {
#pragma unroll
        for (int i = 0; i < 8; ++i) cells[tr * width + norm_cell(a, col + i)] = v[i];
    }
    __syncthreads();
    if (parts < a.together) {
        for (int at = tid; at < width * parts; at += a.threads) {
            V s = cells[at];
            for (int r = at + width * parts; r < width * a.together; r += width * parts) s += cells[r];
            cells[at] = s;
        }
    }
    __syncthreads();
}
// result[g] = the sum of f(cell, channel) over a group's channels and the parts. Ends with a barrier.
template <class F> __device__ __attribute__((always_inline)) inline void norm_groups(const NormArgs& a, double* result, int tid, F f) {
    const int width = 8 * a.octets, parts = norm_parts(a), each_group = a.cg * parts;
    if (each_group <= 8 || a.groups >= a.threads / 4) {
        for (int g = tid; g < a.groups; g += a.threads) {
            double s = 0.0;
            for (int p = 0; p < parts; ++p)
                for (int c = g * a.cg; c < (g + 1) * a.cg; ++c) s += f(p * width + norm_cell(a, c), c);
            result[g] = s;
        }
    } else {
        const int lane = tid & 63;
        for (int g = wave_number(); g < a.groups; g += a.threads / 64) {
            double s = 0.0;
            for (int i = lane; i < each_group; i += 64) {
                const int p = i / a.cg, c = g * a.cg + i - p * a.cg;
                s += f(p * width + norm_cell(a, c), c);
            }
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
    int all, n, tr, col;   // all: the chunk's (or part's) tokens
    unsigned item;
    bool outside, several;
    __device__ NormPlace(const NormArgs& a, unsigned items, int shift) {
        const unsigned id = last_first(blockIdx.x, gridDim.x);
        const int tid = threadIdx.x;
        item = id % items;
        b = a.first_signal + id / items;
        t = find_tile<int>(a.off, a.n_bands, a.rows, 1, shift, static_cast<int>(item), tid & 63);
        all = min(t.len - t.first, 1 << shift);
        outside = t.band < 0 || t.band >= a.n_bands;
        several = t.len > 1 << a.shift;
        tr = tid / a.octets;
        col = 8 * (tid - tr * a.octets);
        n = works(a) ? all : 0;
    }
    // One workgroup a band: all of its tokens (several: more than a chunk); behind
    // the bands a.zeros workgroups a signal, which share the tokens that no band holds.
    __device__ explicit NormPlace(const NormArgs& a) {
        const unsigned items = a.n_bands + a.zeros, id = gridDim.x - 1 - blockIdx.x;
        const int tid = threadIdx.x;
        item = id % items;
        b = a.first_signal + id / items;
        t.band = static_cast<int>(item);
        outside = t.band >= a.n_bands;
        t.start = outside ? 0 : band_bound(a.off, a.n_bands, a.rows, t.band + 1);
        const int end = outside ? 0 : band_bound(a.off, a.n_bands, a.rows, t.band + 2);
        t.len = end > t.start ? end - t.start : 0;
        t.first = 0;
        t.live = outside || t.len > 0;
        all = t.len;
        several = t.len > 1 << a.shift;
        tr = tid / a.octets;
        col = 8 * (tid - tr * a.octets);
        n = works(a) ? all : 0;
    }
    __device__ bool works(const NormArgs& a) const { return tr < a.together; }
    __device__ double2* stats(const NormArgs& a) const { return a.stats + (b * a.n_bands + t.band) * a.groups; }
    template <class T> __device__ T* at(const View& v, int token) const {
        return norm_row<T>(v, b, t.start + t.first + token) + col;
    }
    template <class T, int N, bool WIDE> __device__ void load(const NormArgs& a, const View& v, frag<T> (&f)[N], int from = 0) const {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int token = from + tr + a.together * k;
            f[k] = load8<T, WIDE>(at<T>(v, token < n ? token : 0), token < n ? a.channels - col : 0, col > 0);
        }
    }
};
// Where the parts of a band lie among a signal's.
__device__ inline int64_t norm_part(const NormArgs& a, int64_t b, int band, int start) {
    return b * a.parts + (start >> a.part_shift) + band + 1;
}

// 1 / sqrt(var + eps). What rounding left below 0 is 0; a NaN, of a group that
// holds an infinity or NaN, stays one.
__device__ inline double norm_rstd(double var, double eps) { return 1.0 / sqrt((var < 0.0 ? 0.0 : var) + eps); }

// f(k, token) for the thread's tokens that exist
template <int N, class F> __device__ __attribute__((always_inline)) inline void norm_tokens(const NormArgs& a, const NormPlace& p, F f) {
    each<N>([&](auto k) __attribute__((always_inline)) {
        const int token = p.tr + a.together * k.value;
        if (token < p.n) f(k.value, token);
    });
}

template <class T, bool WIDE> __device__ inline void norm_zero(const NormArgs& a, const NormPlace& p) {
    const int first = band_bound(a.off, a.n_bands, a.rows, 1), last = band_bound(a.off, a.n_bands, a.rows, a.n_bands + 1);
    const int step = a.zeros * a.together;
    if (!p.works(a)) return;
    for (int64_t row = (p.item - a.n_bands) * a.together + p.tr; row < a.rows; row += step)
        if (row < first || row >= last) store8<T>(norm_row<T>(a.y, p.b, row) + p.col, zero8<T>(), a.channels - p.col, WIDE);
}

template <class T, int N, bool WIDE> __device__ inline void norm_out(const NormArgs& a, const NormPlace& p, const NormOctet<T>& o, const frag<T> (&x)[N]) {
    by_act(a.act, [&](auto act) __attribute__((always_inline)) {
        norm_tokens<N>(a, p, [&](int k, int token) __attribute__((always_inline)) {
            store8<T>(p.at<T>(a.y, token), o.template out<act.value>(x[k]), a.channels - p.col, WIDE);
        });
    });
}

// y of bands of one chunk, and zeros where no band is: the mean first, then the
// squares of the differences from it. Bound by the chain of loads, sums and
// barriers of a workgroup: 64 signals of one token of 128 channels 8.3 us.
template <class T, bool WIDE>
__global__ __launch_bounds__(kNormThreads, 2) void k_norm(NormArgs a) {
    constexpr int N = norm_held<T>();
    extern __shared__ __align__(16) double norm_lds[];
    double *const mean = norm_lds + 8 * a.octets * a.together, *const squares = mean + a.groups;   // [groups]
    const int tid = threadIdx.x;
    const NormPlace p(a);
    if (!p.t.live) return;
    if (p.outside) return norm_zero<T, WIDE>(a, p);
    if (p.several) return;
    frag<T> x[N];
    p.load<T, N, WIDE>(a, a.x, x);
    const double count = static_cast<double>(p.all) * a.cg;   // (divided by: the mean of equal values is theirs)
    auto cell = [&](int at, int) { return norm_lds[at]; };
    double s[8] = {};
    norm_tokens<N>(a, p, [&](int k, int) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] += static_cast<double>(static_cast<float>(x[k][i]));
    });
    norm_columns(a, norm_lds, p.works(a), p.tr, p.col, s, tid);
    norm_groups(a, mean, tid, cell);
    for (int g = tid; g < a.groups; g += a.threads) mean[g] /= count;
    __syncthreads();
    NormOctet<T> o(a, p.col);
    float m[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        m[i] = static_cast<float>(mean[o.group[i]]);   // (what it is off by is made up for below)
        s[i] = 0.0;
    }
    norm_tokens<N>(a, p, [&](int k, int) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = static_cast<float>(x[k][i]) - m[i];
            s[i] = fma(static_cast<double>(d), static_cast<double>(d), s[i]);
        }
    });
    norm_columns(a, norm_lds, p.works(a), p.tr, p.col, s, tid);
    norm_groups(a, squares, tid, cell);
    // the mean of the squared differences from m is the variance and the square of the mean's own difference from m
    double2* st = p.stats(a);
    for (int g = tid; g < a.groups; g += a.threads) {
        const double off = mean[g] - static_cast<double>(static_cast<float>(mean[g]));
        squares[g] = norm_rstd(squares[g] / count - off * off, a.eps);
        if (a.stats) st[g] = double2{mean[g], squares[g]};
    }
    __syncthreads();
    if (!p.works(a)) return;
    o.load_affine(a, p.t.band, p.col);
    o.set(a, [&](int g) { return double2{mean[g], squares[g]}; });
    o.fold();
    norm_out<T, N, WIDE>(a, p, o, x);
}

// What a group's values of a longer band are summed as differences from: its first one.
template <class T> __device__ inline double norm_pivot(const NormArgs& a, int64_t b, int start, int group) {
    return static_cast<double>(static_cast<float>(norm_row<const T>(a.x, b, start)[group * a.cg]));
}

// The sums of v and v^2, v = x - norm_pivot, of the parts of longer bands. 446,932 tokens of 128
// channels, bfloat16, 221 bands: 28 us (4.1 TB/s); 710,680 of 77, float16: 51, as
// loads at odd addresses take four accesses of the first cache each.
template <class T, bool WIDE>
__global__ __launch_bounds__(kNormThreads, 2) void k_norm_sum(NormArgs a) {
    constexpr int N = 4;
    extern __shared__ __align__(16) double norm_lds[];
    double *const sum = norm_lds + 8 * a.octets * a.together, *const squares = sum + a.groups;   // [groups]
    const int tid = threadIdx.x;
    const NormPlace p(a, a.parts, a.part_shift);
    if (!p.t.live || p.outside || !p.several) return;
    double s[8] = {}, q[8] = {}, pivot[8];
    frag<T> x[N], next[N];
    p.load<T, N, WIDE>(a, a.x, next);
    const NormOctet<T> o(a, p.col);
    each<8>([&](auto i) __attribute__((always_inline)) {
        pivot[i.value] = i.value && a.octet_groups ? pivot[0] : norm_pivot<T>(a, p.b, p.t.start, o.group[i.value]);
    });
    for (int from = 0; from < p.all; from += N * a.together) {
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = next[k];
        p.load<T, N, WIDE>(a, a.x, next, from + N * a.together);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (from + p.tr + a.together * k >= p.n) break;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double v = static_cast<double>(static_cast<float>(x[k][i])) - pivot[i];
                s[i] += v;
                q[i] = fma(v, v, q[i]);
            }
        }
    }
    auto cell = [&](int at, int) { return norm_lds[at]; };
    norm_columns(a, norm_lds, p.works(a), p.tr, p.col, s, tid);
    norm_groups(a, sum, tid, cell);
    norm_columns(a, norm_lds, p.works(a), p.tr, p.col, q, tid);
    norm_groups(a, squares, tid, cell);
    double2* to = a.part + (p.b * a.parts + p.item) * a.groups;
    for (int g = tid; g < a.groups; g += a.threads) to[g] = double2{sum[g], squares[g]};
}

// Joins the parts of longer bands, in order, a group a thread: into their
// statistics, or (GRAD) their means of d and d xh into the first part's place.
template <class T, bool GRAD> __global__ __launch_bounds__(256) void k_norm_join(NormArgs a) {
    const int64_t id = (a.first_block + blockIdx.x) * 256 + threadIdx.x, place = id / a.groups;
    const int g = static_cast<int>(id % a.groups), band = static_cast<int>(place % a.n_bands);
    const int64_t b = place / a.n_bands;
    if (b >= a.batch) return;
    const int start = band_bound(a.off, a.n_bands, a.rows, band + 1), len = band_bound(a.off, a.n_bands, a.rows, band + 2) - start;
    if (len <= 1 << a.shift) return;
    double2* part = a.part + norm_part(a, b, band, start) * a.groups + g;
    const int count = (len + (1 << a.part_shift) - 1) >> a.part_shift;
    double2 all = {0.0, 0.0};
#pragma unroll 8
    for (int c = 0; c < count; ++c) all += part[static_cast<int64_t>(c) * a.groups];
    all /= static_cast<double>(len) * a.cg;
    if (GRAD)
        part[0] = all;
    else
        a.stats[place * a.groups + g] = double2{norm_pivot<T>(a, b, start, g) + all.x, norm_rstd(all.y - all.x * all.x, a.eps)};
}

// y of longer bands, a part a workgroup: the next tokens are on their way while
// these are computed. The same two cases: 37 us, much of x coming from the
// memory-side cache, and 84.
template <class T, bool WIDE>
__global__ __launch_bounds__(kNormThreads, 2) void k_norm_apply(NormArgs a) {
    constexpr int N = norm_held<T>() / 2;
    const NormPlace p(a, a.parts, a.part_shift);
    if (!p.t.live || p.outside || !p.several || !p.works(a)) return;
    frag<T> x[N], next[N];
    p.load<T, N, WIDE>(a, a.x, next);
    NormOctet<T> o(a, p.col);
    const double2* st = p.stats(a);
    o.load_affine(a, p.t.band, p.col);
    o.set(a, [&](int g) { return st[g]; });
    o.fold();
    by_act(a.act, [&](auto act) __attribute__((always_inline)) {
        for (int from = 0; from < p.n; from += N * a.together) {
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] = next[k];
            p.load<T, N, WIDE>(a, a.x, next, from + N * a.together);
            each<N>([&](auto k) __attribute__((always_inline)) {
                const int token = from + p.tr + a.together * k.value;
                if (token < p.n) store8<T>(p.at<T>(a.y, token), o.template out<act.value>(x[k.value]), a.channels - p.col, WIDE);
            });
        }
    });
}

// From the sums of dz and dz xh of a thread's 8 channels: those of the
// workgroup's channels, to `to` (NULL: not wanted), and times w, of its groups.
template <class T>
__device__ inline void norm_grad_sums(const NormArgs& a, const NormPlace& p, float2* cells, const float2 (&s)[8], float* to,
                                      double* first, double* second, int tid) {
    const int width = 8 * a.octets, parts = norm_parts(a);
    norm_columns(a, cells, p.works(a), p.tr, p.col, s, tid);
    if (to) {
        for (int c = tid; c < a.channels; c += a.threads) {
            float2 v = cells[norm_cell(a, c)];
            for (int k = 1; k < parts; ++k) v += cells[k * width + norm_cell(a, c)];
            to[c] = v.y;
            to[a.channels + c] = v.x;
        }
    }
    const T* wp = static_cast<const T*>(a.w) + p.t.band * a.w_band;
    auto w = [&](int c) { return a.w ? static_cast<double>(static_cast<float>(wp[c])) : 1.0; };
    norm_groups(a, first, tid, [&](int at, int c) { return cells[at].x * w(c); });
    norm_groups(a, second, tid, [&](int at, int c) { return cells[at].y * w(c); });
}

// The means of d and d xh of a thread's 8 channels' groups, and dx.
template <class T> struct NormMeans {
    float first[8], second[8];
    template <class F> __device__ NormMeans(const NormArgs& a, const NormOctet<T>& o, F means) {
        each<8>([&](auto i) __attribute__((always_inline)) {
            if (i.value && a.octet_groups) {
                first[i.value] = first[0];
                second[i.value] = second[0];
            } else {
                const double2 v = means(o.group[i.value]);
                first[i.value] = static_cast<float>(v.x);
                second[i.value] = static_cast<float>(v.y);
            }
        });
    }
    template <int ACT> __device__ frag<T> dx(const NormOctet<T>& o, frag<T> x, frag<T> dy) const {
        float xh[8], dz[8];
        o.template slope<ACT>(x, dy, xh, dz);
        frag<T> f;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = static_cast<T>(o.rstd[i] * (fmaf(dz[i], o.w[i], -first[i]) - xh[i] * second[i]));
        return f;
    }
};

template <int ACT, class T> __device__ inline void norm_grad_add(const NormOctet<T>& o, frag<T> x, frag<T> dy, float2 (&s)[8]) {
    float xh[8], dz[8];
    o.template slope<ACT>(x, dy, xh, dz);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        s[i].x += dz[i];
        s[i].y = fmaf(dz[i], xh[i], s[i].y);
    }
}

// dx of bands of one chunk, and what they add to dw and db.
template <class T, bool WIDE>
__global__ __launch_bounds__(kNormThreads, 2) void k_norm_grad(NormArgs a) {
    constexpr int N = norm_held<T>() / 2;
    extern __shared__ __align__(16) double norm_lds[];
    double *const first = norm_lds + 8 * a.octets * a.together, *const second = first + a.groups;   // [groups]
    const int tid = threadIdx.x;
    const NormPlace p(a);
    if (!p.t.live) return;
    if (p.outside) {
        if (a.y.data) norm_zero<T, WIDE>(a, p);
        return;
    }
    if (p.several) return;
    frag<T> x[N], dy[N];
    p.load<T, N, WIDE>(a, a.x, x);
    p.load<T, N, WIDE>(a, a.dy, dy);
    NormOctet<T> o(a, p.col);
    if (p.works(a)) {
        const double2* st = p.stats(a);
        o.load_affine(a, p.t.band, p.col);
        o.set(a, [&](int g) { return st[g]; });
    }
    float2 s[8] = {};
    by_act(a.act, [&](auto act) __attribute__((always_inline)) {
        norm_tokens<N>(a, p, [&](int k, int) __attribute__((always_inline)) { norm_grad_add<act.value>(o, x[k], dy[k], s); });
    });
    norm_grad_sums<T>(a, p, reinterpret_cast<float2*>(norm_lds), s,
                      a.sums ? a.sums + (p.b * a.n_bands + p.t.band) * 2 * a.channels : nullptr, first, second, tid);
    if (!a.y.data) return;
    const double share = 1.0 / (static_cast<double>(p.t.len) * a.cg);
    const NormMeans<T> means(a, o, [&](int g) { return double2{first[g] * share, second[g] * share}; });
    by_act(a.act, [&](auto act) __attribute__((always_inline)) {
        norm_tokens<N>(a, p, [&](int k, int token) __attribute__((always_inline)) {
            store8<T>(p.at<T>(a.y, token), means.template dx<act.value>(o, x[k], dy[k]), a.channels - p.col, WIDE);
        });
    });
}

// The sums of d and d xh of the parts of longer bands, and what they add to dw
// and db. 446,932 tokens of 128 channels, bfloat16: 58 us (3.9 TB/s).
template <class T, bool WIDE>
__global__ __launch_bounds__(kNormThreads, 2) void k_norm_grad_sum(NormArgs a) {
    constexpr int N = 2;
    extern __shared__ __align__(16) double norm_lds[];
    double *const first = norm_lds + 8 * a.octets * a.together, *const second = first + a.groups;   // [groups]
    const int tid = threadIdx.x;
    const NormPlace p(a, a.parts, a.part_shift);
    if (!p.t.live || p.outside || !p.several) return;
    frag<T> x[N], dy[N], x_next[N], dy_next[N];
    p.load<T, N, WIDE>(a, a.x, x_next);
    p.load<T, N, WIDE>(a, a.dy, dy_next);
    NormOctet<T> o(a, p.col);
    if (p.works(a)) {
        const double2* st = p.stats(a);
        o.load_affine(a, p.t.band, p.col);
        o.set(a, [&](int g) { return st[g]; });
    }
    float2 s[8] = {};
    by_act(a.act, [&](auto act) __attribute__((always_inline)) {
        for (int from = 0; from < p.all; from += N * a.together) {
#pragma unroll
            for (int k = 0; k < N; ++k) {
                x[k] = x_next[k];
                dy[k] = dy_next[k];
            }
            p.load<T, N, WIDE>(a, a.x, x_next, from + N * a.together);
            p.load<T, N, WIDE>(a, a.dy, dy_next, from + N * a.together);
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (from + p.tr + a.together * k < p.n) norm_grad_add<act.value>(o, x[k], dy[k], s);
        }
    });
    norm_grad_sums<T>(a, p, reinterpret_cast<float2*>(norm_lds), s,
                      a.sums ? a.sums + (static_cast<int64_t>(a.batch) * a.n_bands + p.b * a.parts + p.item) * 2 * a.channels : nullptr,
                      first, second, tid);
    double2* to = a.part + (p.b * a.parts + p.item) * a.groups;
    for (int g = tid; g < a.groups; g += a.threads) to[g] = double2{first[g], second[g]};
}

// dx of longer bands, a part a workgroup: 61 us (5.6 TB/s with the memory-side cache).
template <class T, bool WIDE>
__global__ __launch_bounds__(kNormThreads, 2) void k_norm_grad_apply(NormArgs a) {
    constexpr int N = 2;
    const NormPlace p(a, a.parts, a.part_shift);
    if (!p.t.live || p.outside || !p.several || !p.works(a)) return;
    frag<T> x[N], dy[N], x_next[N], dy_next[N];
    p.load<T, N, WIDE>(a, a.x, x_next);
    p.load<T, N, WIDE>(a, a.dy, dy_next);
    NormOctet<T> o(a, p.col);
    const double2 *st = p.stats(a), *sums = a.part + norm_part(a, p.b, p.t.band, p.t.start) * a.groups;
    o.load_affine(a, p.t.band, p.col);
    o.set(a, [&](int g) { return st[g]; });
    const NormMeans<T> means(a, o, [&](int g) { return sums[g]; });
    by_act(a.act, [&](auto act) __attribute__((always_inline)) {
        for (int from = 0; from < p.n; from += N * a.together) {
#pragma unroll
            for (int k = 0; k < N; ++k) {
                x[k] = x_next[k];
                dy[k] = dy_next[k];
            }
            p.load<T, N, WIDE>(a, a.x, x_next, from + N * a.together);
            p.load<T, N, WIDE>(a, a.dy, dy_next, from + N * a.together);
            each<N>([&](auto k) __attribute__((always_inline)) {
                const int token = from + p.tr + a.together * k.value;
                if (token < p.n)
                    store8<T>(p.at<T>(a.y, token), means.template dx<act.value>(o, x[k.value], dy[k.value]), a.channels - p.col, WIDE);
            });
        }
    });
}

// dw and db where bands are so short that what each adds to them would be as
// much as the data: sums over 2^weight_shift rows of a band, token r % len of
// signal r / len.
template <class T, bool WIDE>
__global__ __launch_bounds__(kNormThreads, 2) void k_norm_weight(NormArgs a) {
    extern __shared__ __align__(16) double norm_lds[];
    float2* cells = reinterpret_cast<float2*>(norm_lds);
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t id = a.first_block + die_order(blockIdx.x, gridDim.x);
    const Tile<int64_t> t = find_tile<int64_t>(a.off, a.n_bands, a.rows, a.batch, a.weight_shift, id, lane);
    if (!t.live || t.band < 0 || t.band >= a.n_bands) return;
    const int64_t end = min(t.first + (int64_t(1) << a.weight_shift), static_cast<int64_t>(t.len) * a.batch);
    const int tr = tid / a.octets, col = 8 * (tid - tr * a.octets);
    const bool works = tr < a.together;
    float2 s[8] = {};
    if (works) {
        NormOctet<T> o(a, col);
        o.load_affine(a, t.band, col);
        int64_t signal = -1;
        by_act(a.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll 2
            for (int64_t r = t.first + tr; r < end; r += a.together) {
                const int64_t b = r / t.len, row = t.start + (r - b * t.len);
                const frag<T> x = load8<T, WIDE>(norm_row<T>(a.x, b, row) + col, a.channels - col, col > 0);
                const frag<T> dy = load8<T, WIDE>(norm_row<T>(a.dy, b, row) + col, a.channels - col, col > 0);
                if (b != signal) {
                    const double2* st = a.stats + (b * a.n_bands + t.band) * a.groups;
                    o.set(a, [&](int g) { return st[g]; });
                }
                signal = b;
                norm_grad_add<act.value>(o, x, dy, s);
            }
        });
    }
    norm_columns(a, cells, works, tr, col, s, tid);
    float* to = a.sums + id * 2 * a.channels;
    for (int c = tid; c < a.channels; c += a.threads) {
        float2 v = cells[norm_cell(a, c)];
        for (int k = 1; k < norm_parts(a); ++k) v += cells[k * 8 * a.octets + norm_cell(a, c)];
        to[c] = v.y;
        to[a.channels + c] = v.x;
    }
}

// Adds up what was left for dw and db of each band, in order: by k_norm_weight,
// or with `by_chunk` by the other two. In 64 bits: long rows leave thousands, and
// terms of one sign may all be rounded the same way. S of 1: a thread a channel;
// else the S waves of a workgroup share what was left for 64 channels (8,192 items
// of 1,032 channels: 103 us, and 637 with one thread a channel).
template <class T, int S> __global__ __launch_bounds__(S == 1 ? 256 : 64 * S) void k_norm_weight_join(NormArgs a, bool by_chunk) {
    __shared__ double2 sums[S][64];
    const int64_t block = a.first_block + blockIdx.x;
    const int lane = threadIdx.x & 63, wave = S == 1 ? 0 : wave_number(), slabs = (a.channels + 63) / 64;
    const int64_t id = block * 256 + threadIdx.x;
    const int c = S == 1 ? static_cast<int>(id % a.channels) : static_cast<int>(block % slabs) * 64 + lane;
    const int64_t band = S == 1 ? id / a.channels : block / slabs;
    const bool there = band < a.n_bands && c < a.channels;
    double2 all = {0.0, 0.0};   // dw, db
    if (there) {
        const int at = static_cast<int>(band), start = band_bound(a.off, a.n_bands, a.rows, at + 1);
        const int len = max(band_bound(a.off, a.n_bands, a.rows, at + 2) - start, 0);
        // row (i, j) of i < signals, j < each lies at first + i apart + j
        int64_t first, apart = 0, signals = a.batch, each = 1;
        if (!by_chunk) {
            first = ((static_cast<int64_t>(start) * a.batch) >> a.weight_shift) + band + 1;
            signals = 1;
            each = (static_cast<int64_t>(len) * a.batch + (int64_t(1) << a.weight_shift) - 1) >> a.weight_shift;
        } else if (len > 1 << a.shift) {
            first = static_cast<int64_t>(a.batch) * a.n_bands + norm_part(a, 0, at, start);
            apart = a.parts;
            each = (len + (int64_t(1) << a.part_shift) - 1) >> a.part_shift;
        } else {
            first = band;
            apart = a.n_bands;
            if (len == 0) each = 0;
        }
        const int64_t step = 2 * static_cast<int64_t>(a.channels), lo = signals * each * wave / S, hi = signals * each * (wave + 1) / S;
        int64_t i = each ? lo / each : 0, j = lo - i * each;
        const float* from = a.sums + (first + i * apart + j) * step + c;
#pragma unroll 8
        for (int64_t n = lo; n < hi; ++n) {
            all += double2{from[0], from[a.channels]};
            const bool next = ++j == each;
            from += (next ? apart - each + 1 : 1) * step;
            if (next) j = 0;
        }
    }
    if constexpr (S > 1) {
        sums[wave][lane] = all;
        __syncthreads();
        if (wave > 0) return;
        for (int w = 1; w < S; ++w) all += sums[w][lane];
    }
    if (!there) return;
    const int64_t to = band * a.channels + c;
    if (a.dw) static_cast<T*>(a.dw)[to] = static_cast<T>(static_cast<float>(all.x));
    if (a.db) static_cast<T*>(a.db)[to] = static_cast<T>(static_cast<float>(all.y));
}

}  // namespace nsl
