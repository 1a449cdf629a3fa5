// Windowed attention along the bands: forward and gradient kernels.
//
//   o_i = sum_j p_ij v_j,  p_ij = exp(scale q_i . k_j - lse_i) over the visible j
//   dv_j = sum_i p_ij do_i            ds_ij = p_ij (do_i . v_j - do_i . o_i)
//   dq_i = scale sum_j ds_ij k_j      dk_j = scale sum_i ds_ij q_i
//
// visible(i, j): keep_j and j <= i + right and (j >= i - left or j < sinks).
#pragma once
#include "tile.hpp"

namespace nsl {

struct AttnScale {
    float c, unit;   // scale log2(e): exp(scale s) = exp2(c s); the scores' difference of one power of two, 1 / c
};

// The kernels' WIDE: every view takes 16-byte accesses.
struct AttnArgs {
    View q, k, v, o, d_o, dq, dk, dv;
    float* stats;         // [batch][heads][rows]: log2 of the softmax sum of scores times c; +inf for an empty row
    float* delta;         // [batch][heads][rows]: do . o
    float* part;          // partial dk, dv of the sinks
    const uint8_t* keep;
    int64_t keep_batch;
    const int64_t* off;
    int rows, n_bands, batch, heads, kv_heads, dim;
    int share;            // heads of one kv head that a workgroup takes: 1, 2 or 4
    int left, right, sinks;   // at most rows
    int far;                  // of the sinks, those whose far queries have partial sums (gradient)
    float scale;
    AttnScale by;
};

__device__ inline float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// The base of a running softmax: what is subtracted from the scores before
// the exponential. It is the maximum, but may lag by LAG powers of two: sums
// and outputs are rescaled when it moves by more, which is rare after the
// first keys. Float16 has no numbers between 0 and 2^-24, and keys of smaller
// probabilities may add up to a result: there the base also follows the scores
// of the last 32 keys down where they lie kDown powers of two below it (sums
// and outputs, in 32 bits, then grow; by 2^kDeep at most), and probabilities
// are formed times 2^kLift: the largest of 32 keys lies in 2^-1 .. 2^15.
template <class T, int LAG> struct Base {
    static constexpr bool kHalf = std::is_same<T, _Float16>::value;
    static constexpr float kDown = 8.f, kDeep = 48.f, kLift = kHalf ? 15.f - LAG : 0.f;
    float top = -INFINITY, peak = -INFINITY;   // the base's score; the largest score yet (float16)

    // Takes the largest score of the next keys: true if `factor` has to be
    // applied to what was summed before.
    __device__ bool move(float mx, const AttnScale& by, float& factor) {
        bool far = LAG ? mx > top + LAG * by.unit : mx > top;
        if constexpr (kHalf) {
            peak = fmaxf(peak, mx);
            far |= mx < top - kDown * by.unit && mx > -INFINITY && top > peak - kDeep * by.unit;
        }
        if (!__any(far)) return false;
        float now = fmaxf(top, mx);
        if constexpr (kHalf) now = mx > -INFINITY ? fmaxf(mx, peak - kDeep * by.unit) : top;
        // the difference of the bases as the exponentials take them, rounded
        const float before = of(by);
        const bool first = top == -INFINITY;   // nothing was summed yet
        top = now;
        factor = first ? 1.f : exp2_(before - of(by));
        return true;
    }
    // in powers of two: a key's probability is exp2(c score - of(c))
    __device__ float of(const AttnScale& by) const { return top == -INFINITY ? 0.f : fmaf(top, by.c, -kLift); }
};

// A workgroup has four waves of 32 rows each. Forward and dq: `share` heads of
// one kv head, 128 / share queries of each, so that the waves need (nearly)
// the same keys: with a window of 256 and four heads a workgroup walks 287
// keys and not 383. The key gradient: 128 keys of one kv head.
constexpr int kKeys = 128, kKeyShift = 7;
__host__ __device__ inline int query_shift(int share) { return share == 4 ? 5 : share == 2 ? 6 : 7; }
// Rows of a tile of keys (forward, dq) and of queries (key gradient): short
// enough for two workgroups' tiles in a compute unit's LDS. 223,466 tokens,
// 4 heads of 64 over 2, window 128, float32: 437 us forward and 2263 with
// gradients; with tiles of 64 there 468 and 2799.
template <class T, int DP> constexpr int key_tile() { return row_bytes<T, DP>() > 128 ? 32 : 64; }
template <class T, int DP> constexpr int query_tile() { return sizeof(T) == 4 && DP > 32 ? 32 : 64; }

template <class T> __device__ inline T* row_of(const View& v, int64_t b, int64_t row, int head) {
    return reinterpret_cast<T*>(v.data) + b * v.batch + row * v.row + head * v.head;
}

// The window's keys in tiles of BN: first tiles over the sinks that lie
// before the window of the block's first query, then over the window.
struct KeyRange {
    int sink_end, sink_tiles, begin, end, tiles;
    __device__ KeyRange(const AttnArgs& a, int i_first, int i_last, int len, int bn) {
        begin = i_first > a.left ? i_first - a.left : 0;
        end = static_cast<int>(static_cast<int64_t>(i_last) + a.right + 1 < len ? i_last + a.right + 1 : len);
        sink_end = a.sinks < begin ? a.sinks : begin;
        sink_tiles = (sink_end + bn - 1) / bn;
        tiles = sink_tiles + (end - begin + bn - 1) / bn;
    }
    // Of 32 keys j .. of a tile and a wave's queries i_lo .. i_hi: whether no
    // query sees any of them, and whether some see only some of them.
    __device__ static bool hidden(const AttnArgs& a, int j, int j_end, int i_lo, int i_hi) {
        return j >= j_end || j > i_hi + a.right || (j + 31 < i_lo - a.left && j >= a.sinks);
    }
    __device__ static bool edge(const AttnArgs& a, int j, int i_lo, int i_hi) {
        return j + 31 > i_lo + a.right || (j < i_hi - a.left && j + 31 >= a.sinks);
    }
    // first key of tile t, and the end of the keys it may hold
    __device__ void tile(int t, int bn, int& j0, int& j_end) const {
        const bool s = t < sink_tiles;
        j0 = s ? t * bn : begin + (t - sink_tiles) * bn;
        j_end = s ? sink_end : end;
    }
};

typedef __attribute__((address_space(3))) void lds_void;

// One tile of BN rows x DP columns of two tensors into LDS. Wide tensors go
// there directly, 16 bytes a lane (a wave fills 1 KB of consecutive LDS, so
// the lanes fetch the chunks that belong to their places): no registers, no
// stores, and the next tile is on its way while this one is computed. The
// buffer ends with the tile's last row, and reads past its end give zeros:
// rows that are not there cost nothing; lanes whose column or row is not there
// or not kept aim past the end. Other tensors take element loads and are
// stored from registers.
template <class T, int DP, int BN, bool WIDE> struct Loader {
    static constexpr int kRB = row_bytes<T, DP>(), kBytes = BN * kRB;
    static constexpr int kEach = kBytes / 4096;          // wide: loads of a thread for each tensor
    static constexpr int kChunks = BN * DP / 8;          // else: chunks of 8 values of a tile
    static constexpr unsigned kPast = 0x80000000u;       // past every tile, and less than 2^30 from its end
    // Wide: this lane's offsets in bytes. In rows of 128 bytes a wave's loads
    // are 8 rows apart, where the chunks' order repeats: one offset serves all.
    static constexpr int kOffsets = kRB == 128 ? 1 : kEach;
    unsigned ox[kOffsets], oy[kOffsets];
    int64_t sx, sy;
    int dim;

    // row of load e of this thread in a tile
    static __device__ int row(int e, int wave, int lane) { return ((wave * kEach + e) * 1024 + lane * 16) / kRB; }

    __device__ Loader(int64_t stride_x, int64_t stride_y, int width, int wave, int lane)
        : sx(stride_x), sy(stride_y), dim(width) {
#pragma unroll
        for (int e = 0; e < kOffsets; ++e) {
            const int r = row(e, wave, lane), slot = lane % (kRB / 16 < 64 ? kRB / 16 : 64);
            const unsigned d = (slot ^ turn(r)) * (16 / sizeof(T));
            ox[e] = d < static_cast<unsigned>(dim) ? (r * static_cast<unsigned>(sx) + d) * sizeof(T) : kPast;
            oy[e] = d < static_cast<unsigned>(dim) ? (r * static_cast<unsigned>(sy) + d) * sizeof(T) : kPast;
        }
    }

    static __device__ unsigned offset(const unsigned (&o)[kOffsets], int e, int64_t stride) {
        return kOffsets > 1 ? o[e] : o[0] + e * 8 * static_cast<unsigned>(stride) * static_cast<unsigned>(sizeof(T));
    }

    // rows row0 .. of px, py (below row_end) into tx, ty; kept: for each load
    // of a wide tensor, whether its row may be used (with keep)
    __device__ void load(char* tx, char* ty, const T* px, const T* py, int row0, int row_end, const uint8_t* keep,
                         const bool (&kept)[kEach], int tid) const {
        px += row0 * sx;
        py += row0 * sy;
        const int rows = min(row_end - row0, BN);
        if constexpr (WIDE) {
#ifdef __HIP_DEVICE_COMPILE__   // the host pass does not know a buffer's type
            const int wave = wave_number();
            const auto rx = __builtin_amdgcn_make_buffer_rsrc(
                const_cast<T*>(px), 0, rows * static_cast<unsigned>(sx) * static_cast<unsigned>(sizeof(T)), 0x00020000);
            const auto ry = __builtin_amdgcn_make_buffer_rsrc(
                const_cast<T*>(py), 0, rows * static_cast<unsigned>(sy) * static_cast<unsigned>(sizeof(T)), 0x00020000);
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const int at = (wave * kEach + e) * 1024;
                const bool drop = keep && !kept[e];
                const unsigned x = drop ? kPast : offset(ox, e, sx), y = drop ? kPast : offset(oy, e, sy);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lds_void*)(tx + at), 16, x, 0, 0, 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(ry, (lds_void*)(ty + at), 16, y, 0, 0, 0);
            }
#endif
        } else {
            for (int c = tid; c < kChunks; c += 256) {
                const int r = c / (DP / 8), d = c % (DP / 8) * 8;
                const int n = r < rows && (!keep || keep[row0 + r]) ? dim - d : 0;
                write8<T, kRB>(tx, r, c % (DP / 8), load8<T, false>(px + r * sx + d, n, d > 0));
                write8<T, kRB>(ty, r, c % (DP / 8), load8<T, false>(py + r * sy + d, n, d > 0));
            }
        }
    }
};

// Every LDS write of this wave, the direct ones too, is done; then all waves'.
__device__ inline void tile_barrier() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
}

// S^T of 32 keys (rows row0 .. of a tile) and 32 queries. With a bias (of the
// tile's keys: 0, or -inf for one that is not there or not kept; its row is
// zeros) the sums start there, so that masking costs no instruction.
template <class T, int DP>
__device__ inline acc16 scores(const char* tile, int row0, const frag<T> (&f)[DP / 16], const float* bias, int lane) {
    constexpr int RB = row_bytes<T, DP>();
    const int m = lane & 31, h = lane >> 5;
    if (!bias) {
        acc16 s = zero16();
#pragma unroll
        for (int x = 0; x < DP / 16; ++x) s = mma(read8<T, RB>(tile, row0 + m, 2 * x + h), f[x], s);
        return s;
    }
    acc16 s;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const f4 b = *reinterpret_cast<const f4*>(bias + row0 + 8 * q + 4 * h);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[4 * q + j] = b[j];
    }
#pragma unroll
    for (int x = 0; x < DP / 16; ++x) s = mma(read8<T, RB>(tile, row0 + m, 2 * x + h), f[x], s);
    return s;
}

// The product of 32 rows (from row0 on) of two tiles, transposed: rows of a, columns of b.
template <class T, int DP>
__device__ inline acc16 rows_product(const char* a, int row_a, const char* b, int row_b, int lane) {
    constexpr int RB = row_bytes<T, DP>();
    const int m = lane & 31, h = lane >> 5;
    acc16 s = zero16();
#pragma unroll
    for (int x = 0; x < DP / 16; ++x)
        s = mma(read8<T, RB>(a, row_a + m, 2 * x + h), read8<T, RB>(b, row_b + m, 2 * x + h), s);
    return s;
}

// The window's edges, for tiles that cross one: hides the scores (column:
// query i, rows: keys j0 ..) of keys outside [i - left, i + right] that are
// not sinks, and with GRAD drops what dp holds there (0 * inf would be NaN).
template <bool GRAD>
__device__ inline void hide_edges(acc16& s, acc16& dp, const AttnArgs& a, int i, int j0, int h) {
    const int at = j0 + 4 * h, lo = i - a.left - at;
    const unsigned span = static_cast<unsigned>(a.left) + a.right;
    if (j0 >= a.sinks) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const bool see = static_cast<unsigned>(8 * (r >> 2) + (r & 3) - lo) <= span;
            s[r] = see ? s[r] : -INFINITY;
            if (GRAD) dp[r] = see ? dp[r] : 0.f;
        }
    } else {
        const int hi = i + a.right - at, sink = a.sinks - at;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int e = 8 * (r >> 2) + (r & 3);
            const bool see = e <= hi && (e >= lo || e < sink);
            s[r] = see ? s[r] : -INFINITY;
            if (GRAD) dp[r] = see ? dp[r] : 0.f;
        }
    }
}

// 32 rows of a tensor as fragments (A or B): lane l holds row l % 32.
template <class T, int DP>
__device__ inline void load_rows(frag<T> (&f)[DP / 16], const T* p, bool there, int dim, bool wide, int lane) {
    by_width(wide, [&](auto w) {
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
            const int d = 16 * s + 8 * (lane >> 5);
            f[s] = load8<T, w.value>(p + d, there ? dim - d : 0, d > 0);
        }
    });
}

// Zeros for `count` rows from `first` on (below len) of tokens that no band holds.
template <class T>
__device__ inline void zero_rows(const View& v, int64_t b, int head, int start, int first, int count, int len, int dim,
                                 int tid) {
    for (int r = first; r < first + count && r < len; ++r)
        for (int d = tid; d < dim; d += 256) row_of<T>(v, b, start + r, head)[d] = static_cast<T>(0.f);
}

// The same 32 rows in LDS of the wave's own, to be read as fragments when they
// are needed: registers, and with them the waves on a SIMD, are what the
// gradient kernels are short of (446,932 tokens, 8 heads of 64 over 2, window
// 256, bfloat16: dq 1065 us with three waves, 1292 with two; the key gradient
// 1044 and 1167).
template <class T, int DP>
__device__ inline void keep_rows(char* to, const T* p, bool there, int dim, bool wide, int lane) {
    frag<T> f[DP / 16];
    load_rows<T, DP>(f, p, there, dim, wide, lane);
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) write8<T, row_bytes<T, DP>()>(to, lane & 31, 2 * s + (lane >> 5), f[s]);
}

// What a workgroup of the forward or the dq kernel works on.
struct QueryWork {
    int b, kv, head0, head, i_lo, queries;
    Tile<int> t;
    __device__ QueryWork(const AttnArgs& a, int wave, int lane) {
        const int group = a.heads / a.kv_heads, parts = group / a.share, shift = query_shift(a.share);
        const unsigned id = die_order(blockIdx.x, gridDim.x), units = a.kv_heads * parts, unit = id % units, rest = id / units;
        const unsigned per = static_cast<unsigned>(tile_count(shift, a.n_bands, 1, a.rows));
        b = rest / per;
        kv = unit / parts;
        head0 = kv * group + unit % parts * a.share;
        queries = 1 << shift;
        t = find_tile<int>(a.off, a.n_bands, a.rows, 1, shift, rest - b * per, lane);
        head = head0 + (wave & (a.share - 1));
        i_lo = t.first + 32 * (wave >> (7 - shift));
    }
};

// Forward. One pass over the visible keys with a running maximum and sum. The
// scores are formed transposed (a lane has one query), so a row's maximum and
// sum need one exchange between the wave's halves, and the probabilities are
// the B fragment of o^T = V^T p^T without leaving the registers. In 16 bits p
// goes into that product as two numbers, the rounded one and what the rounding
// left: with one alone o is off by 0.0022 in the 2-norm in bfloat16, with two
// by its own rounding, 0.0016. Sums take p unrounded.
//
// 131,072 tokens, 8 heads of 128 over 2, window 1024: 850 us (667 with p as
// one number), 648 TFLOP/s of visible pairs; 457 at the rate of a large
// product, 685 with p's second number, which is half as many products again.
// The matrix cores wait for the exponentials (a quarter of the vector rate),
// the maxima and the rounding. Tiles of 32 keys there, three waves a SIMD.
// 446,932 tokens in 221 bands, 8 heads of 64 over 2, window 256: 690 us (600
// with p as one number), 232 for reading and writing at the rate of a large copy.
template <class T, int DP, bool WIDE>
__global__ __launch_bounds__(256, sizeof(T) == 4 && DP > 64 ? 1 : WIDE ? 3 : 2) void k_attention(AttnArgs a) {
    constexpr int BN = key_tile<T, DP>(), RB = row_bytes<T, DP>();
    typedef Loader<T, DP, BN, WIDE> Ld;
    __shared__ __align__(1024) char lds[2][2][Ld::kBytes];
    __shared__ __align__(16) float bias[2][BN];
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), m = lane & 31, h = lane >> 5;

    const QueryWork w(a, wave, lane);
    const Tile<int>& t = w.t;
    if (!t.live) return;
    const int64_t b = w.b;
    const int len = t.len, q0 = t.first, kv = w.kv, head = w.head;
    float* stats = a.stats ? a.stats + (b * a.heads + head) * a.rows + t.start : nullptr;
    const int i_lo = w.i_lo, i = i_lo + m, i_hi = min(i_lo + 31, len - 1);
    const bool mine = i < len, active = i_lo < len;
    if (t.band < 0 || t.band >= a.n_bands) {
        for (int x = 0; x < a.share; ++x)
            zero_rows<T>(a.o, b, w.head0 + x, t.start, q0, w.queries, len, a.dim, tid);
        if (stats && mine && h == 0) stats[i] = INFINITY;
        return;
    }
    frag<T> qf[DP / 16];
    load_rows<T, DP>(qf, row_of<T>(a.q, b, t.start + (mine ? i : 0), head), mine, a.dim, WIDE, lane);
    const T* kp = row_of<T>(a.k, b, t.start, kv);
    const T* vp = row_of<T>(a.v, b, t.start, kv);
    const uint8_t* keep = a.keep ? a.keep + b * a.keep_batch + t.start : nullptr;

    acc16 o[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) o[d] = zero16();
    float sum = 0.f;   // this half's
    Base<T, 8> base;

    const KeyRange range(a, q0, min(q0 + w.queries, len) - 1, len, BN);
    const Ld ld(a.k.row, a.v.row, a.dim, wave, lane);
    // what masks tile n is fetched a tile earlier than the tile itself
    bool kept[Ld::kEach];
    float next_bias = 0.f;
    auto fetch_masks = [&](int n) {
        int j0 = 0, j_end = 0;
        if (n < range.tiles) range.tile(n, BN, j0, j_end);
#pragma unroll
        for (int e = 0; e < Ld::kEach; ++e) {
            const int j = j0 + Ld::row(e, wave, lane);
            kept[e] = !keep || (j < j_end && keep[j]);
        }
        next_bias = j0 + tid < j_end && tid < BN && (!keep || keep[j0 + tid]) ? 0.f : -INFINITY;
    };
    auto fetch = [&](int n, int u) {
        int j0, j_end;
        range.tile(n, BN, j0, j_end);
        ld.load(lds[u][0], lds[u][1], kp, vp, j0, j_end, keep, kept, tid);
        if (tid < BN) bias[u][tid] = next_bias;
    };
    fetch_masks(0);
    fetch(0, 0);
    fetch_masks(1);
    tile_barrier();
    for (int n0 = 0; n0 < range.tiles; n0 += 2) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {   // by two, so that a tile's place in LDS is a constant
            const int n = n0 + u;
            if (n >= range.tiles) continue;
            if (n + 1 < range.tiles) {
                fetch(n + 1, u ^ 1);
                fetch_masks(n + 2);
            }
            int j0, j_end;
            range.tile(n, BN, j0, j_end);
            const char* kt = lds[u][0];
            const char* vt = lds[u][1];
#pragma unroll
            for (int kb = 0; kb < BN / 32; ++kb) {
                const int j = j0 + 32 * kb;
                if (!active || KeyRange::hidden(a, j, j_end, i_lo, i_hi)) continue;
                acc16 s = scores<T, DP>(kt, 32 * kb, qf, keep || j + 32 > j_end ? bias[u] : nullptr, lane);
                if (KeyRange::edge(a, j, i_lo, i_hi)) hide_edges<false>(s, s, a, i, j, h);
                float mx = s[0];
#pragma unroll
                for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
                mx = half_max(mx);
                float factor;
                if (base.move(mx, a.by, factor)) {
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
                        const frag<T> vd = read_turned<T, RB>(vt, 32 * kb + 16 * x, 32 * d, lane);
                        o[d] = mma(vd, p, o[d]);
                        if constexpr (sizeof(T) == 2) o[d] = mma(vd, low, o[d]);
                    }
                }
            }
            tile_barrier();
        }
    }
    const float total = half_sum(sum);
    const float inv = total == 0.f ? 0.f : 1.f / total;
    T* out = mine ? row_of<T>(a.o, b, t.start + i, head) : nullptr;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) {
        o[d] *= inv;
        store_column<T>(out, o[d], 32 * d, a.dim, WIDE, lane);
    }
    if (stats && mine && h == 0)
        stats[i] = total == 0.f ? INFINITY : base.of(a.by) + __log2f(total);
}

// --------------------------------------------------------------- gradients

// Float16's range in a product summed over blocks: a lane's 16 values x of a
// block belong to one column of the sums (with those of the lane 32 away), and
// are multiplied by a power of two of the column's that brings the largest of
// a block to 2^-1 .. 2^15: probabilities' gradients pass 65,504 under a scaled
// loss, and lie below 2^-24 under a small one, where dq, dk and dv are float16
// numbers. When the power changes the sums, in 32 bits, change with it; they
// grow by 2^48 at most. In the other types there is nothing to do. (446,932
// tokens, 8 heads of 64 over 2, window 256, forward and gradients: 3524 us in
// float16, 2687 in bfloat16: the powers' registers leave two waves a SIMD.)
template <class T> struct InRange {
    static constexpr bool kHalf = std::is_same<T, _Float16>::value;
    static constexpr float kGrow = 0x1p48f;
    float by = 0.f, least = INFINITY;   // the column's power (0: none yet), and the smallest yet

    template <int N> __device__ void take(acc16& x, acc16 (&sums)[N]) {
        if constexpr (kHalf) {
            float mx = fabsf(x[0]);
#pragma unroll
            for (int r = 1; r < 16; ++r) mx = fmaxf(mx, fabsf(x[r]));
            mx = half_max(mx);
            const float at = mx * by;
            if (__any(at > 0x1p15f || (at < 0.5f && mx > 0.f && by < least * kGrow))) {
                float to = by > 0.f ? by : 1.f;
                if (mx > 0.f && mx < INFINITY)
                    to = fminf(fminf(ldexpf(1.f, 14 - __builtin_amdgcn_frexp_expf(mx)), 0x1p100f), least * kGrow);
                const float change = by > 0.f ? to / by : 1.f;
#pragma unroll
                for (int d = 0; d < N; ++d) sums[d] *= change;
                by = to;
                if (mx > 0.f) least = fminf(least, to);
            }
            x *= by;
        }
    }
    // what takes the sums back
    __device__ float undo() const { return kHalf && by > 0.f ? 1.f / by : 1.f; }
};

// Waves a SIMD of dq and the key gradient, by what their registers allow:
// `large` at heads above 64.
template <class T, int DP, bool WIDE> constexpr int grad_waves(int large) {
    if (DP > 64) return large;
    return sizeof(T) == 2 && WIDE && (DP <= 32 || !InRange<T>::kHalf) ? 3 : 2;
}

// dq, and delta = do . o for the key gradient. In 16 bits ds goes into its
// product as two numbers, the rounded one and what the rounding left: with one
// alone dq is off by 0.0025 in the 2-norm (bfloat16; 0.0017 is its own
// rounding). delta comes from the rounded o; a row of ds sums to zero with the
// exact one, so the sum that is found is delta's error, and the key gradient
// gets the corrected value. Where few keys have a weight (few are seen, or one
// outweighs the others), dp - delta is small beside delta, whose error then
// shows in dq (two keys, bfloat16: 0.0034 in the 2-norm). So a workgroup in
// which that sum passes a quarter of u of the row's sum of |ds| anywhere goes
// through its keys once more with the corrected delta (0.0017). With random
// scores that happens below some 30 keys, at a band's first tokens and where
// few are kept: 446,932 tokens, window of 256, one key in eight and a long
// stretch dropped: 11 % of the workgroups, 1070 us instead of 970; window of 2,
// everywhere: forward and gradients 1390 us instead of 1290.
// Layout as k_attention: the scores and dp are formed transposed, so ds is the
// B fragment of dq^T = K^T ds^T.
template <class T> constexpr float kRest = std::is_same<T, _Float16>::value ? 0x1p-13f : 0x1p-10f;
template <class T, int DP, bool WIDE>
__global__ __launch_bounds__(256, (grad_waves<T, DP, WIDE>(sizeof(T) == 4 ? 1 : 2))) void k_attention_dq(AttnArgs a) {
    constexpr int BN = key_tile<T, DP>(), RB = row_bytes<T, DP>();
    typedef Loader<T, DP, BN, WIDE> Ld;
    __shared__ __align__(1024) char lds[2][2][Ld::kBytes];
    __shared__ __align__(128) char grads[4][32 * RB];   // each wave's rows of do
    __shared__ __align__(16) float bias[2][BN];
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), m = lane & 31, h = lane >> 5;

    const QueryWork w(a, wave, lane);
    const Tile<int>& t = w.t;
    if (!t.live) return;
    const int64_t b = w.b;
    const int len = t.len, q0 = t.first, kv = w.kv, head = w.head;
    if (t.band < 0 || t.band >= a.n_bands) {
        for (int x = 0; x < a.share; ++x)
            zero_rows<T>(a.dq, b, w.head0 + x, t.start, q0, w.queries, len, a.dim, tid);
        return;
    }
    const int64_t at = (b * a.heads + head) * a.rows + t.start;
    const int i_lo = w.i_lo, i = i_lo + m, i_hi = min(i_lo + 31, len - 1);
    const bool mine = i < len, active = i_lo < len;
    const int64_t row = t.start + (mine ? i : 0);
    frag<T> qf[DP / 16];
    load_rows<T, DP>(qf, row_of<T>(a.q, b, row, head), mine, a.dim, WIDE, lane);
    char* own = grads[wave];
    float delta = 0.f;
    {
        frag<T> of[DP / 16], gf[DP / 16];
        load_rows<T, DP>(gf, row_of<T>(a.d_o, b, row, head), mine, a.dim, WIDE, lane);
        load_rows<T, DP>(of, row_of<T>(a.o, b, row, head), mine, a.dim, WIDE, lane);
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
            write8<T, RB>(own, m, 2 * s + h, gf[s]);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                delta = fmaf(static_cast<float>(of[s][j]), static_cast<float>(gf[s][j]), delta);
        }
    }
    delta = half_sum(delta);
    float rest = 0.f;   // the sum of this row's ds: 0 but for delta's error
    InRange<T> range_ds;
    const float lse = mine ? a.stats[at + i] : INFINITY;

    const T* kp = row_of<T>(a.k, b, t.start, kv);
    const T* vp = row_of<T>(a.v, b, t.start, kv);
    const uint8_t* keep = a.keep ? a.keep + b * a.keep_batch + t.start : nullptr;
    acc16 g[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) g[d] = zero16();

    const KeyRange range(a, q0, min(q0 + w.queries, len) - 1, len, BN);
    const Ld ld(a.k.row, a.v.row, a.dim, wave, lane);
    // what masks tile n is fetched a tile earlier than the tile itself
    bool kept[Ld::kEach];
    float next_bias = 0.f;
    auto fetch_masks = [&](int n) {
        int j0 = 0, j_end = 0;
        if (n < range.tiles) range.tile(n, BN, j0, j_end);
#pragma unroll
        for (int e = 0; e < Ld::kEach; ++e) {
            const int j = j0 + Ld::row(e, wave, lane);
            kept[e] = !keep || (j < j_end && keep[j]);
        }
        next_bias = j0 + tid < j_end && tid < BN && (!keep || keep[j0 + tid]) ? 0.f : -INFINITY;
    };
    auto fetch = [&](int n, int u) {
        int j0, j_end;
        range.tile(n, BN, j0, j_end);
        ld.load(lds[u][0], lds[u][1], kp, vp, j0, j_end, keep, kept, tid);
        if (tid < BN) bias[u][tid] = next_bias;
    };
    float size = 0.f;   // the sum of |ds|
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
        const bool load = pass == 0 || range.tiles > 2;   // else both tiles are still in LDS
        if (load) {
            fetch_masks(0);
            fetch(0, 0);
            fetch_masks(1);
            tile_barrier();
        }
        for (int n0 = 0; n0 < range.tiles; n0 += 2) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {   // by two, so that a tile's place in LDS is a constant
                const int n = n0 + u;
                if (n >= range.tiles) continue;
                if (load && n + 1 < range.tiles) {
                    fetch(n + 1, u ^ 1);
                    fetch_masks(n + 2);
                }
                int j0, j_end;
                range.tile(n, BN, j0, j_end);
                const char* kt = lds[u][0];
                const char* vt = lds[u][1];
#pragma unroll
                for (int kb = 0; kb < BN / 32; ++kb) {
                    const int j = j0 + 32 * kb;
                    if (!active || KeyRange::hidden(a, j, j_end, i_lo, i_hi)) continue;
                    acc16 s = scores<T, DP>(kt, 32 * kb, qf, keep || j + 32 > j_end ? bias[u] : nullptr, lane);
                    acc16 dp = rows_product<T, DP>(vt, 32 * kb, own, 0, lane);
                    if (KeyRange::edge(a, j, i_lo, i_hi)) hide_edges<true>(s, dp, a, i, j, h);
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        s[r] = exp2_(fmaf(s[r], a.by.c, -lse)) * (dp[r] - delta);
                        rest += s[r];
                        if (sizeof(T) == 2) size += fabsf(s[r]);
                    }
                    range_ds.take(s, g);
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const frag<T> ds = narrow<T>(s, x), low = rest_of<T>(s, x, ds);
#pragma unroll
                        for (int d = 0; d < DP / 32; ++d) {
                            const frag<T> kd = read_turned<T, RB>(kt, 32 * kb + 16 * x, 32 * d, lane);
                            g[d] = mma(kd, ds, g[d]);
                            if constexpr (sizeof(T) == 2) g[d] = mma(kd, low, g[d]);
                        }
                    }
                }
                tile_barrier();
            }
        }
        rest = half_sum(rest);
        if (sizeof(T) == 4 || pass == 1) break;
        if (!__syncthreads_or(fabsf(rest) > kRest<T> * half_sum(size))) break;
        delta += rest;
        rest = 0.f;
        range_ds = InRange<T>();
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) g[d] = zero16();
    }
    if (mine && h == 0) a.delta[at + i] = delta + rest;
    T* out = mine ? row_of<T>(a.dq, b, t.start + i, head) : nullptr;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) {
        g[d] *= a.scale * range_ds.undo();
        store_column<T>(out, g[d], 32 * d, a.dim, WIDE, lane);
    }
}

// The sinks' keys are seen from everywhere. Queries past the window of a key
// tile's last key ("far" ones) would make one workgroup walk a whole band, so
// k_attention_far takes them in chunks and leaves partial dk, dv, which the
// workgroup of the key tile adds up in the chunks' order. The partial sums
// take 64 dim floats for each 512 tokens and 32 sinks: with kFarSinks twice
// what dk and dv take in 16 bits. Key tiles past those sinks walk the whole
// band after all.
constexpr int kFarShift = 9;   // queries of a chunk
constexpr int kFarSinks = 512;
static_assert(kFarSinks % kKeys == 0, "a key tile is on one side");
__device__ inline int far_begin(const AttnArgs& a, int sink_tile) {   // of 32 keys
    return sink_tile * 32 / kKeys * kKeys + kKeys + a.left;
}
__device__ inline float* far_part(const AttnArgs& a, int64_t b, int kv, int64_t item, int sink_tile) {
    const int64_t per = tile_count(kFarShift, a.n_bands, 1, a.rows);
    const int n = (a.far + 31) / 32;
    return a.part + (((b * a.kv_heads + kv) * per + item) * n + sink_tile) * (2 * 32 * a.dim);
}

// One wave's 32 queries (rows of the tiles qt, gt at r0) against its 32 keys:
// adds to dk^T and dv^T, each times its column's power of two. kf, vt: the
// keys' k as fragments and v in LDS. lse, delta: of the tile's queries, in LDS
// (+inf for a query that is not there: its probabilities are 0). With edge, this lane's
// key is visible to the rows r0 + lo .. r0 + lo + span only. A key that is
// not there or not kept only spoils its own column, which its lane drops.
template <class T, int DP>
__device__ inline void key_grad(const char* qt, const char* gt, const float* lse, const float* delta, int r0,
                                const frag<T> (&kf)[DP / 16], const char* vt, acc16 (&dk)[DP / 32],
                                acc16 (&dv)[DP / 32], InRange<T>& range_ds, InRange<T>& range_p, float c, bool edge,
                                int lo, unsigned span, int lane) {
    constexpr int RB = row_bytes<T, DP>();
    const int h = lane >> 5;
    acc16 s = scores<T, DP>(qt, r0, kf, nullptr, lane), dp = rows_product<T, DP>(gt, r0, vt, 0, lane);
    if (edge) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const bool see = static_cast<unsigned>(8 * (r >> 2) + (r & 3) - (lo - 4 * h)) <= span;
            s[r] = see ? s[r] : -INFINITY;
            dp[r] = see ? dp[r] : 0.f;
        }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const f4 l = *reinterpret_cast<const f4*>(lse + r0 + 8 * q + 4 * h);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[4 * q + j] = exp2_(fmaf(s[4 * q + j], c, -l[j]));
    }
    acc16 pr = s;
    range_p.take(pr, dv);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const frag<T> p = narrow<T>(pr, x), low = rest_of<T>(pr, x, p);
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) {
            const frag<T> g = read_turned<T, RB>(gt, r0 + 16 * x, 32 * d, lane);
            dv[d] = mma(g, p, dv[d]);
            if constexpr (sizeof(T) == 2) dv[d] = mma(g, low, dv[d]);
        }
    }
    if (sizeof(T) == 2) __builtin_amdgcn_sched_barrier(0);   // p's fragments are gone before ds' are made: registers
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const f4 e = *reinterpret_cast<const f4*>(delta + r0 + 8 * q + 4 * h);
#pragma unroll
        for (int j = 0; j < 4; ++j) dp[4 * q + j] = s[4 * q + j] * (dp[4 * q + j] - e[j]);
    }
    range_ds.take(dp, dk);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const frag<T> ds = narrow<T>(dp, x), low = rest_of<T>(dp, x, ds);
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) {
            const frag<T> q = read_turned<T, RB>(qt, r0 + 16 * x, 32 * d, lane);
            dk[d] = mma(q, ds, dk[d]);
            if constexpr (sizeof(T) == 2) dk[d] = mma(q, low, dk[d]);
        }
    }
}

// Past the last query near 128 keys from k0 on. (Their sum passes 31 bits in
// the longest rows.)
__host__ __device__ inline int queries_end(int k0, int left, int len) {
    const int64_t end = static_cast<int64_t>(k0) + kKeys + left;
    return static_cast<int>(end < len ? end : len);
}

// dk, dv of 128 keys (a wave has 32) over the queries near them, for all heads
// of their kv head: no atomics and no partial sums but the sinks'. Scores and
// dp are formed the other way round than in dq (a lane has one key), so p and
// ds are B fragments again. In 16 bits each goes into its product as two
// numbers: with one, dk and dv are off by 0.0026 and 0.0023 in the 2-norm in
// bfloat16, with two by their own rounding, 0.0016.
// 446,932 tokens, 8 heads of 64 over 2, window 256, bfloat16: 1044 us (820 with
// p and ds as one number; dq 1070, far queries 190): 2.8 ms with the forward,
// 273 TFLOP/s of the formulas' work. Bound by waiting: three waves a SIMD,
// half their cycles.
template <class T, int DP, bool WIDE>
__global__ __launch_bounds__(256, (grad_waves<T, DP, WIDE>(1))) void k_attention_dkv(AttnArgs a) {
    constexpr int BQ = query_tile<T, DP>();
    typedef Loader<T, DP, BQ, WIDE> Ld;
    __shared__ __align__(1024) char lds[2][2][Ld::kBytes];
    __shared__ __align__(128) char values[4][32 * Ld::kRB];   // each wave's rows of v
    __shared__ __align__(16) float row_lse[2][BQ], row_delta[2][BQ];
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), m = lane & 31, h = lane >> 5;

    const unsigned id = die_order(blockIdx.x, gridDim.x), rest = id / a.kv_heads;
    const unsigned per = static_cast<unsigned>(tile_count(kKeyShift, a.n_bands, 1, a.rows));
    const int kv = id - rest * a.kv_heads;
    const int64_t b = rest / per;
    const Tile<int> t =
        find_tile<int>(a.off, a.n_bands, a.rows, 1, kKeyShift, rest - static_cast<unsigned>(b) * per, lane);
    if (!t.live) return;
    const int len = t.len, k0 = t.first, group = a.heads / a.kv_heads;
    if (t.band < 0 || t.band >= a.n_bands) {
        zero_rows<T>(a.dk, b, kv, t.start, k0, kKeys, len, a.dim, tid);
        zero_rows<T>(a.dv, b, kv, t.start, k0, kKeys, len, a.dim, tid);
        return;
    }
    const int j_lo = k0 + 32 * wave, j = j_lo + m, j_hi = min(j_lo + 31, len - 1);
    const bool mine = j < len, active = j_lo < len;
    const uint8_t* keep = a.keep ? a.keep + b * a.keep_batch + t.start : nullptr;
    const bool kept = mine && (!keep || keep[j]);
    const int64_t row = t.start + (mine ? j : 0);
    frag<T> kf[DP / 16];
    load_rows<T, DP>(kf, row_of<T>(a.k, b, row, kv), kept, a.dim, WIDE, lane);
    keep_rows<T, DP>(values[wave], row_of<T>(a.v, b, row, kv), kept, a.dim, WIDE, lane);
    acc16 dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) dk[d] = dv[d] = zero16();
    InRange<T> range_ds, range_p;

    const int i_begin = k0 > a.right ? k0 - a.right : 0;
    const int i_end = k0 >= a.far && k0 < a.sinks ? len : queries_end(k0, a.left, len);
    const int q_tiles = (i_end - i_begin + BQ - 1) / BQ, total = q_tiles * group;
    const unsigned span = j < a.sinks ? 0x7fffffffu : static_cast<unsigned>(a.left) + a.right;
    float next_lse = 0.f, next_delta = 0.f;
    const Ld ld(a.q.row, a.d_o.row, a.dim, wave, lane);
    bool every[Ld::kEach];
#pragma unroll
    for (int e = 0; e < Ld::kEach; ++e) every[e] = true;
    auto fetch_stats = [&](int n) {
        if (n < total && tid < BQ) {
            const int head = kv * group + n / q_tiles, i = i_begin + n % q_tiles * BQ + tid;
            const int64_t at = (b * a.heads + head) * a.rows + t.start + i;
            next_lse = i < i_end ? a.stats[at] : INFINITY;
            next_delta = i < i_end ? a.delta[at] : 0.f;
        }
    };
    auto fetch = [&](int n, int u) {
        const int head = kv * group + n / q_tiles, i0 = i_begin + n % q_tiles * BQ;
        ld.load(lds[u][0], lds[u][1], row_of<T>(a.q, b, t.start, head), row_of<T>(a.d_o, b, t.start, head), i0,
                i_end, nullptr, every, tid);
        if (tid < BQ) {
            row_lse[u][tid] = next_lse;
            row_delta[u][tid] = next_delta;
        }
    };
    fetch_stats(0);
    fetch(0, 0);
    fetch_stats(1);
    tile_barrier();
    for (int n0 = 0; n0 < total; n0 += 2) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int n = n0 + u;
            if (n >= total) continue;
            if (n + 1 < total) {
                fetch(n + 1, u ^ 1);
                fetch_stats(n + 2);
            }
            const int i0 = i_begin + n % q_tiles * BQ;
#pragma unroll 1
            for (int qb = 0; qb < BQ / 32; ++qb) {
                const int i_lo = i0 + 32 * qb, i_hi = min(i_lo + 31, i_end - 1);
                const bool skip = !active || i_lo >= i_end || j_lo > i_hi + a.right ||
                                  (j_hi < i_lo - a.left && j_lo >= a.sinks);
                if (!skip) {
                    const bool edge = j_hi > i_lo + a.right || (j_lo < i_hi - a.left && j_hi >= a.sinks);
                    key_grad<T, DP>(lds[u][0], lds[u][1], row_lse[u], row_delta[u], 32 * qb, kf, values[wave], dk, dv,
                                    range_ds, range_p, a.by.c, edge, j - a.right - i_lo, span, lane);
                }
            }
            tile_barrier();
        }
    }
    if constexpr (InRange<T>::kHalf) {
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) {
            dk[d] *= range_ds.undo();
            dv[d] *= range_p.undo();
        }
    }
    // the far queries' share of the sinks
    if (j_lo < a.far && active) {
        const int tile = j_lo / 32;
        const int begin = far_begin(a, tile);
        const int64_t item0 = (t.start >> kFarShift) + t.band + 1;
        if (begin < len)
            for (int ch = begin >> kFarShift; ch <= (len - 1) >> kFarShift; ++ch) {
                const float* p = far_part(a, b, kv, item0 + ch, tile) + m * a.dim;
                if (j < a.far && mine) {
#pragma unroll
                    for (int d = 0; d < DP / 32; ++d) {
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const int c = 32 * d + 8 * (r >> 2) + 4 * h + (r & 3);
                            if (c < a.dim) {
                                dk[d][r] += p[c];
                                dv[d][r] += p[32 * a.dim + c];
                            }
                            if (r % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // few loads at a time: registers
                        }
                    }
                }
            }
    }
    T* ok = mine ? row_of<T>(a.dk, b, t.start + j, kv) : nullptr;
    T* ov = mine ? row_of<T>(a.dv, b, t.start + j, kv) : nullptr;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            dk[d][r] = kept ? dk[d][r] * a.scale : 0.f;
            dv[d][r] = kept ? dv[d][r] : 0.f;
        }
        store_column<T>(ok, dk[d], 32 * d, a.dim, WIDE, lane);
        store_column<T>(ov, dv[d], 32 * d, a.dim, WIDE, lane);
    }
}

// Partial dk, dv of 32 sink keys over the far queries of one chunk. Every wave
// has the same keys and takes a quarter of the queries; the four results are
// added in the waves' order.
template <class T, int DP, bool WIDE>
__global__ __launch_bounds__(256, DP > 64 || (sizeof(T) == 4 && DP > 32) ? 1 : 2) void k_attention_far(AttnArgs a) {
    constexpr int BQ = sizeof(T) == 4 && DP > 64 ? 64 : 128;
    typedef Loader<T, DP, BQ, WIDE> Ld;
    __shared__ __align__(1024) char lds[2][2 * Ld::kBytes];
    __shared__ __align__(128) char values[32 * Ld::kRB];   // the keys' rows of v
    __shared__ __align__(16) float row_lse[2][BQ], row_delta[2][BQ];
    static_assert(sizeof(lds) >= 2 * DP * 33 * 4, "the tiles' room also serves to add up the waves");
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), m = lane & 31, h = lane >> 5;

    const unsigned n_sink = (a.far + 31) / 32, id = die_order(blockIdx.x, gridDim.x);
    const int tile = id % n_sink, kv = id / n_sink % a.kv_heads;
    const unsigned rest = id / n_sink / a.kv_heads;
    const unsigned per = static_cast<unsigned>(tile_count(kFarShift, a.n_bands, 1, a.rows));
    const int64_t b = rest / per;
    const int item = rest - static_cast<unsigned>(b) * per;
    const Tile<int> t = find_tile<int>(a.off, a.n_bands, a.rows, 1, kFarShift, item, lane);
    if (!t.live || t.band < 0 || t.band >= a.n_bands) return;
    const int len = t.len, group = a.heads / a.kv_heads, j = 32 * tile + m, far = far_begin(a, tile);
    const int i_begin = max(t.first, far), i_end = min(t.first + (1 << kFarShift), len);
    if (i_begin >= i_end) return;
    const uint8_t* keep = a.keep ? a.keep + b * a.keep_batch + t.start : nullptr;
    const bool kept = j < a.far && j < len && (!keep || keep[j]);
    const int64_t row = t.start + (j < len ? j : 0);
    frag<T> kf[DP / 16];
    load_rows<T, DP>(kf, row_of<T>(a.k, b, row, kv), kept, a.dim, WIDE, lane);
    if (wave == 0) keep_rows<T, DP>(values, row_of<T>(a.v, b, row, kv), kept, a.dim, WIDE, lane);
    acc16 dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) dk[d] = dv[d] = zero16();
    InRange<T> range_ds, range_p;

    const int q_tiles = (i_end - i_begin + BQ - 1) / BQ, total = q_tiles * group;
    const Ld ld(a.q.row, a.d_o.row, a.dim, wave, lane);
    bool every[Ld::kEach];
#pragma unroll
    for (int e = 0; e < Ld::kEach; ++e) every[e] = true;
    auto fetch = [&](int n) {
        const int head = kv * group + n / q_tiles, i0 = i_begin + n % q_tiles * BQ;
        ld.load(lds[n & 1], lds[n & 1] + Ld::kBytes, row_of<T>(a.q, b, t.start, head), row_of<T>(a.d_o, b, t.start, head),
                i0, i_end, nullptr, every, tid);
        if (tid < BQ) {
            const int64_t at = (b * a.heads + head) * a.rows + t.start + i0 + tid;
            const bool there = i0 + tid < i_end;
            row_lse[n & 1][tid] = there ? a.stats[at] : INFINITY;
            row_delta[n & 1][tid] = there ? a.delta[at] : 0.f;
        }
    };
    fetch(0);
    tile_barrier();
    for (int n = 0; n < total; ++n) {
        if (n + 1 < total) fetch(n + 1);
        if (32 * wave < BQ && i_begin + n % q_tiles * BQ + 32 * wave < i_end)
            key_grad<T, DP>(lds[n & 1], lds[n & 1] + Ld::kBytes, row_lse[n & 1], row_delta[n & 1], 32 * wave, kf,
                            values, dk, dv, range_ds, range_p, a.by.c, false, 0, 0, lane);
        tile_barrier();
    }
    if constexpr (InRange<T>::kHalf) {
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) {
            dk[d] *= range_ds.undo();
            dv[d] *= range_p.undo();
        }
    }
    float(*joined)[DP][33] = reinterpret_cast<float(*)[DP][33]>(&lds[0][0]);
    for (int v = 0; v < 4; ++v) {
        if (wave == v) {
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int c = 32 * d + 8 * (r >> 2) + 4 * h + (r & 3);
                    joined[0][c][m] = (v ? joined[0][c][m] : 0.f) + dk[d][r];
                    joined[1][c][m] = (v ? joined[1][c][m] : 0.f) + dv[d][r];
                }
        }
        __syncthreads();
    }
    const int keys = min(32, a.far - 32 * tile);
    float* out = far_part(a, b, kv, item, tile);
    for (int x = tid; x < 2 * 32 * a.dim; x += 256) {
        const int c = x % a.dim, key = x / a.dim % 32;
        if (key < keys) out[x] = joined[x / (32 * a.dim)][c][key];
    }
}

}  // namespace nsl
