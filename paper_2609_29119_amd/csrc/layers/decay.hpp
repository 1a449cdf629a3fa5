// Linear attention along the bands with a decay for each head, and its step.
//
//   o_t = sum over s <= t of g^(t - s) (q_t . k_s) v_s        (times scale)
//
// Forward and gradients are one operator with its arguments in other places:
//   W(a, b, c)_t = sum_{s <= t} g^(t - s) (a_t . b_s) c_s     W' the same over s >= t
//   o = W(q, k, v)   dq = W(do, v, k)   dk = sum_heads W'(v, do, q)   dv = sum_heads W'(k, q, do)
// and W' is W with a band's tokens numbered from its end.
//
// In tiles of 32 tokens, with S = sum of g^(first - 1 - s) b_s c_s^T over the tokens before the tile:
//   out_i = g^(i + 1) a_i S + sum_{j <= i} g^(i - j) (a_i . b_j) c_j
//   S <- g^32 S + sum_j g^(31 - j) b_j c_j^T
// Every power's exponent is a distance: nothing grows, however fast a head forgets.
#pragma once
#include "pieces.hpp"

namespace nsl {

constexpr int kDecayTile = 32;

// One sum W or W' of a launch. Result head h belongs to key head h / per and
// takes the sources (key head) * many + {0 .. many - 1}.
struct DecayJob {
    View a, b, c, out;
    float* part;         // states within long bands, [batch][slots][kv_heads][dim][dim]
    int heads, per, many;
    bool reverse;        // W'
    bool turned;         // the states are those of the job with b and c exchanged
    bool keep_result;    // keep takes out results (else sources)
};

struct DecayArgs {
    DecayJob job[3];
    const float* log_decay;   // [kv_heads]
    float* state;             // [batch * n_bands][kv_heads][dim][dim] or NULL
    const uint8_t* keep;
    int64_t keep_batch;
    const int64_t* off;
    int rows, n_bands, batch, kv_heads, dim;
    int units;                // result heads of all jobs
    int shift;                // of a segment's length: what k_decay's workgroups walk through
    int fine;                 // of a part's: what k_decay_sum's do, in bands of several segments
    int64_t first_block;      // of a launch of k_decay_scan
    bool single;              // k_decay_sum: bands of one segment, into `state`
    float scale;
};

template <class T> __device__ inline T* decay_row(const View& v, int64_t b, int64_t row, int head) {
    return reinterpret_cast<T*>(v.data) + b * v.batch + row * v.row + head * v.head;
}

// decay^n of a head, rounded once.
__device__ inline float decay_power(double log_decay, int64_t n) {
    return n == 0 ? 1.f : static_cast<float>(exp(log_decay * static_cast<double>(n)));
}

// A state decays by n tokens many times over; with the factor rounded, by the
// same error each time: by 1e-5 after as many tiles as a slow head remembers. So
// where it is near 1 it is kept as its difference from 1,
struct DecayBy {
    bool near;
    float by;
    __device__ DecayBy(double log_decay, int64_t n) {
        const double less = expm1(log_decay * static_cast<double>(n));
        near = less > -0.5;
        by = near ? static_cast<float>(less) : decay_power(log_decay, n);
    }
    template <class V> __device__ V of(V s) const { return near ? s * by + s : s * by; }   // (one multiply-add)
};
// or, where a state's many values should take one multiplication each, its two
// neighbours in 32 bits take turns, so that their product so far is right to one
// rounding.
struct DecayFactors {
    float low, high, share, phase = 0.f;   // share: of the turns that are `high`'s
    __device__ static float uniform(float x) {
        return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x)));
    }
    __device__ DecayFactors(double log_decay, int64_t n) {
        const double factor = exp(log_decay * static_cast<double>(n));
        const float near = static_cast<float>(factor);
        const int bits = __builtin_bit_cast(int, near);
        const bool normal = factor > 1e-30 && factor < 1e30;
        const bool over = static_cast<double>(near) > factor;
        const float below = normal && over ? __builtin_bit_cast(float, bits - 1) : near;
        const float above = normal && !over ? __builtin_bit_cast(float, bits + 1) : near;
        low = uniform(below);
        high = uniform(above);
        share = uniform(normal ? static_cast<float>((factor - below) / (static_cast<double>(above) - below)) : 0.f);
    }
    __device__ float next() {
        phase += share;
        const bool turn = phase >= 1.f;
        phase = uniform(turn ? phase - 1.f : phase);
        return turn ? high : low;
    }
};

// As read_turned, with bits 2 and 3 of the column's number exchanged: a
// product's result whose rows are these columns then holds, in registers
// 8 s .. 8 s + 7 of a lane, the columns 16 s + 8 h + {0 .. 7}, which is the
// order in which `load8` holds a reduction's steps. So a state whose rows are
// b's columns is a fragment for the product with a as it is loaded.
template <class T, int RB> __device__ inline frag<T> read_turned_state(const char* tile, int row0, int col0, int lane) {
    const int h = lane >> 5;
    if constexpr (sizeof(T) == 2) {
        const int l16 = lane & 15, row = row0 + 4 * h + (l16 >> 2);
        const int c = ((col0 + (lane & 16)) >> 3) + (l16 & 1), at = (l16 & 2) << 2;
        const char* a = tile + row * RB + ((c ^ turn(row)) << 4) + at;
        const char* b = tile + (row + 8) * RB + ((c ^ turn(row + 8)) << 4) + at;
        const s4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)a);
        const s4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)b);
        const s8 z = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(frag<T>, z);
    } else {
        const int m = lane & 31, col = col0 + ((m & ~12) | ((m & 4) << 1) | ((m & 8) >> 1));
        frag<T> f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int row = row0 + 4 * h + (j & 3) + 8 * (j >> 2);
            f[j] = *reinterpret_cast<const T*>(tile + row * RB + (((col >> 2) ^ turn(row)) << 4) + ((col & 3) << 2));
        }
        return f;
    }
}

// What a workgroup of either kernel works on.
struct DecayPlace {
    int job, head, kv;
    int64_t b;
    Tile<int> seg;
    int n;          // the segment's (or part's) tokens
    bool outside;   // tokens that no band holds
    bool several;   // the band has more than one segment
    __device__ DecayPlace(const DecayArgs& a, int shift, int lane) {
        const unsigned id = last_first(blockIdx.x, gridDim.x), rest = id / a.units;
        head = static_cast<int>(id - rest * a.units);
        job = 0;
        while (head >= a.job[job].heads) head -= a.job[job++].heads;
        kv = head / a.job[job].per;
        b = rest % a.batch;
        seg = find_tile<int>(a.off, a.n_bands, a.rows, 1, shift, static_cast<int>(rest / a.batch), lane);
        n = min(seg.len - seg.first, 1 << shift);
        outside = seg.band < 0 || seg.band >= a.n_bands;
        several = seg.len > 1 << a.shift;
    }
    __device__ int64_t token(int t, bool reverse) const {   // the row's token of the segment's t-th
        return seg.start + (reverse ? seg.len - 1 - seg.first - t : seg.first + t);
    }
    // keep of tile `tile`, a bit for each of its tokens (all set without keep)
    __device__ unsigned kept(const DecayArgs& a, bool reverse, int tile, int lane) const {
        const int t = kDecayTile * tile + (lane & 31);
        const bool k = t < n && (!a.keep || a.keep[b * a.keep_batch + token(t, reverse)]);
        return static_cast<unsigned>(__ballot(k));
    }
};

// 32 tokens of one head of one tensor on their way into an LDS tile. Wide
// tensors go there directly: a wave's load fills 1 KB of it, its lanes fetch
// the chunks that belong there, and those whose token or column is not there
// or not kept aim past the buffer's end, which gives zeros. Other tensors go
// through registers, two chunks a thread. W' numbers tokens from the band's
// end: its buffers begin at the tile's last token.
template <class T, int DP, bool WIDE> struct DecayLoad {
    static constexpr int kThreads = 2 * DP, RB = row_bytes<T, DP>(), kLoads = kDecayTile * RB / 1024,
                         kEach = WIDE ? (kLoads + DP / 32 - 1) / (DP / 32) : 2;
    static constexpr unsigned kPast = 0x80000000u;   // past every tile, and less than 2^30 from its end
    const char* base;    // of the first tile's buffer
    int64_t step, head;  // bytes from tile to tile, from head to head
    int64_t row;         // and from token to token (wide: below 2^23)
    bool reverse;
    unsigned at[WIDE ? kEach : 1];
    frag<T> f[WIDE ? 1 : 2];

    static __device__ int token_of(int e, int tid) {   // of the thread's e-th chunk in a tile
        return WIDE ? ((wave_number() * kEach + e) * 1024 + (tid & 63) * 16) / RB : (tid + kThreads * e) / (DP / 8);
    }
    __device__ DecayLoad(const DecayArgs& a, const View& v, const DecayPlace& p, int first_head, bool rev, int tid) {
        reverse = rev;
        row = v.row * static_cast<int64_t>(sizeof(T));
        step = (rev ? -v.row : v.row) * static_cast<int64_t>(kDecayTile * sizeof(T));
        head = v.head * static_cast<int64_t>(sizeof(T));
        base = reinterpret_cast<const char*>(decay_row<T>(v, p.b, p.token(rev ? kDecayTile - 1 : 0, rev), first_head));
        if constexpr (WIDE) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const int byte = (wave_number() * kEach + e) * 1024 + (tid & 63) * 16, r = byte / RB;
                const unsigned d = ((byte % RB / 16) ^ turn(r)) * 16;
                at[e] = d < a.dim * sizeof(T) ? (rev ? kDecayTile - 1 - r : r) * static_cast<unsigned>(row) + d : kPast;
            }
        }
    }
    // kept: a bit for each of the tile's tokens that are there and kept
    __device__ void fetch(char* tile, const DecayArgs& a, int number, int g, unsigned kept, int tid) {
        const char* from = base + number * step + g * head;
        if constexpr (WIDE) {
#ifdef __HIP_DEVICE_COMPILE__   // the host pass does not know a buffer's type
            const auto buffer = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(from), 0, kDecayTile * static_cast<unsigned>(row), 0x00020000);
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const int load = wave_number() * kEach + e;
                if (kLoads % (DP / 32) && load >= kLoads) break;
                unsigned x = at[e];
                if (kept != ~0u && !(kept >> token_of(e, tid) & 1)) x = kPast;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer, (lds_void*)(tile + load * 1024), 16, x, 0, 0, 0);
            }
#endif
        } else {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = token_of(e, tid), d = (tid + kThreads * e) % (DP / 8) * 8;
                const T* p = reinterpret_cast<const T*>(from + (reverse ? kDecayTile - 1 - r : r) * row);
                f[e] = load8<T, false>(p + d, kept >> r & 1 ? a.dim - d : 0, d > 0);
            }
        }
    }
    __device__ void put(char* tile, int tid) const {
        if constexpr (!WIDE) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int c = tid + kThreads * e;
                write8<T, RB>(tile, c / (DP / 8), c % (DP / 8), f[e]);
            }
        }
    }
};

// S += b^T (w c): the wave's 32 columns of c, N pieces of w c.
template <class T, int DP, int N>
__device__ inline void decay_add(acc16 (&s)[DP / 32], const char* tb, frag<T> cf, f8 w, int step, int lane) {
    const auto cw = sum_of<T, N>(wide_of(cf) * w);
    each<DP / 32>([&](auto d) __attribute__((always_inline)) {
        const auto bf = data_of(read_turned_state<T, row_bytes<T, DP>()>(tb, 16 * step, 32 * d.value, lane));
        s[d.value] = product(bf, cw, s[d.value]);
    });
}

// 8 weights decay^(last - token), for the tokens of reduction step `step` in read_turned's order.
__device__ inline f8 decay_weights(const float* power, int last, int step, int h) {
    f8 w;
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = power[max(last - (16 * step + 4 * h + (j & 3) + 8 * (j >> 2)), 0)];
    return w;
}

// The state that a segment starts with, or the place of one: element [d][e] of the job's own order.
__device__ inline float* decay_state_of(const DecayArgs& a, const DecayJob& j, const DecayPlace& p, bool& there) {
    const int64_t size = static_cast<int64_t>(a.dim) * a.dim;
    there = true;
    if (p.several)
        return j.part + ((p.b * slot_count(a.rows, a.fine) + slot_of(p.seg.start, p.seg.first >> a.fine, a.fine)) *
                             a.kv_heads + p.kv) * size;
    if (a.state) return a.state + ((p.b * a.n_bands + p.seg.band) * a.kv_heads + p.kv) * size;
    there = false;
    return nullptr;
}

// out of one segment of one result head. The workgroup's waves hold 32 columns
// of the state each, in registers for the whole segment; the score tile, which
// all of them need, is formed by each (8 of 44 products at heads of 128). All
// products are formed transposed, so that the scores, the state and the result
// go from one to the next without a trip through LDS. Tiles of 32 tokens: the
// state's two pieces are formed anew for each, a third of the vector work.
// Scores, states and weighted sources meet 16-bit data as two pieces: off by 2^-16
// of a term, where the results are rounded to 2^-8 (float16: 2^-11) of themselves;
// with three pieces the two cases below take 17 and 28 % longer.
// 446,932 tokens, 8 heads of 64 over 4, bfloat16, 221 bands: 436 us (3.1 TB/s),
// of which loads and stores alone take 353; its three sums of the gradient in
// one launch 937, alone 743. 131,072 tokens, 8 heads of 128: 340 us, alone 228.
// Bound by waiting for rows of 128 and 256 bytes, far apart, with three (two)
// waves a SIMD.
template <class T, int DP, bool WIDE>
__global__ __launch_bounds__(2 * DP, sizeof(T) == 4 && DP >= 96 ? 1 : 2) void k_decay(DecayArgs a) {
    constexpr int RB = row_bytes<T, DP>(), ND = DP / 32, NK = DP / 16;
    constexpr bool kEarly = WIDE || (sizeof(T) == 2 && DP <= 64);   // the next tiles are on their way while these are computed
    __shared__ __align__(128) char ta[2][kDecayTile * RB], tb[2][kDecayTile * RB], tc[2][kDecayTile * RB];
    __shared__ float power[kDecayTile + 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), m = lane & 31, h = lane >> 5;
    const DecayPlace p(a, a.shift, lane);
    if (!p.seg.live) return;
    const DecayJob& j = a.job[p.job];
    const bool reverse = j.reverse;
    if (p.outside) {
        for (int t = m; t < p.n; t += 32)
            store_column<T>(decay_row<T>(j.out, p.b, p.token(t, reverse), p.head), zero16(), 32 * wave, a.dim, WIDE, lane);
        return;
    }
    const int count = (p.n + kDecayTile - 1) / kDecayTile;
    DecayLoad<T, DP, WIDE> la(a, j.a, p, p.head, reverse, tid), lb(a, j.b, p, p.kv * j.many, reverse, tid),
        lc(a, j.c, p, p.kv * j.many, reverse, tid);
    // (where keep takes out results, the sources are all those that exist)
    auto exist = [&](int tile) { return p.n - kDecayTile * tile >= kDecayTile ? ~0u : (1u << (p.n - kDecayTile * tile)) - 1; };
    auto kept_of = [&](int tile) { return a.keep ? p.kept(a, reverse, tile, lane) : exist(tile); };
    auto fetch_a = [&](int tile, unsigned k) { la.fetch(ta[tile & 1], a, tile, 0, j.keep_result ? k : exist(tile), tid); };
    auto fetch_bc = [&](int stage, int tile, int g, unsigned k) {
        const unsigned use = j.keep_result ? exist(tile) : k;
        lb.fetch(tb[stage & 1], a, tile, g, use, tid);
        lc.fetch(tc[stage & 1], a, tile, g, use, tid);
    };
    unsigned kept = kept_of(0), kept_next = 0;
    fetch_a(0, kept);
    fetch_bc(0, 0, 0, kept);
    if (count > 1) kept_next = kept_of(1);
    const double log_decay = a.log_decay[p.kv];
    DecayFactors across(log_decay, kDecayTile);
    if (tid <= kDecayTile) power[tid] = decay_power(log_decay, tid);
    acc16 s[ND];
    bool some;
    const float* from = decay_state_of(a, j, p, some);
    const int col = 32 * wave + m;
#pragma unroll
    for (int d = 0; d < ND; ++d) s[d] = zero16();
    if (some) {
        const int64_t sd = j.turned ? 1 : a.dim, sc = j.turned ? a.dim : 1;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = 32 * d + 16 * (r >> 3) + 8 * h + (r & 7);
                if (row < a.dim && col < a.dim) s[d][r] = from[row * sd + col * sc];
            }
    }
    la.put(ta[0], tid);
    lb.put(tb[0], tid);
    lc.put(tc[0], tid);
    tile_barrier();
    float fade[16];   // scale decay^(i - j) where j <= i
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int lag = m - (8 * (r >> 2) + 4 * h + (r & 3));
        fade[r] = lag < 0 ? 0.f : power[lag] * a.scale;
    }
    const float up = power[m + 1] * a.scale;
    T* to = decay_row<T>(j.out, p.b, p.token(m, reverse), p.head);   // (of the last tile, perhaps past the segment: not used)
    const int64_t to_step = (reverse ? -j.out.row : j.out.row) * kDecayTile;
    int stage = 0;
    for (int tile = 0; tile < count; ++tile) {
        const bool last = tile + 1 == count;
        const char* xa = ta[tile & 1];
        const unsigned kept_now = kept;
        acc16 out = zero16();
        for (int g = 0; g < j.many; ++g, ++stage) {
            const bool end = g + 1 == j.many, more = !(end && last);
            const char *xb = tb[stage & 1], *xc = tc[stage & 1];
            const int next_tile = end ? tile + 1 : tile;
            if (end) kept = kept_next;
            auto fetch = [&]() __attribute__((always_inline)) {
                if (!more) return;
                if (end) fetch_a(next_tile, kept);
                fetch_bc(stage + 1, next_tile, end ? 0 : g + 1, kept);
            };
            if (kEarly) fetch();
            if (end && tile + 2 < count) kept_next = kept_of(tile + 2);
            if (g == 0) {
                each<NK>([&](auto x) __attribute__((always_inline)) {
                    if (DP <= 64 && 16 * x.value >= a.dim) return;   // (wider heads: the branches cost more, 334 -> 368 us)
                    const auto af = data_of(read8<T, RB>(xa, m, 2 * x.value + h));
                    out = product(sum_of<T, 2>(octet(s[x.value / 2], x.value % 2)), af, out);
                });
                out *= up;
                const float by = across.next();
#pragma unroll
                for (int d = 0; d < ND; ++d) s[d] *= by;
            }
            acc16 q = zero16();
            each<NK>([&](auto x) __attribute__((always_inline)) {
                if (DP > 64 || 16 * x.value < a.dim) q = mma(read8<T, RB>(xb, m, 2 * x.value + h), read8<T, RB>(xa, m, 2 * x.value + h), q);
            });
#pragma unroll
            for (int r = 0; r < 16; ++r) q[r] *= fade[r];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const frag<T> cf = read_turned<T, RB>(xc, 16 * x, 32 * wave, lane);
                out = product(data_of(cf), sum_of<T, 2>(octet(q, x)), out);
                if (!last) decay_add<T, DP, 2>(s, xb, cf, decay_weights(power, kDecayTile - 1, x, h), x, lane);
            }
            if (more) {
                if (!kEarly) fetch();
                if (end) la.put(ta[next_tile & 1], tid);
                lb.put(tb[(stage + 1) & 1], tid);
                lc.put(tc[(stage + 1) & 1], tid);
            }
            if (end) {
                if (a.keep && j.keep_result && !(kept_now >> m & 1)) out = zero16();
                store_column<T>(kDecayTile * tile + m < p.n ? to : nullptr, out, 32 * wave, a.dim, WIDE, lane);
                to += to_step;
            }
            tile_barrier();
        }
    }
}

// What a part adds to the state, sum_s g^(n - 1 - s) b_s c_s^T, into its slot:
// for bands of several segments, up to the last one's start (to the band's end
// where a state is kept). single: bands of one segment, whose state in `state`
// goes on. Three pieces of w c: the states are 32-bit results. 131,072 tokens, 8
// heads of 128, bfloat16: 86 us (6.2 TB/s, some of it from the memory-side cache).
template <class T, int DP, bool WIDE>
__global__ __launch_bounds__(2 * DP, 2) void k_decay_sum(DecayArgs a) {
    constexpr int RB = row_bytes<T, DP>(), ND = DP / 32;
    __shared__ __align__(128) char tb[2][kDecayTile * RB], tc[2][kDecayTile * RB];
    __shared__ float power[kDecayTile + 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), m = lane & 31, h = lane >> 5;
    const DecayPlace p(a, a.single ? a.shift : a.fine, lane);
    if (!p.seg.live || p.outside || p.several == a.single) return;
    const DecayJob& j = a.job[p.job];
    if (!a.state && p.seg.first >> a.shift == (p.seg.len - 1) >> a.shift) return;
    const int count = (p.n + kDecayTile - 1) / kDecayTile, stages = count * j.many;
    DecayLoad<T, DP, WIDE> lb(a, j.b, p, p.kv * j.many, j.reverse, tid), lc(a, j.c, p, p.kv * j.many, j.reverse, tid);
    auto use = [&](int tile) {
        if (a.keep && !j.keep_result) return p.kept(a, j.reverse, tile, lane);
        return p.n - kDecayTile * tile >= kDecayTile ? ~0u : (1u << (p.n - kDecayTile * tile)) - 1;
    };
    auto fetch = [&](int stage, int tile, int g, unsigned k) {
        lb.fetch(tb[stage & 1], a, tile, g, k, tid);
        lc.fetch(tc[stage & 1], a, tile, g, k, tid);
    };
    unsigned kept = use(0), kept_next = 0;
    fetch(0, 0, 0, kept);
    if (count > 1) kept_next = use(1);
    const double log_decay = a.log_decay[p.kv];
    DecayFactors across(log_decay, kDecayTile);
    if (tid <= kDecayTile) power[tid] = decay_power(log_decay, tid);
    bool there;
    float* to = decay_state_of(a, j, p, there);
    const int col = 32 * wave + m;
    acc16 s[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = 32 * d + 16 * (r >> 3) + 8 * h + (r & 7);
            s[d][r] = a.single && row < a.dim && col < a.dim ? to[row * a.dim + col] : 0.f;
        }
    lb.put(tb[0], tid);
    lc.put(tc[0], tid);
    tile_barrier();
    int tile = 0, g = 0;
    for (int stage = 0; stage < stages; ++stage) {
        const bool more = stage + 1 < stages, end = g + 1 == j.many;
        const char *xb = tb[stage & 1], *xc = tc[stage & 1];
        const int n = min(p.n - kDecayTile * tile, kDecayTile);
        if (end) kept = kept_next;
        if (more) fetch(stage + 1, end ? tile + 1 : tile, end ? 0 : g + 1, kept);
        if (end && tile + 2 < count) kept_next = use(tile + 2);
        if (g == 0) {
            const float by = n == kDecayTile ? across.next() : power[n];
#pragma unroll
            for (int d = 0; d < ND; ++d) s[d] *= by;
        }
#pragma unroll
        for (int x = 0; x < 2; ++x)
            decay_add<T, DP, 3>(s, xb, read_turned<T, RB>(xc, 16 * x, 32 * wave, lane),
                                decay_weights(power, n - 1, x, h), x, lane);
        if (end) {
            g = 0;
            ++tile;
        } else {
            ++g;
        }
        if (more) {
            lb.put(tb[(stage + 1) & 1], tid);
            lc.put(tc[(stage + 1) & 1], tid);
        }
        tile_barrier();
    }
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = 32 * d + 16 * (r >> 3) + 8 * h + (r & 7);
            if (row < a.dim && col < a.dim) to[row * a.dim + col] = s[d][r];
        }
}

// From what each part adds to the state that each segment starts with, in
// place, along every band of several; `state` goes to the band's end. A thread
// takes V neighbouring elements, 16 parts on their way at once: 128 parts of 8
// heads of 128 x 128 in 29 us.
template <int V> constexpr int decay_scan_part() { return 256 * V; }   // elements of a workgroup
template <int V> __global__ __launch_bounds__(256) void k_decay_scan(DecayArgs a) {
    typedef float vec __attribute__((ext_vector_type(V)));
    const int size = a.dim * a.dim, parts = (size + decay_scan_part<V>() - 1) / decay_scan_part<V>();
    int64_t id = a.first_block + blockIdx.x;
    const int e = (static_cast<int>(id % parts) * 256 + static_cast<int>(threadIdx.x)) * V;
    id /= parts;
    const int u = static_cast<int>(id % a.units), job = u / a.kv_heads, kv = u % a.kv_heads;
    id /= a.units;
    const int band = static_cast<int>(id % a.n_bands);
    const int64_t b = id / a.n_bands;
    const int start = band_bound(a.off, a.n_bands, a.rows, band + 1), len = band_bound(a.off, a.n_bands, a.rows, band + 2) - start;
    if (len <= 1 << a.shift || e >= size) return;
    const double log_decay = a.log_decay[kv];
    const DecayBy across(log_decay, int64_t(1) << a.fine);
    const int count = (len + (1 << a.fine) - 1) >> a.fine, each = (1 << (a.shift - a.fine)) - 1;
    const int last = (len - 1) >> a.shift << (a.shift - a.fine);   // the part that the last segment starts with
    const int64_t step = static_cast<int64_t>(a.kv_heads) * size;
    float* x = a.job[job].part + ((b * slot_count(a.rows, a.fine) + slot_of(start, 0, a.fine)) * a.kv_heads + kv) * size + e;
    float* st = a.state ? a.state + ((b * a.n_bands + band) * a.kv_heads + kv) * size + e : nullptr;
    auto at = [&](int i) -> vec& { return *reinterpret_cast<vec*>(x + i * step); };
    vec s = st ? *reinterpret_cast<vec*>(st) : vec(0.f);
    const int end = st ? count - 1 : last;   // (the band's last part may be a short one)
    constexpr int kAhead = 16;
    for (int i = 0; i < end; i += kAhead) {
        vec add[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) add[k] = i + k < end ? at(i + k) : vec(0.f);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (i + k < end) {
                if (((i + k) & each) == 0) at(i + k) = s;
                s = across.of(s) + add[k];
            }
    }
    if (st) *reinterpret_cast<vec*>(st) = decay_power(log_decay, len - (static_cast<int64_t>(end) << a.fine)) * s + at(end);
    if ((end & each) == 0) at(end) = s;
}

// ------------------------------------------------------------- single tokens

struct DecayStepArgs {
    View q, k, v, o;   // batch stride: from stream to stream
    float* state;      // [streams][kv_heads][dim][dim]
    const int64_t* pos;
    const float* log_decay;
    int heads, kv_heads, dim, group;
    float scale;
};

// S <- g S + k v^T, o = scale q S for the query heads of one key head of one
// stream. A thread holds V neighbouring columns of every kRows-th row of the
// state in registers; the rows' sums meet in LDS. Bound by the states, read and
// written once: 3,536 streams, 4 heads of 64 x 64, 65 us and 88 a call among
// others (92 at the rate of a large copy; a part of them stays in the
// memory-side cache). One stream: 3.8 us.
template <class T, int DP, int V>
__global__ __launch_bounds__(256) void k_decay_step(DecayStepArgs a) {
    constexpr int kCols = DP / V, kRows = 256 / kCols, kEach = DP / kRows, kHeads = 4;
    __shared__ float sums[kHeads][kRows][DP + 4];
    __shared__ float ks[DP], qs[kHeads][DP];
    typedef float vec __attribute__((ext_vector_type(V)));
    const int tid = threadIdx.x, c0 = tid % kCols * V, r0 = tid / kCols;
    const int64_t stream = blockIdx.x / a.kv_heads;
    const int kv = static_cast<int>(blockIdx.x % a.kv_heads);
    const int64_t pos = a.pos[stream];
    auto q_of = [&](int g) { return reinterpret_cast<const T*>(a.q.data) + stream * a.q.batch + static_cast<int64_t>(kv * a.group + g) * a.q.head; };
    auto o_of = [&](int g) { return reinterpret_cast<T*>(a.o.data) + stream * a.o.batch + static_cast<int64_t>(kv * a.group + g) * a.o.head; };
    if (pos < 0) {
        for (int e = tid; e < a.group * a.dim; e += 256) o_of(e / a.dim)[e % a.dim] = static_cast<T>(0.f);
        return;
    }
    const T* kp = reinterpret_cast<const T*>(a.k.data) + stream * a.k.batch + kv * a.k.head;
    const T* vp = reinterpret_cast<const T*>(a.v.data) + stream * a.v.batch + kv * a.v.head;
    float* st = a.state + static_cast<int64_t>(blockIdx.x) * a.dim * a.dim;
    vec s[kEach], v = 0.f;
    if (pos > 0) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int r = r0 + kRows * i;
            s[i] = r < a.dim && c0 < a.dim ? *reinterpret_cast<const vec*>(st + r * a.dim + c0) : vec(0.f);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i) s[i] = 0.f;
    }
    if (c0 < a.dim)
#pragma unroll
        for (int x = 0; x < V; ++x) v[x] = static_cast<float>(vp[c0 + x]);
    const DecayBy fade(a.log_decay[kv], 1);
    if (tid < DP) ks[tid] = tid < a.dim ? static_cast<float>(kp[tid]) : 0.f;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int r = r0 + kRows * i;
        const float kr = ks[r];
#pragma unroll
        for (int x = 0; x < V; ++x) s[i][x] = fmaf(kr, v[x], pos > 0 ? fade.of(s[i][x]) : 0.f);
        if (r < a.dim && c0 < a.dim) *reinterpret_cast<vec*>(st + r * a.dim + c0) = s[i];
    }
    for (int g0 = 0; g0 < a.group; g0 += kHeads) {
        const int n = min(a.group - g0, kHeads);
        __syncthreads();
        for (int e = tid; e < n * DP; e += 256)
            qs[e / DP][e % DP] = e % DP < a.dim ? static_cast<float>(q_of(g0 + e / DP)[e % DP]) : 0.f;
        __syncthreads();
        for (int g = 0; g < n; ++g) {
            vec sum = 0.f;
#pragma unroll
            for (int i = 0; i < kEach; ++i) sum += s[i] * qs[g][r0 + kRows * i];
#pragma unroll
            for (int x = 0; x < V; ++x) sums[g][r0][c0 + x] = sum[x];
        }
        __syncthreads();
        for (int e = tid; e < n * DP; e += 256) {
            const int g = e / DP, c = e % DP;
            float sum = 0.f;
#pragma unroll
            for (int r = 0; r < kRows; ++r) sum += sums[g][r][c];
            if (c < a.dim) o_of(g0 + g)[c] = static_cast<T>(sum * a.scale);
        }
    }
}

}  // namespace nsl
