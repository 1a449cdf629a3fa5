// Matrix fragments, LDS tiles and the search for a block's band: what the
// layer kernels share.
//
// Fragments. Every product is built from 32 x 32 tiles of the matrix cores
// with 16 reduction steps a call. A lane l = 32 h + m holds 8 consecutive
// reduction steps (8 h .. 8 h + 7) of row m of A, or of column m of B. In 16
// bits that is one v_mfma_f32_32x32x16; in 32 bits it is eight
// v_mfma_f32_32x32x2, call j taking step j of either half: the order in which
// a reduction's steps are taken is free as long as A and B agree. So one code
// serves all three types. The result's register r of lane l is element
// (row 8 (r / 4) + 4 h + r % 4, column m).
//
// Chains without a trip through LDS. With the scores formed as S^T = K Q^T
// (row: key, column: query), registers 8 s .. 8 s + 7 of a lane hold keys
// 16 s + 4 h + {0..3} and 16 s + 8 + 4 h + {0..3} of its query. Taken as they
// are, they are a B fragment of the next product's 16 steps, if its A
// fragment takes its steps in that same order (`read_turned`).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace nsl {

typedef float acc16 __attribute__((ext_vector_type(16)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f8 __attribute__((ext_vector_type(8)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef __bf16 b4 __attribute__((ext_vector_type(4)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));
typedef unsigned u2 __attribute__((ext_vector_type(2)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));

template <class T> struct Type;
template <> struct Type<float> { typedef f8 v8; typedef f4 v4; };
template <> struct Type<_Float16> { typedef h8 v8; typedef h4 v4; };
template <> struct Type<__bf16> { typedef b8 v8; typedef b4 v4; };
template <class T> using frag = typename Type<T>::v8;
template <class T> using quad = typename Type<T>::v4;

__device__ inline acc16 mma(h8 a, h8 b, acc16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ inline acc16 mma(b8 a, b8 b, acc16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ inline acc16 mma(f8 a, f8 b, acc16 c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
}

template <class T> __device__ inline frag<T> zero8() {
    frag<T> f;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = static_cast<T>(0.f);
    return f;
}

__device__ inline acc16 zero16() {
    acc16 c;
#pragma unroll
    for (int r = 0; r < 16; ++r) c[r] = 0.f;
    return c;
}

// Registers 8 s .. 8 s + 7 of c, rounded to T: the next product's B fragment.
template <class T> __device__ inline frag<T> narrow(const acc16& c, int s) {
    frag<T> f;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = static_cast<T>(c[8 * s + j]);
    return f;
}

// What `narrow` left of them, rounded to T in turn. The two fragments together
// hold 16 bits of each value in bfloat16 and 22 in float16.
template <class T> __device__ inline frag<T> rest_of(const acc16& c, int s, const frag<T>& f) {
    frag<T> low;
#pragma unroll
    for (int j = 0; j < 8; ++j) low[j] = static_cast<T>(c[8 * s + j] - static_cast<float>(f[j]));
    return low;
}

// 8 values at p, of which the first n are there (n may be <= 0 or past 8).
// WIDE: p is 16-byte aligned and n is never between 0 and 8. Else p is
// aligned to its element only, which the memory pipeline takes too; a row's
// last values come from the 8 that end it (before: 8 values lie in front of
// p) and are shifted down. Callers branch on the alignment around a group of
// loads, not at each one, which would keep them from being in flight together.
template <class T, bool WIDE> __device__ inline frag<T> load8(const T* p, int n, bool before = false) {
    frag<T> f = zero8<T>();
    if constexpr (WIDE) {
        if (n > 0) f = *reinterpret_cast<const frag<T>*>(p);
    } else if (n >= 8) {
        __builtin_memcpy(&f, p, sizeof(f));
    } else if (n > 0) {
        if constexpr (sizeof(T) == 2) {
            if (before) {
                uint64_t u[2];
                __builtin_memcpy(u, p + n - 8, 16);
                const int s = 16 * (8 - n);
                const uint64_t lo = s >= 64 ? u[1] >> (s - 64) : (u[0] >> s) | (u[1] << (64 - s));
                const uint64_t hi = s >= 64 ? 0 : u[1] >> s;
                const u4 w = {static_cast<unsigned>(lo), static_cast<unsigned>(lo >> 32), static_cast<unsigned>(hi),
                              static_cast<unsigned>(hi >> 32)};
                return __builtin_bit_cast(frag<T>, w);
            }
        }
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < n) f[j] = p[j];
    }
    return f;
}

// f(0), ..., f(N - 1) with integral constants: a loop over an array that has to
// stay in registers where the code around it is too large for the unroller.
template <int N, int I = 0, class F> __device__ __attribute__((always_inline)) inline void each(F f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>());
        each<N, I + 1>(f);
    }
}

// f(true_type or false_type)
template <class F> __device__ inline void by_width(bool wide, F f) {
    if (wide)
        f(std::true_type());
    else
        f(std::false_type());
}

// The values of lane l % 32 and lane l % 32 + 32, in every lane.
__device__ inline void halves(float x, float& low, float& high) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const u2 r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const unsigned a = r[0], b = r[1];   // (a bit cast of a vector's element reads element 0)
    low = __builtin_bit_cast(float, a);
    high = __builtin_bit_cast(float, b);
}
__device__ inline float half_max(float x) {
    float a, b;
    halves(x, a, b);
    return fmaxf(a, b);
}
__device__ inline float half_sum(float x) {
    float a, b;
    halves(x, a, b);
    return a + b;
}

// ------------------------------------------------------------------ LDS tiles

// A tile's row takes 128 bytes or a multiple; its 16-byte chunks lie at
// chunk ^ turn(row), so that `read8` (consecutive rows, one chunk) finds eight
// rows in eight different places of 128 bytes, and the transposed read (four
// rows, two chunks) four rows in four. What conflicts are left (between a
// quarter and a half of LDS' active cycles in the attention kernels) cost no
// time: a layout that takes them out of read8 altogether gave the same figures.
template <class T, int D> constexpr int row_bytes() { return (D * static_cast<int>(sizeof(T)) + 127) / 128 * 128; }
__device__ inline int turn(int row) { return ((row & 3) << 1) | ((row >> 2) & 1); }

// Columns 8 c8 .. 8 c8 + 7 of `row`.
template <class T> __device__ inline frag<T> read8(const char* tile, int rb, int row, int c8) {
    const char* r = tile + row * rb;
    const int t = turn(row);
    if constexpr (sizeof(T) == 2) {
        return *reinterpret_cast<const frag<T>*>(r + ((c8 ^ t) << 4));
    } else {
        const f4 a = *reinterpret_cast<const f4*>(r + (((2 * c8) ^ t) << 4));
        const f4 b = *reinterpret_cast<const f4*>(r + (((2 * c8 + 1) ^ t) << 4));
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
}

template <class T, int RB> __device__ inline frag<T> read8(const char* tile, int row, int c8) {
    return read8<T>(tile, RB, row, c8);
}

template <class T> __device__ inline void write8(char* tile, int rb, int row, int c8, frag<T> f) {
    char* r = tile + row * rb;
    const int t = turn(row);
    if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<frag<T>*>(r + ((c8 ^ t) << 4)) = f;
    } else {
        *reinterpret_cast<f4*>(r + (((2 * c8) ^ t) << 4)) = __builtin_shufflevector(f, f, 0, 1, 2, 3);
        *reinterpret_cast<f4*>(r + (((2 * c8 + 1) ^ t) << 4)) = __builtin_shufflevector(f, f, 4, 5, 6, 7);
    }
}

template <class T, int RB> __device__ inline void write8(char* tile, int row, int c8, frag<T> f) {
    write8<T>(tile, RB, row, c8, f);
}

typedef __attribute__((address_space(3))) s4 lds_s4;
typedef __attribute__((address_space(3))) void lds_void;   // where a direct load into LDS goes

// Every LDS write of this wave, the direct ones too, is done; then all waves'.
__device__ inline void tile_barrier() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
}

// A fragment of the tile's transpose: for column col0 + (lane % 32), rows
// row0 + 4 h + {0..3} and row0 + 8 + 4 h + {0..3}, h = lane / 32 (row0 and
// col0 multiples of 16 and 32). In 16 bits ds_read_b64_tr_b16 turns 4 x 16
// blocks on the way out of LDS.
template <class T, int RB> __device__ inline frag<T> read_turned(const char* tile, int row0, int col0, int lane) {
    const int h = lane >> 5;
    if constexpr (sizeof(T) == 2) {
        const int l16 = lane & 15, row = row0 + 4 * h + (l16 >> 2);
        const int c = ((col0 + (lane & 16)) >> 3) + ((l16 & 3) >> 1);
        const char* a = tile + row * RB + ((c ^ turn(row)) << 4) + ((l16 & 1) << 3);
        const char* b = tile + (row + 8) * RB + ((c ^ turn(row + 8)) << 4) + ((l16 & 1) << 3);
        const s4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)a);
        const s4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)b);
        const s8 z = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(frag<T>, z);
    } else {
        const int col = col0 + (lane & 31);
        frag<T> f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int row = row0 + 4 * h + (j & 3) + 8 * (j >> 2);
            f[j] = *reinterpret_cast<const T*>(tile + row * RB + (((col >> 2) ^ turn(row)) << 4) + ((col & 3) << 2));
        }
        return f;
    }
}

// As read_turned, with rows row0 + 8 h + {0..7}: the order in which `load8`
// and `read8` hold a reduction's steps.
template <class T, int RB> __device__ inline frag<T> read_turned8(const char* tile, int row0, int col0, int lane) {
    const int h = lane >> 5;
    if constexpr (sizeof(T) == 2) {
        const int l16 = lane & 15, row = row0 + 8 * h + (l16 >> 2);
        const int c = ((col0 + (lane & 16)) >> 3) + ((l16 & 3) >> 1);
        const char* a = tile + row * RB + ((c ^ turn(row)) << 4) + ((l16 & 1) << 3);
        const char* b = tile + (row + 4) * RB + ((c ^ turn(row + 4)) << 4) + ((l16 & 1) << 3);
        const s4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)a);
        const s4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)b);
        const s8 z = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(frag<T>, z);
    } else {
        const int col = col0 + (lane & 31);
        frag<T> f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int row = row0 + 8 * h + j;
            f[j] = *reinterpret_cast<const T*>(tile + row * RB + (((col >> 2) ^ turn(row)) << 4) + ((col & 3) << 2));
        }
        return f;
    }
}

// ---------------------------------------------------------------------- stores

// Stores rows 0 .. 31 of a result tile, held as registers of column m = one
// token: element d0 + row of the token's row p (NULL: nothing), d below n.
// wide: 16-byte aligned rows and n a multiple of 8; else rows are aligned to
// their element only. In 16 bits the halves of the wave exchange quads, so
// that each lane stores 8 consecutive values.
template <class T> __device__ inline void store_column(T* p, const acc16& c, int d0, int n, bool wide, int lane) {
    const int h = lane >> 5;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const frag<T> f = narrow<T>(c, s);
            const u4 u = __builtin_bit_cast(u4, f);
            const u2 x = __builtin_amdgcn_permlane32_swap(u[0], u[2], false, false);
            const u2 y = __builtin_amdgcn_permlane32_swap(u[1], u[3], false, false);
            const u4 out = {x[0], y[0], x[1], y[1]};
            const int d = d0 + 16 * s + 8 * h;
            if (!p || d >= n) continue;
            if (wide) {
                *reinterpret_cast<u4*>(p + d) = out;
            } else if (d + 8 <= n) {
                __builtin_memcpy(p + d, &out, 16);
            } else {
                const frag<T> g = __builtin_bit_cast(frag<T>, out);
#pragma unroll
                for (int j = 0; j < 7; ++j)
                    if (d + j < n) p[d + j] = g[j];
            }
        }
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int d = d0 + 8 * q + 4 * h;
            const f4 v = {c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]};
            if (!p || d >= n) continue;
            if (wide) {
                *reinterpret_cast<f4*>(p + d) = v;
            } else if (d + 4 <= n) {
                __builtin_memcpy(p + d, &v, 16);
            } else {
#pragma unroll
                for (int j = 0; j < 3; ++j)
                    if (d + j < n) p[d + j] = v[j];
            }
        }
    }
}

// Lane l's pointer.
template <class P> __device__ inline P from_lane(P p, int l) {
    return reinterpret_cast<P>(__shfl(reinterpret_cast<unsigned long long>(p), l));
}

// Stores a wave's result, 128 bytes of each of its rows at a time, through
// 4 KB of LDS of its own: lane l's column is row l % 32; row_out: the rows
// lane / 8 + {0, 8, 16, 24}, of which those below `there` exist.
template <class T, int NB>
__device__ inline void store_rows(char* slab, const acc16 (&acc)[NB], T* const (&row_out)[4], int there, int c0,
                                  int n_col, bool y_wide, int lane) {
    constexpr int kSlab = 128 / (32 * static_cast<int>(sizeof(T)));   // tiles of 32 columns in 128 bytes
    constexpr int kIn16 = 16 / static_cast<int>(sizeof(T));
    const int m = lane & 31, h = lane >> 5;
    each<(NB + kSlab - 1) / kSlab>([&](auto z) __attribute__((always_inline)) {
        constexpr int n0 = decltype(z)::value * kSlab;
        each<kSlab>([&](auto x) __attribute__((always_inline)) {
            constexpr int nb = n0 + decltype(x)::value;
            if constexpr (nb < NB) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    quad<T> v;
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = static_cast<T>(acc[nb][4 * q + j]);
                    const int byte = (32 * decltype(x)::value + 8 * q + 4 * h) * static_cast<int>(sizeof(T));
                    *reinterpret_cast<quad<T>*>(slab + m * 128 + (((byte >> 4) ^ turn(m)) << 4) + (byte & 15)) = v;
                }
            }
        });
        const int d = c0 + 32 * n0 + lane % 8 * kIn16;
        by_width(y_wide, [&](auto wide) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int row = lane / 8 + 8 * e;
                const u4 v = *reinterpret_cast<const u4*>(slab + row * 128 + ((lane % 8 ^ turn(row)) << 4));
                if (row >= there || d >= n_col || 32 * n0 + lane % 8 * kIn16 >= 32 * NB) continue;
                if (wide.value) {
                    *reinterpret_cast<u4*>(row_out[e] + d) = v;
                } else if (d + kIn16 <= n_col) {
                    __builtin_memcpy(row_out[e] + d, &v, 16);
                } else {
                    T x[kIn16];
                    __builtin_memcpy(x, &v, 16);
#pragma unroll
                    for (int j = 0; j < kIn16 - 1; ++j)
                        if (d + j < n_col) row_out[e][d + j] = x[j];
                }
            }
        });
    });
}

// ---------------------------------------------------------------- work items

// Which of n work items block `id` takes. Blocks go to the 8 compute dies in
// turn; each die gets stretches of 16 neighbouring items, which share its L2,
// and stretches from everywhere: bands grow along the row, and with one eighth
// of it for each die the last die has most of the work.
__device__ inline unsigned die_order(unsigned id, unsigned n) {
    constexpr unsigned kStretch = 16;
    if (id >= n / (8 * kStretch) * (8 * kStretch)) return id;
    const unsigned die = id & 7, k = id >> 3;
    return (k / kStretch * 8 + die) * kStretch + k % kStretch;
}

// The same from the row's end: where bands grow along the row, the longest work
// begins first and the shortest fills the end.
__device__ inline unsigned last_first(unsigned id, unsigned n) { return n - 1 - die_order(id, n); }

// I: int where a band's mult * len rows stay below 2^30, else int64_t.
template <class I> struct Tile {
    int band;    // -1: tokens before the first band, n_bands: after the last
    int start;   // the band's first token
    int len;     // and its number of tokens
    I first;     // the tile's first row of the band's mult * len rows
    bool live;   // false: nothing to do
};

// Tiles of 2^shift rows of the bands' mult * len rows each, without a table:
// band i's tiles begin at item floor(mult start_i / 2^shift) + i, which
// leaves room for each band's ragged last tile, so tile_count() items hold
// them all and some items are empty. The band of item p is found by a search
// over the offsets, 64 at a time: one or two rounds of loads.
inline __host__ __device__ int64_t tile_count(int shift, int64_t n_bands, int64_t mult, int64_t rows) {
    return ((mult * rows) >> shift) + n_bands + 2;
}

inline __host__ __device__ int band_bound(const int64_t* off, int n_bands, int rows, int i) {
    if (i <= 0) return 0;
    if (i >= n_bands + 2) return rows;
    const int64_t o = off[i - 1];
    return o < 0 ? 0 : o > rows ? rows : static_cast<int>(o);
}

// The band of item p among the bounds lo .. hi - 1, in rounds of 64 bounds
// that are `step` apart: a round's `count` is how many of them, from lo on,
// begin at or before p. At the end `lo` is the band's bound, which lane `at`
// of the last round held; its next lane held the next bound only if that
// round went in steps of one (a round in larger steps may end the search too:
// when its last bound is the only one left).
struct BandSearch {
    int lo = 0, hi, step = 0, at = 0;
    __host__ __device__ explicit BandSearch(int n_bands) : hi(n_bands + 2) {}
    __host__ __device__ bool more() const { return hi - lo > 1; }
    __host__ __device__ void open() { step = (hi - lo + 63) >> 6; }
    __host__ __device__ void close(int count) {
        at = count > 1 ? count - 1 : 0;
        lo += at * step;
        hi = lo + step < hi ? lo + step : hi;
    }
    __host__ __device__ bool next_held() const { return step == 1 && at < 63; }
};

// Whether item p lies at or behind the first item of bound i, token `bound`.
template <class I> __host__ __device__ inline bool item_from(I mult, int bound, int shift, int i, I p) {
    return ((mult * bound) >> shift) + i <= p;
}

// The tile of item p, between the bounds a (of band lo - 1) and b.
template <class I> __host__ __device__ inline Tile<I> tile_of(int lo, int a, int b, I mult, int shift, I p) {
    Tile<I> t;
    t.band = lo - 1;
    t.start = a;
    t.len = b > a ? b - a : 0;
    t.first = (p - (((mult * a) >> shift) + lo)) << shift;
    t.live = t.first >= 0 && t.first < mult * t.len;
    return t;
}

template <class I>
__device__ inline Tile<I> find_tile(const int64_t* off, int n_bands, int rows, I mult, int shift, I p, int lane) {
    BandSearch s(n_bands);
    int bound = 0;
    while (s.more()) {
        s.open();
        const int i = s.lo + lane * s.step;
        bound = band_bound(off, n_bands, rows, i);
        s.close(__popcll(__ballot(i < s.hi && item_from(mult, bound, shift, i, p))));
    }
    const int lo = __builtin_amdgcn_readfirstlane(s.lo), at = __builtin_amdgcn_readfirstlane(s.at);
    const int a = __builtin_amdgcn_readlane(bound, at);
    const int b = s.next_held() ? __builtin_amdgcn_readlane(bound, at + 1) : band_bound(off, n_bands, rows, lo + 1);
    return tile_of(lo, a, b, mult, shift, p);
}

// Slots for the segments of 2^shift = T tokens of those bands that have
// several, without a table: a band of more than T tokens that starts at token
// `start` has those from floor(2 start / T) on, and its ceil(len / T) segments
// end before the next such band's first, as floor(2 len / T) is no less.
inline __host__ __device__ int64_t slot_count(int64_t rows, int shift) { return ((2 * rows) >> shift) + 1; }
inline __host__ __device__ int64_t slot_of(int64_t start, int64_t segment, int shift) {
    return ((2 * start) >> shift) + segment;
}

// The number of this thread's wave, in a scalar register: what follows from
// it (a wave's range of rows, what it skips) is then scalar work.
__device__ inline int wave_number() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

struct View {
    char* data;
    int64_t batch, row, head;   // strides in elements
};

}  // namespace nsl
