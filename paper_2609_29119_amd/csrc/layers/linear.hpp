// A matrix of its own for each band, over ragged rows.
//
//   y[r] = W[g] x[r] + bias[g]     dx[r] = W[g]^T dy[r]     dW[g] = sum_r dy[r] x[r]^T
//
// A band's rows are those of all signals: row r of its batch * len rows is
// token r % len of signal r / len.
#pragma once
#include "tile.hpp"

namespace nsl {

struct LinearArgs {
    View x, y;            // the product's input and output (for dW: x and dy)
    const void* w;        // [n_bands][n_out][n_in]
    const void* bias;     // [n_bands][n_out] or NULL
    void* dw;
    void* db;
    float* part;          // partial dW (and db) of bands of several chunks
    const int64_t* off;
    int rows, n_bands, batch;
    int n_in, n_out;      // of the layer, whichever direction is computed
    int first_band;       // of a launch of k_linear_join
    int chunk_shift;      // rows of a workgroup of the weights' gradient, or of k_linear_kept
    bool x_wide, y_wide, w_wide;
};

constexpr int kRowShift = 7;   // rows of a workgroup of k_linear: 4 waves of 32
template <class T> constexpr int step_width() { return 128 / static_cast<int>(sizeof(T)); }   // reduction of one LDS tile

template <class T> __device__ inline T* band_row(const View& v, const Tile<int64_t>& t, int64_t r) {
    const int64_t b = r / t.len, c = r - b * t.len;
    return reinterpret_cast<T*>(v.data) + b * v.batch + (t.start + c) * v.row;
}

// y (BACK: dx). The product is formed transposed, y^T = W x^T: a lane's column
// is a row of x, whose 8 consecutive values are its B fragment straight from
// memory, and the result's registers run along y. Only W goes through LDS,
// where the four waves share it; BACK reads it turned. Bound by memory and by
// what each workgroup waits for in turn (the search, its rows, W):
// 446,932 rows, 128 -> 128, bfloat16, 221 bands: y 58 us (4.1 TB/s), dx 61 us,
// of 48 at the rate of a large copy.
template <class T, int NB, bool BACK>
__global__ __launch_bounds__(256, 2) void k_linear(LinearArgs a) {
    constexpr int BK = step_width<T>(), BN = 32 * NB, KS = BK / 16;
    constexpr int WR = BACK ? BK : BN, WC = BACK ? BN : BK;           // rows and columns of the tile of W
    constexpr int RB = row_bytes<T, WC>(), kChunks = WR * WC / 8, kEach = (kChunks + 255) / 256;
    __shared__ __align__(128) char lds[2][WR * RB];
    __shared__ __align__(16) float start[BN];   // where the sums start: the bias
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), m = lane & 31, h = lane >> 5;
    const int n_red = BACK ? a.n_out : a.n_in, n_col = BACK ? a.n_in : a.n_out, cols = (n_col + BN - 1) / BN;

    const unsigned id = die_order(blockIdx.x, gridDim.x), p = id / cols;
    const int c0 = (id - p * cols) * BN;
    const Tile<int64_t> t = find_tile<int64_t>(a.off, a.n_bands, a.rows, a.batch, kRowShift, p, lane);
    if (!t.live) return;
    const int64_t n_rows = static_cast<int64_t>(t.len) * a.batch, r = t.first + 32 * wave + m;
    const bool mine = r < n_rows;
    T* out = mine ? band_row<T>(a.y, t, r) : nullptr;
    if (t.band < 0 || t.band >= a.n_bands) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) store_column<T>(out, zero16(), c0 + 32 * nb, n_col, a.y_wide, lane);
        return;
    }
    const T* in = mine ? band_row<T>(a.x, t, r) : nullptr;
    const T* w = static_cast<const T*>(a.w) + static_cast<int64_t>(t.band) * a.n_out * a.n_in;

    frag<T> wr[kEach], xf[KS], xn[KS];
    auto fetch_w = [&](int k0) {
        by_width(a.w_wide, [&](auto wide) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const int c = tid + 256 * e, row = c / (WC / 8) + (BACK ? k0 : c0);
                const int col = c % (WC / 8) * 8 + (BACK ? c0 : k0);
                const bool there = (kChunks % 256 == 0 || c < kChunks) && row < a.n_out;
                wr[e] = load8<T, wide.value>(w + static_cast<int64_t>(row) * a.n_in + col, there ? a.n_in - col : 0,
                                             col > 0);
            }
        });
    };
    auto put_w = [&](int n) {
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int c = tid + 256 * e;
            if (kChunks % 256 == 0 || c < kChunks) write8<T, RB>(lds[n & 1], c / (WC / 8), c % (WC / 8), wr[e]);
        }
    };
    auto fetch_x = [&](frag<T>(&f)[KS], int k0) {
        by_width(a.x_wide, [&](auto wide) {
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int k = k0 + 16 * s + 8 * h;
                f[s] = load8<T, wide.value>(in + k, mine ? n_red - k : 0, k > 0);
            }
        });
    };
    const int steps = (n_red + BK - 1) / BK;
    fetch_w(0);
    fetch_x(xf, 0);
    if (a.bias && tid < BN)
        start[tid] = c0 + tid < n_col ? static_cast<float>(static_cast<const T*>(
                                            a.bias)[static_cast<int64_t>(t.band) * a.n_out + c0 + tid])
                                      : 0.f;
    put_w(0);
    __syncthreads();
    acc16 acc[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        acc[nb] = zero16();
        if (a.bias) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f4 v = *reinterpret_cast<const f4*>(start + 32 * nb + 8 * q + 4 * h);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[nb][4 * q + j] = v[j];
            }
        }
    }
#pragma unroll 1
    for (int n = 0; n < steps; ++n) {
        if (n + 1 < steps) {
            fetch_w((n + 1) * BK);
            fetch_x(xn, (n + 1) * BK);
        }
        const char* tile = lds[n & 1];
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            if (n * BK + 16 * s < n_red) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    if constexpr (BACK)
                        acc[nb] = mma(read_turned8<T, RB>(tile, 16 * s, 32 * nb, lane), xf[s], acc[nb]);
                    else
                        acc[nb] = mma(read8<T, RB>(tile, 32 * nb + m, 2 * s + h), xf[s], acc[nb]);
                }
            }
        }
        if (n + 1 < steps) {
            put_w(n + 1);
#pragma unroll
            for (int s = 0; s < KS; ++s) xf[s] = xn[s];
        }
        __syncthreads();
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) store_column<T>(out, acc[nb], c0 + 32 * nb, n_col, a.y_wide, lane);
}

// The same product for rows of odd widths or strides, where a band's whole W
// (or 32 NB of its output columns) fits LDS beside 4 KB for each wave: W is
// loaded once, and each wave walks through its share of the workgroup's
// 2^chunk_shift rows on its own, without a barrier. Its rows go through LDS in
// slabs of 128 bytes a row, two on their way while one is computed, and so
// does its result: memory is read and written in runs of 128 bytes a row.
// Straight to fragments, 32 unaligned bytes of each of 32 rows a load, the
// addresses are the limit (193 -> 77 columns, 710,680 rows, float16: 205 us,
// here 149); aligned rows are faster that way, which keeps more waves
// resident (128 -> 128, 446,932 rows, bfloat16: 60 us, here 70).
constexpr int kKeptLds = 65536, kKeptRest = 4 * 4096 + 512;   // rows of the waves, bias
template <class T, bool BACK> __host__ __device__ inline int kept_row_bytes(int n_red, int nb) {
    return ((BACK ? 32 * nb : n_red) * static_cast<int>(sizeof(T)) + 127) / 128 * 128;
}
// Rows of W's tile in LDS: the reduction's in whole steps (BACK), or the columns that exist.
template <bool BACK> __host__ __device__ inline int kept_rows(int n_red, int n_col, int nb) {
    return BACK ? (n_red + 15) / 16 * 16 : n_col < 32 * nb ? n_col : 32 * nb;
}

template <class T, int NB, bool BACK>
__global__ __launch_bounds__(256, 2) void k_linear_kept(LinearArgs a) {
    constexpr int BK = step_width<T>(), BN = 32 * NB, KS = BK / 16, kRowEach = 32 * BK / 8 / 64;
    extern __shared__ __align__(128) char kept_lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), m = lane & 31, h = lane >> 5;
    const int n_red = BACK ? a.n_out : a.n_in, n_col = BACK ? a.n_in : a.n_out, cols = (n_col + BN - 1) / BN;
    char* slab = kept_lds + 4096 * wave;
    float* start = reinterpret_cast<float*>(kept_lds + 4 * 4096);
    char* wt = kept_lds + kKeptRest;

    const unsigned id = die_order(blockIdx.x, gridDim.x), p = id / cols;
    const int c0 = (id - p * cols) * BN;
    const Tile<int64_t> t = find_tile<int64_t>(a.off, a.n_bands, a.rows, a.batch, a.chunk_shift, p, lane);
    if (!t.live) return;
    const int64_t n_rows = static_cast<int64_t>(t.len) * a.batch;
    const int64_t r_end = min(t.first + (int64_t(1) << a.chunk_shift), n_rows);
    const bool outside = t.band < 0 || t.band >= a.n_bands;   // tokens that no band holds: zeros

    const int RB = kept_row_bytes<T, BACK>(n_red, NB);
    // x comes in slabs of 128 bytes of 32 rows; two are on their way while one is computed
    frag<T> xr[2][kRowEach];
    const T* row_in[kRowEach];   // of the fetched rows, this lane's part: chunk lane % (BK / 8) of these
    const int steps = (n_red + BK - 1) / BK;
    int64_t next_r0 = t.first + 32 * wave;   // what is fetched next: rows, and slab of them
    int next_slab = 0;
    auto fetch = [&](frag<T>(&f)[kRowEach]) __attribute__((always_inline)) {
        if (next_r0 >= r_end || outside) return;
        if (next_slab == 0) {
            const T* in = next_r0 + m < r_end ? band_row<T>(a.x, t, next_r0 + m) : nullptr;
#pragma unroll
            for (int e = 0; e < kRowEach; ++e) row_in[e] = from_lane(in, (lane + 64 * e) / (BK / 8));
        }
        by_width(a.x_wide, [&](auto wide) {
            const int k = next_slab * BK + lane % (BK / 8) * 8;
#pragma unroll
            for (int e = 0; e < kRowEach; ++e)
                f[e] = load8<T, wide.value>(row_in[e] + k, row_in[e] ? n_red - k : 0, k > 0);
        });
        if (++next_slab == steps) {
            next_slab = 0;
            next_r0 += 128;
        }
    };
    fetch(xr[0]);
    fetch(xr[1]);

    const int w_rows = kept_rows<BACK>(n_red, n_col, NB);
    if (!outside) {
        const T* w = static_cast<const T*>(a.w) + static_cast<int64_t>(t.band) * a.n_out * a.n_in;
        const int w_cols = BACK ? BN : (n_red + 15) / 16 * 16;
        const int chunks = w_cols / 8, total = w_rows * chunks;
        by_width(a.w_wide, [&](auto wide) {
#pragma unroll 4
            for (int c = tid; c < total; c += 256) {
                const int wr = c / chunks, wc = (c - wr * chunks) * 8;
                const int row = wr + (BACK ? 0 : c0), col = wc + (BACK ? c0 : 0);
                write8<T>(wt, RB, wr, wc / 8,
                          load8<T, wide.value>(w + static_cast<int64_t>(row) * a.n_in + col,
                                               row < a.n_out ? a.n_in - col : 0, col > 0));
            }
        });
        if (tid < BN)
            start[tid] = a.bias && c0 + tid < n_col
                             ? static_cast<float>(static_cast<const T*>(
                                   a.bias)[static_cast<int64_t>(t.band) * a.n_out + c0 + tid])
                             : 0.f;
    }
    __syncthreads();

    int64_t r0 = t.first + 32 * wave;
    int step = 0;
    acc16 acc[NB];
    while (r0 < r_end) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {   // one slab; its registers are then free for the one after the next
            if (r0 >= r_end) continue;
            if (step == 0) {
                each<NB>([&](auto nb) __attribute__((always_inline)) {
                    acc16 v = zero16();
                    if (a.bias && !outside) {
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const f4 u = *reinterpret_cast<const f4*>(start + 32 * nb.value + 8 * q + 4 * h);
#pragma unroll
                            for (int j = 0; j < 4; ++j) v[4 * q + j] = u[j];
                        }
                    }
                    acc[nb.value] = v;
                });
            }
            if (!outside) {
#pragma unroll
                for (int e = 0; e < kRowEach; ++e)
                    write8<T, 128>(slab, (lane + 64 * e) / (BK / 8), lane % (BK / 8), xr[u][e]);
                fetch(xr[u]);
                each<KS>([&](auto s) __attribute__((always_inline)) {
                    if (step * BK + 16 * s.value < n_red) {
                        const frag<T> xf = read8<T, 128>(slab, m, 2 * s.value + h);
                        each<NB>([&](auto nb) __attribute__((always_inline)) {
                            if constexpr (BACK)
                                acc[nb.value] = mma(read_turned8<T, row_bytes<T, BN>()>(wt, step * BK + 16 * s.value,
                                                                                        32 * nb.value, lane),
                                                    xf, acc[nb.value]);
                            else
                                acc[nb.value] = mma(read8<T>(wt, RB, min(32 * nb.value + m, w_rows - 1),
                                                             step * (BK / 8) + 2 * s.value + h),
                                                    xf, acc[nb.value]);
                        });
                    }
                });
            }
            if (++step >= steps || outside) {
                T* out = r0 + m < r_end ? band_row<T>(a.y, t, r0 + m) : nullptr;
                T* row_out[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) row_out[e] = from_lane(out, lane / 8 + 8 * e);
                store_rows<T, NB>(slab, acc, row_out, static_cast<int>(min(r_end - r0, int64_t(32))), c0, n_col,
                                  a.y_wide, lane);
                r0 += 128;
                step = 0;
            }
        }
    }
}

// dW over chunks of 2^chunk_shift rows: 128 outputs x 128 inputs a workgroup, its
// waves 64 x 64 each. Both operands run along the rows, so both are read
// turned from LDS. A band of one chunk is written at once, one of several as
// 32-bit partial sums that k_linear_join adds in order: no atomics, so the sums
// do not vary. 446,932 rows, 128 x 128, bfloat16: 65 us and 17 us for the join
// (chunks of 512 rows: 71 and 23; of 2048: 98 and 13), of 48 at the rate of a
// large copy; bound by waiting for loads, three waves a SIMD.
__device__ inline float* dw_part(const LinearArgs& a, int64_t item) {
    return a.part + item * (static_cast<int64_t>(a.n_out) * a.n_in + a.n_out);
}

template <class T>
__global__ __launch_bounds__(256, 2) void k_linear_dw(LinearArgs a) {
    constexpr int BR = 64, RB = row_bytes<T, 128>();
    constexpr int kEach = BR * 16 / 256;
    __shared__ __align__(128) char lds[2][BR * RB];
    __shared__ float sums[16][128 + 4];
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), m = lane & 31, h = lane >> 5;
    const int ot = (a.n_out + 127) / 128, it = max(1, (a.n_in + 127) / 128);
    const unsigned id = die_order(blockIdx.x, gridDim.x), p = id / (ot * it), at2 = id - p * (ot * it);
    const int o0 = at2 / it * 128, i0 = at2 % it * 128;
    const Tile<int64_t> t = find_tile<int64_t>(a.off, a.n_bands, a.rows, a.batch, a.chunk_shift, p, lane);
    if (!t.live || t.band < 0 || t.band >= a.n_bands) return;
    const int64_t n_rows = static_cast<int64_t>(t.len) * a.batch;
    const int64_t r_end = min(t.first + (int64_t(1) << a.chunk_shift), n_rows);
    const int wo = wave >> 1 << 6, wi = (wave & 1) << 6;

    frag<T> xr[kEach], yr[kEach];
    float colsum[8] = {};
    const bool sum_bias = a.db && i0 == 0;
    auto fetch = [&](int64_t r0) {
        const T *px[kEach], *py[kEach];
        bool there[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int64_t r = r0 + (tid + 256 * e) / 16;
            there[e] = r < r_end;
            px[e] = there[e] ? band_row<T>(a.x, t, r) : nullptr;
            py[e] = there[e] ? band_row<T>(a.y, t, r) : nullptr;
        }
        const int x0 = i0 + tid % 16 * 8, y0 = o0 + tid % 16 * 8;
        by_width(a.x_wide, [&](auto wide) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) xr[e] = load8<T, wide.value>(px[e] + x0, there[e] ? a.n_in - x0 : 0, x0 > 0);
        });
        by_width(a.y_wide, [&](auto wide) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) yr[e] = load8<T, wide.value>(py[e] + y0, there[e] ? a.n_out - y0 : 0, y0 > 0);
        });
    };
    acc16 acc[2][2];
#pragma unroll
    for (int x = 0; x < 4; ++x) acc[x >> 1][x & 1] = zero16();
    fetch(t.first);
    for (int64_t r0 = t.first; r0 < r_end; r0 += BR) {
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int c = tid + 256 * e;
            write8<T, RB>(lds[0], c / 16, c % 16, xr[e]);
            write8<T, RB>(lds[1], c / 16, c % 16, yr[e]);
            if (sum_bias) {
#pragma unroll
                for (int j = 0; j < 8; ++j) colsum[j] += static_cast<float>(yr[e][j]);
            }
        }
        __syncthreads();
        if (r0 + BR < r_end) fetch(r0 + BR);
        if (o0 + wo < a.n_out && i0 + wi < a.n_in) {
#pragma unroll
            for (int s = 0; s < BR / 16; ++s) {
                frag<T> fo[2], fi[2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    fo[x] = read_turned<T, RB>(lds[1], 16 * s, wo + 32 * x, lane);
                    fi[x] = read_turned<T, RB>(lds[0], 16 * s, wi + 32 * x, lane);
                }
#pragma unroll
                for (int x = 0; x < 4; ++x) acc[x >> 1][x & 1] = mma(fo[x >> 1], fi[x & 1], acc[x >> 1][x & 1]);
            }
        }
        __syncthreads();
    }
    const bool whole = n_rows <= (int64_t(1) << a.chunk_shift);
    float* part = dw_part(a, p);
    T* dw = static_cast<T*>(a.dw) + static_cast<int64_t>(t.band) * a.n_out * a.n_in;
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const int o = o0 + wo + 32 * (x >> 1) + 8 * (q >> 2) + 4 * h + (q & 3), i = i0 + wi + 32 * (x & 1) + m;
            if (o < a.n_out && i < a.n_in) {
                const int64_t at = static_cast<int64_t>(o) * a.n_in + i;
                if (whole)
                    dw[at] = static_cast<T>(acc[x >> 1][x & 1][q]);
                else
                    part[at] = acc[x >> 1][x & 1][q];
            }
        }
    if (sum_bias) {   // 16 threads hold sums of the same 8 columns
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[tid / 16][tid % 16 * 8 + j] = colsum[j];
        __syncthreads();
        if (tid < 128 && o0 + tid < a.n_out) {
            float s = 0.f;
            for (int k = 0; k < 16; ++k) s += sums[k][tid];
            if (whole)
                static_cast<T*>(a.db)[static_cast<int64_t>(t.band) * a.n_out + o0 + tid] = static_cast<T>(s);
            else
                part[static_cast<int64_t>(a.n_out) * a.n_in + o0 + tid] = s;
        }
    }
}

// Adds the partial sums of bands of several chunks, and writes zeros for empty bands: bands first_band on.
template <class T>
__global__ __launch_bounds__(256) void k_linear_join(LinearArgs a) {
    const int band = a.first_band + static_cast<int>(blockIdx.y);
    const int64_t b0 = band_bound(a.off, a.n_bands, a.rows, band + 1), b1 = band_bound(a.off, a.n_bands, a.rows, band + 2);
    const int64_t n_rows = b1 > b0 ? (b1 - b0) * a.batch : 0;
    if (n_rows > 0 && n_rows <= (int64_t(1) << a.chunk_shift)) return;
    const int64_t n_w = static_cast<int64_t>(a.n_out) * a.n_in, n = n_w + (a.db ? a.n_out : 0);
    const int64_t chunks = (n_rows + (int64_t(1) << a.chunk_shift) - 1) >> a.chunk_shift;
    const int64_t item = ((b0 * a.batch) >> a.chunk_shift) + band + 1;
    for (int64_t e = blockIdx.x * 256 + threadIdx.x; e < n; e += 256 * gridDim.x) {
        float s = 0.f;
#pragma unroll 8
        for (int64_t c = 0; c < chunks; ++c) s += dw_part(a, item + c)[e];
        if (e < n_w)
            static_cast<T*>(a.dw)[band * n_w + e] = static_cast<T>(s);
        else
            static_cast<T*>(a.db)[static_cast<int64_t>(band) * a.n_out + e - n_w] = static_cast<T>(s);
    }
}

}  // namespace nsl
