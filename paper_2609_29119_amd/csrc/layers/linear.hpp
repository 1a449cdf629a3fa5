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
    bool x_wide, y_wide, w_wide;
};

constexpr int kRowShift = 7;   // rows of a workgroup: 4 waves of 32
template <class T> constexpr int step_width() { return 128 / static_cast<int>(sizeof(T)); }   // reduction of one LDS tile

template <class T> __device__ inline T* band_row(const View& v, const Tile<int64_t>& t, int64_t r) {
    const int64_t b = r / t.len, c = r - b * t.len;
    return reinterpret_cast<T*>(v.data) + b * v.batch + (t.start + c) * v.row;
}

// y (BACK: dx). The product is formed transposed, y^T = W x^T: a lane's column
// is a row of x, whose 8 consecutive values are its B fragment straight from
// memory, and the result's registers run along y. Only W goes through LDS,
// where the four waves share it; BACK reads it turned.
template <class T, int NB, bool BACK>
__global__ __launch_bounds__(256, 2) void k_linear(LinearArgs a) {
    constexpr int BK = step_width<T>(), BN = 32 * NB, KS = BK / 16;
    constexpr int WR = BACK ? BK : BN, WC = BACK ? BN : BK;           // rows and columns of the tile of W
    constexpr int RB = row_bytes<T, WC>(), kChunks = WR * WC / 8, kEach = (kChunks + 255) / 256;
    __shared__ __align__(128) char lds[2][WR * RB];
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
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int c = tid + 256 * e, row = c / (WC / 8) + (BACK ? k0 : c0), col = c % (WC / 8) * 8 + (BACK ? c0 : k0);
            const bool there = (kChunks % 256 == 0 || c < kChunks) && row < a.n_out;
            wr[e] = load8<T>(w + static_cast<int64_t>(row) * a.n_in + col, there ? a.n_in - col : 0, a.w_wide);
        }
    };
    auto put_w = [&](int n) {
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int c = tid + 256 * e;
            if (kChunks % 256 == 0 || c < kChunks) write8<T, RB>(lds[n & 1], c / (WC / 8), c % (WC / 8), wr[e]);
        }
    };
    auto fetch_x = [&](frag<T>(&f)[KS], int k0) {
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int k = k0 + 16 * s + 8 * h;
            f[s] = load8<T>(in + k, mine ? n_red - k : 0, a.x_wide);
        }
    };
    acc16 acc[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) acc[nb] = zero16();
    const int steps = (n_red + BK - 1) / BK;
    fetch_w(0);
    fetch_x(xf, 0);
    put_w(0);
    __syncthreads();
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
                    // turned reads take the steps of a fragment in another order than rows of x have them
                    if constexpr (BACK) {
                        acc[nb] = mma(read_turned8<T, RB>(tile, 16 * s, 32 * nb, lane), xf[s], acc[nb]);
                    } else {
                        acc[nb] = mma(read8<T, RB>(tile, 32 * nb + m, 2 * s + h), xf[s], acc[nb]);
                    }
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
    if (a.bias) {
        const T* bias = static_cast<const T*>(a.bias) + static_cast<int64_t>(t.band) * a.n_out;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const int d = c0 + 32 * nb + 8 * (q >> 2) + 4 * h + (q & 3);
                if (d < n_col) acc[nb][q] += static_cast<float>(bias[d]);
            }
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) store_column<T>(out, acc[nb], c0 + 32 * nb, n_col, a.y_wide, lane);
}

// dW over chunks of 2^SHIFT rows: 128 outputs x 128 inputs a workgroup, its
// waves 64 x 64 each. Both operands run along the rows, so both are read
// turned from LDS. A band of one chunk is written at once, one of several as
// 32-bit partial sums that k_linear_join adds in order.
constexpr int kChunkShift = 11;
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
    const Tile<int64_t> t = find_tile<int64_t>(a.off, a.n_bands, a.rows, a.batch, kChunkShift, p, lane);
    if (!t.live || t.band < 0 || t.band >= a.n_bands) return;
    const int64_t n_rows = static_cast<int64_t>(t.len) * a.batch;
    const int64_t r_end = min(t.first + (int64_t(1) << kChunkShift), n_rows);
    const int wo = wave >> 1 << 6, wi = (wave & 1) << 6;

    frag<T> xr[kEach], yr[kEach];
    float colsum[8] = {};
    const bool sum_bias = a.db && i0 == 0;
    auto fetch = [&](int64_t r0) {
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int c = tid + 256 * e, col = c % 16 * 8;
            const int64_t r = r0 + c / 16;
            const bool there = r < r_end;
            const T* px = there ? band_row<T>(a.x, t, r) : nullptr;
            const T* py = there ? band_row<T>(a.y, t, r) : nullptr;
            xr[e] = load8<T>(px + i0 + col, there ? a.n_in - i0 - col : 0, a.x_wide);
            yr[e] = load8<T>(py + o0 + col, there ? a.n_out - o0 - col : 0, a.y_wide);
        }
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
    const bool whole = n_rows <= (int64_t(1) << kChunkShift);
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

// Adds the partial sums of bands of several chunks, and writes zeros for empty bands.
template <class T>
__global__ __launch_bounds__(256) void k_linear_join(LinearArgs a) {
    const int band = blockIdx.y;
    const int64_t b0 = band_bound(a.off, a.n_bands, a.rows, band + 1), b1 = band_bound(a.off, a.n_bands, a.rows, band + 2);
    const int64_t n_rows = b1 > b0 ? (b1 - b0) * a.batch : 0;
    if (n_rows > 0 && n_rows <= (int64_t(1) << kChunkShift)) return;
    const int64_t n_w = static_cast<int64_t>(a.n_out) * a.n_in, n = n_w + (a.db ? a.n_out : 0);
    const int64_t chunks = (n_rows + (int64_t(1) << kChunkShift) - 1) >> kChunkShift;
    const int64_t item = ((b0 * a.batch) >> kChunkShift) + band + 1;
    for (int64_t e = blockIdx.x * 256 + threadIdx.x; e < n; e += 256 * gridDim.x) {
        float s = 0.f;
        for (int64_t c = 0; c < chunks; ++c) s += dw_part(a, item + c)[e];
        if (e < n_w)
            static_cast<T*>(a.dw)[band * n_w + e] = static_cast<T>(s);
        else
            static_cast<T*>(a.db)[static_cast<int64_t>(band) * a.n_out + e - n_w] = static_cast<T>(s);
    }
}

}  // namespace nsl
