// A gated product of each band: two projections, an activation, their product.
//
//   a = Wa x + ba   u = Wu x + bu   y = act(a) u
//   da = dy u act'(a)   du = dy act(a)   dx = Wa^T da + Wu^T du   dW. = sum d. x^T   db. = sum d.
//
// W of a band: [2][n_out][n_in], Wa before Wu. a and u stay in registers: the
// forward call writes y alone, and each gradient forms them again, which
// costs less than writing and reading them, let alone da and du, each of
// which would have to go to memory as two numbers of 16 bits.
#pragma once
#include "act.hpp"
#include "linear.hpp"
#include "pieces.hpp"

namespace nsl {

struct GatedArgs {
    View x, y, dy;          // (dx is y)
    const void* w;          // [n_bands][2][n_out][n_in]
    const void* bias;       // [n_bands][2][n_out] or NULL
    LinearArgs dw;          // weights' gradient: as of a band_linear of 2 n_out outputs
    const int64_t* off;
    int rows, n_bands, batch;
    int n_in, n_out, act;
    bool x_wide, y_wide, w_wide;
};

template <class T> __device__ inline float gated_bias(const GatedArgs& a, const Tile<int64_t>& t, int which, int o) {
    return a.bias && o < a.n_out
               ? static_cast<float>(static_cast<const T*>(a.bias)[(static_cast<int64_t>(t.band) * 2 + which) * a.n_out + o])
               : 0.f;
}

// y, as k_linear forms its product (transposed, x straight to fragments), with
// 32 NB rows of Wa and as many of Wu in LDS side by side.
template <class T, int NB>
__global__ __launch_bounds__(256, 2) void k_gated(GatedArgs a) {
    constexpr int BK = step_width<T>(), BN = 32 * NB, KS = BK / 16, RB = row_bytes<T, BK>();
    constexpr int kChunks = 2 * BN * BK / 8, kEach = kChunks / 256;
    __shared__ __align__(128) char lds[2][2 * BN * RB];
    __shared__ __align__(16) float start[2 * BN];
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), m = lane & 31, h = lane >> 5;
    const int cols = (a.n_out + BN - 1) / BN;
    const unsigned id = die_order(blockIdx.x, gridDim.x), p = id / cols;
    const int c0 = (id - p * cols) * BN;
    const Tile<int64_t> t = find_tile<int64_t>(a.off, a.n_bands, a.rows, a.batch, kRowShift, p, lane);
    if (!t.live) return;
    const int64_t n_rows = static_cast<int64_t>(t.len) * a.batch, r = t.first + 32 * wave + m;
    const bool mine = r < n_rows;
    T* out = mine ? band_row<T>(a.y, t, r) : nullptr;
    if (t.band < 0 || t.band >= a.n_bands) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) store_column<T>(out, zero16(), c0 + 32 * nb, a.n_out, a.y_wide, lane);
        return;
    }
    const T* in = mine ? band_row<T>(a.x, t, r) : nullptr;
    const T* w = static_cast<const T*>(a.w) + static_cast<int64_t>(t.band) * 2 * a.n_out * a.n_in;
    frag<T> wr[kEach], xf[KS], xn[KS];
    auto fetch_w = [&](int k0) {
        by_width(a.w_wide, [&](auto wide) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const int c = tid + 256 * e, i = c / (BK / 8), o = c0 + i % BN, col = c % (BK / 8) * 8 + k0;
                const int64_t row = static_cast<int64_t>(i / BN) * a.n_out + o;
                wr[e] = load8<T, wide.value>(w + row * a.n_in + col, o < a.n_out ? a.n_in - col : 0, col > 0);
            }
        });
    };
    auto put_w = [&](int n) {
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int c = tid + 256 * e;
            write8<T, RB>(lds[n & 1], c / (BK / 8), c % (BK / 8), wr[e]);
        }
    };
    auto fetch_x = [&](frag<T>(&f)[KS], int k0) {
        by_width(a.x_wide, [&](auto wide) {
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int k = k0 + 16 * s + 8 * h;
                f[s] = load8<T, wide.value>(in + k, mine ? a.n_in - k : 0, k > 0);
            }
        });
    };
    const int steps = (a.n_in + BK - 1) / BK;
    fetch_w(0);
    fetch_x(xf, 0);
    if (tid < 2 * BN) start[tid] = gated_bias<T>(a, t, tid / BN, c0 + tid % BN);
    put_w(0);
    __syncthreads();
    acc16 acc[2 * NB];
#pragma unroll
    for (int nb = 0; nb < 2 * NB; ++nb)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f4 v = *reinterpret_cast<const f4*>(start + 32 * nb + 8 * q + 4 * h);
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[nb][4 * q + j] = v[j];
        }
#pragma unroll 1
    for (int n = 0; n < steps; ++n) {
        if (n + 1 < steps) {
            fetch_w((n + 1) * BK);
            fetch_x(xn, (n + 1) * BK);
        }
#pragma unroll
        for (int s = 0; s < KS; ++s)
            if (n * BK + 16 * s < a.n_in) {
#pragma unroll
                for (int nb = 0; nb < 2 * NB; ++nb)
                    acc[nb] = mma(read8<T, RB>(lds[n & 1], 32 * nb + m, 2 * s + h), xf[s], acc[nb]);
            }
        if (n + 1 < steps) {
            put_w(n + 1);
#pragma unroll
            for (int s = 0; s < KS; ++s) xf[s] = xn[s];
        }
        __syncthreads();
    }
    by_act(a.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[nb][q] = act_of<act.value>(acc[nb][q]) * acc[NB + nb][q];
    });
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) store_column<T>(out, acc[nb], c0 + 32 * nb, a.n_out, a.y_wide, lane);
}

// Inputs that a workgroup of the gradients takes at once.
template <class T> constexpr int gated_inputs() { return sizeof(T) == 4 ? 64 : 128; }

// 4 values at p, of which the first n are there.
template <class T> __device__ inline quad<T> load4(const T* p, int n, bool wide) {
    quad<T> f;
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = static_cast<T>(0.f);
    if (n >= 4) {
        if (wide)
            f = *reinterpret_cast<const quad<T>*>(p);
        else
            __builtin_memcpy(&f, p, sizeof(f));
    } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (j < n) f[j] = p[j];
    }
    return f;
}

// From a, u and dy: da and du, in their places.
template <int ACT> __device__ inline void gated_slope(acc16& a, acc16& u, const float (&dy)[16]) {
#pragma unroll
    for (int q = 0; q < 16; ++q) {
        float slope;
        const float f = act_of<ACT>(a[q], slope);
        a[q] = dy[q] * u[q] * slope;
        u[q] = dy[q] * f;
    }
}

// dx of 128 rows (32 a wave), 128 inputs (64 in 32 bits): along the outputs in blocks of 32,
// whose a and u are formed transposed (a lane's column is a row of x), turned
// into da and du in their registers, and go on from there, as two numbers of
// 16 bits each, into the product with W. Both products read the same tile of W,
// the second one turned. HELD: one tile holds
// a block's rows of W, and the row of x stays in registers.
template <class T, bool HELD>
__global__ __launch_bounds__(256, 2) void k_gated_dx(GatedArgs a) {
    constexpr int BK = gated_inputs<T>(), NB = BK / 32, KS = BK / 16, RB = row_bytes<T, BK>(), kEach = 2 * 32 * BK / 8 / 256;
    __shared__ __align__(128) char lds[2][2][32 * RB];
    __shared__ __align__(16) float start[2][2][32];
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), m = lane & 31, h = lane >> 5;
    const int slabs = (a.n_in + BK - 1) / BK;
    const unsigned id = die_order(blockIdx.x, gridDim.x), p = id / slabs;
    const int my_slab = static_cast<int>(id - p * slabs), c0 = my_slab * BK;
    const Tile<int64_t> t = find_tile<int64_t>(a.off, a.n_bands, a.rows, a.batch, kRowShift, p, lane);
    if (!t.live) return;
    const int64_t n_rows = static_cast<int64_t>(t.len) * a.batch, r = t.first + 32 * wave + m;
    const bool mine = r < n_rows;
    T* out = mine ? band_row<T>(a.y, t, r) : nullptr;
    acc16 dx[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) dx[nb] = zero16();
    if (t.band < 0 || t.band >= a.n_bands || a.n_out == 0) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) store_column<T>(out, dx[nb], c0 + 32 * nb, a.n_in, a.x_wide, lane);
        return;
    }
    const T* in = mine ? band_row<T>(a.x, t, r) : nullptr;
    const T* dy = mine ? band_row<T>(a.dy, t, r) : nullptr;
    const T* w = static_cast<const T*>(a.w) + static_cast<int64_t>(t.band) * 2 * a.n_out * a.n_in;
    const int blocks = (a.n_out + 31) / 32, stages = blocks * slabs;
    // a block's slabs in an order that ends with this workgroup's own
    auto slab_of = [&](int i) { return (my_slab + 1 + i) % slabs; };
    frag<T> wr[kEach], xf[KS];
    auto fetch_w = [&](int stage) {
        const int o0 = stage / slabs * 32, k0 = slab_of(stage % slabs) * BK;
        by_width(a.w_wide, [&](auto wide) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const int c = tid + 256 * e, i = c / (BK / 8), o = o0 + i % 32, col = c % (BK / 8) * 8 + k0;
                const int64_t row = static_cast<int64_t>(i / 32) * a.n_out + o;
                wr[e] = load8<T, wide.value>(w + row * a.n_in + col, o < a.n_out ? a.n_in - col : 0, col > 0);
            }
        });
    };
    auto put_w = [&](int stage) {
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int c = tid + 256 * e, i = c / (BK / 8);
            write8<T, RB>(lds[stage & 1][i / 32], i % 32, c % (BK / 8), wr[e]);
        }
        if (tid < 64) start[stage & 1][tid / 32][tid % 32] = gated_bias<T>(a, t, tid / 32, stage / slabs * 32 + tid % 32);
    };
    auto fetch_x = [&](int slab) {
        by_width(a.x_wide, [&](auto wide) {
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int k = slab * BK + 16 * s + 8 * h;
                xf[s] = load8<T, wide.value>(in + k, mine ? a.n_in - k : 0, k > 0);
            }
        });
    };
    fetch_w(0);
    if (HELD) fetch_x(0);
    put_w(0);
    __syncthreads();
    acc16 za, zu;
#pragma unroll 1
    for (int stage = 0; stage < stages; ++stage) {
        const int at = HELD ? 0 : stage % slabs, o0 = (HELD ? stage : stage / slabs) * 32;
        const char *ta = lds[stage & 1][0], *tu = lds[stage & 1][1];
        if (!HELD) fetch_x(slab_of(at));
        if (stage + 1 < stages) fetch_w(stage + 1);
        const bool whole = at + 1 == slabs;
        quad<T> dyq[4];
        if (whole) {
#pragma unroll
            for (int q = 0; q < 4; ++q) dyq[q] = load4<T>(dy + o0 + 8 * q + 4 * h, mine ? a.n_out - (o0 + 8 * q + 4 * h) : 0, a.y_wide);
        }
        if (at == 0) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f4 va = *reinterpret_cast<const f4*>(&start[stage & 1][0][8 * q + 4 * h]);
                const f4 vu = *reinterpret_cast<const f4*>(&start[stage & 1][1][8 * q + 4 * h]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    za[4 * q + j] = va[j];
                    zu[4 * q + j] = vu[j];
                }
            }
        }
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            za = mma(read8<T, RB>(ta, m, 2 * s + h), xf[s], za);
            zu = mma(read8<T, RB>(tu, m, 2 * s + h), xf[s], zu);
        }
        if (whole) {
            float d[16];
#pragma unroll
            for (int q = 0; q < 16; ++q) d[q] = static_cast<float>(dyq[q >> 2][q & 3]);
            by_act(a.act, [&](auto act) __attribute__((always_inline)) { gated_slope<act.value>(za, zu, d); });
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const auto da = sum_of<T, 2>(octet(za, x)), du = sum_of<T, 2>(octet(zu, x));
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    dx[nb] = product(data_of(read_turned<T, RB>(ta, 16 * x, 32 * nb, lane)), da, dx[nb]);
                    dx[nb] = product(data_of(read_turned<T, RB>(tu, 16 * x, 32 * nb, lane)), du, dx[nb]);
                }
            }
        }
        if (stage + 1 < stages) put_w(stage + 1);
        __syncthreads();
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) store_column<T>(out, dx[nb], c0 + 32 * nb, a.n_in, a.x_wide, lane);
}

// dW and db over chunks of 2^chunk_shift rows: 32 outputs a wave (its part of
// Wa and Wu), 128 inputs (64 in 32
// bits). a and u are formed with rows of x as their rows, so
// that da and du are fragments of the product over the rows as they are; x is
// read both ways from one tile in LDS. HELD: these are all, and the
// wave's rows of W stay in registers for the whole chunk; a wave takes most of
// a SIMD's registers then.
template <class T, bool HELD>
__global__ __launch_bounds__(256, 1) void k_gated_dw(GatedArgs a) {
    constexpr int BK = gated_inputs<T>(), NB = BK / 32, KS = BK / 16, RB = row_bytes<T, 128>(), RX = row_bytes<T, BK>();
    constexpr int kEach = 32 * 128 / 8 / 256, kEachX = 32 * BK / 8 / 256;
    __shared__ __align__(128) char xs[2][32 * RX], dys[2][32 * RB];
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), m = lane & 31, h = lane >> 5;
    const int ot = (a.n_out + 127) / 128, it = max(1, (a.n_in + BK - 1) / BK);
    const unsigned id = die_order(blockIdx.x, gridDim.x), p = id / (ot * it), at2 = id - p * (ot * it);
    const int o0 = at2 / it * 128, i0 = at2 % it * BK;
    const Tile<int64_t> t = find_tile<int64_t>(a.off, a.n_bands, a.rows, a.batch, a.dw.chunk_shift, p, lane);
    if (!t.live || t.band < 0 || t.band >= a.n_bands) return;
    const int64_t n_rows = static_cast<int64_t>(t.len) * a.batch;
    const int64_t r_end = min(t.first + (int64_t(1) << a.dw.chunk_shift), n_rows);
    const int o = o0 + 32 * wave + m;   // this lane's output
    const bool works = o0 + 32 * wave < a.n_out, there = o < a.n_out;
    const T* wa = static_cast<const T*>(a.w) + (static_cast<int64_t>(t.band) * 2 * a.n_out + (there ? o : 0)) * a.n_in;
    const T* wu = wa + static_cast<int64_t>(a.n_out) * a.n_in;
    const float ba = gated_bias<T>(a, t, 0, o), bu = gated_bias<T>(a, t, 1, o);

    frag<T> fa[HELD ? KS : 1], fu[HELD ? KS : 1], xr[kEachX], yr[kEach];
    if constexpr (HELD) {
        by_width(a.w_wide, [&](auto wide) {
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int k = 16 * s + 8 * h, n = there ? a.n_in - k : 0;
                fa[s] = load8<T, wide.value>(wa + k, n, k > 0);
                fu[s] = load8<T, wide.value>(wu + k, n, k > 0);
            }
        });
    }
    auto fetch = [&](int64_t r0) {
        const int x0 = i0 + tid % (BK / 8) * 8, y0 = o0 + tid % 16 * 8;
        by_width(a.x_wide, [&](auto wide) {
#pragma unroll
            for (int e = 0; e < kEachX; ++e) {
                const int64_t r = r0 + (tid + 256 * e) / (BK / 8);
                const bool has = r < r_end;
                xr[e] = load8<T, wide.value>((has ? band_row<T>(a.x, t, r) : nullptr) + x0, has ? a.n_in - x0 : 0, x0 > 0);
            }
        });
        by_width(a.y_wide, [&](auto wide) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const int64_t r = r0 + (tid + 256 * e) / 16;
                const bool has = r < r_end;
                yr[e] = load8<T, wide.value>((has ? band_row<T>(a.dy, t, r) : nullptr) + y0, has ? a.n_out - y0 : 0, y0 > 0);
            }
        });
    };
    auto put = [&](int n) {
#pragma unroll
        for (int e = 0; e < kEachX; ++e) {
            const int c = tid + 256 * e;
            write8<T, RX>(xs[n], c / (BK / 8), c % (BK / 8), xr[e]);
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int c = tid + 256 * e;
            write8<T, RB>(dys[n], c / 16, c % 16, yr[e]);
        }
    };
    acc16 ga[NB], gu[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) ga[nb] = gu[nb] = zero16();
    float sa = 0.f, su = 0.f;
    fetch(t.first);
    put(0);
    __syncthreads();
    int buffer = 0;
#pragma unroll 1
    for (int64_t r0 = t.first; r0 < r_end; r0 += 32) {
        const char *tx = xs[buffer], *ty = dys[buffer];
        if (r0 + 32 < r_end) fetch(r0 + 32);
        if (works) {
            acc16 za, zu;
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                za[q] = ba;
                zu[q] = bu;
            }
            if constexpr (HELD) {
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const frag<T> xf = read8<T, RX>(tx, m, 2 * s + h);
                    za = mma(xf, fa[s], za);
                    zu = mma(xf, fu[s], zu);
                }
            } else {
                const bool mine = r0 + m < r_end;
                const T* in = mine ? band_row<T>(a.x, t, r0 + m) : nullptr;
                for (int k0 = 0; k0 < a.n_in; k0 += 16) {
                    const int k = k0 + 8 * h;
                    const frag<T> xf = load8<T, false>(in + k, mine ? a.n_in - k : 0, k > 0);
                    za = mma(xf, load8<T, false>(wa + k, there ? a.n_in - k : 0, k > 0), za);
                    zu = mma(xf, load8<T, false>(wu + k, there ? a.n_in - k : 0, k > 0), zu);
                }
            }
            float d[16];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const frag<T> f = read_turned<T, RB>(ty, 16 * x, 32 * wave, lane);
#pragma unroll
                for (int j = 0; j < 8; ++j) d[8 * x + j] = static_cast<float>(f[j]);
            }
            by_act(a.act, [&](auto act) __attribute__((always_inline)) { gated_slope<act.value>(za, zu, d); });
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                sa += za[q];
                su += zu[q];
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const auto da = sum_of<T, 2>(octet(za, x)), du = sum_of<T, 2>(octet(zu, x));
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const auto xf = data_of(read_turned<T, RX>(tx, 16 * x, 32 * nb, lane));
                    ga[nb] = product(da, xf, ga[nb]);
                    gu[nb] = product(du, xf, gu[nb]);
                }
            }
        }
        buffer ^= 1;
        if (r0 + 32 < r_end) put(buffer);
        __syncthreads();
    }
    if (!works) return;
    const bool whole = n_rows <= (int64_t(1) << a.dw.chunk_shift);
    const int64_t n_w = static_cast<int64_t>(2) * a.n_out * a.n_in;
    float* part = dw_part(a.dw, p);
    T* dw = static_cast<T*>(a.dw.dw) + t.band * n_w;
    auto store = [&](const acc16(&g)[NB], int which) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const int row = o0 + 32 * wave + 8 * (q >> 2) + 4 * h + (q & 3), i = i0 + 32 * nb + m;
                if (row < a.n_out && i < a.n_in) {
                    const int64_t at = (static_cast<int64_t>(which) * a.n_out + row) * a.n_in + i;
                    if (whole)
                        dw[at] = static_cast<T>(g[nb][q]);
                    else
                        part[at] = g[nb][q];
                }
            }
    };
    store(ga, 0);
    store(gu, 1);
    if (a.dw.db && i0 == 0) {
        sa = half_sum(sa);
        su = half_sum(su);
        if (h == 0 && there) {
            if (whole) {
                T* db = static_cast<T*>(a.dw.db) + static_cast<int64_t>(t.band) * 2 * a.n_out;
                db[o] = static_cast<T>(sa);
                db[a.n_out + o] = static_cast<T>(su);
            } else {
                part[n_w + o] = sa;
                part[n_w + a.n_out + o] = su;
            }
        }
    }
}

}  // namespace nsl
