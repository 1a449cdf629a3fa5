// A gated product of each band: two projections, an activation, their product.
//
//   a = Wa x + ba   u = Wu x + bu   y = act(a) u
//   da = dy u act'(a)   du = dy act(a)   dx = Wa^T da + Wu^T du   dW. = sum d. x^T   db. = sum d.
//
// W of a band: [2][n_out][n_in], Wa before Wu. a and u stay in registers: the
// forward call writes y alone, and each gradient forms them again, a third of
// its products; da and du in memory, each as two numbers of 16 bits, would be
// four times y's bytes, written once and read twice.
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
    int chunk_shift;        // rows of a workgroup of k_gated_kept
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
    const unsigned id = last_first(blockIdx.x, gridDim.x), p = id / cols;
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
            for (int q = 0; q < 16; ++q) acc[nb][q] = act_of<act.value, sizeof(T) == 4>(acc[nb][q]) * acc[NB + nb][q];
    });
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) store_column<T>(out, acc[nb], c0 + 32 * nb, a.n_out, a.y_wide, lane);
}

// A row's place among a band's rows of all signals, moved on without a division as long as it stays in its signal.
struct GatedRow {
    int64_t b;
    int c;
    __device__ GatedRow(const Tile<int64_t>& t, int64_t r) : b(r / t.len), c(static_cast<int>(r - b * t.len)) {}
    __device__ void move(const Tile<int64_t>& t, int by) {
        c += by;
        if (c >= t.len) {
            const int k = c / t.len;
            b += k;
            c -= k * t.len;
        }
    }
    template <class T> __device__ const T* of(const View& v, const Tile<int64_t>& t) const {
        return reinterpret_cast<const T*>(v.data) + b * v.batch + (t.start + c) * v.row;
    }
};

// Inputs that a workgroup of the gradients takes at once.
template <class T> constexpr int gated_inputs() { return sizeof(T) == 4 ? 64 : 128; }

// y where a row of x is one slab of gated_inputs: a workgroup keeps its 32 NB
// rows of Wa and of Wu in LDS, and its waves walk through 2^chunk_shift rows, 32
// at a time, on their own, the next rows on their way while these are computed;
// results leave through LDS, 128 bytes of a row at a time. 446,932 rows, 128 ->
// 256, bfloat16, silu: 163 us (k_gated 187), of 67 at the rate of a large copy;
// 355,340 rows, 96 -> 193, float16, gelu: 140 (179 with 16-byte stores). Bound by
// the activation's vector work (about 66 us) and waiting at two waves a SIMD.
template <class T, int NB>
__global__ __launch_bounds__(256, 2) void k_gated_kept(GatedArgs a) {
    constexpr int BK = gated_inputs<T>(), BN = 32 * NB, KS = BK / 16, RB = row_bytes<T, BK>();
    __shared__ __align__(128) char ws[2 * BN * RB];
    __shared__ __align__(16) float start[2 * BN];
    __shared__ __align__(128) char slabs[4][4096];
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), m = lane & 31, h = lane >> 5;
    const int cols = (a.n_out + BN - 1) / BN;
    const unsigned id = last_first(blockIdx.x, gridDim.x), p = id / cols;
    const int c0 = (id - p * cols) * BN;
    const Tile<int64_t> t = find_tile<int64_t>(a.off, a.n_bands, a.rows, a.batch, a.chunk_shift, p, lane);
    if (!t.live) return;
    const int n = static_cast<int>(min(int64_t(1) << a.chunk_shift, static_cast<int64_t>(t.len) * a.batch - t.first));
    GatedRow row(t, t.first + 32 * wave + m);
    auto out = [&]() { return const_cast<T*>(row.of<T>(a.y, t)); };
    if (t.band < 0 || t.band >= a.n_bands) {
        for (int r = 32 * wave; r < n; r += 128) {
            T* to = r + m < n ? out() : nullptr;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) store_column<T>(to, zero16(), c0 + 32 * nb, a.n_out, a.y_wide, lane);
            row.move(t, 128);
        }
        return;
    }
    frag<T> xf[KS];
    auto fetch = [&](const T* in, bool mine) {
        by_width(a.x_wide, [&](auto wide) {
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int k = 16 * s + 8 * h;
                xf[s] = load8<T, wide.value>(in + k, mine ? a.n_in - k : 0, k > 0);
            }
        });
    };
    fetch(row.of<T>(a.x, t), 32 * wave + m < n);
    const T* w = static_cast<const T*>(a.w) + static_cast<int64_t>(t.band) * 2 * a.n_out * a.n_in;
    by_width(a.w_wide, [&](auto wide) {
#pragma unroll
        for (int e = 0; e < 2 * BN * BK / 8 / 256; ++e) {
            const int c = tid + 256 * e;
            const int i = c / (BK / 8), o = c0 + i % BN, col = c % (BK / 8) * 8;
            const T* from = w + (static_cast<int64_t>(i / BN) * a.n_out + o) * a.n_in + col;
            write8<T, RB>(ws, i, col / 8, load8<T, wide.value>(from, o < a.n_out ? a.n_in - col : 0, col > 0));
        }
    });
    if (tid < 2 * BN) start[tid] = gated_bias<T>(a, t, tid / BN, c0 + tid % BN);
    __syncthreads();
#pragma unroll 1
    for (int r = 32 * wave; r < n; r += 128) {
        T* to = r + m < n ? out() : nullptr;
        acc16 acc[2 * NB];
#pragma unroll
        for (int nb = 0; nb < 2 * NB; ++nb) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f4 v = *reinterpret_cast<const f4*>(start + 32 * nb + 8 * q + 4 * h);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[nb][4 * q + j] = v[j];
            }
        }
#pragma unroll
        for (int s = 0; s < KS; ++s)
            if (16 * s < a.n_in) {
#pragma unroll
                for (int nb = 0; nb < 2 * NB; ++nb)
                    acc[nb] = mma(read8<T, RB>(ws, 32 * nb + m, 2 * s + h), xf[s], acc[nb]);
            }
        row.move(t, 128);
        if (r + 128 < n) fetch(row.of<T>(a.x, t), r + 128 + m < n);
        by_act(a.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int q = 0; q < 16; ++q) acc[nb][q] = act_of<act.value, sizeof(T) == 4>(acc[nb][q]) * acc[NB + nb][q];
        });
        T* row_out[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) row_out[e] = from_lane(to, lane / 8 + 8 * e);
        acc16 y[NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) y[nb] = acc[nb];
        store_rows<T, NB>(slabs[wave], y, row_out, min(n - r, 32), c0, a.n_out, a.y_wide, lane);
    }
}

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
template <int ACT, bool EXACT> __device__ inline void gated_slope(acc16& a, acc16& u, const float (&dy)[16]) {
#pragma unroll
    for (int q = 0; q < 16; ++q) {
        float slope;
        const float f = act_of<ACT, EXACT>(a[q], slope);
        a[q] = dy[q] * u[q] * slope;
        u[q] = dy[q] * f;
    }
}

// dx of 128 rows (32 a wave), 128 inputs (64 in 32 bits): along the outputs in blocks of 32,
// whose a and u are formed transposed (a lane's column is a row of x), turned
// into da and du in their registers, and go on from there, as two numbers of
// 16 bits each, into the product with W. Both products read the same tile of W,
// the second one turned. HELD: one tile holds a block's rows of W, and the row of
// x stays in registers. 446,932 rows, 128 -> 256, bfloat16: 290 us; without the
// activation's slope 245, without loading dy 270: bound by vector work (about 110
// us) and the matrix cores (70), which overlap little at two waves a SIMD.
template <class T, bool HELD>
__global__ __launch_bounds__(256, 2) void k_gated_dx(GatedArgs a) {
    constexpr int BK = gated_inputs<T>(), NB = BK / 32, KS = BK / 16, RB = row_bytes<T, BK>(), kEach = 2 * 32 * BK / 8 / 256;
    __shared__ __align__(128) char lds[2][2][32 * RB];
    __shared__ __align__(16) float start[2][2][32];
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), m = lane & 31, h = lane >> 5;
    const int slabs = (a.n_in + BK - 1) / BK;
    const unsigned id = last_first(blockIdx.x, gridDim.x), p = id / slabs;
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
            by_act(a.act, [&](auto act) __attribute__((always_inline)) { gated_slope<act.value, sizeof(T) == 4>(za, zu, d); });
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

__device__ inline float sum8(f8 x) { return ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7])); }

// A lane's fragments to and from LDS, as they are.
template <class F, int N> __device__ inline void put_pieces(char* at, int lane, const Pieces<F, N>& p) {
    constexpr int kParts = sizeof(F) / 16;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        f4 part[kParts];
        __builtin_memcpy(part, &p.p[i], sizeof(F));
#pragma unroll
        for (int k = 0; k < kParts; ++k) *reinterpret_cast<f4*>(at + ((i * kParts + k) * 64 + lane) * 16) = part[k];
    }
}
template <class F, int N> __device__ inline Pieces<F, N> get_pieces(const char* at, int lane) {
    constexpr int kParts = sizeof(F) / 16;
    Pieces<F, N> p;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        f4 part[kParts];
#pragma unroll
        for (int k = 0; k < kParts; ++k) part[k] = *reinterpret_cast<const f4*>(at + ((i * kParts + k) * 64 + lane) * 16);
        __builtin_memcpy(&p.p[i], part, sizeof(F));
    }
    return p;
}

// dW and db over chunks of 2^chunk_shift rows, 64 at a time: 128 outputs (their
// rows of Wa and of Wu) x 128 inputs (64 in 32 bits) a workgroup. Wave 4 j + i
// forms a and u of 32 of the rows (j) and 32 outputs (i) with rows of x as
// their rows, so that da and du are fragments of the product over the rows as
// they are; through LDS they go to the wave that takes the other half of the
// inputs. x is read both ways from one tile. HELD: the inputs are all there
// are, and W stays on chip for the whole chunk, Wa in registers and Wu in LDS.
// The same case: 365 us and 41 for the join (four waves of all inputs, W in
// registers, one wave a SIMD: 685); without the slope 325, without the second
// product 317. Its two barriers a step keep a SIMD's waves in the same phase, so
// that vector work and matrix cores take turns.
constexpr int kGatedThreads = 512;
template <class T, bool HELD>
__global__ __launch_bounds__(kGatedThreads, 2) void k_gated_dw(GatedArgs a) {
    constexpr int BK = gated_inputs<T>(), NB = BK / 64, KS = BK / 16, RB = row_bytes<T, 128>(), RX = row_bytes<T, BK>();
    constexpr int kEach = 64 * 128 / 8 / 512, kEachX = 64 * BK / 8 / 512, NP = sizeof(T) == 4 ? 1 : 2;
    constexpr int kPieces = NP * static_cast<int>(sizeof(piece<T>)) * 64;   // bytes of a fragment's pieces
    __shared__ __align__(128) char xs[2][64 * RX], dys[64 * RB], ds[8][4 * kPieces];
    __shared__ __align__(128) char wus[HELD ? 128 * RX : 128];   // Wu: with it too in registers there are not enough
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), m = lane & 31, h = lane >> 5;
    const int wi = wave & 3, wj = wave >> 2;
    const int ot = (a.n_out + 127) / 128, it = max(1, (a.n_in + BK - 1) / BK);
    const unsigned id = last_first(blockIdx.x, gridDim.x), p = id / (ot * it), at2 = id - p * (ot * it);
    const int o0 = at2 / it * 128, i0 = at2 % it * BK;
    const Tile<int64_t> t = find_tile<int64_t>(a.off, a.n_bands, a.rows, a.batch, a.dw.chunk_shift, p, lane);
    if (!t.live || t.band < 0 || t.band >= a.n_bands) return;
    const int64_t n_rows = static_cast<int64_t>(t.len) * a.batch;
    const int n = static_cast<int>(min(int64_t(1) << a.dw.chunk_shift, n_rows - t.first));
    const int o = o0 + 32 * wi + m;   // this lane's output
    const bool works = o0 + 32 * wi < a.n_out, there = o < a.n_out;
    const T* wa = static_cast<const T*>(a.w) + (static_cast<int64_t>(t.band) * 2 * a.n_out + (there ? o : 0)) * a.n_in;
    const T* wu = wa + static_cast<int64_t>(a.n_out) * a.n_in;
    const float ba = gated_bias<T>(a, t, 0, o), bu = gated_bias<T>(a, t, 1, o);

    frag<T> fa[HELD ? KS : 1], xr[kEachX], yr[kEach];
    if constexpr (HELD) {
        by_width(a.w_wide, [&](auto wide) {
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int k = 16 * s + 8 * h, n_k = there ? a.n_in - k : 0;
                fa[s] = load8<T, wide.value>(wa + k, n_k, k > 0);
                if (s % 2 == wj) write8<T, RX>(wus, 32 * wi + m, 2 * s + h, load8<T, wide.value>(wu + k, n_k, k > 0));
            }
        });
    }
    // this thread's rows of a step: row tid / 16 and 32 on of dy, and of x as many
    constexpr int kPerX = 512 / (BK / 8);
    GatedRow ry(t, t.first + tid / 16), rx(t, t.first + tid / (BK / 8));
    auto fetch = [&](int r0) {
        const int x0 = i0 + tid % (BK / 8) * 8, y0 = o0 + tid % 16 * 8;
        by_width(a.x_wide, [&](auto wide) {
#pragma unroll
            for (int e = 0; e < kEachX; ++e) {
                const bool has = r0 + tid / (BK / 8) + kPerX * e < n;
                xr[e] = load8<T, wide.value>(rx.of<T>(a.x, t) + x0, has ? a.n_in - x0 : 0, x0 > 0);
                rx.move(t, kPerX);
            }
        });
        by_width(a.y_wide, [&](auto wide) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const bool has = r0 + tid / 16 + 32 * e < n;
                yr[e] = load8<T, wide.value>(ry.of<T>(a.dy, t) + y0, has ? a.n_out - y0 : 0, y0 > 0);
                ry.move(t, 32);
            }
        });
    };
    auto put_x = [&](char* to) {
#pragma unroll
        for (int e = 0; e < kEachX; ++e) write8<T, RX>(to, tid / (BK / 8) + kPerX * e, tid % (BK / 8), xr[e]);
    };
    auto put_y = [&]() {
#pragma unroll
        for (int e = 0; e < kEach; ++e) write8<T, RB>(dys, tid / 16 + 32 * e, tid % 16, yr[e]);
    };
    acc16 ga[NB], gu[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) ga[nb] = gu[nb] = zero16();
    // Up to 128 sums of 8 a lane: where all are rounded the same way, off by 2^-18 in 32 bits.
    std::conditional_t<sizeof(T) == 4, double, float> sa = 0, su = 0;
    fetch(0);
    put_x(xs[0]);
    put_y();
    __syncthreads();
    int buffer = 0;
#pragma unroll 1
    for (int r0 = 0; r0 < n; r0 += 64) {
        const char* tx = xs[buffer];
        const bool more = r0 + 64 < n;
        if (more) fetch(r0 + 64);
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
                    const frag<T> xf = read8<T, RX>(tx, 32 * wj + m, 2 * s + h);
                    za = mma(xf, fa[s], za);
                    zu = mma(xf, read8<T, RX>(wus, 32 * wi + m, 2 * s + h), zu);
                }
            } else {
                const int r = r0 + 32 * wj + m;
                const T* in = r < n ? band_row<T>(a.x, t, t.first + r) : nullptr;
                for (int k0 = 0; k0 < a.n_in; k0 += 16) {
                    const int k = k0 + 8 * h;
                    const frag<T> xf = load8<T, false>(in + k, r < n ? a.n_in - k : 0, k > 0);
                    za = mma(xf, load8<T, false>(wa + k, there ? a.n_in - k : 0, k > 0), za);
                    zu = mma(xf, load8<T, false>(wu + k, there ? a.n_in - k : 0, k > 0), zu);
                }
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const frag<T> d = read_turned<T, RB>(dys, 32 * wj + 16 * x, 32 * wi, lane);
                f8 da, du;
                by_act(a.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        float slope;
                        const float f = act_of<act.value, sizeof(T) == 4>(za[8 * x + j], slope), dy = static_cast<float>(d[j]);
                        da[j] = dy * zu[8 * x + j] * slope;
                        du[j] = dy * f;
                    }
                });
                if (!more) {   // (rows that are not there: x and dy are 0, but a bias may be infinite)
                    const int left = n - (r0 + 32 * wj + 16 * x + 4 * h);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (8 * (j >> 2) + (j & 3) >= left) da[j] = du[j] = 0.f;
                }
                sa += sum8(da);
                su += sum8(du);
                put_pieces(ds[wave] + (2 * x) * kPieces, lane, sum_of<T, 2>(da));
                put_pieces(ds[wave] + (2 * x + 1) * kPieces, lane, sum_of<T, 2>(du));
            }
        }
        __syncthreads();
        buffer ^= 1;
        if (more) {
            put_x(xs[buffer]);
            put_y();
        }
        if (works) {
#pragma unroll
            for (int jj = 0; jj < 2; ++jj)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const char* from = ds[4 * jj + wi] + 2 * x * kPieces;
                    const auto da = get_pieces<piece<T>, NP>(from, lane), du = get_pieces<piece<T>, NP>(from + kPieces, lane);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        const auto xf = data_of(read_turned<T, RX>(tx, 32 * jj + 16 * x, 32 * (NB * wj + nb), lane));
                        ga[nb] = product(da, xf, ga[nb]);
                        gu[nb] = product(du, xf, gu[nb]);
                    }
                }
        }
        __syncthreads();
    }
    // the two waves of an output add up their rows' sums
    float* sums = reinterpret_cast<float*>(ds[0]);
    float ba_sum = half_sum(static_cast<float>(sa)), bu_sum = half_sum(static_cast<float>(su));
    if (wj == 1 && h == 0) {
        sums[2 * (32 * wi + m)] = ba_sum;
        sums[2 * (32 * wi + m) + 1] = bu_sum;
    }
    __syncthreads();
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
                const int row = o0 + 32 * wi + 8 * (q >> 2) + 4 * h + (q & 3), i = i0 + 32 * (NB * wj + nb) + m;
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
    if (a.dw.db && i0 == 0 && wj == 0 && h == 0 && there) {
        ba_sum += sums[2 * (32 * wi + m)];
        bu_sum += sums[2 * (32 * wi + m) + 1];
        if (whole) {
            T* db = static_cast<T*>(a.dw.db) + static_cast<int64_t>(t.band) * 2 * a.n_out;
            db[o] = static_cast<T>(ba_sum);
            db[a.n_out + o] = static_cast<T>(bu_sum);
        } else {
            part[n_w + o] = ba_sum;
            part[n_w + a.n_out + o] = bu_sum;
        }
    }
}

}  // namespace nsl
