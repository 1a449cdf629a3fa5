// C entries of the per-band products.
#include <algorithm>

#include "checks.hpp"
#include "linear.hpp"

using namespace nsl;

namespace {

int check_linear(int dtype, const nsgcqt_rows* r, int64_t n_in, int64_t n_out) {
    CHECK_TRY(check_dtype(dtype));
    CHECK_TRY(check_rows(r));
    if (n_in < 0 || n_out < 0) return set_err(NSGCQT_EINVAL, "a width is negative");
    if (n_in > kMaxWidth || n_out > kMaxWidth) return set_err(NSGCQT_EUNSUPPORTED, "a width above 65,536");
    return NSGCQT_OK;
}

LinearArgs linear_args(const nsgcqt_rows* r, int64_t n_in, int64_t n_out) {
    LinearArgs a{};
    a.off = r->offsets;
    a.rows = static_cast<int>(r->rows);
    a.n_bands = static_cast<int>(r->n_bands);
    a.batch = static_cast<int>(r->batch);
    a.n_in = static_cast<int>(n_in);
    a.n_out = static_cast<int>(n_out);
    a.x_wide = a.y_wide = true;
    return a;
}

// Rows of a chunk of the weights' gradient, 256 to 4096: the most that leave 400
// workgroups. 446,932 rows of 128 x 128: 1024 rows (436 workgroups) 82 us in
// all, 512 rows 94, 2048 rows 111.
int chunk_shift_of(int64_t batch, int64_t rows, int64_t n_in, int64_t n_out) {
    const int64_t tiles = ((n_out + 127) / 128) * (n_in ? (n_in + 127) / 128 : 1);
    int shift = 12;
    while (shift > 8 && ((batch * rows) >> shift) * tiles < 400) --shift;
    return shift;
}

// LDS of k_linear_kept for W.
template <class T, bool BACK> int kept_bytes(int64_t n_red, int64_t n_col, int nb) {
    if (n_red > 4096) return kKeptLds;
    return kept_rows<BACK>(static_cast<int>(n_red), static_cast<int>(n_col), nb) *
           kept_row_bytes<T, BACK>(static_cast<int>(n_red), nb);
}

// Rows of a workgroup of k_linear_kept: up to 1024 for each copy of W into
// LDS, but not so many that fewer than 4 workgroups fall on a compute unit
// (44,374 rows of 2 -> 32: 128 rows 8.0 us, 1024 rows 17; 710,680 rows of
// 193 -> 77: 512 rows 149 us, 128 rows about 200).
int kept_shift(int64_t batch, int64_t rows, int64_t cols) {
    int shift = 10;
    while (shift > 7 && ((batch * rows) >> shift) * cols < 1024) --shift;
    return shift;
}

int check_weights(const void* w, const char* name, int dtype, int64_t count) {
    if (count && !w) return set_err(NSGCQT_EINVAL, std::string(name) + " is NULL");
    if (misaligned(w, elem_bytes(dtype))) return set_err(NSGCQT_EINVAL, std::string(name) + " is not aligned to its element");
    return NSGCQT_OK;
}

// y = W x, or with BACK dx = W^T dy: in has n_red columns, out n_col.
template <bool BACK>
int run_linear(int dtype, const nsgcqt_rows* r, const nsgcqt_view* in, const void* w, const void* bias,
               const nsgcqt_view* out, int64_t n_in, int64_t n_out, void* stream) {
    CHECK_TRY(check_linear(dtype, r, n_in, n_out));
    LinearArgs a = linear_args(r, n_in, n_out);
    const int64_t n_red = BACK ? n_out : n_in, n_col = BACK ? n_in : n_out;
    CHECK_TRY(check_view(in, BACK ? "dy" : "x", dtype, r->batch, r->rows, 1, n_red, a.x_wide));
    CHECK_TRY(check_view(out, BACK ? "dx" : "y", dtype, r->batch, r->rows, 1, n_col, a.y_wide));
    CHECK_TRY(check_weights(w, "w", dtype, r->n_bands * n_in * n_out));
    CHECK_TRY(check_weights(bias, "bias", dtype, 0));
    if (r->batch == 0 || r->rows == 0 || n_col == 0) return NSGCQT_OK;
    a.x = view_of(in);
    a.y = view_of(out);
    a.w = w;
    a.bias = bias;
    a.w_wide = n_in % 8 == 0 && !misaligned(w, 16);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return by_type(dtype, [&](auto t) -> int {
        using T = decltype(t);
        auto go = [&](auto nb) -> int {
            constexpr int NB = decltype(nb)::value;
            const int64_t cols = (n_col + 32 * NB - 1) / (32 * NB);
            const int lds = kKeptRest + kept_bytes<T, BACK>(n_red, n_col, NB);
            if (!a.x_wide && n_red > 0 && lds <= kKeptLds) {
                a.chunk_shift = kept_shift(a.batch, a.rows, cols);
                const int64_t blocks = tile_count(a.chunk_shift, a.n_bands, a.batch, a.rows) * cols;
                CHECK_TRY(check_grid(blocks));
                LAUNCH_TRY(k_linear_kept<T, NB, BACK>, dim3(static_cast<unsigned>(blocks)), dim3(256),
                           static_cast<size_t>(lds), st, a);
                return NSGCQT_OK;
            }
            const int64_t blocks = tile_count(kRowShift, a.n_bands, a.batch, a.rows) * cols;
            CHECK_TRY(check_grid(blocks));
            LAUNCH_TRY(k_linear<T, NB, BACK>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, st, a);
            return NSGCQT_OK;
        };
        if (n_col <= 32) return go(std::integral_constant<int, 1>());
        if (n_col <= 64) return go(std::integral_constant<int, 2>());
        if (n_col <= 96) return go(std::integral_constant<int, 3>());
        return go(std::integral_constant<int, 4>());
    });
}

}  // namespace

extern "C" {

int nsgcqt_band_linear(int dtype, const nsgcqt_rows* r, const nsgcqt_view* x, const void* w, const void* bias,
                       const nsgcqt_view* y, int64_t n_in, int64_t n_out, void* stream) {
    return run_linear<false>(dtype, r, x, w, bias, y, n_in, n_out, stream);
}

int nsgcqt_band_linear_grad_input(int dtype, const nsgcqt_rows* r, const nsgcqt_view* dy, const void* w,
                                  const nsgcqt_view* dx, int64_t n_in, int64_t n_out, void* stream) {
    return run_linear<true>(dtype, r, dy, w, nullptr, dx, n_in, n_out, stream);
}

int64_t nsgcqt_band_linear_workspace(int64_t n_bands, int64_t batch, int64_t rows, int64_t n_in, int64_t n_out) {
    static const int64_t none = 0;
    const nsgcqt_rows r{&none, n_bands, batch, rows};
    CHECK_TRY(check_linear(NSGCQT_F32, &r, n_in, n_out));
    return workspace_of(
        product(4, tile_count(chunk_shift_of(batch, rows, n_in, n_out), n_bands, batch, rows), n_in * n_out + n_out));
}

int nsgcqt_band_linear_grad_weight(int dtype, const nsgcqt_rows* r, const nsgcqt_view* x, const nsgcqt_view* dy,
                                   void* dw, void* db, int64_t n_in, int64_t n_out, void* ws, size_t ws_bytes,
                                   void* stream) {
    CHECK_TRY(check_linear(dtype, r, n_in, n_out));
    LinearArgs a = linear_args(r, n_in, n_out);
    CHECK_TRY(check_view(x, "x", dtype, r->batch, r->rows, 1, n_in, a.x_wide));
    CHECK_TRY(check_view(dy, "dy", dtype, r->batch, r->rows, 1, n_out, a.y_wide));
    CHECK_TRY(check_weights(dw, "dw", dtype, r->n_bands * n_in * n_out));
    CHECK_TRY(check_weights(db, "db", dtype, 0));
    if (r->n_bands == 0 || n_out == 0 || (n_in == 0 && !db)) return NSGCQT_OK;
    const int64_t need = nsgcqt_band_linear_workspace(r->n_bands, r->batch, r->rows, n_in, n_out);
    if (need < 0) return static_cast<int>(need);
    if (static_cast<int64_t>(ws_bytes) < need)
        return set_err(NSGCQT_EWORKSPACE, "workspace of " + std::to_string(ws_bytes) + " bytes, " +
                                              std::to_string(need) + " required");
    if (!ws || misaligned(ws, 16)) return set_err(NSGCQT_EINVAL, "workspace is NULL or not aligned to 16 bytes");
    a.x = view_of(x);
    a.y = view_of(dy);
    a.dw = dw;
    a.db = db;
    a.part = static_cast<float*>(ws);
    a.chunk_shift = chunk_shift_of(r->batch, r->rows, n_in, n_out);
    // with no inputs there is still the sum of dy
    const int64_t ot = (n_out + 127) / 128, it = n_in ? (n_in + 127) / 128 : 1;
    const int64_t blocks = tile_count(a.chunk_shift, a.n_bands, a.batch, a.rows) * ot * it;
    const int64_t join = (n_in * n_out + n_out + 255) / 256;
    CHECK_TRY(check_grid(blocks));
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return by_type(dtype, [&](auto t) -> int {
        using T = decltype(t);
        LAUNCH_TRY(k_linear_dw<T>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, st, a);
        for (; a.first_band < a.n_bands; a.first_band += 65535)   // the most that a grid's second axis holds
            LAUNCH_TRY(k_linear_join<T>, dim3(static_cast<unsigned>(join < 64 ? join : 64),
                                              static_cast<unsigned>(std::min(a.n_bands - a.first_band, 65535))),
                       dim3(256), 0, st, a);
        return NSGCQT_OK;
    });
}

}  // extern "C"
