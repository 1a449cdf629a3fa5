// C entries of the gated product.
#include <algorithm>

#include "checks.hpp"
#include "gated.hpp"

using namespace nsl;

namespace {

int check_gated(int dtype, const nsgcqt_rows* r, int64_t n_in, int64_t n_out, int act) {
    CHECK_TRY(check_dtype(dtype));
    CHECK_TRY(check_rows(r));
    if (n_in < 0 || n_out < 0) return set_err(NSGCQT_EINVAL, "a width is negative");
    if (act < NSGCQT_ACT_NONE || act > NSGCQT_ACT_SIGMOID)
        return set_err(NSGCQT_EINVAL, "unknown activation " + std::to_string(act));
    if (n_in > kMaxWidth || n_out > kMaxWidth / 2) return set_err(NSGCQT_EUNSUPPORTED, "n_in above 65,536 or n_out above 32,768");
    return NSGCQT_OK;
}

int check_parameter(const void* w, const char* name, int dtype, int64_t count) {
    if (count && !w) return set_err(NSGCQT_EINVAL, std::string(name) + " is NULL");
    if (misaligned(w, elem_bytes(dtype))) return set_err(NSGCQT_EINVAL, std::string(name) + " is not aligned to its element");
    return NSGCQT_OK;
}

GatedArgs gated_args(const nsgcqt_rows* r, const void* w, const void* bias, int64_t n_in, int64_t n_out, int act) {
    GatedArgs a{};
    a.w = w;
    a.bias = bias;
    a.off = r->offsets;
    a.rows = static_cast<int>(r->rows);
    a.n_bands = static_cast<int>(r->n_bands);
    a.batch = static_cast<int>(r->batch);
    a.n_in = static_cast<int>(n_in);
    a.n_out = static_cast<int>(n_out);
    a.act = act;
    a.x_wide = a.y_wide = true;
    a.w_wide = n_in % 8 == 0 && !misaligned(w, 16);
    return a;
}

// Rows of a chunk of the weights' gradient, 256 to 4096: the most that leave
// 800 workgroups of 512 threads. 446,932 rows, 128 -> 256: 1024 rows 373 us and
// 40 for the join, 512 rows 434 and 64, 2048 rows 403 and 30.
int gated_chunk_shift(int64_t batch, int64_t rows, int64_t n_out) {
    const int64_t tiles = (n_out + 127) / 128;
    int shift = 12;
    while (shift > 8 && ((batch * rows) >> shift) * tiles < 800) --shift;
    return shift;
}

// Rows of a workgroup of k_gated_kept: up to 2048 for each copy of W into LDS,
// but not so many that fewer than 4 workgroups fall on a compute unit (446,932
// rows, 128 -> 256: 2048 rows 165 us, 1024 rows 175, 512 rows 195).
int kept_rows_shift(int64_t batch, int64_t rows, int64_t cols) {
    int shift = 11;
    while (shift > 7 && ((batch * rows) >> shift) * cols < 1024) --shift;
    return shift;
}

}  // namespace

extern "C" {

int nsgcqt_band_gated(int dtype, const nsgcqt_rows* r, const nsgcqt_view* x, const void* w, const void* bias,
                      const nsgcqt_view* y, int64_t n_in, int64_t n_out, int act, void* stream) {
    CHECK_TRY(check_gated(dtype, r, n_in, n_out, act));
    GatedArgs a = gated_args(r, w, bias, n_in, n_out, act);
    CHECK_TRY(check_view(x, "x", dtype, r->batch, r->rows, 1, n_in, a.x_wide));
    CHECK_TRY(check_view(y, "y", dtype, r->batch, r->rows, 1, n_out, a.y_wide));
    CHECK_TRY(check_parameter(w, "w", dtype, r->n_bands * n_in * n_out));
    CHECK_TRY(check_parameter(bias, "bias", dtype, 0));
    if (r->batch == 0 || r->rows == 0 || n_out == 0) return NSGCQT_OK;
    a.x = view_of(x);
    a.y = view_of(y);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return by_type(dtype, [&](auto t) -> int {
        using T = decltype(t);
        auto go = [&](auto nb) -> int {
            constexpr int NB = decltype(nb)::value;
            const int64_t cols = (n_out + 32 * NB - 1) / (32 * NB);
            if (n_in <= gated_inputs<T>()) {
                a.chunk_shift = kept_rows_shift(a.batch, a.rows, cols);
                const int64_t blocks = tile_count(a.chunk_shift, a.n_bands, a.batch, a.rows) * cols;
                CHECK_TRY(check_grid(blocks));
                LAUNCH_TRY((k_gated_kept<T, NB>), dim3(static_cast<unsigned>(blocks)), dim3(256), 0, st, a);
                return NSGCQT_OK;
            }
            const int64_t blocks = tile_count(kRowShift, a.n_bands, a.batch, a.rows) * cols;
            CHECK_TRY(check_grid(blocks));
            LAUNCH_TRY((k_gated<T, NB>), dim3(static_cast<unsigned>(blocks)), dim3(256), 0, st, a);
            return NSGCQT_OK;
        };
        return n_out <= 32 ? go(std::integral_constant<int, 1>()) : go(std::integral_constant<int, 2>());
    });
}

int64_t nsgcqt_band_gated_workspace(const nsgcqt_rows* r, int64_t n_in, int64_t n_out) {
    CHECK_TRY(check_gated(NSGCQT_F32, r, n_in, n_out, 0));
    return workspace_of(product(4, tile_count(gated_chunk_shift(r->batch, r->rows, n_out), r->n_bands, r->batch, r->rows),
                                2 * n_in * n_out + 2 * n_out));
}

int nsgcqt_band_gated_grad(int dtype, const nsgcqt_rows* r, const nsgcqt_view* x, const void* w, const void* bias,
                           const nsgcqt_view* dy, const nsgcqt_view* dx, void* dw, void* db, int64_t n_in,
                           int64_t n_out, int act, void* ws, size_t ws_bytes, void* stream) {
    CHECK_TRY(check_gated(dtype, r, n_in, n_out, act));
    GatedArgs a = gated_args(r, w, bias, n_in, n_out, act);
    CHECK_TRY(check_view(x, "x", dtype, r->batch, r->rows, 1, n_in, a.x_wide));
    CHECK_TRY(check_view(dy, "dy", dtype, r->batch, r->rows, 1, n_out, a.y_wide));
    if (dx) CHECK_TRY(check_view(dx, "dx", dtype, r->batch, r->rows, 1, n_in, a.x_wide));
    CHECK_TRY(check_parameter(w, "w", dtype, r->n_bands * n_in * n_out));
    CHECK_TRY(check_parameter(bias, "bias", dtype, 0));
    if (misaligned(dw, elem_bytes(dtype)) || misaligned(db, elem_bytes(dtype)))
        return set_err(NSGCQT_EINVAL, "dw or db is not aligned to its element");
    if (db && !dw && n_in) return set_err(NSGCQT_EINVAL, "db without dw");
    a.x = view_of(x);
    a.dy = view_of(dy);
    if (dx) a.y = view_of(dx);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const bool weights = (dw || db) && r->n_bands > 0 && n_out > 0, inputs = dx && r->batch > 0 && r->rows > 0 && n_in > 0;
    const int64_t at_once = dtype == NSGCQT_F32 ? gated_inputs<float>() : gated_inputs<__bf16>();
    const int64_t slabs = (n_in + at_once - 1) / at_once, blocks = tile_count(kRowShift, r->n_bands, r->batch, r->rows) * slabs;
    if (inputs) CHECK_TRY(check_grid(blocks));
    int64_t items = 0;
    if (weights) {
        const int64_t need = nsgcqt_band_gated_workspace(r, n_in, n_out);
        if (need < 0) return static_cast<int>(need);
        if (static_cast<int64_t>(ws_bytes) < need)
            return set_err(NSGCQT_EWORKSPACE, "workspace of " + std::to_string(ws_bytes) + " bytes, " +
                                                  std::to_string(need) + " required");
        if (!ws || misaligned(ws, 16)) return set_err(NSGCQT_EINVAL, "workspace is NULL or not aligned to 16 bytes");
        a.dw.dw = dw;
        a.dw.db = db;
        a.dw.part = static_cast<float*>(ws);
        a.dw.off = r->offsets;
        a.dw.rows = a.rows;
        a.dw.n_bands = a.n_bands;
        a.dw.batch = a.batch;
        a.dw.n_in = a.n_in;
        a.dw.n_out = 2 * a.n_out;
        a.dw.chunk_shift = gated_chunk_shift(r->batch, r->rows, n_out);
        items = tile_count(a.dw.chunk_shift, r->n_bands, r->batch, r->rows) * ((n_out + 127) / 128) *
                (slabs ? slabs : 1);
        CHECK_TRY(check_grid(items, kGatedThreads));
    }
    return by_type(dtype, [&](auto t) -> int {
        using T = decltype(t);
        auto go = [&](auto held) -> int {
            constexpr bool kHeld = decltype(held)::value;
            if (inputs) LAUNCH_TRY((k_gated_dx<T, kHeld>), dim3(static_cast<unsigned>(blocks)), dim3(256), 0, st, a);
            if (weights) {
                LAUNCH_TRY((k_gated_dw<T, kHeld>), dim3(static_cast<unsigned>(items)), dim3(kGatedThreads), 0, st, a);
                const int64_t join = (2 * n_in * n_out + 2 * n_out + 255) / 256;
                for (LinearArgs l = a.dw; l.first_band < l.n_bands; l.first_band += 65535)
                    LAUNCH_TRY(k_linear_join<T>, dim3(static_cast<unsigned>(join < 64 ? join : 64),
                                                      static_cast<unsigned>(std::min(l.n_bands - l.first_band, 65535))),
                               dim3(256), 0, st, l);
            }
            return NSGCQT_OK;
        };
        return n_in <= at_once ? go(std::true_type()) : go(std::false_type());
    });
}

}  // extern "C"
