// Argument checks of the layer calls.
#pragma once
#include "../../../include/nsgcqt_layers.h"
#include "../status.hpp"
#include "tile.hpp"

namespace nsl {

using nsg::launch_kernel;
using nsg::set_err;

constexpr int64_t kMaxRows = int64_t(1) << 30, kMaxCount = int64_t(1) << 30, kMaxBands = int64_t(1) << 24,
                  kMaxWidth = 65536, kMaxGrid = 0xffffffffll / 256;   // a launch takes less than 2^32 threads

inline int elem_bytes(int dtype) { return dtype == NSGCQT_F32 ? 4 : 2; }

inline int check_dtype(int dtype) {
    if (dtype != NSGCQT_F32 && dtype != NSGCQT_F16 && dtype != NSGCQT_BF16)
        return set_err(NSGCQT_EINVAL, "unknown data type " + std::to_string(dtype));
    return NSGCQT_OK;
}

inline bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

inline int check_rows(const nsgcqt_rows* r) {
    if (!r) return set_err(NSGCQT_EINVAL, "rows is NULL");
    if (r->n_bands < 0 || r->batch < 0 || r->rows < 0) return set_err(NSGCQT_EINVAL, "a count of the rows is negative");
    if (!r->offsets) return set_err(NSGCQT_EINVAL, "offsets is NULL");
    if (misaligned(r->offsets, 8)) return set_err(NSGCQT_EINVAL, "offsets is not aligned to 8 bytes");
    if (r->rows >= kMaxRows || r->n_bands > kMaxBands || r->batch > kMaxCount || r->rows * r->batch > (int64_t(1) << 40))
        return set_err(NSGCQT_EUNSUPPORTED, "rows, bands or batch beyond the supported range");
    return NSGCQT_OK;
}

// A tensor [batch][rows][heads][width]: its pointer and alignment; `wide`
// stays true if it takes 16-byte accesses, its rows do not overlap, and a tile
// of up to 128 rows spans less than the 2^31 bytes that a buffer access reaches.
inline int check_view(const nsgcqt_view* v, const char* name, int dtype, int64_t batch, int64_t rows, int64_t heads,
                      int64_t width, bool& wide) {
    if (!v) return set_err(NSGCQT_EINVAL, std::string(name) + " is NULL");
    if (batch == 0 || rows == 0 || heads == 0 || width == 0) return NSGCQT_OK;
    const int e = elem_bytes(dtype);
    if (!v->data) return set_err(NSGCQT_EINVAL, std::string(name) + " has a NULL pointer");
    if (misaligned(v->data, e)) return set_err(NSGCQT_EINVAL, std::string(name) + " is not aligned to its element");
    // the stride of an axis of one element is not read
    if ((batch > 1 && v->batch < 0) || (rows > 1 && v->row < 0) || (heads > 1 && v->head < 0))
        return set_err(NSGCQT_EINVAL, std::string(name) + " has a negative stride");
    const int64_t step = 16 / e;
    if (misaligned(v->data, 16) || width % 8 || (batch > 1 && v->batch % step) || (heads > 1 && v->head % step) ||
        (rows > 1 && (v->row % step || v->row >= (int64_t(1) << 23) / e || v->row < width)))
        wide = false;
    return NSGCQT_OK;
}

inline View view_of(const nsgcqt_view* v) { return View{static_cast<char*>(v->data), v->batch, v->row, v->head}; }

#define CHECK_TRY(expr)                                \
    do {                                               \
        if (int r_ = (expr); r_ != NSGCQT_OK) return r_; \
    } while (0)

// The product of counts that are not negative, or the largest number.
template <class... N> inline int64_t product(int64_t a, N... rest) {
    if constexpr (sizeof...(rest) > 0) {
        int64_t all;
        return __builtin_mul_overflow(a, product(rest...), &all) ? INT64_MAX : all;
    }
    return a;
}

inline int check_grid(int64_t blocks) {
    if (blocks > kMaxGrid) return set_err(NSGCQT_EUNSUPPORTED, "more than 16,777,215 workgroups");
    return NSGCQT_OK;
}

// A workspace's size in bytes.
inline int64_t workspace_of(int64_t bytes) {
    if (bytes > (int64_t(1) << 60)) return set_err(NSGCQT_EUNSUPPORTED, "a workspace above 2^60 bytes");
    return bytes;
}

// f(T()) for the element type of dtype
template <class F> int by_type(int dtype, F f) {
    switch (dtype) {
        case NSGCQT_F32: return f(float());
        case NSGCQT_F16: return f(_Float16());
        default: return f(__bf16());
    }
}

}  // namespace nsl
