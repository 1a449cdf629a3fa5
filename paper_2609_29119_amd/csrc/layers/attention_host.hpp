// What the forward and the gradient entry of the attention share on the host.
#pragma once
#include <cmath>

#include "attention.hpp"
#include "checks.hpp"

namespace nsl {

// The scores' factor in 32 bits, with and without log2(e), has to be a number.
inline int check_scale(double scale) {
    const float c = static_cast<float>(scale * 1.4426950408889634);
    if (!(scale > 0) || !std::isfinite(c) || c < 1e-37f)
        return set_err(NSGCQT_EINVAL, "scale must be positive and finite in 32 bits");
    return NSGCQT_OK;
}

inline AttnScale scale_of(double scale) {
    const double c = scale * 1.4426950408889634;
    return {static_cast<float>(c), static_cast<float>(1.0 / c)};
}

inline int check_shape(const nsgcqt_attention_shape* s) {
    if (!s) return set_err(NSGCQT_EINVAL, "shape is NULL");
    if (s->n_heads < 1 || s->n_kv_heads < 1 || s->n_heads % s->n_kv_heads)
        return set_err(NSGCQT_EINVAL, "n_kv_heads must divide n_heads, both at least 1");
    if (s->head_dim < 1) return set_err(NSGCQT_EINVAL, "head_dim must be at least 1");
    if (s->left < 0 || s->right < 0 || s->sinks < 0)
        return set_err(NSGCQT_EINVAL, "left, right and sinks must not be negative");
    CHECK_TRY(check_scale(s->scale));
    if (s->head_dim > 128) return set_err(NSGCQT_EUNSUPPORTED, "head_dim above 128");
    if (s->n_heads > 65536) return set_err(NSGCQT_EUNSUPPORTED, "more than 65,536 heads");
    return NSGCQT_OK;
}

inline AttnArgs attention_args(const nsgcqt_rows* r, const nsgcqt_attention_shape* s) {
    AttnArgs a{};
    a.keep = s->keep;
    a.keep_batch = s->keep_batch;
    a.off = r->offsets;
    a.rows = static_cast<int>(r->rows);
    a.n_bands = static_cast<int>(r->n_bands);
    a.batch = static_cast<int>(r->batch);
    a.heads = static_cast<int>(s->n_heads);
    a.kv_heads = static_cast<int>(s->n_kv_heads);
    a.dim = static_cast<int>(s->head_dim);
    const int group = a.heads / a.kv_heads;
    a.share = group % 4 == 0 ? 4 : group % 2 == 0 ? 2 : 1;
    auto cut = [&](int64_t v) { return static_cast<int>(v < r->rows ? v : r->rows); };
    a.left = cut(s->left);
    a.right = cut(s->right);
    a.sinks = cut(s->sinks);
    a.far = a.sinks < kFarSinks ? a.sinks : kFarSinks;
    a.scale = static_cast<float>(s->scale);
    a.by = scale_of(s->scale);
    return a;
}

// Workgroups of the kernels that go by queries.
inline int64_t query_blocks(const AttnArgs& a) {
    return product(tile_count(query_shift(a.share), a.n_bands, 1, a.rows), a.batch, a.heads / a.share);
}

// f(T(), DP) with the head width's padded size as an integral constant
template <class F> int by_type_and_width(int dtype, int64_t dim, F f) {
    return by_type(dtype, [&](auto t) {
        if (dim <= 32) return f(t, std::integral_constant<int, 32>());
        if (dim <= 64) return f(t, std::integral_constant<int, 64>());
        return f(t, std::integral_constant<int, 128>());
    });
}

// f(T(), DP, true_type or false_type)
template <class F> int by_shape(int dtype, int64_t dim, bool wide, F f) {
    return by_type_and_width(dtype, dim, [&](auto t, auto dp) {
        return wide ? f(t, dp, std::true_type()) : f(t, dp, std::false_type());
    });
}

}  // namespace nsl
