// C entry of the attention along the bands (forward).
#include "attention_host.hpp"

using namespace nsl;

extern "C" int nsgcqt_band_attention(int dtype, const nsgcqt_rows* r, const nsgcqt_attention_shape* s,
                                     const nsgcqt_view* q, const nsgcqt_view* k, const nsgcqt_view* v,
                                     const nsgcqt_view* o, float* stats, void* stream) {
    CHECK_TRY(check_dtype(dtype));
    CHECK_TRY(check_rows(r));
    CHECK_TRY(check_shape(s));
    AttnArgs a = attention_args(r, s);
    bool wide = r->rows > 1;   // (a lone row's stride may be anything)
    CHECK_TRY(check_view(q, "q", dtype, r->batch, r->rows, s->n_heads, s->head_dim, wide));
    CHECK_TRY(check_view(k, "k", dtype, r->batch, r->rows, s->n_kv_heads, s->head_dim, wide));
    CHECK_TRY(check_view(v, "v", dtype, r->batch, r->rows, s->n_kv_heads, s->head_dim, wide));
    CHECK_TRY(check_view(o, "o", dtype, r->batch, r->rows, s->n_heads, s->head_dim, wide));
    if (misaligned(stats, 4)) return set_err(NSGCQT_EINVAL, "stats is not aligned to 4 bytes");
    if (r->batch == 0 || r->rows == 0) return NSGCQT_OK;
    a.q = view_of(q);
    a.k = view_of(k);
    a.v = view_of(v);
    a.o = view_of(o);
    a.stats = stats;
    const int64_t blocks = query_blocks(a);
    CHECK_TRY(check_grid(blocks));
    return by_shape(dtype, s->head_dim, wide, [&](auto t, auto dp, auto w) -> int {
        LAUNCH_TRY(k_attention<decltype(t), decltype(dp)::value, decltype(w)::value>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0,
                   static_cast<hipStream_t>(stream), a);
        return NSGCQT_OK;
    });
}
