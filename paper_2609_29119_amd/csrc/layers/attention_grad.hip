// C entry of the attention's gradients.
#include "attention_host.hpp"

using namespace nsl;

namespace {

int64_t align256(int64_t b) { return (b + 255) / 256 * 256; }

int64_t delta_bytes(const AttnArgs& a) { return align256(int64_t(4) * a.rows * a.batch * a.heads); }

// Workgroups of the far queries: for each chunk, kv head and 32 sinks.
int64_t far_blocks(const AttnArgs& a) {
    return product(tile_count(kFarShift, a.n_bands, 1, a.rows), a.batch, a.kv_heads, (a.far + 31) / 32);
}

int64_t part_bytes(const AttnArgs& a) { return product(far_blocks(a), 4 * 2 * 32 * a.dim); }

// Whether some query lies past the window of some sink's key tile.
bool has_far(const AttnArgs& a) { return a.sinks > 0 && kKeys + a.left < a.rows; }

int64_t grad_bytes(const AttnArgs& a) {
    const int64_t part = has_far(a) ? workspace_of(part_bytes(a)) : 0;
    return part < 0 ? part : delta_bytes(a) + part;
}

}  // namespace

extern "C" int64_t nsgcqt_band_attention_workspace(const nsgcqt_rows* r, const nsgcqt_attention_shape* s) {
    CHECK_TRY(check_rows(r));
    CHECK_TRY(check_shape(s));
    const AttnArgs a = attention_args(r, s);
    return grad_bytes(a);
}

extern "C" int nsgcqt_band_attention_grad(int dtype, const nsgcqt_rows* r, const nsgcqt_attention_shape* s,
                                          const nsgcqt_view* q, const nsgcqt_view* k, const nsgcqt_view* v,
                                          const nsgcqt_view* o, const float* stats, const nsgcqt_view* d_o,
                                          const nsgcqt_view* dq, const nsgcqt_view* dk, const nsgcqt_view* dv,
                                          void* ws, size_t ws_bytes, void* stream) {
    CHECK_TRY(check_dtype(dtype));
    CHECK_TRY(check_rows(r));
    CHECK_TRY(check_shape(s));
    AttnArgs a = attention_args(r, s);
    bool wide = r->rows > 1;   // (a lone row's stride may be anything)
    const struct {
        const nsgcqt_view* v;
        const char* name;
        View* to;
        int64_t heads;
    } views[] = {{q, "q", &a.q, s->n_heads},       {k, "k", &a.k, s->n_kv_heads},     {v, "v", &a.v, s->n_kv_heads},
                 {o, "o", &a.o, s->n_heads},       {d_o, "d_o", &a.d_o, s->n_heads},  {dq, "dq", &a.dq, s->n_heads},
                 {dk, "dk", &a.dk, s->n_kv_heads}, {dv, "dv", &a.dv, s->n_kv_heads}};
    for (const auto& x : views)
        CHECK_TRY(check_view(x.v, x.name, dtype, r->batch, r->rows, x.heads, s->head_dim, wide));
    if (r->batch == 0 || r->rows == 0) return NSGCQT_OK;
    if (!stats || misaligned(stats, 4)) return set_err(NSGCQT_EINVAL, "stats is NULL or not aligned to 4 bytes");
    const int64_t need = grad_bytes(a);
    if (need < 0) return static_cast<int>(need);
    if (static_cast<int64_t>(ws_bytes) < need)
        return set_err(NSGCQT_EWORKSPACE, "workspace of " + std::to_string(ws_bytes) + " bytes, " +
                                              std::to_string(need) + " required");
    if (!ws || misaligned(ws, 16)) return set_err(NSGCQT_EINVAL, "workspace is NULL or not aligned to 16 bytes");
    for (const auto& x : views) *x.to = view_of(x.v);
    a.stats = const_cast<float*>(stats);
    a.delta = static_cast<float*>(ws);
    a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + delta_bytes(a));
    const int64_t queries = query_blocks(a), far = far_blocks(a);
    const int64_t keys = product(tile_count(kKeyShift, a.n_bands, 1, a.rows), a.batch, a.kv_heads);
    CHECK_TRY(check_grid(queries));
    CHECK_TRY(check_grid(keys));
    if (has_far(a)) CHECK_TRY(check_grid(far));
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return by_shape(dtype, s->head_dim, wide, [&](auto t, auto dp, auto w) -> int {
        using T = decltype(t);
        constexpr int DP = decltype(dp)::value;
        constexpr bool WIDE = decltype(w)::value;
        LAUNCH_TRY(k_attention_dq<T, DP, WIDE>, dim3(static_cast<unsigned>(queries)), dim3(256), 0, st, a);
        if (has_far(a)) LAUNCH_TRY(k_attention_far<T, DP, WIDE>, dim3(static_cast<unsigned>(far)), dim3(256), 0, st, a);
        LAUNCH_TRY(k_attention_dkv<T, DP, WIDE>, dim3(static_cast<unsigned>(keys)), dim3(256), 0, st, a);
        return NSGCQT_OK;
    });
}
