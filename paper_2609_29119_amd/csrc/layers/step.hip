// C entries of the single-token attention step and the cache's fill.
#include <algorithm>

#include "attention_host.hpp"
#include "step.hpp"

using namespace nsl;

namespace {

int check_step(int64_t streams, int64_t heads, int64_t kv_heads, int64_t dim, int64_t window, int64_t sinks) {
    if (streams < 0) return set_err(NSGCQT_EINVAL, "n_streams is negative");
    nsgcqt_attention_shape s{};
    s.n_heads = heads;
    s.n_kv_heads = kv_heads;
    s.head_dim = dim;
    s.sinks = sinks;
    s.scale = 1.0;
    CHECK_TRY(check_shape(&s));
    if (window < 1) return set_err(NSGCQT_EINVAL, "window must be at least 1");
    if (streams > kMaxCount || window >= kMaxCount || sinks >= kMaxCount || window + sinks >= kMaxCount)
        return set_err(NSGCQT_EUNSUPPORTED, "streams or slots beyond the supported range");
    return NSGCQT_OK;
}

int64_t head_blocks(int64_t heads, int64_t kv_heads) { return (heads / kv_heads + 31) / 32; }

// Stretches of a cache: enough workgroups for four on each of the 256 compute
// units, none shorter than 256 slots (two tiles for each wave; a shorter cache
// is one workgroup's and needs no join, which costs 6.5 us).
int64_t splits_of(int64_t streams, int64_t heads, int64_t kv_heads, int64_t slots) {
    const int64_t blocks = std::max<int64_t>(1, streams * kv_heads * head_blocks(heads, kv_heads));
    return std::max<int64_t>(1, std::min<int64_t>({1024 / blocks, slots / 256, 256}));
}

}  // namespace

extern "C" {

int64_t nsgcqt_attention_step_workspace(int64_t n_streams, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim,
                                        int64_t window, int64_t sinks) {
    CHECK_TRY(check_step(n_streams, n_heads, n_kv_heads, head_dim, window, sinks));
    const int64_t splits = splits_of(n_streams, n_heads, n_kv_heads, window + sinks);
    return splits == 1 ? 0 : 4 * n_streams * n_heads * splits * (head_dim + 2);
}

int nsgcqt_attention_step(int dtype, int64_t n_streams, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim,
                          int64_t window, int64_t sinks, double scale, const nsgcqt_view* q, const nsgcqt_view* k,
                          const nsgcqt_view* v, const nsgcqt_view* o, void* k_cache, void* v_cache,
                          const int64_t* pos, void* ws, size_t ws_bytes, void* stream) {
    CHECK_TRY(check_dtype(dtype));
    CHECK_TRY(check_step(n_streams, n_heads, n_kv_heads, head_dim, window, sinks));
    CHECK_TRY(check_scale(scale));
    StepArgs a{};
    bool wide = true;
    CHECK_TRY(check_view(q, "q", dtype, n_streams, 1, n_heads, head_dim, wide));
    CHECK_TRY(check_view(k, "k", dtype, n_streams, 1, n_kv_heads, head_dim, wide));
    CHECK_TRY(check_view(v, "v", dtype, n_streams, 1, n_kv_heads, head_dim, wide));
    CHECK_TRY(check_view(o, "o", dtype, n_streams, 1, n_heads, head_dim, wide));
    if (n_streams == 0) return NSGCQT_OK;
    const size_t e = elem_bytes(dtype);
    if (!k_cache || !v_cache || misaligned(k_cache, e) || misaligned(v_cache, e))
        return set_err(NSGCQT_EINVAL, "a cache is NULL or not aligned to its element");
    if (!pos || misaligned(pos, 8)) return set_err(NSGCQT_EINVAL, "pos is NULL or not aligned to 8 bytes");
    wide = wide && !misaligned(k_cache, 16) && !misaligned(v_cache, 16);
    a.splits = static_cast<int>(splits_of(n_streams, n_heads, n_kv_heads, window + sinks));
    const int64_t need = nsgcqt_attention_step_workspace(n_streams, n_heads, n_kv_heads, head_dim, window, sinks);
    if (static_cast<int64_t>(ws_bytes) < need)
        return set_err(NSGCQT_EWORKSPACE, "workspace of " + std::to_string(ws_bytes) + " bytes, " +
                                              std::to_string(need) + " required");
    if (need > 0 && (!ws || misaligned(ws, 4)))
        return set_err(NSGCQT_EINVAL, "workspace is NULL or not aligned to 4 bytes");
    a.q = view_of(q);
    a.k = view_of(k);
    a.v = view_of(v);
    a.o = view_of(o);
    a.k_cache = k_cache;
    a.v_cache = v_cache;
    a.pos = pos;
    a.part = static_cast<float*>(ws);
    a.streams = n_streams;
    a.heads = static_cast<int>(n_heads);
    a.kv_heads = static_cast<int>(n_kv_heads);
    a.dim = static_cast<int>(head_dim);
    a.group = a.heads / a.kv_heads;
    a.head_blocks = static_cast<int>(head_blocks(n_heads, n_kv_heads));
    a.slots = static_cast<int>(window + sinks);
    a.sinks = static_cast<int>(sinks);
    a.window = static_cast<int>(window);
    a.by = scale_of(scale);
    const int64_t blocks = n_streams * n_kv_heads * a.head_blocks * a.splits;
    CHECK_TRY(check_grid(blocks));
    CHECK_TRY(check_grid(n_streams * n_heads));
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return by_shape(dtype, head_dim, wide, [&](auto t, auto dp, auto w) -> int {
        using T = decltype(t);
        LAUNCH_TRY(k_step<T, decltype(dp)::value, decltype(w)::value>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, st, a);
        if (a.splits > 1)
            LAUNCH_TRY(k_step_join<T>, dim3(static_cast<unsigned>(n_streams * n_heads)), dim3(256), 0, st, a);
        return NSGCQT_OK;
    });
}

int nsgcqt_cache_fill(int dtype, const nsgcqt_rows* r, int64_t n_kv_heads, int64_t head_dim, int64_t window,
                      int64_t sinks, const nsgcqt_view* k, const nsgcqt_view* v, void* k_cache, void* v_cache,
                      void* stream) {
    CHECK_TRY(check_dtype(dtype));
    CHECK_TRY(check_rows(r));
    CHECK_TRY(check_step(r->batch * r->n_bands, n_kv_heads, n_kv_heads, head_dim, window, sinks));
    bool any = true;   // the copies take rows of every alignment
    CHECK_TRY(check_view(k, "k", dtype, r->batch, r->rows, n_kv_heads, head_dim, any));
    CHECK_TRY(check_view(v, "v", dtype, r->batch, r->rows, n_kv_heads, head_dim, any));
    const int64_t streams = r->batch * r->n_bands;
    if (streams == 0 || r->rows == 0) return NSGCQT_OK;
    const size_t e = elem_bytes(dtype);
    if (!k_cache || !v_cache || misaligned(k_cache, e) || misaligned(v_cache, e))
        return set_err(NSGCQT_EINVAL, "a cache is NULL or not aligned to its element");
    if (streams > 65535) return set_err(NSGCQT_EUNSUPPORTED, "more than 65,535 streams in one fill");
    FillArgs a{};
    a.k = view_of(k);
    a.v = view_of(v);
    a.k_cache = k_cache;
    a.v_cache = v_cache;
    a.off = r->offsets;
    a.rows = static_cast<int>(r->rows);
    a.n_bands = static_cast<int>(r->n_bands);
    a.kv_heads = static_cast<int>(n_kv_heads);
    a.dim = static_cast<int>(head_dim);
    a.slots = static_cast<int>(window + sinks);
    a.sinks = static_cast<int>(sinks);
    a.window = static_cast<int>(window);
    const int each = head_dim % 8 ? 1 : 8;
    const int64_t blocks = std::min<int64_t>((n_kv_heads * head_dim / each * (window + sinks) + 255) / 256,
                                             std::max<int64_t>(1, 65536 / streams));
    const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(streams));
    return by_type(dtype, [&](auto t) -> int {
        if (each == 8)
            LAUNCH_TRY(k_fill<decltype(t), 8>, grid, dim3(256), 0, static_cast<hipStream_t>(stream), a);
        else
            LAUNCH_TRY(k_fill<decltype(t), 1>, grid, dim3(256), 0, static_cast<hipStream_t>(stream), a);
        return NSGCQT_OK;
    });
}

}  // extern "C"
