// C entries of the decayed linear attention and its single-token step.
#include <algorithm>
#include <cmath>

#include "checks.hpp"
#include "decay.hpp"

using namespace nsl;

namespace {

int check_decay(const nsgcqt_decay_shape* s) {
    if (!s) return set_err(NSGCQT_EINVAL, "shape is NULL");
    if (s->n_heads < 1 || s->n_kv_heads < 1 || s->n_heads % s->n_kv_heads)
        return set_err(NSGCQT_EINVAL, "n_kv_heads must divide n_heads, both at least 1");
    if (s->head_dim < 1) return set_err(NSGCQT_EINVAL, "head_dim must be at least 1");
    if (!std::isfinite(static_cast<float>(s->scale))) return set_err(NSGCQT_EINVAL, "scale must be finite in 32 bits");
    if (s->head_dim > 128) return set_err(NSGCQT_EUNSUPPORTED, "head_dim above 128");
    if (s->n_heads > 65536) return set_err(NSGCQT_EUNSUPPORTED, "more than 65,536 heads");
    return NSGCQT_OK;
}

int check_log_decay(const float* p) {
    if (!p || misaligned(p, 4)) return set_err(NSGCQT_EINVAL, "log_decay is NULL or not aligned to 4 bytes");
    return NSGCQT_OK;
}

int check_state(const float* p) {
    if (misaligned(p, 4)) return set_err(NSGCQT_EINVAL, "state is not aligned to 4 bytes");
    return NSGCQT_OK;
}

// Tokens of a segment, 64 to 4096 (2048 for the gradients, where some heads
// walk through them several times): the most that leave 1536 workgroups of one
// result head each; and of a part of it, at most 1024, as many of one key head
// (few of a ragged row's tokens lie in bands of several segments). A part's
// state costs as much to write, join and read as 4 head_dim of its tokens: parts
// of less than 8 head_dim tokens only below 1024 workgroups. 131,072 tokens, 8
// heads of 128, bfloat16, all three kernels: 256 tokens 561 us, 512 497, 1024 500,
// 2048 574; 446,932 tokens over 221 bands, 8 heads of 64 over 4: 512 tokens 607,
// 1024 600, 2048 650.
int shift_of(int64_t batch, int64_t rows, int64_t heads, int64_t dim, int shift) {
    while (shift > 6 && product(batch, (rows + (int64_t(1) << shift) - 1) >> shift, heads) < (1 << shift > 8 * dim ? 1536 : 1024)) --shift;
    return shift;
}
struct DecayCut { int shift, fine; };
DecayCut cut_of(const nsgcqt_rows* r, const nsgcqt_decay_shape* s, bool grad) {
    const int64_t heads = grad ? s->n_heads + 2 * s->n_kv_heads : s->n_heads;
    const int shift = shift_of(r->batch, r->rows, heads, s->head_dim, grad ? 11 : 12);
    return {shift, shift_of(r->batch, r->rows, (grad ? 2 : 1) * s->n_kv_heads, s->head_dim, std::min(shift, 10))};
}

// Bytes of the states within bands of several segments.
int64_t decay_workspace(const nsgcqt_rows* r, const nsgcqt_decay_shape* s, bool grad) {
    const DecayCut cut = cut_of(r, s, grad);
    if (r->rows <= int64_t(1) << cut.shift) return 0;   // no band has several segments
    return workspace_of(product(grad ? 8 : 4, r->batch, slot_count(r->rows, cut.fine), s->n_kv_heads, s->head_dim * s->head_dim));
}

int check_workspace(const void* ws, size_t have, int64_t need) {
    if (need < 0) return static_cast<int>(need);
    if (static_cast<int64_t>(have) < need)
        return set_err(NSGCQT_EWORKSPACE, "workspace of " + std::to_string(have) + " bytes, " + std::to_string(need) +
                                              " required");
    if (need > 0 && (!ws || misaligned(ws, 4)))
        return set_err(NSGCQT_EINVAL, "workspace is NULL or not aligned to 4 bytes");
    return NSGCQT_OK;
}

DecayArgs decay_args(const nsgcqt_rows* r, const nsgcqt_decay_shape* s, bool grad) {
    DecayArgs a{};
    a.log_decay = s->log_decay;
    a.keep = s->keep;
    a.keep_batch = s->keep_batch;
    a.off = r->offsets;
    a.rows = static_cast<int>(r->rows);
    a.n_bands = static_cast<int>(r->n_bands);
    a.batch = static_cast<int>(r->batch);
    a.kv_heads = static_cast<int>(s->n_kv_heads);
    a.dim = static_cast<int>(s->head_dim);
    a.units = static_cast<int>(grad ? s->n_heads + 2 * s->n_kv_heads : s->n_heads);
    const DecayCut cut = cut_of(r, s, grad);
    a.shift = cut.shift;
    a.fine = cut.fine;
    a.scale = static_cast<float>(s->scale);
    return a;
}

// f(T(), DP, true_type or false_type)
template <class F> int by_decay_shape(int dtype, int64_t dim, bool wide, F f) {
    return by_type(dtype, [&](auto t) {
        auto with = [&](auto dp) { return wide ? f(t, dp, std::true_type()) : f(t, dp, std::false_type()); };
        if (dim <= 32) return with(std::integral_constant<int, 32>());
        if (dim <= 64) return with(std::integral_constant<int, 64>());
        if (dim <= 96) return with(std::integral_constant<int, 96>());
        return with(std::integral_constant<int, 128>());
    });
}

// The launches of a call: `a` with its jobs, `sums` the ones whose states are formed (the first n_sums jobs of it).
int run_decay(int dtype, const nsgcqt_rows* r, const DecayArgs& a, DecayArgs sums, int n_sums, bool wide, hipStream_t st) {
    const bool several = r->rows > int64_t(1) << a.shift;
    sums.units = n_sums * a.kv_heads;
    const int64_t items = product(r->batch, tile_count(a.shift, a.n_bands, 1, a.rows));
    const int64_t walk = product(items, a.units), single = product(items, sums.units);
    const int64_t sum = product(r->batch, tile_count(a.fine, a.n_bands, 1, a.rows), sums.units);
    // four elements of a state at once where both kinds of states are aligned for it
    const bool quads = a.dim % 2 == 0 && !misaligned(a.state, 16) && !misaligned(a.job[0].part, 16) && !misaligned(a.job[1].part, 16);
    const int64_t part = quads ? decay_scan_part<4>() : decay_scan_part<1>();
    const int64_t parts = (static_cast<int64_t>(a.dim) * a.dim + part - 1) / part;
    const int64_t scan = product(r->batch, r->n_bands, sums.units, parts);
    CHECK_TRY(check_grid(walk));
    CHECK_TRY(check_grid(std::max(single, several ? sum : 0)));
    if (several && scan == INT64_MAX) return set_err(NSGCQT_EUNSUPPORTED, "more workgroups than 64 bits count");
    return by_decay_shape(dtype, a.dim, wide, [&](auto t, auto dp, auto w) -> int {
        using T = decltype(t);
        constexpr int DP = decltype(dp)::value;
        constexpr bool kWide = decltype(w)::value;
        const dim3 block(2 * DP);
        if (several) {
            LAUNCH_TRY(k_decay_sum<T, DP, kWide>, dim3(static_cast<unsigned>(sum)), block, 0, st, sums);
            for (; sums.first_block < scan; sums.first_block += kMaxGrid)
                LAUNCH_TRY(quads ? k_decay_scan<4> : k_decay_scan<1>, dim3(static_cast<unsigned>(std::min(scan - sums.first_block, kMaxGrid))),
                           dim3(256), 0, st, sums);
        }
        LAUNCH_TRY(k_decay<T, DP, kWide>, dim3(static_cast<unsigned>(walk)), block, 0, st, a);
        if (a.state) {
            sums.single = true;
            LAUNCH_TRY(k_decay_sum<T, DP, kWide>, dim3(static_cast<unsigned>(single)), block, 0, st, sums);
        }
        return NSGCQT_OK;
    });
}

// The kernels go by strides from a tile's last token too: a row's stride that
// was not checked, of rows of one token, is not used.
View row_view(const nsgcqt_view* v, const DecayArgs& a) {
    View w = view_of(v);
    if (a.rows == 1) w.row = a.dim;
    return w;
}

DecayJob job_of(const nsgcqt_view* a, const nsgcqt_view* b, const nsgcqt_view* c, const nsgcqt_view* out, float* part,
                const DecayArgs& args, int64_t heads, bool reverse, bool turned) {
    const int group = static_cast<int>(heads / args.kv_heads);
    DecayJob j{};
    j.a = row_view(a, args);
    j.b = row_view(b, args);
    j.c = row_view(c, args);
    if (out) j.out = row_view(out, args);
    j.part = part;
    j.reverse = reverse;
    j.turned = turned;
    j.keep_result = reverse;   // keys and values are the results then
    j.heads = reverse ? args.kv_heads : static_cast<int>(heads);
    j.per = reverse ? 1 : group;
    j.many = reverse ? group : 1;
    return j;
}

}  // namespace

extern "C" {

int64_t nsgcqt_decay_attention_workspace(const nsgcqt_rows* r, const nsgcqt_decay_shape* s, int grad) {
    CHECK_TRY(check_rows(r));
    CHECK_TRY(check_decay(s));
    return decay_workspace(r, s, grad != 0);
}

int nsgcqt_decay_attention(int dtype, const nsgcqt_rows* r, const nsgcqt_decay_shape* s, const nsgcqt_view* q,
                           const nsgcqt_view* k, const nsgcqt_view* v, const nsgcqt_view* o, float* state, void* ws,
                           size_t ws_bytes, void* stream) {
    CHECK_TRY(check_dtype(dtype));
    CHECK_TRY(check_rows(r));
    CHECK_TRY(check_decay(s));
    bool wide = true;
    CHECK_TRY(check_view(q, "q", dtype, r->batch, r->rows, s->n_heads, s->head_dim, wide));
    CHECK_TRY(check_view(k, "k", dtype, r->batch, r->rows, s->n_kv_heads, s->head_dim, wide));
    CHECK_TRY(check_view(v, "v", dtype, r->batch, r->rows, s->n_kv_heads, s->head_dim, wide));
    CHECK_TRY(check_view(o, "o", dtype, r->batch, r->rows, s->n_heads, s->head_dim, wide));
    CHECK_TRY(check_state(state));
    if (r->batch == 0 || r->rows == 0) return NSGCQT_OK;
    CHECK_TRY(check_log_decay(s->log_decay));
    CHECK_TRY(check_workspace(ws, ws_bytes, decay_workspace(r, s, false)));
    DecayArgs a = decay_args(r, s, false);
    a.state = state;
    a.job[0] = job_of(q, k, v, o, static_cast<float*>(ws), a, s->n_heads, false, false);
    DecayArgs sums = a;
    sums.job[0].heads = a.kv_heads;
    sums.job[0].per = 1;
    return run_decay(dtype, r, a, sums, 1, wide, static_cast<hipStream_t>(stream));
}

int nsgcqt_decay_attention_grad(int dtype, const nsgcqt_rows* r, const nsgcqt_decay_shape* s, const nsgcqt_view* q,
                                const nsgcqt_view* k, const nsgcqt_view* v, const nsgcqt_view* d_o,
                                const nsgcqt_view* dq, const nsgcqt_view* dk, const nsgcqt_view* dv, void* ws,
                                size_t ws_bytes, void* stream) {
    CHECK_TRY(check_dtype(dtype));
    CHECK_TRY(check_rows(r));
    CHECK_TRY(check_decay(s));
    bool wide = true;
    const struct { const nsgcqt_view* v; const char* name; int64_t heads; } views[] = {
        {q, "q", s->n_heads}, {k, "k", s->n_kv_heads}, {v, "v", s->n_kv_heads}, {d_o, "d_o", s->n_heads},
        {dq, "dq", s->n_heads}, {dk, "dk", s->n_kv_heads}, {dv, "dv", s->n_kv_heads}};
    for (const auto& t : views)
        CHECK_TRY(check_view(t.v, t.name, dtype, r->batch, r->rows, t.heads, s->head_dim, wide));
    if (r->batch == 0 || r->rows == 0) return NSGCQT_OK;
    CHECK_TRY(check_log_decay(s->log_decay));
    const int64_t need = decay_workspace(r, s, true);
    CHECK_TRY(check_workspace(ws, ws_bytes, need));
    DecayArgs a = decay_args(r, s, true);
    float* before = static_cast<float*>(ws);   // states of what came before, k v^T, and of what follows, q do^T
    float* after = need ? before + need / 8 : before;
    a.job[0] = job_of(d_o, v, k, dq, before, a, s->n_heads, false, true);
    a.job[1] = job_of(v, d_o, q, dk, after, a, s->n_heads, true, true);
    a.job[2] = job_of(k, q, d_o, dv, after, a, s->n_heads, true, false);
    DecayArgs sums = a;
    sums.job[0] = job_of(q, k, v, nullptr, before, a, s->n_heads, false, false);
    sums.job[0].heads = a.kv_heads;
    sums.job[0].per = 1;
    sums.job[1] = job_of(k, q, d_o, nullptr, after, a, s->n_heads, true, false);
    return run_decay(dtype, r, a, sums, 2, wide, static_cast<hipStream_t>(stream));
}

int nsgcqt_decay_step(int dtype, int64_t n_streams, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim, double scale,
                      const nsgcqt_view* q, const nsgcqt_view* k, const nsgcqt_view* v, const nsgcqt_view* o,
                      float* state, const int64_t* pos, const float* log_decay, void* stream) {
    CHECK_TRY(check_dtype(dtype));
    if (n_streams < 0) return set_err(NSGCQT_EINVAL, "n_streams is negative");
    const nsgcqt_decay_shape s{n_heads, n_kv_heads, head_dim, scale, log_decay, nullptr, 0};
    CHECK_TRY(check_decay(&s));
    bool wide = true;
    CHECK_TRY(check_view(q, "q", dtype, n_streams, 1, n_heads, head_dim, wide));
    CHECK_TRY(check_view(k, "k", dtype, n_streams, 1, n_kv_heads, head_dim, wide));
    CHECK_TRY(check_view(v, "v", dtype, n_streams, 1, n_kv_heads, head_dim, wide));
    CHECK_TRY(check_view(o, "o", dtype, n_streams, 1, n_heads, head_dim, wide));
    if (n_streams == 0) return NSGCQT_OK;
    CHECK_TRY(check_log_decay(log_decay));
    if (!state) return set_err(NSGCQT_EINVAL, "state is NULL");
    CHECK_TRY(check_state(state));
    if (!pos || misaligned(pos, 8)) return set_err(NSGCQT_EINVAL, "pos is NULL or not aligned to 8 bytes");
    const int64_t blocks = product(n_streams, n_kv_heads);
    CHECK_TRY(check_grid(blocks));
    DecayStepArgs a{};
    a.q = view_of(q);
    a.k = view_of(k);
    a.v = view_of(v);
    a.o = view_of(o);
    a.state = state;
    a.pos = pos;
    a.log_decay = log_decay;
    a.heads = static_cast<int>(n_heads);
    a.kv_heads = static_cast<int>(n_kv_heads);
    a.dim = static_cast<int>(head_dim);
    a.group = a.heads / a.kv_heads;
    a.scale = static_cast<float>(scale);
    const bool quads = head_dim % 4 == 0 && !misaligned(state, 16);
    return by_type(dtype, [&](auto t) -> int {
        using T = decltype(t);
        auto with = [&](auto dp) -> int {
            constexpr int DP = decltype(dp)::value;
            const dim3 grid(static_cast<unsigned>(blocks)), block(256);
            const hipStream_t st = static_cast<hipStream_t>(stream);
            if (quads)
                LAUNCH_TRY((k_decay_step<T, DP, 4>), grid, block, 0, st, a);
            else
                LAUNCH_TRY((k_decay_step<T, DP, 1>), grid, block, 0, st, a);
            return NSGCQT_OK;
        };
        if (head_dim <= 32) return with(std::integral_constant<int, 32>());
        if (head_dim <= 64) return with(std::integral_constant<int, 64>());
        return with(std::integral_constant<int, 128>());
    });
}

}  // extern "C"
