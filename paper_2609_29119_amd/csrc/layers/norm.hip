// C entries of the group norm on ragged rows.
#include <algorithm>

#include "checks.hpp"
#include "norm.hpp"

using namespace nsl;

namespace {

int check_norm(int dtype, const nsgcqt_rows* r, const nsgcqt_norm_shape* s) {
    CHECK_TRY(check_dtype(dtype));
    CHECK_TRY(check_rows(r));
    if (!s) return set_err(NSGCQT_EINVAL, "shape is NULL");
    if (s->groups < 1 || s->channels < 0 || s->channels % s->groups)
        return set_err(NSGCQT_EINVAL, "groups must divide channels, and be at least 1");
    if (!(s->eps >= 1e-30 && s->eps <= 1e30)) return set_err(NSGCQT_EINVAL, "eps must lie between 1e-30 and 1e30");
    if (s->act < NSGCQT_ACT_NONE || s->act > NSGCQT_ACT_SIGMOID)
        return set_err(NSGCQT_EINVAL, "unknown activation " + std::to_string(s->act));
    if (s->w_band < 0 || s->b_band < 0) return set_err(NSGCQT_EINVAL, "a stride of w or b is negative");
    if (misaligned(s->w, elem_bytes(dtype)) || misaligned(s->b, elem_bytes(dtype)))
        return set_err(NSGCQT_EINVAL, "w or b is not aligned to its element");
    if (s->channels > kNormChannels || s->groups > kNormGroups)
        return set_err(NSGCQT_EUNSUPPORTED, "more than 4,096 channels or 1,024 groups");
    return NSGCQT_OK;
}

void set_threads(NormArgs& a, int threads) {
    a.octets = (a.channels + 7) / 8;
    a.threads = a.octets > 256 ? kNormThreads : threads;   // (of four waves three workgroups fit a compute unit, of eight one)
    a.together = a.threads / a.octets;
}
size_t norm_lds(const NormArgs& a) { return sizeof(double) * (8 * a.octets * a.together + 2 * a.groups); }

// Tokens of a chunk: what a workgroup's registers hold, `held` octets a thread
// (32 KB a workgroup of 256); and of a part, up to 8 chunks, but not so many that
// fewer than 1024 workgroups are left. A workgroup is one wave where the mean
// band is at most an eighth of what a wave holds: more bands are then on their
// way at once. 256 bands of 64 signals, 64 channels in bfloat16, of 8 tokens at the
// mean: 62 us, and 117 with four waves; with gradients, of 4: 165 and 213. With 16
// signals and bands twice as long, more of which take parts: 158 and 92.
void set_chunk(NormArgs& a, int held) {
    set_threads(a, 256);
    const int64_t wave = a.octets <= 64 ? 64 / a.octets * held : 0;   // tokens
    if (8 * static_cast<int64_t>(a.rows) <= wave * a.n_bands) set_threads(a, 64);
    a.shift = 0;
    while ((2 << a.shift) <= a.together * held) ++a.shift;
    a.part_shift = a.shift + 3;
    while (a.part_shift > a.shift && product(static_cast<int64_t>(a.batch), static_cast<int64_t>(a.rows >> a.part_shift)) < 1024) --a.part_shift;
    a.zeros = static_cast<int>(std::min<int64_t>(64, (static_cast<int64_t>(a.rows) + 1023) >> 10));
    a.parts = static_cast<unsigned>(tile_count(a.part_shift, a.n_bands, 1, a.rows));
    a.octet_groups = a.cg % 8 == 0;
}
bool has_parts(const NormArgs& a) { return a.rows > 1 << a.shift; }

// Whether each band of one chunk and each part leaves what it adds to dw and
// db: where these have 16 tokens or more at the mean, that is little beside the data.
bool chunks_sum(const NormArgs& a) { return a.rows >= 16 * static_cast<int64_t>(a.n_bands + 1); }

// Rows of an item of the weights' gradient, 64 to 4096: the most that leave 1024
// items; but no more than 32 a thread, which adds them up one after another in 32
// bits (n equal terms are then off by up to n 2^-25 of their sum).
int weight_shift_of(const NormArgs& a) {
    NormArgs w = a;
    set_threads(w, 256);
    int shift = 12;
    while ((shift > 6 && product(static_cast<int64_t>(a.batch), static_cast<int64_t>(a.rows)) >> shift < 1024) || 1 << shift > 32 * w.together) --shift;
    return shift;
}

NormArgs norm_args(const nsgcqt_rows* r, const nsgcqt_norm_shape* s) {
    NormArgs a{};
    a.w = s->w;
    a.b = s->b;
    a.w_band = s->w_band;
    a.b_band = s->b_band;
    a.off = r->offsets;
    a.rows = static_cast<int>(r->rows);
    a.n_bands = static_cast<int>(r->n_bands);
    a.batch = static_cast<int>(r->batch);
    a.channels = static_cast<int>(s->channels);
    a.groups = static_cast<int>(s->groups);
    a.cg = a.channels / a.groups;
    a.act = s->act;
    a.eps = s->eps;
    return a;
}

int held_of(int dtype, bool grad) { return (dtype == NSGCQT_F32 ? norm_held<float>() : norm_held<__bf16>()) / (grad ? 2 : 1); }

// Bytes of the workspace, whose parts begin at 16-byte boundaries: chunks'
// statistics, then the weights' partial sums.
struct NormSpace { int64_t part, sums; };   // (sums: without gradient, the statistics, for a call that does not ask for them)
NormSpace norm_space(int dtype, const nsgcqt_rows* r, const nsgcqt_norm_shape* s, bool grad, bool weights) {
    NormArgs a = norm_args(r, s);
    if (a.channels == 0) return {0, 0};
    set_chunk(a, held_of(dtype, grad));
    NormSpace n{0, 0};
    if (has_parts(a)) n.part = product(16, r->batch, static_cast<int64_t>(a.parts), a.groups);
    if (has_parts(a) && !grad) n.sums = product(16, r->batch, r->n_bands, a.groups);
    if (grad && weights)
        n.sums = product(8, chunks_sum(a) ? product(r->batch, r->n_bands + static_cast<int64_t>(a.parts))
                                          : tile_count(weight_shift_of(a), r->n_bands, r->batch, r->rows), a.channels);
    return n;
}
int64_t norm_bytes(const NormSpace& n) {
    int64_t all;
    return workspace_of(__builtin_add_overflow(n.part, n.sums, &all) ? INT64_MAX : all);
}

int check_space(const void* ws, size_t have, int64_t need) {
    if (need < 0) return static_cast<int>(need);
    if (static_cast<int64_t>(have) < need)
        return set_err(NSGCQT_EWORKSPACE, "workspace of " + std::to_string(have) + " bytes, " + std::to_string(need) +
                                              " required");
    if (need > 0 && (!ws || misaligned(ws, 16)))
        return set_err(NSGCQT_EINVAL, "workspace is NULL or not aligned to 16 bytes");
    return NSGCQT_OK;
}

// A kernel's workgroups, `each` of every signal, in launches of whole signals.
constexpr int64_t kMaxBlocks = int64_t(1) << 34;
int check_signals(const NormArgs& a, int64_t each) {
    CHECK_TRY(check_grid(each, a.threads));
    if (product(static_cast<int64_t>(a.batch), each) > kMaxBlocks) return set_err(NSGCQT_EUNSUPPORTED, "more than 2^34 workgroups");
    return NSGCQT_OK;
}
template <class K> int launch_signals(K kernel, NormArgs a, int64_t each, size_t lds, hipStream_t st) {
    const int64_t most = 0xffffffffll / a.threads / each;   // signals a launch
    for (; a.first_signal < a.batch; a.first_signal += most)
        LAUNCH_TRY(kernel, dim3(static_cast<unsigned>(std::min(a.batch - a.first_signal, most) * each)), dim3(a.threads), lds, st, a);
    return NSGCQT_OK;
}

// And `blocks` of all signals.
template <class K, class... More> int launch_all(K kernel, NormArgs a, int64_t blocks, int threads, size_t lds, hipStream_t st, More... more) {
    const int64_t most = 0xffffffffll / threads;
    for (; a.first_block < blocks; a.first_block += most)
        LAUNCH_TRY(kernel, dim3(static_cast<unsigned>(std::min(blocks - a.first_block, most))), dim3(threads), lds, st, a, more...);
    return NSGCQT_OK;
}

// f(T(), true_type or false_type)
template <class F> int by_width_of(int dtype, bool wide, F f) {
    return by_type(dtype, [&](auto t) { return wide ? f(t, std::true_type()) : f(t, std::false_type()); });
}

}  // namespace

extern "C" {

int64_t nsgcqt_band_norm_workspace(int dtype, const nsgcqt_rows* r, const nsgcqt_norm_shape* s, int grad, int weights) {
    CHECK_TRY(check_norm(dtype, r, s));
    return norm_bytes(norm_space(dtype, r, s, grad != 0, weights != 0));
}

int nsgcqt_band_norm(int dtype, const nsgcqt_rows* r, const nsgcqt_norm_shape* s, const nsgcqt_view* x,
                     const nsgcqt_view* y, double* stats, void* ws, size_t ws_bytes, void* stream) {
    CHECK_TRY(check_norm(dtype, r, s));
    bool wide = true;
    CHECK_TRY(check_view(x, "x", dtype, r->batch, r->rows, 1, s->channels, wide));
    CHECK_TRY(check_view(y, "y", dtype, r->batch, r->rows, 1, s->channels, wide));
    if (r->batch == 0 || r->rows == 0 || s->channels == 0) return NSGCQT_OK;
    if (misaligned(stats, 16)) return set_err(NSGCQT_EINVAL, "stats is not aligned to 16 bytes");
    const NormSpace space = norm_space(dtype, r, s, false, false);
    CHECK_TRY(check_space(ws, ws_bytes, norm_bytes(space)));
    NormArgs a = norm_args(r, s);
    set_chunk(a, held_of(dtype, false));
    a.x = view_of(x);
    a.y = view_of(y);
    a.part = static_cast<double2*>(ws);
    a.stats = stats ? reinterpret_cast<double2*>(stats)
                    : space.part ? reinterpret_cast<double2*>(static_cast<char*>(ws) + space.part) : nullptr;
    const int64_t blocks = r->n_bands + a.zeros;
    CHECK_TRY(check_signals(a, blocks));
    if (space.part) CHECK_TRY(check_signals(a, a.parts));
    const int64_t groups = product(r->batch, r->n_bands, a.groups);
    if (groups == INT64_MAX) return set_err(NSGCQT_EUNSUPPORTED, "more groups than 64 bits count");
    const size_t lds = norm_lds(a);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return by_width_of(dtype, wide, [&](auto t, auto w) -> int {
        using T = decltype(t);
        constexpr bool kWide = decltype(w)::value;
        CHECK_TRY(launch_signals(k_norm<T, kWide>, a, blocks, lds, st));
        if (space.part) {
            CHECK_TRY(launch_signals(k_norm_sum<T, kWide>, a, a.parts, lds, st));
            CHECK_TRY(launch_all(k_norm_join<T, false>, a, (groups + 255) / 256, 256, 0, st));
            CHECK_TRY(launch_signals(k_norm_apply<T, kWide>, a, a.parts, 0, st));
        }
        return NSGCQT_OK;
    });
}

int nsgcqt_band_norm_grad(int dtype, const nsgcqt_rows* r, const nsgcqt_norm_shape* s, const nsgcqt_view* x,
                          const double* stats, const nsgcqt_view* dy, const nsgcqt_view* dx, void* dw, void* db,
                          void* ws, size_t ws_bytes, void* stream) {
    CHECK_TRY(check_norm(dtype, r, s));
    bool wide = true;
    CHECK_TRY(check_view(x, "x", dtype, r->batch, r->rows, 1, s->channels, wide));
    CHECK_TRY(check_view(dy, "dy", dtype, r->batch, r->rows, 1, s->channels, wide));
    if (dx) CHECK_TRY(check_view(dx, "dx", dtype, r->batch, r->rows, 1, s->channels, wide));
    if (misaligned(dw, elem_bytes(dtype)) || misaligned(db, elem_bytes(dtype)))
        return set_err(NSGCQT_EINVAL, "dw or db is not aligned to its element");
    const bool weights = dw || db;
    if (s->channels == 0 || (!dx && !weights)) return NSGCQT_OK;
    const bool rows = r->batch > 0 && r->rows > 0;
    if (rows && r->n_bands > 0 && (!stats || misaligned(stats, 16)))
        return set_err(NSGCQT_EINVAL, "stats is NULL or not aligned to 16 bytes");
    const NormSpace space = norm_space(dtype, r, s, true, weights);
    CHECK_TRY(check_space(ws, ws_bytes, norm_bytes(space)));
    NormArgs a = norm_args(r, s);
    set_chunk(a, held_of(dtype, true));
    a.weight_shift = weight_shift_of(a);
    a.x = view_of(x);
    a.dy = view_of(dy);
    if (dx) a.y = view_of(dx);
    a.stats = reinterpret_cast<double2*>(const_cast<double*>(stats));
    a.part = static_cast<double2*>(ws);
    float* sums = weights ? reinterpret_cast<float*>(static_cast<char*>(ws) + space.part) : nullptr;
    const bool by_chunk = weights && chunks_sum(a);
    if (by_chunk) a.sums = sums;
    a.dw = dw;
    a.db = db;
    const int64_t blocks = r->n_bands + a.zeros;
    const int64_t items = tile_count(a.weight_shift, r->n_bands, r->batch, r->rows);
    const int64_t groups = product(r->batch, r->n_bands, a.groups);
    const bool bands = (dx || by_chunk) && rows;
    if (bands) CHECK_TRY(check_signals(a, blocks));
    if (bands && space.part) CHECK_TRY(check_signals(a, a.parts));
    if (groups == INT64_MAX) return set_err(NSGCQT_EUNSUPPORTED, "more groups than 64 bits count");
    const size_t lds = norm_lds(a);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return by_width_of(dtype, wide, [&](auto t, auto w) -> int {
        using T = decltype(t);
        constexpr bool kWide = decltype(w)::value;
        if (bands) {
            CHECK_TRY(launch_signals(k_norm_grad<T, kWide>, a, blocks, lds, st));
            if (space.part) {
                CHECK_TRY(launch_signals(k_norm_grad_sum<T, kWide>, a, a.parts, lds, st));
                if (dx) {
                    CHECK_TRY(launch_all(k_norm_join<T, true>, a, (groups + 255) / 256, 256, 0, st));
                    CHECK_TRY(launch_signals(k_norm_grad_apply<T, kWide>, a, a.parts, 0, st));
                }
            }
        }
        if (weights) {
            a.sums = sums;
            if (rows && !by_chunk) {
                set_threads(a, 256);
                CHECK_TRY(launch_all(k_norm_weight<T, kWide>, a, items, a.threads, norm_lds(a), st));
            }
            // 16 waves for 64 channels of a band where 64 or more were left for each at the mean and the workgroups, 1024
            // threads each, are all there at once (64 signals: 200 bands of 64 channels 4.8 us, and 6.8 with a thread a
            // channel; 500 bands of 128 12.2 and 9.3, 10,000 of 8 88 and 11).
            const int64_t left = by_chunk ? product(static_cast<int64_t>(a.parts), r->batch) : items;
            const int64_t shared = r->n_bands * ((s->channels + 63) / 64);
            if (left >= 64 * r->n_bands && shared <= 512)
                CHECK_TRY(launch_all(k_norm_weight_join<T, 16>, a, shared, 1024, 0, st, by_chunk));
            else
                CHECK_TRY(launch_all(k_norm_weight_join<T, 1>, a, (r->n_bands * s->channels + 255) / 256, 256, 0, st, by_chunk));
        }
        return NSGCQT_OK;
    });
}

}  // extern "C"
