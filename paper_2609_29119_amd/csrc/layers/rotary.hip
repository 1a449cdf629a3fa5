// C entry of the rotary positions.
#include <algorithm>

#include "checks.hpp"
#include "rotary.hpp"

using namespace nsl;

extern "C" int nsgcqt_rotary(int dtype, const nsgcqt_view* q, const nsgcqt_view* q_out, int64_t n_q_heads,
                             const nsgcqt_view* k, const nsgcqt_view* k_out, int64_t n_k_heads, int64_t batch,
                             int64_t rows, int64_t head_dim, const void* positions, int pos_type, int64_t pos_axis,
                             int64_t pos_batch, const float* freqs, const int32_t* sections, int n_axes,
                             int interleaved, int inverse, void* stream) {
    CHECK_TRY(check_dtype(dtype));
    if (batch < 0 || rows < 0 || n_q_heads < 0 || n_k_heads < 0 || head_dim < 0)
        return set_err(NSGCQT_EINVAL, "a size is negative");
    if (batch > kMaxCount || rows > kMaxCount || batch * rows > (int64_t(1) << 40) || n_q_heads > 65536 ||
        n_k_heads > 65536 || head_dim > kMaxWidth)
        return set_err(NSGCQT_EUNSUPPORTED, "a size beyond the supported range");
    if (n_axes < 1 || n_axes > 4) return set_err(NSGCQT_EINVAL, "n_axes must be 1 to 4");
    if (!sections) return set_err(NSGCQT_EINVAL, "sections is NULL");
    RotaryArgs a{};
    int64_t pairs = 0;
    for (int x = 0; x < 4; ++x) {
        if (x < n_axes) {
            if (sections[x] < 0) return set_err(NSGCQT_EINVAL, "a section is negative");
            pairs += sections[x];
        }
        if (2 * pairs > head_dim) return set_err(NSGCQT_EINVAL, "the sections hold more than head_dim / 2 pairs");
        // the last axis has every pair that is left, so that no pair reads past the axes
        a.ends[x] = static_cast<int>(x < n_axes - 1 ? pairs : head_dim);
    }
    if (pos_type != NSGCQT_POS_F32 && pos_type != NSGCQT_POS_F64 && pos_type != NSGCQT_POS_I64)
        return set_err(NSGCQT_EINVAL, "unknown type of positions");
    if (pos_axis < 0 || pos_batch < 0) return set_err(NSGCQT_EINVAL, "a stride of the positions is negative");
    bool wide = true;
    if (n_q_heads) {
        CHECK_TRY(check_view(q, "q", dtype, batch, rows, n_q_heads, head_dim, wide));
        CHECK_TRY(check_view(q_out, "q_out", dtype, batch, rows, n_q_heads, head_dim, wide));
        a.in[0] = view_of(q);
        a.out[0] = view_of(q_out);
    }
    if (n_k_heads) {
        CHECK_TRY(check_view(k, "k", dtype, batch, rows, n_k_heads, head_dim, wide));
        CHECK_TRY(check_view(k_out, "k_out", dtype, batch, rows, n_k_heads, head_dim, wide));
        a.in[1] = view_of(k);
        a.out[1] = view_of(k_out);
    }
    if (batch == 0 || rows == 0 || n_q_heads + n_k_heads == 0 || head_dim == 0) return NSGCQT_OK;
    const size_t pb = pos_type == NSGCQT_POS_F32 ? 4 : 8;
    if (pairs && (!positions || misaligned(positions, pb)))
        return set_err(NSGCQT_EINVAL, "positions is NULL or not aligned to its element");
    if (pairs && (!freqs || misaligned(freqs, 4)))
        return set_err(NSGCQT_EINVAL, "freqs is NULL or not aligned to 4 bytes");
    a.heads[0] = static_cast<int>(n_q_heads);
    a.heads[1] = static_cast<int>(n_k_heads);
    a.positions = positions;
    a.pos_axis = pos_axis;
    a.pos_batch = pos_batch;
    a.freqs = freqs;
    a.rows = rows;
    a.tokens = batch * rows;
    a.pos_type = pos_type;
    a.dim = static_cast<int>(head_dim);
    a.pairs = static_cast<int>(pairs);
    a.interleaved = interleaved != 0;
    a.inverse = inverse != 0;
    // the most values an item can take that divide both parts of a head
    const int64_t both = pairs | (head_dim - 2 * pairs);
    const int v = both % 8 == 0 ? 8 : both % 4 == 0 ? 4 : both % 2 == 0 ? 2 : 1;
    a.chunks = static_cast<int>(pairs / v + (head_dim - 2 * pairs) / v);
    const int64_t blocks = (a.tokens * a.chunks + 255) / 256, heads = n_q_heads + n_k_heads;
    CHECK_TRY(check_grid(blocks));
    // one item for all heads where that alone fills the card (8 workgroups on
    // each of 256 compute units); fewer heads an item for few tokens
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(heads, 2048 / blocks));
    a.each = static_cast<int>((heads + parts - 1) / parts);
    const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>((heads + a.each - 1) / a.each));
    return by_type(dtype, [&](auto t) -> int {
        using T = decltype(t);
        auto go = [&](auto width) -> int {
            LAUNCH_TRY(k_rotary<T, decltype(width)::value>, grid, dim3(256), 0, static_cast<hipStream_t>(stream), a);
            return NSGCQT_OK;
        };
        switch (v) {
            case 8: return go(std::integral_constant<int, 8>());
            case 4: return go(std::integral_constant<int, 4>());
            case 2: return go(std::integral_constant<int, 2>());
            default: return go(std::integral_constant<int, 1>());
        }
    });
}
