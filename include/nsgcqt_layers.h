/*
 * nsgcqt_layers.h - C ABI of the layers on the band layout (libnsgcqt.so).
 *
 * A network behind the constant-Q transform works on rows of C tokens (one
 * for each coefficient), cut into bands: band g holds the tokens
 * [offsets[g], offsets[g + 1]) of every signal's row. The calls here take
 * such ragged rows as they are, without padding a band to the longest:
 *
 *   nsgcqt_band_linear*     a matrix of its own for each band, with gradients
 *   nsgcqt_rotary           rotary positions over one to four axes
 *   nsgcqt_band_attention*  attention along each band with a sliding window
 *                           and first tokens that stay visible (sinks)
 *   nsgcqt_attention_step   the same attention for one new token of each of
 *                           many streams, over a ring cache; _cache_fill
 *   nsgcqt_decay_attention* linear attention along each band with a decay for
 *                           each head, from and into a state
 *   nsgcqt_decay_step       the same for one new token of each of many streams
 *   nsgcqt_band_norm*       group norm of each band with an activation
 *   nsgcqt_band_gated*      two projections of each band, an activation and
 *                           their product
 *
 * Conventions
 *   - Data are float32, float16 or bfloat16 (nsgcqt_dtype), one type a call.
 *     Products, sums, softmax statistics and angles are held in 32 bits or
 *     more; each result is rounded once. In 16-bit attention the
 *     probabilities and their gradients enter the matrix products as two
 *     numbers of the data's type, the rounded one and what the rounding
 *     left; an infinity in v, k, q or d_o may therefore come out as NaN.
 *   - A tensor is an nsgcqt_view: a device pointer and the strides, in
 *     elements, of its batch, row (token) and head axes; the last axis is
 *     contiguous. Pointers are aligned to their element. 16-byte aligned
 *     pointers and strides with widths that are multiples of 8 take the wide
 *     loads.
 *   - offsets: n_bands + 1 ascending int64 on the device. They are read by
 *     the kernels only: bands are cut to [0, rows), tokens that no band
 *     holds get zeros in every output, and offsets that do not ascend give
 *     unspecified values but no access out of range.
 *   - rows, widths and counts may be zero; then nothing is launched for
 *     them, except that gradients of weights are written as zeros.
 *   - Calls only enqueue work on `stream` (a hipStream_t or NULL), allocate
 *     nothing and may be captured into a HIP graph. Workspaces are the
 *     caller's; nothing in them needs to start at zero and nothing is kept
 *     in them between calls. Results do not vary from run to run: no
 *     atomics, every sum has a fixed order.
 *   - Errors as in nsgcqt.h: an nsgcqt_status, its text from
 *     nsgcqt_last_error(). EINVAL for null or misaligned pointers, negative
 *     sizes, an unknown type; EUNSUPPORTED for head_dim above 128 and sizes
 *     beyond the stated limits; EWORKSPACE for a workspace below its size.
 *   - Limits: below 2^30 rows, 2^24 bands, 2^30 signals, 2^40 tokens in all,
 *     widths of 65,536, 65,536 heads; and 16,777,215 workgroups a launch,
 *     which comes first for many signals or short bands: with tiles of R
 *     tokens a signal has rows / R + n_bands + 2 of them (R = 128 for the
 *     products and the key gradient, which counts in kv heads; 128 / s with
 *     s = 4, 2 or 1 heads a workgroup, the largest that divides n_heads /
 *     n_kv_heads, for the attention). The step takes a workgroup for each
 *     stream, kv head and 32 query heads of it, and one for each stream and head.
 *     The decayed attention takes one for each segment (64 to 4,096 tokens)
 *     of each band of each signal and head, its step for each stream and kv
 *     head, the gated product for 128 tokens or more of a band and 64 outputs
 *     (256 and 128 for the weights' gradient, 8,388,607 of them a launch). The
 *     norm takes one for each band (and part of a long one) of each signal, in
 *     as many launches of whole signals as that needs, up to 2^34 in all.
 */
#ifndef NSGCQT_LAYERS_H
#define NSGCQT_LAYERS_H

#include "nsgcqt.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { NSGCQT_F32 = 0, NSGCQT_F16 = 1, NSGCQT_BF16 = 2 } nsgcqt_dtype;

typedef enum { NSGCQT_POS_F32 = 0, NSGCQT_POS_F64 = 1, NSGCQT_POS_I64 = 2 } nsgcqt_pos_type;

/* Element [b][r][h][d] of a tensor is data[b batch + r row + h head + d]. */
typedef struct {
    void* data;
    int64_t batch, row, head;   /* strides in elements */
} nsgcqt_view;

/* The ragged rows: every signal of `batch` has `rows` tokens, cut by offsets. */
typedef struct {
    const int64_t* offsets;   /* device, n_bands + 1 */
    int64_t n_bands;
    int64_t batch;
    int64_t rows;             /* C, below 2^30 */
} nsgcqt_rows;

/* y[b][c][:] = W[g] x[b][c][:] + bias[g], g the band of token c.
 * x: [batch][rows][n_in], w: [n_bands][n_out][n_in] contiguous, bias:
 * [n_bands][n_out] contiguous or NULL, y: [batch][rows][n_out]. Views'
 * head strides are not read. n_in and n_out at most 65,536. */
int nsgcqt_band_linear(int dtype, const nsgcqt_rows* r, const nsgcqt_view* x, const void* w, const void* bias,
                       const nsgcqt_view* y, int64_t n_in, int64_t n_out, void* stream);

/* dx[b][c][:] = W[g]^T dy[b][c][:]. */
int nsgcqt_band_linear_grad_input(int dtype, const nsgcqt_rows* r, const nsgcqt_view* dy, const void* w,
                                  const nsgcqt_view* dx, int64_t n_in, int64_t n_out, void* stream);

/* dw[g] = sum over the band's tokens of every signal of dy x^T, and, with db
 * not NULL, db[g] = the sum of dy; laid out as w and bias. */
int nsgcqt_band_linear_grad_weight(int dtype, const nsgcqt_rows* r, const nsgcqt_view* x, const nsgcqt_view* dy,
                                   void* dw, void* db, int64_t n_in, int64_t n_out, void* ws, size_t ws_bytes,
                                   void* stream);

/* Workspace bytes of nsgcqt_band_linear_grad_weight, or a negative status. */
int64_t nsgcqt_band_linear_workspace(int64_t n_bands, int64_t batch, int64_t rows, int64_t n_in, int64_t n_out);

/* Rotary positions. The first 2 P of a head's head_dim values form P pairs,
 * P the sum of sections[0 .. n_axes-1] (1 <= n_axes <= 4, 2 P <= head_dim):
 * values (p, p + P), or (2p, 2p + 1) with interleaved != 0. Pair p belongs
 * to the axis whose section it falls into and is turned by the angle
 * positions[axis] * freqs[p] (by its negative with inverse != 0, which is
 * the gradient); values past 2 P are copied. The angle is formed and reduced
 * in 64 bits.
 * q, k and their outputs: [batch][rows][heads][head_dim]; either q (with
 * n_q_heads) or k (with n_k_heads) may be left out with a NULL view and 0
 * heads. Outputs may be the inputs themselves, and must not overlap them
 * otherwise. positions: element [axis][b][row] at
 * positions[axis pos_axis + b pos_batch + row] of type pos_type (strides in
 * elements; pos_batch 0 shares them among signals). freqs: [P] float32.
 * sections is read on the host. */
int nsgcqt_rotary(int dtype, const nsgcqt_view* q, const nsgcqt_view* q_out, int64_t n_q_heads,
                  const nsgcqt_view* k, const nsgcqt_view* k_out, int64_t n_k_heads, int64_t batch, int64_t rows,
                  int64_t head_dim, const void* positions, int pos_type, int64_t pos_axis, int64_t pos_batch,
                  const float* freqs, const int32_t* sections, int n_axes, int interleaved, int inverse,
                  void* stream);

/* Shape of an attention call. Token i of a band sees token j of the same
 * band and signal when keep[b][j] is not 0 (keep NULL: always),
 * j <= i + right, and j >= i - left or j < sinks (numbers within the band).
 * A token that sees none gets a zero row and passes no gradient. What a
 * token that is not kept holds in k and v is never used, whatever it is; an
 * infinity or NaN of a kept token may, with weight zero, reach tokens of its
 * band near it that do not see it. */
typedef struct {
    int64_t n_heads, n_kv_heads;   /* n_kv_heads divides n_heads; head h reads kv head h / (n_heads / n_kv_heads) */
    int64_t head_dim;              /* 1 .. 128 */
    int64_t left, right, sinks;    /* each >= 0; values past rows mean all */
    double scale;                  /* of the scores, > 0 */
    const uint8_t* keep;           /* device, [batch][rows] with batch stride keep_batch, or NULL */
    int64_t keep_batch;
} nsgcqt_attention_shape;

/* o = attention(q, k, v), and for the gradient stats [batch][n_heads][rows]
 * float32 (the base-2 logarithm of each row's softmax sum; NULL: not
 * written). q, o: [batch][rows][n_heads][head_dim]; k, v with n_kv_heads. */
int nsgcqt_band_attention(int dtype, const nsgcqt_rows* r, const nsgcqt_attention_shape* s, const nsgcqt_view* q,
                          const nsgcqt_view* k, const nsgcqt_view* v, const nsgcqt_view* o, float* stats,
                          void* stream);

/* dq, dk, dv of a loss with gradient d_o at o; o and stats as the forward call
 * wrote them. */
int nsgcqt_band_attention_grad(int dtype, const nsgcqt_rows* r, const nsgcqt_attention_shape* s,
                               const nsgcqt_view* q, const nsgcqt_view* k, const nsgcqt_view* v,
                               const nsgcqt_view* o, const float* stats, const nsgcqt_view* d_o,
                               const nsgcqt_view* dq, const nsgcqt_view* dk, const nsgcqt_view* dv, void* ws,
                               size_t ws_bytes, void* stream);

/* Workspace bytes of nsgcqt_band_attention_grad, or a negative status. */
int64_t nsgcqt_band_attention_workspace(const nsgcqt_rows* r, const nsgcqt_attention_shape* s);

/* One new token of each of n_streams streams. The ring caches
 * k_cache, v_cache: [n_streams][n_kv_heads][sinks + window][head_dim]
 * contiguous hold token t of a stream at slot t for t < sinks and at
 * sinks + (t - sinks) mod window after. pos[s] (device int64) numbers the new
 * token of stream s: its k and v are written to its slot, and its q attends
 * over all tokens that the cache then holds, itself among them. A negative
 * pos leaves the stream's cache alone and gives a zero row.
 * q, o: [n_streams][n_heads][head_dim], k, v: with n_kv_heads: views whose
 * batch stride goes from stream to stream (row strides are not read).
 * sinks >= 0, window >= 1, sinks + window below 2^30. */
int nsgcqt_attention_step(int dtype, int64_t n_streams, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim,
                          int64_t window, int64_t sinks, double scale, const nsgcqt_view* q, const nsgcqt_view* k,
                          const nsgcqt_view* v, const nsgcqt_view* o, void* k_cache, void* v_cache,
                          const int64_t* pos, void* ws, size_t ws_bytes, void* stream);

/* Workspace bytes of nsgcqt_attention_step, or a negative status. */
int64_t nsgcqt_attention_step_workspace(int64_t n_streams, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim,
                                        int64_t window, int64_t sinks);

/* Fills ring caches from whole bands: stream b n_bands + g holds the tokens
 * of band g of signal b, numbered from 0; what its cache would hold after
 * steps over all of them is copied, slots without a token are left alone.
 * k, v: [batch][rows][n_kv_heads][head_dim]. At most 65,535 streams a call. */
int nsgcqt_cache_fill(int dtype, const nsgcqt_rows* r, int64_t n_kv_heads, int64_t head_dim, int64_t window,
                      int64_t sinks, const nsgcqt_view* k, const nsgcqt_view* v, void* k_cache, void* v_cache,
                      void* stream);

/* Shape of a decayed linear attention. Head h of q and o reads key head
 * n = h / (n_heads / n_kv_heads) of k and v, whose decay is
 * exp(log_decay[n]); with keep not NULL, tokens with keep[b][j] = 0 add
 * nothing (what k and v hold there is never used), but count as distance. */
typedef struct {
    int64_t n_heads, n_kv_heads;   /* n_kv_heads divides n_heads */
    int64_t head_dim;              /* 1 .. 128 */
    double scale;                  /* of the results, finite */
    const float* log_decay;        /* device, [n_kv_heads]; a decay of at most 1, log_decay <= 0, is meant */
    const uint8_t* keep;           /* device, [batch][rows] with batch stride keep_batch, or NULL */
    int64_t keep_batch;
} nsgcqt_decay_shape;

/* o_t = scale (decay^(t + 1) q_t S + sum over tokens s <= t of the band of
 * decay^(t - s) (q_t . k_s) v_s), t counted within the band. S is state
 * [batch * n_bands][n_kv_heads][head_dim][head_dim] float32, contiguous, stream
 * b n_bands + g that of band g of signal b; the call leaves in its place
 * decay^len S + sum_s decay^(len - 1 - s) k_s v_s^T (of a band without tokens:
 * S itself). state NULL: S = 0. q, o: [batch][rows][n_heads][head_dim]; k, v
 * with n_kv_heads. Sums whose terms pass 16 bits enter the products of 16-bit
 * data as two numbers of 8 bits, those of the state as three; an infinity or
 * NaN may, with weight zero, reach the 31 tokens before it, and come out as NaN. */
int nsgcqt_decay_attention(int dtype, const nsgcqt_rows* r, const nsgcqt_decay_shape* s, const nsgcqt_view* q,
                           const nsgcqt_view* k, const nsgcqt_view* v, const nsgcqt_view* o, float* state, void* ws,
                           size_t ws_bytes, void* stream);

/* dq, dk, dv of a loss with gradient d_o at o, for state NULL. */
int nsgcqt_decay_attention_grad(int dtype, const nsgcqt_rows* r, const nsgcqt_decay_shape* s, const nsgcqt_view* q,
                                const nsgcqt_view* k, const nsgcqt_view* v, const nsgcqt_view* d_o,
                                const nsgcqt_view* dq, const nsgcqt_view* dk, const nsgcqt_view* dv, void* ws,
                                size_t ws_bytes, void* stream);

/* Workspace bytes of nsgcqt_decay_attention (grad 0) or its gradient, or a negative status. */
int64_t nsgcqt_decay_attention_workspace(const nsgcqt_rows* r, const nsgcqt_decay_shape* s, int grad);

/* One new token of each of n_streams streams: S <- decay S + k v^T,
 * o = scale q S, with S in state [n_streams][n_kv_heads][head_dim][head_dim]
 * float32, contiguous. pos[s] (device int64) above 0: the stream goes on; 0: it
 * begins, what its state holds is not used; below 0: it has no token, its
 * state stays as it is and its row is zero. Views as in nsgcqt_attention_step. */
int nsgcqt_decay_step(int dtype, int64_t n_streams, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim, double scale,
                      const nsgcqt_view* q, const nsgcqt_view* k, const nsgcqt_view* v, const nsgcqt_view* o,
                      float* state, const int64_t* pos, const float* log_decay, void* stream);

/* none: z; silu: z / (1 + exp(-z)); gelu: z Phi(z), Phi the normal
 * distribution's; sigmoid: 1 / (1 + exp(-z)). At infinite z these, and their
 * derivatives, are their limits. */
typedef enum {
    NSGCQT_ACT_NONE = 0, NSGCQT_ACT_SILU = 1, NSGCQT_ACT_GELU = 2, NSGCQT_ACT_SIGMOID = 3
} nsgcqt_act;

/* Shape and parameters of a group norm. */
typedef struct {
    int64_t channels, groups;   /* groups divides channels; at most 4,096 and 1,024 */
    double eps;                 /* 1e-30 .. 1e30 */
    const void *w, *b;          /* device, element [g][c] at [g w_band + c]; NULL: ones, zeros */
    int64_t w_band, b_band;     /* strides in elements, not negative; 0 shares a row among bands */
    int act;                    /* nsgcqt_act */
} nsgcqt_norm_shape;

/* y = act(w (x - mean) / sqrt(var + eps) + b), mean and (biased) variance over
 * the channels of a group and all tokens of a band of one signal. x, y:
 * [batch][rows][channels]. stats: [batch][n_bands][groups][2] float64, 16-byte
 * aligned, receives mean and 1 / sqrt(var + eps) of bands that have tokens, for
 * the gradient; NULL: not wanted. y may be x itself. A group that holds an
 * infinity or NaN in a band has no variance: its y (and dx) are NaN there. */
int nsgcqt_band_norm(int dtype, const nsgcqt_rows* r, const nsgcqt_norm_shape* s, const nsgcqt_view* x,
                     const nsgcqt_view* y, double* stats, void* ws, size_t ws_bytes, void* stream);

/* dx, and with dw or db not NULL the gradients of w and b as
 * [n_bands][channels] contiguous (whatever their strides), of a loss with
 * gradient dy at y; stats as the forward call wrote them. dx may be NULL. */
int nsgcqt_band_norm_grad(int dtype, const nsgcqt_rows* r, const nsgcqt_norm_shape* s, const nsgcqt_view* x,
                          const double* stats, const nsgcqt_view* dy, const nsgcqt_view* dx, void* dw, void* db,
                          void* ws, size_t ws_bytes, void* stream);

/* Workspace bytes of nsgcqt_band_norm (grad 0) or its gradient (weights: with dw or db), or a negative status. */
int64_t nsgcqt_band_norm_workspace(int dtype, const nsgcqt_rows* r, const nsgcqt_norm_shape* s, int grad, int weights);

/* y[b][c][:] = act(Wa x + ba) (Wu x + bu), elementwise, with Wa, Wu = w[g][0],
 * w[g][1] and ba, bu = bias[g][0], bias[g][1], g the band of token c. x:
 * [batch][rows][n_in], w: [n_bands][2][n_out][n_in] contiguous, bias:
 * [n_bands][2][n_out] contiguous or NULL, y: [batch][rows][n_out]; act an
 * nsgcqt_act. n_in at most 65,536, n_out 32,768. */
int nsgcqt_band_gated(int dtype, const nsgcqt_rows* r, const nsgcqt_view* x, const void* w, const void* bias,
                      const nsgcqt_view* y, int64_t n_in, int64_t n_out, int act, void* stream);

/* dx, dw and db (as w and bias) of a loss with gradient dy at y. dx may be
 * NULL, and so may db, or dw and db; the workspace is for dw and db. The
 * gradients at the two projections enter the products of 16-bit data as two
 * numbers of 8 bits. */
int nsgcqt_band_gated_grad(int dtype, const nsgcqt_rows* r, const nsgcqt_view* x, const void* w, const void* bias,
                           const nsgcqt_view* dy, const nsgcqt_view* dx, void* dw, void* db, int64_t n_in,
                           int64_t n_out, int act, void* ws, size_t ws_bytes, void* stream);

/* Workspace bytes of nsgcqt_band_gated_grad, or a negative status. */
int64_t nsgcqt_band_gated_workspace(const nsgcqt_rows* r, int64_t n_in, int64_t n_out);

#ifdef __cplusplus
}
#endif

#endif /* NSGCQT_LAYERS_H */
