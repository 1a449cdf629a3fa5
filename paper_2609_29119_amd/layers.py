"""Layers on the band layout: what a network needs right behind the transform.

A row of C coefficients is a ragged row of tokens: band g holds the tokens
[offsets[g], offsets[g + 1]) (`Plan.band_offsets`). The operators work on that
row as it is, in hand-written HIP kernels behind the C ABI of
include/nsgcqt_layers.h:

  band_linear      a matrix of its own for each band
  rotary           rotary positions over one to four axes (time, frequency, ...)
  band_attention   attention along each band: sliding window, first tokens
                   that stay visible (sinks), shared key heads
  attention_step   the same attention for one new token of each of many
                   streams, over a ring cache; `cache_fill` starts the caches,
                   `StreamCache` holds them
  decay_attention  linear attention along each band, whose past decays at a
                   rate of each head's own; from and into a state
  decay_step       the same for one new token of each of many streams;
                   `DecayState` holds the streams' states
  band_norm        group norm of each band, with an activation
  band_gated       two projections of each band, an activation, their product

All but the steps and fills are differentiable. Data are float32, float16 or bfloat16
CUDA tensors, one type a call; the last axis has to be contiguous, other
strides are free. Calls run on the current stream.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import struct

import torch
from torch.autograd import forward_ad

from .nsgcqt import EINVAL, NsgcqtError, _check, lib

F32, F16, BF16 = 0, 1, 2
POS_F32, POS_F64, POS_I64 = 0, 1, 2

_DTYPES = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
_ACTS = {None: 0, "silu": 1, "gelu": 2, "sigmoid": 3}
_POS = {torch.float32: POS_F32, torch.float64: POS_F64, torch.int64: POS_I64}

EXPORTS = [
    "nsgcqt_band_linear", "nsgcqt_band_linear_grad_input", "nsgcqt_band_linear_grad_weight",
    "nsgcqt_band_linear_workspace", "nsgcqt_rotary", "nsgcqt_band_attention", "nsgcqt_band_attention_grad",
    "nsgcqt_band_attention_workspace", "nsgcqt_attention_step", "nsgcqt_attention_step_workspace",
    "nsgcqt_cache_fill", "nsgcqt_decay_attention", "nsgcqt_decay_attention_grad", "nsgcqt_decay_attention_workspace",
    "nsgcqt_decay_step", "nsgcqt_band_norm", "nsgcqt_band_norm_grad", "nsgcqt_band_norm_workspace",
    "nsgcqt_band_gated", "nsgcqt_band_gated_grad", "nsgcqt_band_gated_workspace",
]


# The structs of the header, packed: a call passes their bytes.
_view = struct.Struct("=4q").pack                # nsgcqt_view: data, strides of batch, row, head
_rows = struct.Struct("=4q").pack                # nsgcqt_rows: offsets, n_bands, batch, rows
_shape = struct.Struct("=6qd2q").pack            # nsgcqt_attention_shape
_decay_shape = struct.Struct("=3qd3q").pack      # nsgcqt_decay_shape
_norm_shape = struct.Struct("=2qd4qi4x").pack    # nsgcqt_norm_shape


_fns = None


def _lib():
    """The library with the layers' signatures."""
    global _fns
    if _fns is None:
        L = lib()
        V, I, I64, D, Z = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_double, ctypes.c_size_t
        sig = {
            "nsgcqt_band_linear": [I, V, V, V, V, V, I64, I64, V],
            "nsgcqt_band_linear_grad_input": [I, V, V, V, V, I64, I64, V],
            "nsgcqt_band_linear_grad_weight": [I, V, V, V, V, V, I64, I64, V, Z, V],
            "nsgcqt_band_linear_workspace": [I64, I64, I64, I64, I64],
            "nsgcqt_rotary": [I, V, V, I64, V, V, I64, I64, I64, I64, V, I, I64, I64, V, V, I, I, I, V],
            "nsgcqt_band_attention": [I, V, V, V, V, V, V, V, V],
            "nsgcqt_band_attention_grad": [I] + [V] * 12 + [Z, V],
            "nsgcqt_band_attention_workspace": [V, V],
            "nsgcqt_attention_step": [I, I64, I64, I64, I64, I64, I64, D, V, V, V, V, V, V, V, V, Z, V],
            "nsgcqt_attention_step_workspace": [I64] * 6,
            "nsgcqt_cache_fill": [I, V, I64, I64, I64, I64, V, V, V, V, V],
            "nsgcqt_decay_attention": [I] + [V] * 8 + [Z, V],
            "nsgcqt_decay_attention_grad": [I] + [V] * 10 + [Z, V],
            "nsgcqt_decay_attention_workspace": [V, V, I],
            "nsgcqt_decay_step": [I, I64, I64, I64, I64, D] + [V] * 8,
            "nsgcqt_band_norm": [I] + [V] * 6 + [Z, V],
            "nsgcqt_band_norm_grad": [I] + [V] * 9 + [Z, V],
            "nsgcqt_band_norm_workspace": [I, V, V, I, I],
            "nsgcqt_band_gated": [I, V, V, V, V, V, I64, I64, I, V],
            "nsgcqt_band_gated_grad": [I] + [V] * 8 + [I64, I64, I, V, Z, V],
            "nsgcqt_band_gated_workspace": [V, I64, I64],
        }
        for name, args in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = I64 if name.endswith("_workspace") else I
        _fns = L
    return _fns


def _bad(msg):
    raise NsgcqtError(EINVAL, msg)


def _bytes(n):
    return _check(int(n)) if n < 0 else n


_here = contextlib.nullcontext()
_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device


def _on(t):
    """A context with t's device current."""
    return _here if t.get_device() == _current_device() else torch.cuda.device(t.device)


def _stream(t):
    """The raw handle of t's device's current stream."""
    return torch._C._cuda_getCurrentRawStream(t.get_device())


def _tensor(t, name, like=None, shape=None, dims=None):
    """Checks one tensor of a call: its device, type, shape and last stride."""
    if dims is not None and t.dim() != dims.count("["):
        raise ValueError(f"{name} has {t.dim()} axes: {dims} is expected")
    if not t.is_cuda:
        raise ValueError(f"{name} is on {t.device}: a cuda tensor is expected")
    if like is None:
        if t.dtype not in _DTYPES:
            raise ValueError(f"{name} is {t.dtype}: float32, float16 or bfloat16 is expected")
    elif t.dtype != like.dtype or t.get_device() != like.get_device():
        raise ValueError(f"{name} is {t.dtype} on {t.device}: {like.dtype} on {like.device} is expected")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}: {tuple(shape)} is expected")
    if t.shape[-1] > 1:
        if t.stride(-1) != 1:
            raise ValueError(f"the last axis of {name} has to be contiguous")
    elif t.is_neg():   # (of the imaginary part of a conjugate: its other strides are even, never 1)
        raise ValueError(f"{name} is a lazy negative: call resolve_neg()")
    return t


def _offsets(offsets, like):
    if offsets.dtype != torch.int64 or offsets.dim() != 1 or offsets.numel() < 1 or not offsets.is_contiguous():
        raise ValueError("offsets has to be a contiguous int64 vector of n_bands + 1 values")
    if offsets.get_device() != like.get_device():
        raise ValueError(f"offsets is on {offsets.device}: {like.device} is expected")
    return offsets


def _ragged(offsets, batch, rows):
    return _rows(offsets.data_ptr(), offsets.shape[0] - 1, batch, rows)


def _view3(t):
    s = t.stride()
    return _view(t.data_ptr(), s[0], s[1], 0)


def _view4(t):
    s = t.stride()
    return _view(t.data_ptr(), s[0], s[1], s[2])


def _view_step(t):
    s = t.stride()
    return _view(t.data_ptr(), s[0], 0, s[1])


def _scale(scale, dim):
    """The scores' factor as given, or D^-1/2 (the call refuses a width of 0)."""
    return float(scale) if scale is not None else dim ** -0.5 if dim else 1.0


def _trains(*tensors):
    """Whether a result has to carry a derivative: an input requires grad, or
    has a forward-mode tangent (which no operator here has a rule for: the
    autograd functions then raise NotImplementedError)."""
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                return True
    if getattr(forward_ad, "_current_level", 0) >= 0:   # (-1: no forward-mode level is open)
        for t in tensors:
            if t is not None and forward_ad.unpack_dual(t).tangent is not None:
                return True
    return False


_increment = getattr(torch._C, "_increment_version", torch.autograd.graph.increment_version)


def _written(*tensors):
    """Tells autograd that a kernel wrote to these: a graph that saved one
    then refuses to run backward with the new values."""
    _increment(tensors)


def _last(t):
    """t with a contiguous last axis and no lazy sign (a gradient may come in any layout)."""
    t = t.resolve_neg()
    return t if t.shape[-1] <= 1 or t.stride(-1) == 1 else t.contiguous()


# ------------------------------------------------------------------ band_linear


def _linear_checks(x, weight, offsets, bias):
    _tensor(x, "x", dims="[batch][rows][n_in]")
    if weight.dim() != 3:
        raise ValueError("weight has to be [n_bands][n_out][n_in]")
    _offsets(offsets, x)
    bands = offsets.numel() - 1
    _tensor(weight, "weight", x, (bands, weight.shape[1], x.shape[2]))
    if not weight.is_contiguous():
        raise ValueError("weight has to be contiguous")
    if bias is not None:
        _tensor(bias, "bias", x, (bands, weight.shape[1]))
        if not bias.is_contiguous():
            raise ValueError("bias has to be contiguous")


def _linear_forward(x, weight, offsets, bias):
    batch, rows, n_in = x.shape
    n_out = weight.shape[1]
    y = x.new_empty((batch, rows, n_out))
    with _on(x):
        _check(_lib().nsgcqt_band_linear(
            _DTYPES[x.dtype], _ragged(offsets, batch, rows), _view3(x), weight.data_ptr(),
            None if bias is None else bias.data_ptr(), _view3(y), n_in, n_out, _stream(x)))
    return y


def _linear_grad_input(dy, weight, offsets):
    batch, rows, n_out = dy.shape
    n_in = weight.shape[2]
    dx = dy.new_empty((batch, rows, n_in))
    with _on(dy):
        _check(_lib().nsgcqt_band_linear_grad_input(
            _DTYPES[dy.dtype], _ragged(offsets, batch, rows), _view3(dy), weight.data_ptr(),
            _view3(dx), n_in, n_out, _stream(dy)))
    return dx


def _linear_grad_weight(x, dy, offsets, with_bias):
    batch, rows, n_in = x.shape
    n_out, bands = dy.shape[2], offsets.numel() - 1
    dw = torch.empty((bands, n_out, n_in), dtype=x.dtype, device=x.device)
    db = torch.empty((bands, n_out), dtype=x.dtype, device=x.device) if with_bias else None
    L = _lib()
    n = _bytes(L.nsgcqt_band_linear_workspace(bands, batch, rows, n_in, n_out))
    ws = torch.empty(max(n, 1), dtype=torch.uint8, device=x.device)
    with _on(x):
        _check(L.nsgcqt_band_linear_grad_weight(
            _DTYPES[x.dtype], _ragged(offsets, batch, rows), _view3(x), _view3(dy), dw.data_ptr(),
            None if db is None else db.data_ptr(), n_in, n_out, ws.data_ptr(), n, _stream(x)))
    return dw, db


class _BandLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, offsets):
        ctx.save_for_backward(x, weight, offsets)
        ctx.has_bias = bias is not None
        return _linear_forward(x, weight, offsets, bias)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, offsets = ctx.saved_tensors
        dy = _last(dy)
        dx = _linear_grad_input(dy, weight, offsets) if ctx.needs_input_grad[0] else None
        dw = db = None
        if ctx.needs_input_grad[1] or ctx.needs_input_grad[2]:
            dw, db = _linear_grad_weight(x, dy, offsets, ctx.has_bias and ctx.needs_input_grad[2])
        return dx, dw if ctx.needs_input_grad[1] else None, db, None


def band_linear(x, weight, offsets, bias=None):
    """y[b, c] = weight[g] @ x[b, c] + bias[g], g the band of token c.

    x [batch][rows][n_in], weight [n_bands][n_out][n_in], bias
    [n_bands][n_out] or None, offsets int64 [n_bands + 1]; returns
    [batch][rows][n_out]. Tokens that no band holds get zeros. Gradients for
    x, weight and bias.
    """
    _linear_checks(x, weight, offsets, bias)
    if not _trains(x, weight, bias):
        return _linear_forward(x, weight, offsets, bias)
    return _BandLinear.apply(x, weight, bias, offsets)


class BandLinear(torch.nn.Module):
    """band_linear with its own weights (uniform in +-n_in^-1/2 at the start)."""

    def __init__(self, n_bands, n_in, n_out, bias=True, device="cuda", dtype=torch.float32):
        super().__init__()
        k = n_in ** -0.5 if n_in else 0.0
        self.weight = torch.nn.Parameter(torch.empty(n_bands, n_out, n_in, device=device, dtype=dtype).uniform_(-k, k))
        self.bias = torch.nn.Parameter(torch.zeros(n_bands, n_out, device=device, dtype=dtype)) if bias else None

    def forward(self, x, offsets):
        return band_linear(x, self.weight, offsets, self.bias)


# ----------------------------------------------------------------------- rotary


def rotary_frequencies(sections, base=10000.0, device="cuda"):
    """Frequencies of `rotary`: base^(-i / s) for the i-th of an axis's s pairs."""
    return torch.cat([base ** (-torch.arange(s, dtype=torch.float64) / max(s, 1)) for s in sections]).float().to(device)


@functools.lru_cache(maxsize=256)
def _sections(sections, dim):
    """The packed sections of a head of dim values, and their number of pairs."""
    pairs = sum(sections)
    if not 1 <= len(sections) <= 4 or min(sections) < 0 or 2 * pairs > dim:
        raise ValueError("sections has to hold 1 to 4 counts of at most D / 2 pairs in all")
    return struct.pack(f"={len(sections)}i", *sections), pairs


def _rotary_call(q, k, positions, freqs, sections, interleaved, inverse):
    outs, views, heads = [], [], []
    for t in (q, k):
        if t is None:
            outs.append(None)
            views += [None, None]
            heads.append(0)
        else:
            o = torch.empty_like(t, memory_format=torch.contiguous_format)
            outs.append(o)
            views += [_view4(t), _view4(o)]
            heads.append(t.shape[2])
    t = q if q is not None else k
    batch, rows, _, dim = t.shape
    s = positions.stride()
    with _on(t):
        _check(_lib().nsgcqt_rotary(
            _DTYPES[t.dtype], views[0], views[1], heads[0], views[2], views[3], heads[1], batch, rows, dim,
            positions.data_ptr(), _POS[positions.dtype], s[0], s[1] if positions.dim() == 3 else 0, freqs.data_ptr(),
            sections, len(sections) // 4, int(interleaved), int(inverse), _stream(t)))
    return outs


def _rotary_forward(q, k, positions, freqs, sections, interleaved):
    return tuple(_rotary_call(q, k, positions, freqs, sections, interleaved, False))


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, positions, freqs, sections, interleaved):
        ctx.save_for_backward(positions, freqs)
        ctx.how = sections, interleaved
        ctx.set_materialize_grads(False)
        return _rotary_forward(q, k, positions, freqs, sections, interleaved)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dq, dk):
        positions, freqs = ctx.saved_tensors
        dq = _last(dq) if dq is not None and ctx.needs_input_grad[0] else None
        dk = _last(dk) if dk is not None and ctx.needs_input_grad[1] else None
        if dq is None and dk is None:
            return (None,) * 6
        dq, dk = _rotary_call(dq, dk, positions, freqs, *ctx.how, True)
        return dq, dk, None, None, None, None


def rotary(q, k, positions, freqs, sections, interleaved=False):
    """q and k with their pairs turned by positions[axis] * freqs[pair].

    q [batch][rows][heads][D] and k with its own heads (or None), positions
    [axes][rows] or [axes][batch][rows] (float32, float64 or int64), freqs
    float32 [sum(sections)], sections: the number of pairs of each of the 1
    to 4 axes. Pairs are values (p, p + P), P = sum(sections), or (2p, 2p + 1)
    with interleaved=True; values past 2 P are copied. Angles are formed in
    64 bits. Gradients for q and k; positions and freqs have none and are
    refused where they would need one. Returns (q, k), or q alone if k is None.
    """
    _tensor(q, "q", dims="[batch][rows][heads][D]")
    batch, rows, _, dim = q.shape
    if k is not None:
        if k.dim() != 4:
            raise ValueError("k has to be [batch][rows][heads][D]")
        _tensor(k, "k", q, (batch, rows, k.shape[2], dim))
    sec, pairs = _sections(tuple(sections), dim)
    axes = len(sections)
    if positions.dtype not in _POS or positions.device != q.device:
        raise ValueError("positions has to be float32, float64 or int64 on the device of q")
    if (positions.shape != (axes, rows) and positions.shape != (axes, batch, rows)) or (
            positions.stride(-1) != 1 if rows > 1 else positions.is_neg()):
        raise ValueError("positions has to be [axes][rows] or [axes][batch][rows], its rows contiguous")
    if freqs.dtype != torch.float32 or freqs.device != q.device or freqs.shape != (pairs,) or not freqs.is_contiguous():
        raise ValueError(f"freqs has to be a float32 vector of {pairs} values on the device of q")
    if _trains(positions, freqs):
        raise ValueError("rotary has no gradient for positions and freqs: detach them")
    call = _Rotary.apply if _trains(q, k) else _rotary_forward
    out = call(q, k, positions, freqs, sec, interleaved)
    return out[0] if k is None else out


# --------------------------------------------------------------- band_attention


def _shape_of(q, k, left, right, sinks, scale, keep):
    return _shape(q.shape[2], k.shape[2], q.shape[3], left, right, sinks, scale,
                          0 if keep is None else keep.data_ptr(), 0 if keep is None else keep.stride(0))


def _attention_forward(q, k, v, offsets, keep, left, right, sinks, scale, stats=None):
    batch, rows, heads, dim = q.shape
    o = torch.empty_like(q, memory_format=torch.contiguous_format)
    with _on(q):
        _check(_lib().nsgcqt_band_attention(
            _DTYPES[q.dtype], _ragged(offsets, batch, rows), _shape_of(q, k, left, right, sinks, scale, keep),
            _view4(q), _view4(k), _view4(v), _view4(o), None if stats is None else stats.data_ptr(), _stream(q)))
    return o


class _BandAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, offsets, keep, left, right, sinks, scale):
        stats = torch.empty((q.shape[0], q.shape[2], q.shape[1]), dtype=torch.float32, device=q.device)
        o = _attention_forward(q, k, v, offsets, keep, left, right, sinks, scale, stats)
        ctx.save_for_backward(q, k, v, o, stats, offsets, keep)
        ctx.how = left, right, sinks, scale
        return o

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, do):
        q, k, v, o, stats, offsets, keep = ctx.saved_tensors
        do = _last(do)
        dq, dk, dv = (torch.empty_like(t, memory_format=torch.contiguous_format) for t in (q, k, v))
        shape, r = _shape_of(q, k, *ctx.how, keep), _ragged(offsets, q.shape[0], q.shape[1])
        L = _lib()
        n = _bytes(L.nsgcqt_band_attention_workspace(r, shape))
        ws = torch.empty(max(n, 1), dtype=torch.uint8, device=q.device)
        with _on(q):
            _check(L.nsgcqt_band_attention_grad(
                _DTYPES[q.dtype], r, shape, _view4(q), _view4(k), _view4(v),
                _view4(o), stats.data_ptr(), _view4(do), _view4(dq), _view4(dk),
                _view4(dv), ws.data_ptr(), n, _stream(q)))
        return dq, dk, dv, None, None, None, None, None, None


def _keep(keep, like, batch, rows):
    if keep is not None and (keep.dtype != torch.bool or keep.device != like.device or keep.shape != (batch, rows) or (
            rows > 1 and keep.stride(1) != 1)):
        raise ValueError("keep has to be bool [batch][rows] on the device of q, its rows contiguous")


def band_attention(q, k, v, offsets, left, right=0, sinks=0, scale=None, keep=None):
    """Attention along each band of each signal.

    q [batch][rows][heads][D], k and v with kv_heads heads, a divisor of
    heads (D at most 128). Token i of a band sees token j of it when
    j <= i + right and either j >= i - left or j < sinks, and keep[b, j] (bool
    [batch][rows]) is set or keep is None; numbers count within the band.
    left or right None: no bound. scale: of the scores, D^-1/2 by default. A
    token that sees none gets zeros and passes no gradient, and what k and v
    hold at tokens that are not kept is never used. Gradients for q, k, v.
    """
    _tensor(q, "q", dims="[batch][rows][heads][D]")
    if k.dim() != 4:
        raise ValueError("k has to be [batch][rows][kv_heads][D]")
    batch, rows, heads, dim = q.shape
    _tensor(k, "k", q, (batch, rows, k.shape[2], dim))
    _tensor(v, "v", q, k.shape)
    _offsets(offsets, q)
    _keep(keep, q, batch, rows)
    far = 1 << 40
    call = _BandAttention.apply if _trains(q, k, v) else _attention_forward
    return call(q, k, v, offsets, keep, far if left is None else int(left), far if right is None else int(right),
                int(sinks), _scale(scale, dim))


# ------------------------------------------------------------- single-token step


def _caches(k_cache, v_cache, like, streams, kv_heads, dim):
    if k_cache.dim() != 4:
        raise ValueError("k_cache has to be [streams][kv_heads][slots][D]")
    shape = (streams, kv_heads, k_cache.shape[2], dim)
    for t, name in ((k_cache, "k_cache"), (v_cache, "v_cache")):
        _tensor(t, name, like, shape)
        if not t.is_contiguous():
            raise ValueError(f"{name} has to be contiguous")
    return k_cache.shape[2]


@functools.lru_cache(maxsize=256)
def _step_workspace(*sizes):
    return _bytes(_lib().nsgcqt_attention_step_workspace(*sizes))


def attention_step(q, k, v, k_cache, v_cache, pos, sinks=0, scale=None, out=None):
    """Attention of one new token of each stream over its ring cache.

    q [streams][heads][D], k and v [streams][kv_heads][D]: the new token
    number pos[s] (int64 [streams]) of stream s. k_cache and v_cache
    [streams][kv_heads][slots][D] hold the first `sinks` tokens and the last
    slots - sinks others; the new k and v are written there in place, then q
    attends over all tokens held. pos < 0: the stream has no token in this
    step, its cache stays as it is and its row is zero. Not differentiable.
    """
    _tensor(q, "q", dims="[streams][heads][D]")
    if k.dim() != 3:
        raise ValueError("k has to be [streams][kv_heads][D]")
    streams, heads, dim = q.shape
    kv_heads = k.shape[1]
    _tensor(k, "k", q, (streams, kv_heads, dim))
    _tensor(v, "v", q, k.shape)
    slots = _caches(k_cache, v_cache, q, streams, kv_heads, dim)
    if pos.dtype != torch.int64 or pos.device != q.device or pos.shape != (streams,) or not pos.is_contiguous():
        raise ValueError("pos has to be int64 [streams] on the device of q")
    if _trains(q, k, v, k_cache, v_cache, out):
        raise ValueError("attention_step has no gradient: call it under torch.no_grad()")
    o = torch.empty_like(q, memory_format=torch.contiguous_format) if out is None else _tensor(out, "out", q, q.shape)
    sinks = int(sinks)
    n = _step_workspace(streams, heads, kv_heads, dim, slots - sinks, sinks)
    ws = torch.empty(n, dtype=torch.uint8, device=q.device) if n else None
    with _on(q):
        _check(_lib().nsgcqt_attention_step(
            _DTYPES[q.dtype], streams, heads, kv_heads, dim, slots - sinks, sinks,
            _scale(scale, dim), _view_step(q), _view_step(k), _view_step(v), _view_step(o),
            k_cache.data_ptr(), v_cache.data_ptr(), pos.data_ptr(), ws.data_ptr() if n else None, n, _stream(q)))
    _written(k_cache, v_cache, *(() if out is None else (out,)))
    return o


def cache_fill(k, v, offsets, k_cache, v_cache, sinks=0):
    """Fills ring caches from whole bands: stream b * n_bands + g gets band g of signal b.

    k and v [batch][rows][kv_heads][D]; the caches are those of
    `attention_step`. Afterwards a stream's next token is number
    offsets[g + 1] - offsets[g]. Slots without a token are left alone. Not
    differentiable.
    """
    _tensor(k, "k", dims="[batch][rows][kv_heads][D]")
    batch, rows, kv_heads, dim = k.shape
    _tensor(v, "v", k, k.shape)
    _offsets(offsets, k)
    slots = _caches(k_cache, v_cache, k, batch * (offsets.numel() - 1), kv_heads, dim)
    if _trains(k, v, k_cache, v_cache):
        raise ValueError("cache_fill has no gradient: call it under torch.no_grad()")
    with _on(k):
        _check(_lib().nsgcqt_cache_fill(
            _DTYPES[k.dtype], _ragged(offsets, batch, rows), kv_heads, dim, slots - int(sinks), int(sinks),
            _view4(k), _view4(v), k_cache.data_ptr(), v_cache.data_ptr(), _stream(k)))
    _written(k_cache, v_cache)


class StreamCache:
    """Ring caches of many streams: the first `sinks` tokens and the last `window` others of each.

    `pos` holds the number of each stream's next token; a stream whose pos is
    below 0 is idle: its cache and its pos stay as they are.
    """

    def __init__(self, streams, kv_heads, head_dim, window, sinks=0, dtype=torch.bfloat16, device="cuda"):
        if window < 1 or sinks < 0:
            _bad("window must be at least 1 and sinks at least 0")
        self.sinks = sinks
        shape = (streams, kv_heads, sinks + window, head_dim)
        self.k = torch.zeros(shape, dtype=dtype, device=device)
        self.v = torch.zeros(shape, dtype=dtype, device=device)
        self.pos = torch.zeros(streams, dtype=torch.int64, device=device)

    def fill(self, k, v, offsets):
        """Starts the streams with whole bands (`cache_fill`)."""
        cache_fill(k, v, offsets, self.k, self.v, self.sinks)
        ends = offsets.clamp(0, k.shape[1])     # bands are cut to the row, as the kernels cut them
        self.pos.copy_((ends[1:] - ends[:-1]).repeat(k.shape[0]))

    def step(self, q, k, v, scale=None):
        """`attention_step` of every stream's next token (zeros for an idle one)."""
        o = attention_step(q, k, v, self.k, self.v, self.pos, self.sinks, scale)
        self.pos += self.pos >= 0
        return o


# -------------------------------------------------------------- decay_attention


def _decay_of(log_decay, like, kv_heads):
    if log_decay.dtype != torch.float32 or log_decay.device != like.device or log_decay.shape != (kv_heads,) or (
            not log_decay.is_contiguous()):
        raise ValueError(f"log_decay has to be a float32 vector of {kv_heads} values on the device of q")


def _states(state, like, streams, kv_heads, dim):
    if state.dtype != torch.float32 or state.device != like.device or (
            state.shape != (streams, kv_heads, dim, dim)) or not state.is_contiguous():
        raise ValueError(f"state has to be contiguous float32 {[streams, kv_heads, dim, dim]} on the device of q")


def _decay_shape_of(q, k, log_decay, keep, scale):
    return _decay_shape(q.shape[2], k.shape[2], q.shape[3], scale, log_decay.data_ptr(),
                        0 if keep is None else keep.data_ptr(), 0 if keep is None else keep.stride(0))


@functools.lru_cache(maxsize=256)
def _decay_bytes(bands, batch, rows, heads, kv_heads, dim, grad):
    here = ctypes.c_int64(0)   # offsets and decays that are not read
    at = ctypes.addressof(here)
    return _bytes(_lib().nsgcqt_decay_attention_workspace(_rows(at, bands, batch, rows),
                                                          _decay_shape(heads, kv_heads, dim, 1.0, at, 0, 0), grad))


def _decay_sizes(q, k, log_decay, keep, scale, offsets):
    """Refuses a shape as the call itself does."""
    _bytes(_lib().nsgcqt_decay_attention_workspace(_ragged(offsets, q.shape[0], q.shape[1]),
                                                   _decay_shape_of(q, k, log_decay, keep, scale), 0))


def _decay_workspace(q, kv_heads, offsets, grad):
    n = _decay_bytes(offsets.shape[0] - 1, q.shape[0], q.shape[1], q.shape[2], kv_heads, q.shape[3], grad)
    return torch.empty(n, dtype=torch.uint8, device=q.device) if n else None, n


def _decay_forward(q, k, v, offsets, log_decay, keep, state, scale):
    o = torch.empty_like(q, memory_format=torch.contiguous_format)
    shape, r = _decay_shape_of(q, k, log_decay, keep, scale), _ragged(offsets, q.shape[0], q.shape[1])
    with _on(q):
        ws, n = _decay_workspace(q, k.shape[2], offsets, 0)
        _check(_lib().nsgcqt_decay_attention(
            _DTYPES[q.dtype], r, shape, _view4(q), _view4(k), _view4(v), _view4(o),
            None if state is None else state.data_ptr(), ws.data_ptr() if n else None, n, _stream(q)))
    return o


class _DecayAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, offsets, log_decay, keep, state, scale):
        ctx.save_for_backward(q, k, v, offsets, log_decay, keep)
        ctx.scale = scale
        return _decay_forward(q, k, v, offsets, log_decay, keep, state, scale)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, do):
        q, k, v, offsets, log_decay, keep = ctx.saved_tensors
        do = _last(do)
        dq, dk, dv = (torch.empty_like(t, memory_format=torch.contiguous_format) for t in (q, k, v))
        shape, r = _decay_shape_of(q, k, log_decay, keep, ctx.scale), _ragged(offsets, q.shape[0], q.shape[1])
        with _on(q):
            ws, n = _decay_workspace(q, k.shape[2], offsets, 1)
            _check(_lib().nsgcqt_decay_attention_grad(
                _DTYPES[q.dtype], r, shape, _view4(q), _view4(k), _view4(v), _view4(do), _view4(dq), _view4(dk),
                _view4(dv), ws.data_ptr() if n else None, n, _stream(q)))
        return dq, dk, dv, None, None, None, None, None


def _decay_checks(q, k, v, offsets, log_decay, scale, keep, state):
    """Checks a call's arguments; the function to call, and the scale."""
    _tensor(q, "q", dims="[batch][rows][heads][D]")
    if k.dim() != 4:
        raise ValueError("k has to be [batch][rows][kv_heads][D]")
    batch, rows, _, dim = q.shape
    kv_heads = k.shape[2]
    _tensor(k, "k", q, (batch, rows, kv_heads, dim))
    _tensor(v, "v", q, k.shape)
    _offsets(offsets, q)
    _keep(keep, q, batch, rows)
    _decay_of(log_decay, q, kv_heads)
    if _trains(log_decay):
        raise ValueError("decay_attention has no gradient for log_decay: detach it")
    trains = _trains(q, k, v)
    if state is not None:
        _states(state, q, batch * (offsets.numel() - 1), kv_heads, dim)
        if trains or _trains(state):
            raise ValueError("decay_attention has no gradient from or into a state: call it under torch.no_grad()")
    return _DecayAttention.apply if trains else _decay_forward, _scale(scale, dim)


def decay_attention(q, k, v, offsets, log_decay, scale=None, keep=None, state=None):
    """Linear attention along each band, the past decaying by exp(log_decay) a token.

    o_t = scale * sum over s <= t of exp(log_decay (t - s)) (q_t . k_s) v_s,
    within token t's band. q [batch][rows][heads][D], k and v with kv_heads
    heads, a divisor of heads (D at most 128); log_decay float32 [kv_heads], at
    most 0. scale: D^-1/2 by default. keep (bool [batch][rows] or None): tokens
    that add nothing, though they count as distance; what k and v hold there is
    never used. state (float32 [batch * n_bands][kv_heads][D][D] or None): the
    sum of exp(..) k_s v_s^T over what came before each band, row b * n_bands +
    g for band g of signal b; it is replaced by that sum at the band's end.
    Gradients for q, k and v, where no state is given; log_decay has none.
    Tokens are taken 32 at a time: an infinity or NaN of a kept token, or a
    product with it that passes 32 bits, may make the results of up to 31 tokens
    before it NaN (in the gradients for k and v, of up to 31 after it).
    """
    call, scale = _decay_checks(q, k, v, offsets, log_decay, scale, keep, state)
    o = call(q, k, v, offsets, log_decay, keep, state, scale)
    if state is not None:
        _written(state)
    return o


def decay_step(q, k, v, state, pos, log_decay, scale=None, out=None):
    """`decay_attention` of one new token of each stream.

    q [streams][heads][D], k and v [streams][kv_heads][D]; state float32
    [streams][kv_heads][D][D] takes the token in place, then q meets it. pos
    int64 [streams] numbers the token: 0 starts a stream, whatever its state
    holds; below 0 the stream has no token in this step, its state stays as it
    is and its row is zero. Not differentiable.
    """
    _tensor(q, "q", dims="[streams][heads][D]")
    if k.dim() != 3:
        raise ValueError("k has to be [streams][kv_heads][D]")
    streams, heads, dim = q.shape
    kv_heads = k.shape[1]
    _tensor(k, "k", q, (streams, kv_heads, dim))
    _tensor(v, "v", q, k.shape)
    _decay_of(log_decay, q, kv_heads)
    _states(state, q, streams, kv_heads, dim)
    if pos.dtype != torch.int64 or pos.device != q.device or pos.shape != (streams,) or not pos.is_contiguous():
        raise ValueError("pos has to be int64 [streams] on the device of q")
    if _trains(q, k, v, state, log_decay, out):
        raise ValueError("decay_step has no gradient: call it under torch.no_grad()")
    o = torch.empty_like(q, memory_format=torch.contiguous_format) if out is None else _tensor(out, "out", q, q.shape)
    with _on(q):
        _check(_lib().nsgcqt_decay_step(
            _DTYPES[q.dtype], streams, heads, kv_heads, dim, _scale(scale, dim), _view_step(q), _view_step(k),
            _view_step(v), _view_step(o), state.data_ptr(), pos.data_ptr(), log_decay.data_ptr(), _stream(q)))
    _written(state, *(() if out is None else (out,)))
    return o


class DecayState:
    """The states of many streams of `decay_attention`: one matrix a key head, however long a stream is.

    `pos` holds the number of each stream's next token; a stream whose pos is
    below 0 is idle: its state and its pos stay as they are, until `read` has
    tokens for it.
    """

    def __init__(self, streams, kv_heads, head_dim, device="cuda"):
        self.state = torch.zeros((streams, kv_heads, head_dim, head_dim), dtype=torch.float32, device=device)
        self.pos = torch.zeros(streams, dtype=torch.int64, device=device)

    def read(self, q, k, v, offsets, log_decay, scale=None, keep=None):
        """`decay_attention` of whole bands: band g of signal b continues stream b * n_bands + g, or begins it where
        its pos is 0, or below 0 and the band has tokens. A call that is refused leaves states and pos as they are."""
        _, factor = _decay_checks(q, k, v, offsets, log_decay, scale, keep, self.state)
        _decay_sizes(q, k, log_decay, keep, factor, offsets)
        ends = offsets.clamp(0, q.shape[1])     # bands are cut to the row, as the kernels cut them
        more = (ends[1:] - ends[:-1]).clamp_(min=0).repeat(q.shape[0])
        self.state.masked_fill_(((self.pos == 0) | ((self.pos < 0) & (more > 0)))[:, None, None, None], 0.0)
        o = decay_attention(q, k, v, offsets, log_decay, factor, keep, self.state)
        self.pos.copy_(torch.where(more > 0, self.pos.clamp(min=0) + more, self.pos))
        return o

    def step(self, q, k, v, log_decay, scale=None):
        """`decay_step` of every stream's next token (zeros for an idle one)."""
        o = decay_step(q, k, v, self.state, self.pos, log_decay, scale)
        self.pos += self.pos >= 0
        return o


# -------------------------------------------------------------------- band_norm


def _act(activation):
    if activation not in _ACTS:
        raise ValueError(f"activation is {activation!r}: None, 'silu', 'gelu' or 'sigmoid' is expected")
    return _ACTS[activation]


def _norm_shape_of(x, weight, bias, groups, act, eps):
    w, b = ((0, 0) if t is None else (t.data_ptr(), t.stride(0) if t.shape[0] > 1 else 0) for t in (weight, bias))
    return _norm_shape(x.shape[2], groups, eps, w[0], b[0], w[1], b[1], act)


@functools.lru_cache(maxsize=256)
def _norm_bytes(dtype, bands, batch, rows, channels, groups, act, eps, grad, weights):
    here = ctypes.c_int64(0)   # offsets that are not read
    return _bytes(_lib().nsgcqt_band_norm_workspace(dtype, _rows(ctypes.addressof(here), bands, batch, rows),
                                                    _norm_shape(channels, groups, eps, 0, 0, 0, 0, act), grad, weights))


def _norm_workspace(x, bands, groups, act, eps, grad, weights):
    n = _norm_bytes(_DTYPES[x.dtype], bands, x.shape[0], x.shape[1], x.shape[2], groups, act, eps, grad, weights)
    return torch.empty(n, dtype=torch.uint8, device=x.device) if n else None, n


def _norm_call(x, offsets, weight, bias, groups, act, eps, stats=None):
    batch, rows, _ = x.shape
    y = torch.empty_like(x, memory_format=torch.contiguous_format)
    shape, r = _norm_shape_of(x, weight, bias, groups, act, eps), _ragged(offsets, batch, rows)
    with _on(x):
        ws, n = _norm_workspace(x, offsets.shape[0] - 1, groups, act, eps, 0, 0)
        _check(_lib().nsgcqt_band_norm(_DTYPES[x.dtype], r, shape, _view3(x), _view3(y),
                                       None if stats is None else stats.data_ptr(), ws.data_ptr() if n else None, n,
                                       _stream(x)))
    return y


def _norm_forward(x, weight, bias, offsets, groups, act, eps):
    return _norm_call(x, offsets, weight, bias, groups, act, eps)


class _BandNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, offsets, groups, act, eps):
        stats = torch.empty((x.shape[0], offsets.numel() - 1, groups, 2), dtype=torch.float64, device=x.device)
        y = _norm_call(x, offsets, weight, bias, groups, act, eps, stats)
        ctx.save_for_backward(x, weight, bias, offsets, stats)
        ctx.how = groups, act, eps
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, bias, offsets, stats = ctx.saved_tensors
        dy = _last(dy)
        need = ctx.needs_input_grad
        dx = torch.empty_like(x, memory_format=torch.contiguous_format) if need[0] else None
        dw, db = (torch.empty(t.shape, dtype=t.dtype, device=t.device) if n else None
                  for t, n in ((weight, need[1]), (bias, need[2])))
        shape, r = _norm_shape_of(x, weight, bias, *ctx.how), _ragged(offsets, x.shape[0], x.shape[1])
        with _on(x):
            ws, n = _norm_workspace(x, offsets.shape[0] - 1, *ctx.how, 1, int(dw is not None or db is not None))
            _check(_lib().nsgcqt_band_norm_grad(
                _DTYPES[x.dtype], r, shape, _view3(x), stats.data_ptr(), _view3(dy),
                None if dx is None else _view3(dx), None if dw is None else dw.data_ptr(),
                None if db is None else db.data_ptr(), ws.data_ptr() if n else None, n, _stream(x)))
        return dx, dw, db, None, None, None, None


def band_norm(x, offsets, weight=None, bias=None, groups=1, activation=None, eps=1e-5):
    """Group norm of each band of each signal, with an activation.

    x [batch][rows][channels]: mean and (biased) variance go over the channels
    of one of `groups` equal groups and all tokens of one band. weight and bias
    [n_bands][channels] or None: y = act(weight * (x - mean) / sqrt(var + eps)
    + bias); a row shared by the bands may be expanded to them. activation:
    None, "silu", "gelu" (by the normal distribution) or "sigmoid". Tokens that
    no band holds get zeros. Tokens are normalised each by itself as rows of one
    token: x [tokens][1][channels], offsets [0, 1]. At most 4,096 channels and
    1,024 groups. Gradients for x, weight and bias.
    """
    _tensor(x, "x", dims="[batch][rows][channels]")
    _offsets(offsets, x)
    for t, name in ((weight, "weight"), (bias, "bias")):
        if t is not None:
            _tensor(t, name, x, (offsets.numel() - 1, x.shape[2]))
    act, groups = _act(activation), int(groups)
    if groups < 1 or x.shape[2] % groups:
        _bad("groups must divide channels, and be at least 1")
    call = _BandNorm.apply if _trains(x, weight, bias) else _norm_forward
    return call(x, weight, bias, offsets, groups, act, float(eps))


class BandNorm(torch.nn.Module):
    """band_norm with its own weights (ones and zeros at the start)."""

    def __init__(self, n_bands, channels, groups=1, activation=None, eps=1e-5, device="cuda", dtype=torch.float32):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.ones(n_bands, channels, device=device, dtype=dtype))
        self.bias = torch.nn.Parameter(torch.zeros(n_bands, channels, device=device, dtype=dtype))
        self.groups, self.activation, self.eps = groups, activation, eps

    def forward(self, x, offsets):
        return band_norm(x, offsets, self.weight, self.bias, self.groups, self.activation, self.eps)


# ------------------------------------------------------------------- band_gated


def _gated_forward(x, weight, bias, offsets, act):
    batch, rows, n_in = x.shape
    n_out = weight.shape[2]
    y = x.new_empty((batch, rows, n_out))
    with _on(x):
        _check(_lib().nsgcqt_band_gated(
            _DTYPES[x.dtype], _ragged(offsets, batch, rows), _view3(x), weight.data_ptr(),
            None if bias is None else bias.data_ptr(), _view3(y), n_in, n_out, act, _stream(x)))
    return y


class _BandGated(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, offsets, act):
        ctx.save_for_backward(x, weight, bias, offsets)
        ctx.act = act
        return _gated_forward(x, weight, bias, offsets, act)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, bias, offsets = ctx.saved_tensors
        dy = _last(dy)
        batch, rows, n_in = x.shape
        n_out = weight.shape[2]
        need = ctx.needs_input_grad
        dx = torch.empty_like(x, memory_format=torch.contiguous_format) if need[0] else None
        dw = torch.empty_like(weight) if need[1] or need[2] else None
        db = torch.empty_like(bias) if need[2] else None
        L, r = _lib(), _ragged(offsets, batch, rows)
        n = _bytes(L.nsgcqt_band_gated_workspace(r, n_in, n_out)) if dw is not None else 0
        ws = torch.empty(max(n, 1), dtype=torch.uint8, device=x.device)
        with _on(x):
            _check(L.nsgcqt_band_gated_grad(
                _DTYPES[x.dtype], r, _view3(x), weight.data_ptr(), None if bias is None else bias.data_ptr(), _view3(dy),
                None if dx is None else _view3(dx), None if dw is None else dw.data_ptr(),
                None if db is None else db.data_ptr(), n_in, n_out, ctx.act, ws.data_ptr(), n, _stream(x)))
        return dx, dw if need[1] else None, db, None, None


def band_gated(x, weight, offsets, bias=None, activation="silu"):
    """y[b, c] = act(weight[g, 0] @ x[b, c] + bias[g, 0]) * (weight[g, 1] @ x[b, c] + bias[g, 1]), g the band of token c.

    x [batch][rows][n_in], weight [n_bands][2][n_out][n_in], bias
    [n_bands][2][n_out] or None, offsets int64 [n_bands + 1]; activation None,
    "silu", "gelu" (by the normal distribution) or "sigmoid"; returns
    [batch][rows][n_out]. Tokens that no band holds get zeros. Gradients for
    x, weight and bias; they form both projections again.
    """
    _tensor(x, "x", dims="[batch][rows][n_in]")
    if weight.dim() != 4:
        raise ValueError("weight has to be [n_bands][2][n_out][n_in]")
    _offsets(offsets, x)
    bands, n_out = offsets.numel() - 1, weight.shape[2]
    _tensor(weight, "weight", x, (bands, 2, n_out, x.shape[2]))
    if not weight.is_contiguous():
        raise ValueError("weight has to be contiguous")
    if bias is not None:
        _tensor(bias, "bias", x, (bands, 2, n_out))
        if not bias.is_contiguous():
            raise ValueError("bias has to be contiguous")
    act = _act(activation)
    call = _BandGated.apply if _trains(x, weight, bias) else _gated_forward
    return call(x, weight, bias, offsets, act)


class BandGated(torch.nn.Module):
    """band_gated with its own weights (uniform in +-n_in^-1/2 at the start)."""

    def __init__(self, n_bands, n_in, n_out, activation="silu", bias=True, device="cuda", dtype=torch.float32):
        super().__init__()
        k = n_in ** -0.5 if n_in else 0.0
        self.weight = torch.nn.Parameter(
            torch.empty(n_bands, 2, n_out, n_in, device=device, dtype=dtype).uniform_(-k, k))
        self.bias = torch.nn.Parameter(torch.zeros(n_bands, 2, n_out, device=device, dtype=dtype)) if bias else None
        self.activation = activation

    def forward(self, x, offsets):
        return band_gated(x, self.weight, offsets, self.bias, self.activation)
