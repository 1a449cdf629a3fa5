"""GPU tests of the layers that make up a streaming block, against plain forms in 64 bits.

Bounds. u is the unit roundoff of the data's type (2^-24, 2^-11, 2^-8): a
result is off by its one rounding, at most u of each value. What its sums leave
is measured by `size`, the same result with every term's magnitude in the place
of its value: in 32 bits 2^-24 for each of the factors and partial sums of a
term (fewer than sixteen of them matter here, so 2^-20); with 16-bit data a
term's 32-bit factors enter the matrix products as two numbers of 8 bits, off by
2^-17 each, the two last ones' product is left out (2^-16), and no term has more
than three such factors: 2^-14 holds them all.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2609_29119_amd as nc  # noqa: E402
from paper_2609_29119_amd import layers  # noqa: E402

pytestmark = pytest.mark.gpu

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nc.lib()


def sums_of(dtype):
    return 2.0 ** -20 if dtype == torch.float32 else 2.0 ** -14


def close(got, ref, size, what, sums=None, tiny=0.0):
    """Each value within its own rounding (got's type) and `sums` of its terms' size; tiny: the type's smallest step."""
    u = U[got.dtype]
    got, ref, size = (t.detach().double().cpu() for t in (got, ref, size))
    assert got.shape == ref.shape, what
    assert torch.isfinite(got).all(), f"{what}: not finite"
    if ref.numel() == 0:
        return
    over = ((got - ref).abs() - (u * ref.abs() + sums * size + tiny)).max().item()
    at = int(((got - ref).abs() - (u * ref.abs() + sums * size + tiny)).argmax())
    assert over <= 0, f"{what}: value {at} is {got.flatten()[at]}, not {ref.flatten()[at]}, of size {size.flatten()[at]}"


def offsets_of(lengths, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(lengths)]).astype(np.int64), device="cuda")


def randn(seed, *shape, dtype=torch.float32, by=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g, dtype=torch.float64) * by).to(dtype).cuda()


# -------------------------------------------------------------- decay_attention


def decays_of(heads, seed=0):
    """From a head that forgets at once to one that hardly does."""
    g = torch.Generator().manual_seed(seed)
    return -(10.0 ** -(4 * torch.rand(heads, generator=g))).cuda()


def decay_reference(q, k, v, lengths, first, log_decay, scale, keep=None, state=None, do=None):
    """Every pair of tokens, in 64 bits: (o, dq, dk, dv, state after) and the same of the terms' magnitudes."""
    dev = "cuda"
    q, k, v = (t.detach().double().to(dev) for t in (q, k, v))
    do = torch.zeros_like(q) if do is None else do.detach().double().to(dev)
    h, hk, B, G = q.shape[2], k.shape[2], q.shape[0], len(lengths)
    lam = log_decay.double().to(dev)
    out = []
    for size in (False, True):
        Q, K, V, DO = (t.abs() if size else t for t in (q, k, v, do))
        if keep is not None:
            K, V = (torch.where(keep[:, :, None, None], t, 0.0) for t in (K, V))
        o, dq, dk, dv = (torch.zeros_like(t) for t in (Q, Q, K, K))
        st = None
        if state is not None:
            st = state.detach().double().to(dev).view(B, G, hk, q.shape[3], -1).clone()
            st = st.abs() if size else st
        at = first
        for g, n in enumerate(lengths):
            s = slice(at, at + n)
            at += n
            if n == 0:
                continue
            i = torch.arange(n, device=dev, dtype=torch.float64)
            lag = i[:, None] - i
            for a in range(h):
                c = a // (h // hk)
                fade = torch.where(lag >= 0, (lam[c] * lag.clamp(min=0)).exp(), 0.0) * (abs(scale) if size else scale)
                Qa, Kc, Vc, Da = Q[:, s, a], K[:, s, c], V[:, s, c], DO[:, s, a]
                p, dp = torch.matmul(Qa, Kc.mT.contiguous()) * fade, torch.matmul(Da, Vc.mT.contiguous()) * fade
                o[:, s, a] = torch.matmul(p, Vc)
                if st is not None:
                    grow = (lam[c] * (i + 1)).exp()[None, :, None] * (abs(scale) if size else scale)
                    o[:, s, a] += torch.matmul(Qa, st[:, g, c]) * grow
                dq[:, s, a] = torch.matmul(dp, Kc)
                dk[:, s, c] += torch.matmul(dp.mT.contiguous(), Qa)
                dv[:, s, c] += torch.matmul(p.mT.contiguous(), Da)
            if st is not None:
                for c in range(hk):
                    w = (lam[c] * (n - 1 - i)).exp()[None, :, None]
                    st[:, g, c] = st[:, g, c] * (lam[c] * n).exp() + torch.matmul((K[:, s, c] * w).mT.contiguous(), V[:, s, c])
        if keep is not None:
            dk, dv = (torch.where(keep[:, :, None, None], t, 0.0) for t in (dk, dv))
        out.append((o, dq, dk, dv, None if st is None else st.reshape(state.shape)))
    return out


DECAY = [
    # lengths, batch, heads, kv_heads, dim
    ([1], 1, 1, 1, 1),
    ([1, 2, 0, 3], 2, 2, 1, 8),
    ([31, 32, 33, 64, 65], 1, 4, 2, 32),
    ([70, 0, 129], 2, 3, 3, 64),
    ([128, 127], 1, 6, 2, 40),
    ([257, 5], 1, 2, 1, 96),
    ([300], 2, 2, 2, 128),
    ([129, 260], 1, 2, 1, 17),
    ([1000, 3, 0, 555], 1, 2, 1, 64),        # several segments
    ([3] * 140, 1, 2, 2, 16),
    ([700], 1, 3, 1, 100),
    ([0, 0], 2, 1, 1, 4),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("case", range(len(DECAY)))
def test_decay_attention(case, masked, dtype):
    lengths, batch, h, hk, d = DECAY[case]
    rows = sum(lengths)
    qkv = randn(case, batch, rows, h + 2 * hk, d, dtype=dtype)
    q, k, v = (t.detach().requires_grad_() for t in qkv.split([h, hk, hk], 2))
    do = randn(case + 30, batch, rows, h, d, dtype=dtype)
    keep = None
    if masked:
        keep = torch.rand(batch, rows, generator=torch.Generator().manual_seed(case)) > 0.3
        keep[:, : rows // 3] = False
        keep = keep.cuda()
    off, lam = offsets_of(lengths), decays_of(hk, case)
    o = layers.decay_attention(q, k, v, off, lam, keep=keep)
    got = (o, *torch.autograd.grad(o, [q, k, v], do))
    ref, size = decay_reference(q, k, v, lengths, 0, lam, d ** -0.5, keep, do=do)
    for t, r, z, name in zip(got, ref, size, ("o", "dq", "dk", "dv")):
        close(t, r, z, name, sums_of(dtype), 2.0 ** -25 if dtype == torch.float16 else 1e-37)
    if masked:
        assert not got[2][~keep].any() and not got[3][~keep].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(DECAY)))
def test_decay_attention_from_and_into_a_state(case, dtype):
    lengths, batch, h, hk, d = DECAY[case]
    rows = sum(lengths)
    q, k, v = (randn(case + i, batch, rows, n, d, dtype=dtype) for i, n in enumerate((h, hk, hk)))
    state = randn(case + 40, batch * len(lengths), hk, d, d, by=3.0)
    off, lam = offsets_of(lengths), decays_of(hk, case)
    ref, size = decay_reference(q, k, v, lengths, 0, lam, 0.3, state=state)
    before = state.clone()
    o = layers.decay_attention(q, k, v, off, lam, 0.3, state=state)
    close(o, ref[0], size[0], "o", sums_of(dtype), 2.0 ** -25 if dtype == torch.float16 else 1e-37)
    close(state, ref[4], size[4], "state", 2.0 ** -20)     # three numbers of 8 bits: 32-bit results
    # bands in two calls are bands in one
    cut = [n // 2 for n in lengths]
    if rows:
        first = torch.cat([torch.arange(a, a + n) for a, n in zip(off.tolist(), cut)] + [torch.zeros(0)]).long().cuda()
        rest = torch.cat([torch.arange(a + c, a + n) for a, c, n in zip(off.tolist(), cut, lengths)]).long().cuda()
        two = [layers.decay_attention(q[:, at], k[:, at], v[:, at], offsets_of(n), lam, 0.3, state=before)
               for at, n in ((first, cut), (rest, [n - c for n, c in zip(lengths, cut)]))]
        close(two[0], ref[0][:, first], size[0][:, first], "o", sums_of(dtype), 2.0 ** -25)
        close(two[1], ref[0][:, rest], size[0][:, rest], "o", sums_of(dtype), 2.0 ** -25)
        close(before, ref[4], size[4], "state", 2.0 ** -20)


STEP = [
    # streams, heads, kv_heads, dim, tokens
    (1, 1, 1, 1, 3),
    (3, 2, 1, 8, 5),
    (5, 8, 2, 64, 4),
    (2, 6, 3, 33, 4),
    (2, 4, 4, 128, 3),
    (4, 12, 1, 20, 4),
    (2, 5, 1, 90, 3),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(STEP)))
def test_decay_step_from_the_first_token(case, dtype):
    """Steps against the whole stream at once; a state that holds anything at pos 0, an idle stream."""
    streams, h, hk, d, tokens = STEP[case]
    q, k, v = (randn(case + i, streams, tokens, n, d, dtype=dtype) for i, n in enumerate((h, hk, hk)))
    lam = decays_of(hk, case)
    held = layers.DecayState(streams + 1, hk, d)
    held.state.fill_(float("nan"))
    held.state[streams] = 7.0
    held.pos[streams] = -1
    pad = lambda t: torch.cat([t, t[:1]])  # noqa: E731
    rows = []
    for t in range(tokens):
        o = held.step(*(pad(x[:, t]) for x in (q, k, v)), lam)
        assert o[streams].abs().max() == 0
        rows.append(o[:streams])
    assert (held.state[streams] == 7.0).all() and held.pos.tolist() == [tokens] * streams + [-1]
    zero = torch.zeros(streams, hk, d, d, device="cuda")
    ref, size = decay_reference(q, k, v, [tokens], 0, lam, d ** -0.5, state=zero)
    close(torch.stack(rows, 1), ref[0], size[0], "o", 2.0 ** -20, 2.0 ** -25)
    close(held.state[:streams], ref[4], size[4], "state", 2.0 ** -20)


# -------------------------------------------------------------------- band_norm

ACTS = [None, "silu", "gelu", "sigmoid"]


def act_reference(z, how):
    """act(z) and act'(z), in 64 bits."""
    if how is None:
        return z, torch.ones_like(z)
    if how == "gelu":
        phi = 0.5 * torch.special.erfc(-z / 2 ** 0.5)
        return z * phi, phi + z * (-z * z / 2).exp() / (2 * np.pi) ** 0.5
    s = torch.sigmoid(z)
    return (s, s * torch.sigmoid(-z)) if how == "sigmoid" else (z * s, s + z * s * torch.sigmoid(-z))


def norm_reference(x, lengths, first, w, b, groups, act, eps, dy):
    """(y, dx, dw, db) in 64 bits, and the sizes of their terms: a value's own magnitude, the mean's and the shift's
    stand in z, and each sum has its terms' magnitudes."""
    x, dy = x.detach().double(), dy.detach().double()
    B, _, ch = x.shape
    G = len(lengths)
    w = torch.ones(G, ch, device="cuda").double() if w is None else w.detach().double()
    b = torch.zeros(G, ch, device="cuda").double() if b is None else b.detach().double()
    ref = [torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(w), torch.zeros_like(w)]
    size = [torch.zeros_like(t) for t in ref]
    at = first
    for g, n in enumerate(lengths):
        s = slice(at, at + n)
        at += n
        if n == 0:
            continue
        split = lambda t: t.reshape(*t.shape[:-1], groups, -1)  # noqa: E731
        t = split(x[:, s])
        mean, var = t.mean((1, 3), keepdim=True), t.var((1, 3), correction=0, keepdim=True)
        r = (var + eps) ** -0.5
        hat, hat_size = (t - mean) * r, (t.abs() + mean.abs()) * r
        wg, bg = split(w[g]), split(b[g])
        z, z_size = wg * hat + bg, wg.abs() * hat_size + bg.abs()
        y, slope = act_reference(z, act)
        ref[0][:, s], size[0][:, s] = y.flatten(2), (y.abs() + (slope.abs() + 0.4) * z_size).flatten(2)
        d0 = split(dy[:, s])
        dz, dz_size = d0 * slope, d0.abs() * (slope.abs() + z_size)
        d, d_size = dz * wg, dz_size * wg.abs()
        mean2 = lambda v: v.mean((1, 3), keepdim=True)  # noqa: E731
        ref[1][:, s] = (r * (d - mean2(d) - hat * mean2(d * hat))).flatten(2)
        size[1][:, s] = (r * (d_size + mean2(d_size) + hat_size * mean2(d_size * hat_size))).flatten(2)
        ref[2][g], size[2][g] = (dz * hat).sum((0, 1)).flatten(), (dz_size * hat_size).sum((0, 1)).flatten()
        ref[3][g], size[3][g] = dz.sum((0, 1)).flatten(), dz_size.sum((0, 1)).flatten()
    return ref, size


NORM = [
    # lengths, batch, channels, groups, affine
    ([1], 1, 1, 1, True),
    ([1], 5, 24, 3, True),                  # single tokens
    ([5, 0, 3], 2, 8, 8, True),
    ([130, 1, 257], 3, 12, 4, True),
    ([300, 7, 0, 0, 129], 2, 128, 8, True),
    ([64, 200], 1, 77, 7, True),
    ([700, 900], 1, 64, 1, True),           # several chunks
    ([6000], 2, 9, 1, False),
    ([31, 33], 2, 1000, 10, True),
    ([9, 20], 1, 4096, 4, True),
    ([40], 1, 2600, 2, False),
    ([3] * 150 + [0, 1], 1, 16, 2, True),
    ([0, 0], 2, 4, 2, True),
    ([17, 5], 40, 33, 33, True),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(NORM)))
def test_band_norm(case, dtype):
    lengths, batch, ch, groups, affine = NORM[case]
    rows, G, act = sum(lengths), len(lengths), ACTS[case % 4]
    x = (randn(case, batch, rows, ch) + 2 * randn(case + 1, ch)).to(dtype).requires_grad_()
    w, b = (((randn(case + n, G, ch, by=0.4) + 1).to(dtype).requires_grad_() if affine else None) for n in (50, 60))
    dy = randn(case + 70, batch, rows, ch, dtype=dtype)
    y = layers.band_norm(x, offsets_of(lengths), w, b, groups, act, 1e-3)
    got = [y, *torch.autograd.grad(y, [t for t in (x, w, b) if t is not None], dy)]
    ref, size = norm_reference(x, lengths, 0, w, b, groups, act, 1e-3, dy)
    for t, r, z, name in zip(got, ref, size, ("y", "dx", "dw", "db")):
        close(t, r, z, name, 2.0 ** -20, 2.0 ** -25)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS)
def test_band_norm_strides_uncovered_tokens_and_shared_weights(act, dtype):
    """Odd strides, tokens of no band, one row of weights for all bands, whose gradients are then its sum."""
    lengths, first, rows, batch, ch = [17, 1150], 9, 1190, 2, 40
    big = randn(3, batch, rows + 3, 2 * ch + 1, dtype=dtype)
    w, b = (randn(n, ch, dtype=dtype).requires_grad_() for n in (4, 5))
    dy = randn(6, rows, batch, ch, dtype=dtype).transpose(0, 1)
    for lo in (0, 1):
        x = big[:, 1:rows + 1, lo:lo + ch].detach().requires_grad_()
        y = layers.band_norm(x, offsets_of(lengths, first), w.expand(2, -1), b.expand(2, -1), 5, act)
        got = torch.autograd.grad(y, [x, w, b], dy)
        ref, size = norm_reference(x, lengths, first, w.expand(2, -1), b.expand(2, -1), 5, act, 1e-5, dy)
        close(y, ref[0], size[0], "y", 2.0 ** -20, 2.0 ** -25)
        close(got[0], ref[1], size[1], "dx", 2.0 ** -20, 2.0 ** -25)
        # autograd adds the two bands' rows, each rounded: one rounding of each row, and one of the sum
        for t, r, z, name in zip(got[1:], ref[2:], size[2:], ("dw", "db")):
            u = U[dtype]
            assert ((t.double() - r.sum(0)).abs() <= 2.0 ** -20 * z.sum(0) + u * (r.abs().sum(0) + 1.01 * r.sum(0).abs()) * 1.01 + 2.0 ** -24).all(), name
        for t in (y, got[0]):
            assert t[:, :first].abs().max() == 0 and t[:, first + 1167:].abs().max() == 0


def test_band_norm_far_from_zero():
    """A mean of 10^4 standard deviations: the statistics are differences from the mean, not of squares."""
    for n in (40, 5000):
        x = 1e4 + randn(1, 2, n, 16)
        y = layers.band_norm(x, offsets_of([n]), groups=2)
        ref, _ = norm_reference(x, [n], 0, None, None, 2, None, 1e-5, x)
        assert (y.double() - ref[0]).abs().max() < 2.0 ** -20
        same = layers.band_norm(torch.full((1, n, 16), 3e4, device="cuda"), offsets_of([n]), activation="silu")
        assert not same.any()


# ------------------------------------------------------------------- band_gated


def gated_reference(x, w, b, lengths, first, act, dy):
    """(y, dx, dw, db) in 64 bits, and their sizes: projections' errors, 2^-20 of their terms, pass through the
    activation and its slope (both change by at most their argument's change, 0.8 of it for the slope)."""
    x, w, dy = (t.detach().double() for t in (x, w, dy))
    b = torch.zeros(*w.shape[:3], device="cuda").double() if b is None else b.detach().double()
    ref = [torch.zeros(*x.shape[:2], w.shape[2], device="cuda").double(), torch.zeros_like(x), torch.zeros_like(w),
           torch.zeros_like(b)]
    size = [torch.zeros_like(t) for t in ref]
    at = first
    for g, n in enumerate(lengths):
        s = slice(at, at + n)
        at += n
        if n == 0:
            continue
        xs, d = x[:, s], dy[:, s]
        a, u = (torch.matmul(xs, w[g, i].T.contiguous()) + b[g, i] for i in (0, 1))
        za, zu = (torch.matmul(xs.abs(), w[g, i].T.abs().contiguous()) + b[g, i].abs() for i in (0, 1))
        f, slope = act_reference(a, act)
        fz, sz = f.abs() + slope.abs() * za + za * 2.0 ** -20, slope.abs() + za
        ref[0][:, s], size[0][:, s] = f * u, fz * zu
        da, du, da_z, du_z = d * u * slope, d * f, d.abs() * zu * sz, d.abs() * fz
        ref[1][:, s] = torch.matmul(da, w[g, 0]) + torch.matmul(du, w[g, 1])
        size[1][:, s] = torch.matmul(da_z, w[g, 0].abs()) + torch.matmul(du_z, w[g, 1].abs())
        for i, (t, z) in enumerate(((da, da_z), (du, du_z))):
            ref[2][g, i] = torch.matmul(t.flatten(0, 1).T.contiguous(), xs.flatten(0, 1))
            size[2][g, i] = torch.matmul(z.flatten(0, 1).T.contiguous(), xs.flatten(0, 1).abs())
            ref[3][g, i], size[3][g, i] = t.sum((0, 1)), z.sum((0, 1))
    return ref, size


GATED = [
    # lengths, batch, n_in, n_out, bias
    ([1], 1, 1, 1, True),
    ([5, 0, 3], 2, 2, 32, True),
    ([130, 1, 257], 3, 8, 8, False),
    ([64, 200], 1, 33, 77, True),
    ([300, 7, 0, 0, 129], 2, 128, 128, True),
    ([150], 2, 72, 200, True),
    ([40, 90], 1, 200, 40, False),
    ([31, 33], 2, 257, 65, True),
    ([1500, 600], 3, 24, 16, True),        # several chunks of the weights' gradient
    ([3] * 150 + [0, 1], 1, 16, 24, True),
    ([0, 0], 2, 4, 4, True),
    ([70, 131], 2, 520, 130, True),
    ([1] * 40, 5, 64, 96, True),
    ([12], 1, 0, 8, True),                 # nothing but the bias
    ([12, 4], 1, 8, 0, False),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(GATED)))
def test_band_gated(case, dtype):
    lengths, batch, n_in, n_out, bias = GATED[case]
    rows, G, act = sum(lengths), len(lengths), ACTS[(case + 1) % 4]
    x = randn(case, batch, rows, n_in, dtype=dtype).requires_grad_()
    w = randn(case + 50, G, 2, n_out, n_in, dtype=dtype, by=max(n_in, 1) ** -0.5).requires_grad_()
    b = randn(case + 90, G, 2, n_out, dtype=dtype).requires_grad_() if bias else None
    dy = randn(case + 70, batch, rows, n_out, dtype=dtype)
    y = layers.band_gated(x, w, offsets_of(lengths), b, act)
    got = [y, *torch.autograd.grad(y, [t for t in (x, w, b) if t is not None], dy)]
    ref, size = gated_reference(x, w, b, lengths, 0, act, dy)
    close(y, ref[0], size[0], "y", 2.0 ** -20, 2.0 ** -25)
    for t, r, z, name in zip(got[1:], ref[1:], size[1:], ("dx", "dw", "db")):
        close(t, r, z, name, 2.0 ** -20 if name == "db" else sums_of(dtype), 2.0 ** -25)


@pytest.mark.parametrize("dtype", TYPES)
def test_band_gated_strides_and_uncovered_tokens(dtype):
    lengths, first, rows, batch, n_in, n_out = [17, 150], 9, 190, 2, 48, 40
    big = randn(3, batch, rows + 3, 2 * n_in + 1, dtype=dtype)
    for lo in (0, 1):
        x = big[:, 1:rows + 1, lo:lo + n_in].detach().requires_grad_()
        w = randn(4, 2, 2, n_out, n_in, dtype=dtype, by=0.2).requires_grad_()
        dy = randn(5, rows, batch, n_out, dtype=dtype).transpose(0, 1)
        y = layers.band_gated(x, w, offsets_of(lengths, first), activation="gelu")
        dx, dw = torch.autograd.grad(y, [x, w], dy)
        ref, size = gated_reference(x, w, None, lengths, first, "gelu", dy)
        close(y, ref[0], size[0], "y", 2.0 ** -20, 2.0 ** -25)
        close(dx, ref[1], size[1], "dx", sums_of(dtype), 2.0 ** -25)
        close(dw, ref[2], size[2], "dw", sums_of(dtype), 2.0 ** -25)
        for t in (y, dx):
            assert t[:, :first].abs().max() == 0 and t[:, first + 167:].abs().max() == 0
