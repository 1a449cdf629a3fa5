"""GPU tests of the streaming block's layers at values and sizes where their arithmetic can go wrong: groups of equal
values, levels far above the differences, infinite and extreme arguments, very long sums, very many signals.

Bounds, beside test_block_gpu's: what a norm makes of a value is off by 2^-20 of the normalised value and of 1 (the
level's own rest, 2^-24 of a level of 10^6 deviations), however high the level is.
"""
import ctypes

import pytest

torch = pytest.importorskip("torch")
import paper_2609_29119_amd as nc  # noqa: E402
from paper_2609_29119_amd import layers  # noqa: E402
from test_block_gpu import ACTS, TYPES, U, act_reference, close, offsets_of, randn  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nc.lib()


def norm_of(x, lengths, w, b, groups, act, eps, dy):
    """(y, dx, dw, db) in 64 bits, and the sizes of their terms: those of the normalised values, not of the level."""
    x, dy, w, b = (t.detach().double() for t in (x, dy, w, b))
    ref = [torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(w), torch.zeros_like(w)]
    size = [torch.zeros_like(t) for t in ref]
    at = 0
    for g, n in enumerate(lengths):
        s = slice(at, at + n)
        at += n
        split = lambda t: t.reshape(*t.shape[:-1], groups, -1)  # noqa: E731
        mean2 = lambda v: v.mean((1, 3), keepdim=True)  # noqa: E731
        t = split(x[:, s])
        t = t - mean2(t)
        t = t - mean2(t)                       # (what the level's own rounding left)
        r = (mean2(t * t) + eps) ** -0.5
        hat = t * r
        hat_size = hat.abs() + 2.0
        wg, bg = split(w[g]), split(b[g])
        z, z_size = wg * hat + bg, wg.abs() * hat_size + bg.abs()
        y, slope = act_reference(z, act)
        ref[0][:, s], size[0][:, s] = y.flatten(2), (y.abs() + (slope.abs() + 0.4) * z_size).flatten(2)
        d0 = split(dy[:, s])
        dz, dz_size = d0 * slope, d0.abs() * (slope.abs() + z_size)
        d, d_size = dz * wg, dz_size * wg.abs()
        ref[1][:, s] = (r * (d - mean2(d) - hat * mean2(d * hat))).flatten(2)
        size[1][:, s] = (r * (d_size + mean2(d_size) + hat_size * mean2(d_size * hat_size))).flatten(2)
        ref[2][g], size[2][g] = (dz * hat).sum((0, 1)).flatten(), (dz_size * hat_size).sum((0, 1)).flatten()
        ref[3][g], size[3][g] = dz.sum((0, 1)).flatten(), dz_size.sum((0, 1)).flatten()
    return ref, size


def norm_and_gradients(x, lengths, w, b, groups, act, eps, dy):
    x, w, b = (t.detach().requires_grad_() for t in (x, w, b))
    y = layers.band_norm(x, offsets_of(lengths), w, b, groups, act, eps)
    return [y.detach(), *torch.autograd.grad(y, (x, w, b), dy)]


LEVEL = {torch.float32: (1000.0, -3e6), torch.float16: (1000.0, 30000.0, -60000.0), torch.bfloat16: (1000.0, -1e6)}
EQUAL = [
    # lengths, batch, channels, groups
    ([1], 40, 16, 16),        # single tokens, a group a channel
    ([7, 1, 30], 2, 24, 4),
    ([9000, 3], 1, 24, 3),    # parts
    ([2500], 2, 5, 5),
]


# --------------------------------------------------------------------------------------------- groups of equal values


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(EQUAL)))
def test_band_norm_of_equal_values(case, dtype):
    """A group without differences: the normalised value is 0 at any level, y is act(b), and w has no gradient."""
    lengths, batch, ch, groups = EQUAL[case]
    rows, G = sum(lengths), len(lengths)
    w, b = (randn(n, G, ch, dtype=dtype) for n in (case, case + 10))
    dy = randn(case + 20, batch, rows, ch, dtype=dtype)
    for level in LEVEL[dtype]:
        each = level * (1 - torch.arange(groups, device="cuda") / (4 * groups))       # a level of its own for each group
        x = each.repeat_interleave(ch // groups).to(dtype).expand(batch, rows, ch).contiguous()
        for act in ACTS:
            got = norm_and_gradients(x, lengths, w, b, groups, act, 1e-5, dy)
            ref, size = norm_of(x, lengths, w, b, groups, act, 1e-5, dy)
            if act is None:
                assert torch.equal(got[0], b.repeat_interleave(torch.tensor(lengths, device="cuda"), 0).expand_as(got[0]))
            assert not got[2].any(), (level, act)
            for t, r, z, name in zip(got, ref, size, ("y", "dx", "dw", "db")):
                close(t, r, z, f"{name} at {level}, {act}", 2.0 ** -20, 2.0 ** -25)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(EQUAL)))
def test_band_norm_of_nearly_equal_values(case, dtype):
    """One value in forty is a step of the type above the level: the others are next to the mean, not on it."""
    lengths, batch, ch, groups = EQUAL[case]
    rows, G = sum(lengths), len(lengths)
    w, b = (randn(n, G, ch, dtype=dtype) for n in (case, case + 10))
    dy = randn(case + 20, batch, rows, ch, dtype=dtype)
    some = (torch.rand(batch, rows, ch, generator=torch.Generator().manual_seed(case)) < 1 / 40).cuda()
    for level in LEVEL[dtype]:
        level = torch.tensor(level).to(dtype).item()
        x = torch.where(some, level + 2 * U[dtype] * abs(level), level).to(dtype)
        got = norm_and_gradients(x, lengths, w, b, groups, "silu", 1e-5, dy)
        ref, size = norm_of(x, lengths, w, b, groups, "silu", 1e-5, dy)
        for t, r, z, name in zip(got, ref, size, ("y", "dx", "dw", "db")):
            close(t, r, z, f"{name} at {level}", 2.0 ** -20, 2.0 ** -25)


# ----------------------------------------------------------------------------------------------- levels far from zero


@pytest.mark.parametrize("tokens", [40, 5000])
def test_band_norm_of_a_level_of_a_million_deviations(tokens):
    """In 32 bits: squares of the values themselves would leave 2^-53 of 10^12 deviations."""
    x, dy = 1e6 + randn(1, 2, tokens, 16), randn(2, 2, tokens, 16)
    w, b = randn(3, 1, 16), randn(4, 1, 16)
    got = norm_and_gradients(x, [tokens], w, b, 2, "silu", 1e-5, dy)
    ref, size = norm_of(x, [tokens], w, b, 2, "silu", 1e-5, dy)
    for t, r, z, name in zip(got, ref, size, ("y", "dx", "dw", "db")):
        close(t, r, z, name, 2.0 ** -20, 2.0 ** -25)


# ------------------------------------------------------------------------------- very long sums of the norm's weights


@pytest.mark.parametrize("lengths,batch,channels", [
    ([2_000_000], 1, 16),        # thousands of parts
    ([1], 262_144, 1032),        # one token of many signals, a thread's sum over as many rows as an item has
])
def test_long_sums_of_a_norm_s_weights(lengths, batch, channels):
    """Terms of one sign, whose additions may all round the same way: n equal terms added in turn are off by up to
    n 2^-25 of their sum. The chains in 32 bits have 32 terms here, 8 + 8 + 16 (a thread, its columns, their sum) or 32 of
    a thread; what follows is in 64 bits, and rounded once."""
    rows = lengths[0]
    x = torch.randn(batch, rows, channels, device="cuda")
    dy = (0.5 + (torch.arange(channels, device="cuda") + 0.3) / (2 * channels)).expand(batch, rows, channels)
    b = torch.zeros(1, channels, device="cuda").requires_grad_()
    db = torch.autograd.grad(layers.band_norm(x, offsets_of(lengths), None, b), b, dy)[0].double()
    want = dy[0, :1].double() * (batch * rows)
    assert ((db - want).abs() <= (2.0 ** -20 + 2.0 ** -24) * want).all(), ((db / want - 1).abs().max() * 2 ** 20).item()


# --------------------------------------------------------------------------------------------------------- many parts


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths,batch", [([20000, 1, 0, 300], 5), ([1, 1], 5000)])
def test_many_parts_of_a_norm_s_weights(lengths, batch, dtype):
    """Parts of several signals, and items of short bands, so many that the waves of a workgroup share them; 70 channels."""
    rows, G = sum(lengths), len(lengths)
    x, dy = randn(1, batch, rows, 70, dtype=dtype), randn(2, batch, rows, 70, dtype=dtype)
    w, b = (randn(n, G, 70, dtype=dtype) for n in (3, 4))
    got = norm_and_gradients(x, lengths, w, b, 7, "silu", 1e-3, dy)
    full = [n for n in range(G) if lengths[n]]
    ref, size = norm_of(x, [lengths[n] for n in full], w[full], b[full], 7, "silu", 1e-3, dy)
    for t, r, z, name in zip([*got[:2], got[2][full], got[3][full]], ref, size, ("y", "dx", "dw", "db")):
        close(t, r, z, name, 2.0 ** -20, 2.0 ** -25)
    assert not any(got[i][n].any() for i in (2, 3) for n in range(G) if not lengths[n])


# ----------------------------------------------------------------------------------------- and of the gated product's


def test_long_sums_of_a_gated_product_s_biases():
    """As for the norm's weights: 4,000,000 rows of one band."""
    rows, n_out = 4_000_000, 8
    x = torch.zeros(1, rows, 1, device="cuda")
    w = randn(1, 1, 2, n_out, 1)
    b = randn(2, 1, 2, n_out).requires_grad_()
    dy = (0.5 + (torch.arange(n_out, device="cuda") + 0.3) / 16).expand(1, rows, n_out)
    y = layers.band_gated(x, w, offsets_of([rows]), b, None)
    db = torch.autograd.grad(y, b, dy)[0].double()
    want = dy[0, 0].double() * b.detach().double().flip(1) * rows
    assert ((db - want).abs() <= 2.0 ** -20 * want.abs()).all(), ((db / want - 1).abs().max() * 2 ** 20).item()


# -------------------------------------------------------------------------------------------- rows that are not there


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, n_in", [(1, 8), (33, 8), (70, 130)])
def test_rows_that_are_not_there_add_nothing_to_infinite_values(rows, n_in, dtype):
    """A gate or a value that a bias makes infinite: its gradient is infinite or, by the other bias, a sum over its rows."""
    x, dy = randn(1, 1, rows, n_in, dtype=dtype), randn(2, 1, rows, 4, dtype=dtype).abs() + 0.5
    w = randn(3, 1, 2, 4, n_in, dtype=dtype, by=0.1)
    bias = torch.tensor([[[float("inf"), 1.0, 1.0, 2.0], [1.0, float("inf"), 1.0, 2.0]]], device="cuda").to(dtype).requires_grad_()
    y = layers.band_gated(x, w, offsets_of([rows]), bias, None)
    db = torch.autograd.grad(y, bias, dy)[0][0].double()
    a, u = (torch.matmul(x[0].double(), w[0, i].double().T.contiguous()) + bias.detach()[0, i].double() for i in (0, 1))
    want = torch.stack([(dy[0].double() * t).sum(0) for t in (u, a)])
    size = torch.stack([(dy[0].double() * (1 + x[0].double().abs().sum(1, keepdim=True) + t.abs())).sum(0) for t in (u, a)])
    assert torch.equal(db.isinf(), want.isinf()) and (db[want.isinf()] > 0).all()
    fine = want.isfinite()
    assert ((db - want)[fine].abs() <= U[dtype] * want[fine].abs() + 2.0 ** -20 * size[fine]).all()


# -------------------------------------------------------------------------------------------------- activations' ends


def act_limits(z, how):
    """act_reference, with its limits at the infinities."""
    far = z.isinf()
    f, slope = act_reference(torch.where(far, 0.0, z), how)
    up = (z > 0).double()
    if how is None:
        return z, torch.ones_like(z)
    value = up if how == "sigmoid" else torch.where(z > 0, z, 0.0)
    return torch.where(far, value, f), torch.where(far, 0.0 if how == "sigmoid" else up, slope)


def extremes(dtype):
    most = torch.finfo(dtype).max
    z = [0.0, 1.0, 3.0, 10.0, 13.25, 14.5, 20.0, 88.0, 104.0, 127.0, 200.0, 1e4, 1e19, 1e30, 1e36, 1e38, 2.5e38, 3e38, most]
    z = torch.tensor([v for v in z if v <= most] + [float("inf")], dtype=torch.float64)
    return torch.cat([z, -z]).to(dtype).cuda()


def check_act(got, want, z, what):
    """Equal where infinite; else one rounding and 2^-20 of the value, times the argument where it is an exponent. An
    exponential below 2^-126 may be taken for 0, and is multiplied by at most 1 + |z|, with |z| < 128 where it is not 0."""
    got, want, z = got.double(), want.double(), z.detach()
    by = 1 + z.double().abs().clamp(max=128)
    tiny = 2.0 ** -25 if z.dtype == torch.float16 else by * 2.0 ** -126
    fine = torch.where(want.isinf(), got == want, (got - want).abs() <= (U[z.dtype] + 2.0 ** -20 * by) * want.abs() + tiny)
    assert fine.all(), f"{what}: {z[~fine].tolist()} give {got[~fine].tolist()}, not {want[~fine].tolist()}"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS)
def test_activations_at_their_ends(act, dtype):
    """Infinite and the largest arguments, as biases set them, in both operators; slopes as db has them."""
    z = extremes(dtype)
    n = z.numel()
    want, slope = act_limits(z.double(), act)
    off = offsets_of([1])
    bias = torch.stack([z, torch.ones_like(z)])[None].requires_grad_()
    x, w = randn(1, 1, 1, 8, dtype=dtype).requires_grad_(), torch.zeros(1, 2, n, 8, dtype=dtype, device="cuda")
    y = layers.band_gated(x, w, off, bias, act)
    dx, db = torch.autograd.grad(y, [x, bias], torch.ones_like(y))
    check_act(y[0, 0], want, z, "gated")
    check_act(db[0, 0], slope, z, "gated slope")
    check_act(db[0, 1], want, z, "gated, other bias")
    y = layers.band_gated(x.detach().expand(1, 1, 8), w, off, bias.detach(), act)
    check_act(y[0, 0], want, z, "gated forward")
    for rows in (1, 9000):
        level = torch.full((1, rows, n), 3.0, dtype=dtype, device="cuda")
        b = z[None].detach().requires_grad_()
        y = layers.band_norm(level, offsets_of([rows]), torch.ones_like(b), b, 1, act)
        dy = torch.zeros_like(y)
        dy[:, rows // 2] = 1.0
        db = torch.autograd.grad(y, b, dy)[0]
        check_act(y[0, 0], want, z, "norm")
        check_act(y[0, -1], want, z, "norm")
        check_act(db[0], slope, z, "norm slope")
    # a NaN stays one
    assert layers.band_gated(x.detach(), w, off, torch.full_like(bias, float("nan")).detach(), act).isnan().all()


# --------------------------------------------------------------------------------------------------------- infinities


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_a_group_with_an_infinity_has_no_norm(bad, act, dtype):
    """No variance: the group's values in that band and signal are NaN, in y and dx; all others are as they were."""
    lengths, batch, ch = [5, 9000, 3], 2, 24
    x = randn(1, batch, 9008, ch, dtype=dtype)
    w, b = (randn(n, 3, ch, dtype=dtype) for n in (2, 3))
    dy = randn(4, batch, 9008, ch, dtype=dtype)
    want = norm_and_gradients(x, lengths, w, b, 3, act, 1e-5, dy)
    hit = torch.zeros_like(x, dtype=torch.bool)
    for signal, band, token, channel in ((0, slice(0, 5), 4, 3), (1, slice(5, 9005), 5, 8), (0, slice(5, 9005), 7000, 20)):
        x[signal, token, channel] = bad
        hit[signal, band, channel // 8 * 8:channel // 8 * 8 + 8] = True
    got = norm_and_gradients(x, lengths, w, b, 3, act, 1e-5, dy)
    for a, e, name in zip(got[:2], want[:2], ("y", "dx")):
        assert a[hit].isnan().all(), name
        assert torch.equal(a[~hit], e[~hit]), name
    for a, name in zip(got[2:], ("dw", "db")):
        if name == "dw" or act is not None:
            assert a[0, :8].isnan().all() and a[1, 8:].isnan().all(), name
        assert torch.isfinite(a[2]).all() and torch.isfinite(a[0, 8:]).all() and torch.isfinite(a[1, :8]).all(), name


# -------------------------------------------------------------------------------------------------- ends of the range


@pytest.mark.parametrize("by", [1e30, 1e-30])
@pytest.mark.parametrize("tokens", [40, 5000])
def test_band_norm_of_values_near_the_ends_of_their_range(tokens, by):
    x, dy = (randn(1, 2, tokens, 16) * by).float(), randn(2, 2, tokens, 16)
    w, b = randn(3, 1, 16), randn(4, 1, 16)
    got = norm_and_gradients(x, [tokens], w, b, 2, "silu", 1e-30, dy)
    ref, size = norm_of(x, [tokens], w, b, 2, "silu", 1e-30, dy)
    for t, r, z, name in zip(got, ref, size, ("y", "dx", "dw", "db")):
        close(t, r, z, name, 2.0 ** -20, 1e-37)


# ---------------------------------------------------------------------------------- more workgroups than a launch has


def test_band_norm_of_more_signals_than_a_launch_has_workgroups():
    """Single tokens of 33,554,435 signals: two launches of each kernel."""
    n = (1 << 25) + 3
    x = torch.randn(n, 1, 2, device="cuda").bfloat16().requires_grad_()
    w = torch.tensor([[1.5, -2.0]], device="cuda").bfloat16().requires_grad_()
    dy = torch.randn(n, 1, 2, device="cuda").bfloat16()
    y = layers.band_norm(x, torch.tensor([0, 1], device="cuda"), w, eps=1e-3)
    dx, dw = torch.autograd.grad(y, (x, w), dy)
    for at in (slice(0, 1 << 20), slice((1 << 25) - (1 << 20), n)):   # around the launches' border and at both ends
        ref, size = zip(*[norm_of_pairs(t[at].detach(), d[at], w) for t, d in ((x, dy),)])
        close(y[at], ref[0][0], size[0][0], "y", 2.0 ** -20, 1e-37)
        close(dx[at], ref[0][1], size[0][1], "dx", 2.0 ** -20, 1e-37)
    assert not (y == 0).all(2).logical_and((x[:, :, 0] != x[:, :, 1])).any()
    want, terms = torch.zeros(2, device="cuda").double(), torch.zeros(2, device="cuda").double()
    for i in range(0, n, 1 << 22):
        t = x[i:i + (1 << 22), 0].detach().double()
        h = (t - t.mean(1, keepdim=True)) * (t.var(1, correction=0, keepdim=True) + 1e-3) ** -0.5 * dy[i:i + (1 << 22), 0].double()
        want, terms = want + h.sum(0), terms + h.abs().sum(0)
    close(dw[0], want, terms, "dw", 2.0 ** -20)


def norm_of_pairs(x, dy, w, eps=1e-3):
    """(y, dx) of groups of two values, in 64 bits, and their sizes."""
    x, dy, w = (t.detach().double() for t in (x, dy, w))
    t = x - x.mean(2, keepdim=True)
    r = ((t * t).mean(2, keepdim=True) + eps) ** -0.5
    hat, d = t * r, dy * w
    dx = r * (d - d.mean(2, keepdim=True) - hat * (d * hat).mean(2, keepdim=True))
    return (hat * w, dx), ((hat.abs() + 2) * w.abs(), r * (d.abs() + d.abs().mean(2, keepdim=True)) * (2 + (hat.abs() + 2) ** 2))


# -------------------------------------------------------------------------------------------------- an infinite token


@pytest.mark.parametrize("dtype", TYPES)
def test_an_infinite_token_reaches_the_tiles_it_lies_in_only(dtype):
    """Tiles of 32 tokens from the band's start for o and dq, from its end for dk and dv (136 .. 167 is one)."""
    q, k, v, do = (randn(i, 1, 200, 2, 32, dtype=dtype) for i in (1, 2, 3, 4))
    off, lam = offsets_of([200]), torch.tensor([-0.1, -0.01], device="cuda")

    def run(q, k, v, do):
        q, k, v = (t.clone().requires_grad_() for t in (q, k, v))
        o = layers.decay_attention(q, k, v, off, lam)
        return (o, *torch.autograd.grad(o, [q, k, v], do))

    want = run(q, k, v, do)
    q[:, 130], k[:, 131], v[:, 132], do[:, 133] = float("inf"), float("nan"), float("inf"), -float("inf")
    got = run(q, k, v, do)
    for a, b, at in zip(got, want, (slice(0, 128), slice(0, 128), slice(136, 200), slice(136, 200))):
        assert torch.equal(a[:, at], b[:, at])


# ------------------------------------------------------------------------------------------------------------ streams


def test_streams_that_a_read_begins_continues_and_leaves_alone():
    """Streams at 0, idle or going on, with and without tokens; a refused call changes nothing."""
    lengths, off, lam = [5, 0, 7, 0, 3, 0], offsets_of([5, 0, 7, 0, 3, 0]), torch.tensor([-0.1, -0.01], device="cuda")
    q, k, v = (randn(i, 1, 15, 2, 8) for i in (1, 2, 3))
    held = layers.DecayState(6, 2, 8)
    held.state.copy_(randn(4, 6, 2, 8, 8))
    held.pos.copy_(torch.tensor([0, 0, -1, -2, 9, 4], device="cuda"))
    state, pos = held.state.clone(), held.pos.clone()
    for bad, error in ((dict(scale=float("inf")), nc.NsgcqtError), (dict(scale=1e300), nc.NsgcqtError),
                       (dict(keep=torch.ones(1, 14, dtype=torch.bool, device="cuda")), ValueError)):
        with pytest.raises(error):
            held.read(q, k, v, off, lam, **bad)
        assert torch.equal(held.state, state) and torch.equal(held.pos, pos)
    start = state.clone()
    start[[0, 2]] = 0.0          # those that begin
    want = layers.decay_attention(q, k, v, off, lam, state=start)
    assert torch.equal(held.read(q, k, v, off, lam), want)
    assert held.pos.tolist() == [5, 0, 7, -2, 12, 4]
    for n in (0, 2, 3, 4, 5):    # (what the state at pos 0 holds is not used)
        assert torch.equal(held.state[n], start[n] if lengths[n] else state[n]), n


# ----------------------------------------------------------------------------------------------- claims of the header


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("channels, odd", [(64, 0), (77, 0), (40, 1)])
def test_band_norm_may_write_over_its_input(channels, odd, dtype):
    """Through the C call, which takes one tensor as x and y: short bands, long ones and tokens of no band."""
    lengths, first, rows = [9, 0, 9000, 40], 4, 9060
    x = randn(1, 2, rows, channels + odd, dtype=dtype)[..., odd:]
    want = layers.band_norm(x, offsets_of(lengths, first), activation="gelu")
    L, off = layers._lib(), offsets_of(lengths, first)
    r = layers._ragged(off, 2, rows)
    shape = layers._norm_shape(channels, 1, 1e-5, 0, 0, 0, 0, 2)
    n = L.nsgcqt_band_norm_workspace(layers._DTYPES[dtype], r, shape, 0, 0)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    assert L.nsgcqt_band_norm(layers._DTYPES[dtype], r, shape, layers._view3(x), layers._view3(x), None, ws.data_ptr(), n,
                              ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == nc.OK
    assert torch.equal(x, want)


def test_the_norm_s_module():
    m = layers.BandNorm(3, 24, groups=4, activation="silu", eps=1e-3)
    x, off = randn(1, 2, 60, 24).requires_grad_(), offsets_of([20, 0, 40])
    with torch.no_grad():
        m.weight.copy_(randn(2, 3, 24))
        m.bias.copy_(randn(3, 3, 24))
    y = m(x, off)
    assert torch.equal(y, layers.band_norm(x, off, m.weight, m.bias, 4, "silu", 1e-3))
    got = torch.autograd.grad(y.square().sum(), [x, m.weight, m.bias])
    assert all(torch.isfinite(g).all() and g.any() for g in got)
    assert [n for n, _ in m.named_parameters()] == ["weight", "bias"]
