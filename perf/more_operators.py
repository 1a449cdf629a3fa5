"""The calls whose speed matters to a user of a whole block of a streaming network on the band layout.

A block behind the constant-Q transform normalises the features of each band
(`band_norm`: group norm with an activation, channels last), mixes a band's
tokens by linear attention whose past decays at a rate of each head's own
(`decay_attention`, whose memory of a stream is one matrix a head, and
`decay_step` for single tokens), and passes them through a gated product
(`band_gated`: two projections, an activation and their product). Rows are
ragged: C tokens (coefficients) a signal, cut into bands of unequal length.

Band layouts are those of the repository's workloads, computed here from the
constant-Q definition, or free ones (any lengths, empty ones among them).
Where `own` is false, `run` computes the plain form in 32 bits: bands are cut
into blocks of tokens, the last one padded.
"""
import math
import random

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}

# ---------------------------------------------------------------------- cases

_TINY = {"layout": "cq", "fs": 22050.0, "fmin": 110.0, "bins": 12, "n": 16384}
_TRAIN = {"layout": "cq", "fs": 44100.0, "fmin": 40.0, "bins": 24, "n": 220500}
_STRESS = {"layout": "cq", "fs": 22050.0, "fmin": 55.0, "bins": 36, "n": 88200}


def listed():
    return [
        # one token of each of 64 streams, normalised by itself: latency
        {"name": "norm_step", "op": "norm", "layout": "free", "bands": 1, "tokens": 1, "shape_seed": 0, "batch": 64,
         "dtype": "bf16", "channels": 128, "groups": 4, "act": "silu", "affine": True},
        # features of a batch of clips in a mask estimator: odd widths, seven groups of eleven channels
        {"name": "norm_stress", "op": "norm", **_STRESS, "batch": 8, "dtype": "f16", "channels": 77, "groups": 7,
         "act": "gelu", "affine": True},
        # a hidden layer's norm in training, with the gradients of input, weights and bias: 5 s clips
        {"name": "norm_train", "op": "norm_train", **_TRAIN, "batch": 2, "dtype": "bf16", "channels": 128, "groups": 8,
         "act": "silu", "affine": True},
        # one token of every band of 16 signals, each band with matrices of its own: the weights are what is read
        {"name": "gated_bands", "op": "gated", "layout": "each", "bands": 221, "batch": 16, "dtype": "bf16", "k": 128,
         "m": 256, "act": "silu", "bias": False},
        # a batch of clips in 16 bits, an odd width on one side
        {"name": "gated_stress", "op": "gated", **_STRESS, "batch": 4, "dtype": "f16", "k": 96, "m": 193, "act": "gelu",
         "bias": True},
        # the feed-forward part of a block in training: 5 s clips
        {"name": "gated_train", "op": "gated_train", **_TRAIN, "batch": 2, "dtype": "bf16", "k": 128, "m": 256,
         "act": "silu", "bias": True},
        # a short clip in 32 bits: the smallest whole row
        {"name": "decay_clip", "op": "decay", **_TINY, "batch": 1, "dtype": "f32", "heads": 4, "kv_heads": 4, "dim": 32,
         "keep": False, "state": False},
        # narrow heads of an odd count over shared key heads, silent coefficients dropped
        {"name": "decay_stress", "op": "decay", **_STRESS, "batch": 4, "dtype": "f16", "heads": 6, "kv_heads": 3,
         "dim": 40, "keep": True, "state": False},
        # training over every band of 5 s clips: silent coefficients dropped, shared key heads
        {"name": "decay_train", "op": "decay_train", **_TRAIN, "batch": 2, "dtype": "bf16", "heads": 8, "kv_heads": 4,
         "dim": 64, "keep": True, "state": False},
        # one long stream read in on top of what its state holds (the prompt of a streaming session)
        {"name": "decay_long", "op": "decay", "layout": "free", "bands": 1, "tokens": 131072, "shape_seed": 0,
         "batch": 1, "dtype": "bf16", "heads": 8, "kv_heads": 8, "dim": 128, "keep": False, "state": True},
        # one token of one stream: latency
        {"name": "step_one", "op": "step", "streams": 1, "dtype": "bf16", "heads": 8, "kv_heads": 4, "dim": 64},
        # one token of every band of 16 signals, each band a stream of its own
        {"name": "step_bands", "op": "step", "streams": 3536, "dtype": "bf16", "heads": 8, "kv_heads": 4, "dim": 64},
    ]


def _log(rng, lo, hi):
    return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def draw(rng):
    """One more case: sizes spread over the logarithm of the range."""
    op = rng.choice(["norm", "norm", "norm_train", "gated", "gated", "gated_train", "decay", "decay", "decay_train",
                     "step", "step"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    kv = rng.choice([1, 2, 3, 4])
    heads = kv * rng.choice([1, 1, 2, 3])
    dim = rng.choice([16, 32, 40, 64, 64, 80, 96, 128, rng.randint(3, 128)])
    if op == "step":
        most = 4e8 / (8 * kv * dim * dim)
        return {"op": op, "streams": max(1, min(_log(rng, 1, 8192), int(most))), "dtype": dtype, "heads": heads,
                "kv_heads": kv, "dim": dim}
    kind = rng.random()
    if kind < 0.55:
        fs = rng.choice([16000.0, 22050.0, 44100.0])
        c = {"op": op, "layout": "cq", "fs": fs, "fmin": round(rng.uniform(30.0, 120.0), 1),
             "bins": rng.randint(4, 48), "n": 2 * _log(rng, 2000, 110250)}
    elif kind < 0.9:
        c = {"op": op, "layout": "free", "bands": _log(rng, 1, 300), "tokens": _log(rng, 1, 130000),
             "shape_seed": rng.randrange(1 << 20)}
    else:
        c = {"op": op, "layout": "each", "bands": _log(rng, 1, 600)}
    tokens = max(1, sum(_lengths(c)))
    c["dtype"] = dtype
    if op.startswith("norm"):
        groups = rng.choice([1, 1, 2, 4, 8, rng.randint(1, 20)])
        channels = groups * max(1, round(_log(rng, 2, 512) / groups))
        share = max(1, int(min(440e3 * 128 / max(channels, 32) / tokens, 4096)))
        c.update(batch=_log(rng, 1, share), channels=channels, groups=groups,
                 act=rng.choice(["silu", "silu", "gelu", "sigmoid", "none"]), affine=rng.random() < 0.8)
        return c
    if op.startswith("gated"):
        k, m = _log(rng, 2, 320), _log(rng, 2, 640)
        share = max(1, int(min(440e3 * 128 * 256 / max(k, 32) / max(m, 64) / tokens, 440e3 / tokens, 256)))
        c.update(batch=_log(rng, 1, share), k=k, m=m, act=rng.choice(["silu", "silu", "gelu", "sigmoid", "none"]),
                 bias=rng.random() < 0.6)
        return c
    share = max(1, int(min(440e3 * 8 * 64 / (heads * max(dim, 32)) / tokens, 256)))
    c.update(batch=_log(rng, 1, share), heads=heads, kv_heads=kv, dim=dim, keep=rng.random() < 0.4,
             state=op == "decay" and rng.random() < 0.4)
    return c


def _lengths(case):
    """Tokens of each band."""
    if case["layout"] == "each":
        return [1] * case["bands"]
    if case["layout"] == "free":
        bands, tokens = case["bands"], case["tokens"]
        if bands == 1:
            return [tokens]
        r = random.Random(case["shape_seed"])
        share = [0.0 if r.random() < 0.1 else r.expovariate(1.0) for _ in range(bands)]
        share[-1] = share[-1] if any(share) else 1.0
        cuts, at = [0], 0.0
        for s in share:
            at += s
            cuts.append(round(tokens * at / sum(share)))
        return [b - a for a, b in zip(cuts, cuts[1:])]
    fs, n, bins = case["fs"], case["n"], case["bins"]
    half, q, xs, j = n // 2, 1.0 / (2.0 ** (1.0 / bins) - 1.0), [], 0
    while case["fmin"] * 2.0 ** (j / bins) < fs / 2:
        xs.append(case["fmin"] * 2.0 ** (j / bins) * n / fs)
        j += 1
    got = [min(half, math.ceil(xs[0]) - 1) + 1]
    got += [min(half, math.ceil(x + x / q) - 1) - max(0, math.floor(x - x / q) + 1) + 1 for x in xs]
    return [m for m in got + [half - math.floor(xs[-1])] if m > 0]


# --------------------------------------------------------------------- inputs


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = _TYPES[case["dtype"]]

    def normal(*shape, by=1.0, about=0.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * by + about).to(kind)

    def decays(n):
        # a head forgets within ten tokens, the last one within a thousand
        x = 3.0 + 7.0 * torch.arange(n, device="cuda") / max(n - 1, 1) + torch.rand(n, generator=gen, device="cuda")
        return torch.log1p(-(2.0 ** -x))

    if case["op"] == "step":
        b, h, hk, d = case["streams"], case["heads"], case["kv_heads"], case["dim"]
        s = {"case": case, "q": normal(b, h, d), "k": normal(b, hk, d), "v": normal(b, hk, d), "log_decay": decays(hk),
             "state": torch.randn(b, hk, d, d, generator=gen, device="cuda") * 4.0}
        # most streams are under way, some begin with this token, a few have none in this step
        age = torch.rand(b, generator=gen, device="cuda")
        on = torch.randint(1, 100000, (b,), generator=gen, device="cuda")
        s["pos"] = torch.where(age < 0.9, on, torch.where(age < 0.96, 0, -1)) if b > 8 else on
        return s
    lengths, batch = _lengths(case), case["batch"]
    tokens, bands = sum(lengths), len(lengths)
    n = torch.tensor(lengths, dtype=torch.int64)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]).cuda()
    s = {"case": case, "offsets": offsets, "lengths": n.cuda(),
         "band": torch.arange(bands, device="cuda").repeat_interleave(n.cuda())}
    # the plain form's plan: blocks of tokens of one band, the last one of a band padded
    size = max(1, min(128, max(lengths)))
    blocks = (n + size - 1) // size
    s["size"], s["of"] = size, torch.arange(bands).repeat_interleave(blocks).cuda()
    s["first"] = ((torch.arange(int(blocks.sum())) - (blocks.cumsum(0) - blocks).repeat_interleave(blocks)) * size).cuda()
    # features of a band have the band's own level: low bands are louder
    level = torch.logspace(0.5, -0.5, bands, device="cuda")[s["band"]][None, :, None]
    if case["op"].startswith("norm"):
        ch = case["channels"]
        centre = torch.randn(ch, generator=gen, device="cuda")
        s["x"] = ((torch.randn(batch, tokens, ch, generator=gen, device="cuda") + centre) * level).to(kind)
        s["weight"] = normal(bands, ch, by=0.2, about=1.0) if case["affine"] else None
        s["bias"] = normal(bands, ch, by=0.2) if case["affine"] else None
        if case["op"] == "norm_train":
            s["dy"] = normal(batch, tokens, ch)
            for name in ("x", "weight", "bias"):
                if s[name] is not None:
                    s[name].requires_grad_(True)
        return s
    if case["op"].startswith("gated"):
        k, m = case["k"], case["m"]
        s["x"] = (torch.randn(batch, tokens, k, generator=gen, device="cuda") * level).to(kind)
        s["weight"] = normal(bands, 2, m, k, by=k ** -0.5)
        s["bias"] = normal(bands, 2, m, by=0.1) if case["bias"] else None
        if case["op"] == "gated_train":
            s["dy"] = normal(batch, tokens, m)
            for name in ("x", "weight", "bias"):
                if s[name] is not None:
                    s[name].requires_grad_(True)
        return s
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    # query, key and value are parts of one projection's output, as a model has them
    s["q"], s["k"], s["v"] = normal(batch, tokens, h + 2 * hk, d).split([h, hk, hk], 2)
    s["log_decay"], s["keep"], s["state"] = decays(hk), None, None
    if case["keep"]:  # silent coefficients: one in eight, and one stretch
        s["keep"] = torch.rand(batch, tokens, generator=gen, device="cuda") > 0.125
        at = int(torch.randint(0, tokens, (1,), generator=gen, device="cuda"))
        s["keep"][:, at:at + 300] = False
    if case["state"]:
        s["state"] = torch.randn(batch * bands, hk, d, d, generator=gen, device="cuda") * 4.0
    if case["op"] == "decay_train":
        s["do"] = normal(batch, tokens, h, d)
        for name in ("q", "k", "v"):
            s[name] = s[name].detach().requires_grad_(True)
    return s


# ---------------------------------------------------------------- plain forms


def _act(z, how):
    """act(z) and act'(z)."""
    if how == "none":
        return z, torch.ones_like(z)
    if how == "gelu":
        phi = 0.5 * (1.0 + torch.erf(z * 0.5 ** 0.5))
        return z * phi, phi + z * (-0.5 * z * z).exp() * (2.0 * math.pi) ** -0.5
    sig = 1.0 / (1.0 + (-z).exp())
    return (sig, sig * (1.0 - sig)) if how == "sigmoid" else (z * sig, sig * (1.0 + z * (1.0 - sig)))


def _norm(s):
    with torch.no_grad():
        c, x, kind = s["case"], s["x"], s["x"].dtype
        batch, tokens, ch = x.shape
        groups, band = c["groups"], s["band"]
        count = (s["lengths"] * (ch // groups)).clamp(min=1).double()[None, :, None]

        at, there = _blocks(s)

        def over_bands(t):                        # [n, tokens, width] -> [n, bands, width]: each block's sum, then theirs
            part = (t[:, at.reshape(-1)].view(len(t), *at.shape, -1) * there[..., None]).sum(2)
            return torch.zeros(len(t), len(s["lengths"]), part.shape[2], dtype=t.dtype, device=t.device).index_add_(
                1, s["of"], part)

        def sums(t):                              # over a group's channels and a band's tokens
            return over_bands(t.view(batch, tokens, groups, -1).sum(-1, dtype=torch.float64))

        def spread(t):                            # [batch, bands, groups] -> [batch, tokens, channels]
            return t.float()[:, band].repeat_interleave(ch // groups, 2)

        xf = x.float()
        xc = xf - spread(sums(xf) / count)
        rstd = spread((sums(xc * xc) / count + 1e-5).rsqrt())
        xh = xc * rstd
        w = s["weight"].float()[band][None] if c["affine"] else 1.0
        z = xh * w + s["bias"].float()[band][None] if c["affine"] else xh
        y, slope = _act(z, c["act"])
        out = {"y": y.to(kind)}
        if "dy" in s:
            dz = s["dy"].float() * slope
            d = dz * w
            out["dx"] = (rstd * (d - spread(sums(d) / count) - xh * spread(sums(d * xh) / count))).to(kind)
            if c["affine"]:
                out["dw"] = over_bands((dz * xh).sum(0, True, dtype=torch.float64))[0].to(kind)
                out["db"] = over_bands(dz.sum(0, True, dtype=torch.float64))[0].to(kind)
        return out


def _blocks(s, reverse=False):
    """Tokens of each block [blocks, size], and which of them are there."""
    i = s["first"][:, None] + torch.arange(s["size"], device=s["first"].device)
    length, start = s["lengths"][s["of"]][:, None], s["offsets"][:-1][s["of"]][:, None]
    there = i < length
    return torch.where(there, start + (length - 1 - i if reverse else i), 0), there


def _gated(s):
    with torch.no_grad():
        c, kind, of = s["case"], s["x"].dtype, s["of"]
        at, there = _blocks(s)
        nb, size = at.shape
        batch, tokens, k = s["x"].shape

        def rows(t):                              # [batch, tokens, width] -> [blocks, batch * size, width]
            t = t.float()[:, at.reshape(-1)].view(batch, nb, size, -1) * there[None, :, :, None]
            return t.transpose(0, 1).reshape(nb, batch * size, -1)

        def back(t):
            t = t.view(nb, batch, size, -1).transpose(0, 1)
            out = torch.zeros(batch, tokens, t.shape[-1], device=t.device)
            out[:, at[there]] = t[:, there]
            return out

        def over_band(t):
            return torch.zeros(len(s["lengths"]), *t.shape[1:], device=t.device).index_add_(0, of, t)

        x, w = rows(s["x"]), s["weight"].float()
        wa, wu = w[of, 0], w[of, 1]
        a = torch.bmm(x, wa.transpose(1, 2).contiguous())
        u = torch.bmm(x, wu.transpose(1, 2).contiguous())
        if c["bias"]:
            a, u = a + s["bias"].float()[of, 0, None], u + s["bias"].float()[of, 1, None]
        f, slope = _act(a, c["act"])
        out = {"y": back(f * u).to(kind)}
        if "dy" in s:
            dy = rows(s["dy"])
            da, du = dy * u * slope, dy * f
            out["dx"] = back(torch.bmm(da, wa) + torch.bmm(du, wu)).to(kind)
            dw = [over_band(torch.bmm(t.transpose(1, 2).contiguous(), x)) for t in (da, du)]
            out["dw"] = torch.stack(dw, 1).to(kind)
            if c["bias"]:
                out["db"] = torch.stack([over_band(t.sum(1)) for t in (da, du)], 1).to(kind)
        return out


def _powers(s, n):
    """exp(log_decay)^n for each key head, [heads, *n.shape]; the exponents in 64 bits."""
    return (s["log_decay"].double().view(-1, *[1] * n.dim()) * n).exp().float()


def _decayed(s, a, b, c, reverse=False, state=None):
    """sum over the earlier (reverse: later) tokens j of a band of decay^|i - j| (a_i . b_j) c_j, and the state after it.

    a, b and c are [batch, tokens, heads, D] in 32 bits; where one side has more heads than there are decays, they
    share a key head: each has a result of its own (a), or their sums are one (b and c)."""
    at, there = _blocks(s, reverse)
    nb, size = at.shape
    batch, tokens, _, d = a.shape
    hk, dev = len(s["log_decay"]), a.device

    def heads(x):                                 # [batch, blocks, key heads, group, size, D]
        x = x[:, at.reshape(-1)].view(batch, nb, size, hk, -1, d) * there[None, :, :, None, None, None]
        return x.permute(0, 1, 3, 4, 2, 5).contiguous()

    shared = b.shape[2] > hk
    a, b, c = heads(a), heads(b), heads(c)
    i = torch.arange(size, device=dev)
    lag = i[:, None] - i
    near = torch.where(lag >= 0, _powers(s, lag.clamp(min=0)), 0.0)[:, None]
    out = torch.matmul(torch.matmul(a, b.transpose(-1, -2).contiguous()) * near, c)
    out = out.sum(3, keepdim=True) if shared else out
    # what each block adds to the state, as it stands at the block's end, and the state at each block's start
    count = there.sum(1)
    left = (count[:, None] - 1 - i).clamp(min=0)
    weighted = b * _powers(s, left).transpose(0, 1)[None, :, :, None, :, None]
    added = torch.matmul(weighted.transpose(-1, -2).contiguous(), c).sum(3).transpose(1, 2).reshape(batch, hk, nb, d * d)
    first, of, ends = s["first"], s["of"], s["first"] + count
    gap = first[:, None] - ends
    join = torch.where((of[:, None] == of) & (gap >= 0), _powers(s, gap.clamp(min=0)), 0.0)
    begin = torch.matmul(join, added)
    if state is not None:
        old = state.view(batch, -1, hk, d * d).transpose(1, 2)
        begin = begin + old[:, :, of] * _powers(s, first)[..., None]
    begin = begin.view(batch, hk, nb, d, d).transpose(1, 2)[:, :, :, None]
    out = out + torch.matmul(a * _powers(s, i + 1)[None, None, :, None, :, None], begin)
    full = torch.zeros(batch, tokens, out.shape[2] * out.shape[3], d, device=dev)
    full[:, at[there]] = out.permute(0, 1, 4, 2, 3, 5).reshape(batch, nb, size, -1, d)[:, there]
    if state is None:
        return full, None
    last = (s["lengths"][:, None] - ends).clamp(min=0)
    join = torch.where(torch.arange(len(s["lengths"]), device=dev)[:, None] == of, _powers(s, last), 0.0)
    after = torch.matmul(join, added) + old * _powers(s, s["lengths"])[..., None]
    return full, after.transpose(1, 2).reshape(state.shape)


def _decay(s):
    with torch.no_grad():
        kind, scale = s["q"].dtype, s["q"].shape[3] ** -0.5
        q, k, v = (s[n].float() for n in "qkv")
        if s["keep"] is not None:
            k, v = (torch.where(s["keep"][:, :, None, None], t, 0.0) for t in (k, v))
        o, after = _decayed(s, q, k, v, state=s["state"])
        out = {"o": (o * scale).to(kind)}
        if after is not None:
            s["state"].copy_(after)
            out["state"] = s["state"]
        if "do" in s:
            do = s["do"].float()
            out["dq"] = (_decayed(s, do, v, k)[0] * scale).to(kind)
            for name, a, b, c in (("dk", v, do, q), ("dv", k, q, do)):
                g = _decayed(s, a, b, c, reverse=True)[0] * scale
                out[name] = (g if s["keep"] is None else torch.where(s["keep"][:, :, None, None], g, 0.0)).to(kind)
        return out


def _step(s):
    b, h, d = s["q"].shape
    hk, pos, state = len(s["log_decay"]), s["pos"], s["state"]
    q, k, v = (s[n].float().view(b, hk, -1, d) for n in "qkv")
    g = s["log_decay"].exp()[None, :, None, None] * (pos > 0)[:, None, None, None]
    on = (pos >= 0)[:, None, None, None]
    state.copy_(torch.where(on, state * g + k.transpose(2, 3) * v, state))
    o = torch.where(on, torch.matmul(q, state) * d ** -0.5, 0.0)
    return {"o": o.view(b, h, d).to(s["q"].dtype), "state": state}


def run(s):
    op = s["case"]["op"]
    if own:
        return _own(s)
    if op.startswith("norm"):
        return _norm(s)
    if op.startswith("gated"):
        return _gated(s)
    return _step(s) if op == "step" else _decay(s)


def _own(s):
    from paper_2609_29119_amd import layers

    c = s["case"]
    if c["op"] == "step":
        o = layers.decay_step(s["q"], s["k"], s["v"], s["state"], s["pos"], s["log_decay"])
        return {"o": o, "state": s["state"]}
    if c["op"].startswith("decay"):
        o = layers.decay_attention(s["q"], s["k"], s["v"], s["offsets"], s["log_decay"], keep=s["keep"],
                                   state=s["state"])
        out = {"o": o.detach()}
        if s["state"] is not None:
            out["state"] = s["state"]
        if "do" in s:
            out.update(zip(("dq", "dk", "dv"), torch.autograd.grad(o, [s["q"], s["k"], s["v"]], s["do"])))
        return out
    act = None if c["act"] == "none" else c["act"]
    if c["op"].startswith("norm"):
        y = layers.band_norm(s["x"], s["offsets"], s["weight"], s["bias"], c["groups"], act)
    else:
        y = layers.band_gated(s["x"], s["weight"], s["offsets"], s["bias"], act)
    out = {"y": y.detach()}
    if "dy" in s:
        have = [(n, t) for n, t in (("dx", s["x"]), ("dw", s["weight"]), ("db", s["bias"])) if t is not None]
        out.update(zip([n for n, _ in have], torch.autograd.grad(y, [t for _, t in have], s["dy"])))
    return out


# ----------------------------------------------------------------------- work


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "step":
        b, h, hk, d = case["streams"], case["heads"], case["kv_heads"], case["dim"]
        return {"bytes": 8 * b * hk * d * d + e * b * d * (2 * h + 2 * hk) + 8 * b + 4 * hk,
                "flops": b * d * d * (3 * hk + 2 * h)}
    lengths, train = _lengths(case), case["op"].endswith("_train")
    rows = case["batch"] * sum(lengths)
    if case["op"].startswith("norm"):
        ch, w = case["channels"], 2 * len(lengths) * case["channels"] if case["affine"] else 0
        return {"bytes": e * (rows * ch * (4 if train else 2) + w * (2 if train else 1)),
                "flops": rows * ch * (40 if train else 14)}
    if case["op"].startswith("gated"):
        k, m = case["k"], case["m"]
        w = sum(1 for n in lengths if n) * 2 * m * (k + int(case["bias"]))
        if train:
            return {"bytes": e * (rows * (2 * k + 2 * m) + 2 * w), "flops": 12 * rows * k * m}
        return {"bytes": e * (rows * (k + m) + w), "flops": 4 * rows * k * m}
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    flops = rows * d * d * (2 * h + 3 * hk)
    if train:   # then one more sum over the past, and two over what follows
        return {"bytes": e * rows * d * (4 * h + 4 * hk), "flops": 2 * flops + 2 * rows * d * d * (3 * h + 2 * hk)}
    state = 8 * case["batch"] * len(lengths) * hk * d * d if case["state"] else 0
    return {"bytes": e * rows * d * (2 * h + 2 * hk) + state, "flops": flops}


# ---------------------------------------------------- the definition in 64 bits


def exact(case, seed):
    with torch.no_grad():
        s = prepare(case, seed)
        if case["op"] == "step":
            return _exact_step(s)
        if case["op"].startswith("norm"):
            return _exact_norm(s)
        return _exact_gated(s) if case["op"].startswith("gated") else _exact_decay(s)


def _exact_slope(z, how):
    """The activation and its derivative, from the functions' own names."""
    with torch.enable_grad():
        z = z.detach().requires_grad_(True)
        f = {"none": lambda t: t * 1.0, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu,
             "sigmoid": torch.sigmoid}[how](z)
        return f.detach(), torch.autograd.grad(f.sum(), z)[0]


def _exact_norm(s):
    c, ends, x = s["case"], s["offsets"].tolist(), s["x"]
    groups, ch = c["groups"], c["channels"]
    out = {"y": torch.zeros(x.shape, dtype=torch.float64, device=x.device)}
    if "dy" in s:
        out["dx"] = torch.zeros_like(out["y"])
        if c["affine"]:
            out.update(dw=torch.zeros(len(ends) - 1, ch, dtype=torch.float64, device=x.device),
                       db=torch.zeros(len(ends) - 1, ch, dtype=torch.float64, device=x.device))
    for g, (a, b) in enumerate(zip(ends, ends[1:])):
        if a == b:
            continue
        t = x[:, a:b].double().unflatten(2, (groups, -1))
        var, mean = torch.var_mean(t, (1, 3), correction=0, keepdim=True)
        r = 1.0 / (var + 1e-5).sqrt()
        xh = (t - mean) * r
        w = s["weight"][g].double().view(groups, -1) if c["affine"] else torch.ones_like(xh[0, 0])
        z = xh * w + (s["bias"][g].double().view(groups, -1) if c["affine"] else 0.0)
        f, slope = _exact_slope(z, c["act"])
        out["y"][:, a:b] = f.flatten(2)
        if "dy" in s:
            dz = s["dy"][:, a:b].double().unflatten(2, (groups, -1)) * slope
            d = dz * w
            d = r * (d - d.mean((1, 3), keepdim=True) - xh * (d * xh).mean((1, 3), keepdim=True))
            out["dx"][:, a:b] = d.flatten(2)
            if c["affine"]:
                out["dw"][g], out["db"][g] = (dz * xh).sum((0, 1)).flatten(), dz.sum((0, 1)).flatten()
    return out


def _exact_gated(s):
    c, ends, x, w = s["case"], s["offsets"].tolist(), s["x"], s["weight"].double()
    out = {"y": torch.zeros(*x.shape[:2], c["m"], dtype=torch.float64, device=x.device)}
    if "dy" in s:
        out.update(dx=torch.zeros(x.shape, dtype=torch.float64, device=x.device), dw=torch.zeros_like(w))
        if c["bias"]:
            out["db"] = torch.zeros_like(w[..., 0])
    for g, (a, b) in enumerate(zip(ends, ends[1:])):
        xg = x[:, a:b].double()
        gate, value = (xg @ w[g, i].T + (s["bias"][g, i].double() if c["bias"] else 0.0) for i in (0, 1))
        f, slope = _exact_slope(gate, c["act"])
        out["y"][:, a:b] = f * value
        if "dy" in s:
            dy = s["dy"][:, a:b].double()
            for i, d in enumerate((dy * value * slope, dy * f)):
                out["dx"][:, a:b] += d @ w[g, i]
                out["dw"][g, i] = d.flatten(0, 1).T @ xg.flatten(0, 1)
                if c["bias"]:
                    out["db"][g, i] = d.sum((0, 1))
    return out


def _exact_decay(s):
    """Every pair of tokens of a band, a stretch of later tokens against all before them."""
    c, lengths, ends, dev = s["case"], _lengths(s["case"]), s["offsets"].tolist(), s["q"].device
    h, hk, d, batch = c["heads"], c["kv_heads"], c["dim"], c["batch"]
    back, scale = "do" in s, d ** -0.5
    if batch * h * sum(m * m for m in lengths) * (d + 16) * (3 if back else 1) > 4e13:
        return None
    lam = s["log_decay"].double().repeat_interleave(h // hk)[None, :, None, None]
    double = {"dtype": torch.float64, "device": dev}
    out = {"o": torch.zeros(s["q"].shape, **double)}
    if c["state"]:
        out["state"] = s["state"].double().view(batch, len(lengths), hk, d, d)
    if back:
        out.update(dq=torch.zeros_like(out["o"]), dk=torch.zeros(s["k"].shape, **double),
                   dv=torch.zeros(s["k"].shape, **double))
    for g, (a, b) in enumerate(zip(ends, ends[1:])):
        q, k, v = (s[n][:, a:b].double().transpose(1, 2) for n in "qkv")
        if s["keep"] is not None:
            k, v = (t.masked_fill(~s["keep"][:, None, a:b, None], 0.0) for t in (k, v))
        k1, v1 = k, v
        k, v = (t.repeat_interleave(h // hk, 1) for t in (k, v))
        far = max(1, min(512, int(2e8 // (batch * h * max(b - a, 1)))))
        for i0 in range(0, b - a, far):
            i1 = min(i0 + far, b - a)
            lag = torch.arange(i0, i1, device=dev)[:, None] - torch.arange(i1, device=dev)
            fade = (lam * lag).exp().masked_fill(lag < 0, 0.0) * scale
            p = (q[:, :, i0:i1] @ k[:, :, :i1].mT) * fade
            o = p @ v[:, :, :i1]
            if c["state"]:
                i = torch.arange(i0 + 1, i1 + 1, device=dev)[None, None, :, None]
                old = s["state"].double().view(batch, len(lengths), hk, d, d)[:, g].repeat_interleave(h // hk, 1)
                o += (q[:, :, i0:i1] @ old) * (lam * i).exp() * scale
            out["o"][:, a + i0:a + i1] = o.transpose(1, 2)
            if back:
                do = s["do"][:, a + i0:a + i1].double().transpose(1, 2)
                dp = (do @ v[:, :, :i1].mT) * fade
                out["dq"][:, a + i0:a + i1] = (dp @ k[:, :, :i1]).transpose(1, 2)
                for name, x in (("dk", dp.mT @ q[:, :, i0:i1]), ("dv", p.mT @ do)):
                    out[name][:, a:a + i1] += x.unflatten(1, (hk, -1)).sum(2).transpose(1, 2)
        if back and s["keep"] is not None:
            for name in ("dk", "dv"):
                out[name][:, a:b].masked_fill_(~s["keep"][:, a:b, None, None], 0.0)
        if c["state"] and b > a:
            lk = s["log_decay"].double()[None, :, None, None]
            since = torch.arange(b - a - 1, -1, -1, device=dev)[None, None, :, None]
            out["state"][:, g] = out["state"][:, g] * (lk * (b - a)).exp() + (k1 * (lk * since).exp()).mT @ v1
    if c["state"]:
        out["state"] = out["state"].reshape(s["state"].shape)
    return out


def _exact_step(s):
    c, pos, lam = s["case"], s["pos"], s["log_decay"].double()
    h, hk, d = c["heads"], c["kv_heads"], c["dim"]
    state = s["state"].double()
    fresh, on = pos == 0, pos >= 0
    state[fresh] = 0.0
    state[on] = state[on] * lam.exp()[:, None, None] + torch.einsum("bhi,bhj->bhij", s["k"][on].double(), s["v"][on].double())
    rows = [torch.einsum("bi,bij->bj", s["q"][:, i].double(), state[:, i // (h // hk)]) for i in range(h)]
    o = torch.stack(rows, 1) * d ** -0.5
    o[~on] = 0.0
    return {"o": o, "state": state}
