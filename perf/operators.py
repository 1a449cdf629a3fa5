"""The calls whose speed matters to a user of the layers on the band layout.

A model behind the constant-Q transform works on a ragged row: C tokens
(coefficients) a signal, cut into bands of unequal length. Each case is one
call as such a program makes it: a matrix of its own for each band
(`band_linear`), rotary positions over time and frequency (`rotary`),
attention along each band with a sliding window and a few first tokens that
stay visible (`band_attention`), and the same attention for single tokens of
many streams over a ring cache (`attention_step`).

Band layouts are those of the repository's workloads, computed here from the
constant-Q definition, or free ones (any lengths, empty ones among them).
Where `own` is false, `run` computes the plain form in 32 bits: bands padded to
the longest, keys gathered for blocks of queries.
"""
import math
import random

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}

# ---------------------------------------------------------------------- cases

_TINY = {"layout": "cq", "fs": 22050.0, "fmin": 110.0, "bins": 12, "n": 16384}
_SINGLE = {"layout": "cq", "fs": 44100.0, "fmin": 32.7, "bins": 48, "n": 44100}
_TRAIN = {"layout": "cq", "fs": 44100.0, "fmin": 40.0, "bins": 24, "n": 220500}
_STRESS = {"layout": "cq", "fs": 22050.0, "fmin": 55.0, "bins": 36, "n": 88200}


def listed():
    return [
        # the first layer on one second of audio: (re, im) of each coefficient to 32 features, the smallest product
        {"name": "embed_single", "op": "linear", **_SINGLE, "batch": 1, "dtype": "f32", "k": 2, "m": 32, "bias": True},
        # the last layer of a mask estimator on a batch of clips: an odd width on either side
        {"name": "mask_stress", "op": "linear", **_STRESS, "batch": 8, "dtype": "f16", "k": 193, "m": 77, "bias": True},
        # a hidden layer in training, with the gradients of input, weights and bias: 5 s clips
        {"name": "hidden_train", "op": "linear_train", **_TRAIN, "batch": 2, "dtype": "bf16", "k": 128, "m": 128,
         "bias": True},
        # positions of one token of each of 64 streams: latency
        {"name": "rotary_step", "op": "rotary", "layout": "free", "bands": 1, "tokens": 64, "shape_seed": 0, "batch": 1,
         "dtype": "bf16", "heads": 8, "kv_heads": 2, "dim": 64, "axes": 2, "interleaved": False, "rotated": 64},
        # time, band and channel as axes on a clip, adjacent pairs, part of the head rotated, 32 bits
        {"name": "rotary_axes", "op": "rotary", **_STRESS, "batch": 1, "dtype": "f32", "heads": 6, "kv_heads": 3,
         "dim": 80, "axes": 3, "interleaved": True, "rotated": 60},
        # (time, frequency) positions in training: 5 s clips, there and back
        {"name": "rotary_train", "op": "rotary_train", **_TRAIN, "batch": 2, "dtype": "bf16", "heads": 8, "kv_heads": 2,
         "dim": 64, "axes": 2, "interleaved": False, "rotated": 64},
        # a short clip in 32 bits, both sides of the window visible: the smallest attention
        {"name": "attention_clip", "op": "attention", **_TINY, "batch": 1, "dtype": "f32", "heads": 4, "kv_heads": 4,
         "dim": 32, "left": 63, "right": 63, "sinks": 0, "keep": False},
        # attention in training over every band of 5 s clips: silent coefficients dropped, shared heads, sinks
        {"name": "attention_train", "op": "attention_train", **_TRAIN, "batch": 2, "dtype": "bf16", "heads": 8,
         "kv_heads": 2, "dim": 64, "left": 255, "right": 0, "sinks": 4, "keep": True},
        # one long stream read in (the prompt of a streaming session): the largest product
        {"name": "attention_long", "op": "attention", "layout": "free", "bands": 1, "tokens": 131072, "shape_seed": 0,
         "batch": 1, "dtype": "bf16", "heads": 8, "kv_heads": 2, "dim": 128, "left": 1023, "right": 0, "sinks": 4,
         "keep": False},
        # one token of one stream: latency
        {"name": "step_one", "op": "step", "streams": 1, "dtype": "bf16", "heads": 8, "kv_heads": 2, "dim": 64,
         "window": 256, "sinks": 4},
        # one token of every band of 16 signals, each band a stream of its own
        {"name": "step_bands", "op": "step", "streams": 3536, "dtype": "bf16", "heads": 8, "kv_heads": 2, "dim": 64,
         "window": 256, "sinks": 4},
        # a few streams with a long memory: the cache is split and the parts joined
        {"name": "step_long", "op": "step", "streams": 4, "dtype": "f16", "heads": 8, "kv_heads": 2, "dim": 128,
         "window": 131072, "sinks": 4},
    ]


def _log(rng, lo, hi):
    return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def draw(rng):
    """One more case: sizes spread over the logarithm of the range."""
    op = rng.choice(["linear", "linear", "linear_train", "rotary", "rotary_train", "attention", "attention",
                     "attention_train", "step", "step"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    kv = rng.choice([1, 2, 3, 4])
    heads = kv * rng.choice([1, 2, 3, 4])
    dim = rng.choice([16, 32, 40, 64, 64, 80, 96, 128, rng.randint(3, 128)])
    if op == "step":
        window = _log(rng, 1, 131072)
        most = 5e8 / (2 * kv * dim * window * (4 if dtype == "f32" else 2))
        return {"op": op, "streams": max(1, min(_log(rng, 1, 4096), int(most))), "dtype": dtype, "heads": heads,
                "kv_heads": kv, "dim": dim, "window": window, "sinks": rng.choice([0, 1, 4, rng.randint(0, 70)])}
    if rng.random() < 0.6:
        fs = rng.choice([16000.0, 22050.0, 44100.0])
        c = {"op": op, "layout": "cq", "fs": fs, "fmin": round(rng.uniform(30.0, 120.0), 1),
             "bins": rng.randint(4, 48), "n": 2 * _log(rng, 2000, 110250)}
    else:
        c = {"op": op, "layout": "free", "bands": _log(rng, 1, 300), "tokens": _log(rng, 1, 200000),
             "shape_seed": rng.randrange(1 << 20)}
    lengths = _lengths(c)
    tokens, padded = max(1, sum(lengths)), len(lengths) * max(lengths + [1])
    c["dtype"] = dtype
    if op.startswith("linear"):
        k, m = (2 if rng.random() < 0.2 else _log(rng, 3, 512)), _log(rng, 1, 512)
        share = max(1, int(min(450e3 * 128 / max(k, m) / tokens, 2.8e6 * 128 / max(k, m) / padded, 16)))
        c.update(batch=_log(rng, 1, share), k=k, m=m, bias=rng.random() < 0.7)
        return c
    share = max(1, int(min(450e3 * 8 * 64 / (heads * dim) / tokens, 16)))
    c.update(batch=_log(rng, 1, share), heads=heads, kv_heads=kv, dim=dim)
    if op.startswith("rotary"):
        c.update(axes=rng.randint(1, 4), interleaved=rng.random() < 0.4)
        c["rotated"] = 2 * max(1, dim // 2 if rng.random() < 0.6 else rng.randint(1, dim // 2))
        return c
    c.update(left=_log(rng, 1, 1024) - 1, right=rng.choice([0, 0, _log(rng, 1, 256) - 1]),
             sinks=rng.choice([0, 1, 4, rng.randint(0, 40)]), keep=rng.random() < 0.4)
    cost = lambda: c["batch"] * tokens * heads * (c["left"] + c["right"] + c["sinks"] + 160)  # noqa: E731
    while cost() > 0.6e9 and c["batch"] > 1:
        c["batch"] -= 1
    while cost() > 0.6e9 and c["left"] + c["right"] > 8:
        c["left"] //= 2
        c["right"] //= 2
    return c


def _lengths(case):
    """Tokens of each band."""
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

    def normal(*shape, by=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * by).to(kind)

    if case["op"] == "step":
        b, hk, d, slots = case["streams"], case["kv_heads"], case["dim"], case["window"] + case["sinks"]
        s = {"case": case, "q": normal(b, case["heads"], d, by=1.5), "k": normal(b, hk, d), "v": normal(b, hk, d),
             "k_cache": normal(b, hk, slots, d), "v_cache": normal(b, hk, slots, d)}
        # most streams are past their first window, some are young, a few have no token in this step
        age = torch.rand(b, generator=gen, device="cuda")
        far = torch.randint(slots, 3 * slots + 8, (b,), generator=gen, device="cuda")
        young = torch.randint(0, slots, (b,), generator=gen, device="cuda")
        s["pos"] = torch.where(age < 0.85, far, torch.where(age < 0.97, young, -1)) if b > 8 else far
        return s
    lengths, batch = _lengths(case), case["batch"]
    tokens = sum(lengths)
    n = torch.tensor(lengths, dtype=torch.int64)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]).cuda()
    s = {"case": case, "offsets": offsets}
    if case["op"].startswith("linear"):
        k, m = case["k"], case["m"]
        # features of a band have the band's own level: low bands are louder
        level = torch.logspace(0.5, -0.5, len(lengths), device="cuda").repeat_interleave(n.cuda())
        s["x"] = (torch.randn(batch, tokens, k, generator=gen, device="cuda") * level[None, :, None]).to(kind)
        s["weight"] = normal(len(lengths), m, k, by=k ** -0.5)
        s["bias"] = normal(len(lengths), m, by=0.1) if case["bias"] else None
        if case["op"] == "linear_train":
            s["dy"] = normal(batch, tokens, m)
            for name in ("x", "weight", "bias"):
                if s[name] is not None:
                    s[name].requires_grad_(True)
        # the plain form's plan: where each band's rows lie when all are padded to the longest
        band = torch.arange(len(lengths), device="cuda").repeat_interleave(n.cuda())
        within = torch.arange(tokens, device="cuda") - offsets[band]
        s["longest"] = max(max(lengths), 1)
        s["back"] = band * s["longest"] + within
        return s
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    # query and key are parts of one projection's output, as a model has them
    both = normal(batch, tokens, h + hk, d)
    s["q"], s["k"] = both[:, :, :h], both[:, :, h:]
    if case["op"].startswith("rotary"):
        pairs, axes = case["rotated"] // 2, case["axes"]
        s["sections"] = [pairs * (a + 1) // axes - pairs * a // axes for a in range(axes)]
        s["freqs"] = torch.cat([10000.0 ** (-torch.arange(p, dtype=torch.float64) / max(p, 1)) for p in s["sections"]]
                               ).float().cuda()
        # time in hops of the longest band from a random start, the band's number, then ordinals
        m = n.cuda().repeat_interleave(n.cuda()).double()
        within = torch.arange(tokens, device="cuda") - offsets[:-1].repeat_interleave(n.cuda())
        start = torch.rand(1, generator=gen, device="cuda", dtype=torch.float64) * 5000.0
        axis = [start + within * (max(max(lengths), 1) / m),
                torch.arange(len(lengths), device="cuda").repeat_interleave(n.cuda()).double(),
                (torch.arange(tokens, device="cuda") % 5).double(), (torch.arange(tokens, device="cuda") % 7).double()]
        s["positions"] = torch.stack(axis[:axes]).contiguous()
        if case["op"] == "rotary_train":
            s["dq"], s["dk"] = normal(batch, tokens, h, d), normal(batch, tokens, hk, d)
            s["q"] = s["q"].detach().requires_grad_(True)
            s["k"] = s["k"].detach().requires_grad_(True)
        return s
    s["v"] = normal(batch, tokens, hk, d)
    s["keep"] = None
    if case["keep"]:  # silent coefficients: one in eight, and one stretch that leaves whole windows empty
        keep = torch.rand(batch, tokens, generator=gen, device="cuda") > 0.125
        at = int(torch.randint(0, tokens, (1,), generator=gen, device="cuda"))
        keep[:, at:at + 2 * case["left"] + 40] = False
        s["keep"] = keep
    if case["op"] == "attention_train":
        s["do"] = normal(batch, tokens, h, d)
        for name in ("q", "k", "v"):
            s[name] = s[name].detach().requires_grad_(True)
    # the plain form's plan: blocks of queries of one band, and each block's keys
    size = 512 if case["left"] + case["right"] >= 512 else 128
    blocks = (n + size - 1) // size
    band = torch.arange(len(lengths)).repeat_interleave(blocks)
    first = torch.arange(int(blocks.sum())) - (blocks.cumsum(0) - blocks)[band]
    s["size"], s["band"], s["first"] = size, band.cuda(), (first * size).cuda()
    s["lengths"] = n.cuda()
    return s


# ---------------------------------------------------------------- plain forms


def _padded(x, s):
    """[batch, C, K] -> [bands, batch * longest, K] in 32 bits, zeros past a band's end."""
    bands, batch = len(s["offsets"]) - 1, x.shape[0]
    full = torch.zeros(batch, bands * s["longest"], x.shape[2], device=x.device)
    full[:, s["back"]] = x.float()
    return full.view(batch, bands, s["longest"], -1).transpose(0, 1).reshape(bands, batch * s["longest"], -1)


def _rows(y, s, batch):
    bands = y.shape[0]
    return y.view(bands, batch, s["longest"], -1).transpose(0, 1).reshape(batch, bands * s["longest"], -1)[:, s["back"]]


def _linear(s):
    with torch.no_grad():
        x, w, bias, kind = s["x"], s["weight"], s["bias"], s["x"].dtype
        xp, wf = _padded(x, s), w.float()
        yp = torch.bmm(xp, wf.transpose(1, 2).contiguous())
        if bias is not None:
            yp = yp + bias.float()[:, None, :]
        out = {"y": _rows(yp, s, x.shape[0]).to(kind)}
        if "dy" in s:
            dyp = _padded(s["dy"], s)
            out["dx"] = _rows(torch.bmm(dyp, wf), s, x.shape[0]).to(kind)
            out["dw"] = torch.bmm(dyp.transpose(1, 2).contiguous(), xp).to(kind)
            if bias is not None:
                out["db"] = dyp.sum(1).to(kind)
        return out


def _turned(x, s, sign):
    """The pairs of x [batch, C, heads, D] turned by their angles. The angles are the only thing in 64 bits:
    a 32-bit product of a position in the thousands and a frequency is off by more than the result's rounding."""
    axis = torch.repeat_interleave(torch.arange(len(s["sections"]), device=x.device),
                                   torch.tensor(s["sections"], device=x.device), output_size=len(s["freqs"]))
    angle = s["positions"][axis].T * s["freqs"].double()
    cos, sin = angle.cos().float()[None, :, None], sign * angle.sin().float()[None, :, None]
    r = s["case"]["rotated"]
    xf, y = x.float(), x.float().clone()
    at = (slice(0, r, 2), slice(1, r, 2)) if s["case"]["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
    a, b = xf[..., at[0]], xf[..., at[1]]
    y[..., at[0]] = a * cos - b * sin
    y[..., at[1]] = a * sin + b * cos
    return y.to(x.dtype)


def _attention(s):
    with torch.no_grad():
        c, kind = s["case"], s["q"].dtype
        batch, tokens, h, d = s["q"].shape
        hk, size, scale = c["kv_heads"], s["size"], s["q"].shape[3] ** -0.5
        dev = s["q"].device
        start, length = s["offsets"][:-1][s["band"]][:, None], s["lengths"][s["band"]][:, None]
        i = s["first"][:, None] + torch.arange(size, device=dev)                                   # [nb, size]
        near = s["first"][:, None] - c["left"] + torch.arange(size + c["left"] + c["right"], device=dev)
        sink = torch.arange(c["sinks"], device=dev).expand(len(i), -1)
        sink = torch.where(sink < s["first"][:, None] - c["left"], sink, -1)                       # not seen twice
        j = torch.cat([sink, near], 1)                                                             # [nb, keys]
        there = (j >= 0) & (j < length)
        see = there[:, None] & (j[:, None] <= i[..., None] + c["right"])
        see &= (j[:, None] >= i[..., None] - c["left"]) | (j[:, None] < c["sinks"])
        qi, kj = (start + i).clamp(max=max(tokens - 1, 0)), (start + j).clamp(0, max(tokens - 1, 0))
        see = see[None].expand(batch, -1, -1, -1)
        if s["keep"] is not None:
            see = see & s["keep"][:, kj][:, :, None]
        see = see[:, :, None, None]                                                  # [batch, nb, 1, 1, size, keys]

        def heads(x, at):                                                            # [batch, nb, hk, group, at, D]
            x = x.float()[:, at.reshape(-1)].view(batch, *at.shape, hk, -1, d)
            return x.permute(0, 1, 3, 4, 2, 5).contiguous()

        q, k, v = heads(s["q"], qi), heads(s["k"], kj), heads(s["v"], kj)
        logit = torch.matmul(q, k.transpose(-1, -2)) * scale
        logit = logit.masked_fill(~see, float("-inf"))
        top = logit.amax(-1, keepdim=True).clamp(min=-3e38)
        p = (logit - top).exp()
        total = p.sum(-1, keepdim=True)
        p = p / torch.where(total > 0, total, 1.0)
        o = torch.matmul(p, v)
        mine = (i < length).reshape(-1)
        at = (start + i).reshape(-1)[mine]

        def tokens_of(x):                                                            # back to [batch, C, h, D]
            x = x.permute(0, 1, 4, 2, 3, 5).reshape(batch, -1, h, d)
            full = torch.zeros(batch, tokens, h, d, device=dev)
            full[:, at] = x[:, mine]
            return full

        out = {"o": tokens_of(o).to(kind)}
        if "do" in s:
            do = heads(s["do"], qi) * (i < length)[None, :, None, None, :, None]
            dp = torch.matmul(do, v.transpose(-1, -2))
            ds = p * (dp - (do * o).sum(-1, keepdim=True)) * scale
            out["dq"] = tokens_of(torch.matmul(ds, k)).to(kind)
            to = torch.where(there, start + j, 0).reshape(-1)
            for name, left, right in (("dk", ds, q), ("dv", p, do)):
                part = torch.matmul(left.transpose(-1, -2), right).sum(3) * there[None, :, None, :, None]
                part = part.permute(0, 1, 3, 2, 4).reshape(batch, -1, hk, d)
                out[name] = torch.zeros(batch, tokens, hk, d, device=dev).index_add_(1, to, part).to(kind)
        return out


def _step(s):
    c, kind = s["case"], s["q"].dtype
    b, h, d = s["q"].shape
    hk, slots, pos = c["kv_heads"], s["k_cache"].shape[2], s["pos"]
    slot = torch.where(pos < c["sinks"], pos, c["sinks"] + (pos - c["sinks"]) % c["window"]).clamp(min=0)
    rows, at = torch.arange(b, device=pos.device), (pos >= 0)[:, None, None]
    for cache, new in ((s["k_cache"], s["k"]), (s["v_cache"], s["v"])):
        cache[rows, :, slot] = torch.where(at, new, cache[rows, :, slot])
    see = torch.arange(slots, device=pos.device) <= pos[:, None]
    q = s["q"].float().view(b, hk, h // hk, d)
    logit = torch.matmul(q, s["k_cache"].float().transpose(-1, -2)) * d ** -0.5
    logit = logit.masked_fill(~see[:, None, None], float("-inf"))
    p = (logit - logit.amax(-1, keepdim=True).clamp(min=-3e38)).exp()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p / torch.where(total > 0, total, 1.0), s["v_cache"].float())
    return {"o": o.view(b, h, d).to(kind), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def run(s):
    c = s["case"]
    if own:
        return _own(s)
    if c["op"].startswith("linear"):
        return _linear(s)
    if c["op"].startswith("rotary"):
        with torch.no_grad():
            out = {"q": _turned(s["q"], s, 1.0), "k": _turned(s["k"], s, 1.0)}
            if "dq" in s:
                out.update(dq=_turned(s["dq"], s, -1.0), dk=_turned(s["dk"], s, -1.0))
        return out
    return _step(s) if c["op"] == "step" else _attention(s)


def _own(s):
    from paper_2609_29119_amd import layers

    c = s["case"]
    if c["op"] == "step":
        o = layers.attention_step(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["pos"], c["sinks"])
        return {"o": o, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if c["op"].startswith("linear"):
        y = layers.band_linear(s["x"], s["weight"], s["offsets"], s["bias"])
        out = {"y": y.detach()}
        if "dy" in s:
            names = ["dx", "dw", "db"][:2 if s["bias"] is None else 3]
            out.update(zip(names, torch.autograd.grad(y, [s["x"], s["weight"], s["bias"]][:len(names)], s["dy"])))
        return out
    if c["op"].startswith("rotary"):
        q, k = layers.rotary(s["q"], s["k"], s["positions"], s["freqs"], s["sections"], c["interleaved"])
        out = {"q": q.detach(), "k": k.detach()}
        if "dq" in s:
            out.update(zip(("dq", "dk"), torch.autograd.grad([q, k], [s["q"], s["k"]], [s["dq"], s["dk"]])))
        return out
    o = layers.band_attention(s["q"], s["k"], s["v"], s["offsets"], c["left"], c["right"], c["sinks"], keep=s["keep"])
    out = {"o": o.detach()}
    if "do" in s:
        out.update(zip(("dq", "dk", "dv"), torch.autograd.grad(o, [s["q"], s["k"], s["v"]], s["do"])))
    return out


# ----------------------------------------------------------------------- work


def _pairs(case):
    """Visible (query, key) pairs of one signal and head, with every key kept."""
    total, left, right, sinks = 0, case["left"], case["right"], case["sinks"]
    for m in _lengths(case):
        i = torch.arange(m, dtype=torch.int64)
        lo, hi = (i - left).clamp(min=0), (i + right).clamp(max=m - 1)
        total += int((hi - lo + 1 + torch.minimum(torch.full_like(i, sinks), lo)).sum())
    return total


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "step":
        s = prepare(case, 1)
        seen = int((s["pos"] + 1).clamp(max=s["k_cache"].shape[2]).sum())
        b, h, hk, d = case["streams"], case["heads"], case["kv_heads"], case["dim"]
        return {"bytes": e * d * (2 * seen * hk + 2 * b * h + 4 * b * hk) + 8 * b, "flops": 4 * seen * h * d}
    lengths, batch = _lengths(case), case["batch"]
    rows = batch * sum(lengths)
    if case["op"].startswith("linear"):
        k, m, w = case["k"], case["m"], len(lengths) * case["m"] * (case["k"] + int(case["bias"]))
        if case["op"] == "linear":
            return {"bytes": e * (rows * (k + m) + w), "flops": 2 * rows * k * m}
        return {"bytes": e * (rows * (2 * k + 2 * m) + 2 * w), "flops": 6 * rows * k * m}
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    if case["op"].startswith("rotary"):
        times = 2 if case["op"] == "rotary_train" else 1
        return {"bytes": times * 2 * e * rows * (h + hk) * d + 8 * case["axes"] * sum(lengths),
                "flops": times * 3 * rows * (h + hk) * case["rotated"]}
    pairs = batch * h * _pairs(case)
    if case["op"] == "attention":
        return {"bytes": e * rows * d * (2 * h + 2 * hk), "flops": 4 * d * pairs}
    # o, then q, k, v, do read and dq, dk, dv written
    return {"bytes": e * rows * d * (4 * h + 4 * hk), "flops": 14 * d * pairs}


# ---------------------------------------------------- the definition in 64 bits


def exact(case, seed):
    with torch.no_grad():
        s = prepare(case, seed)
        if case["op"] == "step":
            return _exact_step(s)
        if case["op"].startswith("linear"):
            return _exact_linear(s)
        return _exact_rotary(s) if case["op"].startswith("rotary") else _exact_attention(s)


def _exact_linear(s):
    ends = s["offsets"].tolist()
    x, w = s["x"], s["weight"].double()
    out = {"y": torch.zeros(*x.shape[:2], w.shape[1], dtype=torch.float64, device=x.device)}
    if "dy" in s:
        out.update(dx=torch.zeros(*x.shape, dtype=torch.float64, device=x.device), dw=torch.zeros_like(w))
        if s["bias"] is not None:
            out["db"] = torch.zeros_like(w[:, :, 0])
    for g, (a, b) in enumerate(zip(ends, ends[1:])):
        xg = x[:, a:b].double()
        out["y"][:, a:b] = xg @ w[g].T + (s["bias"][g].double() if s["bias"] is not None else 0.0)
        if "dy" in s:
            dy = s["dy"][:, a:b].double()
            out["dx"][:, a:b] = dy @ w[g]
            out["dw"][g] = dy.reshape(-1, dy.shape[2]).T @ xg.reshape(-1, xg.shape[2])
            if s["bias"] is not None:
                out["db"][g] = dy.sum((0, 1))
    return out


def _exact_rotary(s):
    c, r = s["case"], s["case"]["rotated"]
    rows, at = [], 0
    for axis, count in enumerate(s["sections"]):
        rows += [s["positions"][axis] * s["freqs"][at + p].double() for p in range(count)]
        at += count
    turn = torch.polar(torch.ones_like(torch.stack(rows, 1)), torch.stack(rows, 1))[None, :, None, :]

    def turned(x, by):
        y = x.double().clone()
        pair = (lambda t: t.unflatten(-1, (r // 2, 2))) if c["interleaved"] else (
            lambda t: t.unflatten(-1, (2, r // 2)).transpose(-1, -2))
        z = torch.view_as_complex(pair(y[..., :r]).contiguous()) * by
        z = torch.view_as_real(z)
        y[..., :r] = (z if c["interleaved"] else z.transpose(-1, -2)).flatten(-2)
        return y

    out = {"q": turned(s["q"], turn), "k": turned(s["k"], turn)}
    if "dq" in s:
        out.update(dq=turned(s["dq"], turn.conj()), dk=turned(s["dk"], turn.conj()))
    return out


def _exact_attention(s):
    """Band by band, a stretch of queries at a time against a slice of the keys."""
    c, ends = s["case"], s["offsets"].tolist()
    h, hk, d = c["heads"], c["kv_heads"], c["dim"]
    left, right, sinks = c["left"], c["right"], c["sinks"]
    back, dev = "do" in s, s["q"].device
    out = {"o": torch.zeros(s["q"].shape, dtype=torch.float64, device=dev)}
    if back:
        out.update(dq=torch.zeros_like(out["o"]), dk=torch.zeros(s["k"].shape, dtype=torch.float64, device=dev),
                   dv=torch.zeros(s["k"].shape, dtype=torch.float64, device=dev))
    for a, b in zip(ends, ends[1:]):
        for i0 in range(0, b - a, 256):
            i1 = min(i0 + 256, b - a)
            j0, j1 = max(0, i0 - left), min(b - a, i1 + right)
            some = min(sinks, j0)
            js = torch.cat([torch.arange(some, device=dev), torch.arange(j0, j1, device=dev)])
            i = torch.arange(i0, i1, device=dev)[:, None]
            hide = (js > i + right) | ((js < i - left) & (js >= sinks))
            hide = hide[None].expand(c["batch"], -1, -1)
            if s["keep"] is not None:
                hide = hide | ~s["keep"][:, a + js][:, None]
            hide = hide[:, None]
            q = s["q"][:, a + i0:a + i1].double().transpose(1, 2)
            k = s["k"][:, a + js].double().transpose(1, 2).repeat_interleave(h // hk, 1)
            v = s["v"][:, a + js].double().transpose(1, 2).repeat_interleave(h // hk, 1)
            p = (q @ k.mT * d ** -0.5).masked_fill(hide, float("-inf")).softmax(-1).nan_to_num(0.0)
            o = p @ v
            out["o"][:, a + i0:a + i1] = o.transpose(1, 2)
            if back:
                do = s["do"][:, a + i0:a + i1].double().transpose(1, 2)
                ds = p * (do @ v.mT - (do * o).sum(-1, keepdim=True)) * d ** -0.5
                out["dq"][:, a + i0:a + i1] = (ds @ k).transpose(1, 2)
                for name, x in (("dk", ds.mT @ q), ("dv", p.mT @ do)):
                    x = x.unflatten(1, (hk, h // hk)).sum(2).transpose(1, 2)
                    out[name][:, a:a + some] += x[:, :some]
                    out[name][:, a + j0:a + j1] += x[:, some:]
    return out


def _exact_step(s):
    """The visible tokens of each stream, one of its heads at a time."""
    c = s["case"]
    if c["streams"] * c["heads"] > 40000:
        return None
    pos, sinks, window = s["pos"].tolist(), c["sinks"], c["window"]
    k, v = s["k_cache"], s["v_cache"]
    for b, t in enumerate(pos):
        if t >= 0:
            at = t if t < sinks else sinks + (t - sinks) % window
            k[b, :, at], v[b, :, at] = s["k"][b], s["v"][b]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device=k.device)
    group = c["heads"] // c["kv_heads"]
    for b, t in enumerate(pos):
        seen = min(t + 1, sinks + window)
        if seen > 0:
            q = s["q"][b].double().view(c["kv_heads"], group, -1)
            p = (q @ k[b, :, :seen].double().mT * c["dim"] ** -0.5).softmax(-1)
            o[b] = (p @ v[b, :, :seen].double()).view(c["heads"], -1)
    # the caches only hold copies of inputs: compared with the plain form's
    return {"o": o, "k_cache": k.double(), "v_cache": v.double()}
