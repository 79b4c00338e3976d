"""The operators of token-predicting tenants: what they compute, over the sizes their users have.

A case is a dict of plain values; its ``kind`` names the public entry point it goes through:

  qk       ``jn_qk_norm_rope``: norms of queries and keys for each head and their rotation by positions of one to
           three axes, in one pass over the rows of a fused q | k | v projection
  qk_bwd   ``jn_qk_norm_rope_bwd``: the gradients of its input rows and of the two norms' gains
  tokens   ``jn_tenant_tokens_fwd_bwd``: every tenant's softmax cross entropy over its own vocabulary, with the
           gradients of its head's weights and, where asked for, of the rows it reads
  decode   ``jn_tenant_tokens_decode``: the likeliest token of each row and its log-probability

``own`` says which side ``run`` takes: these entry points, or the same definitions in elementary torch operations.
Shapes follow from a case's numbers alone, values from the seed that ``prepare`` gets.
"""
from __future__ import annotations

import math
from typing import List

import torch

own = False

DEV = "cuda"
EPS = 1e-6
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


# ------------------------------------------------------------------ cases ---


def listed() -> List[dict]:
    return [
        # One robot's decode step: a new token of each of eight streams, far into their episodes, grouped heads. Latency.
        dict(name="qk_8_rows", kind="qk", rows=8, heads=16, kv=2, hd=128, axes=3, norm=True, interleaved=True,
             theta=1e6, far=250_000),
        # One observation (an image and its instruction) through one layer of the 2B-shaped backbone, one axis.
        dict(name="qk_301_rows", kind="qk", rows=301, heads=8, kv=1, hd=256, axes=1, norm=True, interleaved=False,
             theta=1e4, far=0),
        # A training group's packed rows (eight tenants x 32 samples), three position axes, wide heads.
        dict(name="qk_75k_rows", kind="qk", rows=75_923, heads=16, kv=2, hd=128, axes=3, norm=True, interleaved=False,
             theta=1e6, far=0),
        # Gradients for a small tenant's own samples, heads of an odd width.
        dict(name="qk_bwd_1k_rows", kind="qk_bwd", rows=1_021, heads=12, kv=4, hd=96, axes=3, norm=True,
             interleaved=True, theta=1e5, far=0),
        # Gradients over a whole group's rows.
        dict(name="qk_bwd_75k_rows", kind="qk_bwd", rows=75_923, heads=16, kv=2, hd=128, axes=3, norm=True,
             interleaved=False, theta=1e6, far=0),
        # The smallest training call: one tenant, seven action tokens in 256 bins. Launches and host work.
        dict(name="tokens_bins_7", kind="tokens", tenants=1, rows=7, vocab=256, d=768, dh=False, empty=False),
        # Eight tenants of unequal sizes with discretised actions, one of them without any target in this group.
        dict(name="tokens_bins_8x", kind="tokens", tenants=8, rows=2_003, vocab=2_049, d=768, dh=True, empty=True),
        # One tenant's instruction and answer tokens over a language vocabulary.
        dict(name="tokens_32k_700", kind="tokens", tenants=1, rows=701, vocab=32_003, d=2048, dh=True, empty=False),
        # A group's text tokens over a large vocabulary: bound by the matrix cores.
        dict(name="tokens_160k_8k", kind="tokens", tenants=1, rows=8_192, vocab=160_001, d=2048, dh=True, empty=False),
        # Serving one robot's next action token: launches, then the head's weights.
        dict(name="decode_1_bins", kind="decode", tenants=1, rows=1, vocab=1_024, d=768),
        # Eight tenants' streams, one token each, every tenant with a vocabulary head of its own.
        dict(name="decode_8x1", kind="decode", tenants=8, rows=8, vocab=32_003, d=2048),
        # A serving batch over a large vocabulary: bound by reading the weights.
        dict(name="decode_160k_61", kind="decode", tenants=1, rows=61, vocab=160_001, d=2048),
    ]


# (query heads, key/value heads, head width) of the backbones' variants, and of narrower ones
_HEADS = ((8, 8, 256), (8, 1, 256), (16, 2, 128), (16, 16, 128), (12, 12, 64), (12, 4, 96), (4, 4, 32), (6, 2, 80))
_WIDTHS = (128, 768, 1024, 2048)


def _log(rng, lo: int, hi: int) -> int:
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng) -> dict:
    kind = rng.choice(("qk", "qk_bwd", "tokens", "decode"))
    if kind in ("qk", "qk_bwd"):
        heads, kv, hd = rng.choice(_HEADS)
        most = 75_923 * 18 * 128 // ((heads + kv) * hd)
        return dict(kind=kind, rows=_log(rng, 1, min(75_923, most)), heads=heads, kv=kv, hd=hd,
                    axes=rng.choice((1, 2, 3)), norm=rng.random() < 0.8, interleaved=rng.random() < 0.5,
                    theta=rng.choice((1e4, 1e5, 1e6)), far=rng.choice((0, 0, _log(rng, 1, 1_000_000))))
    d = rng.choice(_WIDTHS)
    tenants = rng.choice((1, 1, 2, 3, 5, 8))
    if kind == "decode":
        return dict(kind=kind, tenants=tenants, rows=_log(rng, tenants, 64), d=d,
                    vocab=_log(rng, 100, 160_001 // tenants))
    dh = rng.random() < 0.5
    return dict(kind=kind, tenants=tenants, rows=_log(rng, tenants, 8_192), vocab=_log(rng, 200, 160_001 // tenants),
                d=d, dh=dh, empty=tenants > 1 and rng.random() < 0.3)


def _sections(c: dict) -> List[int]:
    """Pairs of each axis: a half for the first of three (time) rounded so that all add up."""
    half, axes = c["hd"] // 2, c["axes"]
    rest = half // 4 if axes == 3 else half // 3
    return [half - rest * (axes - 1)] + [rest] * (axes - 1)


def _pair_axis(c: dict) -> List[int]:
    """Axis of every pair of a head: runs of sections[a] pairs, or dealt in turn while an axis has pairs left."""
    sec, axes, half = _sections(c), c["axes"], c["hd"] // 2
    if not c["interleaved"]:
        return [a for a in range(axes) for _ in range(sec[a])]
    return [i % axes if i // axes < sec[i % axes] else 0 for i in range(half)]


def _shares(c: dict) -> List[tuple]:
    """(target rows, vocabulary) of every tenant: unequal shares of the rows, vocabularies of several sizes."""
    g = c["tenants"]
    live = g - 1 if c.get("empty") else g
    w = [1.0 / (k + 1) for k in range(live)]
    n = [max(1, int(c["rows"] * x / sum(w))) for x in w]
    n[0] = max(1, c["rows"] - sum(n[1:]))
    n += [0] * (g - live)
    return [(n[k], max(2, c["vocab"] - 5 * k)) for k in range(g)]


# ----------------------------------------------------------------- inputs ---


def _positions(c: dict, gen) -> torch.Tensor:
    """int32 [rows][axes]: samples of 16 x 16 image patches at one time and text after them; `far` moves all of them."""
    r = torch.arange(c["rows"], device=DEV)
    j, sample = r % 297, r // 297
    text = j >= 256
    t = torch.where(text, 16 + j - 256, 0)
    ax = [t, torch.where(text, t, j // 16), torch.where(text, t, j % 16)][: c["axes"]]
    far = c["far"] + torch.randint(0, 8, (c["rows"] // 297 + 1,), generator=gen, device=DEV)[sample]
    return (torch.stack(ax, 1) + far[:, None]).to(torch.int32).contiguous()


def prepare(case: dict, seed: int) -> dict:
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = {"case": dict(case)}
    randn = lambda *n: torch.randn(*n, generator=gen, device=DEV)  # noqa: E731
    if case["kind"] in ("qk", "qk_bwd"):
        hd, width = case["hd"], (case["heads"] + case["kv"]) * case["hd"]
        x = randn(case["rows"], width + case["kv"] * hd)
        x *= 0.2 + 2.0 * torch.rand(case["rows"], 1, generator=gen, device=DEV)
        if case["rows"] > 40:
            x[torch.randint(0, case["rows"], (case["rows"] // 40,), generator=gen, device=DEV)] = 0  # alignment rows
        s["x"] = x.to(BF16)
        s["gq"] = (1 + 0.2 * randn(hd)).to(BF16) if case["norm"] else None
        s["gk"] = (1 + 0.2 * randn(hd)).to(BF16) if case["norm"] else None
        s["pos"] = _positions(case, gen)
        if case["kind"] == "qk_bwd":
            s["dout"] = randn(case["rows"], width).to(BF16)
        return s
    d, shares = case["d"], _shares(case)
    total = min(4 * sum(n for n, _ in shares) + 16, 40_000)
    hidden = randn(total, d)
    s["heads"], s["rows"], s["targets"] = [], [], []
    for n, v in shares:
        w = (randn(v, d) / math.sqrt(d)).to(BF16)
        rows = torch.randperm(total, generator=gen, device=DEV)[:n].sort()[0]
        target = torch.randint(0, v, (n,), generator=gen, device=DEV)
        # three rows in four belong to a trained head's surer predictions (logits of deviation 1, theirs 10 higher)
        sure = torch.rand(n, generator=gen, device=DEV) < 0.75
        hidden[rows[sure]] += 10.0 * w[target[sure]].float()
        none = torch.rand(n, generator=gen, device=DEV) < 0.1
        s["heads"].append(w)
        s["rows"].append(rows.to(torch.int32))
        s["targets"].append(torch.where(none, -1, target).to(torch.int32))
    s["hidden"] = hidden.to(BF16)
    return s


# ------------------------------------------------------------- plain form ---


def _angles(c: dict, pos: torch.Tensor):
    i = torch.arange(c["hd"] // 2, device=DEV, dtype=F64)
    a = pos.to(F64)[:, torch.tensor(_pair_axis(c), device=DEV)] * c["theta"] ** (-2.0 * i / c["hd"])
    return a.cos().to(F32)[:, None], a.sin().to(F32)[:, None]  # far positions need the angle in 64 bits


def _gains(s: dict) -> torch.Tensor:
    """fp32 [heads + kv][hd]: the gain of every query and key head, ones without a norm."""
    c = s["case"]
    if not c["norm"]:
        return torch.ones(c["heads"] + c["kv"], c["hd"], device=DEV)
    return torch.cat([s["gq"].float().expand(c["heads"], -1), s["gk"].float().expand(c["kv"], -1)])


def _split(c: dict, x: torch.Tensor) -> torch.Tensor:
    return x[:, : (c["heads"] + c["kv"]) * c["hd"]].float().view(c["rows"], c["heads"] + c["kv"], c["hd"])


def _rsqrt(c: dict, x: torch.Tensor) -> torch.Tensor:
    return torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) if c["norm"] else torch.ones_like(x[..., :1])


def _qk_plain(s: dict):
    c = s["case"]
    x = _split(c, s["x"])
    cos, sin = _angles(c, s["pos"])
    u = x * _rsqrt(c, x) * _gains(s)
    a, b = u.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(BF16).view(c["rows"], -1)


def _qk_bwd_plain(s: dict):
    c = s["case"]
    x = _split(c, s["x"])
    cos, sin = _angles(c, s["pos"])
    a, b = _split(c, s["dout"]).chunk(2, -1)
    du = torch.cat([a * cos + b * sin, b * cos - a * sin], -1)
    if not c["norm"]:
        return {"dx": du.to(BF16).view(c["rows"], -1)}
    r = _rsqrt(c, x)
    xh, gdu = x * r, du * _gains(s)
    dx = r * (gdu - xh * (xh * gdu).mean(-1, keepdim=True))
    dg = (du * xh).sum(0, dtype=F64)
    return {"dx": dx.to(BF16).view(c["rows"], -1), "dgq": dg[: c["heads"]].sum(0).to(F32),
            "dgk": dg[c["heads"]:].sum(0).to(F32)}


def _softmax(z: torch.Tensor):
    """z less its rows' largest, what the others' exponentials add to, exp(z) and where the largest was.

    The largest is left out of the sum so that log1p of it keeps the small log-probabilities of sure rows.
    """
    m, top = z.max(1, keepdim=True)
    z -= m
    e = z.exp().scatter_(1, top, 0.0)
    return z, e.sum(1, keepdim=True), e.scatter_(1, top, 1.0), top


def _tokens_plain(s: dict, w: torch.Tensor, rows: torch.Tensor, target: torch.Tensor):
    h, wf = s["hidden"][rows.long()].float(), w.float()
    live = ((target >= 0) & (target < w.shape[0]))[:, None]
    at = target.long().clamp(0, w.shape[0] - 1)[:, None]
    z, rest, e, _ = _softmax(h @ wf.T)
    logp = z.gather(1, at) - rest.log1p()
    count = live.sum().clamp(min=1)
    e /= 1 + rest
    e.scatter_(1, at, logp.expm1())
    e *= live / count
    logp = torch.where(live, logp, 0.0)[:, 0]
    out = {"logp": logp, "loss": -(logp.sum() / count).view(1), "dW": (e.T @ h).to(BF16)}
    if s["case"]["dh"]:
        out["dh"] = (e @ wf).to(BF16)
    return out


def _decode_plain(s: dict, w: torch.Tensor, rows: torch.Tensor):
    _, rest, _, top = _softmax(s["hidden"][rows.long()].float() @ w.float().T)
    return {"token": top[:, 0].to(torch.int32), "logp": -rest[:, 0].log1p()}


# --------------------------------------------------------- the framework's ---


def _call(s: dict):
    """The objects a program of this framework keeps beside its inputs: heads, outputs, a workspace."""
    import paper_2607_16074_amd as jn

    c, ctx = s["case"], _context()
    if c["kind"] in ("qk", "qk_bwd"):
        width = (c["heads"] + c["kv"]) * c["hd"]
        qk = jn.QKNormRope(c["heads"], c["kv"], c["hd"], EPS, s["gq"], s["gk"], c["theta"], _sections(c),
                           c["interleaved"])
        out = torch.empty(c["rows"], width, dtype=BF16, device=DEV)
        if c["kind"] == "qk":
            return lambda: jn.jn_qk_norm_rope(ctx, qk, s["x"], s["pos"], out), out
        dg = [torch.empty(c["hd"], dtype=F32, device=DEV) if c["norm"] else None for _ in range(2)]
        ws = torch.empty(jn.jn_qk_norm_rope_workspace_size(qk, c["rows"]), dtype=torch.uint8, device=DEV)
        res = {"dx": out, "dgq": dg[0], "dgk": dg[1]} if c["norm"] else {"dx": out}
        return lambda: jn.jn_qk_norm_rope_bwd(ctx, qk, s["x"], s["pos"], s["dout"], out, dg[0], dg[1], ws), res
    heads = [jn.TokenHead(w) for w in s["heads"]]
    f32 = lambda n: torch.empty(n, dtype=F32, device=DEV)  # noqa: E731
    if c["kind"] == "decode":
        res = [{"token": torch.empty(r.numel(), dtype=torch.int32, device=DEV), "logp": f32(r.numel())}
               for r in s["rows"]]
        picks = [jn.TokenPick(r, o["token"], o["logp"]) for r, o in zip(s["rows"], res)]
        ws = torch.empty(jn.jn_tokens_decode_workspace_size(heads, picks), dtype=torch.uint8, device=DEV)
        return lambda: jn.jn_tenant_tokens_decode(ctx, s["hidden"], heads, picks, ws), res
    res = [{"logp": f32(r.numel()), "loss": f32(1), "dW": torch.empty_like(w)} for r, w in zip(s["rows"], s["heads"])]
    if c["dh"]:
        res = [dict(o, dh=torch.empty(r.numel(), c["d"], dtype=BF16, device=DEV)) for o, r in zip(res, s["rows"])]
    ios = [jn.TokenIO(r, t, o["logp"], o["loss"], o["dW"], o.get("dh"))
           for r, t, o in zip(s["rows"], s["targets"], res)]
    ws = torch.empty(jn.jn_tokens_workspace_size(heads, ios), dtype=torch.uint8, device=DEV)
    return lambda: jn.jn_tenant_tokens_fwd_bwd(ctx, s["hidden"], heads, ios, ws), res


_contexts: dict = {}


def _context():
    import paper_2607_16074_amd as jn

    stream = torch.cuda.current_stream()
    if stream.cuda_stream not in _contexts:
        _contexts[stream.cuda_stream] = jn.Context(stream)
    return _contexts[stream.cuda_stream]


def run(state: dict):
    if own:
        if "call" not in state:
            state["call"] = _call(state)
        go, out = state["call"]
        go()
        return out
    kind = state["case"]["kind"]
    if kind == "qk":
        return _qk_plain(state)
    if kind == "qk_bwd":
        return _qk_bwd_plain(state)
    if kind == "decode":
        return [_decode_plain(state, w, r) for w, r in zip(state["heads"], state["rows"])]
    return [_tokens_plain(state, w, r, t) for w, r, t in zip(state["heads"], state["rows"], state["targets"])]


# ------------------------------------------------------------------- work ---


def work(case: dict) -> dict:
    if case["kind"] in ("qk", "qk_bwd"):
        elems = case["rows"] * (case["heads"] + case["kv"]) * case["hd"]
        back = case["kind"] == "qk_bwd"
        return {"bytes": elems * (6 if back else 4) + 4 * case["rows"] * case["axes"],
                "flops": elems * (20 if back else 9)}
    d, total = case["d"], {"bytes": 0, "flops": 0}
    for n, v in _shares(case):
        if case["kind"] == "decode":
            total["bytes"] += 2 * d * (n + v) + 12 * n
            total["flops"] += 2 * n * v * d
        else:
            products = 3 if case["dh"] else 2  # logits, weight gradient, row gradient
            total["bytes"] += 2 * d * (n + 2 * v + (n if case["dh"] else 0)) + 12 * n
            total["flops"] += 2 * products * n * v * d
    return total


# ------------------------------------------------------ 64-bit definitions ---


def _turn(c: dict, v: torch.Tensor, pos: torch.Tensor, sign: float) -> torch.Tensor:
    """Every pair (i, i + hd/2) of v [rows][heads][hd] as a complex number, turned by its axis's angle."""
    half = c["hd"] // 2
    freq = torch.tensor([c["theta"] ** (-2.0 * i / c["hd"]) for i in range(half)], dtype=F64, device=DEV)
    ang = sign * torch.stack([pos[:, a].double() * freq[i] for i, a in enumerate(_pair_axis(c))], 1)
    z = torch.complex(v[..., :half], v[..., half:]) * torch.polar(torch.ones_like(ang), ang)[:, None]
    return torch.cat([z.real, z.imag], -1)


def _qk_exact(s: dict):
    c, parts = s["case"], []
    dg = [torch.zeros(c["hd"], dtype=F64, device=DEV) for _ in range(2)]
    for r0 in range(0, c["rows"], 8192):
        x = _split(dict(c, rows=min(8192, c["rows"] - r0)), s["x"][r0: r0 + 8192]).double()
        pos = s["pos"][r0: r0 + 8192]
        norm = (x.pow(2).sum(-1, keepdim=True) / c["hd"] + EPS).sqrt() if c["norm"] else 1.0
        gain = torch.ones(c["heads"] + c["kv"], c["hd"], dtype=F64, device=DEV)
        if c["norm"]:
            gain[: c["heads"]], gain[c["heads"]:] = s["gq"].double(), s["gk"].double()
        if c["kind"] == "qk":
            parts.append(_turn(c, x / norm * gain, pos, 1.0).flatten(1))
            continue
        back = _turn(c, s["dout"][r0: r0 + 8192].double().view(x.shape), pos, -1.0)
        if not c["norm"]:
            parts.append(back.flatten(1))
            continue
        # the norm's Jacobian is (I - x x^T / (hd norm^2)) / norm
        t = back * gain
        parts.append(((t - x * (x * t).sum(-1, keepdim=True) / (c["hd"] * norm * norm)) / norm).flatten(1))
        dg[0] += (back * x / norm)[:, : c["heads"]].sum((0, 1))
        dg[1] += (back * x / norm)[:, c["heads"]:].sum((0, 1))
    out = torch.cat(parts)
    if c["kind"] == "qk":
        return out
    return {"dx": out, "dgq": dg[0], "dgk": dg[1]} if c["norm"] else {"dx": out}


def _tokens_exact(s: dict, w: torch.Tensor, rows: torch.Tensor, target: torch.Tensor):
    w64, d = w.double(), s["case"]["d"]
    live = (target >= 0) & (target < w.shape[0])
    count = max(1, int(live.sum()))
    logp, dh, dw = [], [], torch.zeros(w.shape, dtype=F64, device=DEV)
    for r0 in range(0, rows.numel(), 1024):  # a bounded slice of the logits at a time
        at, on = target[r0: r0 + 1024].long(), live[r0: r0 + 1024]
        h = s["hidden"][rows[r0: r0 + 1024].long()].double()
        lp = torch.log_softmax(h @ w64.t(), 1)
        hit = torch.zeros_like(lp)
        k = on.nonzero()[:, 0]
        hit[k, at[k]] = 1.0
        logp.append((lp * hit).sum(1))
        g = (lp.exp() - hit) * (on.double() / count)[:, None]
        dw += g.t() @ h
        dh.append(g @ w64)
    empty = torch.zeros(0, dtype=F64, device=DEV)
    logp = torch.cat(logp + [empty])
    out = {"logp": logp, "loss": (-logp.sum() / count).view(1), "dW": dw}
    if s["case"]["dh"]:
        out["dh"] = torch.cat(dh + [empty.view(0, d)])
    return out


def exact(case: dict, seed: int):
    s = prepare(case, seed)
    if case["kind"] in ("qk", "qk_bwd"):
        return _qk_exact(s)
    if case["kind"] == "decode":
        out = []
        for w, r in zip(s["heads"], s["rows"]):
            lp = torch.log_softmax(s["hidden"][r.long()].double() @ w.double().t(), 1)
            out.append({"token": lp.argmax(1).to(torch.int32), "logp": lp.amax(1)})
        return out
    return [_tokens_exact(s, w, r, t) for w, r, t in zip(s["heads"], s["rows"], s["targets"])]
