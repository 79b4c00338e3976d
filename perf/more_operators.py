"""The operators of tenants that write tokens over a cache: what they compute, over the sizes their users have.

A sequence's keys and values lie in pages of a cache; a call brings each sequence some new rows: one token, a tree of
drafted tokens, a piece of a prompt. A case is a dict of plain values; its ``kind`` names the public entry point:

  append   ``jn_kv_append``: norms and rotation of the new rows' queries and keys; keys and values go to their pages
  attend   ``jn_kv_attention``: the new rows' attention over the cached rows and over each other, by the tree's branches
  verify   ``jn_tenant_tokens_verify``: which drafted tokens the target's probabilities let stand, and the token after them
  keep     ``jn_kv_keep``: the standing branch's keys and values of every layer, moved behind the sequence

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
BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32


# ------------------------------------------------------------------ cases ---


def listed() -> List[dict]:
    return [
        # One token of each of eight robots' streams, far into their episodes, three position axes. Latency.
        dict(name="append_8_tokens", kind="append", seqs=8, new=1, past=4_001, heads=16, kv=2, hd=128, page=64,
             mask="chain", norm=True, theta=1e6, axes=3),
        # A group's observations (256 of an image and its instruction each) go to the cache in one call.
        dict(name="append_75k_rows", kind="append", seqs=256, new=297, past=0, heads=16, kv=2, hd=128, page=128,
             mask="chain", norm=True, theta=1e6, axes=1),
        # One stream's next token. Latency, then the work of few workgroups.
        dict(name="attend_1_token", kind="attend", seqs=1, new=1, past=1_021, heads=16, kv=2, hd=128, page=64,
             mask="chain"),
        # A serving batch: 64 streams of unequal lengths, one token each. Bound by reading the cache.
        dict(name="attend_64_streams", kind="attend", seqs=64, new=1, past=16_000, heads=16, kv=2, hd=128, page=64,
             mask="chain"),
        # Eight streams' drafted trees over the 2B-shaped backbone's single key head, small pages.
        dict(name="attend_trees_8", kind="attend", seqs=8, new=25, past=4_000, heads=8, kv=1, hd=256, page=16,
             mask="tree"),
        # One drafted tree at the end of a very long context, every query head with keys of its own.
        dict(name="attend_tree_131k", kind="attend", seqs=1, new=61, past=131_009, heads=8, kv=8, hd=128, page=256,
             mask="tree"),
        # Pieces of two prompts behind what is cached of them: bound by the matrix cores.
        dict(name="attend_pieces_2k", kind="attend", seqs=2, new=2_048, past=6_001, heads=16, kv=2, hd=128, page=128,
             mask="chain"),
        # One stream's chain of four drafted tokens, drawn from the draft's own probabilities. Latency.
        dict(name="verify_chain", kind="verify", tenants=1, trees=1, nodes=5, vocab=32_003, tree=False, drawn=True),
        # A serving batch's trees of the draft's likeliest tokens, two tenants.
        dict(name="verify_trees_64", kind="verify", tenants=2, trees=64, nodes=25, vocab=32_003, tree=True, drawn=False),
        # Trees drawn from the draft's probabilities over a large vocabulary.
        dict(name="verify_trees_160k", kind="verify", tenants=1, trees=16, nodes=9, vocab=160_001, tree=True, drawn=True),
        # One stream's standing branch, a few layers. Latency.
        dict(name="keep_1", kind="keep", seqs=1, new=9, past=1_021, layers=4, kv=2, hd=128, page=64, path=4),
        # A serving batch's standing branches in every layer of the 2B-shaped backbone's depth.
        dict(name="keep_64", kind="keep", seqs=64, new=25, past=700, layers=18, kv=8, hd=128, page=64, path=6),
    ]


# (query heads, key/value heads, head width) of the backbones' variants
_HEADS = ((8, 8, 256), (8, 1, 256), (16, 2, 128), (16, 16, 128), (12, 12, 64), (4, 4, 32), (16, 4, 64), (8, 2, 32))
_PAGES = (16, 32, 64, 128, 256)


def _log(rng, lo: int, hi: int) -> int:
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng) -> dict:
    kind = rng.choice(("append", "attend", "attend", "verify", "keep"))
    if kind == "verify":
        vocab, tenants = _log(rng, 100, 160_001), rng.choice((1, 1, 2, 5))
        nodes = _log(rng, 1, 61)
        trees = _log(rng, tenants, max(tenants, min(64, 25_000_000 // (vocab * nodes))))
        return dict(kind=kind, tenants=tenants, trees=trees, nodes=nodes, vocab=vocab, tree=rng.random() < 0.6,
                    drawn=rng.random() < 0.5)
    heads, kv, hd = rng.choice(_HEADS)
    page = rng.choice(_PAGES)
    if kind == "keep":
        new = _log(rng, 4, 64)
        return dict(kind=kind, seqs=_log(rng, 1, 64), new=new, past=_log(rng, 1, 1_000), layers=_log(rng, 1, 18), kv=kv,
                    hd=hd, page=page, path=rng.randint(2, new // 2))
    mask = rng.choice(("chain", "tree", "tree", "whole"))
    if kind == "append":
        seqs = _log(rng, 1, 256)
        new = _log(rng, 1, 64 if mask == "tree" else max(1, min(2_048, 60_000 * 20 * 128 // ((heads + 2 * kv) * hd * seqs))))
        return dict(kind=kind, seqs=seqs, new=new, past=rng.choice((0, _log(rng, 1, 2_000))), heads=heads, kv=kv, hd=hd,
                    page=page, mask=mask, norm=rng.random() < 0.5, theta=rng.choice((0.0, 1e4, 1e6)),
                    axes=rng.choice((1, 1, 2, 3)))
    seqs = _log(rng, 1, 64)
    new = _log(rng, 1, 64 if mask == "tree" else 2_000 // seqs)
    past = _log(rng, 1, max(1, min(131_009, 250_000_000 // (seqs * kv * hd), 120_000_000 // (seqs * heads * new) - new)))
    return dict(kind=kind, seqs=seqs, new=new, past=past, heads=heads, kv=kv, hd=hd, page=page, mask=mask)


def _lengths(c: dict) -> tuple:
    """(cached rows, new rows) of every sequence: unequal shares of the case's largest, some of them one row or none."""
    past = [c["past"] * ((37 * s) % 64 + 1) // 64 if s else c["past"] for s in range(c["seqs"])]
    new = [1 + (c["new"] - 1) * ((29 * s) % 16 + 1) // 16 if s else c["new"] for s in range(c["seqs"])]
    return past, new


def _cu(n: List[int]) -> List[int]:
    cu = [0]
    for x in n:
        cu.append(cu[-1] + x)
    return cu


def _shares(c: dict) -> List[tuple]:
    """(nodes of each tree, vocabulary) of every tenant."""
    g, out, at = c["tenants"], [], 0
    for k in range(g):
        trees = c["trees"] // g + (1 if k < c["trees"] % g else 0)
        out.append(([1 + (c["nodes"] - 1) * ((29 * (at + s)) % 16 + 1) // 16 if at + s else c["nodes"]
                     for s in range(trees)], max(2, c["vocab"] - 7 * k)))
        at += trees
    return out


# ----------------------------------------------------------------- inputs ---


def _ints(v) -> torch.Tensor:
    return torch.tensor(v, dtype=I32, device=DEV)


def _parents(new: List[int], tree: bool, gen) -> torch.Tensor:
    """int32, every row's parent in its own sequence: the first row has none, later ones an earlier row near the first."""
    j = torch.cat([torch.arange(n, device=DEV) for n in new])
    if not tree:
        return (j - 1).to(I32)
    u = torch.rand(j.numel(), generator=gen, device=DEV, dtype=F64)
    return torch.where(j > 0, (u * u * j).floor().clamp(max=j - 1), -1).to(I32)


def prepare(case: dict, seed: int) -> dict:
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    c = dict(case)
    s = {"case": c}
    randn = lambda *n: torch.randn(*n, generator=gen, device=DEV)  # noqa: E731
    if c["kind"] == "verify":
        s["tenants"] = [_drafts(c, n, v, gen) for n, v in _shares(c)]
        return s
    past, new = _lengths(c)
    cap = [(p + n + c["page"] - 1) // c["page"] for p, n in zip(past, new)]
    c["max_pages"] = max(cap)
    pool = torch.randperm(sum(cap) + 3, generator=gen, device=DEV).to(I32)
    table = torch.full((c["seqs"], c["max_pages"]), -1, dtype=I32)  # a sequence has the pages that it needs
    at = torch.arange(c["max_pages"])[None] < torch.tensor(cap)[:, None]
    table = table.to(DEV)
    table[at.to(DEV)] = pool[: sum(cap)]
    s["pages"], s["past"], s["cu"] = table, _ints(past), _ints(_cu(new))
    s["parents"] = _parents(new, True, gen) if c.get("mask") == "tree" else None
    # one layer where the call is one layer's; others than the first have what the model left there
    shape = (c.get("layers", 1), sum(cap) + 3, c["kv"], c["page"], c["hd"])
    cache = lambda: torch.empty(shape, dtype=BF16, device=DEV).normal_(generator=gen)  # noqa: E731
    s["k"], s["v"] = cache(), cache()
    c["live"], c["rows"] = sum(new), sum(new) + (5 if c["seqs"] > 1 else 0)  # a batch's rows have room for more
    if c["kind"] == "keep":
        # ascending rows of the tree; those that move come from behind where the branch goes
        path = torch.full((c["seqs"], c["path"]), -1, dtype=I32)
        count = [max(1, min(c["path"], n // 2)) for n in new]
        u = torch.rand(c["seqs"], c["new"], generator=gen, device=DEV).cpu()
        for i, (n, k) in enumerate(zip(new, count)):
            u[i, :k] = u[i, n:] = 2.0
            path[i, 0] = 0
            path[i, 1:k] = u[i].argsort()[: k - 1].sort()[0]
        s["path"], s["count"], s["behind"] = path.to(DEV), _ints(count), torch.zeros_like(s["past"])
        return s
    if c["kind"] == "append":
        x = randn(c["rows"], (c["heads"] + 2 * c["kv"]) * c["hd"])
        s["x"] = (x * (0.2 + 2.0 * torch.rand(c["rows"], 1, generator=gen, device=DEV))).to(BF16)
        s["gq"] = (1 + 0.2 * randn(c["hd"])).to(BF16) if c["norm"] else None
        s["gk"] = (1 + 0.2 * randn(c["hd"])).to(BF16) if c["norm"] else None
        s["q"] = torch.zeros(c["rows"], c["heads"] * c["hd"], dtype=BF16, device=DEV)
        s["pos"] = None  # one axis: a row's place behind its sequence (along its branch)
        if c["axes"] > 1 and c["theta"]:
            s["pos"] = torch.randint(0, 5_000, (c["rows"], c["axes"]), generator=gen, device=DEV).to(I32)
        return s
    s["q"] = (1.5 * randn(c["rows"], c["heads"] * c["hd"])).to(BF16)
    s["out"] = torch.zeros(c["rows"], c["heads"] * c["hd"], dtype=BF16, device=DEV)
    return s


def _drafts(c: dict, nodes: List[int], vocab: int, gen) -> dict:
    """A tenant's trees: the target's probabilities near the draft's; tokens drawn from the draft's, or its likeliest."""
    n = sum(nodes)
    z = 2.5 * torch.randn(n, vocab, generator=gen, device=DEV)
    p = torch.softmax(z + 0.7 * torch.randn(n, vocab, generator=gen, device=DEV), 1)
    q = torch.softmax(z, 1)
    parents = _parents(nodes, c["tree"], gen)
    first = torch.repeat_interleave(torch.tensor(_cu(nodes)[:-1], device=DEV), torch.tensor(nodes, device=DEV))
    up = first + parents.clamp(min=0)
    if c["drawn"]:
        # (one number a token by the exponentials' race: a drawn token's chance is its probability)
        race = torch.empty(n, vocab, device=DEV).exponential_(generator=gen)
        tokens = race.reciprocal_().mul_(q[up]).argmax(1)
    else:
        order = torch.arange(n, device=DEV)
        rank = ((up[:, None] == up[None]) & (order[None] < order[:, None]) & (parents[None] >= 0)).sum(1)
        best = q.topk(min(vocab, 64), 1)[1]
        tokens = best[up, rank.clamp(max=best.shape[1] - 1)]
    u = lambda m: torch.rand(m, generator=gen, device=DEV)  # noqa: E731
    return {"cu": _ints(_cu(nodes)), "nodes": max(nodes), "parents": parents if c["tree"] else None,
            "tokens": tokens.to(I32), "p": p, "q": q if c["drawn"] else None, "u": u(n), "r": u(len(nodes))}


# ------------------------------------------------------------- plain form ---


def _places(s: dict, live: int):
    """Of the first `live` rows: sequence, index in it, and the cache's (page, row of the page) of place past + index."""
    r = torch.arange(live, device=DEV)
    seq = torch.searchsorted(s["cu"][1:].long(), r, right=True)
    j = r - s["cu"].long()[seq]
    at = s["past"].long()[seq] + j
    page = s["case"]["page"]
    return seq, j, s["pages"].long()[seq, at // page], at % page


def _sees(parents: torch.Tensor) -> torch.Tensor:
    """bool [trees][n][n]: row i sees row j of its tree, its ancestors and itself: (1 - A)^-1 for the parents' matrix A."""
    n = parents.shape[1]
    hit = (parents[:, :, None] == torch.arange(n, device=DEV)).to(F32)
    one = torch.eye(n, device=DEV)
    return torch.linalg.solve_triangular(one - hit, one.expand_as(hit), upper=False, unitriangular=True) > 0.5


def _padded(s: dict, rows: torch.Tensor, fill=0) -> torch.Tensor:
    """[seqs][most new rows][...] of rows, `fill` where a sequence has fewer."""
    c = s["case"]
    seq, j, _, _ = _places(s, c["live"])
    out = torch.full((c["seqs"], c["new"], *rows.shape[1:]), fill, dtype=rows.dtype, device=DEV)
    out[seq, j] = rows[: c["live"]]
    return out


def _pair_axis(c: dict) -> List[int]:
    """Axis of every pair of a head: runs of the sections' lengths."""
    return [a for a, k in enumerate(_sections(c)) for _ in range(k)]


def _sections(c: dict) -> List[int]:
    half, axes = c["hd"] // 2, c["axes"]
    rest = half // 4 if axes == 3 else half // 3
    return [half - rest * (axes - 1)] + [rest] * (axes - 1)


def _append_plain(s: dict):
    c, hd = s["case"], s["case"]["hd"]
    seq, j, page, row = _places(s, c["live"])
    x = s["x"][: c["live"]].float().view(c["live"], -1, hd)
    u = x[:, : c["heads"] + c["kv"]]
    if c["norm"]:
        u = u * torch.rsqrt(u.square().mean(-1, keepdim=True) + EPS)
        u = torch.cat([u[:, : c["heads"]] * s["gq"].float(), u[:, c["heads"]:] * s["gk"].float()], 1)
    if c["theta"]:
        if s["pos"] is None:
            deep = j if s["parents"] is None else _sees(_padded(s, s["parents"], -1))[seq, j].sum(-1) - 1
            pos = (s["past"].long()[seq] + deep)[:, None].expand(-1, hd // 2)
        else:
            pos = s["pos"][: c["live"]].long()[:, torch.tensor(_pair_axis(c), device=DEV)]
        # far positions need the angle in 64 bits
        a = pos.to(F64) * c["theta"] ** (-2.0 * torch.arange(hd // 2, device=DEV, dtype=F64) / hd)
        cos, sin = a.cos().to(F32)[:, None], a.sin().to(F32)[:, None]
        lo, hi = u.chunk(2, -1)
        u = torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1)
    s["q"][: c["live"]] = u[:, : c["heads"]].to(BF16).flatten(1)
    s["k"][-1][page, :, row] = u[:, c["heads"]:].to(BF16)
    s["v"][-1][page, :, row] = x[:, c["heads"] + c["kv"]:].to(BF16)
    return {"q": s["q"], "k": s["k"], "v": s["v"]}


def _cached(s: dict, cache: torch.Tensor, most: int) -> torch.Tensor:
    """fp32 [seqs][kv][most][hd] of a cache's layer: every sequence's rows in order (others' behind its end)."""
    c = s["case"]
    t = cache[s["pages"].long().clamp(min=0)].transpose(1, 2).reshape(c["seqs"], c["kv"], -1, c["hd"])
    return t[:, :, :most].float()


def _attend_plain(s: dict):
    c, group = s["case"], s["case"]["heads"] // s["case"]["kv"]
    past, n = s["past"].long(), (s["cu"][1:] - s["cu"][:-1]).long()
    most = max(p + m for p, m in zip(*_lengths(c)))
    q = _padded(s, s["q"].float()).view(c["seqs"], c["new"], c["kv"], group, c["hd"])
    q = q.permute(0, 2, 3, 1, 4).reshape(c["seqs"] * c["kv"], group * c["new"], c["hd"])
    key = torch.arange(most, device=DEV) - past[:, None]  # of the new rows from 0 on
    i = torch.arange(c["new"], device=DEV)[None, :, None]
    new = (key >= 0) & (key < n[:, None])
    if c["mask"] == "tree":
        sees = _sees(_padded(s, s["parents"], -1)).gather(2, key.clamp(0, c["new"] - 1)[:, None].expand(-1, c["new"], -1))
    else:
        sees = key[:, None] <= i if c["mask"] == "chain" else torch.ones_like(key[:, None] <= i)
    sees = (key < 0)[:, None] | (sees & new[:, None])
    z = q @ _cached(s, s["k"][-1], most).flatten(0, 1).transpose(1, 2)
    z = (z / math.sqrt(c["hd"])).view(c["seqs"], c["kv"] * group, c["new"], most)
    z.masked_fill_(~sees[:, None], -math.inf)
    z -= z.amax(-1, keepdim=True)
    z.exp_()
    z /= z.sum(-1, keepdim=True)
    o = z.view(c["seqs"] * c["kv"], -1, most) @ _cached(s, s["v"][-1], most).flatten(0, 1)
    o = o.view(c["seqs"], c["kv"] * group, c["new"], c["hd"]).transpose(1, 2).flatten(2)
    seq, j, _, _ = _places(s, c["live"])
    s["out"][: c["live"]] = o[seq, j].to(BF16)
    return s["out"]


def _verify_plain(t: dict):
    """All trees together, node after node: a node whose parent is the last standing one is tried.

    What is left of a node's probabilities after rejections is max(p - a q, 0): each adds the sum of what was left,
    over what the number's acceptance is taken of, to a. Likeliest tokens are taken out of p instead.
    """
    p, q, cu = t["p"], t["q"], t["cu"].long()
    first, n = cu[:-1], cu[1:] - cu[:-1]
    trees, ar = n.numel(), torch.arange(n.numel(), device=DEV)
    cur = torch.zeros_like(n)
    a, left = torch.zeros(trees, dtype=F64, device=DEV), torch.ones(trees, dtype=F64, device=DEV)
    # max(p - a q, 0) of the node before its last rejection stays the answer where nothing is left after it
    before = torch.zeros_like(a)
    out = torch.zeros(trees, p.shape[1], dtype=torch.bool, device=DEV)  # tokens taken out
    path = torch.full((trees, t["nodes"]), -1, dtype=I32, device=DEV)
    path[:, 0], count = 0, torch.ones_like(n)
    rest = lambda a: (p[first + cur].double() - a[:, None] * q[first + cur].double()).clamp_(min=0)  # noqa: E731
    for j in range(1, t["nodes"]):
        at = first + min(j, t["nodes"]) * (j < n)
        up = torch.full_like(n, j - 1) if t["parents"] is None else t["parents"].long()[at]
        tried = (j < n) & (up == cur)
        x = t["tokens"].long()[at]
        px, u = p[first + cur, x].double(), t["u"][at].double()
        if q is None:
            px = torch.where(out[ar, x], 0.0, px)
            stands = tried & (u * left < px)
            left = torch.where(tried, left - px, left)
            out[ar, x] |= tried
        else:
            qx = q[first + cur, x].double()
            stands = tried & (u * qx * left < (px - a * qx).clamp(min=0))
            fails = tried & ~stands & (left > 0)
            before = torch.where(fails, a, before)
            a = torch.where(fails, a + left, a)
            left = torch.where(fails, rest(a).sum(1), left)
        cur = torch.where(stands, j, cur)
        path[ar, torch.where(stands, count, 0)] = torch.where(stands, j, 0).to(I32)
        count = count + stands
        a, before, left = (torch.where(stands, v, w) for v, w in ((0.0, a), (0.0, before), (1.0, left)))
        out &= ~stands[:, None]
    if q is None:
        w = p[first + cur].double().masked_fill_(out, 0.0)
    else:
        w = rest(a)
        w = torch.where((w.sum(1) > 0)[:, None], w, rest(before))
    sums = w.cumsum(1)
    nxt = (sums <= t["r"].double()[:, None] * sums[:, -1:]).sum(1)
    return {"path": path, "count": count.to(I32), "next": nxt.to(I32)}


def _keep_plain(s: dict):
    c = s["case"]
    k = torch.arange(c["path"], device=DEV)
    live = k < s["count"][:, None]
    seq, k = live.nonzero(as_tuple=True)
    page = lambda at: (s["pages"].long()[seq, at // c["page"]], at % c["page"])  # noqa: E731
    past = s["past"].long()[seq]
    (p0, r0), (p1, r1) = page(past + s["path"].long()[seq, k]), page(past + k)
    for cache in (s["k"], s["v"]):
        cache[:, p1, :, r1] = cache[:, p0, :, r0]
    torch.add(s["past"], s["count"], out=s["behind"])
    return {"k": s["k"], "v": s["v"], "past": s["behind"]}


# --------------------------------------------------------- the framework's ---


def _call(s: dict):
    """The objects a program of this framework keeps beside its inputs: cache, batch, outputs, a workspace."""
    import paper_2607_16074_amd as jn

    c, ctx = s["case"], _context()
    if c["kind"] == "verify":
        res, ios = [], []
        for t in s["tenants"]:
            trees = t["cu"].numel() - 1
            ints = lambda *n: torch.empty(n, dtype=I32, device=DEV)  # noqa: E731
            o = {"path": ints(trees, t["nodes"]), "count": ints(trees), "next": ints(trees)}
            ios.append(jn.TokenVerify(t["cu"], t["tokens"], o["path"], o["count"], o["next"], p=t["p"], q=t["q"],
                                      u=t["u"], r=t["r"], parents=t["parents"]))
            res.append(o)
        ws = torch.empty(jn.jn_tokens_verify_workspace_size(ios), dtype=torch.uint8, device=DEV)
        return lambda: jn.jn_tenant_tokens_verify(ctx, ios, ws), res
    cache = jn.KVCache(s["k"], s["v"])
    rows = c["rows"] if s["parents"] is None else c["live"]  # (every row of a call with trees has its parent)
    batch = jn.KVBatch(s["pages"], s["past"], s["cu"], rows, c["new"], s["parents"], c.get("mask") == "whole")
    if c["kind"] == "keep":
        return (lambda: jn.jn_kv_keep(ctx, cache, batch, s["path"], s["count"], s["behind"]),
                {"k": s["k"], "v": s["v"], "past": s["behind"]})
    if c["kind"] == "append":
        qk = jn.QKNormRope(c["heads"], c["kv"], c["hd"], EPS, s["gq"], s["gk"], c["theta"],
                           _sections(c) if s["pos"] is not None else ())
        x, q, pos = s["x"][:rows], s["q"][:rows], s["pos"][:rows] if s["pos"] is not None else None
        return (lambda: jn.jn_kv_append(ctx, cache, 0, batch, qk, x, pos, q),
                {"q": s["q"], "k": s["k"], "v": s["v"]})
    ws = torch.empty(jn.jn_kv_attention_workspace_size(cache, batch, c["heads"]), dtype=torch.uint8, device=DEV)
    q, out = s["q"][:rows], s["out"][:rows]
    return lambda: jn.jn_kv_attention(ctx, cache, 0, batch, c["heads"], q, out, ws), s["out"]


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
    if kind == "verify":
        return [_verify_plain(t) for t in state["tenants"]]
    return {"append": _append_plain, "attend": _attend_plain, "keep": _keep_plain}[kind](state)


# ------------------------------------------------------------------- work ---


def work(case: dict) -> dict:
    c = case
    if c["kind"] == "verify":
        # Each standing or last node's token probabilities, and one row of them (the last node's) to the next token's draw.
        rows = [(len(n), sum(n), v) for n, v in _shares(c)]
        per = 8 if c["drawn"] else 4
        return {"bytes": sum(t * v * per + 16 * n + 8 * t for t, n, v in rows), "flops": sum(4 * t * v for t, _, v in rows)}
    past, new = _lengths(c)
    if c["kind"] == "keep":
        moved = sum(max(1, min(c["path"], n // 2)) - 1 for n in new) * c["layers"] * c["kv"] * c["hd"]
        return {"bytes": 8 * moved + 8 * c["seqs"], "flops": 0}
    if c["kind"] == "append":
        elems = sum(new) * (c["heads"] + 2 * c["kv"]) * c["hd"]
        return {"bytes": 4 * elems + 4 * sum(new), "flops": 9 * elems}
    pairs = sum(n * p + (n * n if c["mask"] == "whole" else n * (n + 1) // 2) for p, n in zip(past, new))
    cached = sum(p + n for p, n in zip(past, new)) * c["kv"] * c["hd"]
    return {"bytes": 4 * cached + 4 * sum(new) * c["heads"] * c["hd"], "flops": 4 * pairs * c["heads"] * c["hd"]}


# ------------------------------------------------------ 64-bit definitions ---


def _branch(parents: List[int], j: int) -> List[int]:
    """Row j and its ancestors, from the row up."""
    out = [j]
    while parents[out[-1]] >= 0:
        out.append(parents[out[-1]])
    return out


def _of_seq(s: dict, i: int):
    """(cached rows, first new row, new rows, parents or None) of a sequence."""
    past, new = _lengths(s["case"])
    at = _cu(new)[i]
    up = s["parents"][at: at + new[i]].tolist() if s["parents"] is not None else None
    return past[i], at, new[i], up


def _slots(s: dict, i: int, lo: int, hi: int) -> torch.Tensor:
    """Rows of the cache, pages laid end to end, that hold places lo .. hi - 1 of sequence i."""
    at = torch.arange(lo, hi, device=DEV)
    return s["pages"][i].long()[at // s["case"]["page"]] * s["case"]["page"] + at % s["case"]["page"]


def _append_exact(s: dict):
    c, hd, half = s["case"], s["case"]["hd"], s["case"]["hd"] // 2
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    flat = [t[0].transpose(1, 2).reshape(-1, c["kv"], hd).clone() for t in (k, v)]
    freq = torch.tensor([c["theta"] ** (-2.0 * e / hd) if c["theta"] else 0.0 for e in range(half)], dtype=F64, device=DEV)
    for i in range(c["seqs"]):
        past, at, n, up = _of_seq(s, i)
        x = s["x"][at: at + n].double().view(n, -1, hd)
        qh, kh, vh = x.split([c["heads"], c["kv"], c["kv"]], 1)
        if c["norm"]:
            qh, kh = (t / (t.pow(2).sum(-1, keepdim=True) / hd + EPS).sqrt() * g.double() for t, g in ((qh, s["gq"]), (kh, s["gk"])))
        if s["pos"] is not None:
            place = torch.stack([s["pos"][at: at + n, a].double() for a in _pair_axis(c)], 1)
        else:
            deep = [len(_branch(up, j)) - 1 for j in range(n)] if up else list(range(n))
            place = (past + torch.tensor(deep, dtype=F64, device=DEV))[:, None]
        turn = torch.polar(torch.ones(n, half, dtype=F64, device=DEV), (place * freq).expand(n, half).contiguous())[:, None]
        rows = []
        for t in (qh, kh):
            z = torch.complex(t[..., :half].contiguous(), t[..., half:].contiguous()) * turn
            rows.append(torch.cat([z.real, z.imag], -1))
        q[at: at + n] = rows[0].flatten(1)
        slot = _slots(s, i, past, past + n)
        flat[0][slot], flat[1][slot] = rows[1], vh
    k, v = (t.view(k.shape[1], c["page"], c["kv"], hd).transpose(1, 2)[None] for t in flat)
    return {"q": q, "k": k, "v": v}


def _attend_exact(s: dict):
    c, group = s["case"], s["case"]["heads"] // s["case"]["kv"]
    out = s["out"].double().view(c["rows"], c["heads"], c["hd"])
    for i in range(c["seqs"]):
        past, at, n, up = _of_seq(s, i)
        slot = _slots(s, i, 0, past + n)
        hidden = torch.ones(n, past + n, dtype=torch.bool, device=DEV)
        hidden[:, :past] = False
        if c["mask"] == "whole":
            hidden[:] = False
        elif c["mask"] == "chain":
            hidden[:, past:] = torch.ones(n, n, device=DEV).triu(1).bool()
        else:
            for j in range(n):
                hidden[j, [past + b for b in _branch(up, j)]] = False
        page, row = slot // c["page"], slot % c["page"]
        for h in range(c["heads"]):
            keys, values = (t[0][page, h // group, row].double() for t in (s["k"], s["v"]))
            z = s["q"][at: at + n, h * c["hd"]: (h + 1) * c["hd"]].double() @ keys.t() * c["hd"] ** -0.5
            out[at: at + n, h] = torch.softmax(z.masked_fill(hidden, -math.inf), 1) @ values
    return out.flatten(1)


def _verify_exact(t: dict):
    """Tree after tree; the residual distributions are formed and normalised one after the other."""
    cu, tokens, us, rs = (t[k].tolist() for k in ("cu", "tokens", "u", "r"))
    path, count, nxt = torch.full((len(rs), t["nodes"]), -1, dtype=I32), [], []
    for i, r in enumerate(rs):
        first, n = cu[i], cu[i + 1] - cu[i]
        up = t["parents"][first: first + n].tolist() if t["parents"] is not None else list(range(-1, n - 1))
        stand, cur = [0], None
        while cur != stand[-1]:
            cur = stand[-1]
            left = t["p"][first + cur].double()
            for j in [j for j in range(cur + 1, n) if up[j] == cur]:
                x = tokens[first + j]
                draft = t["q"][first + cur].double() if t["q"] is not None else None
                chance = float(left[x] / draft[x]) if draft is not None else float(left[x])
                if us[first + j] < chance:
                    stand.append(j)
                    break
                if draft is None:
                    left = left / (1.0 - chance)
                    left[x] = 0.0
                    continue
                new = (left - draft).clamp(min=0)
                if float(new.sum()) > 0:
                    left = new / new.sum()
        sums = (left / left.sum()).cumsum(0)
        nxt.append(int(torch.searchsorted(sums, torch.tensor([r], dtype=F64, device=DEV), right=True)))
        path[i, : len(stand)] = torch.tensor(stand, dtype=I32)
        count.append(len(stand))
    return {"path": path.to(DEV), "count": _ints(count), "next": _ints(nxt)}


def _keep_exact(s: dict):
    """The moves one after the other: nothing is computed, so there is nothing to round."""
    c = s["case"]
    k, v = s["k"].double(), s["v"].double()
    for i, n in enumerate(s["count"].tolist()):
        past = _lengths(c)[0][i]
        for to, frm in enumerate(s["path"][i, :n].tolist()):
            (p0, r0), (p1, r1) = (divmod(int(_slots(s, i, past + x, past + x + 1)), c["page"]) for x in (frm, to))
            k[:, p1, :, r1], v[:, p1, :, r1] = k[:, p0, :, r0].clone(), v[:, p0, :, r0].clone()
    return {"k": k, "v": v, "past": s["past"] + s["count"]}


def exact(case: dict, seed: int):
    s = prepare(case, seed)
    if case["kind"] == "verify":
        return [_verify_exact(t) for t in s["tenants"]]
    return {"append": _append_exact, "attend": _attend_exact, "keep": _keep_exact}[case["kind"]](s)
