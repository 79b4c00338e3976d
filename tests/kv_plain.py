"""Plain 64-bit definitions of the calls over a cache of keys and values, on the CPU, one row at a time."""
import math

import torch

F64 = torch.float64


def sequences(b):
    """(past, first row, new rows) of every sequence, bounded as joynexus.h says."""
    cu, past = b["cu"].tolist(), b["past"].tolist()
    places = b["pages"].shape[1] * b["page"]
    out = []
    for s in range(len(past)):
        row0 = min(max(cu[s], 0), b["rows"])
        out.append((min(max(past[s], 0), places), row0, min(max(min(cu[s + 1], b["rows"]) - row0, 0), b["max_new"])))
    return out


def place(b, n_pages, s, t):
    """(page, row of the page) of place t of sequence s, or None."""
    if t < 0 or t // b["page"] >= b["pages"].shape[1]:
        return None
    g = int(b["pages"][s, t // b["page"]])
    return (g, t % b["page"]) if 0 <= g < n_pages else None


def parent(b, row0, j):
    p = int(b["parents"][row0 + j])
    return p if 0 <= p < j else -1


def branch(b, row0, j):
    """Row j and its ancestors."""
    out = [j]
    while parent(b, row0, out[-1]) >= 0:
        out.append(parent(b, row0, out[-1]))
    return out


def sees(b, row0, n, j):
    """New rows that row j sees."""
    if b.get("parents") is not None:
        return sorted(branch(b, row0, j))
    return list(range(n if b.get("whole") else j + 1))


def norm_rope(x, g, eps, theta, pos, axis):
    """x [heads][hd] in 64 bits; pos: position of every axis, axis: axis of every pair."""
    hd = x.shape[1]
    if g is not None:
        x = x / torch.sqrt(x.pow(2).mean(1, keepdim=True) + eps) * g.to(F64)
    if theta:
        i = torch.arange(hd // 2, dtype=F64)
        ang = torch.tensor([pos[a] for a in axis], dtype=F64) * theta ** (-2 * i / hd)
        lo, hi = x[:, : hd // 2], x[:, hd // 2:]
        x = torch.cat([lo * ang.cos() - hi * ang.sin(), hi * ang.cos() + lo * ang.sin()], 1)
    return x


def append(b, k, v, x, heads, kv, gq, gk, eps, theta, pos, axis, q):
    """64-bit copies of k, v [pages][kv][page][hd] and q with the new rows in their places, and whether each was written."""
    hd = k.shape[-1]
    k, v, q = k.to(F64).clone(), v.to(F64).clone(), q.to(F64).clone()
    hit = torch.zeros(k.shape[0], k.shape[2], dtype=torch.bool)
    for s, (past, row0, n) in enumerate(sequences(b)):
        for j in range(n):
            r = x[row0 + j, : (heads + 2 * kv) * hd].to(F64).view(-1, hd)
            if pos is not None:
                at = pos[row0 + j].tolist()
            else:
                at = [past + (len(branch(b, row0, j)) - 1 if b.get("parents") is not None else j)]
            q[row0 + j, : heads * hd] = norm_rope(r[:heads], gq, eps, theta, at, axis).flatten()
            where = place(b, k.shape[0], s, past + j)
            if where:
                k[where[0], :, where[1]] = norm_rope(r[heads: heads + kv], gk, eps, theta, at, axis)
                v[where[0], :, where[1]] = r[heads + kv:]
                hit[where] = True
    return k, v, q, hit


def attention(b, k, v, q, heads, out, scale=0.0):
    """(out, tolerance) in 64 bits: rows that no sequence has keep what they were, with tolerance 0.

    A result is off by at most half a step of bf16, the rounding of every probability to bf16 (2^-8 of sum p |v|), and
    what 32-bit scores, exponentials and sums lose: a score's dot product over hd terms and its scaling, n sums.
    """
    kv, hd = k.shape[1], k.shape[-1]
    out = out.to(F64).clone()
    tol = torch.zeros_like(out)
    scale = scale or 1 / math.sqrt(hd)
    for s, (past, row0, n) in enumerate(sequences(b)):
        at = [place(b, k.shape[0], s, t) for t in range(past + n)]
        for j in range(n):
            keys = [at[t] for t in [*range(past), *(past + i for i in sees(b, row0, n, j))] if at[t]]
            cols = slice(0, heads * hd)
            if not keys:
                out[row0 + j, cols] = 0
                continue
            g, r = (torch.tensor(x) for x in zip(*keys))
            kk, vv = k[g, :, r].to(F64), v[g, :, r].to(F64)  # [keys][kv][hd]
            qq = q[row0 + j, cols].to(F64).view(kv, heads // kv, hd)
            z = torch.einsum("hgd,khd->hgk", qq, kk) * scale
            p = torch.softmax(z, -1)
            o, a = torch.einsum("hgk,khd->hgd", p, vv), torch.einsum("hgk,khd->hgd", p, vv.abs())
            big = (torch.einsum("hgd,khd->hgk", qq.abs(), kk.abs()) * scale).amax(-1, keepdim=True)
            dz = (hd + 8) * 2.0 ** -24 * big
            e = 2.0 ** -8 + 2 * dz + 2.0 ** -20 + 2 * len(keys) * 2.0 ** -24
            out[row0 + j, cols] = o.flatten()
            tol[row0 + j, cols] = (2.0 ** -8 * o.abs() + e * a * 1.01).flatten()
    return out, tol


def keep(b, k, v, path, n_path):
    """k, v [layers][pages][kv][page][hd] with the paths' rows moved one after the other, and past."""
    k, v, past_out = k.clone(), v.clone(), []
    for s, (past, _, _) in enumerate(sequences(b)):
        n, last = min(max(int(n_path[s]), 0), path.shape[1]), -1
        past_out.append(past + n)
        for i in range(n):
            j = int(path[s, i])
            if j <= last or j < i or j >= b["max_new"]:
                continue
            last = j
            frm, to = place(b, k.shape[1], s, past + j), place(b, k.shape[1], s, past + i)
            if frm and to:
                k[:, to[0], :, to[1]] = k[:, frm[0], :, frm[1]].clone()
                v[:, to[0], :, to[1]] = v[:, frm[0], :, frm[1]].clone()
    return k, v, past_out


def verify(cu, tokens, parents, p, q, greedy, u, r, vocab, max_path, n_all, tree_rows=256):
    """(paths, next) of every tree, by the definition in joynexus.h."""
    paths, nxt = [], []
    clean = lambda w: torch.nan_to_num(w, nan=0.0, posinf=math.inf).clamp(min=0)  # noqa: E731
    for t in range(len(cu) - 1):
        first = min(max(int(cu[t]), 0), n_all)
        n = min(max(min(int(cu[t + 1]), n_all) - first, 0), tree_rows if parents is not None else max_path)
        if n == 0:
            paths.append([])
            nxt.append(-1)
            continue
        path, c = [0], 0
        fresh = lambda c: clean(p[first + c, :vocab].to(F64)) if p is not None else None  # noqa: E731
        w, a, T = fresh(0), 0.0, 1.0
        before = w
        j = 0
        while j + 1 < n and len(path) < max_path:
            j += 1
            up = int(parents[first + j]) if parents is not None else j - 1
            x = int(tokens[first + j])
            if up != c or not 0 <= x < vocab:
                continue
            if p is None:
                ok = int(greedy[first + c]) == x
            elif q is not None:
                ok = float(u[first + j]) * float(q[first + c, x]) * T < float(w[x])
                if not ok and T > 0:
                    before = w
                    a += T
                    w = clean(p[first + c, :vocab].to(F64) - a * q[first + c, :vocab].to(F64))
                    T = float(w.sum())
            else:
                ok = float(u[first + j]) * T < float(w[x])
                if not ok:
                    T -= float(w[x])
                    w = w.clone()
                    w[x] = 0
            if ok:
                path.append(j)
                c, a, T = j, 0.0, 1.0
                w = before = fresh(c)
        paths.append(path)
        if p is None:
            nxt.append(int(greedy[first + c]))
            continue
        if q is not None and float(w.sum()) == 0:
            w = before
        sums = w.cumsum(0)
        over = (sums > float(r[t]) * sums[-1]).nonzero()
        nxt.append(int(over[0]) if len(over) else int(w.nonzero()[-1]) if float(w.sum()) > 0 else -1)
    return paths, nxt
