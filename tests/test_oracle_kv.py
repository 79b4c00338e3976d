"""CPU pins of the plain definitions behind the calls over a paged cache and the verification of drafts."""
import numpy as np
import pytest
import torch

import kv_plain as plain
from test_gpu_kv import make
from test_gpu_verify import trees

F64 = torch.float64


@pytest.mark.parametrize("mask", ["chain", "whole", "tree"])
def test_attention_is_the_libraries(mask):
    """Against torch's scaled_dot_product_attention in 64 bits over the gathered rows, masks written as matrices."""
    b, k, v, gen = make(1, 2, 32, 16, [20, 0, 37], [5, 9, 1], mask)
    q = torch.randn(b["rows"], 4 * 32, generator=gen).to(torch.bfloat16)
    out, tol = plain.attention(b, k[0], v[0], q, 4, torch.full((b["rows"], 128), 7.0))
    for s, (past, row0, n) in enumerate(plain.sequences(b)):
        at = [plain.place(b, k.shape[1], s, t) for t in range(past + n)]
        kk, vv = (torch.stack([c[0][g, :, r] for g, r in at], 1).to(F64) for c in (k, v))
        new = torch.ones(n, n, dtype=torch.bool)
        if mask == "chain":
            new = new.tril()
        elif mask == "tree":
            up = b["parents"][row0: row0 + n].tolist()
            hop = torch.zeros(n, n, dtype=F64)
            for j, p in enumerate(up):
                if p >= 0:
                    hop[j, p] = 1
            new = torch.linalg.inv(torch.eye(n, dtype=F64) - hop) > 0.5
        m = torch.cat([torch.ones(n, past, dtype=torch.bool), new], 1)
        qq = q[row0: row0 + n].to(F64).view(n, 4, 32).transpose(0, 1)
        w = torch.nn.functional.scaled_dot_product_attention(qq, kk.repeat_interleave(2, 0), vv.repeat_interleave(2, 0), m)
        assert torch.allclose(out[row0: row0 + n], w.transpose(0, 1).flatten(1), atol=1e-12)
    assert bool((out[-2:] == 7).all()) and bool((tol[-2:] == 0).all())


def test_turns_are_those_of_complex_numbers():
    x = torch.randn(3, 16, dtype=F64)
    got = plain.norm_rope(x, None, 1e-6, 1e4, [37], [0] * 8)
    z = torch.complex(x[:, :8], x[:, 8:]) * torch.polar(torch.ones(8, dtype=F64), 37 * 1e4 ** (-torch.arange(8, dtype=F64) / 8))
    assert torch.allclose(got, torch.cat([z.real, z.imag], 1), atol=1e-12)
    g = torch.randn(16)
    assert torch.allclose(plain.norm_rope(x, g, 0.0, 0.0, [0], [0] * 8), torch.nn.functional.rms_norm(x, (16,), g.to(F64), 0.0))


def test_lengths_and_places_are_bounded():
    b, k, _, _ = make(2, 1, 16, 16, [5, 40], [3, 4], bad=[(1, 1, -1)])
    b["cu"], b["past"], b["max_new"] = torch.tensor([-7, 3, 99]), torch.tensor([-1, 10 ** 6]), 4
    places = 16 * b["pages"].shape[1]
    assert plain.sequences(b) == [(0, 0, 3), (places, 3, 4)]
    assert plain.place(b, k.shape[1], 1, 16) is None and plain.place(b, k.shape[1], 0, places) is None


def test_a_kept_path_moves_in_order():
    b, k, v, _ = make(3, 1, 16, 16, [3], [6])
    n = k.clone()
    wk, _, past = plain.keep(b, k, v, torch.tensor([[0, 2, 5, 1]]), [4])
    at = [plain.place(b, k.shape[1], 0, 3 + j) for j in range(6)]
    for to, frm in ((0, 0), (1, 2), (2, 5), (3, 3)):
        assert torch.equal(wk[0][at[to][0], 0, at[to][1]], n[0][at[frm][0], 0, at[frm][1]])
    assert past == [7]


@pytest.mark.parametrize("drawn", [True, False])
def test_a_verified_token_has_the_targets_chance(drawn):
    """Sum over all outcomes of one node with two children, by the intervals of the numbers: exactly p."""
    p = torch.tensor([0.4, 0.1, 0.3, 0.2], dtype=F64)
    q = torch.tensor([0.1, 0.5, 0.2, 0.2], dtype=F64)
    got = torch.zeros(4, dtype=F64)
    kids = [(x, y) for x in range(4) for y in range(4)] if drawn else [(1, 0)]
    for x, y in kids:
        chance = float(q[x] * q[y]) if drawn else 1.0
        # first child, second child, then what is left
        w, left = p, 1.0
        for c in (x, y):
            ok = min(1.0, float(w[c] / w.sum()) / float(q[c])) if drawn else float(w[c] / w.sum())
            got[c] += chance * left * ok
            left *= 1 - ok
            if left <= 0:
                break
            w = w / w.sum()
            if drawn:
                w = (w - q).clamp(min=0)
            else:
                w = w.clone()
                w[c] = 0
        if left > 1e-15:
            got += chance * left * w / w.sum()
    assert torch.allclose(got, p, atol=1e-12)
    # and the definition's walk takes these decisions, at numbers on either side of each border
    t = {"cu": [0, 3], "tok": torch.tensor([0, 1, 1]), "up": torch.tensor([-1, 0, 0])}
    rows = lambda v: v.expand(3, 4)  # noqa: E731
    border = min(1.0, float(p[1] / q[1])) if drawn else float(p[1])
    for du, want in ((-1e-9, [0, 1]), (1e-9, None)):
        path, _ = plain.verify(t["cu"], t["tok"], t["up"], rows(p), rows(q) if drawn else None, None,
                               torch.tensor([0, border + du, 0.999], dtype=F64), torch.tensor([0.5], dtype=F64), 4, 3, 3)
        assert path[0] == (want or [0])


def test_residuals_by_one_number_are_the_residuals():
    """max(p_k - q, 0) / T, repeated, is max(p - a q, 0) over its sum with a the sum of the sums before."""
    r = np.random.default_rng(0)
    p, q = (torch.from_numpy(r.dirichlet(np.ones(50))) for _ in range(2))
    w, a, T = p, 0.0, 1.0
    for _ in range(4):
        w = (w / w.sum() - q).clamp(min=0)
        a += T
        f = (p - a * q).clamp(min=0)
        T = float(f.sum())
        if T == 0:
            break
        assert torch.allclose(w / w.sum(), f / T, atol=1e-12)


def test_trees_are_made_of_their_parents_rows():
    t = trees(1, [5, 1, 7], 30)
    assert t["cu"].tolist() == [0, 5, 6, 13] and all(-1 <= int(u) < j for u, j in zip(t["parents"], [*range(5), 0, *range(7)]))
