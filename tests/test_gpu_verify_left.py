"""Picked drafts whose rejections take every token that the target has: the token behind is drawn from what was there
before the last of them."""
import pytest
import torch

from test_gpu_verify import run, trees

pytestmark = pytest.mark.gpu
I32 = torch.int32


def wide(p, tokens, u, r=0.5):
    """One tree of a root and its children, picked."""
    n = len(tokens) + 1
    rows = torch.zeros(n, len(p))
    rows[0] = torch.tensor(p)
    return {"cu": torch.tensor([0, n], dtype=I32), "tokens": torch.tensor([0, *tokens], dtype=I32),
            "parents": torch.tensor([-1] + [0] * (n - 1), dtype=I32), "p": rows, "q": None, "u": torch.tensor([0.0, *u]),
            "r": torch.tensor([r])}


def definition(t):
    """joynexus.h's walk of picked drafts, a tree at a time: (paths, next)."""
    cu, paths, nxt = t["cu"].tolist(), [], []
    tokens, u = t["tokens"].tolist(), t["u"].double().tolist()
    for i in range(len(cu) - 1):
        first, n = cu[i], cu[i + 1] - cu[i]
        up = t["parents"][first: first + n].tolist() if t["parents"] is not None else list(range(-1, n - 1))
        weights = lambda c: {k: x for k, x in enumerate(t["p"][first + c].double().tolist()) if x > 0}  # noqa: E731
        path, w, before, T = [0], weights(0), {}, 1.0
        for j in range(1, n):
            if up[j] != path[-1]:
                continue
            x = tokens[first + j]
            if u[first + j] * T < w.get(x, 0.0):
                path.append(j)
                w, before, T = weights(j), {}, 1.0
            elif x in w:
                before, T = dict(w), T - w[x]
                del w[x]
        w, at = w or before, 0.0
        token = -1
        for k in sorted(w):
            at += w[k]
            if at > float(t["r"][i]) * sum(w.values()):
                token = k
                break
        paths.append(path)
        nxt.append(token)
    return paths, nxt


# rejected for certain: each number times what is left is above the token's probability
GONE = [([0.5, 0.25], [0, 1], 1), ([0.5, 0.25], [1, 0], 0), ([0.25], [0], 0), ([0.0, 0.25, 0.0], [1], 1),
        ([0.5, 0.25, 0.0], [0, 1, 1, 2], 1), ([0.5, 0.25, 0.0], [0, 0, 2, 1, 0], 1), ([0.125, 0.25, 0.125, 0.25], [3, 0, 2, 1], 1),
        ([0.0, 0.0], [0, 1], -1), ([float("nan"), -1.0], [0, 1], -1)]


@pytest.mark.parametrize("p,tokens,want", GONE)
def test_the_last_rejected_token_comes_back(lib, p, tokens, want):
    for r in (0.0, 0.5, 1.0 - 2.0 ** -24):
        t = wide(p, tokens, [0.99] * len(tokens), r)
        assert definition(t) == ([[0]], [want])
        assert run(lib, [t], len(tokens) + 1)[0] == ([[0]], [want])


def test_an_ordinary_rejection_is_what_it_was(lib):
    """Tokens that are left go before the one that was rejected last."""
    t = wide([0.5, 0.25, 0.125], [0, 1], [0.99, 0.99])
    assert run(lib, [t], 3)[0] == ([[0]], [2])


def cut(seed, nodes, vocab, tree, keep):
    """Trees of picked drafts whose targets hold `keep` tokens, in quarters, eighths and so on, all of them drafted."""
    t = trees(seed, nodes, vocab, tree, False)
    gen = torch.Generator().manual_seed(seed)
    best = torch.randperm(vocab, generator=gen)[:keep]
    t["p"].zero_()
    t["p"][:, best] = 2.0 ** -(2.0 + torch.arange(keep))
    t["tokens"] = best[torch.randint(0, keep, t["tokens"].shape, generator=gen)].to(I32)
    return t


@pytest.mark.parametrize("vocab", [3, 300, 20011, 60001])
@pytest.mark.parametrize("tree", [True, False])
def test_targets_of_few_tokens(lib, vocab, tree):
    """Every token's piece of a long row, behind standing nodes too."""
    t = cut(vocab, 3 * [25, 9, 1, 40, 2, 17], vocab, tree, 1 + (vocab > 3))
    want = definition(t)
    assert -1 not in want[1] and any(len(p) > 1 for p in want[0])
    assert run(lib, [t], 40)[0] == want


def test_beside_drawn_drafts_and_likeliest_tokens(lib):
    """Tenants of every kind in one call: several launches over rows, of which picked drafts need one."""
    sets = [trees(1, [9, 9], 9000, True, True), cut(2, [12, 3], 9000, True, 2), cut(3, [5], 70, False, 1)]
    got = run(lib, sets, 12)
    assert got[1:] == [definition(t) for t in sets[1:]]
    assert got[0] == run(lib, sets[:1], 12)[0]
