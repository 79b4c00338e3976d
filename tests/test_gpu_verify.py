"""Verification of drafted tokens on the GPU against its definition in 64 bits: whole numbers, equal."""
import pytest
import torch

import kv_plain as plain

pytestmark = pytest.mark.gpu
F32, I32 = torch.float32, torch.int32


def trees(seed, nodes, vocab, tree=True, drawn=True, near=0.7, normal=True):
    """Trees of these numbers of nodes with drafts from q (or q's likeliest tokens), on the CPU."""
    gen = torch.Generator().manual_seed(seed)
    n = sum(nodes)
    z = 2 * torch.randn(n, vocab, generator=gen)
    p, q = torch.softmax(z + near * torch.randn(n, vocab, generator=gen), 1), torch.softmax(z, 1)
    j = torch.cat([torch.arange(m) for m in nodes] + [torch.zeros(0, dtype=torch.long)])
    up = torch.where(j > 0, (torch.rand(n, generator=gen) ** 2 * j).long().clamp(max=(j - 1).clamp(min=0)), -1) if tree else j - 1
    cu = torch.tensor([0] + torch.tensor(nodes, dtype=torch.long).cumsum(0).tolist(), dtype=torch.long)
    first = torch.repeat_interleave(cu[:-1], torch.tensor(nodes, dtype=torch.long))
    rows = first + up.clamp(min=0)
    if drawn:
        tok = torch.tensor([int(torch.multinomial(q[int(i)], 1, generator=gen)) for i in rows], dtype=I32)
    else:
        best = q.topk(min(vocab, 8), 1)[1]
        tok = torch.tensor([int(best[int(i), int(k) % best.shape[1]]) for i, k in zip(rows, j)], dtype=I32)
    return {"cu": cu.to(I32), "tokens": tok.to(I32), "parents": up.to(I32) if tree else None, "p": p,
            "q": q if drawn else None, "u": torch.rand(n, generator=gen), "r": torch.rand(len(nodes), generator=gen)}


def run(lib, sets, max_path, vocab=None, ctx=None, pad=0):
    """[(paths, next)] of the tenants, every output checked to be whole."""
    ios, outs = [], []
    for t in sets:
        m = t["cu"].numel() - 1
        o = [torch.full(s, 77, dtype=I32, device="cuda") for s in ((m, max_path), (m,), (m,))]
        dev = {k: x.cuda() if x is not None else None for k, x in t.items()}
        if pad:
            for k in ("p", "q"):
                if dev[k] is not None:
                    dev[k] = torch.cat([dev[k], torch.full((dev[k].shape[0], pad), 9.0, device="cuda")], 1)[:, : dev[k].shape[1]]
        ios.append(lib.TokenVerify(dev["cu"], dev["tokens"], *o, p=dev["p"], greedy=dev.get("greedy"), q=dev["q"], u=dev["u"],
                                   r=dev["r"], parents=dev["parents"], vocab=vocab))
        outs.append(o)
    ws = torch.empty(max(1, lib.jn_tokens_verify_workspace_size(ios)), dtype=torch.uint8, device="cuda").fill_(0xff)
    lib.jn_tenant_tokens_verify(ctx or lib.Context(), ios, ws)
    torch.cuda.synchronize()
    got = []
    for path, count, nxt in outs:
        rows = [r[:c] for r, c in zip(path.tolist(), count.tolist())]
        assert all(set(r[c:]) <= {-1} for r, c in zip(path.tolist(), count.tolist()))
        got.append((rows, nxt.tolist()))
    return got


def check(lib, sets, max_path, vocab=None, pad=0):
    got = run(lib, sets, max_path, vocab, pad=pad)
    for t, g in zip(sets, got):
        want = plain.verify(t["cu"].tolist(), t["tokens"], t["parents"], t["p"], t["q"], t.get("greedy"), t["u"], t["r"],
                            vocab or t["p"].shape[1], max_path, t["tokens"].numel())
        assert g == (want[0], want[1])
    return got


@pytest.mark.parametrize("vocab", [1, 2, 7, 300, 1025, 32003])
@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("drawn", [True, False])
def test_trees(lib, vocab, tree, drawn):
    check(lib, [trees(vocab + tree, [1, 5, 0, 9, 25, 2], vocab, tree, drawn)], 25)


@pytest.mark.parametrize("drawn", [True, False])
def test_many_rejections(lib, drawn):
    """Drafts far from the target: every child of a wide node is tried."""
    t = trees(3, [40, 33], 500, True, drawn, near=6.0)
    t["parents"] = torch.where(torch.arange(73) % 5 == 4, t["parents"], torch.tensor(0)).to(I32)
    got = check(lib, [t], 40)
    assert all(len(p) < 20 for p in got[0][0])


def test_equal_distributions_stand(lib):
    """p == q: a drawn draft stands whatever its number."""
    t = trees(4, [9, 4], 300, False, True)
    t["p"] = t["q"].clone()
    assert [len(p) for p in check(lib, [t], 9)[0][0]] == [9, 4]


def test_nothing_left(lib):
    """A rejection that leaves no weight falls back to the weights before it; no weight at all draws nothing."""
    t = trees(5, [2, 2, 1], 16, False, True)
    t["p"].zero_()
    t["p"][0, 3], t["p"][2, 5] = 0.25, 0.0
    t["q"].fill_(0.5)
    t["tokens"].fill_(3)
    t["u"].fill_(0.9)
    got = check(lib, [t], 4)
    assert got[0] == ([[0], [0], [0]], [3, -1, -1])


def test_weights_that_are_none(lib):
    """NaN and negative weights count as nothing, tokens outside the vocabulary are passed over, bad parents not reached."""
    t = trees(6, [8, 6], 64, True, False)
    t["p"][:, ::3] = float("nan")
    t["p"][:, 1::3] *= -1
    t["tokens"] = torch.tensor([0, 2, -1, 64, 5, 2 ** 31 - 1, 8, 11, 0, 2, 2, 2, 5, 8], dtype=I32)
    t["parents"] = torch.tensor([-1, 0, 0, 0, 1, 1, 99, 6, 3, -4, 0, 0, 2, 3], dtype=I32)
    check(lib, [t], 8)
    t["q"] = torch.softmax(torch.randn(14, 64), 1)
    t["q"][:, 5] = float("nan")
    check(lib, [t], 8)


def test_numbers_at_their_ends(lib):
    """u = 0 lets any possible token stand, r = 0 draws the first, r just below 1 the last."""
    t = trees(7, [6, 6, 6], 100, True, True)
    t["u"].zero_()
    t["r"] = torch.tensor([0.0, 1.0 - 2.0 ** -24, 0.5])
    check(lib, [t], 6)
    one = trees(8, [1, 1], 50, False, False)
    one["r"] = torch.tensor([0.0, 1.0 - 2.0 ** -24])
    one["p"][:, :4] = 0
    one["p"][:, 40:] = 0
    got = check(lib, [one], 1)
    assert got[0][1] == [4, 39]


def test_short_paths_and_outer_rows(lib):
    """max_path ends the walk; cu_nodes outside its range is bounded; wider rows than the vocabulary."""
    t = trees(9, [9, 7, 5], 90, True, True, near=0.1)
    check(lib, [t], 3, pad=13)
    check(lib, [t], 1)
    t["cu"] = torch.tensor([-3, 9, 16, 10 ** 9], dtype=I32)
    check(lib, [t], 9)
    t["cu"] = torch.tensor([0, 9, 4, 21], dtype=I32)
    check(lib, [t], 9, vocab=90)


def test_chains_longer_than_a_tree_may_be(lib):
    t = trees(10, [400], 20, False, True)
    t["p"] = t["q"].clone()
    assert len(check(lib, [t], 400)[0][0][0]) == 400
    wide = trees(11, [300], 20, True, False)  # of a tree 256 nodes are looked at
    wide["p"].fill_(0.0)
    wide["p"][:, 1] = 1.0
    wide["tokens"].fill_(1)
    wide["parents"] = (torch.arange(300) - 1).to(I32)
    assert len(check(lib, [wide], 300)[0][0][0]) == 256


def test_greedy_targets(lib):
    t = trees(12, [9, 5, 1], 50, True, False)
    t["greedy"] = torch.randint(0, 50, (15,), dtype=I32)
    t["greedy"][0] = t["tokens"][1]
    t["p"] = t["u"] = t["r"] = None
    got = run(lib, [t], 9, vocab=50)
    want = plain.verify(t["cu"].tolist(), t["tokens"], t["parents"], None, None, t["greedy"], None, None, 50, 9, 15)
    assert got[0] == want


@pytest.mark.parametrize("tenants", [1, 3, 24, 25, 60])
def test_tenants_of_their_own(lib, tenants):
    """More tenants than one launch takes; a tenant without trees."""
    sets = [trees(20 + g, [1 + g % 5, 3] if g != 1 else [], 40 + g, g % 2 == 0, g % 3 != 0) for g in range(tenants)]
    check(lib, sets, 7)


def test_chances(lib):
    """A drawn draft stands with chance sum min(p, q), and a token comes out with the target's probability."""
    n, vocab = 6000, 5
    p, q = torch.tensor([0.5, 0.2, 0.1, 0.15, 0.05]), torch.tensor([0.1, 0.3, 0.3, 0.1, 0.2])
    gen = torch.Generator().manual_seed(1)
    drafts = torch.multinomial(q, 2 * n, True, generator=gen).view(n, 2)
    t = {"cu": torch.arange(0, 3 * n + 1, 3).to(I32), "parents": torch.tensor([-1, 0, 0] * n, dtype=I32),
         "tokens": torch.cat([torch.zeros(n, 1), drafts], 1).flatten().to(I32), "p": p.expand(3 * n, 5).contiguous(),
         "q": q.expand(3 * n, 5).contiguous(), "u": torch.rand(3 * n, generator=gen), "r": torch.rand(n, generator=gen)}
    paths, nxt = run(lib, [t], 3)[0]
    out = [int(t["tokens"][3 * i + p_[1]]) if len(p_) > 1 else x for i, (p_, x) in enumerate(zip(paths, nxt))]
    share = torch.bincount(torch.tensor(out), minlength=5) / n
    # five deviations of a count of n draws
    assert bool(((share - p).abs() < 5 * (p * (1 - p) / n).sqrt()).all())
