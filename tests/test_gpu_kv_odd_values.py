"""Keys and values that are not finite: what sees them, what does not, with a bound for every result."""
import pytest
import torch

import kv_plain as plain
from test_gpu_kv import BF16, attend, check_rows, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv,hd,new", [(1, 1, 64, 1), (8, 2, 128, 3), (8, 1, 256, 40), (4, 2, 32, 70)])
def test_a_key_of_minus_infinity_is_nothing(lib, margin, heads, kv, hd, new):
    """Its score is -inf where the query is positive: the result is that of the other keys, within their tolerance."""
    b, k, v, gen = make(6, kv, hd, 16, [40], [new], "whole", pad=0)
    q = (0.1 + torch.rand(new, heads * hd, generator=gen)).to(BF16)
    # the same batch with its key 16 .. 31's page taken away, against one whose keys there are -inf
    without = dict(b, pages=b["pages"].clone())
    without["pages"][0, 1] = -1
    want, tol = plain.attention(without, k[0], v[0], q, heads, torch.full(q.shape, float("nan")))
    assert bool(torch.isfinite(want).all() and torch.isfinite(tol).all() and (tol < 0.1).all())
    k[0, b["pages"][0, 1]] = -float("inf")
    check_rows(attend(lib, b, k, v, q, heads), want, tol, margin)


@pytest.mark.parametrize("heads,kv,hd", [(4, 1, 64), (16, 2, 128), (8, 1, 256), (2, 2, 32)])
@pytest.mark.parametrize("past,new", [(45, 5), (0, 9), (45, 70), (64, 200), (3, 150)])
def test_values_of_a_chains_later_rows(lib, margin, heads, kv, hd, past, new):
    """NaN and infinities in new rows reach the rows from there on, in their own columns, and no row before them."""
    b, k, v, gen = make(past + new, kv, hd, 32, [past, 7], [new, 3], "chain", pad=1)
    odd = {new // 3: (0, float("nan")), new // 2: (5, float("inf")), new - 1: (hd - 1, -float("inf"))}
    clean = v.clone()
    for j, (col, x) in odd.items():
        g, r = plain.place(b, k.shape[1], 0, past + j)
        v[0, g, :, r, col] = x
        clean[0, g, :, r, col] = 0.0
    q = torch.randn(b["rows"], heads * hd, generator=gen).to(BF16)
    got = attend(lib, b, k, v, q, heads).double()
    want, tol = plain.attention(b, k[0], clean[0], q, heads, torch.full(got.shape, float("nan")))
    for j, (col, x) in odd.items():
        for a in range(heads):
            want[j: new, a * hd + col] = float("nan") if x != x else x
    live = torch.arange(b["rows"]) < new + 3
    fine = torch.isfinite(want) & live[:, None]
    err = (got - want).abs()[fine] / tol[fine]
    margin("attention", float(err.max()), 1.0)
    assert bool((err <= 1).all())
    for x in (float("inf"), -float("inf")):
        assert torch.equal((got == x) & live[:, None], want == x)
    assert torch.equal(torch.isnan(got) & live[:, None], torch.isnan(want) & live[:, None])
    assert bool(torch.isnan(got[~live]).all())
