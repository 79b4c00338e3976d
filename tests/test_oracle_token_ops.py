"""The formulas behind the GPU tests of head norms, rotation and token heads, on the CPU: gradients against central
differences, the rotation's invariances, and the plain forms of perf/operators.py against its 64-bit definitions."""
import importlib.util
import os

import pytest
import torch

from test_gpu_qk import pair_axes, reference

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F64 = torch.float64


def test_pair_axes_of_known_sections():
    assert pair_axes(16, [4, 2, 2], False) == [0, 0, 0, 0, 1, 1, 2, 2]
    assert pair_axes(16, [4, 2, 2], True) == [0, 1, 2, 0, 1, 2, 0, 0]
    assert pair_axes(16, [3, 3, 2], True) == [0, 1, 2, 0, 1, 2, 0, 1]
    assert pair_axes(16, [0, 8], False) == [1] * 8
    assert pair_axes(16, [], True) == [0] * 8
    for sec in ([8, 4, 4], [6, 5, 5], [16, 0, 0]):
        got = pair_axes(32, sec, True)
        assert [got.count(a) for a in range(3)] == sec


@pytest.mark.parametrize("axes,interleaved", [(1, False), (3, False), (3, True)])
@pytest.mark.parametrize("norm", [True, False])
def test_qk_gradients_against_differences(axes, interleaved, norm):
    g = torch.Generator().manual_seed(3)
    rows, heads, kv, hd = 4, 2, 1, 16
    x = torch.randn(rows, (heads + kv) * hd, generator=g, dtype=F64)
    dy = torch.randn(rows, (heads + kv) * hd, generator=g, dtype=F64)
    gains = [1 + 0.3 * torch.randn(hd, generator=g, dtype=F64) for _ in range(2)] if norm else [None, None]
    pos = torch.randint(0, 50, (rows, axes), generator=g).to(torch.int32)
    sec = [8 - 2 * (axes - 1)] + [2] * (axes - 1) if axes > 1 else []
    args = (pos, heads, kv, hd, 1e4, sec, interleaved)
    (dx, _), gq, gk = reference(x, *gains, *args, dy=dy)

    def loss(x_, gains_):
        return float((reference(x_, *gains_, *args)[0] * dy).sum())

    e = 1e-5
    for i in (0, 17, 47, 100):
        a, b = x.clone(), x.clone()
        a.view(-1)[i] += e
        b.view(-1)[i] -= e
        assert abs((loss(a, gains) - loss(b, gains)) / (2 * e) - float(dx.view(-1)[i])) < 1e-7
    for k, got in enumerate((gq, gk)):
        if not norm:
            assert got is None
            continue
        for i in (0, 9):
            p, m = [list(gains) for _ in range(2)]
            p[k], m[k] = gains[k].clone(), gains[k].clone()
            p[k][i] += e
            m[k][i] -= e
            assert abs((loss(x, p) - loss(x, m)) / (2 * e) - float(got[0][i])) < 1e-7


def test_rotation_depends_on_differences_of_positions():
    """A common shift of an axis leaves the products of queries and keys of a row pair as they were."""
    g = torch.Generator().manual_seed(4)
    x = torch.randn(2, 2 * 32, generator=g, dtype=F64)
    pos = torch.tensor([[3, 7, 2], [11, 0, 5]], dtype=torch.int32)
    dots = []
    for shift in ([0, 0, 0], [100, 0, 0], [5, -9, 1000]):
        y = reference(x, None, None, pos + torch.tensor(shift, dtype=torch.int32), 1, 1, 32, 1e4, [8, 4, 4], True)[0]
        dots.append(float(y[0, :32] @ y[1, 32:]))
    assert max(dots) - min(dots) < 1e-11


def test_cross_entropy_gradients_against_differences():
    g = torch.Generator().manual_seed(5)
    n, v, d = 5, 11, 6
    h, w = torch.randn(n, d, generator=g, dtype=F64), torch.randn(v, d, generator=g, dtype=F64)
    t = torch.tensor([3, 0, 10, 3, 7])

    def loss(h_, w_):
        return float(-torch.log_softmax(h_ @ w_.T, 1).gather(1, t[:, None]).mean())

    dz = torch.softmax(h @ w.T, 1)
    dz[torch.arange(n), t] -= 1
    dz /= n
    e = 1e-6
    for x, got, f in ((w, dz.T @ h, lambda y: loss(h, y)), (h, dz @ w, lambda y: loss(y, w))):
        for i in range(0, x.numel(), 7):
            a, b = x.clone(), x.clone()
            a.view(-1)[i] += e
            b.view(-1)[i] -= e
            assert abs((f(a) - f(b)) / (2 * e) - float(got.reshape(-1)[i])) < 1e-8


def test_plain_forms_agree_with_their_definitions():
    spec = importlib.util.spec_from_file_location("operators", os.path.join(ROOT, "perf", "operators.py"))
    ops = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ops)
    ops.DEV = "cpu"

    def leaves(v, path=""):
        if isinstance(v, torch.Tensor):
            yield path, v
        for k, x in v.items() if isinstance(v, dict) else enumerate(v) if isinstance(v, list) else ():
            yield from leaves(x, f"{path}.{k}")

    for c in ops.listed():
        c = dict(c, rows=min(c["rows"], 50)) | ({"vocab": min(c["vocab"], 300), "d": 128} if "vocab" in c else {})
        got, want = dict(leaves(ops.run(ops.prepare(c, 1)))), dict(leaves(ops.exact(c, 1)))
        assert got.keys() == want.keys()
        for k, x in got.items():
            if not x.is_floating_point():
                assert torch.equal(x, want[k])
                continue
            # fp32 arithmetic, one rounding of bf16 results
            bar = 2e-5 if x.dtype == torch.float32 else 4e-3
            assert float((x.double() - want[k]).norm()) <= bar * float(want[k].norm()) + 1e-30, (c["name"], k)
