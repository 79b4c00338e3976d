"""Steps of one model, each with positions of its own: what one step ran with reaches no other."""
from types import SimpleNamespace

import pytest
import torch

from test_gpu_token_bits import check
from test_gpu_token_step import Problem

pytestmark = pytest.mark.gpu


def with_heads(lib, **kw):
    p = Problem(**kw)
    g = torch.Generator(device="cuda").manual_seed(1)
    randn = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    p.model.heads = [lib.Head([randn(5, p.d)], [randn(5)], 5, 1) for _ in range(2)]
    return p


def served(st):
    st.launch()
    st.synchronize()
    eager = [a.clone() for a in st.actions]
    for a in st.actions:
        a.fill_(9.0)
    torch.cuda.synchronize()
    st.capture()
    st.replay()
    st.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(eager, st.actions))
    return torch.cat([a.flatten() for a in eager])


def test_serving_after_a_group_with_positions(lib):
    """One axis, the same packed rows: a plan without positions turns by its rows' own."""
    p = with_heads(lib, seed=11, norms=False, sections=())
    for q in p.positions:
        q *= 7
    before = served(p.jstep.InferStep(p.model, p.requests, [0, 1]))
    st = p.jstep.GroupStep(p.model, p.requests, p.targets, [0, 1], positions=p.positions)
    st.run()
    torch.cuda.synchronize()
    after = served(p.jstep.InferStep(p.model, p.requests, [0, 1]))
    assert torch.equal(before, after)
    mine = served(p.jstep.InferStep(p.model, p.requests, [0, 1], positions=p.positions))
    assert not torch.equal(before, mine)
    # its hidden rows are the group's, so its actions are heads on their means
    for g in range(2):
        h = [st.out_hidden[r][j, :n].double().mean(0) for r, t in enumerate(p.tenant) if t == g
             for j, n in enumerate(p.lengths[r])]
        want = torch.stack(h) @ p.model.heads[g].W[0].double().T + p.model.heads[g].b[0].double()
        got = mine[:10] if g == 0 else mine[10:]
        # fp32 mean and product of d = 256 terms: 2 x 256 x 2^-24 of the terms' magnitudes
        bar = 2.0 ** -15 * (torch.stack(h).abs() @ p.model.heads[g].W[0].double().T.abs() + 1)
        assert bool(((got.view_as(want).double() - want).abs() <= bar).all())


def test_serving_with_several_axes(lib):
    p = with_heads(lib, seed=12)
    a = p.jstep.InferStep(p.model, p.requests, [0, 1], positions=p.positions)
    first = served(a)
    other = [q.copy() for q in p.positions]
    for q in other:
        q[..., 1] *= 3
    second = served(p.jstep.InferStep(p.model, p.requests, [0, 1], positions=other))
    assert not torch.equal(first, second) and torch.equal(first, served(a))
    with pytest.raises(lib.JNError):  # several axes and no positions
        p.jstep.InferStep(p.model, p.requests, [0, 1])


def test_isolated_runs_of_a_group_with_positions(lib):
    p = Problem(seed=13, sections=())
    for q in p.positions:
        q *= 5
    st = p.jstep.GroupStep(p.model, p.requests, p.targets, [0, 1], positions=p.positions)
    st.run()
    iso = p.jstep.isolated_runs(p.model, p.requests, p.targets, [0, 1], ctx=st.ctx, positions=p.positions)
    for g, one in enumerate(iso):
        one.run()
        torch.cuda.synchronize()
        mine = [k for k, t in enumerate(p.tenant) if t == g]
        assert all(torch.equal(one.out_hidden[j], st.out_hidden[k]) for j, k in enumerate(mine))
    p.check_hidden(st)


def test_weight_gradients_grouped_and_isolated(lib):
    """Element by element, each against the definition: no small row hides behind a large one."""
    p = Problem(seed=14)
    st = p.jstep.GroupStep(p.model, p.requests, p.targets, [0, 1], positions=p.positions)
    iso = p.jstep.isolated_runs(p.model, p.requests, p.targets, [0, 1], ctx=st.ctx, positions=p.positions)
    for step, k, g in ((st, 0, 0), (st, 1, 1), (iso[0], 0, 0), (iso[1], 0, 1)):
        step.run()
        torch.cuda.synchronize()
        io, rows = step.ios[k], step.ios[k].rows.long()
        assert io.dW.dtype is torch.float32 and int((rows < 0).sum()) == 2
        t = SimpleNamespace(rows=io.rows, W=step.token_heads[k].W, targets=torch.where(rows < 0, -1, io.targets), dh=None,
                            dW=io.dW.flatten())
        check(t, step.hidden[rows.clamp(min=0)], 2.0 ** -16)


def test_one_row_between_others(lib):
    """Rows of odd widths, where there is one of them."""
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(1, 3 * 64 + 5, generator=g, device="cuda").to(torch.bfloat16)
    pos = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    qk = lib.QKNormRope(2, 1, 64, theta=1e4)
    y, z = torch.full((1, 197), 7.0, dtype=torch.bfloat16, device="cuda"), torch.empty(1, 192, dtype=torch.bfloat16, device="cuda")
    ctx = lib.Context()
    lib.jn_qk_norm_rope(ctx, qk, x, pos, y)
    lib.jn_qk_norm_rope(ctx, qk, x[:, :192].contiguous(), pos, z)
    assert torch.equal(y[:, :192], z) and bool((y[:, 192:] == 7.0).all())
