"""Steps of one model, each with positions of its own: what one step ran with reaches no other."""
import pytest
import torch

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
