"""Positions belong to a step, not to the model it shares: which ones the library is called with (CPU; the device calls
are recorded in their place)."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch  # before the library: both then share one HIP runtime

D, HEADS = 128, 4
LENGTHS, TENANTS = [[3, 5], [4], [2]], [0, 1, 0]


@pytest.fixture
def calls(lib, monkeypatch):
    """Positions of every forward, in order, as the library got them."""
    seen = []

    def pack(h, req, R, ten, G, o, maps, mb, tokens, tb, out):
        out._obj.T = tokens_rows(req, R)
        return 0

    def tokens_rows(req, R):
        return sum(sum(req[i].lengths[j] for j in range(req[i].n_samples)) for i in range(R))

    monkeypatch.setattr(lib._lib, "jn_pack_group", pack)
    monkeypatch.setattr(lib._lib, "jn_backbone_forward", lambda h, bb, p, hid, ws, n: seen.append(bb._obj.pos) or 0)
    monkeypatch.setattr(lib._lib, "jn_tenant_tokens_decode", lambda *a: 0)
    return seen


def model(lib, sections=(4, 6, 6)):
    from paper_2607_16074_amd import step
    bf = lambda *n: np.zeros(n, np.uint16)  # noqa: E731
    hd = D // HEADS
    layer = {"wqkv": bf(3 * D, D), "wo": bf(D, D), "w_up": bf(D, D), "w_down": bf(D, D), "g1": bf(D), "g2": bf(D),
             "gq": bf(hd), "gk": bf(hd)}
    return step.Model.from_arrays([layer], bf(D), HEADS, 1e-6, [None, None], [{"action_dim": 1, "chunk": 1}] * 2, 7, "cpu",
                                  rope_theta=1e4, rope_sections=sections, token_heads=[bf(50, D), bf(60, D)])


def group(lib, m, positions, **kw):
    from paper_2607_16074_amd import step
    reqs = requests(lib)
    return step.GroupStep(m, reqs, targets(), [0, 1], ctx=SimpleNamespace(handle=None), device="cpu", positions=positions, **kw)


def requests(lib):
    return [lib.Request(t, torch.zeros(len(ln), 6, D, dtype=torch.bfloat16), ln) for t, ln in zip(TENANTS, LENGTHS)]


def targets():
    one = np.zeros(1, np.int32)
    return {0: (one, one, one), 1: (one, one, one)}


def positions(axes, start):
    return [start + 100 * k + np.arange(len(ln) * 6 * axes, dtype=np.int32).reshape(len(ln), 6, axes)
            for k, ln in enumerate(LENGTHS)]


def test_a_step_leaves_the_model_as_it_was(lib, calls):
    m = model(lib)
    a, b = group(lib, m, positions(3, 0)), group(lib, m, positions(3, 5000))
    for st in (a, b, a):
        st.pack()
        st.backbone()
        assert m.backbone.struct.pos is None and m.backbone.pos is None
    assert calls == [a.pos.data_ptr(), b.pos.data_ptr(), a.pos.data_ptr()]
    assert a.pos[:3, 0].tolist() == [0, 3, 6] and not torch.equal(a.pos, b.pos)


def test_a_step_without_positions_leaves_the_users(lib, calls):
    m = model(lib, ())
    own = torch.arange(14, dtype=torch.int32)[:, None].contiguous()
    m.backbone.set_positions(own)
    plain, with_own = group(lib, m, None), group(lib, m, positions(1, 9))
    for st in (plain, with_own, plain):
        st.pack()
        st.backbone()
        assert m.backbone.pos is own and m.backbone.struct.pos == own.data_ptr()
    assert calls == [own.data_ptr(), with_own.pos.data_ptr(), own.data_ptr()]
    m.backbone.set_positions(None)
    plain.backbone()
    assert calls[-1] is None


def test_decoding(lib, calls):
    from paper_2607_16074_amd import step
    m = model(lib)
    st = step.DecodeStep(m, requests(lib), [0, 1], ctx=SimpleNamespace(handle=None), device="cpu", positions=positions(3, 3))
    st.run()
    assert calls == [st.pos.data_ptr()] and m.backbone.struct.pos is None


def test_isolated_steps_have_their_tenants_positions(lib, calls):
    from paper_2607_16074_amd import step
    m, p = model(lib, ()), positions(1, 7)
    iso = step.isolated_runs(m, requests(lib), targets(), [0, 1], ctx=SimpleNamespace(handle=None), device="cpu", positions=p)
    for st in iso:
        st.pack()
        st.backbone()
    assert calls == [st.pos.data_ptr() for st in iso]
    assert iso[0].pos[:, 0].tolist() == [*p[0][0, :3, 0], *p[0][1, :5, 0], *p[2][0, :2, 0]]
    assert iso[1].pos[:, 0].tolist() == p[1][0, :4, 0].tolist()


def test_positions_of_another_size_are_refused(lib, calls):
    m = model(lib)
    st = group(lib, m, positions(3, 0))
    st.pack()
    for bad, error in ((st.pos[:-1].contiguous(), ValueError), (st.pos[:, 0].contiguous(), ValueError),
                       (st.pos[:, :2].contiguous(), TypeError), (st.pos.long(), TypeError)):
        with pytest.raises(error):
            lib.jn_backbone_forward(st.ctx, m.backbone, st.packed, st.hidden, st.bb_ws, bad)
    assert calls == []


def test_misaligned_positions_are_refused(lib):
    m = model(lib)
    heads = [lib.Head([torch.zeros(2, D)], [torch.zeros(2)], 2, 1) for _ in range(2)]
    table, reqs = [lib.Tenant(7, D)] * 2, requests(lib)
    pos = torch.zeros(14, 3, dtype=torch.int32)

    def size():
        return lib.jn_infer_workspace_size(reqs, table, D, 1, m.backbone, heads)

    m.backbone.set_positions(pos)
    assert size() > 0
    for off in (1, 2, 3):
        m.backbone.struct.pos = pos.data_ptr() + off
        with pytest.raises(lib.JNError) as e:
            size()
        assert e.value.status == lib._abi.JN_EINVAL
