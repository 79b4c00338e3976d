"""Token-predicting tenants end to end, as a program runs them: pack, backbone with head norms and several position
axes, cross entropy with gradients, per-tenant AdamW, decoding.  Hidden rows against a float64 evaluation of the same
backbone (2e-2 max-relative, the bar of every backbone test here); everything behind them stage-wise from the GPU's
own hidden rows, with the bars of test_gpu_tokens.py."""
import numpy as np
import pytest
import torch

from oracle import backbone as obb
from test_gpu_qk import pair_axes
from test_gpu_tokens import BF

pytestmark = pytest.mark.gpu

EPS = 1e-6


def bits(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)


class Problem:
    """Two tenants with vocabularies of their own; samples of a 4 x 4 image grid and text."""

    def __init__(self, d=256, heads=4, kv=2, layers=2, ffn=512, norms=True, sections=(16, 8, 8), interleaved=True, seed=0,
                 causal=True, theta=1e4):
        from paper_2607_16074_amd import Request
        from paper_2607_16074_amd import step as jstep
        self.jstep = jstep
        r = np.random.default_rng(seed)
        hd = d // heads
        self.d, self.heads, self.kv, self.causal, self.theta = d, heads, kv, causal, theta
        self.sections, self.interleaved = sections, interleaved
        w = lambda *s: bits(r.normal(size=s) * (1.0 / s[-1]) ** 0.5)  # noqa: E731
        gain = lambda n: bits(1 + 0.2 * r.normal(size=n))  # noqa: E731
        self.layers = []
        for _ in range(layers):
            L = {"wqkv": w((heads + 2 * kv) * hd, d), "wo": w(d, d), "w_up": w(ffn, d), "w_down": w(d, ffn), "g1": gain(d),
                 "g2": gain(d)}
            if norms:
                L |= {"gq": gain(hd), "gk": gain(hd)}
            self.layers.append(L)
        self.gf = gain(d)
        self.vocab = [301, 1000]
        self.W = [w(v, d) for v in self.vocab]
        meta = [{"action_dim": 1, "chunk": 1}] * 2
        self.model = jstep.Model.from_arrays(self.layers, self.gf, heads, EPS, [None, None], meta, 77, "cuda",
                                             n_kv_heads=kv, causal=causal, rope_theta=theta, rope_sections=sections,
                                             rope_interleaved=interleaved, token_heads=self.W)
        self.lengths = [[20, 33], [17], [40, 21, 25]]
        self.tenant = [0, 1, 1]
        self.embeds, self.positions, self.requests = [], [], []
        for t, ln in zip(self.tenant, self.lengths):
            m = max(ln) + 3
            e = bits(r.normal(size=(len(ln), m, d)))
            p = np.zeros((len(ln), m, max(1, len(sections))), np.int32)
            for j in range(m):
                p[:, j] = [0, j // 4, j % 4, 0][: p.shape[-1]] if j < 16 else 4 + j - 16
            p += r.integers(0, 100, (len(ln), 1, 1)).astype(np.int32)
            self.embeds.append(e)
            self.positions.append(p)
            self.requests.append(Request(t, jstep._dev_bf16(e, "cuda"), ln))
        self.targets = {}
        for g in range(2):
            own = [n for t, ln in zip(self.tenant, self.lengths) if t == g for n in ln]
            pairs = [(s, j) for s, n in enumerate(own) for j in range(15, n - 1)]
            pairs += [(0, own[0] - 1), (len(own), 0), (0, own[0])]  # a last row, and two that do not exist
            sample, row = (np.array(x, np.int32) for x in zip(*pairs))
            token = r.integers(0, self.vocab[g], len(pairs)).astype(np.int32)
            token[-3] = -1
            self.targets[g] = (sample, row, token)

    def hidden(self, embeds, pos):
        """float64 hidden rows of one sample."""
        x = obb.bf16_to_f64(embeds)
        hd = self.d // self.heads
        ax = pair_axes(hd, list(self.sections), self.interleaved)
        for L in self.layers:
            lw = obb.LayerF64(L, False)
            qkv = obb.rms_norm(x, lw.g1, EPS) @ lw.wqkv.T
            parts = [qkv[:, : self.d], qkv[:, self.d: self.d + self.kv * hd]]
            for k, (n, name) in enumerate(((self.heads, "gq"), (self.kv, "gk"))):
                v = parts[k].reshape(len(x), n, hd)
                if name in L:
                    v = obb.rms_norm(v, obb.bf16_to_f64(L[name]), EPS)
                if self.theta > 0:
                    freq = self.theta ** (-2.0 * np.arange(hd // 2) / hd)
                    a = (pos[:, ax].astype(np.float64) * freq)[:, None]
                    p, o = v[..., : hd // 2], v[..., hd // 2:]
                    v = np.concatenate([p * np.cos(a) - o * np.sin(a), o * np.cos(a) + p * np.sin(a)], -1)
                parts[k] = v.reshape(len(x), -1)
            a = obb.attention(parts[0], parts[1], qkv[:, self.d + self.kv * hd:], self.heads, self.kv, self.causal)
            x = x + a @ lw.wo.T
            x = x + obb.gelu(obb.rms_norm(x, lw.g2, EPS) @ lw.w_up.T) @ lw.w_down.T
        return obb.rms_norm(x, obb.bf16_to_f64(self.gf), EPS)

    def check_hidden(self, step):
        step.unpack()
        torch.cuda.synchronize()
        for r, ln in enumerate(self.lengths):
            got = step.out_hidden[r].double().cpu().numpy()
            for s, n in enumerate(ln):
                want = self.hidden(self.embeds[r][s, :n], self.positions[r][s, :n])
                assert np.abs(got[s, :n] - want).max() / np.abs(want).max() < 2e-2, (r, s)


@pytest.mark.parametrize("kind", ["norms-3-axes", "norms-1-axis", "norms-own-rows", "norms-only", "3-axes-runs", "1-axis"])
def test_backbone(lib, kind):
    kw = {"norms-3-axes": {}, "norms-1-axis": dict(sections=()), "norms-own-rows": dict(sections=()),
          "norms-only": dict(sections=(), theta=0.0), "3-axes-runs": dict(norms=False, interleaved=False, causal=False),
          "1-axis": dict(norms=False, sections=())}[kind]
    p = Problem(seed=3, **kw)
    if kind == "norms-own-rows":
        for q in p.positions:
            q[:] = np.arange(q.shape[1])[None, :, None]
    positions = None if kind in ("norms-own-rows", "norms-only") else p.positions
    for align in (1, 16):
        st = p.jstep.GroupStep(p.model, p.requests, p.targets, [0, 1], align, positions=positions)
        st.pack()
        st.backbone()
        p.check_hidden(st)


def test_old_rotation_keeps_its_bits(lib):
    """One axis, no norms, the rows' own positions: the rotation of before, whatever jn_qk_norm_rope does."""
    p = Problem(seed=4, norms=False, sections=())
    for q in p.positions:
        q[:] = np.arange(q.shape[1])[None, :, None]
    a = p.jstep.GroupStep(p.model, p.requests, p.targets, [0, 1])
    a.ctx.set_trace(True)
    a.pack()
    a.backbone()
    ops = [t[0] for t in a.ctx.trace_read()]
    assert "rope" in ops and "qk_norm_rope" not in ops
    p.check_hidden(a)


def test_training_step_and_decode(lib):
    p = Problem(seed=5)
    st = p.jstep.GroupStep(p.model, p.requests, p.targets, [0, 1], positions=p.positions)
    opt = p.jstep.TenantOptimizer(st, lr=3e-3, weight_decay=0.01)
    lr, wd, b1, b2, eps = (float(np.float32(x)) for x in (3e-3, 0.01, 0.9, 0.999, 1e-8))
    master = [h.W.double() for h in st.token_heads]
    m = [torch.zeros_like(w) for w in master]
    v = [torch.zeros_like(w) for w in master]
    for t in (1, 2):
        st.run()
        torch.cuda.synchronize()
        p.check_hidden(st)
        for g in range(2):
            sample, row, token = p.targets[g]
            io, W = st.ios[g], st.token_heads[g].W
            host = lib.jn_pack_maps_host(st.requests, st.table, p.d, 1)
            own = host["tenant_perm"][host["tenant_sample_off"][g]: host["tenant_sample_off"][g + 1]]
            live = [k for k in range(len(token)) if token[k] >= 0 and sample[k] < len(own) and row[k] < host["seqlens"][own[sample[k]]]]
            assert live == list(range(len(token) - 3))
            at = torch.tensor([int(host["cu_seqlens"][own[sample[k]]] + row[k]) for k in live], device="cuda")
            h, w = st.hidden[at].double(), W.double()
            y = torch.tensor(token[live], device="cuda", dtype=torch.int64)[:, None]
            z = h @ w.T
            lp = torch.log_softmax(z, 1)
            D = p.d * 2.0 ** -24 * (h.abs() @ w.abs().T).amax(1)
            logp = lp.gather(1, y)[:, 0]
            assert bool(((io.logp[: len(live)].double() - logp).abs() <= 2 * D + 2.0 ** -20 * (1 + logp.abs())).all())
            assert bool((io.logp[len(live):] == 0).all())
            assert abs(float(io.loss) + float(logp.mean())) <= float(2 * D.max()) + 2.0 ** -16
            dz = lp.exp().scatter_add(1, y, -torch.ones_like(y, dtype=torch.float64)) / len(live)
            bar = (dz.abs() * (BF + 2.0 ** -9) + lp.exp() * (2 * D / len(live))[:, None]).T @ h.abs()
            assert bool(((io.dW.double() - dz.T @ h).abs() <= 1.01 * bar + 1e-30).all())
            # the optimizer takes the library's own gradient
            gr = io.dW.double()
            m[g] = b1 * m[g] + (1 - b1) * gr
            v[g] = b2 * v[g] + (1 - b2) * gr * gr
            master[g] = master[g] * (1 - lr * wd) - lr / (1 - b1 ** t) * m[g] / ((v[g] / (1 - b2 ** t)).sqrt() + eps)
        opt.step()
        torch.cuda.synchronize()
        for g in range(2):
            got = opt.sets[g][0][0].double()
            # a step off by 4e-7 of the parameter and 2e-6 of the rate, as in the optimizer's own test; two of them
            assert bool(((got - master[g]).abs() <= t * (4e-7 * master[g].abs() + 2e-6 * 3e-3)).all())
            assert torch.equal(st.token_heads[g].W, opt.sets[g][0][0].to(torch.bfloat16))
    dec = p.jstep.DecodeStep(p.model, p.requests, [0, 1], positions=p.positions)
    dec.run()
    torch.cuda.synchronize()
    assert torch.equal(dec.hidden, st.hidden)
    for g in range(2):
        rows = dec.picks[g].rows.long()
        z = dec.hidden[rows].double() @ p.model.token_heads[g].W.double().T
        best = z.gather(1, dec.tokens[g].long()[:, None])[:, 0]
        assert bool((best >= z.amax(1) - 1e-4).all())
        assert bool(((dec.logp[g].double() - torch.log_softmax(z, 1).amax(1)).abs() < 1e-4).all())


def test_grouped_and_isolated(lib):
    """A tenant alone and in a group: the same hidden rows bit for bit; the softmax sums are added in an order that
    follows the launches' shapes, so log-probabilities agree to twice their own bar (the sums' roundings, 2^-20 of 1 +
    |logp|: the logits themselves are the same additions)."""
    p = Problem(seed=6)
    st = p.jstep.GroupStep(p.model, p.requests, p.targets, [0, 1], positions=p.positions)
    st.run()
    for g in range(2):
        idx = [k for k, r in enumerate(p.requests) if r.tenant == g]
        one = p.jstep.GroupStep(p.model, [p.requests[k] for k in idx], p.targets, [g], positions=[p.positions[k] for k in idx])
        one.run()
        torch.cuda.synchronize()
        assert all(torch.equal(one.out_hidden[j], st.out_hidden[k]) for j, k in enumerate(idx))
        a, b = one.ios[0].logp, st.ios[g].logp
        assert bool(((a - b).abs() <= 2 * 2.0 ** -20 * (1 + a.abs())).all())
        # a gradient's bf16 rounding may fall to the other side where the sums differ: a whole step, 2^-7, of each term
        scale = (one.ios[0].dW.abs() + st.ios[g].dW.abs()).max()
        assert float((one.ios[0].dW - st.ios[g].dW).abs().max()) <= 2.0 ** -7 * float(scale)


def test_positions_of_an_inference_plan(lib):
    """The plan reads the positions as they are at a launch, captured or not."""
    p = Problem(seed=7)
    d = p.d
    head = lib.Head([torch.randn(7, d, device="cuda")], [torch.randn(7, device="cuda")], 7, 1)
    table = [lib.Tenant(77, d)] * 2
    host = lib.jn_pack_maps_host(p.requests, table, d, 1)
    pos = p.jstep._dev_i32(p.jstep.packed_positions(p.requests, host, p.positions), "cuda")
    bb = p.model.backbone
    bb.set_positions(pos)
    n = [sum(r.n for r in p.requests if r.tenant == g) for g in range(2)]
    acts = [torch.zeros(k, 7, device="cuda") for k in n]
    ws = torch.empty(lib.jn_infer_workspace_size(p.requests, table, d, 1, bb, [head, head]), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    ctx = lib.Context(stream)
    torch.cuda.synchronize()
    plan = lib.InferPlan(ctx, p.requests, table, d, 1, bb, [head, head], acts, ws)
    plan.capture()
    seen = []
    for shift in (0, 0, 5000):
        # an axis at a time: a common shift of all would leave attention as it was
        pos[:, 1] += shift
        torch.cuda.synchronize()
        plan.launch()
        torch.cuda.synchronize()
        eager = [a.clone() for a in acts]
        for a in acts:
            a.zero_()
        torch.cuda.synchronize()
        plan.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, acts))
        seen.append(torch.cat([a.flatten() for a in eager]))
    assert torch.equal(seen[0], seen[1])
    with pytest.raises(ValueError):
        bb.set_positions(pos[:-1].contiguous())
        lib.InferPlan(ctx, p.requests, table, d, 1, bb, [head, head], acts, ws)


def test_backbone_refusals(lib):
    p = Problem(seed=8)
    st = p.jstep.GroupStep(p.model, p.requests, p.targets, [0, 1], positions=p.positions)
    st.pack()
    abi, bb = lib._abi, p.model.backbone
    st.hidden.fill_(7.0)
    bb.set_positions(st.pos)

    def refused(code):
        with pytest.raises(lib.JNError) as e:
            lib.jn_backbone_forward(st.ctx, bb, st.packed, st.hidden, st.bb_ws)
        assert e.value.status == code, e.value

    keep = abi.jn_backbone.from_buffer_copy(bb.struct)

    def change(code, **kw):
        for k, x in kw.items():
            setattr(bb.struct, k, x)
        refused(code)
        for k in kw:
            setattr(bb.struct, k, getattr(keep, k))

    import ctypes as C
    change(abi.JN_EINVAL, rope_axes=5)
    change(abi.JN_EINVAL, rope_axes=-1)
    change(abi.JN_EINVAL, rope_interleaved=2)
    change(abi.JN_EINVAL, rope_sections=(C.c_int32 * 4)(16, 8, 7, 0))
    change(abi.JN_EINVAL, rope_sections=(C.c_int32 * 4)(4, 14, 14, 0))
    change(abi.JN_EINVAL, rope_theta=0.0)
    change(abi.JN_EINVAL, pos=None)
    gk = bb._arr[1].gk
    bb._arr[1].gk = None
    refused(abi.JN_EINVAL)
    bb._arr[1].gk = gk + 2
    refused(abi.JN_EUNSUPPORTED)
    bb._arr[1].gk = gk
    torch.cuda.synchronize()
    assert bool((st.hidden == 7.0).all())
    with pytest.raises(ValueError):
        bb.set_positions(st.pos[:-1].contiguous())
        lib.jn_backbone_forward(st.ctx, bb, st.packed, st.hidden, st.bb_ws)
    st.backbone()
    p.check_hidden(st)
