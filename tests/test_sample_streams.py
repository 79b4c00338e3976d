"""Sampled steps of token streams on a stream of the context's own: verification follows the caller's stream, and the
caller's tensors outlive it."""
import contextlib
from types import SimpleNamespace

import pytest
import torch

I32 = torch.int32


class Noted(torch.Tensor):
    """A tensor that notes which streams it is recorded on."""

    notes: list = []

    def record_stream(self, stream):
        Noted.notes.append((self.untyped_storage().data_ptr(), stream))


class FakeStream:
    def __init__(self, log):
        self.log = log

    def wait_stream(self, other):
        self.log.append(("wait", self, other))


@pytest.mark.parametrize("same", [False, True])
def test_verification_waits_for_the_callers_stream(lib, monkeypatch, same):
    """On the CPU, with streams that only note their calls."""
    from paper_2607_16074_amd import step
    log = []
    here = FakeStream(log)
    there = here if same else FakeStream(log)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: here)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(step, "jn_tenant_tokens_verify", lambda *a: log.append(("verify",)))
    Noted.notes = []
    st = object.__new__(step.SpeculativeStep)
    i = lambda *s: torch.zeros(s, dtype=I32)  # noqa: E731
    st.ctx, st.n, st.nodes, st.max_len = SimpleNamespace(stream=there), 3, 2, 8
    st.tokens, st.path, st.n_path, st.next, st.past, st.tree = i(6), i(3, 2), i(3), i(3), i(3), None
    st.full = torch.zeros(3, dtype=torch.bool)
    st.cu = torch.arange(4, dtype=I32) * 2
    st.slices = [(slice(0, 1), slice(0, 2)), (slice(1, 3), slice(2, 6))]
    t = [torch.rand(*s).as_subclass(Noted) for s in ((2, 5), (4, 7), (2, 5), (4, 7), (6,), (3,))]
    st.sample(t[:2], t[4], t[5], t[2:4])
    assert ("verify",) in log
    if same:
        return
    at = log.index(("verify",))
    assert ("wait", there, here) in log[:at]
    kept = {x for x, s in Noted.notes if s is there}
    assert kept == {x.untyped_storage().data_ptr() for x in t}


@pytest.mark.gpu
def test_probabilities_of_another_stream_than_the_contexts(lib):
    """Formed behind much work on the caller's stream and gone when the call returns."""
    import kv_plain as plain
    from paper_2607_16074_amd import step
    from test_gpu_speculative import Speaker
    sp, gen = Speaker(lib, 13), torch.Generator().manual_seed(5)
    st = step.SpeculativeStep(sp.model, [0, 1], [1, 2], 64, 4, None, 16, lib.Context(torch.cuda.Stream()))
    z = [torch.randn(n, h.shape[0], generator=gen) for n, h in zip((4, 8), sp.heads)]
    draft = [2 * torch.randn(n, h.shape[0], generator=gen) for n, h in zip((4, 8), sp.heads)]
    u, r = torch.rand(12, generator=gen), torch.rand(3, generator=gen)
    tokens = torch.randint(0, 33, (12,), generator=gen).to(I32)
    dev = [x.cuda() for x in (*z, *draft, u, r)]
    st.tokens.copy_(tokens)
    busy = torch.zeros(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    for _ in range(50):
        busy = busy @ busy
    p, q = [torch.softmax(x, 1) for x in dev[:2]], [torch.softmax(x, 1) for x in dev[2:4]]
    host = [x.clone() for x in (*p, *q)]
    st.sample(p, dev[4] * 1.0, dev[5] * 1.0, q)
    del p, q
    # what the allocator would hand out again
    again = [torch.full(s, 0.5, device="cuda") for s in ((4, 40), (8, 33), (4, 40), (8, 33), (12,), (3,))]
    torch.cuda.synchronize()
    want = []
    for k, (a, n) in enumerate(((0, 1), (1, 2))):
        rows = slice(4 * a, 4 * a + 4 * n)
        w = plain.verify([4 * i for i in range(n + 1)], tokens[rows], None, host[k].cpu(), host[2 + k].cpu(), None, u[rows],
                         r[a: a + n], sp.heads[k].shape[0], 4, 4 * n)
        want += list(zip(w[0], w[1]))
    got = [x[:c] for x, c in zip(st.path.tolist(), st.n_path.tolist())]
    assert [(g, x) for g, x in zip(got, st.next.tolist())] == want
    assert all(bool((x == 0.5).all()) for x in again)


@pytest.mark.gpu
def test_a_captured_sampled_run_follows_its_buffers(lib):
    """Extend, sample and keep in one graph, replayed over new probabilities, against the same run eagerly."""
    from paper_2607_16074_amd import step
    from test_gpu_speculative import Speaker
    sp, gen = Speaker(lib, 14), torch.Generator().manual_seed(6)
    side = torch.cuda.Stream()
    parents = [-1, 0, 0, 1, 2]
    with torch.cuda.stream(side):
        steps = [step.SpeculativeStep(sp.model, [0, 1], [1, 2], 24, 5, parents, 16, lib.Context(side)) for _ in range(2)]
        x = torch.randn(20, 256, generator=gen).to(torch.bfloat16).cuda()
        for st in steps:
            st.prefill(x, [14, 0, 6])
        p, q = ([torch.zeros(n, h.shape[0], device="cuda") for n, h in zip((5, 10), sp.heads)] for _ in range(2))
        u, r = torch.zeros(15, device="cuda"), torch.zeros(3, device="cuda")

        def run(st):
            st.extend()
            st.sample(p, u, r, q)
            st.keep()

        past = steps[0].past.clone()
        run(steps[0])  # (everything is loaded before a capture)
        steps[0].past.copy_(past)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run(steps[0])
        for turn in range(12):
            for t in (*p, *q):
                t.copy_(torch.softmax(torch.randn(t.shape, generator=gen), 1))
            u.copy_(torch.rand(15, generator=gen))
            r.copy_(torch.rand(3, generator=gen))
            rows, tokens = torch.randn(15, 256, generator=gen), torch.randint(0, 33, (15,), generator=gen)
            for st in steps:
                st.embeds.copy_(rows)
                st.tokens.copy_(tokens)
            graph.replay()
            run(steps[1])
            side.synchronize()
            for name in ("past", "path", "n_path", "next"):
                assert torch.equal(getattr(steps[0], name), getattr(steps[1], name)), (turn, name)
            assert torch.equal(steps[0].cache.k, steps[1].cache.k) and torch.equal(steps[0].cache.v, steps[1].cache.v)
        assert steps[0].past.tolist()[0] >= 24 and steps[0].n_path.tolist()[0] == 0
