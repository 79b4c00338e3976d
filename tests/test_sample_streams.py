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
