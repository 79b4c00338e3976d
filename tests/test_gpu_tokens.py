"""Token heads: softmax cross entropy over a tenant's vocabulary with its gradients, and greedy decoding, against the
definitions in float64.

Bars.  A logit is a sum of d exact products accumulated in fp32 in some order: off by at most D = d 2^-24 sum|h w| of
it.  logp = z_t - m - log1p(rest): off by at most 2 max D and a few roundings of 1 + |logp|.  The gradient of a logit
is rounded to bf16 (half a step: 2^-8) and off by p 2 D before; dW and dh are sums of them against bf16 values in
fp32 (the additions' roundings stay below 2^-9 of the terms' magnitudes, 2^-24 for each of up to 2^15 additions) and
are rounded once more."""
import pytest
import torch  # before the library: both then share one HIP runtime

pytestmark = pytest.mark.gpu

BF = 2.0 ** -8


def draw(n, v, d, T, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    W = (torch.randn(v, d, generator=g, device="cuda") * (scale / d ** 0.5)).to(torch.bfloat16)
    rows = torch.randint(0, T, (n,), generator=g, device="cuda").to(torch.int32)
    targets = torch.randint(0, v, (n,), generator=g, device="cuda").to(torch.int32)
    return W, rows, targets


class Tenant:
    def __init__(self, lib, W, rows, targets, dh, f32=False):
        n, (v, d) = rows.numel(), W.shape
        self.W, self.rows, self.targets = W, rows, targets
        self.logp = torch.full((n + 4,), 9.0, device="cuda")
        self.loss = torch.full((2,), 9.0, device="cuda")
        self.dW = torch.full((v * d + 16,), 9.0, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
        self.dh = torch.full((n * d + 16,), 9.0, dtype=torch.bfloat16, device="cuda") if dh else None
        self.head = lib.TokenHead(W)
        self.io = lib.TokenIO(rows, targets, self.logp[:n], self.loss[:1], self.dW[: v * d].view(v, d),
                              self.dh[: n * d].view(n, d) if dh else None)

    def outputs(self):
        return [t for t in (self.logp, self.loss, self.dW, self.dh) if t is not None]

    def check(self, hidden, margin=None):
        n, (v, d) = self.rows.numel(), self.W.shape
        T = hidden.shape[0]
        r, t = self.rows.long(), self.targets.long()
        live = (r >= 0) & (r < T) & (t >= 0) & (t < v)
        h = torch.where(live[:, None], hidden[r.clamp(0, T - 1)].double(), 0.0)
        w = self.W.double()
        z = h @ w.T
        D = d * 2.0 ** -24 * (h.abs() @ w.abs().T).amax(1) if n else z.sum(1)
        lp = torch.log_softmax(z, 1) if n else z
        at = t.clamp(0, v - 1)[:, None]
        logp = torch.where(live, lp.gather(1, at)[:, 0], 0.0)
        off = (self.logp[:n].double() - logp).abs()
        bar = 2 * D + 16 * 2.0 ** -24 * (1 + logp.abs())
        assert bool((off <= bar).all()), float((off / bar).max())
        assert bool((self.logp[:n][~live] == 0).all())
        count = max(1, int(live.sum()))
        loss = -float(logp.sum()) / count
        lbar = float(bar.sum()) / count + n * 2.0 ** -24 * float(logp.abs().sum()) / count
        assert abs(float(self.loss[0]) - loss) <= lbar + 1e-30
        p = lp.exp()
        dz = p.scatter_add(1, at, torch.full_like(logp, -1.0)[:, None]) * (live.double() / count)[:, None]
        err = BF * dz.abs() + p * (2 * D * live.double() / count)[:, None]
        terms = err + 2.0 ** -9 * dz.abs()

        def within(got, ref, spread, what):
            o = (got.double() - ref).abs()
            b = BF * ref.abs() + (1 + BF) * spread + 1e-37
            assert bool((o <= b).all()), (what, float((o / b).max()))
            rel = float(o.pow(2).sum().sqrt() / ref.pow(2).sum().sqrt().clamp(min=1e-300))
            if margin and ref.numel() and count > 1:
                margin(what, rel, 1e-2)

        # (an fp32 dW misses the last rounding only: the same bar holds)
        within(self.dW[: v * d].view(v, d), dz.T @ h, terms.T @ h.abs(), "dW")
        if self.dh is not None:
            within(self.dh[: n * d].view(n, d), dz @ w, terms @ w.abs(), "dh")
            assert bool((self.dh[: n * d].view(n, d)[~live] == 0).all())
            assert bool((self.dh[n * d:] == 9.0).all())
        assert bool((self.dW[v * d:] == 9.0).all()) and bool((self.logp[n:] == 9.0).all()) and float(self.loss[1]) == 9.0


def step(lib, ctx, hidden, tenants):
    heads, ios = [t.head for t in tenants], [t.io for t in tenants]
    need = lib.jn_tokens_workspace_size(heads, ios)
    ws = torch.full((need + 64,), 0x7f, dtype=torch.uint8, device="cuda")  # a NaN pattern in bf16 and fp32
    lib.jn_tenant_tokens_fwd_bwd(ctx, hidden, heads, ios, ws[:need])
    torch.cuda.synchronize()
    assert bool((ws[need:] == 0x7f).all())


def feature(T, d, seed=5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(T, d, generator=g, device="cuda").to(torch.bfloat16)


CASES = [
    # n, vocab, d: one value, one row, odd and ragged ones, every tile shape and its edges
    (1, 1, 64), (1, 2, 64), (1, 7, 128), (2, 64, 64), (5, 63, 128), (7, 256, 768), (1, 1024, 768), (33, 65, 192),
    (95, 127, 64), (96, 128, 64), (97, 129, 64), (130, 1000, 320), (255, 2049, 128), (700, 513, 2048), (64, 5001, 2048),
    (513, 8193, 256), (2048, 4096, 512), (2300, 9001, 192), (20, 40001, 64),
    # few rows at every width the streaming kernels split differently, and one row more than they take
    (16, 700, 576), (17, 700, 1024), (32, 333, 1088), (64, 999, 2048), (65, 999, 2048), (33, 500, 2176), (32, 500, 4096),
    (16, 300, 4160), (16, 300, 8192), (17, 300, 8192),
]


@pytest.mark.parametrize("dh", [False, True], ids=["w", "wh"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_one_tenant(lib, case, dh, margin):
    n, v, d = case
    hidden = feature(max(3, 2 * n), d)
    t = Tenant(lib, *draw(n, v, d, hidden.shape[0], 11), dh)
    step(lib, lib.Context(), hidden, [t])
    t.check(hidden, margin if n * v > 1e5 else None)


def test_pieces_of_the_vocabulary(lib, margin):
    """More logits than a piece holds: the row gradients are summed over pieces, the last one ragged."""
    hidden = feature(3000, 64)
    a = Tenant(lib, *draw(2000, 300007, 64, 3000, 12), True)
    b = Tenant(lib, *draw(31, 70, 64, 3000, 13), True)  # fewer pieces than its neighbour
    c = Tenant(lib, *draw(12, 90001, 64, 3000, 14), False)
    step(lib, lib.Context(), hidden, [b, a, c])
    for t in (a, b, c):
        t.check(hidden, margin)


@pytest.mark.parametrize("case", [(5, 100001, 128), (32, 20003, 1024), (40, 35003, 2048), (33, 600011, 128),
                                  (16, 1601, 8192), (17, 3203, 4160), (1, 197003, 64)], ids=lambda c: "-".join(map(str, c)))
def test_row_gradients_of_few_rows_and_large_heads(lib, case):
    """Row gradients behind the streaming launches, at both of their row counts and every width."""
    n, v, d = case
    hidden = feature(n + 3, d)
    t = Tenant(lib, *draw(n, v, d, n + 3, 41), True)
    if n > 2:
        t.rows[1], t.targets[2] = -1, v
    step(lib, lib.Context(), hidden, [t])
    t.check(hidden)


def test_row_gradients_of_few_rows_and_many_heads(lib):
    hidden = feature(50, 192)
    ts = [Tenant(lib, *draw(n, v, 192, 50, 42 + k), dh)
          for k, (n, v, dh) in enumerate([(9, 40003, True), (0, 77, True), (31, 30001, False), (1, 1, True), (16, 9001, True)])]
    step(lib, lib.Context(), hidden, ts)
    for t in ts:
        t.check(hidden)


def test_few_rows_of_a_vocabulary_beyond_a_piece(lib):
    """33 rows whose logits in fp32 are more than the workspace may hold: not the streaming launches."""
    hidden = feature(40, 64)
    t = Tenant(lib, *draw(33, 4300001, 64, 40, 38), True)
    assert lib.jn_tokens_workspace_size([t.head], [t.io]) < 1 << 30
    step(lib, lib.Context(), hidden, [t])
    t.check(hidden)


@pytest.mark.parametrize("case", [(1, 300, 64), (7, 256, 768), (50, 777, 2176), (300, 1003, 320), (2048, 4096, 512)],
                         ids=lambda c: "-".join(map(str, c)))
def test_fp32_weight_gradients(lib, case):
    """The same products without the last rounding: rounded, they are the bf16 result bit for bit."""
    n, v, d = case
    hidden = feature(max(3, 2 * n), d)
    args = draw(n, v, d, hidden.shape[0], 15)
    for dh in (False, True):
        a, b = Tenant(lib, *args, dh), Tenant(lib, *args, dh, f32=True)
        empty = [Tenant(lib, *draw(0, 77, d, 4, 16), False, f32=x) for x in (False, True)]
        ctx = lib.Context()
        step(lib, ctx, hidden, [a, empty[0]])
        step(lib, ctx, hidden, [b, empty[1]])
        b.check(hidden)
        assert torch.equal(b.dW[: v * d].to(torch.bfloat16), a.dW[: v * d]) and torch.equal(a.logp, b.logp)
        for e in empty:
            e.check(hidden)
    with pytest.raises(lib.JNError):
        lib.jn_tokens_workspace_size([a.head, b.head], [a.io, b.io])


def test_tenants_of_unequal_sizes(lib):
    hidden = feature(900, 256)
    sizes = [(0, 130), (400, 2049), (1, 3), (0, 1), (77, 999), (257, 300), (0, 64)]
    ts = [Tenant(lib, *draw(n, v, 256, 900, 20 + k), k % 2 == 1) for k, (n, v) in enumerate(sizes)]
    step(lib, lib.Context(), hidden, ts)
    for t in ts:
        t.check(hidden)
    # nothing of a tenant depends on its neighbours but the order of equal sums
    for k in (1, 4, 5):
        alone = Tenant(lib, *draw(*sizes[k], 256, 900, 20 + k), k % 2 == 1)
        step(lib, lib.Context(), hidden, [alone])
        alone.check(hidden)
    only = [Tenant(lib, *draw(0, 130, 256, 900, 1), True)]
    step(lib, lib.Context(), hidden, only)
    assert float(only[0].loss[0]) == 0.0 and float(only[0].dW[: 130 * 256].abs().max()) == 0.0
    assert torch.equal(hidden, feature(900, 256))


def test_entries_without_a_target(lib):
    """Padded entries, rows outside the feature and tokens outside the vocabulary; what the feature holds at rows that
    have no target (NaN, infinities) reaches nothing."""
    n, v, d, T = 150, 700, 192, 300
    hidden = feature(T, d)
    W, rows, targets = draw(n, v, d, T - 20, 30)
    targets[::3] = -1
    targets[1] = v
    targets[4] = 2 ** 31 - 1
    rows[7], rows[10], rows[13] = -1, T, 2 ** 31 - 1
    rows[16] = -2 ** 31
    rows[0], rows[3] = T - 1, T - 2
    hidden[T - 1] = float("nan")
    hidden[T - 2] = float("inf")
    t = Tenant(lib, W, rows, targets, True)
    ctx = lib.Context()
    step(lib, ctx, hidden, [t])
    t.check(hidden)
    targets[:] = -1
    step(lib, ctx, hidden, [t])
    t.check(hidden)
    assert float(t.loss[0]) == 0.0 and float(t.dW[: v * d].abs().max()) == 0.0


def test_same_row_and_same_token_many_times(lib):
    hidden = feature(4, 128)
    W, rows, targets = draw(200, 333, 128, 4, 31)
    rows[:] = 2
    targets[:100] = 5
    t = Tenant(lib, W, rows, targets, True)
    step(lib, lib.Context(), hidden, [t])
    t.check(hidden)


def test_sure_rows_keep_their_small_losses(lib):
    """A row whose target holds all but 1e-6 of the probability: logp to a relative 1e-3 (the logits' own error), not
    the 6e-8 / 1e-6 that 1 - p would leave."""
    d, v = 256, 500
    hidden = feature(60, d)
    W, rows, targets = draw(60, v, d, 60, 32)
    rows[:] = torch.arange(60)
    hidden = (hidden.float() + 20.0 * W[targets.long()].float()).to(torch.bfloat16)
    t = Tenant(lib, W, rows, targets, True)
    step(lib, lib.Context(), hidden, [t])
    t.check(hidden)
    lp = torch.log_softmax(hidden.double() @ W.double().T, 1)[torch.arange(60), targets.long()]
    assert float(lp.max()) > -1e-4
    assert float(((t.logp[:60].double() - lp) / lp).abs().max()) < 1e-3


def test_equal_logits_and_large_logits(lib):
    hidden = torch.zeros(8, 64, dtype=torch.bfloat16, device="cuda")
    W, rows, targets = draw(8, 1001, 64, 8, 33)
    t = Tenant(lib, W, rows, targets, True)
    step(lib, lib.Context(), hidden, [t])
    t.check(hidden)
    hidden = feature(8, 64) * 300
    W, rows, targets = draw(8, 1001, 64, 8, 33, scale=300.0)
    t = Tenant(lib, W, rows, targets, True)
    step(lib, lib.Context(), hidden, [t])
    lp = torch.log_softmax(hidden[rows.long()].double() @ W.double().T, 1).gather(1, targets.long()[:, None])[:, 0]
    assert bool(torch.isfinite(t.logp[:8]).all())
    D = 64 * 2.0 ** -24 * (hidden[rows.long()].double().abs() @ W.double().abs().T).amax(1)
    assert bool(((t.logp[:8].double() - lp).abs() <= 2 * D + 2.0 ** -20 * (1 + lp.abs())).all())


def test_nan_of_a_target_is_not_hidden(lib):
    hidden = feature(6, 64)
    hidden[2, 3] = float("nan")
    W, rows, targets = draw(6, 100, 64, 6, 34)
    for i in range(6):
        rows[i] = i
    t = Tenant(lib, W, rows, targets, True)
    step(lib, lib.Context(), hidden, [t])
    bad = t.logp[:6].isnan()
    assert bad.tolist() == [False, False, True, False, False, False] and bool(t.loss[:1].isnan())


@pytest.mark.parametrize("n", [3, 40, 200])
def test_a_token_of_no_probability(lib, n):
    """Logits of -inf (a row of W of -inf where the feature is positive, else 0): as if the vocabulary held no such token."""
    d, v, ban = 128, 600, 0
    hidden = feature(n, d)
    hidden[:, 0] = 1.0
    W, rows, targets = draw(n, v, d, n, 36)
    targets.clamp_(min=1)
    W[ban] = 0.0
    W[ban, 0] = float("-inf")
    t = Tenant(lib, W, rows, targets, False)
    step(lib, lib.Context(), hidden, [t])
    assert bool((t.dW[:d] == 0).all())
    rest = Tenant(lib, W[1:].contiguous(), rows, targets - 1, False)
    rest.logp.copy_(t.logp)
    rest.loss.copy_(t.loss)
    rest.dW.copy_(t.dW[d:])
    rest.check(hidden)
    pick = Pick(lib, W, rows)
    decode(lib, lib.Context(), hidden, [pick])
    assert bool((pick.token[:n] != ban).all()) and bool(torch.isfinite(pick.logp[:n]).all())


@pytest.mark.parametrize("n,v,ban", [(5, 600, 0), (64, 600, 300), (200, 600, 1), (2000, 300007, 3), (2000, 300007, 300001)])
def test_a_token_of_no_probability_and_rows_without_a_target(lib, n, v, ban):
    """As above; an entry without a target meets the infinity with nothing and gets no gradient."""
    d = 64
    hidden = feature(n, d)
    hidden[:, 0] = 1.0
    W, rows, targets = draw(n, v, d, n, 37)
    targets[targets == ban] = 7
    rows[1], targets[2], rows[n - 1] = -1, -1, n
    W[ban] = 0.0
    W[ban, 0] = float("-inf")
    t = Tenant(lib, W, rows, targets, False)
    step(lib, lib.Context(), hidden, [t])
    assert bool((t.dW[ban * d: (ban + 1) * d] == 0).all())
    keep = torch.arange(v, device="cuda") != ban
    rest = Tenant(lib, W[keep], rows, torch.where(targets > ban, targets - 1, targets), False)
    rest.logp.copy_(t.logp)
    rest.loss.copy_(t.loss)
    rest.dW.copy_(torch.cat([t.dW[: v * d].view(v, d)[keep].reshape(-1), t.dW[v * d:]]))
    rest.check(hidden)


def test_same_bits_twice_and_on_another_stream(lib):
    hidden = feature(800, 256)
    a = Tenant(lib, *draw(500, 3001, 256, 800, 35), True)
    step(lib, lib.Context(), hidden, [a])
    first = [t.clone() for t in a.outputs()]
    stream = torch.cuda.Stream()
    ctx = lib.Context(stream)
    for t in a.outputs():
        t.fill_(9.0)
    torch.cuda.synchronize()
    step(lib, ctx, hidden, [a])
    assert all(torch.equal(x, y) for x, y in zip(first, a.outputs()))


def test_captured_and_replayed(lib):
    """Replays read rows, targets, feature and weights as they are then; two captured calls have workspaces of their own."""
    hidden = feature(600, 128)
    ts = [Tenant(lib, *draw(300, 2001, 128, 600, 36), True), Tenant(lib, *draw(40, 777, 128, 600, 37), False)]
    us = [Tenant(lib, *draw(90, 555, 128, 600, 38), True)]
    stream = torch.cuda.Stream()
    ctx = lib.Context(stream)
    runs = []
    for group in (ts, us):
        heads, ios = [t.head for t in group], [t.io for t in group]
        ws = torch.empty(lib.jn_tokens_workspace_size(heads, ios), dtype=torch.uint8, device="cuda")
        runs.append(lambda heads=heads, ios=ios, ws=ws: lib.jn_tenant_tokens_fwd_bwd(ctx, hidden, heads, ios, ws))
    torch.cuda.synchronize()
    graphs = []
    for run in runs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            run()
        graphs.append(graph)
    every = ts + us
    for k in range(3):
        hidden.copy_(torch.randn(600, 128, device="cuda"))
        for t in every:
            t.rows.copy_(torch.randint(-1, 600, t.rows.shape, device="cuda"))
            t.targets.copy_(torch.randint(-5, t.W.shape[0], t.targets.shape, device="cuda"))
            t.W.copy_(torch.randn(t.W.shape, device="cuda") / 12)
        torch.cuda.synchronize()
        for run in runs:
            run()
        torch.cuda.synchronize()
        want = [[o.clone() for o in t.outputs()] for t in every]
        for t in every:
            t.check(hidden)
            for o in t.outputs():
                o.fill_(9.0)
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for t, w in zip(every, want) for a, b in zip(t.outputs(), w))


# ------------------------------------------------------------------ decode ---


class Pick:
    def __init__(self, lib, W, rows):
        n = rows.numel()
        self.W, self.rows = W, rows
        self.token = torch.full((n + 4,), 77, dtype=torch.int32, device="cuda")
        self.logp = torch.full((n + 4,), 9.0, device="cuda")
        self.head = lib.TokenHead(W)
        self.io = lib.TokenPick(rows, self.token[:n], self.logp[:n])

    def check(self, hidden):
        n, (v, d) = self.rows.numel(), self.W.shape
        T = hidden.shape[0]
        r = self.rows.long()
        live = (r >= 0) & (r < T)
        h, w = hidden[r.clamp(0, T - 1)].double(), self.W.double()
        z = h @ w.T
        D = d * 2.0 ** -24 * (h.abs() @ w.abs().T).amax(1)
        token = self.token[:n].long()
        assert bool((token[~live] == -1).all()) and bool((self.logp[:n][~live] == 0).all())
        token, z, D, logp = token[live], z[live], D[live], self.logp[:n][live]
        assert bool(((token >= 0) & (token < v)).all())
        best = z.amax(1)
        got = z.gather(1, token[:, None])[:, 0]
        assert bool((got >= best - 2 * D).all())  # the largest, up to the logits' own error
        want = torch.log_softmax(z, 1).amax(1)
        assert bool(((logp.double() - want).abs() <= 2 * D + 16 * 2.0 ** -24 * (1 + want.abs())).all())
        assert bool((self.token[n:] == 77).all()) and bool((self.logp[n:] == 9.0).all())


def decode(lib, ctx, hidden, picks):
    heads, ios = [p.head for p in picks], [p.io for p in picks]
    need = lib.jn_tokens_decode_workspace_size(heads, ios)
    ws = torch.full((need + 64,), 0x7f, dtype=torch.uint8, device="cuda")
    lib.jn_tenant_tokens_decode(ctx, hidden, heads, ios, ws[:need])
    torch.cuda.synchronize()
    assert bool((ws[need:] == 0x7f).all())


@pytest.mark.parametrize("case", CASES + [(1, 100003, 128), (300, 20001, 768)], ids=lambda c: "-".join(map(str, c)))
def test_decode(lib, case):
    n, v, d = case
    hidden = feature(max(3, 2 * n), d, seed=6)
    W, rows, _ = draw(n, v, d, hidden.shape[0], 40)
    if n > 3:
        rows[1], rows[2] = -1, hidden.shape[0]
    p = Pick(lib, W, rows)
    decode(lib, lib.Context(), hidden, [p])
    p.check(hidden)


def test_decode_tenants(lib):
    hidden = feature(64, 512)
    picks = [Pick(lib, *draw(n, v, 512, 64, 50 + k)[:2]) for k, (n, v) in enumerate([(3, 999), (0, 5), (64, 1), (1, 20001), (0, 7)])]
    decode(lib, lib.Context(), hidden, picks)
    for p in picks:
        p.check(hidden)
    shared = [Pick(lib, picks[3].W, picks[2].rows[:9].clone()), Pick(lib, picks[3].W, picks[2].rows[9:].clone())]
    decode(lib, lib.Context(), hidden, shared)
    for p in shared:
        p.check(hidden)


def test_decode_ties_take_the_lowest(lib):
    hidden = feature(9, 64)
    W, rows, _ = draw(9, 1500, 64, 9, 60)
    rows[:] = torch.arange(9)
    copies = [3, 17, 130, 131, 700, 1499]
    for i in range(9):
        # row i's own best direction, at every place from the i-th on
        W[copies[i % 6:]] = (hidden[i] * 4).to(torch.bfloat16) if i < 6 else W[copies[i % 6:]]
        p = Pick(lib, W.clone(), rows[i: i + 1].clone())
        decode(lib, lib.Context(), hidden, [p])
        if i < 6:
            assert int(p.token[0]) == copies[i]
    zero = torch.zeros(9, 64, dtype=torch.bfloat16, device="cuda")
    p = Pick(lib, W, rows)
    decode(lib, lib.Context(), zero, [p])
    assert bool((p.token[:9] == 0).all())


def test_decode_of_nan_stays_in_the_vocabulary(lib):
    hidden = feature(5, 64)
    hidden[1] = float("nan")
    W, rows, _ = draw(5, 301, 64, 5, 61)
    for i in range(5):
        rows[i] = i
    p = Pick(lib, W, rows)
    decode(lib, lib.Context(), hidden, [p])
    assert 0 <= int(p.token[1]) < 301 and p.logp[:5].isnan().tolist() == [False, True, False, False, False]


def test_decode_captured_and_replayed(lib):
    hidden = feature(100, 256)
    picks = [Pick(lib, *draw(7, 4001, 256, 100, 62)[:2]), Pick(lib, *draw(20, 800, 256, 100, 63)[:2])]
    heads, ios = [p.head for p in picks], [p.io for p in picks]
    ws = torch.empty(lib.jn_tokens_decode_workspace_size(heads, ios), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    ctx = lib.Context(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        lib.jn_tenant_tokens_decode(ctx, hidden, heads, ios, ws)
    for _ in range(3):
        hidden.copy_(torch.randn(100, 256, device="cuda"))
        for p in picks:
            p.rows.copy_(torch.randint(-1, 100, p.rows.shape, device="cuda"))
            p.token[:-4].fill_(5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for p in picks:
            p.check(hidden)


# --------------------------------------------------------------- refusals ---


def test_refusals(lib):
    abi = lib._abi
    hidden = feature(10, 64)
    t = Tenant(lib, *draw(5, 50, 64, 10, 70), True)
    ctx = lib.Context()
    ws = torch.empty(lib.jn_tokens_workspace_size([t.head], [t.io]), dtype=torch.uint8, device="cuda")

    def refused(code, change, small=False, h=hidden):
        head, io = type(t.head.struct).from_buffer_copy(t.head.struct), type(t.io.struct).from_buffer_copy(t.io.struct)
        d = change(head, io) or 64
        st = lib._lib.jn_tenant_tokens_fwd_bwd(ctx.handle, h.data_ptr() if h is not None else None, 10, d, head, io, 1,
                                               ws.data_ptr(), ws.numel() - (1 if small else 0))
        assert st == code, (st, lib._lib.jn_last_error(ctx.handle))

    def put(where, name, value):
        return lambda head, io: setattr(head if where == "head" else io, name, value)

    refused(abi.JN_ENOSPACE, lambda a, b: None, small=True)
    refused(abi.JN_EUNSUPPORTED, lambda a, b: 96)
    refused(abi.JN_EUNSUPPORTED, lambda a, b: 16384)
    refused(abi.JN_ESHAPE, put("head", "vocab", 0))
    refused(abi.JN_ESHAPE, put("head", "vocab", (1 << 24) + 1))
    refused(abi.JN_EINVAL, put("head", "W", None))
    refused(abi.JN_EUNSUPPORTED, put("head", "W", t.W.data_ptr() + 2))
    refused(abi.JN_ESHAPE, put("io", "n", -1))
    refused(abi.JN_ESHAPE, put("io", "n", (1 << 20) + 1))
    for name in ("rows", "targets", "logp", "loss", "dW"):
        refused(abi.JN_EINVAL, put("io", name, None))
    refused(abi.JN_EUNSUPPORTED, put("io", "dh", t.dh.data_ptr() + 2))
    refused(abi.JN_EUNSUPPORTED, put("io", "rows", t.rows.data_ptr() + 2))
    refused(abi.JN_EINVAL, lambda a, b: None, h=None)
    torch.cuda.synchronize()
    assert all(bool((o == 9.0).all()) for o in t.outputs())
    with pytest.raises(TypeError):
        lib.jn_tenant_tokens_fwd_bwd(ctx, feature(10, 128), [t.head], [t.io], ws)
    with pytest.raises(TypeError):
        lib.TokenIO(t.rows.long(), t.targets, t.logp[:5], t.loss[:1], t.io.dW)
    with pytest.raises(ValueError):
        lib.jn_tokens_workspace_size([t.head], [])
