"""The calls over a paged cache on the GPU: appending, attention, keeping a branch, against 64-bit definitions."""
import itertools

import pytest
import torch

import kv_plain as plain

pytestmark = pytest.mark.gpu
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def make(seed, kv, hd, page, past, new, mask="chain", layers=1, spare=3, pad=2, max_new=None, bad=(), parents=None):
    """A cache, and a batch of sequences with these lengths, on the CPU; bad: (sequence, page index, id) of bad pages."""
    gen = torch.Generator().manual_seed(seed)
    per = max(1, max((p + n + page - 1) // page for p, n in zip(past, new)))
    n = len(past) * per + spare
    pages = torch.randperm(n, generator=gen)[: len(past) * per].view(len(past), per).to(I32)
    for s, i, g in bad:
        pages[s, i] = g
    cu = torch.tensor([0] + list(itertools.accumulate(new)), dtype=I32)
    b = {"pages": pages, "past": torch.tensor(past, dtype=I32), "cu": cu, "rows": int(cu[-1]) + pad,
         "max_new": max_new or max(1, max(new)), "page": page, "whole": mask == "whole"}
    if mask == "tree":
        j = torch.cat([torch.arange(m) for m in new] + [torch.zeros(pad, dtype=torch.long)])
        u = torch.rand(b["rows"], generator=gen)
        up = torch.where(j > 0, (u * u * j).long().clamp(max=(j - 1).clamp(min=0)), -1)
        b["parents"] = (up if parents is None else torch.tensor(parents + [-1] * pad)).to(I32)
    k, v = (torch.randn(layers, n, kv, page, hd, generator=gen).to(BF16) for _ in range(2))
    return b, k, v, gen


def batch(lib, b, dev="cuda"):
    up = b["parents"].to(dev) if b.get("parents") is not None else None
    return lib.KVBatch(b["pages"].to(dev), b["past"].to(dev), b["cu"].to(dev), b["rows"], b["max_new"], up, b["whole"])


def attend(lib, b, k, v, q, heads, scale=0.0, out=None, ctx=None, layer=0):
    """out on the CPU, which starts as NaN."""
    ctx = ctx or lib.Context()
    cache, bt = lib.KVCache(k.cuda(), v.cuda()), batch(lib, b)
    hd = k.shape[-1]
    out = torch.full((b["rows"], heads * hd), float("nan"), dtype=BF16, device="cuda") if out is None else out
    ws = torch.empty(lib.jn_kv_attention_workspace_size(cache, bt, heads), dtype=torch.uint8, device="cuda")
    ws.fill_(0xff)  # NaN wherever something unwritten is read
    lib.jn_kv_attention(ctx, cache, layer, bt, heads, q.cuda(), out, ws, scale)
    torch.cuda.synchronize()
    return out.cpu()


def check_rows(got, want, tol, margin=None, what="attention"):
    """Rows that no sequence has are untouched (NaN here), the others within the tolerance."""
    idle = torch.isnan(want)
    assert torch.equal(torch.isnan(got), idle)
    err = (got.double() - want).abs()[~idle]
    t = tol[~idle]
    if margin is not None and err.numel():
        margin(what, float((err / t.clamp(min=1e-30)).max()), 1.0)
    assert bool((err <= t).all()), f"worst {float((err - t).max())}"


def attention_case(lib, margin, b, k, v, gen, heads, scale=0.0, spread=1.5):
    q = (spread * torch.randn(b["rows"], heads * k.shape[-1], generator=gen)).to(BF16)
    got = attend(lib, b, k, v, q, heads, scale)
    want, tol = plain.attention(b, k[0], v[0], q, heads, torch.full(got.shape, float("nan")), scale)
    check_rows(got, want, tol, margin)


SHAPES = [(8, 8, 256), (8, 1, 256), (16, 2, 128), (4, 4, 128), (12, 4, 64), (6, 1, 64), (4, 4, 32), (16, 1, 32)]


@pytest.mark.parametrize("heads,kv,hd", SHAPES)
@pytest.mark.parametrize("mask", ["chain", "tree", "whole"])
def test_attention_of_uneven_sequences(lib, margin, heads, kv, hd, mask):
    """No rows, one row, lengths around pages and tiles, an empty cache."""
    b, k, v, gen = make(hd + heads, kv, hd, 16, [0, 5, 63, 64, 130, 300, 1], [3, 1, 7, 0, 17, 2, 1], mask)
    attention_case(lib, margin, b, k, v, gen, heads)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("past,new", [(0, 1), (1, 1), (255, 1), (256, 3), (1000, 5), (2500, 1)])
def test_attention_over_pages(lib, margin, page, past, new):
    b, k, v, gen = make(page + past, 2, 64, page, [past, past // 2], [new, new], "chain")
    attention_case(lib, margin, b, k, v, gen, 8)


@pytest.mark.parametrize("heads,kv,hd", [(8, 1, 256), (16, 2, 128), (4, 4, 64), (2, 2, 32)])
@pytest.mark.parametrize("past,new", [(0, 200), (37, 131), (300, 64), (5, 33)])
@pytest.mark.parametrize("mask", ["chain", "whole"])
def test_attention_of_pieces(lib, margin, heads, kv, hd, past, new, mask):
    """Pieces of a prompt: more query rows than a tile."""
    b, k, v, gen = make(past + new, kv, hd, 32, [past, 3], [new, new // 2], mask)
    attention_case(lib, margin, b, k, v, gen, heads)


@pytest.mark.parametrize("heads,kv,hd", [(8, 1, 256), (16, 2, 128), (8, 8, 32)])
@pytest.mark.parametrize("new", [2, 61, 64, 65, 200, 256])
def test_attention_of_trees(lib, margin, heads, kv, hd, new):
    b, k, v, gen = make(new, kv, hd, 64, [90, 0], [new, max(1, new // 3)], "tree")
    attention_case(lib, margin, b, k, v, gen, heads)


def test_parents_that_are_none(lib, margin):
    """Later rows, the row itself, numbers far outside: the row hangs on the cached rows."""
    up = [-1, 0, 1, 3, 9, -5, 2 ** 31 - 1, 5, -2 ** 31, 3]
    b, k, v, gen = make(1, 2, 64, 16, [20], [10], "tree", parents=up)
    attention_case(lib, margin, b, k, v, gen, 4)
    b, k, v, gen = make(1, 2, 64, 16, [0], [10], "tree", parents=up)
    attention_case(lib, margin, b, k, v, gen, 4)


def test_bad_pages_and_rows_that_see_nothing(lib, margin):
    """Pages outside the cache are not seen; a row without any key is zeros."""
    bad = [(0, 1, -1), (0, 3, 10 ** 9), (1, 0, -7), (2, 0, 2 ** 31 - 1), (2, 1, -2 ** 31)]
    b, k, v, gen = make(3, 2, 64, 16, [70, 0, 20], [3, 2, 1], bad=bad)
    assert not any(plain.place(b, k.shape[1], 1, t) for t in range(2))
    attention_case(lib, margin, b, k, v, gen, 4)


def test_lengths_outside_their_range(lib, margin):
    """cu_rows behind the call's rows, more rows than max_new, past beyond the pages or negative."""
    b, k, v, gen = make(4, 1, 64, 16, [40, 10, 0], [5, 6, 4], pad=0)
    b["past"] = torch.tensor([10 ** 9, -3, 2 ** 31 - 1], dtype=I32)
    b["cu"] = torch.tensor([-4, 5, 11, 2 ** 31 - 1], dtype=I32)
    b["max_new"] = 4
    attention_case(lib, margin, b, k, v, gen, 4)
    b["cu"] = torch.tensor([9, 5, 5, 11], dtype=I32)  # a sequence of less than no rows
    attention_case(lib, margin, b, k, v, gen, 4)


@pytest.mark.parametrize("heads,kv,hd", [(8, 1, 256), (16, 2, 128), (4, 4, 64), (4, 2, 32)])
@pytest.mark.parametrize("new", [1, 9, 70])
def test_what_a_row_does_not_see_leaves_it_alone(lib, margin, heads, kv, hd, new):
    """NaN and infinities behind the sequences' ends and in other branches of a tree."""
    b, k, v, gen = make(5, kv, hd, 32, [45, 0], [new, new], "tree", parents=([-1] + [0] * (new - 1)) * 2)
    seen = torch.zeros(k.shape[1], 32, dtype=torch.bool)
    for s, (past, row0, n) in enumerate(plain.sequences(b)):
        for t in range(past + n):
            seen[plain.place(b, k.shape[1], s, t)] = True
    poison = torch.tensor([float("nan"), float("inf"), -float("inf")])
    hole = (~seen).nonzero()
    fill = poison[torch.randint(0, 3, (len(hole), kv, hd), generator=gen)].to(BF16)
    k[0][hole[:, 0], :, hole[:, 1]] = fill
    v[0][hole[:, 0], :, hole[:, 1]] = fill.flip(0)
    q = torch.randn(b["rows"], heads * hd, generator=gen).to(BF16)
    clean, _ = plain.attention(b, k[0], v[0], q, heads, torch.full((b["rows"], heads * hd), float("nan")))
    got = attend(lib, b, k, v, q, heads)
    want, tol = plain.attention(b, k[0], v[0], q, heads, torch.full(got.shape, float("nan")))
    check_rows(got, want, tol, margin)
    if new < 3:
        return
    # the last row of each tree: it alone sees itself
    for s, (past, row0, n) in enumerate(plain.sequences(b)):
        g, r = plain.place(b, k.shape[1], s, past + n - 1)
        v[0][g, :, r] = torch.tensor([float("nan"), float("inf")])[s]
        k[0][g, :, r] = 0.5
    got = attend(lib, b, k, v, q, heads).double()
    want, tol = plain.attention(b, k[0], v[0], q, heads, torch.full(got.shape, float("nan")))
    for s, (past, row0, n) in enumerate(plain.sequences(b)):
        others = slice(row0, row0 + n - 1)
        assert bool(((got - want).abs()[others] <= tol[others]).all())
        last = got[row0 + n - 1]
        assert bool(torch.isnan(last).all() if s == 0 else (last == float("inf")).all())


@pytest.mark.parametrize("heads,kv,new", [(4, 1, 2), (4, 1, 40)])
def test_values_that_all_rows_see_stay_what_they_are(lib, heads, kv, new):
    """An infinity among the cached rows reaches every row, also beside a page that is none."""
    b, k, v, gen = make(12, kv, 64, 16, [100], [new], bad=[(0, 2, -1)], pad=0)
    g, r = plain.place(b, k.shape[1], 0, 50)  # (the bad page holds places 32 .. 47)
    v[0][g, :, r, 3], v[0][g, :, r, 40] = float("inf"), -float("inf")
    q = torch.randn(b["rows"], heads * 64, generator=gen).to(BF16)
    got = attend(lib, b, k, v, q, heads).double().view(new, heads, 64)
    want, tol = plain.attention(b, k[0], v[0], q, heads, torch.full((new, heads * 64), float("nan")))
    want, tol = want.view(got.shape), tol.view(got.shape)
    assert bool((got[..., 3] == float("inf")).all() and (got[..., 40] == -float("inf")).all())
    rest = [i for i in range(64) if i not in (3, 40)]
    assert bool(((got - want).abs()[..., rest] <= tol[..., rest]).all())


def test_infinite_keys(lib):
    """A key of +inf where the query is positive: NaN, as a softmax of an infinite score is; a key of -inf is nothing."""
    b, k, v, gen = make(6, 1, 64, 16, [40], [1], pad=0)
    q = torch.ones(1, 64, dtype=BF16)
    g, r = plain.place(b, k.shape[1], 0, 17)
    k[0][g, 0, r] = -float("inf")
    got = attend(lib, b, k, v, q, 1).double()
    g2 = b["pages"].clone()
    want, tol = plain.attention(b, k[0], v[0], q, 1, torch.full((1, 64), float("nan")))
    assert bool(torch.isfinite(want).all()) and bool(((got - want).abs() <= tol.nan_to_num(2.0 ** -6)).all())
    k[0][g, 0, r] = float("inf")
    assert bool(torch.isnan(attend(lib, b, k, v, q, 1)).all())
    assert torch.equal(g2, b["pages"])


@pytest.mark.parametrize("scale", [0.01, 1.0, 30.0])
def test_scales_and_sure_rows(lib, margin, scale):
    """Scores far apart, of either sign, where the running maximum moves late."""
    b, k, v, gen = make(7, 2, 128, 64, [700, 3], [2, 5])
    order = torch.linspace(0.2, 3.0, k.shape[3])[None, None, None, :, None]
    attention_case(lib, margin, b, (k * order).to(BF16), v, gen, 8, scale, 0.5)


def test_equal_scores_give_the_mean(lib):
    b, k, v, gen = make(8, 2, 64, 16, [511, 4096], [1, 1])
    k.fill_(1.0)
    v.fill_(0.5)
    q = torch.randn(b["rows"], 4 * 64, generator=gen).to(BF16)
    got = attend(lib, b, k, v, q, 4)[:2]
    assert bool((got == 0.5).all())


def test_sequences_that_share_pages(lib, margin):
    """A common prompt is read by all of its sequences from the same pages."""
    b, k, v, gen = make(13, 2, 64, 32, [64, 64, 90], [5, 1, 40])
    b["pages"][1, :2] = b["pages"][0, :2]
    b["pages"][2, :2] = b["pages"][0, :2]
    attention_case(lib, margin, b, k, v, gen, 8)


def test_many_sequences(lib, margin):
    """More than a search's 64, uneven, some of them empty."""
    past, new = [(37 * i) % 200 for i in range(150)], [(i % 4 != 1) * (1 + i % 3) for i in range(150)]
    b, k, v, gen = make(14, 1, 32, 16, past, new)
    attention_case(lib, margin, b, k, v, gen, 4)
    b, k, v, gen = make(15, 1, 32, 16, past[:80], [i % 40 for i in range(80)])
    attention_case(lib, margin, b, k, v, gen, 4)


@pytest.mark.parametrize("heads,kv", [(2, 2), (6, 2), (5, 1), (14, 2), (32, 1)])
@pytest.mark.parametrize("cut", [0, 9])
def test_long_pieces_of_odd_head_groups(lib, margin, heads, kv, cut):
    """Chains of many row tiles, with `cut` pages too few for the last rows: the tiles of a run are counted by a formula."""
    b, k, v, gen = make(heads, kv, 32, 16, [700, 61, 0, 5], [601, 1, 333, 1240], "chain")
    b["pages"] = b["pages"][:, : b["pages"].shape[1] - cut].contiguous()
    attention_case(lib, margin, b, k, v, gen, heads)


def test_sizes_far_beyond_what_a_batch_holds(lib, margin):
    """A program's buffers and max_new are made for its largest call."""
    b, k, v, gen = make(3, 2, 32, 16, [s % 40 for s in range(300)], [1 + s % 3 for s in range(300)], "chain", pad=70000,
                        max_new=70000)
    attention_case(lib, margin, b, k, v, gen, 16)


def test_calls_of_nothing(lib):
    b, k, v, gen = make(16, 2, 64, 16, [5], [2], pad=0)
    ctx, cache = lib.Context(), lib.KVCache(k.cuda(), v.cuda())
    i = lambda *n: torch.zeros(n, dtype=I32, device="cuda")  # noqa: E731
    for bt in (lib.KVBatch(i(0, 3), i(0), i(1), 4, 1), lib.KVBatch(i(2, 3), i(2), i(3), 0, 1)):
        rows = bt.struct.rows
        x, q, out = (torch.ones(rows, w, dtype=BF16, device="cuda") for w in (512, 256, 256))
        assert lib.jn_kv_attention_workspace_size(cache, bt, 4) == 0
        lib.jn_kv_append(ctx, cache, 0, bt, lib.QKNormRope(4, 2, 64, theta=1e4), x, None, q)
        lib.jn_kv_attention(ctx, cache, 0, bt, 4, q, out, None)
        lib.jn_kv_keep(ctx, cache, bt, i(bt.struct.n_seqs, 2), i(bt.struct.n_seqs))
        torch.cuda.synchronize()
        assert bool((out == 1).all() and (q == 1).all())
    # a batch whose sequences have no rows
    bt = lib.KVBatch(i(2, 3), i(2), i(3), 4, 2)
    q, out = (torch.ones(4, 256, dtype=BF16, device="cuda") for _ in range(2))
    ws = torch.empty(lib.jn_kv_attention_workspace_size(cache, bt, 4), dtype=torch.uint8, device="cuda").fill_(0xff)
    lib.jn_kv_attention(ctx, cache, 0, bt, 4, q, out, ws)
    torch.cuda.synchronize()
    assert bool((out == 1).all()) and torch.equal(cache.k.cpu(), k)


def test_the_launch_trace_names_the_calls(lib):
    b, k, v, gen = make(17, 2, 64, 16, [5], [2], pad=0)
    ctx, cache, bt = lib.Context(), lib.KVCache(k.cuda(), v.cuda()), batch(lib, b)
    x = torch.randn(2, 8 * 64, generator=gen).to(BF16).cuda()
    q, out = (torch.zeros(2, 4 * 64, dtype=BF16, device="cuda") for _ in range(2))
    ws = torch.empty(lib.jn_kv_attention_workspace_size(cache, bt, 4), dtype=torch.uint8, device="cuda")
    ctx.set_trace(True)
    lib.jn_kv_append(ctx, cache, 0, bt, lib.QKNormRope(4, 2, 64, theta=1e4), x, None, q)
    lib.jn_kv_attention(ctx, cache, 0, bt, 4, q, out, ws)
    lib.jn_kv_keep(ctx, cache, bt, torch.zeros(1, 1, dtype=I32, device="cuda"), torch.ones(1, dtype=I32, device="cuda"))
    got = ctx.trace_read()
    assert [(e[0], e[1], e[2]) for e in got] == [("kv_append", 2, 512), ("kv_attention", 2, 256), ("kv_keep", 1, 128)]
    assert all(0 < e[4] < 1000 for e in got)


def test_strided_rows_cache_and_layers(lib, margin):
    """Rows inside wider ones, layers of a page together, the second layer."""
    heads, kv, hd = 4, 2, 64
    b, k, v, gen = make(9, kv, hd, 16, [50, 7], [3, 2], layers=3)
    wide = torch.randn(b["rows"], heads * hd + 40, generator=gen).to(BF16)
    q = wide[:, 8: 8 + heads * hd]
    big = torch.full((b["rows"], heads * hd + 24), float("nan"), dtype=BF16, device="cuda")
    out = big[:, 16: 16 + heads * hd]
    kk, vv = (t.transpose(0, 1).contiguous().cuda().transpose(0, 1) for t in (k, v))
    assert not kk.is_contiguous()
    cache, bt = lib.KVCache(kk, vv), batch(lib, b)
    ws = torch.empty(lib.jn_kv_attention_workspace_size(cache, bt, heads), dtype=torch.uint8, device="cuda")
    lib.jn_kv_attention(lib.Context(), cache, 1, bt, heads, wide.cuda()[:, 8: 8 + heads * hd], out, ws)
    want, tol = plain.attention(b, k[1], v[1], q, heads, torch.full((b["rows"], heads * hd), float("nan")))
    check_rows(out.cpu(), want, tol, margin)
    assert bool(torch.isnan(big[:, :16]).all() and torch.isnan(big[:, 16 + heads * hd:]).all())


def test_offsets_beyond_32_bits(lib, margin):
    """Pages more than 2^31 elements apart: reads, writes and moves."""
    heads, kv, hd, page, far = 4, 2, 64, 16, (1 << 30) + 8 * 123
    b, k, v, gen = make(10, kv, hd, page, [20], [9], spare=3, pad=0)
    n = k.shape[1]
    assert n * far > 1 << 32
    pool = torch.empty(2, (n - 1) * far + kv * page * hd, dtype=BF16, device="cuda")
    view = [torch.as_strided(pool[i], (1, n, kv, page, hd), (0, far, page * hd, hd, 1)) for i in range(2)]
    view[0].copy_(k)
    view[1].copy_(v)
    cache, bt = lib.KVCache(*view), batch(lib, b)
    q = torch.randn(b["rows"], heads * hd, generator=gen).to(BF16)
    out = torch.full((b["rows"], heads * hd), float("nan"), dtype=BF16, device="cuda")
    ws = torch.empty(lib.jn_kv_attention_workspace_size(cache, bt, heads), dtype=torch.uint8, device="cuda")
    ctx = lib.Context()
    lib.jn_kv_attention(ctx, cache, 0, bt, heads, q.cuda(), out, ws)
    want, tol = plain.attention(b, k[0], v[0], q, heads, torch.full(out.shape, float("nan")))
    check_rows(out.cpu(), want, tol, margin)
    path, count = torch.tensor([[0, 2, 5, 8]], dtype=I32), torch.tensor([4], dtype=I32)
    lib.jn_kv_keep(ctx, cache, bt, path.cuda(), count.cuda())
    wk, wv, _ = plain.keep(b, k, v, path, count)
    assert torch.equal(view[0].cpu(), wk) and torch.equal(view[1].cpu(), wv)
    x = torch.randn(b["rows"], 2 * kv * hd, generator=gen).to(BF16)
    lib.jn_kv_append(ctx, cache, 0, bt, lib.QKNormRope(0, kv, hd), x.cuda(), None, None)
    wk, wv, _, _ = plain.append(b, wk[0], wv[0], x, 0, kv, None, None, 1e-6, 0.0, None, None, x[:, :0])
    assert torch.equal(view[0].cpu()[0].double(), wk) and torch.equal(view[1].cpu()[0].double(), wv)


def test_attention_repeats_its_bits_and_follows_its_inputs_in_a_graph(lib, margin):
    """Replays read lengths, tables, cache and queries as they are then; two graphs share one workspace."""
    heads, kv, hd = 8, 2, 128
    b, k, v, gen = make(11, kv, hd, 32, [900, 40, 3], [3, 1, 6], "tree")
    side = torch.cuda.Stream()
    ctx = lib.Context(side)
    cache, bt = lib.KVCache(k.cuda(), v.cuda()), batch(lib, b)
    qs = [torch.randn(b["rows"], heads * hd, generator=gen).to(BF16) for _ in range(2)]
    q = [t.cuda() for t in qs]
    out = [torch.full((b["rows"], heads * hd), float("nan"), dtype=BF16, device="cuda") for _ in range(2)]
    ws = torch.empty(lib.jn_kv_attention_workspace_size(cache, bt, heads), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            lib.jn_kv_attention(ctx, cache, 0, bt, heads, q[i], out[i], ws)
        graphs.append(g)
    for past, cu in (([900, 40, 3], [0, 3, 4, 10]), ([17, 0, 64], [0, 6, 9, 10]), ([905, 100, 50], [0, 0, 5, 10])):
        b["past"], b["cu"] = torch.tensor(past, dtype=I32), torch.tensor(cu, dtype=I32)
        bt.past.copy_(b["past"])
        bt.cu_rows.copy_(b["cu"])
        for o in out:
            o.fill_(float("nan"))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graphs[0].replay()
            graphs[1].replay()
        torch.cuda.synchronize()
        for i in range(2):
            want, tol = plain.attention(b, k[0], v[0], qs[i], heads, torch.full(out[i].shape, float("nan")))
            check_rows(out[i].cpu(), want, tol, margin)
            again = attend(lib, b, k, v, qs[i], heads)
            assert torch.equal(again.view(torch.int16), out[i].cpu().view(torch.int16))


# ------------------------------------------------------------------ append ---


def append_case(lib, margin, b, k, v, gen, heads, norm, theta, sections=(), interleaved=False, inplace=False, axes=1):
    kv, hd = k.shape[2], k.shape[-1]
    x = (torch.randn(b["rows"], (heads + 2 * kv) * hd, generator=gen) * 2).to(BF16)
    gq, gk = ((1 + 0.3 * torch.randn(hd, generator=gen)).to(BF16) if norm else None for _ in range(2))
    pos = torch.randint(-50, 10 ** 6, (b["rows"], axes), generator=gen).to(I32) if axes > 1 else None
    if axes == 1:
        axis = [0] * (hd // 2)
    elif interleaved:
        axis = [i % axes if i // axes < sections[i % axes] else 0 for i in range(hd // 2)]
    else:
        axis = [a for a in range(axes) for _ in range(sections[a])]
    dev = lambda t: t.cuda() if t is not None else None  # noqa: E731
    qk = lib.QKNormRope(heads, kv, hd, 1e-6, dev(gq), dev(gk), theta, sections, interleaved)
    cache, bt, xd = lib.KVCache(k.cuda(), v.cuda()), batch(lib, b), x.cuda()
    qd = xd if inplace else torch.full((b["rows"], heads * hd + 16), 7.0, dtype=BF16, device="cuda")
    layer = k.shape[0] - 1
    lib.jn_kv_append(lib.Context(), cache, layer, bt, qk, xd, dev(pos), qd)
    torch.cuda.synchronize()
    q0 = x if inplace else torch.full(qd.shape, 7.0)
    wk, wv, wq, hit = plain.append(b, k[layer], v[layer], x, heads, kv, gq, gk, 1e-6, theta, pos, axis, q0)
    # half a step of bf16; sums of hd squares, products and turns of 32 bits; an angle's rounding to 2^-24 turns
    size = x.abs().max().double() * (1.0 + (gq.abs().max().double() if norm else 0.0)) * (4.0 if norm else 1.0)
    room = lambda w: 2.0 ** -8 * w.abs() + 2.0 ** -19 * size  # noqa: E731
    gotk, gotv = cache.k[layer].cpu(), cache.v[layer].cpu()
    assert torch.equal(gotv.double(), wv)
    assert bool(((gotk.double() - wk).abs() <= room(wk)).all())
    assert bool(((qd.cpu().double() - wq).abs() <= room(wq)).all())
    # what is not a new row's is as it was, bit for bit
    same = ~hit
    assert torch.equal(gotk.transpose(1, 2)[same], k[layer].transpose(1, 2)[same])
    idle = torch.ones(b["rows"], dtype=torch.bool)
    for _, row0, n in plain.sequences(b):
        idle[row0: row0 + n] = False
    assert torch.equal(qd.cpu().double()[idle], q0.double()[idle])
    assert torch.equal(qd.cpu().double()[:, heads * hd:], q0.double()[:, heads * hd:])
    for i in range(layer):
        assert torch.equal(cache.k[i].cpu(), k[i]) and torch.equal(cache.v[i].cpu(), v[i])


@pytest.mark.parametrize("heads,kv,hd", [(8, 1, 256), (16, 2, 128), (3, 3, 96), (4, 4, 32), (2, 1, 16), (5, 1, 80)])
@pytest.mark.parametrize("norm,theta", [(True, 1e4), (False, 1e6), (True, 0.0), (False, 0.0)])
@pytest.mark.parametrize("mask", ["chain", "tree"])
def test_append(lib, margin, heads, kv, hd, norm, theta, mask):
    b, k, v, gen = make(hd, kv, hd, 16, [0, 30, 15, 100], [5, 1, 0, 40], mask, layers=2)
    append_case(lib, margin, b, k, v, gen, heads, norm, theta)


@pytest.mark.parametrize("interleaved", [False, True])
def test_append_with_axes_in_place(lib, margin, interleaved):
    b, k, v, gen = make(21, 2, 64, 64, [3, 0], [70, 1])
    append_case(lib, margin, b, k, v, gen, 4, True, 1e5, (16, 8, 8), interleaved, True, 3)


def test_append_of_many_rows_and_sequences(lib, margin):
    """Beyond kQkFewRows; more sequences than a search's 64, and than 64 x 64."""
    b, k, v, gen = make(22, 1, 32, 16, [3] * 100, [17] * 100)
    append_case(lib, margin, b, k, v, gen, 2, True, 1e4)
    new = [(i % 3 == 0) * 1 for i in range(5000)]
    b, k, v, gen = make(23, 1, 16, 16, [i % 29 for i in range(5000)], new)
    append_case(lib, margin, b, k, v, gen, 1, False, 1e4)


def test_append_past_pages_and_rows(lib, margin):
    """Bad pages, places behind the last page, rows behind the last sequence: nothing is written for them."""
    b, k, v, gen = make(24, 2, 64, 16, [0, 14, 40], [20, 5, 9], bad=[(0, 1, -1), (1, 0, 10 ** 8)], pad=6)
    b["past"][2] = 16 * b["pages"].shape[1] - 4
    append_case(lib, margin, b, k, v, gen, 4, True, 1e4)
    b["max_new"] = 3
    append_case(lib, margin, b, k, v, gen, 4, True, 1e4)


# -------------------------------------------------------------------- keep ---


@pytest.mark.parametrize("layers,kv,hd,page", [(1, 1, 32, 16), (3, 2, 64, 32), (18, 8, 128, 64), (2, 1, 256, 256), (2, 3, 48, 16)])
@pytest.mark.parametrize("own", [False, True])
def test_keep(lib, layers, kv, hd, page, own):
    """Branches whose rows move onto rows that move themselves; none, one and all rows kept; longer than a step."""
    b, k, v, gen = make(page + hd, kv, hd, page, [0, 30, 15, 100, 7], [5, 12, 40, 40, 1], layers=layers)
    path = torch.full((5, 40), -1, dtype=I32)
    keepers = [[0, 1, 2, 3, 4], [], [0, 2, 3, 5, 6, 9, 10, 11, 20, 21, 22, 30, 31, 39], list(range(1, 40)), [0]]
    for s, p in enumerate(keepers):
        path[s, : len(p)] = torch.tensor(p, dtype=I32)
    count = torch.tensor([len(p) for p in keepers], dtype=I32)
    cache, bt = lib.KVCache(k.cuda(), v.cuda()), batch(lib, b)
    past = bt.past if own else torch.zeros(5, dtype=I32, device="cuda")
    lib.jn_kv_keep(lib.Context(), cache, bt, path.cuda(), count.cuda(), past)
    wk, wv, wp = plain.keep(b, k, v, path, count)
    assert torch.equal(cache.k.cpu(), wk) and torch.equal(cache.v.cpu(), wv) and past.tolist() == wp
    assert own or bt.past.tolist() == b["past"].tolist()


def test_keep_of_paths_that_are_none(lib):
    """Entries that do not ascend, are out of range or stand in bad pages move nothing."""
    b, k, v, gen = make(31, 2, 64, 16, [3, 20, 0], [12, 12, 12], bad=[(1, 1, -1)])
    path = torch.tensor([[0, 3, 2, 5, 5, 4, 99, -1], [1, 2, 11, 3, 0, 0, 0, 0], [7, 8, 9, 2 ** 31 - 1, -2 ** 31, 10, 11, 11]], dtype=I32)
    count = torch.tensor([100, 3, -5], dtype=I32)
    cache, bt = lib.KVCache(k.cuda(), v.cuda()), batch(lib, b)
    past = torch.zeros(3, dtype=I32, device="cuda")
    lib.jn_kv_keep(lib.Context(), cache, bt, path.cuda(), count.cuda(), past)
    wk, wv, wp = plain.keep(b, k, v, path, count)
    assert torch.equal(cache.k.cpu(), wk) and torch.equal(cache.v.cpu(), wv) and past.tolist() == wp == [11, 23, 0]


def test_calls_refused_on_the_gpu(lib):
    """What only the library's own checks see; nothing is written."""
    b, k, v, gen = make(41, 2, 64, 16, [5], [2], pad=0)
    ctx, cache, bt = lib.Context(), lib.KVCache(k.cuda(), v.cuda()), batch(lib, b)
    q, out = torch.zeros(2, 4 * 64, dtype=BF16, device="cuda"), torch.ones(2, 4 * 64, dtype=BF16, device="cuda")
    ws = torch.empty(max(1, lib.jn_kv_attention_workspace_size(cache, bt, 4)), dtype=torch.uint8, device="cuda")
    with pytest.raises(lib.JNError, match="EINVAL"):
        lib.jn_kv_attention(ctx, cache, 0, bt, 4, q, q, ws)
    with pytest.raises(lib.JNError, match="ESHAPE"):
        lib.jn_kv_attention(ctx, cache, 1, bt, 4, q, out, ws)
    with pytest.raises(lib.JNError, match="EINVAL"):
        lib.jn_kv_attention(ctx, cache, 0, bt, 3, q, out, ws)
    with pytest.raises(lib.JNError, match="EINVAL"):
        lib.jn_kv_attention(ctx, cache, 0, bt, 4, q, out, ws, float("inf"))
    with pytest.raises(lib.JNError, match="EINVAL"):
        lib.jn_kv_append(ctx, cache, 0, bt, lib.QKNormRope(0, 1, 64), torch.zeros(2, 256, dtype=BF16, device="cuda"), None, None)
    with pytest.raises(lib.JNError, match="EINVAL"):
        lib.jn_kv_append(ctx, cache, 0, bt, lib.QKNormRope(1, 2, 64), torch.zeros(2, 320, dtype=BF16, device="cuda"), None, None)
    assert bool((out == 1).all()) and torch.equal(cache.k.cpu(), k)
