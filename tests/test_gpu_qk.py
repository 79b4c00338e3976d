"""Norms of queries and keys for each head and their rotation by one to four position axes, forward and gradients,
against the definitions in float64.

Bars, per element (half a bf16 step is 2^-8 of a value, an fp32 rounding 2^-24): the output is rounded once, 2^-8 of
it; before that every value passes the norm's sum (at most 16 + 4 additions, halved by the root), three products and
the rotation's two products, one sum and two table values of 2 steps each: under 40 roundings of the pair's
magnitude, below 2^-18 of it.  The input's gradient has one more sum over the head: below 2^-17 of the magnitudes
it is made of.  Gain gradients are fp32 sums: one rounding per addition in the longest chain, plus 64 for each term,
of the sum of the terms' magnitudes."""
import math

import pytest
import torch  # before the library: both then share one HIP runtime

pytestmark = pytest.mark.gpu

EPS = 1e-6


def make(lib, rows, heads, kv, hd, axes, norm, interleaved, theta=1e4, far=0, seed=0, pad=8):
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = (heads + kv) * hd
    x = torch.randn(rows, width + kv * hd + pad, generator=g, device="cuda").to(torch.bfloat16)
    gq = (1 + 0.3 * torch.randn(hd, generator=g, device="cuda")).to(torch.bfloat16) if norm else None
    gk = (1 + 0.3 * torch.randn(hd, generator=g, device="cuda")).to(torch.bfloat16) if norm else None
    pos = (torch.randint(0, 700, (rows, max(axes, 1)), generator=g, device="cuda") + far).to(torch.int32)
    half = hd // 2
    rest = half // (axes + 1) if axes > 1 else 0
    sections = [half - rest * (axes - 1)] + [rest] * (axes - 1) if axes > 1 else []
    qk = lib.QKNormRope(heads, kv, hd, EPS, gq, gk, theta, sections, interleaved)
    return x, gq, gk, pos, sections, qk


def pair_axes(hd, sections, interleaved):
    """The rule of the header, pair by pair."""
    axes, half = len(sections), hd // 2
    if axes < 2:
        return [0] * half
    left, out = list(sections), []
    for i in range(half):
        if interleaved:
            a = i % axes
            if a > 0 and left[a] > 0:
                left[a] -= 1
            else:
                a = 0
        else:
            a = next(k for k in range(axes) if left[k] > 0)
            left[a] -= 1
        out.append(a)
    return out


def reference(x, gq, gk, pos, heads, kv, hd, theta, sections, interleaved, dy=None):
    """float64 y, or (dx, dgq, dgk) and the magnitudes their bars refer to."""
    rows, n = x.shape[0], heads + kv
    v = x[:, : n * hd].double().view(rows, n, hd)
    half = hd // 2
    if gq is not None:
        gain = torch.cat([gq.double().expand(heads, hd), gk.double().expand(kv, hd)])
        r = 1 / (v.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
    else:
        gain, r = torch.ones(n, hd, dtype=torch.float64, device=x.device), torch.ones_like(v[..., :1])
    if theta > 0:
        freq = torch.tensor([theta ** (-2.0 * i / hd) for i in range(half)], dtype=torch.float64, device=x.device)
        ang = pos.view(rows, -1).double()[:, torch.tensor(pair_axes(hd, sections, interleaved), device=x.device)] * freq
    else:
        ang = torch.zeros(rows, half, dtype=torch.float64, device=x.device)
    c, s = ang.cos()[:, None], ang.sin()[:, None]

    def turn(t, sign):
        a, b = t[..., :half], t[..., half:]
        return torch.cat([a * c - sign * b * s, b * c + sign * a * s], -1)

    def pairs(t):
        m = (t[..., :half] ** 2 + t[..., half:] ** 2).sqrt()
        return torch.cat([m, m], -1)

    if dy is None:
        u = v * r * gain
        return turn(u, 1.0).view(rows, -1), pairs(u).view(rows, -1)
    du = turn(dy.double().view(rows, n, hd), -1.0)
    if gq is None:
        return (du.view(rows, -1), pairs(du).view(rows, -1)), None, None
    xh, t = v * r, du * gain
    dx = r * (t - xh * (xh * t).mean(-1, keepdim=True))
    mag = r * (pairs(du) * gain.abs() + xh.abs() * (xh.abs() * pairs(du) * gain.abs()).mean(-1, keepdim=True))
    terms = du * xh
    mags = pairs(du) * xh.abs()
    return ((dx.view(rows, -1), mag.view(rows, -1)), (terms[:, :heads].sum((0, 1)), mags[:, :heads].sum((0, 1))),
            (terms[:, heads:].sum((0, 1)), mags[:, heads:].sum((0, 1))))


def within(got, ref, bar):
    bad = (got.double() - ref).abs() > bar
    assert not bool(bad.any()), (int(bad.sum()), float(((got.double() - ref).abs() / bar.clamp(min=1e-300)).max()))


SHAPES = [
    # rows, heads, kv, hd, axes, norm, interleaved
    (1, 1, 1, 16, 1, True, False),
    (1, 16, 2, 128, 3, True, True),
    (3, 8, 1, 256, 1, True, False),
    (5, 5, 0, 32, 2, True, False),
    (7, 0, 3, 48, 3, True, True),
    (257, 12, 4, 96, 3, True, True),
    (64, 3, 2, 80, 4, True, False),
    (301, 12, 12, 64, 1, False, False),
    (130, 6, 2, 240, 4, False, True),
    (1023, 9, 3, 112, 2, True, True),
    (1024, 16, 2, 128, 3, True, False),   # one wavefront per row from here on
    (5003, 8, 8, 256, 3, True, False),
    (9001, 4, 1, 32, 2, False, True),
    (60001, 20, 12, 80, 3, True, True),   # results beyond the last-level cache
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_forward(lib, shape):
    rows, heads, kv, hd, axes, norm, inter = shape
    x, gq, gk, pos, sec, qk = make(lib, *shape, seed=1)
    ctx = lib.Context()
    width = (heads + kv) * hd
    want, mag = reference(x, gq, gk, pos, heads, kv, hd, 1e4, sec, inter)
    y = torch.full((rows, width + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    lib.jn_qk_norm_rope(ctx, qk, x, pos, y)
    within(y[:, :width], want, 2.0 ** -8 * want.abs() + 2.0 ** -18 * mag)
    assert bool((y[:, width:] == 7.0).all())
    again = x.clone()
    lib.jn_qk_norm_rope(ctx, qk, again, pos, again)  # in place; what is behind the heads stays
    assert torch.equal(again[:, :width], y[:, :width]) and torch.equal(again[:, width:], x[:, width:])


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_gradients(lib, shape):
    rows, heads, kv, hd, axes, norm, inter = shape
    x, gq, gk, pos, sec, qk = make(lib, *shape, seed=2)
    ctx = lib.Context()
    width = (heads + kv) * hd
    dy = torch.randn(rows, width + 24, device="cuda").to(torch.bfloat16)
    dx = torch.full((rows, width + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    need = lib.jn_qk_norm_rope_workspace_size(qk, rows)
    ws = torch.full((need + 64,), 3, dtype=torch.uint8, device="cuda")
    dgq, dgk = (torch.full((hd + 4,), 5.0, device="cuda") for _ in range(2))
    args = (dgq[:hd], dgk[:hd]) if norm else (None, None)
    lib.jn_qk_norm_rope_bwd(ctx, qk, x if norm else None, pos, dy, dx, *args, ws)
    (want, mag), rq, rk = reference(x, gq, gk, pos, heads, kv, hd, 1e4, sec, inter, dy[:, :width])
    within(dx[:, :width], want, 2.0 ** -8 * want.abs() + 2.0 ** -17 * mag)
    assert bool((dx[:, width:] == 7.0).all()) and bool((ws[need:] == 3).all())
    if not norm:
        return
    chain = math.ceil(rows / 4096) * (heads + kv) + min(1024, rows) / 16 + 64
    for got, (ref, m) in ((dgq, rq), (dgk, rk)):
        within(got[:hd], ref, chain * 2.0 ** -24 * m + 1e-30)
        assert bool((got[hd:] == 5.0).all())
    # in place over dy, and twice the same bits
    dx2, old = dy.clone(), (dgq.clone(), dgk.clone())
    lib.jn_qk_norm_rope_bwd(ctx, qk, x, pos, dx2, dx2, *args, ws)
    assert torch.equal(dx2[:, :width], dx[:, :width]) and torch.equal(dgq, old[0]) and torch.equal(dgk, old[1])
    # over x
    dx3 = x.clone()
    lib.jn_qk_norm_rope_bwd(ctx, qk, dx3, pos, dy, dx3, *args, ws)
    assert torch.equal(dx3[:, :width], dx[:, :width]) and torch.equal(dgq, old[0])


@pytest.mark.parametrize("far", [0, 10 ** 6, 2 ** 31 - 1000, -2 ** 31])
def test_far_positions(lib, far):
    """The angle of a far position is as exact as a near one's."""
    shape = (33, 4, 1, 128, 3, True, True)
    x, gq, gk, pos, sec, qk = make(lib, *shape, theta=1e6, far=far, seed=3)
    y = torch.empty(33, 5 * 128, dtype=torch.bfloat16, device="cuda")
    lib.jn_qk_norm_rope(lib.Context(), qk, x, pos, y)
    want, mag = reference(x, gq, gk, pos, 4, 1, 128, 1e6, sec, True)
    # the float64 product pos * frequency rounds by 2^-53 of up to 2^31 turns on both sides
    within(y, want, 2.0 ** -8 * want.abs() + 2.0 ** -18 * mag)


def test_norm_without_rotation(lib):
    x, gq, gk, _, _, _ = make(lib, 19, 3, 2, 64, 1, True, False, seed=4)
    qk = lib.QKNormRope(3, 2, 64, EPS, gq, gk)
    y = torch.empty(19, 320, dtype=torch.bfloat16, device="cuda")
    ctx = lib.Context()
    lib.jn_qk_norm_rope(ctx, qk, x, None, y)
    want, mag = reference(x, gq, gk, None, 3, 2, 64, 0.0, [], False)
    within(y, want, 2.0 ** -8 * want.abs() + 2.0 ** -18 * mag)
    dy = torch.randn(19, 320, device="cuda").to(torch.bfloat16)
    dx, dgq, dgk = torch.empty_like(dy), torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
    ws = torch.empty(lib.jn_qk_norm_rope_workspace_size(qk, 19), dtype=torch.uint8, device="cuda")
    lib.jn_qk_norm_rope_bwd(ctx, qk, x, None, dy, dx, dgq, dgk, ws)
    (want, mag), rq, _ = reference(x, gq, gk, None, 3, 2, 64, 0.0, [], False, dy)
    within(dx, want, 2.0 ** -8 * want.abs() + 2.0 ** -17 * mag)
    within(dgq, rq[0], 100 * 2.0 ** -24 * rq[1])


def test_no_rows(lib):
    x, gq, gk, pos, sec, qk = make(lib, 1, 2, 1, 32, 1, True, False)
    ctx = lib.Context()
    e = torch.empty(0, 96, dtype=torch.bfloat16, device="cuda")
    lib.jn_qk_norm_rope(ctx, qk, e, pos[:0], e)
    dgq, dgk = torch.full((32,), 5.0, device="cuda"), torch.full((32,), 5.0, device="cuda")
    ws = torch.empty(16, dtype=torch.uint8, device="cuda")
    lib.jn_qk_norm_rope_bwd(ctx, qk, e, pos[:0], e, e, dgq, dgk, ws)
    assert float(dgq.abs().max()) == 0.0 and float(dgk.abs().max()) == 0.0


def test_zero_rows_and_nan_rows_stay_to_themselves(lib):
    x, gq, gk, pos, sec, qk = make(lib, 40, 4, 2, 128, 3, True, False, seed=5)
    ctx = lib.Context()
    y, y2 = (torch.empty(40, 768, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lib.jn_qk_norm_rope(ctx, qk, x, pos, y)
    x2 = x.clone()
    x2[7] = 0
    x2[9, 128:256] = float("nan")
    x2[11, 0] = float("inf")
    lib.jn_qk_norm_rope(ctx, qk, x2, pos, y2)
    assert float(y2[7].abs().max()) == 0.0
    assert bool(y2[9, 128:256].isnan().all()) and torch.equal(y2[9, :128], y[9, :128]) and torch.equal(y2[9, 256:], y[9, 256:])
    keep = [i for i in range(40) if i not in (7, 9, 11)]
    assert torch.equal(y2[keep], y[keep]) and torch.equal(y2[11, 128:], y[11, 128:])


def test_captured_and_replayed(lib):
    shape = (777, 8, 2, 128, 3, True, True)
    x, gq, gk, pos, sec, qk = make(lib, *shape, seed=6)
    dy = torch.randn(777, 1280, device="cuda").to(torch.bfloat16)
    y, dx = torch.empty_like(dy), torch.empty_like(dy)
    dgq, dgk = torch.empty(128, device="cuda"), torch.empty(128, device="cuda")
    ws = torch.empty(lib.jn_qk_norm_rope_workspace_size(qk, 777), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    ctx = lib.Context(stream)

    def both():
        lib.jn_qk_norm_rope(ctx, qk, x, pos, y)
        lib.jn_qk_norm_rope_bwd(ctx, qk, x, pos, dy, dx, dgq, dgk, ws)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        both()
    for k in range(3):
        x.copy_(torch.randn(x.shape, device="cuda"))
        pos.add_(11 * k)
        torch.cuda.synchronize()
        both()
        torch.cuda.synchronize()
        want = [t.clone() for t in (y, dx, dgq, dgk)]
        for t in (y, dx, dgq, dgk):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (y, dx, dgq, dgk)))


def test_refusals(lib):
    x, gq, gk, pos, sec, qk = make(lib, 8, 4, 2, 64, 1, True, False, pad=0)
    ctx = lib.Context()
    y = torch.full((8, 384), 7.0, dtype=torch.bfloat16, device="cuda")
    abi = lib._abi

    def refused(code, q, xx=x, yy=y, p=pos):
        with pytest.raises(lib.JNError) as e:
            lib.jn_qk_norm_rope(ctx, q, xx, p, yy)
        assert e.value.status == code, e.value

    refused(abi.JN_EUNSUPPORTED, lib.QKNormRope(4, 2, 24, EPS, gq, gk, 1e4))
    refused(abi.JN_EUNSUPPORTED, lib.QKNormRope(1, 0, 272, EPS, gq, gk, 1e4))
    refused(abi.JN_EINVAL, lib.QKNormRope(4, 2, 64, 0.0, gq, gk, 1e4))
    refused(abi.JN_EINVAL, lib.QKNormRope(4, 2, 64, EPS, gq, None, 1e4))
    refused(abi.JN_EINVAL, lib.QKNormRope(4, 2, 64, EPS))
    refused(abi.JN_EINVAL, lib.QKNormRope(4, 2, 64, EPS, gq, gk, -1.0))
    refused(abi.JN_EINVAL, lib.QKNormRope(4, 2, 64, EPS, gq, gk, float("inf")))
    p2 = pos.repeat(1, 2).contiguous()
    refused(abi.JN_EINVAL, lib.QKNormRope(4, 2, 64, EPS, gq, gk, 1e4, [16, 15]), p=p2)
    refused(abi.JN_EINVAL, lib.QKNormRope(4, 2, 64, EPS, gq, gk, 1e4, [33, -1]), p=p2)
    refused(abi.JN_EINVAL, lib.QKNormRope(4, 2, 64, EPS, gq, gk, 1e4, [15, 17], True), p=p2)
    refused(abi.JN_EINVAL, qk, p=None)
    refused(abi.JN_EUNSUPPORTED, qk, xx=torch.empty(8 * 516, dtype=torch.bfloat16, device="cuda").view(8, 516))
    flat = torch.empty(8 * 384 + 1, dtype=torch.bfloat16, device="cuda")
    refused(abi.JN_EUNSUPPORTED, qk, yy=flat[1:].view(8, 384))
    assert bool((y == 7.0).all())
    dg = torch.full((64,), 5.0, device="cuda")
    dy = torch.empty_like(y)
    ws = torch.empty(lib.jn_qk_norm_rope_workspace_size(qk, 8), dtype=torch.uint8, device="cuda")
    for a in ((dg, None, ws), (dg, dg, ws[:-1]), (dg, dg, None)):
        with pytest.raises(lib.JNError):
            lib.jn_qk_norm_rope_bwd(ctx, qk, x, pos, dy, y, *a)
    torch.cuda.synchronize()
    assert bool((dg == 5.0).all()) and bool((y == 7.0).all())
