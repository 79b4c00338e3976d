"""How many bits of the logits' gradient dz reach the weight and row gradients of token heads.

Every tenant here has logits near its targets' (probabilities of 0.02 to 0.98), so that dz is no power of two.  Bars, of
one term dz h: a logit is off by at most D = d 2^-24 sum|h w|, so p by p 2D, and by 2^-21 (1 + max|z|) of it for lse2,
the exponential and their roundings; what dz is rounded to adds its own share (given at each test); sums of up to 640
terms in fp32 add 2^-24 of the terms' magnitudes each."""
import pytest
import torch  # before the library: both then share one HIP runtime

from test_gpu_tokens import BF, Tenant, draw, feature, step

pytestmark = pytest.mark.gpu


def problem(lib, n, v, d, dh, f32, live=None, seed=80):
    """Tenant and feature: entry i reads row i, and its target holds a share of the probability."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    W, rows, targets = draw(n, v, d, n, seed)
    rows.copy_(torch.arange(n))
    if live is not None:
        targets[live:] = -1
    share = 0.02 + 0.96 * torch.rand(n, 1, generator=g, device="cuda")
    up = torch.log(v * share / (1 - share))  # the target's logit, where the others' are near 0
    w = W[targets.clamp(min=0).long()].float()
    hidden = (up * w / w.square().sum(1, keepdim=True) + 0.05 * feature(n, d, seed).float()).to(torch.bfloat16)
    return Tenant(lib, W, rows, targets, dh, f32), hidden


def check(t, hidden, rounding, adds=640, adds_dh=None):
    """`rounding`: of dz, relative; `adds`: the longest sum of dW, and of dh where nothing else is said."""
    n, (v, d) = t.rows.numel(), t.W.shape
    y, live = t.targets.long().clamp(min=0)[:, None], (t.targets >= 0)[:, None]
    h, w = torch.where(live, hidden.double(), 0.0), t.W.double()
    z = h @ w.T
    D = d * 2.0 ** -24 * (h.abs() @ w.abs().T).amax(1, keepdim=True)
    p = torch.softmax(z, 1)
    count = int(live.sum())
    dz = torch.where(live, p.scatter_add(1, y, torch.full((n, 1), -1.0, dtype=torch.float64, device="cuda")), 0.0) / count
    err = dz.abs() * (rounding + 8 * 2.0 ** -24)
    err += torch.where(live, p, 0.0) * (2 * D + 2.0 ** -21 * (1 + z.abs().amax(1, keepdim=True))) / count
    sums = [err + adds * 2.0 ** -24 * dz.abs() for adds in (adds, adds_dh or adds)]

    def within(got, ref, spread, what):
        own = 0.0 if got.dtype is torch.float32 else BF
        o, b = (got.double() - ref).abs(), own * ref.abs() + (1 + own) * spread + 1e-37
        assert bool((o <= b).all()), (what, float((o / b).max()))

    within(t.dW[: v * d].view(v, d), dz.T @ h, sums[0].T @ h.abs(), "dW")
    if t.dh is not None:
        within(t.dh[: n * d].view(n, d), dz @ w, sums[1] @ w.abs(), "dh")


@pytest.mark.parametrize("f32", [True, False], ids=["fp32", "bf16"])
@pytest.mark.parametrize("case", [(1, 256, 64), (2, 300, 64), (7, 256, 128), (16, 999, 192), (33, 600, 64), (64, 999, 128),
                                  (20, 333, 1088), (40, 400, 2048)], ids=lambda c: "-".join(map(str, c)))
def test_few_rows_keep_dz(lib, case, f32):
    """Groups of at most 64 rows a tenant: dz as two bf16, half a step of the second below half a step of the first."""
    t, hidden = problem(lib, *case, False, f32)
    step(lib, lib.Context(), hidden, [t])
    check(t, hidden, 2.0 ** -16)


@pytest.mark.parametrize("case", [(1, 100003, 128), (5, 120001, 128), (32, 110003, 128), (33, 530001, 128), (64, 530003, 128),
                                  (3, 1601, 8192)],
                         ids=lambda c: "-".join(map(str, c)))
def test_few_rows_keep_dz_in_row_gradients(lib, case):
    t, hidden = problem(lib, *case, True, True)
    step(lib, lib.Context(), hidden, [t])
    # sums over ranges of 512 to 4,160 columns, then over up to 256 of them
    check(t, hidden, 2.0 ** -16, 4500)


@pytest.mark.parametrize("f32", [True, False], ids=["fp32", "bf16"])
@pytest.mark.parametrize("case", [(100, 3001, 64, 1), (100, 3001, 64, 100), (300, 2049, 128, 3), (700, 8193, 64, 2),
                                  (2000, 300007, 64, 1)], ids=lambda c: "-".join(map(str, c)))
def test_dz_of_many_rows_is_rounded_once(lib, case, f32):
    """Groups of more rows: dz to bf16 (2^-8) from logits kept in 16 bits (ln 2 / 1024 < 2^-10 of the exponential) or formed
    again.  One or a few targets, so that the weight gradients show single terms."""
    n, v, d, live = case
    t, hidden = problem(lib, n, v, d, True, f32, live)
    step(lib, lib.Context(), hidden, [t])
    check(t, hidden, BF + 2.0 ** -10, n, v)
