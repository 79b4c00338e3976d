"""Token heads where W or the feature is not finite, at the sizes and paths where that could reach what it should not."""
import pytest
import torch  # before the library: both then share one HIP runtime

from test_gpu_tokens import Pick, Tenant, decode, draw, feature, step

pytestmark = pytest.mark.gpu


def without(lib, t, ban):
    """Tenant `t` as if its vocabulary held no token `ban`: the same outputs less that token's."""
    v, d = t.W.shape
    keep = torch.arange(v, device="cuda") != ban
    rest = Tenant(lib, t.W[keep], t.rows, torch.where(t.targets > ban, t.targets - 1, t.targets), t.dh is not None,
                  t.dW.dtype is torch.float32)
    rest.logp.copy_(t.logp)
    rest.loss.copy_(t.loss)
    rest.dW.copy_(torch.cat([t.dW[: v * d].view(v, d)[keep].reshape(-1), t.dW[v * d:]]))
    return rest


@pytest.mark.parametrize("d", [2112, 4096, 4160, 5120, 6144, 8192])
def test_a_token_of_no_probability_in_wide_heads(lib, d):
    """The streaming launches take a wide row's contraction in chunks; an infinity in any of them stays in its token."""
    n, v, ban = 16, 600, 17
    for k in (0, 5 * 32 + 3, 10 * 32 + 1, 15 * 32 + 31, d // 8 - 1, d // 2 + 9, d - 1):
        hidden = feature(n, d)
        hidden[:, k] = 1.0
        W, rows, targets = draw(n, v, d, n, 90)
        rows.copy_(torch.arange(n))
        targets[targets == ban] = 3
        W[ban] = 0.0
        W[ban, k] = float("-inf")
        t = Tenant(lib, W, rows, targets, False)
        step(lib, lib.Context(), hidden, [t])
        assert bool((t.dW[ban * d: (ban + 1) * d] == 0).all()), k
        without(lib, t, ban).check(hidden)
        pick = Pick(lib, W, rows)
        decode(lib, lib.Context(), hidden, [pick])
        assert bool((pick.token[:n] != ban).all()) and bool(torch.isfinite(pick.logp[:n]).all()), k


@pytest.mark.parametrize("value", ["-inf", "inf", "nan"])
@pytest.mark.parametrize("case", [(20, 100003, 128), (40, 530001, 128), (20, 600, 64), (100, 400, 64), (300, 3001, 128),
                                  (200, 20001, 256), (2000, 300007, 64)], ids=lambda c: "-".join(map(str, c)))
def test_row_gradients_of_entries_without_a_target(lib, case, value):
    """Their gradient is zero whatever W holds: behind the streaming launches, of one plane, of several, of several pieces."""
    n, v, d = case
    hidden = feature(n, d)
    hidden[:, 0] = 1.0
    W, rows, targets = draw(n, v, d, n, 91)
    rows[1], targets[2], rows[n - 1], targets[n // 2] = -1, -1, n, v
    W[v // 3] = 0.0
    W[v // 3, 0] = float(value)
    W[v - 2, 5] = float(value)
    for f32 in (False, True):
        t = Tenant(lib, W, rows, targets, True, f32)
        step(lib, lib.Context(), hidden, [t])
        dead = (rows < 0) | (rows >= n) | (targets < 0) | (targets >= v)
        assert int(dead.sum()) == 4
        dh = t.dh[: n * d].view(n, d)
        assert bool((dh[dead] == 0).all()) and bool((t.logp[:n][dead] == 0).all())
        assert bool(dh[~dead].isnan().any())  # (a live row's product with an infinity is what the formula says)


@pytest.mark.parametrize("case", [(5, 600, 64, 300), (40, 100003, 128, 7), (100, 600, 64, 300), (2000, 300007, 64, 3),
                                  (2000, 300007, 64, 300001)], ids=lambda c: "-".join(map(str, c)))
def test_an_infinite_logit_of_a_target_is_not_hidden(lib, case):
    """Such a row has no softmax: its loss is infinite, and its gradient does not read as that of a row without a target,
    nor reach other tokens' rows where the infinite token's block is not theirs."""
    n, v, d, bad = case
    hidden = feature(n, d)
    hidden[:, 0] = 0.0
    hidden[1, 0] = 1.0  # the others meet the infinity with 0 * inf, so they have no target
    W, rows, targets = draw(n, v, d, n, 92)
    rows.copy_(torch.arange(n))
    targets[targets == bad] = 0
    targets[0], targets[2:] = -1, -1
    W[bad] = 0.0
    W[bad, 0] = float("inf")
    t = Tenant(lib, W, rows, targets, False, True)
    step(lib, lib.Context(), hidden, [t])
    assert float(t.loss[0]) == float("inf") and float(t.logp[1]) == -float("inf")
    dW = t.dW[: v * d].view(v, d)
    assert bool(dW[bad].isnan().all())
    far = (bad + v // 2) % v
    y = int(targets[1])
    assert bool(torch.isfinite(dW[far]).all()) and (abs(y - bad) <= 256 or bool((dW[y] == -hidden[1].float()).all()))


@pytest.mark.parametrize("case", [(1, 1, 64), (5, 37, 64), (16, 301, 768), (64, 1003, 2048), (16, 700, 8192), (3, 20001, 320),
                                  (100, 301, 64), (70, 20001, 128)], ids=lambda c: "-".join(map(str, c)))
def test_decode_of_equal_infinite_logits_takes_the_lowest(lib, case):
    """All logits -inf, or all but the last ones: still the lowest of equal ones."""
    n, v, d = case
    hidden = feature(n, d)
    hidden[:, 0] = 1.0
    W, rows, _ = draw(n, v, d, n, 93)
    rows.copy_(torch.arange(n))
    W[:] = 0.0
    W[:, 0] = float("-inf")
    pick = Pick(lib, W, rows)
    decode(lib, lib.Context(), hidden, [pick])
    assert bool((pick.token[:n] == 0).all()) and bool(pick.logp[:n].isnan().all())
    if v > 2:
        W[v - 2:, 0] = 1.0
        decode(lib, lib.Context(), hidden, [pick])
        assert bool((pick.token[:n] == v - 2).all())
        assert float((pick.logp[:n] + 0.6931472).abs().max()) < 1e-6
