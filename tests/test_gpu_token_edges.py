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
