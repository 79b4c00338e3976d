"""Rows of targets where maps name a tenant without samples, and where pairs are far outside (CPU)."""
import numpy as np
import pytest
import torch  # before the library: both then share one HIP runtime  # noqa: F401


@pytest.mark.parametrize("slot", [0, 1, 2, 3])
def test_tenants_without_samples(lib, slot):
    from paper_2607_16074_amd import step
    # three samples of 3, 5 and 2 rows at 0, 4 and 12, all of them tenant 1's
    maps = {"tenant_sample_off": np.array([0, 0, 3, 3, 3]), "tenant_perm": np.array([0, 1, 2]),
            "seqlens": np.array([3, 5, 2]), "cu_seqlens": np.array([0, 4, 12, 16])}
    sample, row = np.array([-1, 0, 2, 3, 0, 1]), np.array([-1, 0, 1, 0, 3, 4])
    want = [-1, 0, 13, -1, -1, 8] if slot == 1 else [-1] * 6
    got = step.target_rows(maps, slot, sample, row)
    assert got.tolist() == want and got.dtype == np.int32
    none = np.array([], np.int64)
    assert step.target_rows(maps, slot, none, none).shape == (0,)
    far = np.array([2 ** 40, -2 ** 40, 0])
    assert step.target_rows(maps, slot, far, np.array([0, 0, 2 ** 40])).tolist() == [-1] * 3


def test_one_sample_and_many_rows(lib):
    from paper_2607_16074_amd import step
    maps = {"tenant_sample_off": np.array([0, 0, 3]), "tenant_perm": np.array([0, 1, 2]), "seqlens": np.array([3, 5, 2]),
            "cu_seqlens": np.array([0, 4, 12, 16])}
    assert step.target_rows(maps, 1, 1, np.arange(-1, 6)).tolist() == [-1, 4, 5, 6, 7, 8, -1]
    assert step.target_rows(maps, 1, np.array([[0], [2]]), np.arange(3)).tolist() == [[0, 1, 2], [12, 13, -1]]
    assert step.target_rows(maps, 1, [2, 0], [1, 9]).tolist() == [13, -1]
    assert int(step.target_rows(maps, 1, 2, 1)) == 13 and int(step.target_rows(maps, 0, 0, 0)) == -1
