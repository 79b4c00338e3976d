"""Row strides that the binding hands to the head-norm calls (CPU)."""
import pytest
import torch  # before the library: both then share one HIP runtime


@pytest.mark.parametrize("width", [64, 65, 70, 72, 516])
def test_one_row_of_any_width(lib, width):
    """A single row is not apart from anything, so that no stride of it is refused (strides are multiples of 8)."""
    qk = lib.QKNormRope(1, 0, 64, theta=1e4)
    pos = torch.zeros(1, dtype=torch.int32)
    x = torch.zeros(1, width, dtype=torch.bfloat16)
    a = qk.at(1, pos, x, x)
    assert a.ld_in == a.ld_out and a.ld_in % 8 == 0 and a.ld_in >= width
    part = torch.zeros(5, 72, dtype=torch.bfloat16)[3:4, :64]
    assert qk.at(1, pos, part, x).ld_in == 72
    two = torch.zeros(2, width, dtype=torch.bfloat16)
    assert qk.at(2, torch.zeros(2, dtype=torch.int32), two, two).ld_in == width
    assert qk.at(0, pos[:0], x[:0], x[:0]).ld_in % 8 == 0
