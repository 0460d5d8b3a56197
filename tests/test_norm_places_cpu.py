"""The row strides that the layer norm takes from tensors: a check on the host, so that the host's memory will do."""
import pytest
import torch

from paper_2606_00539_gb300 import LayerNorm
from paper_2606_00539_gb300 import build as native_build


@pytest.fixture(scope="module")
def norms():
    native_build.build()
    n = LayerNorm()
    n.device_index = -1                            # what a tensor of the host says
    return n


def test_one_row_has_no_stride(norms):
    """The same row seen as one of every second, or of a far longer stride, lies where it lies: in place is in place, and no distance is too far."""
    rows = torch.zeros(8, 40)
    for x in (rows[:1], rows[::2][:1], rows[::5][1:], torch.as_strided(rows, (1, 40), (1 << 40, 1)), torch.as_strided(rows, (1, 40), (0, 1))):
        assert norms._matrix(x, "x", None, (torch.float32,)) == (1, 40, 40)
    assert norms._matrix(rows[::2], "x", None, (torch.float32,)) == (4, 40, 80)
    assert norms._matrix(rows[:0], "x", None, (torch.float32,)) == (0, 40, 40)
    assert norms._matrix(rows[:, :1], "x", None, (torch.float32,)) == (8, 1, 40)
