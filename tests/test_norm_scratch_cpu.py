"""The scratch memory of the layer norm's backward pass: sums over the rows in parts, of which there are no more than rows (and one,
where every second row starts alike), nor more than 512."""
import pytest

from paper_2606_00539_gb300 import _native as N
from paper_2606_00539_gb300 import build as native_build


@pytest.fixture(scope="module", autouse=True)
def library():
    native_build.build()
    return N.load()


def bytes_for(rows, cols, dweight=4096, dbias=4096):
    p = N.gnmr_norm()
    p.rows, p.cols, p.d_dweight, p.d_dbias = rows, cols, dweight, dbias
    return N.gnmr_layer_norm_scratch_bytes(p)


@pytest.mark.parametrize("cols", [1, 7, 5120, 131072, 1 << 30])
@pytest.mark.parametrize("rows", [1, 2, 3, 100, 511, 512, 20000, 2 ** 31 - 1])
def test_scratch_goes_by_the_rows(rows, cols):
    need = bytes_for(rows, cols)
    most = min(rows + 1, 512)
    assert 2 * min(rows, 512) * cols * 4 <= need <= 2 * most * cols * 4 + 255 and need % 256 == 0
    assert bytes_for(rows, cols, dbias=None) == bytes_for(rows, cols, dweight=None) == need
    assert bytes_for(rows, cols, None, None) == 0


def test_a_row_of_the_widest_kind_fits_a_card():
    assert bytes_for(1, 1 << 30) <= 17 << 30


def test_no_rows_need_none():
    assert bytes_for(0, 5120) == 0


@pytest.mark.parametrize("rows,cols", [(-1, 8), (1 << 31, 8), (1, 0), (1, (1 << 30) + 1)])
def test_sizes_out_of_range(rows, cols):
    with pytest.raises(N.GnmrError) as e:
        bytes_for(rows, cols)
    assert e.value.status == N.GNMR_ERR_INVALID_ARG
