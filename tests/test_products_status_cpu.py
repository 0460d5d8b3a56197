"""Status calls of the expert products without a GPU."""
import pytest

from paper_2606_00539_gb300 import ExpertProducts, GnmrError
from paper_2606_00539_gb300 import _native as N
from paper_2606_00539_gb300 import build as native_build


@pytest.fixture(scope="module", autouse=True)
def lib():
    native_build.build()
    return N.load()


def test_refusals_without_a_handle():
    for call in (lambda: N.gnmr_products_status(None), lambda: N.gnmr_products_set_wait_limit(None, 5)):
        with pytest.raises(GnmrError) as e:
            call()
        assert e.value.status == N.GNMR_ERR_INVALID_ARG and "products:" in e.value.detail


def test_a_handle_is_freed_once_whatever_its_destruction_reports(monkeypatch):
    """What gnmr_products_destroy reports reaches the caller of close(), who may then close again."""
    freed = []

    def destroy(h):
        freed.append(h)
        raise GnmrError(N.GNMR_ERR_STATE, "products: a product of this handle gave up waiting inside the GPU")

    monkeypatch.setattr(N, "gnmr_products_destroy", destroy)
    p = ExpertProducts.__new__(ExpertProducts)
    p._h = 4096
    with pytest.raises(GnmrError):
        p.close()
    p.close()
    assert freed == [4096]
    with pytest.raises(ValueError):
        p.check()


def test_gradients_of_groups_side_by_side_are_allowed_and_overlapping_ones_are_not():
    p = N.gnmr_product(op=N.GNMR_PRODUCT_WEIGHT_GRAD, groups=3, rows=10, n_out=16, n_in=8, dtype=N.GNMR_DTYPE_BF16,
                       out_dtype=N.GNMR_DTYPE_F32, d_offsets=4096, d_x=4096, x_stride=8, d_dy=4096, dy_stride=16, d_out=4096)
    for row, group, fine in ((24, 8, True), (40, 16, True), (23, 8, False), (24, 7, False), (8, 128, True), (8, 127, False),
                             (25, 8, True), (24, 0, False), (24, -8, False)):
        p.out_stride, p.out_group_stride = row, group
        if fine:
            assert N.gnmr_products_scratch_bytes(p) == 0
        else:
            with pytest.raises(GnmrError) as e:
                N.gnmr_products_scratch_bytes(p)
            assert e.value.status == N.GNMR_ERR_LAYOUT
