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
