"""Expert products: repeated calls, sums that several SMs share, and the memory that a call
may touch.  Tolerances are those of test_gpu_products."""
import pytest

from paper_2606_00539_gb300 import ExpertProducts

pytestmark = pytest.mark.gpu

import torch  # noqa: E402

from .test_gpu_products import check, gen, normal, offsets_of, spans  # noqa: E402


@pytest.fixture(scope="module")
def products():
    p = ExpertProducts(device=0)
    yield p
    p.close()


@pytest.mark.parametrize("counts,n,k", [([1, 0, 2, 1, 1, 1], 1408, 2048), ([1], 264, 8200), ([40], 200, 5000)])
def test_joined_parts_are_whole_and_the_same_each_time(products, counts, n, k):
    """Few tiles, so that several pairs of SMs share each: every one of many calls has all parts of all lanes."""
    g, t, R = gen(n + k), torch.bfloat16, sum(counts)
    x, w, off = normal(g, R, k, dtype=t), normal(g, len(counts), n, k, dtype=t, size=k ** -0.5), offsets_of(counts)
    first = products.forward(x, w, off)
    for e, at in spans(counts):
        X, W = x[at].double(), w[e].double()
        check(first[at], X @ W.T, X.abs() @ W.abs().T, k, "bf16")
    outs = [products.forward(x, w, off) for _ in range(300)]
    assert all(torch.equal(y, first) for y in outs)
