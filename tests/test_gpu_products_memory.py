"""Expert products: repeated calls, sums that several SMs share, and the memory that a call
may touch.  Tolerances are those of test_gpu_products."""
import numpy as np
import pytest

from paper_2606_00539_gb300 import ExpertProducts
from paper_2606_00539_gb300 import _native as N

pytestmark = pytest.mark.gpu

import torch  # noqa: E402

from .test_gpu_products import check, codes_oracle, gen, normal, offsets_of, spans  # noqa: E402


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


@pytest.mark.parametrize("k,stride", [(100, 128), (1264, 1280), (65, 128), (128, 128), (100, 192), (70, 70)])
def test_widened_codes_hold_no_columns_but_the_rows_own(products, k, stride):
    """Rows that the 8-bit product widens in scratch: zeros after the last column, whatever the memory
    between rows holds (rows as far apart as the widened ones are, among others).  The bytes after the last
    row, which are not the operand's, are inside a larger allocation here."""
    rows, groups, n = 150, 2, 24
    g = gen(k)
    base = torch.full((rows * stride + 4096,), 5, dtype=torch.int8, device="cuda")
    xq = torch.as_strided(base, (rows, k), (stride, 1))
    xq.copy_(torch.randint(-127, 128, (rows, k), device="cuda", generator=g, dtype=torch.int8))
    held = -(-k // 16) * 16
    wq = torch.zeros(groups, n, held, dtype=torch.int8, device="cuda")[..., :k]
    wq.copy_(torch.randint(-127, 128, wq.shape, device="cuda", generator=g, dtype=torch.int8))
    xs, ws, off = torch.ones(rows, device="cuda"), torch.ones(groups, n, device="cuda"), offsets_of([90, 60])
    out = torch.empty(rows, n, device="cuda")
    p = N.gnmr_product(op=N.GNMR_PRODUCT_FORWARD_I8, groups=groups, rows=rows, n_out=n, n_in=k, out_dtype=N.GNMR_DTYPE_F32,
                       d_offsets=off.data_ptr(), d_x=xq.data_ptr(), x_stride=stride, d_w=wq.data_ptr(), w_stride=held,
                       w_group_stride=n * held, d_x_scale=xs.data_ptr(), d_w_scale=ws.data_ptr(), d_out=out.data_ptr(),
                       out_stride=n)
    wide = -(-k // 64) * 64
    need = N.gnmr_products_scratch_bytes(p)
    assert need >= rows * wide * 2
    scratch = torch.full((need,), 77, dtype=torch.uint8, device="cuda")
    p.d_scratch, p.scratch_bytes = scratch.data_ptr(), need
    N.gnmr_products_run(products._h, p, torch.cuda.current_stream().cuda_stream)
    held16 = scratch[need - -(-rows * wide * 2 // 256) * 256:].view(torch.float16)[:rows * wide].view(rows, wide)
    assert torch.equal(held16[:, :k].char(), xq) and not held16[:, k:].any()
    for e, at in spans([90, 60]):
        assert torch.equal(out[at].double(), xq[at].double() @ wq[e].double().T)


def test_column_codes_of_clusters_whose_ctas_end_at_different_times(products):
    """Rows that leave a cluster's last CTA a single row, so that it is through while others still read
    its maxima: codes and scales of every column, and the same ones in every one of many calls."""
    for rows, cols in ((769, 200), (8 * 128 + 1, 64), (3 * 128 * 7 + 1, 136)):
        x = normal(gen(rows), 3, rows, cols, dtype=torch.bfloat16, size=3.0)
        x[:, rows - 1] *= 64                                     # the maxima lie in the last CTA's row
        q, s = products.quantize_columns(x)
        wq, ws = codes_oracle(x.transpose(1, 2))
        assert np.array_equal(q.cpu().numpy(), wq) and np.array_equal(s.cpu().numpy(), ws)
        for q2, s2 in [products.quantize_columns(x) for _ in range(50)]:
            assert torch.equal(q, q2) and torch.equal(s, s2)
