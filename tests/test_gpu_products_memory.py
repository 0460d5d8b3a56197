"""Expert products: repeated calls, sums that several SMs share, and the memory that a call
may touch.  Tolerances are those of test_gpu_products."""
import numpy as np
import pytest

from paper_2606_00539_gb300 import ExpertProducts, GnmrError, expert_linear
from paper_2606_00539_gb300 import _native as N

pytestmark = pytest.mark.gpu

import torch  # noqa: E402

from .test_gpu_products import TYPES, check, codes_oracle, gen, normal, offsets_of, spans  # noqa: E402


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


def test_cleared_tails_of_both_ctas_reach_the_multiplies(products):
    """Groups of rows that end inside a stage, infinities in the rows after them, over hundreds of tiles:
    both CTAs of a pair clear their half of such a stage, and the first one's multiplies read both."""
    counts = [70, 1, 131, 64, 193, 5, 0, 257, 63, 65, 130, 17]
    g, t, G, R, n, k = gen(21), torch.bfloat16, 12, sum(counts), 1000, 1544
    x, dy = normal(g, R, k, dtype=t), normal(g, R, n, dtype=t)
    off = offsets_of(counts)
    want = {e: (dy[at].double().T @ x[at].double(), dy[at].double().abs().T @ x[at].double().abs()) for e, at in spans(counts)}
    for odd in (0, 1):                                           # every other group's rows, in turn, are infinities
        x2, dy2 = x.clone(), dy.clone()
        for e, at in spans(counts):
            if e % 2 == odd:
                x2[at], dy2[at] = float("inf"), float("-inf")
        first = products.weight_grad(dy2, x2, off, out=torch.empty(G, n, k, device="cuda"))
        for e, at in spans(counts):
            if e % 2 != odd:
                check(first[e], *want[e], counts[e], "f32")
        for _ in range(20):
            again = products.weight_grad(dy2, x2, off, out=torch.empty(G, n, k, device="cuda"))
            assert torch.equal(torch.nan_to_num(again), torch.nan_to_num(first))


@pytest.mark.parametrize("counts,n,k", [([3, 1, 40, 0, 7, 16, 2, 33, 1, 5, 12, 31, 9, 4, 1, 30], 2000, 1400),
                                        ([1], 30000, 1500), ([90], 1100, 3000), ([1] * 700, 300, 136)])
def test_few_rows_of_codes_over_many_tiles(products, counts, n, k):
    """Rows that are widened on the SM, over more tiles than there are SMs: every output."""
    g, G, R = gen(n), len(counts), sum(counts)
    held = -(-k // 16) * 16
    xq = torch.randint(-128, 128, (R, held), device="cuda", generator=g, dtype=torch.int8)[:, :k]
    wq = torch.randint(-128, 128, (G, n, held), device="cuda", generator=g, dtype=torch.int8)[..., :k]
    off, xs, ws = offsets_of(counts), torch.ones(R, device="cuda"), torch.ones(G, n, device="cuda")
    for _ in range(5):
        y = products.forward_i8(xq, xs, wq, ws, off, out_dtype="f32")
        for e, at in spans(counts):
            assert torch.equal(y[at], (xq[at].double() @ wq[e].double().T).float())


CALLS = {                                                        # each kernel; rows that end inside a stage among them
    "few rows": lambda p, a: p.forward(a["x"][:9], a["w"], a["few"]),
    "many rows": lambda p, a: p.forward(a["x"], a["w"], a["off"]),
    "input gradient": lambda p, a: p.input_grad(a["dy"], a["w"], a["off"]),
    "weight gradient": lambda p, a: p.weight_grad(a["dy"], a["x"], a["off"], out=torch.empty(4, 700, 1100, device="cuda")),
    "few codes": lambda p, a: p.forward_i8(a["xq"][:9], a["xs"][:9], a["wq"], a["ws"], a["few"]),
    "many codes": lambda p, a: p.forward_i8(a["xq"], a["xs"], a["wq"], a["ws"], a["off"]),
}


@pytest.mark.parametrize("name", CALLS)
def test_a_wait_that_runs_out_ends_the_product_and_is_reported(name):
    """With no time at all nothing is loaded, so that every role waits for what never comes, and gives up.  The kernel ends, the
    handle says so and takes no more products, and another handle, on the same context, is not affected."""
    g, t = gen(31), torch.bfloat16
    a = dict(x=normal(g, 900, 1100, dtype=t), dy=normal(g, 900, 700, dtype=t), w=normal(g, 4, 700, 1100, dtype=t),
             off=offsets_of([300, 299, 1, 300]), few=offsets_of([3, 0, 5, 1]))
    with ExpertProducts(device=0) as fine:
        a["xq"], a["xs"] = fine.quantize_rows(a["x"])
        a["wq"], a["ws"] = fine.quantize_rows(a["w"])
        want = CALLS[name](fine, a)
        fine.check()
        p = ExpertProducts(device=0)
        N.gnmr_products_set_wait_limit(p._h, 0)
        CALLS[name](p, a)
        torch.cuda.synchronize()
        for call in (p.check, lambda: CALLS[name](p, a), p.close):
            with pytest.raises(GnmrError) as e:
                call()
            assert e.value.status == N.GNMR_ERR_STATE and "gave up" in e.value.detail
        p.close()
        assert torch.equal(CALLS[name](fine, a), want)
        N.gnmr_products_set_wait_limit(fine._h, 10 ** 9)
        assert torch.equal(CALLS[name](fine, a), want)
        torch.cuda.synchronize()
        fine.check()


def test_expert_linear_adds_micro_batches_to_the_arena(products):
    """Two micro-batches and a weight used twice, into an fp32 arena, with nothing that requires a gradient."""
    counts, n, k, g, t = [40, 0, 30], 72, 136, gen(33), torch.bfloat16
    off, R = offsets_of(counts), 70
    w = normal(g, 3, n, k, dtype=t, size=0.1)
    arena = torch.zeros(3, n, k, device="cuda")
    want, size = (torch.zeros(3, n, k, dtype=torch.float64, device="cuda") for _ in range(2))
    for _ in range(2):
        xs, dys = [normal(g, R, k, dtype=t) for _ in range(2)], [normal(g, R, n, dtype=t) for _ in range(2)]
        ys = [expert_linear(products, x, w, off, None, arena, add=True) for x in xs]
        torch.autograd.backward(ys, dys)
        for x, dy in zip(xs, dys):
            for e, at in spans(counts):
                want[e] += dy[at].double().T @ x[at].double()
                size[e] += dy[at].double().abs().T @ x[at].double().abs()
    check(arena, want, 4 * size, 40, "f32")                      # four sums, each added with a rounding of its own


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_gradients_of_groups_side_by_side(products, kind):
    """Row n of every group's gradient beside the others': [n_out, groups, n_in] in memory."""
    counts, n, k, g, t = [70, 0, 33], 136, 72, gen(35), torch.bfloat16
    x, dy, off = normal(g, 103, k, dtype=t), normal(g, 103, n, dtype=t), offsets_of(counts)
    held = normal(g, n, 3, k, dtype=TYPES[kind])
    old = held.clone()
    products.weight_grad(dy, x, off, out=held.transpose(0, 1), add=True)
    for e, at in spans(counts):
        X, D, before = x[at].double(), dy[at].double(), old[:, e].double()
        check(held[:, e], D.T @ X + before, D.abs().T @ X.abs() + before.abs(), counts[e], kind)
