"""Expert products over several hundred tiles of many stages each, so that every pair of SMs takes
several tiles, of different groups: the rings of operands, the halves of tensor memory and the stages that
rows end in carry over from one to the next.  Every output is compared; tolerances are those of
test_gpu_products."""
import pytest

from paper_2606_00539_gb300 import ExpertProducts

pytestmark = pytest.mark.gpu

import torch  # noqa: E402

from .test_gpu_products import ROUND, TYPES, check, gen, normal, offsets_of, spans  # noqa: E402


@pytest.fixture(scope="module")
def products():
    p = ExpertProducts(device=0)
    yield p
    p.close()


# rows: whole stages of 64, some left over, one, none, more than one piece
UNEVEN = [640, 1, 0, 1027, 320, 63, 65, 64, 0, 1600, 17, 129, 2050, 33]


@pytest.mark.parametrize("n,k", [(1024, 1544), (1003, 1371), (1472, 1032)])
@pytest.mark.parametrize("kind,add", [("f32", False), ("f32", True), ("bf16", False), ("bf16", True)])
def test_weight_grad(products, n, k, kind, add):
    g, t, G, R = gen(n + k), torch.bfloat16, len(UNEVEN), sum(UNEVEN)
    x, dy, off = normal(g, R, k, dtype=t), normal(g, R, n, dtype=t), offsets_of(UNEVEN)
    old = normal(g, G, n, k, dtype=TYPES[kind])
    got = products.weight_grad(dy, x, off, out=old.clone(), add=add)
    for e, at in spans(UNEVEN):
        X, D = x[at].double(), dy[at].double()
        before = old[e].double() if add else torch.zeros((), dtype=torch.float64, device="cuda")
        check(got[e], D.T @ X + before, D.abs().T @ X.abs() + before.abs(), UNEVEN[e], kind)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,k", [(704, 1100), (1003, 1371), (2056, 520)])
def test_forward_and_input_grad(products, n, k, dtype):
    counts = [3 * c for c in UNEVEN]
    g, t, R = gen(n - k + 5000), TYPES[dtype], sum(counts)
    x, dy, off = normal(g, R, k, dtype=t), normal(g, R, n, dtype=t), offsets_of(counts)
    w = normal(g, len(counts), n, k, dtype=t, size=k ** -0.5)
    y, dx = products.forward(x, w, off), products.input_grad(dy, w, off)
    for e, at in spans(counts):
        X, D, W = x[at].double(), dy[at].double(), w[e].double()
        check(y[at], X @ W.T, X.abs() @ W.abs().T, k, dtype)
        check(dx[at], D @ W, D.abs() @ W.abs(), n, dtype)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("n,k", [(1024, 1544), (1003, 1371), (700, 4000)])
def test_forward_i8(products, n, k, out):
    """Rows widened before the product, and scales that differ from row to row and channel to channel."""
    g, G, R = gen(n * k), len(UNEVEN), sum(UNEVEN)
    held = -(-k // 16) * 16
    xq = torch.randint(-128, 128, (R, held), device="cuda", generator=g, dtype=torch.int8)[:, :k]
    wq = torch.randint(-128, 128, (G, n, held), device="cuda", generator=g, dtype=torch.int8)[..., :k]
    xs, ws = torch.rand(R, device="cuda", generator=g) * 1e-2, torch.rand(G, n, device="cuda", generator=g) * 1e-2
    y = products.forward_i8(xq, xs, wq, ws, offsets_of(UNEVEN), out_dtype=out)
    for e, at in spans(UNEVEN):
        want = (xq[at].double() @ wq[e].double().T) * xs[at].double()[:, None] * ws[e].double()
        assert ((y[at].double() - want).abs() <= want.abs() * (3 * 2.0 ** -24 + ROUND[out]) * (1 + 2.0 ** -8)).all()


def test_skewed_groups(products):
    """An average of few rows to a group, nearly all of them one group's: the narrow tiles, many times over."""
    counts = [1] * 30 + [1800, 0] + [2] * 32
    n, k, g, t = 520, 904, gen(77), torch.bfloat16
    x, w, off = normal(g, sum(counts), k, dtype=t), normal(g, 64, n, k, dtype=t, size=k ** -0.5), offsets_of(counts)
    y = products.forward(x, w, off)
    (xq, xs), (wq, ws) = products.quantize_rows(x), products.quantize_rows(w)
    low = products.forward_i8(xq, xs, wq, ws, off, out_dtype="f32")
    for e, at in spans(counts):
        X, W = x[at].double(), w[e].double()
        check(y[at], X @ W.T, X.abs() @ W.abs().T, k, "bf16")
        want = (xq[at].double() @ wq[e].double().T) * xs[at].double()[:, None] * ws[e].double()
        assert ((low[at].double() - want).abs() <= want.abs() * 2.0 ** -21).all()
