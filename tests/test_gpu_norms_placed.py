"""Layer norm of batches inside other memory: rows among wider ones, outputs over the inputs, parameters and their gradients at any element
of an arena, with values around all of them that have to stay.  Sizes of each way that rows are held: by a warp, by
several, by pairs of elements, by a CTA, and read several times.  Tolerances: those of the same rows in memory of their own."""
import pytest

from paper_2606_00539_gb300 import LayerNorm

pytestmark = pytest.mark.gpu

import torch  # noqa: E402

from tests.test_gpu_norms import check_backward, check_forward  # noqa: E402
from tests.test_gpu_products import TYPES, gen, normal  # noqa: E402


@pytest.fixture(scope="module")
def norms():
    return LayerNorm(device=0)


class Placed:
    """A matrix, or a vector, in a buffer of values of its own: `view` may be written, what is around it not."""

    def __init__(self, g, rows, cols, lead, pad, kind, offset=0.0):
        self.lead, self.cols = lead, cols
        self.buffer = (normal(g, rows, lead + cols + pad, dtype=torch.float32) + offset).to(TYPES[kind])
        self.view = self.buffer[:, lead:lead + cols]
        self.was = self.buffer.clone()

    @property
    def old(self):
        return self.was[:, self.lead:self.lead + self.cols]

    def around_is_left(self):
        b, w, end = self.buffer, self.was, self.lead + self.cols
        return torch.equal(b[:, :self.lead], w[:, :self.lead]) and torch.equal(b[:, end:], w[:, end:])

    def again(self):
        self.buffer.copy_(self.was)
        return self.view


# rows, cols; elements before and behind a row of x, dy and the outputs; before the parameters
PLACES = [
    (1501, 512, (0, 0), (0, 0), (0, 0), 0), (1501, 520, (8, 8), (16, 0), (8, 24), 3), (1501, 1000, (0, 8), (8, 0), (24, 0), 1),
    (1501, 2048, (16, 0), (0, 16), (8, 8), 5), (1501, 2056, (8, 0), (0, 0), (0, 8), 1), (1501, 5120, (8, 8), (0, 64), (64, 0), 3),
    (1501, 5120, (0, 0), (0, 0), (0, 0), 0), (701, 8192, (8, 8), (16, 16), (0, 8), 7),
    # odd starts: by pairs where x, dy and the outputs are odd and even together, though not at one offset; else by elements
    (1501, 1371, (0, 0), (0, 0), (0, 0), 0), (1501, 1371, (1, 0), (3, 2), (5, 4), 1), (1501, 1371, (2, 3), (4, 1), (0, 1), 2),
    (1501, 1371, (1, 1), (3, 3), (1, 5), 3), (1501, 1371, (0, 1), (1, 2), (0, 3), 1), (1501, 520, (1, 0), (1, 2), (3, 0), 3),
    (1501, 5120, (1, 1), (3, 1), (1, 1), 1), (901, 5121, (0, 0), (2, 0), (4, 2), 2), (501, 12285, (1, 1), (1, 1), (3, 1), 1),
    (501, 64, (1, 0), (1, 0), (1, 0), 1), (501, 2, (0, 1), (2, 1), (0, 1), 1), (501, 1, (0, 0), (0, 0), (0, 0), 0), (501, 1, (1, 1), (3, 1), (1, 3), 0),
    # wide rows
    (301, 16384, (8, 8), (0, 24), (8, 0), 1), (301, 16384, (0, 0), (0, 0), (0, 0), 0), (201, 20001, (0, 0), (0, 0), (0, 0), 0),
    (201, 20001, (1, 2), (3, 2), (5, 0), 3), (101, 32776, (8, 0), (0, 8), (0, 0), 1),
]


@pytest.mark.parametrize("dtype,params", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("place", range(len(PLACES)))
def test_batches_among_other_values(norms, place, dtype, params):
    rows, cols, of_x, of_dy, of_out, lead = PLACES[place]
    g = gen(place)
    x, dy, out = Placed(g, rows, cols, *of_x, dtype, 0.5), Placed(g, rows, cols, *of_dy, dtype), Placed(g, rows, cols, *of_out, dtype)
    arena = Placed(g, 1, 2 * cols + 3, lead, 5, params)
    w, b = arena.view[0, :cols], arena.view[0, cols + 3:]

    y, mean, rstd = norms.forward(x.view, w, b, out=out.view)
    check_forward(y, mean, rstd, x.view, w, b, 1e-5, dtype)
    assert out.around_is_left() and torch.equal(x.buffer, x.was) and torch.equal(arena.buffer, arena.was)
    again = norms.forward(x.view, w, b, out=x.view)                              # in place
    assert again[0] is x.view
    check_forward(*again, x.old, w, b, 1e-5, dtype)
    assert x.around_is_left()
    x.again()

    grads = Placed(g, 1, 2 * cols + 3, lead, 5, "f32")
    dw, db = grads.view[0, :cols], grads.view[0, cols + 3:]
    dx = norms.backward(dy.view, x.view, w, mean, rstd, out=out.again(), weight_grad=dw, bias_grad=db)
    check_backward(dx, dw, db, dy.view, x.view, w, mean, rstd, dtype, "f32")
    assert out.around_is_left() and torch.equal(x.buffer, x.was) and torch.equal(dy.buffer, dy.was) and torch.equal(arena.buffer, arena.was)
    assert grads.around_is_left() and torch.equal(grads.view[0, cols:cols + 3], grads.old[0, cols:cols + 3])
    grads.again()
    dx = norms.backward(dy.view, x.view, w, mean, rstd, out=dy.view, weight_grad=dw, bias_grad=db, add=True)     # over dy
    assert dx is dy.view
    check_backward(dx, dw, db, dy.old, x.view, w, mean, rstd, dtype, "f32", (grads.old[0, :cols].double(), grads.old[0, cols + 3:].double()))
    assert dy.around_is_left() and torch.equal(x.buffer, x.was) and grads.around_is_left()
    dx = norms.backward(dy.again(), x.view, w, mean, rstd, out=dy.view)                                          # and that alone
    check_backward(dx, None, None, dy.old, x.view, w, mean, rstd, dtype, "f32")
    assert dy.around_is_left() and torch.equal(x.buffer, x.was)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [1371, 5120])
def test_one_row_of_any_stride_in_place(norms, cols, dtype):
    g = gen(cols)
    rows = normal(g, 4, cols, dtype=TYPES[dtype])
    old, dy = rows.clone(), normal(g, 4, cols, dtype=TYPES[dtype])
    check_forward(*norms.forward(rows[::2][:1], out=rows[:1]), old[:1], None, None, 1e-5, dtype)
    assert torch.equal(rows[1:], old[1:])
    _, mean, rstd = norms.forward(old[:1])
    was = dy.clone()
    check_backward(norms.backward(dy[::2][:1], old[::3][:1], None, mean, rstd, out=dy[:1]), None, None, was[:1], old[:1], None, mean, rstd, dtype, "f32")
    assert torch.equal(dy[1:], was[1:])
