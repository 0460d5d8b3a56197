"""expert_linear's autograd without a GPU: the products are torch's, written into `out` as the
kernels do, so that autograd sees nothing of them."""
import pytest
import torch

from paper_2606_00539_gb300 import expert_linear, products as module


class Products:
    """One group, 64 bits."""

    def forward(self, x, w, offsets=None, *, out, mask=None):
        out.copy_(x.detach() @ w.detach().T)

    def input_grad(self, dy, w, offsets=None, *, out, mask=None):
        out.copy_(dy.detach() @ w.detach())

    def weight_grad(self, dy, x, offsets=None, *, out, add=False, mask=None):
        dw = dy.detach().T @ x.detach()
        out.copy_(out + dw if add else dw)


@pytest.fixture(autouse=True)
def loaded():
    if module.torch is None:
        module._load_torch()


def tensors(x_grad=True, w_grad=True):
    g = torch.Generator().manual_seed(3)
    x = torch.randn(7, 5, dtype=torch.float64, generator=g, requires_grad=x_grad)
    w = torch.randn(4, 5, dtype=torch.float64, generator=g, requires_grad=w_grad)
    return x, w


def test_first_derivatives():
    x, w = tensors()
    got = torch.autograd.grad((expert_linear(Products(), x, w) ** 3).sum(), (x, w))
    want = torch.autograd.grad(((x @ w.T) ** 3).sum(), (x, w))
    assert all(torch.allclose(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("cube", [True, False])
def test_second_derivatives_are_refused(cube):
    """A loss that contains the gradient: of a cube, whose gradient depends on y, and of a sum, whose
    gradient depends on the weights alone.  The values are right; passing them back is an error."""
    x, w = tensors()
    y = expert_linear(Products(), x, w)
    g, = torch.autograd.grad((y ** 3 if cube else y).sum(), x, create_graph=True)
    z = x @ w.T
    want, = torch.autograd.grad((z ** 3 if cube else z).sum(), x)
    assert torch.allclose(g, want)
    with pytest.raises(RuntimeError, match="second derivatives"):
        ((y ** 2).sum() + (g ** 2).sum()).backward()


def test_the_arena_is_written_when_nothing_else_requires_a_gradient():
    x, w = tensors(x_grad=False, w_grad=False)
    arena = torch.full((4, 5), 7.0, dtype=torch.float64)
    (expert_linear(Products(), x, w, grad=arena) ** 2).sum().backward()
    assert torch.allclose(arena, 2 * (x @ w.T).T @ x)
    with torch.no_grad():
        assert not expert_linear(Products(), x, w, grad=arena).requires_grad
    assert not expert_linear(Products(), x, w).requires_grad


def test_a_shared_weight_and_micro_batches_add_to_the_arena():
    """Two uses of one weight in one graph, then another micro-batch: the sum, as autograd has it."""
    x, w = tensors()
    arena = torch.zeros(4, 5, dtype=torch.float64)
    want = torch.zeros(4, 5, dtype=torch.float64)
    for scale in (1.0, 3.0):
        y = expert_linear(Products(), x, w, grad=arena, add=True)
        ((y ** 2).sum() + (expert_linear(Products(), scale * x, w, grad=arena, add=True) ** 3).sum()).backward()
        z = x @ w.T
        want += torch.autograd.grad((z ** 2).sum() + ((scale * x @ w.T) ** 3).sum(), w)[0]
    assert w.grad is None and torch.allclose(arena, want)
    (expert_linear(Products(), x, w, grad=arena) ** 2).sum().backward()          # without add: written
    assert torch.allclose(arena, torch.autograd.grad(((x @ w.T) ** 2).sum(), w)[0])


@pytest.mark.parametrize("which", [0, 1])
def test_products_refuse_operands_whose_gradient_would_be_lost(which):
    """Before anything is enqueued; not under no_grad, where nothing is lost."""
    p = module.ExpertProducts.__new__(module.ExpertProducts)
    p._h, p.device_index, p._sixteen = None, -1, (torch.bfloat16, torch.float16)      # -1: tensors in host memory
    x, dy, w = (torch.zeros(s, dtype=torch.bfloat16) for s in ((6, 8), (6, 16), (16, 8)))
    out = torch.zeros(16, 8)
    calls = [(lambda: p.forward(x, w, out=dy), (x, w)), (lambda: p.input_grad(dy, w, out=x), (dy, w)),
             (lambda: p.weight_grad(dy, x, out=out), (dy, x))]
    for call, operands in calls:
        operands[which].requires_grad_()
        with pytest.raises(ValueError, match="expert_linear"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="closed"):
            call()
        operands[which].requires_grad_(False)
        with pytest.raises(ValueError, match="closed"):
            call()
