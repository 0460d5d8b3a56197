"""The gated blocks, the layer norm and the clipping without a GPU: the C layout of the argument structs, the
argument checks, which come before any CUDA call, and the layers' autograd over torch's own arithmetic."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2606_00539_gb300 import GnmrError, expert_gated, layer_norm
from paper_2606_00539_gb300 import _native as N
from paper_2606_00539_gb300 import build as native_build
from paper_2606_00539_gb300 import norms as norms_module
from paper_2606_00539_gb300 import products as module

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, LAYOUT = N.GNMR_ERR_INVALID_ARG, N.GNMR_ERR_LAYOUT


@pytest.fixture(scope="module", autouse=True)
def lib():
    native_build.build()
    if module.torch is None:
        module._load_torch()
    norms_module.torch = torch
    return N.load()


@pytest.mark.parametrize("struct", [N.gnmr_gated, N.gnmr_norm])
def test_struct_layout_matches_c(tmp_path, struct):
    name, fields = struct.__name__, [f for f, _ in struct._fields_]
    prints = "\n".join(f'printf("{f} %zu\\n", offsetof({name}, {f}));' for f in fields)
    src, exe = tmp_path / "probe.c", tmp_path / "probe"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "gnmr.h"\nint main(void) {\n'
                   f'printf("sizeof %zu\\n", sizeof({name}));\n{prints}\nreturn 0; }}\n')
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    said = dict(line.split() for line in subprocess.check_output([str(exe)], text=True).splitlines())
    assert int(said["sizeof"]) == ctypes.sizeof(struct)
    for f in fields:
        assert int(said[f]) == getattr(struct, f).offset, f


def gated(**over):
    """Arguments that pass the checks; nothing here is dereferenced."""
    p = N.gnmr_gated()
    kw = dict(groups=2, rows=10, n=8, n_in=8, dtype=N.GNMR_DTYPE_BF16, d_offsets=4096, d_x=4096, x_stride=8, d_w=4096, w_stride=8,
              w_group_stride=128, d_out=4096, out_stride=8, d_keep=4096, keep_stride=16)
    kw.update(over)
    for key, v in kw.items():
        setattr(p, key, v)
    return p


def test_gated_scratch():
    """Nothing for operands read in place; an odd start, row or group stride copies that operand, in whole 256 bytes."""
    assert N.gnmr_gated_scratch_bytes(gated()) == 0
    assert N.gnmr_gated_scratch_bytes(gated(d_keep=None, keep_stride=0, out_stride=9, d_out=4098)) == 0
    assert N.gnmr_gated_scratch_bytes(gated(d_x=4098)) == 256                       # 10 x 8
    assert N.gnmr_gated_scratch_bytes(gated(n_in=9, x_stride=9, w_stride=16, w_group_stride=256)) == 512       # 10 x 16
    assert N.gnmr_gated_scratch_bytes(gated(w_group_stride=129)) == 512             # 2 x 16 x 8


@pytest.mark.parametrize("status,over", [
    (INVALID, dict(activation=2)), (INVALID, dict(activation=-1)), (INVALID, dict(groups=0)), (INVALID, dict(groups=2049)),
    (INVALID, dict(rows=-1)), (INVALID, dict(rows=1 << 30)), (INVALID, dict(n=0)), (INVALID, dict(n=1 << 30)), (INVALID, dict(n_in=0)),
    (INVALID, dict(dtype=N.GNMR_DTYPE_F32)), (INVALID, dict(d_offsets=None)), (INVALID, dict(d_x=None)), (INVALID, dict(d_w=None)),
    (INVALID, dict(d_out=None)), (LAYOUT, dict(x_stride=7)), (LAYOUT, dict(w_stride=7)), (LAYOUT, dict(w_group_stride=-1)),
    (LAYOUT, dict(out_stride=7)), (LAYOUT, dict(keep_stride=15)), (LAYOUT, dict(d_x=4097)), (LAYOUT, dict(d_keep=4097)),
    (LAYOUT, dict(d_out=4097)), (LAYOUT, dict(out_stride=1 << 37)), (LAYOUT, dict(keep_stride=1 << 37)), (LAYOUT, dict(d_offsets=4100)),
    (LAYOUT, dict(d_mask=4096, mask_stride=0)),
])
def test_gated_refusals(lib, status, over):
    with pytest.raises(GnmrError) as e:
        N.gnmr_gated_scratch_bytes(gated(**over))
    assert e.value.status == status
    assert lib.gnmr_products_gated(None, ctypes.addressof(gated(**over)), None) == INVALID
    assert lib.gnmr_gated_scratch_bytes(None, None) == INVALID


GATE = dict(gu=4096, dtype=N.GNMR_DTYPE_BF16, act=0, groups=2, rows=10, n=8, gu_stride=16, offsets=4096, mask=None, mask_stride=1,
            h=8192, h_stride=8, stream=None)
GRAD = dict(dh=4096, dtype=N.GNMR_DTYPE_BF16, act=0, rows=10, n=8, dh_stride=8, gu=4096, gu_stride=16, dgu=8192, dgu_stride=16, stream=None)


@pytest.mark.parametrize("status,over", [
    (INVALID, dict(dtype=0)), (INVALID, dict(act=2)), (INVALID, dict(groups=0)), (INVALID, dict(groups=2049)), (INVALID, dict(rows=-1)),
    (INVALID, dict(n=0)), (INVALID, dict(offsets=None)), (INVALID, dict(gu=None)), (INVALID, dict(h=None)), (LAYOUT, dict(gu_stride=15)),
    (LAYOUT, dict(h_stride=7)), (LAYOUT, dict(gu=4097)), (LAYOUT, dict(h=4097)), (LAYOUT, dict(offsets=4100)),
    (LAYOUT, dict(mask=4096, mask_stride=0)), (LAYOUT, dict(gu_stride=1 << 32)), (N.GNMR_OK, dict(rows=0)),
])
def test_gate_refusals(lib, status, over):
    assert lib.gnmr_gate(*{**GATE, **over}.values()) == status


@pytest.mark.parametrize("status,over", [
    (INVALID, dict(dtype=0)), (INVALID, dict(act=-1)), (INVALID, dict(rows=-1)), (INVALID, dict(n=0)), (INVALID, dict(dh=None)),
    (INVALID, dict(gu=None)), (INVALID, dict(dgu=None)), (LAYOUT, dict(dh_stride=7)), (LAYOUT, dict(gu_stride=15)), (LAYOUT, dict(dgu_stride=15)),
    (LAYOUT, dict(dh=4097)), (LAYOUT, dict(dgu=4096, dgu_stride=24)), (N.GNMR_OK, dict(rows=0)),
])
def test_gate_grad_refusals(lib, status, over):
    assert lib.gnmr_gate_grad(*{**GRAD, **over}.values()) == status


def norm(**over):
    p = N.gnmr_norm()
    kw = dict(rows=4, cols=8, dtype=N.GNMR_DTYPE_BF16, param_dtype=N.GNMR_DTYPE_F32, eps=1e-5, d_x=4096, x_stride=8, d_weight=4096, d_bias=4096,
              d_mean=4096, d_rstd=4096, d_y=8192, y_stride=8, d_dy=12288, dy_stride=8, d_dx=8192, dx_stride=8, d_dweight=4096, d_dbias=4096,
              grad_dtype=N.GNMR_DTYPE_F32, d_scratch=4096, scratch_bytes=1 << 30)
    kw.update(over)
    for key, v in kw.items():
        setattr(p, key, v)
    return p


BOTH = [(INVALID, dict(dtype=3)), (INVALID, dict(param_dtype=N.GNMR_DTYPE_F16)), (INVALID, dict(rows=-1)), (INVALID, dict(rows=1 << 31)),
        (INVALID, dict(cols=0)), (INVALID, dict(cols=(1 << 30) + 1)), (INVALID, dict(d_x=None)), (LAYOUT, dict(x_stride=7)),
        (LAYOUT, dict(x_stride=1 << 32)), (LAYOUT, dict(d_x=4097)), (LAYOUT, dict(d_weight=4098)), (LAYOUT, dict(d_mean=4098))]


@pytest.mark.parametrize("status,over", BOTH + [
    (INVALID, dict(eps=-1.0)), (INVALID, dict(eps=float("nan"))), (INVALID, dict(eps=float("inf"))), (INVALID, dict(d_y=None)),
    (LAYOUT, dict(y_stride=7)), (LAYOUT, dict(d_y=8193)), (LAYOUT, dict(d_bias=4098)), (LAYOUT, dict(d_y=4096, y_stride=16)),
    (N.GNMR_OK, dict(rows=0, d_x=None, d_y=None))])
def test_layer_norm_refusals(lib, status, over):
    assert lib.gnmr_layer_norm(ctypes.addressof(norm(**over)), None) == status
    assert lib.gnmr_layer_norm(None, None) == INVALID


@pytest.mark.parametrize("status,over", BOTH + [
    (INVALID, dict(grad_dtype=5)), (INVALID, dict(d_dy=None)), (INVALID, dict(d_mean=None)), (INVALID, dict(d_rstd=None)),
    (LAYOUT, dict(dy_stride=7)), (LAYOUT, dict(dx_stride=7)), (LAYOUT, dict(d_dy=4097)), (LAYOUT, dict(d_dx=4097)),
    (LAYOUT, dict(d_dweight=4098)), (LAYOUT, dict(d_scratch=None)), (LAYOUT, dict(d_scratch=4100)), (LAYOUT, dict(scratch_bytes=0)),
    (LAYOUT, dict(d_dx=12288, dx_stride=16))])
def test_layer_norm_grad_refusals(lib, status, over):
    assert lib.gnmr_layer_norm_grad(ctypes.addressof(norm(**over)), None) == status


def test_layer_norm_scratch(lib):
    assert N.gnmr_layer_norm_scratch_bytes(norm(d_dweight=None, d_dbias=None)) == 0
    assert N.gnmr_layer_norm_scratch_bytes(norm()) > 0
    assert lib.gnmr_layer_norm_scratch_bytes(None, None) == INVALID


def test_clip_refusals(lib):
    lengths, dtypes = (ctypes.c_int64 * 2)(5, 6), (ctypes.c_int32 * 2)(0, 1)
    out = ctypes.c_void_p()
    make = lib.gnmr_clip_create
    assert make(2, lengths, dtypes, 0, None) == INVALID
    assert make(-1, lengths, dtypes, 0, ctypes.byref(out)) == INVALID
    assert make(2, None, dtypes, 0, ctypes.byref(out)) == INVALID
    assert make(2, lengths, None, 0, ctypes.byref(out)) == INVALID
    assert make(2, (ctypes.c_int64 * 2)(5, -6), dtypes, 0, ctypes.byref(out)) == INVALID
    assert make(2, (ctypes.c_int64 * 2)(5, 1 << 62), dtypes, 0, ctypes.byref(out)) == INVALID
    assert make(2, lengths, (ctypes.c_int32 * 2)(0, 3), 0, ctypes.byref(out)) == INVALID
    assert out.value is None
    if not torch.cuda.is_available():
        assert make(2, lengths, dtypes, 0, ctypes.byref(out)) == N.GNMR_ERR_CUDA
    assert lib.gnmr_clip_run(None, 4096, None, None, 1.0, None, 0, 4096, 4096, 1 << 20, None) == INVALID
    assert lib.gnmr_clip_scratch_bytes(None, None) == lib.gnmr_clip_table_bytes(None, None) == lib.gnmr_clip_write_table(None, None) == INVALID
    assert lib.gnmr_clip_destroy(None) == N.GNMR_OK


# -- the layers' autograd ---------------------------------------------------------

class Products:
    """One group, 64 bits, silu."""

    def gated(self, x, w, offsets=None, *, out, keep=None, mask=None, activation="silu"):
        ab = x.detach() @ w.detach().T
        a, b = ab.chunk(2, 1)
        out.copy_(a * torch.sigmoid(a) * b)
        if keep is not None:
            keep.copy_(ab)

    def gate_grad(self, dh, ab, *, activation="silu"):
        a, b = ab.chunk(2, 1)
        s = torch.sigmoid(a)
        return torch.cat([dh * b * s * (1 + a * (1 - s)), dh * a * s], 1)

    def input_grad(self, dy, w, offsets=None, *, out, mask=None):
        out.copy_(dy.detach() @ w.detach())

    def weight_grad(self, dy, x, offsets=None, *, out, add=False, mask=None):
        dw = dy.detach().T @ x.detach()
        out.copy_(out + dw if add else dw)


class Norms:
    """64 bits."""

    def forward(self, x, weight=None, bias=None, *, eps):
        mean = x.mean(1)
        rstd = (x.var(1, unbiased=False) + eps).rsqrt()
        y = (x - mean[:, None]) * rstd[:, None]
        y = y if weight is None else y * weight
        return (y if bias is None else y + bias), mean, rstd

    def backward(self, dy, x, weight, mean, rstd, *, input_grad, weight_grad, bias_grad, add):
        hat = (x - mean[:, None]) * rstd[:, None]
        for to, v in ((weight_grad, (dy * hat).sum(0)), (bias_grad, dy.sum(0))):
            if to is not None:
                to.copy_(to + v if add else v)
        t = dy if weight is None else dy * weight
        return rstd[:, None] * (t - t.mean(1, keepdim=True) - hat * (t * hat).mean(1, keepdim=True)) if input_grad else None


def tensors(*shapes):
    g = torch.Generator().manual_seed(3)
    return [torch.randn(*s, dtype=torch.float64, generator=g, requires_grad=True) for s in shapes]


def layers():
    x, w = tensors((7, 5), (8, 5))
    yield (lambda x, w, **kw: expert_gated(Products(), x, w, **kw),
           lambda x, w: torch.nn.functional.silu((x @ w.T)[:, :4]) * (x @ w.T)[:, 4:], x, w)
    x, w = tensors((7, 6), (6,))
    yield (lambda x, w, grad=None, **kw: layer_norm(Norms(), x, w, None, None if grad is None else (grad, None), **kw),
           lambda x, w: torch.nn.functional.layer_norm(x, (6,), w), x, w)


@pytest.mark.parametrize("which", [0, 1])
def test_first_derivatives_and_no_second(which):
    mine, theirs, x, w = list(layers())[which]
    for inputs in ((x, w), (x,), (w,)):
        got, want = (torch.autograd.grad((f(x, w) ** 3).sum(), inputs) for f in (mine, theirs))
        assert all(torch.allclose(a, b) for a, b in zip(got, want))
    assert torch.autograd.gradcheck(mine, (x, w))
    g, = torch.autograd.grad((mine(x, w) ** 2).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivatives"):
        (g ** 2).sum().backward()
    with torch.no_grad():
        assert not mine(x, w).requires_grad


@pytest.mark.parametrize("which", [0, 1])
def test_the_arena_is_written_and_added_to(which):
    mine, theirs, x, w = list(layers())[which]
    arena = torch.full_like(w, 7.0).detach()
    (mine(x.detach(), w.detach(), grad=arena) ** 2).sum().backward()
    want = torch.autograd.grad((theirs(x, w) ** 2).sum(), w)[0]
    assert torch.allclose(arena, want)
    ((mine(x, w, grad=arena, add=True) ** 2).sum() + (mine(x, w, grad=arena, add=True) ** 2).sum()).backward()
    assert torch.allclose(arena, 3 * want) and w.grad is None and x.grad is not None
    with torch.no_grad():
        assert not mine(x.detach(), w.detach(), grad=arena).requires_grad
    assert not mine(x.detach(), w.detach()).requires_grad


def test_layer_norm_of_more_dimensions():
    x, w, b = tensors((2, 3, 4, 5), (5,), (5,))
    got = torch.autograd.grad((layer_norm(Norms(), x, w, b) ** 3).sum(), (x, w, b))
    want = torch.autograd.grad((torch.nn.functional.layer_norm(x, (5,), w, b) ** 3).sum(), (x, w, b))
    assert all(a.shape == z.shape and torch.allclose(a, z) for a, z in zip(got, want))
    v, = tensors((5,))
    assert layer_norm(Norms(), v, w, b).shape == (5,)


def test_gradients_that_do_not_lie_in_order():
    """dh and dy as autograd hands them out after a transpose or an expanded sum."""
    mine, theirs, x, w = list(layers())[0]
    got, want = (torch.autograd.grad((f(x, w).T.contiguous() ** 2).T.sum() + f(x, w).sum(), x)[0] for f in (mine, theirs))
    assert torch.allclose(got, want)
