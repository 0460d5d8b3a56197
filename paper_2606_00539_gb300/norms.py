"""torch-facing wrapper of the layer norm: by row, forward and backward, with the reduction of the
parameters' gradients straight into the arena that the monitor reads.  PyTorch supplies device memory and
the stream; every value is computed by libgnmr's kernels."""
from __future__ import annotations

import ctypes

from . import _native as N
from . import products as P

torch = None                                       # loaded with the first LayerNorm
_DTYPES = P._DTYPES


class LayerNorm:
    """Layer norm over the last dimension of matrices on one device:
    y = (x - mean) * rstd * weight + bias, rstd = 1 / sqrt(mean of (x - mean)^2 + eps).

    x: [rows, cols], bf16, f16 or fp32, contiguous rows at any stride; weight, bias: [cols] of x's
    type or fp32 (both of one type), or None.  Statistics are fp32.  stream: a torch stream, default
    the current one; tensors made on another stream are the caller's to order.  An instance holds nothing that a call
    writes: it may be used from several streams at once.

    Autograd records none of these calls (layer_norm is the layer that it knows), so they refuse
    operands that require a gradient while it records."""

    def __init__(self, device=0):
        global torch
        if torch is None:
            if P.torch is None:
                P._load_torch()
            torch = P.torch
        self.device_index = int(device.index if hasattr(device, "index") else device)
        self._lib = N.load()
        self._scratch = {}
        self._device = torch.device("cuda", self.device_index)
        self._types = tuple(_DTYPES)
        self._raw_stream = torch._C._cuda_getCurrentRawStream

    # -- argument checks ------------------------------------------------------
    # A few rows take the GPU 3 us: these checks are written to cost the host little more.
    def _refuse(self, t, name, dims, dtypes):
        if not isinstance(t, torch.Tensor) or t.get_device() != self.device_index:
            raise ValueError(f"{name} must be a CUDA tensor on device {self.device_index}")
        if t.dtype not in dtypes:
            raise ValueError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, got {t.dtype}")
        raise ValueError(f"{name} must have {dims} dimensions, got {t.dim()}")

    def _matrix(self, t, name, shape, dtypes):
        """(rows, columns, row stride) of a matrix of contiguous rows."""
        if not isinstance(t, torch.Tensor) or t.get_device() != self.device_index or t.dtype not in dtypes or t.dim() != 2:
            self._refuse(t, name, 2, dtypes)
        rows, cols = t.shape
        if shape is not None and (rows, cols) != shape:
            raise ValueError(f"{name} must be {list(shape)}, got {[rows, cols]}")
        step, one = t.stride()
        if one != 1 and cols > 1:
            raise ValueError(f"{name} must have contiguous rows")
        return rows, cols, step if rows > 1 else cols    # a single row has no stride, and torch may give it any

    def _vector(self, t, name, n, dtypes):
        if t is None:
            return None
        if not isinstance(t, torch.Tensor) or t.get_device() != self.device_index or t.dtype not in dtypes or t.dim() != 1:
            self._refuse(t, name, 1, dtypes)
        if t.numel() != n or not t.is_contiguous():
            raise ValueError(f"{name} must hold {n} contiguous entries")
        return t.data_ptr()

    def _params(self, weight, bias, dtype, cols):
        """The parameters' type, and where they are."""
        kinds = (dtype, torch.float32)
        w, b = self._vector(weight, "weight", cols, kinds), self._vector(bias, "bias", cols, kinds)
        kind = dtype if weight is None and bias is None else bias.dtype if weight is None else weight.dtype
        if weight is not None and bias is not None and bias.dtype != kind:
            raise ValueError("weight and bias must be of one type")
        return _DTYPES[kind], w, b

    @staticmethod
    def _no_graph(a, b, c):
        if (a.requires_grad or (b is not None and b.requires_grad) or (c is not None and c.requires_grad)) and torch.is_grad_enabled():
            raise ValueError("autograd records nothing of these calls: use layer_norm, or detach() or torch.no_grad()")

    def _new(self, shape, dtype, stream):
        if stream is None:
            return torch.empty(shape, dtype=dtype, device=self._device)
        with torch.cuda.stream(stream):
            return torch.empty(shape, dtype=dtype, device=self._device)

    def _enqueue(self, fn, p, stream):
        handle = self._raw_stream(self.device_index) if stream is None else stream.cuda_stream
        if torch._C._cuda_getDevice() == self.device_index:
            status = fn(ctypes.addressof(p), handle)
        else:
            with torch.cuda.device(self.device_index):
                status = fn(ctypes.addressof(p), handle)
        if status:
            N._check(status, None)

    # -- the passes -------------------------------------------------------------
    def forward(self, x, weight=None, bias=None, *, eps=1e-5, out=None, stream=None):
        """(y, mean, rstd): y of x's type (in `out`, which may be x, if given), statistics fp32 [rows]."""
        rows, cols, step = self._matrix(x, "x", None, self._types)
        if cols < 1:
            raise ValueError("x must have at least one column")
        dtype = x.dtype
        kind, w, b = self._params(weight, bias, dtype, cols)
        self._no_graph(x, weight, bias)
        if out is None:
            out, across = self._new((rows, cols), dtype, stream), cols
        else:
            _, _, across = self._matrix(out, "out", (rows, cols), (dtype,))
        mean, rstd = self._new(rows, torch.float32, stream), self._new(rows, torch.float32, stream)
        p = N.gnmr_norm(rows, cols, _DTYPES[dtype], kind, eps, x.data_ptr(), step, w, b, mean.data_ptr(), rstd.data_ptr(),
                        out.data_ptr(), across)
        self._enqueue(self._lib.gnmr_layer_norm, p, stream)
        return out, mean, rstd

    def backward(self, dy, x, weight, mean, rstd, *, out=None, input_grad=True, weight_grad=None, bias_grad=None,
                 add=False, stream=None):
        """dx (in `out`, which may be dy, if given; None with input_grad=False).

        weight_grad, bias_grad: [cols] tensors of one type (bf16, f16 or fp32) that get the sums over the rows
        of dy * (x - mean) * rstd and of dy, e.g. views of the gradient arena; with add, these are added to
        what is there.  No rows give zeros (nothing is added)."""
        rows, cols, step = self._matrix(x, "x", None, self._types)
        if cols < 1:
            raise ValueError("x must have at least one column")
        dtype = x.dtype
        _, _, apart = self._matrix(dy, "dy", (rows, cols), (dtype,))
        kind, w, _ = self._params(weight, None, dtype, cols)
        self._no_graph(dy, x, weight)
        if mean is None or rstd is None:
            raise ValueError("mean and rstd must be given")
        m, r = self._vector(mean, "mean", rows, (torch.float32,)), self._vector(rstd, "rstd", rows, (torch.float32,))
        to_w, to_b = self._vector(weight_grad, "weight_grad", cols, self._types), self._vector(bias_grad, "bias_grad", cols, self._types)
        if weight_grad is not None and bias_grad is not None and weight_grad.dtype != bias_grad.dtype:
            raise ValueError("weight_grad and bias_grad must be of one type")
        grads = next((_DTYPES[t.dtype] for t in (weight_grad, bias_grad) if t is not None), _DTYPES[dtype])
        at, across = None, 0
        if not input_grad:
            if out is not None:
                raise ValueError("out is for the input's gradient")
        elif out is None:
            out, across = self._new((rows, cols), dtype, stream), cols
            at = out.data_ptr()
        else:
            _, _, across = self._matrix(out, "out", (rows, cols), (dtype,))
            at = out.data_ptr()
        p = N.gnmr_norm(rows, cols, _DTYPES[dtype], kind, 0.0, x.data_ptr(), step, w, None, m, r, None, 0, dy.data_ptr(), apart,
                        at, across, to_w, to_b, grads, bool(add))
        if rows and (to_w or to_b):
            of, need = self._scratch.get(cols, (0, 0))           # of the rows that this width was last called with
            if of != rows:
                need = N.gnmr_layer_norm_scratch_bytes(p)
                self._scratch[cols] = rows, need
            scratch = self._new(need, torch.uint8, stream)
            p.scratch_bytes = need
            p.d_scratch = scratch.data_ptr()
        self._enqueue(self._lib.gnmr_layer_norm_grad, p, stream)
        return out


def _layer_norm_function():
    Once = P._once_function("layer_norm")

    class Function(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, bias, norms, eps, grad, add, anchor):
            flat = x.detach().reshape(-1, x.shape[-1])
            weight, bias = (t if t is None else t.detach() for t in (weight, bias))
            y, mean, rstd = norms.forward(flat, weight, bias, eps=eps)
            ctx.norms, ctx.grad, ctx.add, ctx.bias = norms, grad, add, None if bias is None else bias.dtype
            ctx.save_for_backward(flat, weight, mean, rstd)
            return y.view(x.shape)

        @staticmethod
        def backward(ctx, dy):
            return P._first_gradients(Once, Function.gradients, ctx, dy) + (None,) * 5

        @staticmethod
        def gradients(ctx, dy):
            x, weight, mean, rstd = ctx.saved_tensors
            dw = db = None
            if ctx.grad is not None:
                to_w, to_b = ctx.grad
            else:
                if ctx.needs_input_grad[1]:
                    dw = torch.empty_like(weight)
                if ctx.needs_input_grad[2]:
                    db = torch.empty(x.shape[-1], dtype=ctx.bias, device=x.device)
                to_w, to_b = dw, db
            dx = ctx.norms.backward(dy.reshape(x.shape).contiguous(), x, weight, mean, rstd,
                                    input_grad=ctx.needs_input_grad[0], weight_grad=to_w, bias_grad=to_b,
                                    add=ctx.add and ctx.grad is not None)
            return (None if dx is None else dx.view(dy.shape)), dw, db

    return Function


_LayerNorm = None


def layer_norm(norms, x, weight=None, bias=None, grad=None, *, eps=1e-5, add=False):
    """Layer norm over x's last dimension with a backward pass.  norms: a :class:`LayerNorm`; x: any number
    of dimensions; weight and bias as there.

    grad: (weight_grad, bias_grad), where the parameters' gradients are written, e.g. parts of the arena that
    the monitor reads (either may be None); the backward pass then writes all of them, whether or not x or a parameter
    requires a gradient (so y does), and the parameters get none from autograd.  They hold the one backward
    pass that ran last: for parameters that are used several times, or several micro-batches, clear them before the first
    and give add=True, which adds to what is there.

    The gradients have no gradients of their own: differentiating them raises RuntimeError."""
    global _LayerNorm
    if _LayerNorm is None:
        _LayerNorm = _layer_norm_function()
    if grad is not None and len(grad) != 2:
        raise ValueError("grad must be (weight_grad, bias_grad)")
    return _LayerNorm.apply(x, weight, bias, norms, eps, grad, add, P._anchor(grad, x, weight, bias))
