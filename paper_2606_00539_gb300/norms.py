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
        self._device = torch.device("cuda", self.device_index)
        self._types = tuple(_DTYPES)
        self._raw_stream = torch._C._cuda_getCurrentRawStream

    # -- argument checks ------------------------------------------------------
    def _tensor(self, t, name, dims, dtypes):
        if not isinstance(t, torch.Tensor) or t.get_device() != self.device_index:
            raise ValueError(f"{name} must be a CUDA tensor on device {self.device_index}")
        if t.dtype not in dtypes:
            raise ValueError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, got {t.dtype}")
        if t.dim() != dims:
            raise ValueError(f"{name} must have {dims} dimensions, got {t.dim()}")

    def _matrix(self, t, name, shape, dtypes):
        """The row stride of a matrix of contiguous rows."""
        self._tensor(t, name, 2, dtypes)
        rows, cols = t.shape
        if shape is not None and (rows, cols) != shape:
            raise ValueError(f"{name} must be {list(shape)}, got {[rows, cols]}")
        if t.stride(1) != 1 and cols > 1:
            raise ValueError(f"{name} must have contiguous rows")
        return t.stride(0) if rows > 1 else max(t.stride(0), cols)

    def _vector(self, t, name, n, dtypes):
        if t is None:
            return None
        self._tensor(t, name, 1, dtypes)
        if t.numel() != n or not t.is_contiguous():
            raise ValueError(f"{name} must hold {n} contiguous entries")
        return t.data_ptr()

    def _params(self, p, weight, bias, dtype):
        p.param_dtype = p.dtype
        for t in (weight, bias):
            if t is not None:
                if t.dtype not in (dtype, torch.float32):
                    raise ValueError(f"weight and bias must be {dtype} or torch.float32, got {t.dtype}")
                p.param_dtype = _DTYPES[t.dtype]
        if weight is not None and bias is not None and weight.dtype != bias.dtype:
            raise ValueError("weight and bias must be of one type")
        p.d_weight = self._vector(weight, "weight", p.cols, (dtype, torch.float32))
        p.d_bias = self._vector(bias, "bias", p.cols, (dtype, torch.float32))

    @staticmethod
    def _no_graph(*operands):
        if any(t is not None and t.requires_grad for t in operands) and torch.is_grad_enabled():
            raise ValueError("autograd records nothing of these calls: use layer_norm, or detach() or torch.no_grad()")

    def _new(self, shape, dtype, stream):
        if stream is None:
            return torch.empty(shape, dtype=dtype, device=self._device)
        with torch.cuda.stream(stream):
            return torch.empty(shape, dtype=dtype, device=self._device)

    def _enqueue(self, fn, p, stream):
        handle = self._raw_stream(self.device_index) if stream is None else stream.cuda_stream
        if torch.cuda.current_device() == self.device_index:
            status = fn(ctypes.addressof(p), handle)
        else:
            with torch.cuda.device(self.device_index):
                status = fn(ctypes.addressof(p), handle)
        if status:
            N._check(status, None)

    # -- the passes -------------------------------------------------------------
    def forward(self, x, weight=None, bias=None, *, eps=1e-5, out=None, stream=None):
        """(y, mean, rstd): y of x's type (in `out`, which may be x, if given), statistics fp32 [rows]."""
        step = self._matrix(x, "x", None, self._types)
        rows, cols = x.shape
        if cols < 1:
            raise ValueError("x must have at least one column")
        self._no_graph(x, weight, bias)
        p = N.gnmr_norm(rows, cols, _DTYPES[x.dtype])
        self._params(p, weight, bias, x.dtype)
        if out is None:
            out, across = self._new((rows, cols), x.dtype, stream), cols
        else:
            across = self._matrix(out, "out", (rows, cols), (x.dtype,))
        mean, rstd = (self._new(rows, torch.float32, stream) for _ in range(2))
        p.eps, p.d_x, p.x_stride, p.d_y, p.y_stride = eps, x.data_ptr(), step, out.data_ptr(), across
        p.d_mean, p.d_rstd = mean.data_ptr(), rstd.data_ptr()
        self._enqueue(self._lib.gnmr_layer_norm, p, stream)
        return out, mean, rstd

    def backward(self, dy, x, weight, mean, rstd, *, out=None, input_grad=True, weight_grad=None, bias_grad=None,
                 add=False, stream=None):
        """dx (in `out`, which may be dy, if given; None with input_grad=False).

        weight_grad, bias_grad: [cols] tensors of one type (bf16, f16 or fp32) that get the sums over the rows
        of dy * (x - mean) * rstd and of dy, e.g. views of the gradient arena; with add, these are added to
        what is there.  No rows give zeros (nothing is added)."""
        step = self._matrix(x, "x", None, self._types)
        rows, cols = x.shape
        if cols < 1:
            raise ValueError("x must have at least one column")
        dtype = x.dtype
        apart = self._matrix(dy, "dy", (rows, cols), (dtype,))
        self._no_graph(dy, x, weight)
        p = N.gnmr_norm(rows, cols, _DTYPES[dtype])
        self._params(p, weight, None, dtype)
        p.d_x, p.x_stride, p.d_dy, p.dy_stride = x.data_ptr(), step, dy.data_ptr(), apart
        p.d_mean = self._vector(mean, "mean", rows, (torch.float32,))
        p.d_rstd = self._vector(rstd, "rstd", rows, (torch.float32,))
        if mean is None or rstd is None:
            raise ValueError("mean and rstd must be given")
        if not input_grad:
            if out is not None:
                raise ValueError("out is for the input's gradient")
        elif out is None:
            out = self._new((rows, cols), dtype, stream)
            p.d_dx, p.dx_stride = out.data_ptr(), cols
        else:
            p.dx_stride = self._matrix(out, "out", (rows, cols), (dtype,))
            p.d_dx = out.data_ptr()
        p.add = bool(add)
        p.grad_dtype = p.dtype
        scratch = None
        if weight_grad is not None or bias_grad is not None:
            p.d_dweight = self._vector(weight_grad, "weight_grad", cols, self._types)
            p.d_dbias = self._vector(bias_grad, "bias_grad", cols, self._types)
            kinds = {t.dtype for t in (weight_grad, bias_grad) if t is not None}
            if len(kinds) > 1:
                raise ValueError("weight_grad and bias_grad must be of one type")
            p.grad_dtype = _DTYPES[kinds.pop()]
            if rows:
                p.scratch_bytes = N.gnmr_layer_norm_scratch_bytes(p)
                scratch = self._new(p.scratch_bytes, torch.uint8, stream)
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
