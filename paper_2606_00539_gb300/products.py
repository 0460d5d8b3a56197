"""torch-facing wrapper of the expert products: the linear units that the recovery mask
chooses a path for, in 16 bits (recovery path) and on 8-bit integer codes (low-cost
path), grouped by expert over ragged rows.  PyTorch supplies device memory and the
stream; every product and every code is computed by libgnmr's kernels."""
from __future__ import annotations

import ctypes

from . import _native as N


torch = None                                       # loaded with the first ExpertProducts, as the monitor does
_DTYPES: dict = {}                                 # torch type -> gnmr_dtype
_NAMED: dict = {}                                  # name -> torch type
_ACTIVATIONS = {"silu": N.GNMR_ACT_SILU, "gelu": N.GNMR_ACT_GELU}


def _load_torch():
    global torch
    import torch as module
    torch = module
    _DTYPES.update({torch.bfloat16: N.GNMR_DTYPE_BF16, torch.float16: N.GNMR_DTYPE_F16,
                    torch.float32: N.GNMR_DTYPE_F32})
    _NAMED.update({"bf16": torch.bfloat16, "bfloat16": torch.bfloat16, "f16": torch.float16,
                   "float16": torch.float16, "f32": torch.float32, "float32": torch.float32})


def _named_dtype(name):
    if name in _NAMED:
        return _NAMED[name]
    if name in _DTYPES:
        return name
    raise ValueError(f"out_dtype must be one of {sorted(_NAMED)} or the torch type, got {name!r}")


def _activation(name):
    if name not in _ACTIVATIONS:
        raise ValueError(f"activation must be one of {sorted(_ACTIVATIONS)}, got {name!r}")
    return _ACTIVATIONS[name]


class ExpertProducts:
    """Products of linear units grouped by expert, on one device.

    Rows lie group by group: group g has the rows offsets[g] up to offsets[g + 1] of the
    activations (offsets: int64 tensor [groups + 1] on the device, as a router's cumulative
    counts give it; None for one group of all rows).  Weights are [groups, n_out, n_in], or
    [n_out, n_in] for one group, with contiguous rows and any strides between rows and
    groups, so views of a flat arena will do.

    mask: uint8 tensor [groups] on the device (any stride), as Monitor.step returns it for
    the experts' units: the 16-bit products compute the groups whose entry is not 0, forward_i8 those
    whose entry is 0, and both leave the other groups' outputs as they are.

    Rows of `out` that belong to no group are left as they are.  stream: a torch stream, default the
    current one; as with any torch call, tensors that were made on another stream are the
    caller's to order.  One instance serves any sizes; use it from one stream at a time.

    Autograd records none of these calls (expert_linear is the layer that it knows), so the
    16-bit products refuse operands that require a gradient while it records."""

    def __init__(self, device=0):
        self._h = None
        self.device_index = int(device.index if hasattr(device, "index") else device)
        if torch is None:
            _load_torch()
        self._h = N.gnmr_products_create(self.device_index)
        self._run = N.load().gnmr_products_run
        self._run_gated = N.load().gnmr_products_gated
        self._device = torch.device("cuda", self.device_index)
        self._sixteen = (torch.bfloat16, torch.float16)
        self._any = tuple(_DTYPES)
        self._raw_stream = torch._C._cuda_getCurrentRawStream

    # -- lifetime -----------------------------------------------------------
    def close(self) -> None:
        """Waits for the device and frees the handle; raises what :meth:`check` does."""
        if self._h:
            h, self._h = self._h, None
            N.gnmr_products_destroy(h)

    def check(self) -> None:
        """Raises GnmrError if a product gave up waiting inside the GPU (its output is not valid, and
        no further product is taken).  Waits for nothing: synchronize first for the products enqueued so far."""
        if not self._h:
            raise ValueError("the products were closed")
        N.gnmr_products_status(self._h)

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- argument checks ------------------------------------------------------
    # A small product takes the GPU under 10 us: these checks are written to cost the host
    # no more than that.
    def _refuse(self, t, name, dims, dtypes):
        if not isinstance(t, torch.Tensor) or t.get_device() != self.device_index:
            raise ValueError(f"{name} must be a CUDA tensor on device {self.device_index}")
        if t.dtype not in dtypes:
            raise ValueError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, got {t.dtype}")
        raise ValueError(f"{name} must have {' or '.join(str(d) for d in dims)} dimensions, got {t.dim()}")

    def _tensor(self, t, name, dims, dtypes):
        if not isinstance(t, torch.Tensor) or t.get_device() != self.device_index or t.dtype not in dtypes or \
                t.dim() not in dims:
            self._refuse(t, name, dims, dtypes)

    def _matrix(self, t, name, dims, dtypes):
        """(groups, rows, columns, row stride, group stride) of a tensor of contiguous rows."""
        if not isinstance(t, torch.Tensor) or t.get_device() != self.device_index or t.dtype not in dtypes:
            self._refuse(t, name, dims, dtypes)
        shape, stride = t.shape, t.stride()
        if len(shape) not in dims:
            self._refuse(t, name, dims, dtypes)
        *lead, rows, cols = shape
        if stride[-1] != 1 and cols > 1:
            raise ValueError(f"{name} must have contiguous rows")
        # a single row, or group, has no stride of its own, and torch may give it any
        row = stride[-2] if rows > 1 else max(stride[-2], cols)
        if not lead:
            return 1, rows, cols, row, 0
        return lead[0], rows, cols, row, stride[0] if lead[0] > 1 else 0

    def _mask(self, mask, groups):
        """Device pointer of the mask, and its stride."""
        if mask is None:
            return None, 1
        self._tensor(mask, "mask", (1,), (torch.uint8,))
        if mask.numel() != groups:
            raise ValueError(f"mask must have one entry per group ({groups})")
        return mask.data_ptr(), mask.stride(0) if groups > 1 else 1

    def _grouping(self, groups, offsets, mask):
        """Device pointers of offsets and mask, and the mask's stride."""
        at = None
        if offsets is not None:
            self._tensor(offsets, "offsets", (1,), (torch.int64,))
            if offsets.numel() != groups + 1 or not offsets.is_contiguous():
                raise ValueError(f"offsets must hold groups + 1 = {groups + 1} contiguous entries")
            at = offsets.data_ptr()
        elif groups != 1:
            raise ValueError("offsets may be None for one group only")
        return (at, *self._mask(mask, groups))

    def _new(self, shape, dtype, stream):
        if stream is None:
            return torch.empty(shape, dtype=dtype, device=self._device)
        with torch.cuda.stream(stream):
            return torch.empty(shape, dtype=dtype, device=self._device)

    def _stream(self, stream):
        return self._raw_stream(self.device_index) if stream is None else stream.cuda_stream

    def _out(self, out, rows, width, dtypes, stream):
        """(out, its row stride): the tensor given, checked, or a new one of the first type."""
        if out is None:
            return self._new((rows, width), dtypes[0], stream), width
        _, r, c, step, _ = self._matrix(out, "out", (2,), dtypes)
        if (r, c) != (rows, width):
            raise ValueError(f"out must be [{rows}, {width}], got [{r}, {c}]")
        return out, step

    def _enqueue(self, p, stream, run=None, scratch_bytes=N.gnmr_products_scratch_bytes):
        if not self._h:
            raise ValueError("the products were closed")
        handle = self._stream(stream)
        run = run or self._run
        status = run(self._h, ctypes.addressof(p), handle)
        if status == N.GNMR_ERR_LAYOUT:
            # operands that cannot be read in place: room for their copies, on the same stream
            need = scratch_bytes(p)
            if need > p.scratch_bytes:
                scratch = self._new(need, torch.uint8, stream)
                p.d_scratch, p.scratch_bytes = scratch.data_ptr(), need
                status = run(self._h, ctypes.addressof(p), handle)
        if status:
            N._check(status, None)

    # -- 16-bit products ------------------------------------------------------
    @staticmethod
    def _no_graph(a, b=None):
        if (a.requires_grad or (b is not None and b.requires_grad)) and torch.is_grad_enabled():
            raise ValueError("autograd records nothing of a product: use expert_linear or expert_gated, or detach() or torch.no_grad()")

    def forward(self, x, w, offsets=None, *, out=None, mask=None, stream=None):
        """y[r] = W_g x[r] for the rows r of every group g: x [rows, n_in] -> [rows, n_out]."""
        groups, n_out, n_in, row, group = self._matrix(w, "w", (2, 3), self._sixteen)
        dtype = w.dtype
        _, rows, cols, step, _ = self._matrix(x, "x", (2,), (dtype,))
        if cols != n_in:
            raise ValueError(f"x must have {n_in} columns, got {cols}")
        self._no_graph(x, w)
        at, bits, each = self._grouping(groups, offsets, mask)
        out, across = self._out(out, rows, n_out, (dtype,), stream)
        code = _DTYPES[dtype]
        self._enqueue(N.gnmr_product(N.GNMR_PRODUCT_FORWARD, groups, rows, n_out, n_in, code, code, at, bits, each,
                                     x.data_ptr(), step, None, 0, w.data_ptr(), row, group, None, None,
                                     out.data_ptr(), across), stream)
        return out

    def input_grad(self, dy, w, offsets=None, *, out=None, mask=None, stream=None):
        """dx[r] = W_g^T dy[r]: dy [rows, n_out] -> [rows, n_in]."""
        groups, n_out, n_in, row, group = self._matrix(w, "w", (2, 3), self._sixteen)
        dtype = w.dtype
        _, rows, cols, step, _ = self._matrix(dy, "dy", (2,), (dtype,))
        if cols != n_out:
            raise ValueError(f"dy must have {n_out} columns, got {cols}")
        self._no_graph(dy, w)
        at, bits, each = self._grouping(groups, offsets, mask)
        out, across = self._out(out, rows, n_in, (dtype,), stream)
        code = _DTYPES[dtype]
        self._enqueue(N.gnmr_product(N.GNMR_PRODUCT_INPUT_GRAD, groups, rows, n_out, n_in, code, code, at, bits, each,
                                     None, 0, dy.data_ptr(), step, w.data_ptr(), row, group, None, None,
                                     out.data_ptr(), across), stream)
        return out

    def weight_grad(self, dy, x, offsets=None, *, out, add=False, mask=None, stream=None):
        """out_g = sum over the group's rows of dy[r] x[r]^T, or that added to out_g.

        out: [groups, n_out, n_in] (or [n_out, n_in]) of dy's type or fp32, e.g. a view of
        the gradient arena that the monitor reads.  A group without rows gets zeros
        (nothing is added)."""
        _, rows, n_out, dy_step, _ = self._matrix(dy, "dy", (2,), self._sixteen)
        dtype = dy.dtype
        _, x_rows, n_in, x_step, _ = self._matrix(x, "x", (2,), (dtype,))
        if x_rows != rows:
            raise ValueError("dy and x must have the same number of rows")
        groups, high, wide, row, group = self._matrix(out, "out", (2, 3), (dtype, torch.float32))
        if (high, wide) != (n_out, n_in):
            raise ValueError(f"out must be [{n_out}, {n_in}] for each group, got [{high}, {wide}]")
        self._no_graph(dy, x)
        at, bits, each = self._grouping(groups, offsets, mask)
        self._enqueue(N.gnmr_product(N.GNMR_PRODUCT_WEIGHT_GRAD, groups, rows, n_out, n_in, _DTYPES[dtype],
                                     _DTYPES[out.dtype], at, bits, each, x.data_ptr(), x_step, dy.data_ptr(), dy_step,
                                     None, 0, 0, None, None, out.data_ptr(), row, group, bool(add)), stream)
        return out

    # -- gated blocks -----------------------------------------------------------
    def gated(self, x, w, offsets=None, *, out=None, keep=None, mask=None, activation="silu", stream=None):
        """h[r] = act(a) * b with [a, b] = W_g x[r]: both projections of a gated block, the activation
        ("silu" or "gelu", the one with erf) and the product in one kernel.  w: [groups, 2 n, n_in] (or
        [2 n, n_in]), the n rows of the gate a before those of b; -> [rows, n].

        keep: a [rows, 2 n] tensor of x's type that gets [a, b] as well, for gate_grad.  The rest of the
        backward pass are products on w as it lies: dx = input_grad(dab, w, ...), dw = weight_grad(dab, x, ...)."""
        act = _activation(activation)
        groups, both, n_in, row, group = self._matrix(w, "w", (2, 3), self._sixteen)
        dtype = w.dtype
        _, rows, cols, step, _ = self._matrix(x, "x", (2,), (dtype,))
        if cols != n_in:
            raise ValueError(f"x must have {n_in} columns, got {cols}")
        if both % 2:
            raise ValueError(f"w must have the rows of two projections, got {both}")
        self._no_graph(x, w)
        at, bits, each = self._grouping(groups, offsets, mask)
        out, across = self._out(out, rows, both // 2, (dtype,), stream)
        kept, apart = None, 0
        if keep is not None:
            _, r, c, apart, _ = self._matrix(keep, "keep", (2,), (dtype,))
            if (r, c) != (rows, both):
                raise ValueError(f"keep must be [{rows}, {both}], got [{r}, {c}]")
            kept = keep.data_ptr()
        p = N.gnmr_gated(groups, act, rows, both // 2, n_in, _DTYPES[dtype], at, bits, each, x.data_ptr(), step,
                         w.data_ptr(), row, group, out.data_ptr(), across, kept, apart)
        self._enqueue(p, stream, self._run_gated, N.gnmr_gated_scratch_bytes)
        return out

    def gate(self, ab, offsets=None, *, out=None, mask=None, activation="silu", stream=None):
        """h = act(a) * b from [a, b] = ab ([rows, 2 n]), for the groups whose mask entry is 0: those whose
        projections forward_i8 computes."""
        act = _activation(activation)
        _, rows, both, step, _ = self._matrix(ab, "ab", (2,), self._sixteen)
        if both % 2:
            raise ValueError(f"ab must have the columns of two projections, got {both}")
        if offsets is None:
            if isinstance(mask, torch.Tensor) and mask.numel() != 1:
                raise ValueError("offsets may be None for one group only")
            groups = 1
        else:
            self._tensor(offsets, "offsets", (1,), (torch.int64,))
            groups = offsets.numel() - 1
        at, bits, each = self._grouping(groups, offsets, mask)
        self._no_graph(ab)
        out, across = self._out(out, rows, both // 2, (ab.dtype,), stream)
        self._on_device(N.load().gnmr_gate, ab.data_ptr(), _DTYPES[ab.dtype], act, groups, rows, both // 2, step, at, bits,
                        each, out.data_ptr(), across, self._stream(stream))
        return out

    def gate_grad(self, dh, ab, *, out=None, activation="silu", stream=None):
        """The gradient of [a, b] = ab ([rows, 2 n], as gated keeps it) from that of h, dh: [rows, n], for
        all rows.  out may be ab, which is then overwritten."""
        act = _activation(activation)
        _, rows, both, step, _ = self._matrix(ab, "ab", (2,), self._sixteen)
        _, r, n, apart, _ = self._matrix(dh, "dh", (2,), (ab.dtype,))
        if (r, 2 * n) != (rows, both):
            raise ValueError(f"ab must be [{r}, {2 * n}] for this dh, got [{rows}, {both}]")
        self._no_graph(dh, ab)
        out, across = self._out(out, rows, both, (ab.dtype,), stream)
        self._on_device(N.load().gnmr_gate_grad, dh.data_ptr(), _DTYPES[ab.dtype], act, rows, n, apart, ab.data_ptr(), step,
                        out.data_ptr(), across, self._stream(stream))
        return out

    # -- 8-bit products -------------------------------------------------------
    def _on_device(self, fn, *args):
        """A call that runs on the current device, on this one."""
        if not self._h:
            raise ValueError("the products were closed")
        if torch.cuda.current_device() == self.device_index:
            status = fn(*args)
        else:
            with torch.cuda.device(self.device_index):
                status = fn(*args)
        if status:
            N._check(status, None)

    def _quantize(self, x, columns, mask, stream):
        groups, rows, cols, row, group = self._matrix(x, "x", (2, 3), self._any)
        bits, step = self._mask(mask, groups)
        high, wide = (cols, rows) if columns else (rows, cols)
        held = (wide + 15) // 16 * 16              # rows of codes start at multiples of 16 bytes
        lead = x.shape[:-2]
        q = self._new((*lead, high, held), torch.int8, stream)
        scale = self._new((*lead, high), torch.float32, stream)
        fn = N.gnmr_quantize_columns if columns else N.gnmr_quantize_rows
        args = (x.data_ptr(), _DTYPES[x.dtype], groups, rows, cols, row, group, bits, step, q.data_ptr(), held,
                high * held, scale.data_ptr(), self._stream(stream))
        if torch.cuda.current_device() == self.device_index:
            fn(*args)
        else:
            with torch.cuda.device(self.device_index):
                fn(*args)
        return q if held == wide else q[..., :wide], scale

    def quantize_rows(self, x, *, mask=None, stream=None):
        """8-bit codes of every row of x ([rows, cols] or [groups, rows, cols]; bf16, f16 or
        fp32) and its scale: (int8 codes of x's shape, fp32 scales).  round(x * (127 * (1 / amax))),
        halves to even; x is about codes * scale.  Activations by token, weights by output channel.
        mask: groups whose entry is not 0, which forward_i8 leaves out, get no codes."""
        return self._quantize(x, False, mask, stream)

    def quantize_columns(self, w, *, mask=None, stream=None):
        """8-bit codes of every column of w, transposed, and its scale: ([..., cols, rows],
        [..., cols]).  Weights by input channel, for the backward product of the 8-bit path:
        dx = forward_i8(codes of dy, ..., codes of w's columns, ...)."""
        return self._quantize(w, True, mask, stream)

    def forward_i8(self, xq, x_scale, wq, w_scale, offsets=None, *, out=None, out_dtype="bf16", mask=None,
                   stream=None):
        """y[r] = x_scale[r] * w_scale_g * (Wq_g xq[r]) on 8-bit codes; the sum is an exact
        integer (n_in up to 131,071), converted and scaled in fp32 (by x_scale first, a rounding
        each), then rounded to out's type."""
        groups, n_out, n_in, row, group = self._matrix(wq, "wq", (2, 3), (torch.int8,))
        _, rows, cols, step, _ = self._matrix(xq, "xq", (2,), (torch.int8,))
        if cols != n_in:
            raise ValueError(f"xq must have {n_in} columns, got {cols}")
        for t, name, n in ((x_scale, "x_scale", rows), (w_scale, "w_scale", groups * n_out)):
            self._tensor(t, name, (1, 2), (torch.float32,))
            if t.numel() != n or not t.is_contiguous():
                raise ValueError(f"{name} must hold {n} contiguous entries")
        at, bits, each = self._grouping(groups, offsets, mask)
        out, across = self._out(out, rows, n_out, (_named_dtype(out_dtype),) if out is None else self._any, stream)
        self._enqueue(N.gnmr_product(N.GNMR_PRODUCT_FORWARD_I8, groups, rows, n_out, n_in, 0, _DTYPES[out.dtype], at,
                                     bits, each, xq.data_ptr(), step, None, 0, wq.data_ptr(), row, group,
                                     x_scale.data_ptr(), w_scale.data_ptr(), out.data_ptr(), across), stream)
        return out


def _once_function(name):
    class Once(torch.autograd.Function):
        """A gradient that has none of its own: passing one back through it is an error."""

        @staticmethod
        def forward(ctx, anchor, g):
            return g.view_as(g)

        @staticmethod
        def backward(ctx, _):
            raise RuntimeError(f"{name} has no second derivatives: its gradients cannot be differentiated")

    return Once


def _first_gradients(once, gradients, ctx, *dy):
    """gradients(ctx, *dy), of which autograd records nothing, and no gradients of these."""
    if not torch.is_grad_enabled():
        return gradients(ctx, *dy)
    with torch.no_grad():                          # create_graph
        got = gradients(ctx, *dy)
    anchor = torch.empty(0, requires_grad=True)
    return tuple(g if g is None else once.apply(anchor, g) for g in got)


def _anchor(grad, *operands):
    """A tensor that requires a gradient, where a gradient is to be written and no operand requires
    one: without it autograd would leave the backward pass out."""
    if grad is not None and torch.is_grad_enabled() and not any(t is not None and t.requires_grad for t in operands):
        return torch.empty(0, requires_grad=True)
    return None


def _expert_linear_function():
    Once = _once_function("expert_linear")

    class ExpertLinear(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, products, offsets, mask, grad, add, codes, anchor):
            x, w = x.detach(), w.detach()
            y = torch.empty(x.shape[0], w.shape[-2], dtype=x.dtype, device=x.device)
            products.forward(x, w, offsets, out=y, mask=mask)
            if mask is not None:
                xq, xs = products.quantize_rows(x)
                wq, ws = codes[:2] if codes is not None else products.quantize_rows(w, mask=mask)
                products.forward_i8(xq, xs, wq, ws, offsets, out=y, mask=mask)
            ctx.products, ctx.grad, ctx.add, ctx.codes = products, grad, add, codes
            ctx.save_for_backward(x, w, *(t for t in (offsets, mask) if t is not None))
            ctx.has = (offsets is not None, mask is not None)
            return y

        @staticmethod
        def backward(ctx, dy):
            return _first_gradients(Once, ExpertLinear.gradients, ctx, dy) + (None,) * 7

        @staticmethod
        def gradients(ctx, dy):
            x, w, *rest = ctx.saved_tensors
            offsets = rest.pop(0) if ctx.has[0] else None
            mask = rest.pop(0) if ctx.has[1] else None
            products, dx, dw = ctx.products, None, None
            dy = dy.contiguous()
            if ctx.needs_input_grad[0]:
                dx = torch.empty_like(x, memory_format=torch.contiguous_format)
                products.input_grad(dy, w, offsets, out=dx, mask=mask)
                if mask is not None:
                    dq, ds = products.quantize_rows(dy)
                    vq, vs = ctx.codes[2:] if ctx.codes is not None else products.quantize_columns(w, mask=mask)
                    products.forward_i8(dq, ds, vq, vs, offsets, out=dx, mask=mask)
            if ctx.grad is not None:
                products.weight_grad(dy, x, offsets, out=ctx.grad, add=ctx.add)
            elif ctx.needs_input_grad[1]:
                dw = torch.empty_like(w, memory_format=torch.contiguous_format)
                products.weight_grad(dy, x, offsets, out=dw)
            return dx, dw

    return ExpertLinear


_ExpertLinear = None


def expert_linear(products, x, w, offsets=None, mask=None, grad=None, *, add=False, codes=None):
    """A linear layer of experts with a backward pass, each expert on the path that the
    mask gives it: 16 bits where its entry is not 0, 8-bit codes where it is 0 (16 bits
    everywhere without a mask).

    x: [rows, n_in], every row in some group; w: [groups, n_out, n_in]; offsets and mask as in
    :class:`ExpertProducts`; the mask is read again in the backward pass, which follows the
    same paths.  Gradients pass through the codes as if they were the values they stand for
    (straight through); the weights' gradient is the 16-bit product for every expert.

    grad: where the weights' gradient is written, e.g. the experts' part of the arena that
    the monitor reads; the backward pass then writes all of it, whether or not x or w
    requires a gradient (so y does), and w gets no gradient from autograd.  It holds the one
    backward pass that ran last: for a weight that is used several times, or several micro-batches, clear
    it before the first and give add=True, which adds to what is there.  codes: (wq, ws, vq, vs) of quantize_rows(w) and quantize_columns(w), for
    weights that do not change; by default both are made anew in each pass.

    The gradients have no gradients of their own: differentiating them raises RuntimeError."""
    global _ExpertLinear
    if _ExpertLinear is None:
        _ExpertLinear = _expert_linear_function()
    return _ExpertLinear.apply(x, w, products, offsets, mask, grad, add, codes, _anchor(grad, x, w))


def _expert_gated_function():
    Once = _once_function("expert_gated")

    class ExpertGated(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, products, offsets, mask, grad, add, codes, activation, keeps, anchor):
            x, w = x.detach(), w.detach()
            rows, both = x.shape[0], w.shape[-2]
            h = torch.empty(rows, both // 2, dtype=x.dtype, device=x.device)
            ab = torch.empty(rows, both, dtype=x.dtype, device=x.device) if keeps or mask is not None else None
            products.gated(x, w, offsets, out=h, keep=ab if keeps else None, mask=mask, activation=activation)
            if mask is not None:
                xq, xs = products.quantize_rows(x)
                wq, ws = codes[:2] if codes is not None else products.quantize_rows(w, mask=mask)
                products.forward_i8(xq, xs, wq, ws, offsets, out=ab, mask=mask)
                products.gate(ab, offsets, out=h, mask=mask, activation=activation)
            ctx.products, ctx.grad, ctx.add, ctx.codes, ctx.activation = products, grad, add, codes, activation
            ctx.has = (offsets is not None, mask is not None)
            if keeps:
                ctx.save_for_backward(x, w, ab, *(t for t in (offsets, mask) if t is not None))
            return h

        @staticmethod
        def backward(ctx, dh):
            return _first_gradients(Once, ExpertGated.gradients, ctx, dh) + (None,) * 9

        @staticmethod
        def gradients(ctx, dh):
            x, w, ab, *rest = ctx.saved_tensors
            offsets = rest.pop(0) if ctx.has[0] else None
            mask = rest.pop(0) if ctx.has[1] else None
            products, dx, dw = ctx.products, None, None
            dab = products.gate_grad(dh.contiguous(), ab, activation=ctx.activation)
            if ctx.needs_input_grad[0]:
                dx = torch.empty_like(x, memory_format=torch.contiguous_format)
                products.input_grad(dab, w, offsets, out=dx, mask=mask)
                if mask is not None:
                    dq, ds = products.quantize_rows(dab)
                    vq, vs = ctx.codes[2:] if ctx.codes is not None else products.quantize_columns(w, mask=mask)
                    products.forward_i8(dq, ds, vq, vs, offsets, out=dx, mask=mask)
            if ctx.grad is not None:
                products.weight_grad(dab, x, offsets, out=ctx.grad, add=ctx.add)
            elif ctx.needs_input_grad[1]:
                dw = torch.empty_like(w, memory_format=torch.contiguous_format)
                products.weight_grad(dab, x, offsets, out=dw)
            return dx, dw

    return ExpertGated


_ExpertGated = None


def expert_gated(products, x, w, offsets=None, mask=None, grad=None, *, add=False, codes=None, activation="silu"):
    """The first half of a gated feed-forward layer of experts with a backward pass: h = act(a) * b,
    [a, b] = W_g x, each expert on the path that the mask gives it (expert_linear is the second half).

    w: [groups, 2 n, n_in], the gate's rows first, as in :meth:`ExpertProducts.gated`; everything
    else as in :func:`expert_linear`, codes of w as it lies.  On the low-cost path [a, b] is the 8-bit
    product rounded to x's type, and h is formed from that; the backward pass takes [a, b] in x's type
    on both paths, and their gradient's 8-bit codes by row for the low-cost one.

    The gradients have no gradients of their own: differentiating them raises RuntimeError."""
    global _ExpertGated
    if _ExpertGated is None:
        _ExpertGated = _expert_gated_function()
    anchor = _anchor(grad, x, w)
    keeps = torch.is_grad_enabled() and (anchor is not None or x.requires_grad or w.requires_grad)
    return _ExpertGated.apply(x, w, products, offsets, mask, grad, add, codes, activation, keeps, anchor)
