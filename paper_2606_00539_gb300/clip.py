"""torch-facing wrapper of the gradient norm and the clipping.  PyTorch supplies device memory and the stream;
libgnmr's kernels form the norm and scale the gradients."""
from __future__ import annotations

import ctypes
from bisect import bisect_right
from operator import add, gt

from . import _native as N
from . import products as P

torch = None                                       # loaded with the first GradientClip


def _refuse_overlaps(at, to, norm, sizes):
    """A call's warps go in no order: memory that is written twice, or written where another tensor is still to be read, would
    get values that go by timing.  at, to: where the gradients and the outputs begin (to None: scaled where they lie); norm: where a
    given norm is, or None; sizes: bytes."""
    if 0 in sizes:
        at, to, sizes = ([v for v, n in zip(of, sizes) if n] if of is not None else None for of in (at, to, sizes))
    first = at if to is None else to
    end = list(map(add, first, sizes))
    if norm is not None:
        first, end = [*first, norm], [*end, norm + 4]
    order = range(len(first))
    if any(map(gt, end, first[1:])):               # not in order, or worse
        order = sorted(order, key=first.__getitem__)
        first, end = [first[i] for i in order], [end[i] for i in order]
        if any(map(gt, end, first[1:])):
            raise ValueError("the same memory is written twice: no two of the tensors may overlap")
    if to is None or not at or end[-1] <= min(at) or max(map(add, at, sizes)) <= first[0]:
        return
    for i, (p, n) in enumerate(zip(at, sizes)):
        k = bisect_right(end, p)                   # the first written range that ends behind p: this gradient's own, or beyond it
        if k < len(end) and first[k] < p + n and (first[k] != p or order[k] != i):
            raise ValueError("out must not be where another gradient lies")


class GradientClip:
    """The norm over many gradients, and the gradients scaled down to a limit:
    norm = sqrt(sum of x^2 over all of them), and where norm > max_norm every element times max_norm / norm.

    tensors: the gradients, or others of the same sizes and types (bf16, f16 or fp32, mixed as they
    come; contiguous; a flat arena is one tensor).  Their sizes and types are the plan, made once; where they lie comes with each
    call, which reads no address of an earlier one.  A norm that is not finite scales nothing.

    stream: a torch stream, default the current one.  A plan holds nothing that a call writes: calls on several streams,
    or in several graphs, do not disturb each other."""

    def __init__(self, tensors, device=0):
        global torch
        self._h = None
        if torch is None:
            if P.torch is None:
                P._load_torch()
            torch = P.torch
        self.device_index = int(device.index if hasattr(device, "index") else device)
        self._device = torch.device("cuda", self.device_index)
        tensors = list(tensors)
        if not all(isinstance(t, torch.Tensor) and t.dtype in P._DTYPES for t in tensors):
            bad = next(i for i, t in enumerate(tensors) if not isinstance(t, torch.Tensor) or t.dtype not in P._DTYPES)
            raise ValueError(f"tensor {bad} must be a tensor of {' or '.join(str(d) for d in P._DTYPES)}")
        self._lengths, self._dtypes = [t.numel() for t in tensors], [t.dtype for t in tensors]
        self._bytes = [t.numel() * t.element_size() for t in tensors]
        self._h = N.gnmr_clip_create(self._lengths, [P._DTYPES[d] for d in self._dtypes], self.device_index)
        self._table = torch.from_numpy(N.gnmr_clip_table(self._h)).to(self._device)
        self._made_on = torch._C._cuda_getCurrentRawStream(self.device_index)
        self._scratch_bytes = N.gnmr_clip_scratch_bytes(self._h)

    # -- lifetime -----------------------------------------------------------
    def close(self) -> None:
        """Frees the plan; no CUDA call but what torch's allocator makes of its table."""
        if self._h:
            N.gnmr_clip_destroy(self._h)
            self._h = self._table = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the calls ------------------------------------------------------------
    def _places(self, tensors, name):
        tensors = list(tensors)
        if len(tensors) != len(self._lengths):
            raise ValueError(f"{name} must be {len(self._lengths)} tensors, got {len(tensors)}")
        here, isin = self.device_index, torch.Tensor
        if not all(isinstance(t, isin) and t.get_device() == here for t in tensors):
            bad = next(i for i, t in enumerate(tensors) if not isinstance(t, isin) or t.get_device() != here)
            raise ValueError(f"{name}[{bad}] must be a CUDA tensor on device {here}")
        if [t.numel() for t in tensors] != self._lengths or [t.dtype for t in tensors] != self._dtypes or \
                not all(t.is_contiguous() for t in tensors):
            for i, (t, n, dtype) in enumerate(zip(tensors, self._lengths, self._dtypes)):
                if t.numel() != n or t.dtype != dtype or not t.is_contiguous():
                    raise ValueError(f"{name}[{i}] must be {n} contiguous elements of {dtype}")
        return tensors, [t.data_ptr() for t in tensors]

    def _new(self, shape, dtype, stream):
        if stream is None:
            return torch.empty(shape, dtype=dtype, device=self._device)
        with torch.cuda.stream(stream):
            return torch.empty(shape, dtype=dtype, device=self._device)

    def prepare_clip(self, grads, max_norm, *, out=None, unit_norms=None, norm=None, stream=None):
        """Validates and marshals clip()'s arguments once and returns a callable that enqueues one pass with
        them: each call is one C call, and returns the norm's tensor.  The tensors' storage and the stream are fixed at preparation, their
        contents may change between calls; one such callable is for one stream at a time (it has scratch memory of its own).  Keep it
        as long as a graph that captured one of its calls is replayed."""
        if not self._h:
            raise ValueError("the plan was closed")
        max_norm = float(max_norm)
        if not max_norm >= 0:
            raise ValueError(f"max_norm must be 0 or more, got {max_norm}")
        grads, at = self._places(grads, "grads")
        outs, to = (None, None) if out is None else self._places(out, "out")
        units, count = None, 0
        if unit_norms is not None:
            if not isinstance(unit_norms, torch.Tensor) or unit_norms.get_device() != self.device_index or \
                    unit_norms.dtype != torch.float64 or not unit_norms.is_contiguous():
                raise ValueError(f"unit_norms must be a contiguous fp64 tensor on device {self.device_index}")
        given = None
        if norm is None:
            norm = self._new((), torch.float32, stream)
        elif not isinstance(norm, torch.Tensor) or norm.get_device() != self.device_index or norm.dtype != torch.float32 or \
                norm.numel() != 1:
            raise ValueError(f"norm must be one fp32 element on device {self.device_index}")
        else:
            given = norm.data_ptr()
        _refuse_overlaps(at, to, given, self._bytes)
        scratch = self._new(self._scratch_bytes, torch.uint8, stream)
        if unit_norms is not None:                 # (an empty tensor has no address)
            units, count = unit_norms.data_ptr() or scratch.data_ptr(), unit_norms.numel()
        handle = torch._C._cuda_getCurrentRawStream(self.device_index) if stream is None else stream.cuda_stream
        if handle != self._made_on:                # the table's memory is not given away before that stream is done with it
            self._table.record_stream(torch.cuda.current_stream(self._device) if stream is None else stream)
        plan, fn = self._h, N.load().gnmr_clip_run
        places = ctypes.c_void_p * len(at)
        args = (plan, self._table.data_ptr(), places(*at), None if to is None else places(*to), max_norm, units, count, norm.data_ptr(), scratch.data_ptr(), self._scratch_bytes, handle)
        keep = (norm, grads, outs, unit_norms, scratch, self._table)          # storage the prepared call points into

        def run():
            if self._h != plan:
                raise ValueError("the plan was closed")
            status = fn(*args)
            if status:
                N._check(status, None)
            return keep[0]

        return run

    def clip(self, grads, max_norm, *, out=None, unit_norms=None, norm=None, stream=None):
        """Enqueues one pass and returns the norm before scaling, an fp32 tensor (`norm`, if given).

        grads: tensors of the plan's sizes and types, no two of which overlap, scaled where they lie, or, with out (as many, of the same types), left as
        they are and written there, scaled or not (out[i] may be grads[i], and overlaps no other).  Tensors that
        overlap otherwise, or a `norm` among them, are refused.  max_norm: 0 or more; infinity only takes the norm.
        unit_norms: fp64 tensor of the norms of parts that make up the gradients, as the monitor's stats["norm"]
        after a step on the same arena: the norm is formed from them, and no gradient is read for it."""
        return self.prepare_clip(grads, max_norm, out=out, unit_norms=unit_norms, norm=norm, stream=stream)()
