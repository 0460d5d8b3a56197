"""Which memory a clipping call takes: the check comes before any CUDA call, so that the host's memory will do."""
import pytest
import torch

from paper_2606_00539_gb300 import GradientClip
from paper_2606_00539_gb300 import build as native_build
from paper_2606_00539_gb300 import clip as module
from paper_2606_00539_gb300 import products


@pytest.fixture(scope="module", autouse=True)
def library():
    native_build.build()
    if products.torch is None:
        products._load_torch()
    module.torch = torch


class HostPlan(GradientClip):
    """A plan whose tensors are the host's.  Calls are prepared, none is made."""

    def __init__(self, tensors):
        self._h, self._table, self.device_index = 1, tensors[0], -1
        self._lengths, self._dtypes = [t.numel() for t in tensors], [t.dtype for t in tensors]
        self._bytes = [t.numel() * t.element_size() for t in tensors]
        self._made_on = self.cuda_stream = self._scratch_bytes = 0

    def _new(self, shape, dtype, stream):
        return torch.empty(shape, dtype=dtype)

    def close(self):
        pass

    def take(self, grads, out=None, norm=None):
        assert callable(self.prepare_clip(grads, 1.0, out=out, norm=norm, stream=self))


def parts(t, *spans):
    return [t[i:j] for i, j in spans]


def test_memory_that_is_written_twice_or_still_to_be_read():
    """Neighbours may touch; ranges that meet in an element are refused, wherever each of them begins and in whatever order they come."""
    flat, to = torch.zeros(64), torch.zeros(64)
    free = parts(to, (0, 10), (10, 20), (20, 23))
    plan = HostPlan(free)
    apart = parts(flat, (10, 20), (0, 10), (20, 23))
    plan.take(apart)
    plan.take(apart, out=parts(to, (3, 13), (13, 23), (0, 3)))
    plan.take(apart, out=apart)                                      # each where it lies
    plan.take(apart, out=[apart[0], *parts(to, (0, 10), (10, 13))])
    plan.take(apart, out=parts(flat, (23, 33), (33, 43), (43, 46)))
    plan.take(parts(flat, (0, 10), (5, 15), (7, 10)), out=free)      # only read
    for spans in ([(0, 10), (5, 15), (20, 23)], [(5, 15), (0, 10), (20, 23)], [(0, 10), (10, 20), (9, 12)], [(0, 10), (20, 30), (3, 6)],
                  [(0, 10), (0, 10), (20, 23)], [(20, 30), (0, 10), (29, 32)]):
        with pytest.raises(ValueError, match="twice"):
            plan.take(parts(flat, *spans))
        with pytest.raises(ValueError, match="twice"):
            plan.take(free, out=parts(flat, *spans))
    for out in ([apart[1], apart[0], apart[2]], parts(flat, (11, 21), (30, 40), (50, 53)), parts(flat, (30, 40), (1, 11), (50, 53)),
                parts(flat, (30, 40), (50, 60), (19, 22)), parts(flat, (30, 40), (50, 60), (4, 7)), parts(flat, (22, 32), (50, 60), (40, 43))):
        with pytest.raises(ValueError, match="another gradient"):
            plan.take(apart, out=out)


def test_a_norm_where_a_tensor_lies():
    flat, to = torch.zeros(24), torch.zeros(24)
    plan = HostPlan([flat[:10], flat[10:20]])
    grads, outs = parts(flat, (10, 20), (0, 10)), parts(to, (0, 10), (10, 20))
    plan.take(grads, norm=flat[23])
    plan.take(grads, out=outs, norm=to[20:21])
    for out, norm, why in ((None, flat[19], "twice"), (None, flat[0], "twice"), (outs, to[10], "twice"), (outs, flat[7], "another gradient")):
        with pytest.raises(ValueError, match=why):
            plan.take(grads, out=out, norm=norm)


def test_ranges_are_bytes_and_empty_tensors_have_none():
    memory = torch.zeros(64, dtype=torch.uint8)
    f32, bf16 = memory.view(torch.float32), memory.view(torch.bfloat16)
    plan = HostPlan([f32[:2], bf16[:3], f32[:0], bf16[:0]])
    plan.take([f32[2:4], bf16[1:4], f32[3:3], bf16[5:5]])
    plan.take([f32[2:4], bf16[8:11], torch.empty(0), bf16[9:9]])
    for at in (2, 4, 7):
        with pytest.raises(ValueError, match="twice"):
            plan.take([f32[2:4], bf16[at:at + 3], f32[:0], bf16[:0]])
    HostPlan([f32[:0], f32[:0]]).take([f32[:0], f32[:0]], out=[f32[:0], f32[:0]])
    HostPlan([f32[:4]]).take([f32[:4]])


def test_thousands_of_tensors():
    many = torch.zeros(3000 * 5)
    rows = [many[5 * i:5 * i + 5] for i in reversed(range(3000))]
    plan = HostPlan(rows)
    plan.take(rows)
    plan.take(rows, out=[t.clone() for t in rows])
    with pytest.raises(ValueError, match="twice"):
        plan.take(rows[:2999] + [rows[1234]])
    with pytest.raises(ValueError, match="twice"):
        plan.take(rows[:2999] + [many[7002:7007]])
    with pytest.raises(ValueError, match="another gradient"):
        plan.take(rows, out=rows[:1500] + [t.clone() for t in rows[1500:2999]] + [rows[1600]])
