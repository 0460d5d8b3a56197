"""The norm over many gradients and the clipping against 64 bits: mixed types, lengths from none to millions, odd starts,
other memory and in place, limits, the monitor's norms in place of a pass, values at the ends of the types' ranges.

Tolerances, u = 2^-24.  A lane adds the squares of at most 16 rounds of 8 vectors before it goes on in pairs of floats: no square passes
through more than 32 fp32 roundings, the lanes' fractions round once more: the sum of squares is at most 34 u off, the norm half that
and its rounding to fp32: 18 u.  The scale has the norm's error in 64 bits and a rounding, an output one in fp32 and its type's."""
import pytest

from paper_2606_00539_gb300 import GnmrError, GradientClip, Monitor

pytestmark = pytest.mark.gpu

import torch  # noqa: E402

from tests.test_gpu_products import LEAST, ROUND, TYPES, gen, normal  # noqa: E402

U = 2.0 ** -24
NAMES = {t: n for n, t in TYPES.items()}


def exact(tensors):
    return float(sum((t.double().square().sum() for t in tensors), torch.zeros((), dtype=torch.float64, device="cuda")).sqrt())


def check(norm, outs, grads, max_norm, total=None):
    total = exact(grads) if total is None else total
    assert norm.shape == () and norm.dtype == torch.float32
    if total >= torch.finfo(torch.float32).max * (1 + U):             # the norm's type has nothing larger than infinity
        assert norm.isinf()
    else:                                                            # below 2^-126 fp32 is a grid of 2^-149, half of which a rounding is off
        assert abs(norm.double().item() - total) <= 18 * U * total + 2.0 ** -150
    scale = min(1.0, max_norm / total) if total else 1.0
    for i, (o, x) in enumerate(zip(outs, grads)):
        want, kind = x.double() * scale, NAMES[x.dtype]
        # next to the limit the norm may be on its other side: a scale of 1
        tol = want.abs() * (20 * U + ROUND[kind] * (1 + 20 * U)) + LEAST[kind] + 2.0 ** -149
        bad = ~((o.double() - want).abs() <= tol)
        assert not bad.any(), f"tensor {i}: {int(bad.sum())} outside, {o[bad][0].item()} for {want[bad][0].item()}"


def views(g, lengths, kinds, gap=0, scale=1.0):
    """Tensors in one buffer for each type, each starting `gap` elements behind the one before it."""
    flat = {k: torch.full((sum(n + gap for n, q in zip(lengths, kinds) if q == k) + 1,), 7.0, dtype=TYPES[k], device="cuda") for k in set(kinds)}
    at, got = dict.fromkeys(flat, 0), []
    for n, k in zip(lengths, kinds):
        v = flat[k][at[k]:at[k] + n]
        v.copy_(normal(g, n, dtype=torch.float32, size=scale))
        got.append(v)
        at[k] += n + gap
    return got, flat


LAYOUTS = [
    ([1], ["f32"]), ([1], ["f16"]), ([0], ["bf16"]), ([], []), ([7], ["bf16"]), ([0, 3, 0, 0, 1], ["f32", "bf16", "f16", "f32", "f32"]),
    ([4096], ["bf16"]), ([1 << 20], ["f32"]), ([3_000_017], ["bf16"]), ([5] * 300, ["f32", "bf16", "f16"] * 100),
    ([1000, 2048, 2049, 33, 100000, 8, 1], ["bf16", "f32", "f16", "bf16", "f16", "f32", "bf16"]), ([777] * 64, ["f32"] * 64),
    ([513] * 65, ["bf16"] * 65), ([129] * 401, ["f16"] * 401), ([31] * 1901, ["f32"] * 1901), ([17] * 4100, ["bf16", "f32"] * 2050),
]


@pytest.mark.parametrize("gap", [0, 1, 8])
@pytest.mark.parametrize("case", range(len(LAYOUTS)))
def test_norm_and_scale(case, gap):
    lengths, kinds = LAYOUTS[case]
    g = gen(case + 100 * gap)
    grads, flat = views(g, lengths, kinds, gap)
    outs, out_flat = views(g, lengths, kinds, gap)
    total = exact(grads)
    before = {k: f.clone() for k, f in flat.items()}
    for f in out_flat.values():
        f.fill_(7.0)
    with GradientClip(grads) as plan:
        for limit in (0.25, 3.0):
            norm = plan.clip(grads, limit * total, out=outs)
            check(norm, outs, grads, limit * total, total)
            assert all(torch.equal(flat[k], before[k]) for k in flat)
            assert limit < 1 or all(torch.equal(a, b) for a, b in zip(outs, grads))
        for k, f in out_flat.items():                                # what lies between the tensors
            taken = torch.zeros(len(f), dtype=torch.bool, device="cuda")
            for o in outs:
                if o.dtype == f.dtype and len(o):
                    taken[o.storage_offset():o.storage_offset() + len(o)] = True
            assert (f[~taken] == 7).all()
        want = [o.clone() for o in outs]
        norm = plan.clip(grads, 3 * total)                           # in place, below the limit
        check(norm, grads, grads, 3 * total, total)
        assert all(torch.equal(flat[k], before[k]) for k in flat)
        norm = plan.clip(grads, 0.25 * total)                        # and above it
        old = [before[NAMES[v.dtype]][v.storage_offset():v.storage_offset() + len(v)] for v in grads]
        check(norm, grads, old, 0.25 * total, total)
        assert want is not None and abs(exact(grads) - 0.25 * total) <= 2.0 ** -8 * total


def test_outputs_that_start_otherwise_than_the_gradients():
    g = gen(1)
    for kind in ("bf16", "f32", "f16"):
        x = normal(g, 5000, dtype=TYPES[kind])
        to = torch.zeros(5016, dtype=TYPES[kind], device="cuda")
        for a in (0, 1, 3):
            for b in (0, 2, 5):
                grads, outs = [x[a:a + 4000]], [to[b:b + 4000]]
                with GradientClip(grads) as plan:
                    check(plan.clip(grads, 1.0, out=outs), outs, grads, 1.0)


def test_limits():
    g = gen(2)
    x = [normal(g, 1000, dtype=torch.float32), normal(g, 300, dtype=torch.bfloat16)]
    old = [v.clone() for v in x]
    with GradientClip(x) as plan:
        assert abs(plan.clip(x, float("inf")).item() - exact(old)) < 1e-4 and all(torch.equal(a, b) for a, b in zip(x, old))
        out = [torch.empty_like(v) for v in x]
        plan.clip(x, 0.0, out=out)
        assert all((v == 0).all() for v in out)
        zero = [torch.zeros_like(v) for v in x]
        assert plan.clip(zero, 0.0).item() == 0 and all((v == 0).all() for v in zero)
        for bad in (-1.0, float("nan")):
            with pytest.raises(ValueError, match="max_norm"):
                plan.clip(x, bad)


@pytest.mark.parametrize("kind,size", [("f32", 1e-30), ("f32", 1e-42), ("f32", 1e30), ("f32", 3e37), ("bf16", 1e-30), ("bf16", 1e36),
                                       ("f16", 6e-8), ("f16", 6e4)])
def test_values_whose_squares_leave_the_range(kind, size):
    """The norm is right where squares are past fp32, or below it, beside ordinary tensors, and the scale with it."""
    g = gen(3)
    x = [(normal(g, 3000, dtype=torch.float64).clamp(-1, 1) * size).to(TYPES[kind])]
    total = exact(x)
    with GradientClip(x) as plan:
        out = [torch.empty_like(x[0])]
        check(plan.clip(x, total / 3, out=out), out, x, total / 3)
    if kind == "f32" and size > 1:
        y = [x[0], normal(g, 9, dtype=torch.float32)]
        with GradientClip(y) as plan:
            out = [torch.empty_like(v) for v in y]
            check(plan.clip(y, total / 3, out=out), out, y, total / 3)


def test_a_norm_past_fp32_still_scales():
    x = [torch.full((100,), 3e38, device="cuda")]
    with GradientClip(x) as plan:
        norm = plan.clip(x, 1.0)
        assert norm.isinf() and torch.allclose(x[0], torch.full_like(x[0], 0.1))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_norm_that_is_not_finite_scales_nothing(bad):
    g = gen(4)
    x = [normal(g, 1000, dtype=torch.float32), normal(g, 5000, dtype=torch.bfloat16)]
    x[1][777] = bad
    old = [v.clone() for v in x]
    with GradientClip(x) as plan:
        norm = plan.clip(x, 0.1)
        out = [torch.zeros_like(v) for v in x]
        plan.clip(x, 0.1, out=out)
    assert not norm.isfinite() and norm.isnan() == (bad != bad)
    for a, b, c in zip(x, old, out):
        assert torch.equal(a.nan_to_num(123.0), b.nan_to_num(123.0)) and torch.equal(c.nan_to_num(123.0), b.nan_to_num(123.0))


def test_the_monitors_norms():
    """After a step on the arena: the same limit, with and without the monitor's norms; and many of them."""
    g = gen(5)
    lengths = [640, 13, 4096, 100000, 7]
    off, pos = [], 0
    for n in lengths:
        off.append(pos)
        pos += (n + 3) // 4 * 4
    arena = torch.zeros(pos, device="cuda")
    for o, n in zip(off, lengths):
        arena[o:o + n] = normal(g, n, dtype=torch.float32)
    mon = Monitor(off, lengths, dtype="f32")
    stats = mon.new_stats()
    mon.step(arena, stats=stats)
    old = arena.clone()
    with GradientClip([arena]) as plan:
        norm = plan.clip([arena], 10.0, unit_norms=stats["norm"])
        check(norm, [arena], [old], 10.0)
        many = torch.rand(200_001, dtype=torch.float64, device="cuda", generator=g)
        out = [torch.empty_like(old)]
        norm = plan.clip([old], 5.0, unit_norms=many, out=out)
        total = float(many.square().sum().sqrt())
        assert abs(norm.item() - total) <= 2 * U * total
        assert torch.allclose(out[0], old * (5.0 / total), rtol=1e-6, atol=0)
        none = plan.clip([old], 5.0, unit_norms=many[:0], out=out)
        assert none.item() == 0 and torch.equal(out[0], old)
    mon.close()


@pytest.mark.parametrize("size", [1e-170, 1e-150, 1e-140, 1e-100, 1e-30, 1.0, 3.0, 1e10, 1e38, 1e100, 1e150])
def test_roots_over_the_range_of_64_bits(size):
    """Norms that a caller gives may be anything whose square is a number; the limit is right for each (norm / 8, so exactly 1 / 8)."""
    x = [torch.full((5,), 8.0, device="cuda")]
    out = [torch.zeros(5, device="cuda")]
    with GradientClip(x) as plan:
        for k in (1.0, 1.7, 2.0, 3.1):
            units = torch.tensor([3.0, 4.0], dtype=torch.float64, device="cuda") * (size * k)
            norm = plan.clip(x, 5.0 * size * k / 8, unit_norms=units, out=out)
            want = 5.0 * size * k
            if want * want < 1e-300:                             # squares below 64 bits' normal numbers keep fewer
                continue
            assert (out[0].double() - 1).abs().max() <= 2 * U
            assert norm.isinf() if want > 3.5e38 else abs(norm.double().item() - want) <= 2 * U * want + 2.0 ** -150


def test_prepared_captured_and_from_two_streams():
    g = gen(6)
    x = [normal(g, 300_000, dtype=torch.bfloat16), normal(g, 70_001, dtype=torch.float32)]
    outs = [[torch.zeros_like(v) for v in x] for _ in range(3)]
    plan = GradientClip(x)
    plan.clip(x, 5.0, out=outs[2])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    calls = [plan.prepare_clip(x, 5.0, out=o, stream=s) for s, o in zip(streams, outs)]
    for _ in range(20):
        norms = [c() for c in calls]
    torch.cuda.synchronize()
    assert norms[0] is calls[0]() and torch.equal(norms[0], norms[1])
    for o in outs[:2]:
        assert all(torch.equal(a, b) for a, b in zip(o, outs[2]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = plan.clip(x, 5.0, out=outs[0])
    x[0].mul_(0.5)
    graph.replay()
    graph.replay()
    check(norm, outs[0], x, 5.0)
    other = [v.clone() for v in x]                                   # the plan goes by the call's tensors
    other[0].mul_(4)
    check(plan.clip(other, 5.0, out=outs[1]), outs[1], other, 5.0)
    plan.close()
    with pytest.raises(ValueError, match="closed"):
        calls[0]()
    with pytest.raises(ValueError, match="closed"):
        plan.clip(x, 1.0)


def test_plans_come_and_go_while_a_stream_is_captured():
    """A plan that is freed during a capture, as when a name is bound anew there, does not end the capture; the same for a
    prepared call.  Calls that were enqueued on another stream before their plan went are what they were."""
    g = gen(8)
    x = [normal(g, 5000, dtype=torch.float32), normal(g, 77, dtype=torch.bfloat16)]
    out = [torch.zeros_like(v) for v in x]
    old = GradientClip(x)
    call = old.prepare_clip(x, 1.0, out=out)
    plan = GradientClip(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = plan.clip(x, 2.0, out=out)
        del old
        call = None
    graph.replay()
    check(norm, out, x, 2.0)
    side = torch.cuda.Stream()
    for _ in range(50):
        plan = GradientClip(x)
        norm = plan.clip(x, 2.0, out=out, stream=side)
        del plan
        torch.full((1 << 10,), 7, dtype=torch.uint8, device="cuda")          # would land where the table was
    torch.cuda.synchronize()
    check(norm, out, x, 2.0)
    assert call is None


def test_offsets_past_31_bits():
    n = (1 << 31) + (1 << 20) + 3
    x = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    x[-3:] = 4.0
    x[0] = 1.0
    with GradientClip([x]) as plan:
        norm = plan.clip([x], 3.5)
    assert norm.item() == 7.0 and (x[-3:] == 2.0).all() and x[0] == 0.5 and x[n // 2] == 0


def test_outputs_where_gradients_lie():
    """out[i] may be grads[i]; where it is another gradient, which is still to be read, the call is refused."""
    g = torch.Generator(device="cuda").manual_seed(5)
    x = [torch.randn(5000, device="cuda", generator=g) for _ in range(3)]
    was = [t.clone() for t in x]
    with GradientClip(x) as plan:
        other = torch.empty_like(x[0])
        for out in ([x[1], x[0], x[2]], [x[0], x[2], other], [other, x[1], x[0]]):
            with pytest.raises(ValueError, match="another gradient"):
                plan.clip(x, 1.0, out=out)
        assert all(torch.equal(a, b) for a, b in zip(x, was))
        norm = plan.clip(x, 1.0, out=[x[0], other, x[2]])
        coef = torch.tensor(1.0, device="cuda") / norm           # half steps: the norm, the division and the product here, the last two there
        assert all(torch.allclose(a, b * coef, rtol=6 * 2.0 ** -24, atol=0) for a, b in zip((x[0], other, x[2]), was))
        assert torch.equal(x[1], was[1])


def test_refusals():
    x = [torch.zeros(10, device="cuda"), torch.zeros(4, dtype=torch.bfloat16, device="cuda")]
    for tensors in ([x[0].double()], [3], [x[0].int()]):
        with pytest.raises(ValueError, match="must be"):
            GradientClip(tensors)
    with pytest.raises(GnmrError):
        GradientClip(x, device=99)
    with GradientClip(x) as plan:
        for call, why in [
            (lambda: plan.clip(x[:1], 1.0), "2 tensors"), (lambda: plan.clip([x[0], x[0]], 1.0), "contiguous elements"),
            (lambda: plan.clip([x[0].cpu(), x[1]], 1.0), "CUDA"), (lambda: plan.clip([torch.zeros(20, device="cuda")[::2], x[1]], 1.0), "contiguous"),
            (lambda: plan.clip(x, 1.0, out=x[:1]), "out must"), (lambda: plan.clip(x, 1.0, unit_norms=x[0]), "unit_norms"),
            (lambda: plan.clip(x, 1.0, norm=x[0]), "norm must"), (lambda: GradientClip([x[0], x[0]]).clip([x[0], x[0]], 1.0), "twice"),
            (lambda: GradientClip([x[0], x[0]]).clip([x[0], x[0].clone()], 1.0, out=[x[0], x[0]]), "twice"),
        ]:
            with pytest.raises(ValueError, match=why):
                call()


def test_tensors_that_overlap_are_refused_and_left_as_they_are():
    flat, to = torch.ones(64, device="cuda"), torch.ones(64, device="cuda")
    with GradientClip([flat[:10], flat[:10]]) as plan:
        for grads, out, why in (([flat[0:10], flat[5:15]], None, "twice"), ([flat[0:10], flat[20:30]], [to[0:10], to[9:19]], "twice"),
                                ([flat[0:10], flat[20:30]], [flat[40:50], flat[9:19]], "another gradient")):
            with pytest.raises(ValueError, match=why):
                plan.clip(grads, 1.0, out=out)
        with pytest.raises(ValueError, match="twice"):
            plan.clip([flat[0:10], flat[10:20]], 1.0, norm=flat[19])
        assert (flat == 1).all() and (to == 1).all()
        norm = plan.clip([flat[10:20], flat[0:10]], 1.0, norm=flat[20])                # neighbours
        assert norm.item() == flat[20].item() and abs(norm.item() - 20 ** 0.5) <= 18 * U * 20 ** 0.5
        assert (flat[21:] == 1).all() and ((flat[:20].double() - 20 ** -0.5).abs() <= 20 * U).all()


@pytest.mark.parametrize("gap", [0, 1, 8])
@pytest.mark.parametrize("case", range(len(LAYOUTS)))
def test_in_place_and_into_other_memory_give_the_same_bits(case, gap):
    """The same norm, the same scale and one product for each element, whichever kernel's shares it falls in; and what lies between stays."""
    lengths, kinds = LAYOUTS[case]
    g = gen(case + 100 * gap + 7)
    grads, flat = views(g, lengths, kinds, gap)
    outs, _ = views(g, lengths, kinds, gap)
    total = exact(grads)
    was = {k: f.clone() for k, f in flat.items()}
    with GradientClip(grads) as plan:
        for limit in (0.25, 0.9, 1.5):
            norm = plan.clip(grads, limit * total, out=outs)
            at = plan.clip(grads, limit * total)
            assert torch.equal(norm, at) and all(torch.equal(a, b) for a, b in zip(grads, outs))
            for k, f in flat.items():
                between = torch.ones(len(f), dtype=torch.bool, device="cuda")
                for v in grads:
                    if NAMES[v.dtype] == k:
                        between[v.storage_offset():v.storage_offset() + len(v)] = False
                assert torch.equal(f[between], was[k][between])
                f.copy_(was[k])
