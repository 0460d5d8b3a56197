"""Gated feed-forward blocks against the definition in 64 bits: types, activations, strides, groupings, masks,
rows of no group, non-finite values, and the gradient of the two projections.

Tolerances.  With u = 2^-23: a projection's sum is off by at most E = (128 + k / 512) u S, S the sum of the terms'
magnitudes (tests of the products say why).  h = act(a) b then is off by at most 1.13 E_a |b| + |act(a)| E_b + E_a E_b
(no slope of either activation is above 1.13), and by what fp32 makes of the formula: exp is off by 2 + 1.2 |a| u, erfc by 4 u and
its argument's rounding, (a^2 + 2) u, and eight u cover the other operations: (8 + 1.2 |a| + a^2) u |h|.  The slopes' formulas are
bounded likewise, term by term.  Results under fp32's smallest normal number, 2^-126, may be lost.  The output's own rounding is half a step."""
import numpy as np
import pytest

from paper_2606_00539_gb300 import ExpertProducts, expert_gated, expert_linear

pytestmark = pytest.mark.gpu

import torch  # noqa: E402

from tests.test_gpu_products import LEAST, ROUND, TYPES, gen, normal, offsets_of, spans  # noqa: E402

U = 2.0 ** -23
LOST = 2.0 ** -126


@pytest.fixture(scope="module")
def products():
    p = ExpertProducts(device=0)
    yield p
    p.close()


def act(a, kind):
    """act(a), act'(a) in 64 bits."""
    if kind == "silu":
        s = torch.sigmoid(a)
        return a * s, s + a * s * torch.sigmoid(-a)
    p = 0.5 * torch.erfc(-a * 0.5 ** 0.5)
    return a * p, p + a * torch.exp(-a * a / 2) / (2 * np.pi) ** 0.5


def close(got, want, tol, kind):
    got = got.double()
    tol = tol + ROUND[kind] * (want.abs() + tol) + LEAST[kind]
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (f"{int(bad.sum())} of {bad.numel()} outside, first at {bad.nonzero()[0].tolist()}: "
                           f"{got[bad][0].item()} for {want[bad][0].item()}")


def check_h(h, keep, x, w, kind, name):
    n, k = w.shape[0] // 2, w.shape[1]
    ab = x.double() @ w.double().T
    err = (128 + k / 512) * U * (x.double().abs() @ w.double().abs().T)
    if keep is not None:
        close(keep, ab, err, name)
    a, b, ea, eb = ab[:, :n], ab[:, n:], err[:, :n], err[:, n:]
    v, _ = act(a, kind)
    close(h, v * b, 1.13 * ea * b.abs() + v.abs() * eb + 1.13 * ea * eb + (8 + 1.2 * a.abs() + a * a) * U * (v * b).abs() +
          LOST * (1 + a.abs()) * (1 + b.abs()), name)


# groups' rows, n, n_in: single rows, odd sizes, tiles of outputs (128) and rows and their edges, split contractions
SHAPES = [
    ([1], 8, 8), ([1], 1, 1), ([3], 5, 7), ([17], 64, 64), ([1], 128, 512), ([5], 500, 136), ([33], 127, 200),
    ([255], 129, 264), ([256], 128, 64), ([257], 256, 1024), ([700], 100, 2056), ([0], 40, 48), ([0, 0, 0], 40, 48),
    ([1, 0, 2, 0, 0, 31, 33], 136, 200), ([64, 65, 63, 1], 131, 129), ([300, 0, 511, 16, 15, 17, 1], 160, 520),
    ([2] * 40, 132, 72), ([1100, 3], 48, 88), ([31] * 3, 1003, 371), ([40], 64, 4096),
]


@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_forward(products, case, dtype, kind):
    counts, n, k = SHAPES[case]
    g, t, G, R = gen(case), TYPES[dtype], len(counts), sum(counts)
    x, w = normal(g, R, k, dtype=t), normal(g, G, 2 * n, k, dtype=t, size=2 * k ** -0.5)
    off = offsets_of(counts)
    keep = torch.empty(R, 2 * n, dtype=t, device="cuda")
    h = products.gated(x, w, off, activation=kind, keep=keep)
    bare = products.gated(x, w, off, activation=kind)
    assert torch.equal(h, bare) and h.shape == (R, n) and h.dtype == t
    for e, at in spans(counts):
        check_h(h[at], keep[at], x[at], w[e], kind, dtype)


def test_strides_and_what_lies_around(products):
    """Operands and outputs inside larger buffers, at odd starts; nothing around them is written."""
    counts, n, k = [37, 0, 129], 70, 200
    t, g, R = torch.bfloat16, gen(5), 166
    off = offsets_of(counts)
    for pad, lead in ((0, 0), (8, 8), (3, 1), (1, 16), (5, 2)):
        x = normal(g, R, k + pad + lead, dtype=t)[:, lead:lead + k]
        flat = normal(g, lead + 3 * (2 * n * k + 24 + pad), dtype=t, size=0.1)
        w = torch.as_strided(flat, (3, 2 * n, k), (2 * n * k + 24 + pad, k, 1), lead)
        out = torch.full((R, n + pad + lead + 1), 7.0, device="cuda", dtype=t)
        kept = torch.full((R, 2 * n + pad + lead + 1), 7.0, device="cuda", dtype=t)
        h, keep = out[:, lead:lead + n], kept[:, lead:lead + 2 * n]
        assert products.gated(x, w, off, out=h, keep=keep) is h
        for m, wide in ((out, n), (kept, 2 * n)):
            assert (m[:, :lead] == 7).all() and (m[:, lead + wide:] == 7).all()
        for e, at in spans(counts):
            check_h(h[at], keep[at], x[at], w[e], "silu", "bf16")


def test_one_weight_for_all_groups_and_rows_of_none(products):
    """A group stride of zero, a mask of any stride, rows before the first group and behind the last: left as they were."""
    counts, n, k, t, g = [9, 70, 0, 40], 72, 136, torch.float16, gen(8)
    first, R = 6, 140
    x, w = normal(g, R, k, dtype=t), normal(g, 2 * n, k, dtype=t, size=0.2)
    mask = torch.tensor([1, 9, 0, 9, 1, 9, 255, 9], dtype=torch.uint8, device="cuda")[::2]
    h, keep = torch.full((R, n), 7.0, device="cuda", dtype=t), torch.full((R, 2 * n), 7.0, device="cuda", dtype=t)
    products.gated(x, w.expand(4, 2 * n, k), offsets_of(counts, first), out=h, keep=keep, mask=mask)
    done = torch.zeros(R, dtype=torch.bool, device="cuda")
    for e, at in spans(counts, first):
        if mask[e]:
            check_h(h[at], keep[at], x[at], w, "silu", "f16")
            done[at] = True
    assert (h[~done] == 7).all() and (keep[~done] == 7).all() and 0 < done.sum() < R


def test_non_finite_values_stay_in_their_rows(products):
    """Of the activations: in the row; of a gate's row of weights: in the column; of the values behind a group: nowhere."""
    n, k, t, g = 150, 264, torch.bfloat16, gen(9)
    x, w = normal(g, 90, k, dtype=t), normal(g, 2 * n, k, dtype=t, size=0.1)
    clean = products.gated(x, w)
    x[40, 3], x[41, 5] = float("nan"), float("inf")
    h = products.gated(x, w)
    keep = torch.ones(90, dtype=torch.bool, device="cuda")
    keep[40:42] = False
    assert torch.equal(h[keep], clean[keep]) and h[40].isnan().all() and not h[41].isfinite().any()
    x[40:42] = 1
    w[n + 3, 7] = float("nan")
    h = products.gated(x, w)
    assert h[:, 3].isnan().all() and h[:, :3].isfinite().all() and h[:, 4:].isfinite().all()


def test_extreme_gates(products):
    """Gates far beyond exp's range: silu and gelu are then a or nothing."""
    k, t = 8, torch.bfloat16
    x = torch.tensor([1e4, 200, 90, 88, 30, 1, -1, -30, -88, -90, -200, -1e4], device="cuda")[:, None]
    x = torch.cat([x, torch.ones_like(x), torch.zeros(12, k - 2, device="cuda")], 1).to(t)
    w = torch.zeros(2, k, device="cuda", dtype=t)
    w[0, 0], w[1, 1] = 1, 3
    for kind in ("silu", "gelu"):
        check_h(products.gated(x, w, activation=kind), None, x, w, kind, "bf16")


@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,n,pad,lead", [(1, 1, 0, 0), (1, 8, 0, 0), (7, 5, 0, 0), (33, 1408, 0, 0), (64, 136, 8, 8),
                                             (19, 136, 3, 0), (50, 1003, 0, 1), (3, 13824, 0, 0), (0, 8, 0, 0)])
def test_gate_and_its_gradient(products, rows, n, pad, lead, dtype, kind):
    g, t = gen(rows + n), TYPES[dtype]
    wide = pad + lead
    dh = normal(g, rows, n + wide, dtype=t)[:, lead:lead + n]
    ab = normal(g, rows, 2 * n + wide, dtype=t, size=3.0)[:, lead:lead + 2 * n]
    out = torch.full((rows, 2 * n + wide + 1), 7.0, device="cuda", dtype=t)
    dab = products.gate_grad(dh, ab, activation=kind, out=out[:, lead:lead + 2 * n])
    assert (out[:, :lead] == 7).all() and (out[:, lead + 2 * n:] == 7).all()
    h = products.gate(ab, activation=kind)
    d, a, b = dh.double(), ab[:, :n].double(), ab[:, n:].double()
    v, slope = act(a, kind)
    m = a.abs()
    rough = (8 + 1.2 * m + a * a) * U
    close(h, v * b, rough * (v * b).abs() + LOST * (1 + m) * (1 + b.abs()), dtype)
    close(dab[:, n:], d * v, rough * (d * v).abs() + LOST * (1 + m) * (1 + d.abs()), dtype)
    if kind == "silu":
        s = torch.sigmoid(a)
        err = U * ((8 + 1.2 * m) * (slope.abs() + s * s * m) + 4 * s * (1 + m))
    else:
        p, tail = 0.5 * torch.erfc(-a * 0.5 ** 0.5), m * torch.exp(-a * a / 2) / (2 * np.pi) ** 0.5
        err = U * ((8 + a * a) * p + (8 + 1.2 * a * a) * tail + slope.abs())
    close(dab[:, :n], d * b * slope, (d * b).abs() * (err + LOST * (1 + m)) + 4 * U * (d * b * slope).abs(), dtype)
    same = products.gate_grad(dh.contiguous(), ab.contiguous(), activation=kind)
    assert torch.equal(same, dab)
    own = ab.clone()
    assert products.gate_grad(dh, own, out=own, activation=kind) is own and torch.equal(own, dab)


def test_gate_takes_the_other_paths_groups(products):
    """h of groups whose entry is 0; others, and rows of no group, are left."""
    counts, n, first, R = [5, 0, 33, 1, 7], 24, 2, 60
    g = gen(4)
    ab = normal(g, R, 2 * n, dtype=torch.bfloat16)
    mask = torch.tensor([0, 0, 1, 0, 1], dtype=torch.uint8, device="cuda")
    out = torch.full((R, n), 7.0, device="cuda", dtype=torch.bfloat16)
    products.gate(ab, offsets_of(counts, first), out=out, mask=mask)
    every = products.gate(ab)
    done = torch.zeros(R, dtype=torch.bool, device="cuda")
    for e, at in spans(counts, first):
        done[at] = not mask[e]
    assert torch.equal(out[done], every[done]) and (out[~done] == 7).all() and done.sum() == 6
    only = products.gate(ab, mask=mask[2:3], out=torch.full_like(out, 7.0))
    assert (only == 7).all()


def test_offsets_out_of_range_and_falling_are_taken_as_the_nearest_allowed(products):
    n, k, R, g = 24, 40, 50, gen(6)
    x, w = normal(g, R, k, dtype=torch.bfloat16), normal(g, 4, 2 * n, k, dtype=torch.bfloat16, size=0.2)
    off = torch.tensor([-5, 20, 10, 1 << 40, 7], dtype=torch.int64, device="cuda")
    h = products.gated(x, w, off)
    for e, at in ((0, slice(0, 20)), (2, slice(20, 50))):
        check_h(h[at], None, x[at], w[e], "silu", "bf16")
    out = torch.full((R, n), 7.0, dtype=torch.bfloat16, device="cuda")
    ab = normal(g, R, 2 * n, dtype=torch.bfloat16)
    products.gate(ab, off, out=out, mask=torch.tensor([0, 1, 1, 0], dtype=torch.uint8, device="cuda"))
    assert torch.equal(out[:20], products.gate(ab)[:20]) and (out[20:] == 7).all()


def test_repeated_captured_and_on_another_stream(products):
    counts, n, k, t, g = [120, 7, 300], 136, 264, torch.bfloat16, gen(11)
    x, w, off = normal(g, 427, k, dtype=t), normal(g, 3, 2 * n, k, dtype=t, size=0.1), offsets_of(counts)
    dh = normal(g, 427, n, dtype=t)
    keep = torch.empty(427, 2 * n, dtype=t, device="cuda")
    want = products.gated(x, w, off, keep=keep).clone(), keep.clone(), products.gate_grad(dh, keep).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = products.gated(x, w, off, keep=keep, stream=side)
    dab = products.gate_grad(dh, keep, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((got, keep, dab), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h = products.gated(x, w, off, keep=keep)
        dab = products.gate_grad(dh, keep)
    x.copy_(normal(g, 427, k, dtype=t))
    for _ in range(3):
        graph.replay()
    again = products.gated(x, w, off, keep=keep)
    assert torch.equal(h, again) and not torch.equal(h, want[0]) and torch.equal(dab, products.gate_grad(dh, keep))


def test_offsets_past_31_bits_of_elements(products):
    """Rows whose elements lie beyond 2^31 in every buffer: the last ones of a tall batch."""
    R, n, k, t = (1 << 21) + 9, 512, 8, torch.bfloat16
    x = torch.zeros(R, k, dtype=t, device="cuda")
    g = gen(12)
    x[-20:] = normal(g, 20, k, dtype=t)
    w = normal(g, 2 * n, k, dtype=t)
    keep = torch.empty(R, 2 * n, dtype=t, device="cuda")
    h = products.gated(x, w, keep=keep)
    check_h(h[-20:], keep[-20:], x[-20:], w, "silu", "bf16")
    dab = products.gate_grad(h, keep, out=keep)
    ab = x[-20:].double() @ w.double().T
    v, _ = act(ab[:, :n], "silu")
    assert torch.allclose(dab[-20:, n:].double(), v * v * ab[:, n:], rtol=2.0 ** -5, atol=1e-3)


def codes(x, dim):
    top = x.float().abs().amax(dim, keepdim=True)
    return (x.float() * (127 * (1 / top))).round().double() * (top / 127).double()


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_layer_on_both_paths(products, kind):
    """expert_gated forward and backward, masked and not, against autograd in 64 bits on the same path.  On the low-cost
    path the codes are those of what the path holds: a rounding to bf16 of [a, b], or of its gradient, in between."""
    counts, n, k, t, g = [40, 0, 70, 33], 72, 136, torch.bfloat16, gen(20)
    x = normal(g, 143, k, dtype=t).requires_grad_()
    w = normal(g, 4, 2 * n, k, dtype=t, size=0.1).requires_grad_()
    dh, off = normal(g, 143, n, dtype=t), offsets_of(counts)
    mask = torch.tensor([1, 0, 0, 1], dtype=torch.uint8, device="cuda")
    for bits in (None, mask):
        arena = torch.full((4, 2 * n, k), 7.0, device="cuda")
        h = expert_gated(products, x, w, off, bits, arena, activation=kind)
        dx, = torch.autograd.grad(h, x, dh, retain_graph=True)
        free = expert_gated(products, x, w, off, bits, activation=kind)
        dx2, dw2 = torch.autograd.grad(free, (x, w), dh)
        assert torch.equal(h, free) and torch.equal(dx, dx2)
        for e, at in spans(counts):
            X, W, D = x.detach()[at].double(), w.detach()[e].double(), dh[at].double()
            low = bits is not None and not bits[e]
            ab = codes(x.detach()[at], 1) @ codes(w.detach()[e], 1).T if low and len(X) else X @ W.T
            a, b = (ab.to(t).double() if low else ab).chunk(2, 1)
            v, _ = act(a, kind)
            # a rounding that falls the other way where [a, b] lies next to a border: one more step of a and of b
            assert ((h[at].double() - v * b).abs() <= 2.0 ** -6 * ((v * b).abs() + a.abs() * b.abs()) + 2.0 ** -12).all()
            a, b = ab.to(t).double().chunk(2, 1)
            v, slope = act(a, kind)
            dab = torch.cat([D * b * slope, D * v], 1)
            size = torch.cat([D.abs() * (b.abs() * (slope.abs() + 1) + a.abs()), D.abs() * (v.abs() + a.abs())], 1)
            # dw: dab is a rounding (2^-8) and [a, b]'s (2^-8, through slopes under 1.13 and curvatures under 1) off
            off_by = 2.0 ** -6 * size
            assert ((arena[e].double() - dab.T @ X).abs() <= off_by.T @ X.abs() + 1e-4).all()
            assert ((dw2[e].double() - dab.T @ X).abs() <= off_by.T @ X.abs() + 2.0 ** -8 * (dab.T @ X).abs() + 1e-4).all()
            if not low:
                assert ((dx[at].double() - dab @ W).abs() <= off_by @ W.abs() + 2.0 ** -8 * (dab @ W).abs() + 1e-4).all()
            elif len(X):
                want = codes(dab.to(t), 1) @ codes(w.detach()[e], 0)
                # besides, a code of dab may fall the other way: a step is amax / 127
                step = dab.abs().amax(1, keepdim=True) / 127
                assert ((dx[at].double() - want).abs() <= (off_by + step) @ W.abs() * 1.02 + 2.0 ** -7 * want.abs() + 1e-4).all()
    before = arena.clone()
    expert_gated(products, x, w, off, mask, arena, add=True, activation=kind).backward(dh)
    assert torch.allclose(arena, 2 * before, rtol=1e-6, atol=1e-6)


def test_given_codes_and_masks_of_one_kind(products):
    """Codes of the weights made once give the same bits as made anew; with every expert on one path the other's calls write nothing."""
    counts, n, k, t, g = [40, 0, 70, 33], 72, 136, torch.bfloat16, gen(22)
    x, w = normal(g, 143, k, dtype=t).requires_grad_(), normal(g, 4, 2 * n, k, dtype=t, size=0.1)
    dh, off = normal(g, 143, n, dtype=t), offsets_of(counts)
    codes_of_w = (*products.quantize_rows(w), *products.quantize_columns(w))
    for bits in ([0, 1, 0, 1], [0] * 4, [1] * 4):
        mask = torch.tensor(bits, dtype=torch.uint8, device="cuda")
        got = []
        for held in (None, codes_of_w):
            arena = torch.empty(4, 2 * n, k, device="cuda")
            h = expert_gated(products, x, w, off, mask, arena, codes=held)
            got.append((h, *torch.autograd.grad(h, x, dh), arena))
        assert all(torch.equal(a, b) for a, b in zip(*got))
        if all(bits):
            plain = expert_gated(products, x, w, off)
            assert torch.equal(got[0][0], plain) and torch.equal(got[0][1], torch.autograd.grad(plain, x, dh)[0])
    with torch.no_grad():
        assert torch.equal(expert_gated(products, x, w, off, mask), plain)
    out = torch.full((143, n), 7.0, dtype=t, device="cuda")
    products.gated(x.detach(), w, off, out=out, mask=torch.zeros_like(mask))
    assert (out == 7).all()


def test_gradients_against_differences(products):
    """The layer's directional derivative against a difference of losses formed in 64 bits from its own outputs: the
    step moves h by about 1 %, its rounding (2^-11 of each of 60 x 40 values, at random) adds up to 2^-11 * 49 * |h|."""
    g, t = gen(31), torch.float16
    x, w = normal(g, 60, 64, dtype=t).requires_grad_(), normal(g, 80, 64, dtype=t, size=0.125)
    c = normal(g, 60, 40, dtype=torch.float64)
    h = expert_gated(products, x, w)
    dx, = torch.autograd.grad((h.double() * c).sum(), x)
    way = normal(g, 60, 64, dtype=torch.float64)
    step = 2.0 ** -5
    up, down = ((x.detach().double() + s * step * way).to(t) for s in (1, -1))
    moved = up.double() - down.double()                              # what the rounded inputs moved by
    with torch.no_grad():
        got = ((expert_gated(products, up, w).double() - expert_gated(products, down, w).double()) * c).sum()
    want = (dx.double() * moved).sum()
    # third derivatives: (step |way|)^3 / 24 of each output's scale; roundings as above, both sides
    assert (got - want).abs() <= 2 * 2.0 ** -11 * h.double().norm() * 4 + 0.05 * want.abs()


def test_two_layers_train_into_one_arena(products):
    """Gated block and down projection: gradients of both weights side by side, against autograd in 32 bits."""
    n, k, t, g = 40, 64, torch.bfloat16, gen(33)
    x = normal(g, 96, k, dtype=t).requires_grad_()
    w1, w2 = normal(g, 2 * n, k, dtype=t, size=0.15), normal(g, k, n, dtype=t, size=0.15)
    arena = torch.zeros(3 * n * k, device="cuda")
    y = expert_linear(products, expert_gated(products, x, w1, grad=arena[:2 * n * k].view(2 * n, k)), w2, grad=arena[2 * n * k:].view(k, n))
    y.float().square().mean().backward()
    X, A, B = (v.detach().float().requires_grad_() for v in (x, w1, w2))
    a, b = (X @ A.T).chunk(2, 1)
    ((torch.nn.functional.silu(a) * b) @ B.T).square().mean().backward()
    for got, want in ((arena[:2 * n * k].view(2 * n, k), A.grad), (arena[2 * n * k:].view(k, n), B.grad), (x.grad.float(), X.grad)):
        # h, [a, b], dh, dab and y each rounded to bf16 on the way: about 2^-8 each
        assert (got - want).norm() <= 6 * 2.0 ** -8 * want.norm()


def test_refusals(products):
    t = torch.bfloat16
    x, w = torch.zeros(6, 16, dtype=t, device="cuda"), torch.zeros(8, 16, dtype=t, device="cuda")
    ab, dh = torch.zeros(6, 8, dtype=t, device="cuda"), torch.zeros(6, 4, dtype=t, device="cuda")
    for call, why in [
        (lambda: products.gated(x, w[:7]), "two projections"), (lambda: products.gated(x[:, :8], w), "columns"),
        (lambda: products.gated(x, w, activation="relu"), "activation"), (lambda: products.gated(x.half(), w), "must be"),
        (lambda: products.gated(x.float(), w.float()), "must be"), (lambda: products.gated(x.cpu(), w), "CUDA"),
        (lambda: products.gated(x, w, keep=ab[:, :6]), "keep"), (lambda: products.gated(x, w, keep=ab.half()), "keep"),
        (lambda: products.gated(x, w, out=ab), "out"), (lambda: products.gated(x, w.T.contiguous().T), "contiguous"),
        (lambda: products.gated(x, w.view(2, 4, 16)), "offsets"), (lambda: products.gate(ab[:, :7]), "two projections"),
        (lambda: products.gate(ab, mask=torch.zeros(2, dtype=torch.uint8, device="cuda")), "one group"),
        (lambda: products.gate_grad(dh, ab[:, :6]), "ab must be"), (lambda: products.gate_grad(dh[:5], ab), "ab must be"),
        (lambda: products.gate_grad(dh, ab, activation=0), "activation"), (lambda: products.gate_grad(dh.half(), ab), "must be"),
        (lambda: products.gated(x.requires_grad_(), w), "autograd"),
    ]:
        with pytest.raises(ValueError, match=why):
            call()


def test_gate_refuses_what_is_no_tensor(products):
    ab = torch.zeros(6, 8, dtype=torch.bfloat16, device="cuda")
    for call, why in [
        (lambda: products.gate(ab, mask=[0]), "mask must"), (lambda: products.gate(ab, [0, 6]), "offsets must"),
        (lambda: products.gate(ab, torch.tensor([0, 6])), "offsets must"), (lambda: products.gate(ab, torch.tensor([0., 6.]).cuda()), "offsets must"),
    ]:
        with pytest.raises(ValueError, match=why):
            call()


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_one_row_of_any_stride_in_place(products, kind):
    g, n = gen(12), 136
    ab, dh = normal(g, 4, 2 * n, dtype=torch.bfloat16), normal(g, 4, n, dtype=torch.bfloat16)
    old, want = ab.clone(), products.gate_grad(dh, ab, activation=kind)
    products.gate_grad(dh[::3][:1], ab[::2][:1], out=ab[:1], activation=kind)
    assert torch.equal(ab[:1], want[:1]) and torch.equal(ab[1:], old[1:])


@pytest.mark.parametrize("n", [24, 5])
@pytest.mark.parametrize("groups", [31, 32, 33, 64, 70, 257, 2048])
def test_gate_of_many_groups(products, groups, n):
    """Groups' first rows are found 32 at a time: groups of none to four rows, ahead of the first and behind the last group rows of none,
    every other group on the other path; offsets that fall are as in the products."""
    rng, g = np.random.default_rng(groups), gen(groups)
    counts, first = rng.integers(0, 5, groups).tolist(), 3
    counts[groups // 2] = 0
    R = sum(counts) + first + 4
    ab = normal(g, R, 2 * n, dtype=torch.bfloat16)
    mask = torch.from_numpy(rng.integers(0, 2, groups).astype(np.uint8)).cuda()
    every = products.gate(ab)
    off = offsets_of(counts, first)
    out = torch.full((R, n), 7.0, device="cuda", dtype=torch.bfloat16)
    products.gate(ab, off, out=out, mask=mask)
    wanted = torch.zeros(R, dtype=torch.bool)
    for e, at in spans(counts, first):
        wanted[at] = not mask[e].item()
    wanted = wanted.cuda()
    assert torch.equal(out[wanted], every[wanted]) and (out[~wanted] == 7).all()
    # one that falls in the middle is taken as the largest before it: its group is empty, and the next one begins there
    off[groups // 2] = 0
    out.fill_(7.0)
    products.gate(ab, off, out=out)
    assert torch.equal(out[first:R - 4], every[first:R - 4]) and (out[:first] == 7).all() and (out[R - 4:] == 7).all()
