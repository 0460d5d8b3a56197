"""Expert products against the definition in 64 bits: every direction, type, stride and
grouping, masks, empty groups, non-finite values, and the 8-bit codes.

Tolerances.  A 16-bit product's sum of d terms is held in fp32: pieces of at most
1,024 terms, of which the tensor cores add 16 at a time, so at most 64 steps that
round (or cut) by at most 2^-23 of the sum S of the terms' magnitudes, one more for the
terms of a step, and an addition for each piece: |error| <= (66 + d / 512) 2^-23 S, and
the output's own rounding (2^-8 bf16, 2^-11 f16, 2^-24 fp32 of the value, or half of
f16's smallest step).  128 in place of 66 leaves room for the order within a step.  An 8-bit product's sum is an exact
integer; converting and scaling it rounds three times, 3 * 2^-24 of the value."""
import numpy as np
import pytest

from paper_2606_00539_gb300 import ExpertProducts, GnmrError, expert_linear

pytestmark = pytest.mark.gpu

import torch  # noqa: E402

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ROUND = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
LEAST = {"bf16": 0.0, "f16": 2.0 ** -25, "f32": 0.0}


@pytest.fixture(scope="module")
def products():
    p = ExpertProducts(device=0)
    yield p
    p.close()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype, size=1.0):
    return (torch.randn(*shape, device="cuda", generator=g) * size).to(dtype)


def offsets_of(counts, first=0):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]) + first, dtype=torch.int64, device="cuda")


def spans(counts, first=0):
    at = first
    for e, c in enumerate(counts):
        yield e, slice(at, at + c)
        at += c


def check(got, want, size, depth, kind):
    got, want, size = got.double(), want.double(), size.double()
    tol = (128 + depth / 512) * 2.0 ** -23 * size
    tol = tol + ROUND[kind] * (want.abs() + tol) + LEAST[kind]
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (f"{int(bad.sum())} of {bad.numel()} outside, first at {bad.nonzero()[0].tolist()}: "
                           f"{got[bad][0].item()} for {want[bad][0].item()}")


# groups' rows, n_out, n_in: one row, a few, odd, tiles and pieces and their edges, no rows at all
SHAPES = [
    ([1], 8, 8), ([1], 1, 1), ([3], 5, 7), ([17], 64, 64), ([1], 256, 512), ([5], 1000, 136),
    ([255], 257, 264), ([256], 256, 64), ([257], 128, 1024), ([513], 384, 1032), ([700], 200, 2056),
    ([0], 40, 48), ([0, 0, 0], 40, 48), ([1, 0, 2, 0, 0, 31, 33], 136, 200), ([64, 65, 63, 1], 257, 129),
    ([300, 0, 511, 16, 15, 17, 1], 320, 520), ([2] * 40, 264, 72), ([1100, 3], 96, 88), ([31] * 3, 1003, 1371),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_forward_and_gradients(products, case, dtype):
    counts, n, k = SHAPES[case]
    g, t, G, R = gen(case), TYPES[dtype], len(counts), sum(counts)
    x, dy = normal(g, R, k, dtype=t), normal(g, R, n, dtype=t)
    w = normal(g, G, n, k, dtype=t, size=k ** -0.5)
    off = offsets_of(counts)
    y, dx = products.forward(x, w, off), products.input_grad(dy, w, off)
    old = normal(g, G, n, k, dtype=torch.float32)
    dw32, dw16, more = old.clone(), old.to(t), old.clone()
    products.weight_grad(dy, x, off, out=dw32)
    products.weight_grad(dy, x, off, out=dw16)
    products.weight_grad(dy, x, off, out=more, add=True)
    torch.cuda.synchronize()
    assert y.shape == (R, n) and dx.shape == (R, k)
    for e, at in spans(counts):
        X, D, W = x[at].double(), dy[at].double(), w[e].double()
        check(y[at], X @ W.T, X.abs() @ W.abs().T, k, dtype)
        check(dx[at], D @ W, D.abs() @ W.abs(), n, dtype)
        dw, size = D.T @ X, D.abs().T @ X.abs()
        check(dw32[e], dw, size, counts[e], "f32")
        check(dw16[e], dw, size, counts[e], dtype)
        check(more[e], dw + old[e].double(), size + old[e].double().abs(), counts[e], "f32")


@pytest.mark.parametrize("dtype,add", [("bf16", True), ("f16", True)])
def test_add_to_a_16_bit_arena(products, dtype, add):
    t, g = TYPES[dtype], gen(3)
    x, dy = normal(g, 300, 200, dtype=t), normal(g, 300, 136, dtype=t)
    old = normal(g, 136, 200, dtype=t)
    got = products.weight_grad(dy, x, out=old.clone(), add=add)
    X, D = x.double(), dy.double()
    check(got, D.T @ X + old.double(), D.abs().T @ X.abs() + old.double().abs(), 300, dtype)


@pytest.mark.parametrize("depth", [8192, 50001])
def test_long_sums_keep_32_bits(products, depth):
    """Tens of thousands of rows into one gradient, all terms of one sign: nothing piles up."""
    g = gen(depth)
    x = torch.rand(depth, 72, device="cuda", generator=g).bfloat16()
    dy = torch.rand(depth, 40, device="cuda", generator=g).bfloat16()
    got = products.weight_grad(dy, x, out=torch.empty(40, 72, device="cuda"))
    want = dy.double().T @ x.double()
    check(got, want, want, depth, "f32")


def test_strides_and_views(products):
    """Operands inside larger buffers: padded rows, group strides, a transposed group order, odd starts."""
    counts, n, k = [37, 0, 129], 136, 200
    t, g, R = torch.bfloat16, gen(5), 166
    off = offsets_of(counts)
    for pad, lead in ((0, 0), (8, 8), (3, 1), (1, 16)):
        x = normal(g, R, k + pad, dtype=t)[:, :k] if pad else normal(g, R, k, dtype=t)
        dy = normal(g, R, n + pad + lead, dtype=t)[:, lead:lead + n]
        flat = normal(g, lead + 3 * (2 * n * k + 24 + pad), dtype=t, size=0.1)
        w = torch.as_strided(flat, (3, n, k), (2 * n * k + 24 + pad, k, 1), lead)
        arena = torch.zeros(lead + 3 * (n * k + 40 + pad), device="cuda")
        dw = torch.as_strided(arena, (3, n, k), (n * k + 40 + pad, k, 1), lead)
        y = torch.full((R, n + 5), 7.0, device="cuda", dtype=t)
        products.forward(x, w, off, out=y[:, 2:2 + n])
        dx = products.input_grad(dy, w, off)
        products.weight_grad(dy, x, off, out=dw)
        assert (y[:, :2] == 7).all() and (y[:, 2 + n:] == 7).all()
        taken = torch.zeros_like(arena, dtype=torch.bool)
        torch.as_strided(taken, dw.shape, dw.stride(), lead).fill_(True)
        assert (arena[~taken] == 0).all()
        for e, at in spans(counts):
            X, D, W = x[at].double(), dy[at].double(), w[e].double()
            check(y[at, 2:2 + n], X @ W.T, X.abs() @ W.abs().T, k, "bf16")
            check(dx[at], D @ W, D.abs() @ W.abs(), n, "bf16")
            check(dw[e], D.T @ X, D.abs().T @ X.abs(), counts[e], "f32")


@pytest.mark.parametrize("n,k,held,lead", [(40, 65, 72, 0), (33, 130, 136, 8), (41, 67, 71, 1), (72, 63, 64, 3)])
def test_what_lies_between_rows_has_no_influence(products, n, k, held, lead):
    """NaN after the last column of every row, in operands read in place and in copied ones."""
    counts, t, g = [50, 0, 21, 200], torch.bfloat16, gen(n)
    off, R = offsets_of(counts), 271

    def inside(*shape):
        flat = torch.full((shape[0] * (shape[1] if len(shape) == 3 else 1) * (held + 16) + lead + 64,), float("nan"),
                          dtype=t, device="cuda")
        row = held if shape[-1] <= held else shape[-1]
        strides = (row * shape[1] + 8, row, 1) if len(shape) == 3 else (row, 1)
        v = torch.as_strided(flat, shape, strides, lead)
        v.copy_(normal(g, *shape, dtype=t))
        return v

    x, w, dy = inside(R, k), inside(4, n, k), inside(R, n)
    y, dx = products.forward(x, w, off), products.input_grad(dy, w, off)
    dw = products.weight_grad(dy, x, off, out=torch.empty(4, n, k, device="cuda"))
    for e, at in spans(counts):
        X, D, W = x[at].double(), dy[at].double(), w[e].double()
        check(y[at], X @ W.T, X.abs() @ W.abs().T, k, "bf16")
        check(dx[at], D @ W, D.abs() @ W.abs(), n, "bf16")
        check(dw[e], D.T @ X, D.abs().T @ X.abs(), counts[e], "f32")


def test_offsets_past_32_bits(products):
    """Rows, and an arena, of more than 2^31 elements: what lies at their ends."""
    rows, k, n = 1_100_001, 2048, 24
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    g, t = gen(17), torch.bfloat16
    x = torch.empty(rows, k, dtype=t, device="cuda").normal_(generator=g)
    w, dy = normal(g, 2, n, k, dtype=t), torch.zeros(rows, n, dtype=t, device="cuda")
    dy[rows - 9:] = normal(g, 9, n, dtype=t)
    off = torch.tensor([0, rows - 7, rows], dtype=torch.int64, device="cuda")
    y = products.forward(x, w, off)
    for at, e in ((slice(rows - 7, rows), 1), (slice(rows - 60, rows - 7), 0), (slice(0, 50), 0)):
        X, W = x[at].double(), w[e].double()
        check(y[at], X @ W.T, X.abs() @ W.abs().T, k, "bf16")
    arena = torch.zeros(2 ** 31 + 2 * n * k, device="cuda")
    out = torch.as_strided(arena, (2, n, k), (2 ** 31 + n * k, k, 1))
    products.weight_grad(dy, x, off, out=out)
    for e, at in ((0, slice(rows - 9, rows - 7)), (1, slice(rows - 7, rows))):
        X, D = x[at].double(), dy[at].double()
        check(out[e], D.T @ X, D.abs().T @ X.abs(), rows if e == 0 else 7, "f32")
    assert int((arena != 0).sum()) == int((out != 0).sum())
    del arena, out, y
    q, s = products.quantize_rows(x)
    wq, ws = codes_oracle(x[-5:])
    assert np.array_equal(q[-5:].cpu().numpy(), wq) and np.array_equal(s[-5:].cpu().numpy(), ws)
    (vq, vs) = products.quantize_rows(w)
    low = products.forward_i8(q, s, vq, vs, off, out_dtype="f32")
    at = slice(rows - 7, rows)
    want = (q[at].double() @ vq[1].double().T) * s[at].double()[:, None] * vs[1].double()
    assert ((low[at].double() - want).abs() <= want.abs() * 2.0 ** -21).all()


@pytest.mark.parametrize("groups", [270, 2048])
def test_many_groups(products, groups):
    """Tables that leave room for fewer stages, and most groups without rows."""
    g, t = gen(groups), torch.bfloat16
    counts = [0] * groups
    for e, c in ((0, 3), (7, 70), (groups // 2, 1), (groups - 2, 300), (groups - 1, 33)):
        counts[e] = c
    R, n, k = sum(counts), 40, 72
    off = offsets_of(counts)
    x, dy, w = normal(g, R, k, dtype=t), normal(g, R, n, dtype=t), normal(g, groups, n, k, dtype=t)
    y, dx = products.forward(x, w, off), products.input_grad(dy, w, off)
    dw = products.weight_grad(dy, x, off, out=torch.full((groups, n, k), 7.0, device="cuda"))
    (xq, xs), (wq, ws) = products.quantize_rows(x), products.quantize_rows(w)
    low = products.forward_i8(xq, xs, wq, ws, off, out_dtype="f32")
    for e, at in spans(counts):
        X, D, W = x[at].double(), dy[at].double(), w[e].double()
        check(y[at], X @ W.T, X.abs() @ W.abs().T, k, "bf16")
        check(dx[at], D @ W, D.abs() @ W.abs(), n, "bf16")
        check(dw[e], D.T @ X, D.abs().T @ X.abs(), counts[e], "f32")
        want = (xq[at].double() @ wq[e].double().T) * xs[at].double()[:, None] * ws[e].double()
        assert ((low[at].double() - want).abs() <= want.abs() * 2.0 ** -21).all()


def test_groups_may_share_a_weight(products):
    g = gen(6)
    x, w = normal(g, 90, 64, dtype=torch.float16), normal(g, 72, 64, dtype=torch.float16)
    y = products.forward(x, w.expand(3, 72, 64), offsets_of([20, 30, 40]))
    check(y, x.double() @ w.double().T, x.double().abs() @ w.double().abs().T, 64, "f16")


def test_rows_of_no_group_and_masked_groups_keep_their_outputs(products):
    counts, n, k, first, R = [40, 0, 300, 17], 264, 136, 5, 400
    t, g = torch.bfloat16, gen(7)
    x, w, dy = normal(g, R, k, dtype=t), normal(g, 4, n, k, dtype=t), normal(g, R, n, dtype=t)
    off = offsets_of(counts, first)
    for bits in ([1, 1, 1, 1], [0, 0, 0, 0], [1, 0, 0, 255], [0, 1, 1, 0]):
        mask = torch.tensor(bits, dtype=torch.uint8, device="cuda").repeat_interleave(3)[1::3]
        y = products.forward(x, w, off, mask=mask, out=torch.full((R, n), 7.0, dtype=t, device="cuda"))
        dx = products.input_grad(dy, w, off, mask=mask, out=torch.full((R, k), 7.0, dtype=t, device="cuda"))
        dw = products.weight_grad(dy, x, off, mask=mask, out=torch.full((4, n, k), 7.0, device="cuda"))
        left = torch.ones(R, dtype=torch.bool)
        for e, at in spans(counts, first):
            if not bits[e]:
                assert (dw[e] == 7).all()
                continue
            left[at] = False
            X, D, W = x[at].double(), dy[at].double(), w[e].double()
            check(y[at], X @ W.T, X.abs() @ W.abs().T, k, "bf16")
            check(dx[at], D @ W, D.abs() @ W.abs(), n, "bf16")
            check(dw[e], D.T @ X, D.abs().T @ X.abs(), counts[e], "f32")
        assert (y[left] == 7).all() and (dx[left] == 7).all()


def test_offsets_out_of_range_are_taken_as_the_nearest_allowed(products):
    g = gen(8)
    x, w = normal(g, 50, 64, dtype=torch.bfloat16), normal(g, 4, 72, 64, dtype=torch.bfloat16)
    off = torch.tensor([-9, 20, 10, 2 ** 40, 7], dtype=torch.int64, device="cuda")   # 0..20, none, 20..50, none
    y = products.forward(x, w, off)
    for e, at in ((0, slice(0, 20)), (2, slice(20, 50))):
        check(y[at], x[at].double() @ w[e].double().T, x[at].double().abs() @ w[e].double().abs().T, 64, "bf16")
    dw = products.weight_grad(y, x, off, out=torch.full((4, 72, 64), 7.0, device="cuda"))
    assert (dw[1] == 0).all() and (dw[3] == 0).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_non_finite_values_stay_where_they_belong(products, bad):
    counts, n, k = [33, 70, 5], 136, 200
    t, g, R = torch.bfloat16, gen(9), 108
    off = offsets_of(counts)
    x, w, dy = normal(g, R, k, dtype=t), normal(g, 3, n, k, dtype=t), normal(g, R, n, dtype=t)
    y0, dx0 = products.forward(x, w, off), products.input_grad(dy, w, off)
    dw0 = products.weight_grad(dy, x, off, out=torch.empty(3, n, k, device="cuda"))
    x[33, 199], dy[33, 3], w[2, 7, 9] = bad, bad, bad        # the second group's first row, the third's weight
    y, dx = products.forward(x, w, off), products.input_grad(dy, w, off)
    dw = products.weight_grad(dy, x, off, out=torch.empty(3, n, k, device="cuda"))
    same = torch.ones(R, n, dtype=torch.bool, device="cuda")
    same[33], same[103:, 7] = False, False
    assert torch.equal(y[same], y0[same]) and not y[~same].isfinite().any()
    same = torch.ones(R, k, dtype=torch.bool, device="cuda")
    same[33], same[103:, 9] = False, False
    assert torch.equal(dx[same], dx0[same]) and not dx[~same].isfinite().any()
    same = torch.ones(3, n, k, dtype=torch.bool, device="cuda")
    same[1, 3], same[1, :, 199] = False, False
    assert torch.equal(dw[same], dw0[same]) and not dw[~same].isfinite().any()


def test_gradients_against_differences(products):
    """The products are linear, so on small integers, where every sum is exact in bf16, a
    difference of outputs equals the gradient's product with the difference of inputs."""
    counts, n, k = [13, 0, 30], 40, 24
    g, R, t = gen(10), 43, torch.bfloat16
    off = offsets_of(counts)

    def small(*shape):
        return (torch.randint(0, 8, shape, device="cuda", generator=g) == 0).to(t) * \
            torch.randint(-1, 2, shape, device="cuda", generator=g).to(t)

    x, w, dy, ex, ew = small(R, k), small(3, n, k), small(R, n), small(R, k), small(3, n, k)
    f = products.forward
    dx = products.input_grad(dy, w, off)
    dw = products.weight_grad(dy, x, off, out=torch.empty(3, n, k, device="cuda"))
    by_x = (dy.double() * (f(x + ex, w, off).double() - f(x, w, off).double())).sum()
    by_w = (dy.double() * (f(x, w + ew, off).double() - f(x, w, off).double())).sum()
    assert by_x == (dx.double() * ex.double()).sum() and by_w == (dw.double() * ew.double()).sum()
    assert by_x != 0 and by_w != 0


def test_the_same_call_gives_the_same_bits_and_other_streams_work(products):
    g = gen(11)
    x, w, dy = normal(g, 40, 2048, dtype=torch.bfloat16), normal(g, 2, 264, 2048, dtype=torch.bfloat16), normal(g, 40, 264, dtype=torch.bfloat16)
    off = offsets_of([3, 37])
    y = products.forward(x, w, off)
    dw = products.weight_grad(dy, x, off, out=torch.empty(2, 264, 2048, device="cuda"))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        y2 = products.forward(x, w, off, stream=side)
        side.synchronize()
        assert torch.equal(y, y2)
        with torch.cuda.stream(side):
            dw2 = products.weight_grad(dy, x, off, out=torch.empty(2, 264, 2048, device="cuda"))
        side.synchronize()
        assert torch.equal(dw, dw2)


# -- 8-bit codes ----------------------------------------------------------------

def codes_oracle(x):
    """By row, in numpy: fp32 factors, products rounded to fp32, halves to even."""
    x = x.float().cpu().numpy()
    with np.errstate(all="ignore"):
        top = np.abs(x).max(axis=-1, initial=0.0, keepdims=True).astype(np.float32)
        up = np.float32(127) * (np.float32(1) / top)
        down = top / np.float32(127)
        zero, lost = ~np.isfinite(up), ~np.isfinite(np.abs(x).sum(axis=-1, keepdims=True, dtype=np.float64))
        q = np.where(zero | lost, 0, np.rint(x * np.where(zero | lost, np.float32(0), up)))
        q[np.broadcast_to(lost, q.shape)] = 0
        down = np.where(lost, np.float32("nan"), np.where(zero, np.float32(0), down))
    return q.astype(np.int8), down[..., 0].astype(np.float32)


CODE_SHAPES = [(1, 1, 1), (1, 1, 8), (1, 7, 5), (1, 33, 64), (1, 300, 129), (3, 130, 72), (1, 5, 1024), (2, 9, 1032),
               (1, 4, 5120), (1, 3, 20008), (1, 3, 9001), (4, 257, 200), (1, 2000, 136), (1, 0, 16), (1, 16, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("case", range(len(CODE_SHAPES)))
def test_codes(products, case, dtype):
    G, r, c = CODE_SHAPES[case]
    g = gen(100 + case)
    x = normal(g, G, r, c, dtype=TYPES[dtype], size=3.0)
    if c > 4 and r > 4:
        x[0, 1] = 0
        x[0, 2, 1] = float("nan")
        x[0, 3, c - 1] = -float("inf")
        if dtype != "f16":
            x[0, 4] = 0
            x[0, 4, 0] = 1e-38
    x2 = x if G > 1 else x[0]
    q, s = products.quantize_rows(x2)
    wq, ws = codes_oracle(x2)
    assert q.shape == x2.shape and np.array_equal(q.cpu().numpy(), wq)
    assert np.array_equal(s.cpu().numpy(), ws, equal_nan=True)
    q, s = products.quantize_columns(x2)
    wq, ws = codes_oracle(x2.transpose(-1, -2))
    assert q.shape == x2.transpose(-1, -2).shape and np.array_equal(q.cpu().numpy(), wq)
    assert np.array_equal(s.cpu().numpy(), ws, equal_nan=True)


def test_codes_of_views(products):
    g = gen(12)
    flat = normal(g, 4 * 70 * 100 + 50, dtype=torch.bfloat16)
    for lead, row, group in ((0, 64, 70 * 64), (8, 72, 70 * 72 + 8), (1, 65, 70 * 100)):
        x = torch.as_strided(flat, (3, 70, 64), (group, row, 1), lead)
        for q, want in ((products.quantize_rows(x), x), (products.quantize_columns(x), x.transpose(1, 2))):
            wq, ws = codes_oracle(want)
            assert np.array_equal(q[0].cpu().numpy(), wq) and np.array_equal(q[1].cpu().numpy(), ws)


@pytest.mark.parametrize("shape", [(5, 130, 72), (5, 9, 1032), (5, 7, 5), (5, 3, 9000)])
def test_codes_of_masked_groups_are_left_as_they_are(products, shape):
    x = normal(gen(15), *shape, dtype=torch.bfloat16)
    mask = torch.tensor([0, 7, 1, 0, 9, 255, 0, 7, 0], dtype=torch.uint8, device="cuda")[::2]     # 0 1 9 0 0
    for fn, want in ((products.quantize_rows, x), (products.quantize_columns, x.transpose(1, 2))):
        q, s = fn(x, mask=mask)
        wq, ws = codes_oracle(want)
        for e in (0, 3, 4):
            assert np.array_equal(q[e].cpu().numpy(), wq[e]) and np.array_equal(s[e].cpu().numpy(), ws[e])
    held = torch.full((5, 130, 16), 77, dtype=torch.int8, device="cuda")
    scale = torch.full((5, 130), 7.0, device="cuda")
    from paper_2606_00539_gb300 import _native as N
    y = normal(gen(16), 5, 130, 16, dtype=torch.float32)
    every = torch.ones(5, dtype=torch.uint8, device="cuda")
    N.gnmr_quantize_rows(y.data_ptr(), N.GNMR_DTYPE_F32, 5, 130, 16, 16, 130 * 16, every.data_ptr(), 1, held.data_ptr(),
                         16, 130 * 16, scale.data_ptr(), torch.cuda.current_stream().cuda_stream)
    N.gnmr_quantize_columns(y.data_ptr(), N.GNMR_DTYPE_F32, 5, 130, 16, 16, 130 * 16, every.data_ptr(), 1,
                            held.data_ptr(), 130, 130 * 16, scale.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert (held == 77).all() and (scale == 7).all()


def codes(g, *shape, low=-127):
    return torch.randint(low, 128, shape, device="cuda", generator=g, dtype=torch.int8)


@pytest.mark.parametrize("out", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_forward_i8(products, case, out):
    counts, n, k = SHAPES[case]
    g, G, R = gen(200 + case), len(counts), sum(counts)
    xq, wq = codes(g, R, k), codes(g, G, n, k)
    xs = torch.rand(R, device="cuda", generator=g) * 1e-2
    ws = torch.rand(G, n, device="cuda", generator=g) * 1e-2
    y = products.forward_i8(xq, xs, wq, ws, offsets_of(counts), out_dtype=out)
    assert y.dtype == TYPES[out] and y.shape == (R, n)
    for e, at in spans(counts):
        want = (xq[at].double() @ wq[e].double().T) * xs[at].double()[:, None] * ws[e].double()
        err = (y[at].double() - want).abs()
        assert (err <= want.abs() * (3 * 2.0 ** -24 + ROUND[out]) * (1 + 2.0 ** -8) + LEAST[out]).all()


@pytest.mark.parametrize("k", [1040, 4096, 131071])
@pytest.mark.parametrize("rows", [3, 300])
def test_forward_i8_sums_are_exact_integers(products, k, rows):
    """All codes at their largest, sums far past 2^24: each the exact integer, rounded once."""
    xq = torch.full((rows, k), 127, dtype=torch.int8, device="cuda")
    wq = torch.full((40, k), 127, dtype=torch.int8, device="cuda")
    xq[1::2], wq[5] = -128, -128
    xq[2, ::2] = -127
    xq[0, k - 1] = 1
    one = torch.ones(rows, device="cuda")
    y = products.forward_i8(xq, one, wq, torch.ones(40, device="cuda"), out_dtype="f32")
    want = (xq.double() @ wq.double().T).to(torch.float32)       # exact in 64 bits
    assert torch.equal(y, want)


def test_forward_i8_mask_strides_and_scales(products):
    counts, n, k, R = [40, 1, 0, 300], 136, 72, 341
    g, off = gen(13), offsets_of(counts)
    xq, wq = codes(g, R, 80)[:, 4:76], codes(g, 4, n + 1, k + 9)[:, :n, :k]
    xs, ws = torch.rand(R, device="cuda", generator=g), torch.rand(4, n, device="cuda", generator=g)
    xs[41], ws[3, 5] = float("nan"), 0.0
    mask = torch.tensor([0, 1, 0, 0], dtype=torch.uint8, device="cuda")
    y = products.forward_i8(xq, xs, wq, ws, off, out=torch.full((R, n), 7.0, device="cuda"), mask=mask)
    assert (y[40] == 7).all() and y[41].isnan().all()
    for e, at in ((0, slice(0, 40)), (3, slice(42, 341))):
        want = (xq[at].double() @ wq[e].double().T) * xs[at].double()[:, None] * ws[e].double()
        assert ((y[at].double() - want).abs() <= want.abs() * 2.0 ** -21).all()


def test_refusals(products):
    t = torch.bfloat16
    x, w = torch.zeros(6, 8, dtype=t, device="cuda"), torch.zeros(2, 16, 8, dtype=t, device="cuda")
    off = offsets_of([2, 4])
    for call in (lambda: products.forward(x.cpu(), w, off), lambda: products.forward(x.float(), w, off),
                 lambda: products.forward(x.half(), w, off), lambda: products.forward(x[:, :7], w, off),
                 lambda: products.forward(x, w), lambda: products.forward(x, w, off.int()),
                 lambda: products.forward(x, w, off[:2]), lambda: products.forward(x, w, off, mask=off),
                 lambda: products.forward(x, w, off, mask=torch.zeros(3, dtype=torch.uint8, device="cuda")),
                 lambda: products.forward(x, w, off, out=torch.zeros(6, 15, dtype=t, device="cuda")),
                 lambda: products.forward(x, w, off, out=torch.zeros(6, 16, device="cuda")),
                 lambda: products.forward(x.T, w, off), lambda: products.forward(x[0], w, off),
                 lambda: products.forward(x, w.transpose(1, 2), off),
                 lambda: products.weight_grad(x, x[:5], off, out=w),
                 lambda: products.weight_grad(x, x, off, out=w.half()),
                 lambda: products.forward_i8(x, x, w, w, off),
                 lambda: products.forward_i8(x.char(), x.float()[:, 0], w.char(), w.float()[:, :, 0].contiguous(), off),
                 lambda: products.forward_i8(x.char(), torch.zeros(6, device="cuda"), w.char(),
                                             torch.zeros(2, 16, device="cuda"), off, out_dtype="i8"),
                 lambda: products.quantize_rows(x.char()), lambda: products.quantize_rows(x[0])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(GnmrError):                                # groups that overlap in the output
        products.weight_grad(torch.zeros(6, 16, dtype=t, device="cuda"), x, off, out=torch.as_strided(w, (2, 16, 8), (8, 8, 1)))
    p = ExpertProducts(device=0)
    p.close()
    with pytest.raises(ValueError):
        p.forward(x, w, off)


# -- the layer --------------------------------------------------------------------

@pytest.mark.parametrize("bits", [None, [0, 1, 0, 1], [0, 0, 0, 0], [1, 1, 1, 1]])
def test_expert_linear(products, bits):
    """Forward and backward on both paths, and the gradient in the arena, against the
    definition on the same codes."""
    counts, n, k = [40, 70, 0, 9], 72, 136
    g, t, R = gen(14), torch.bfloat16, 119
    off = offsets_of(counts)
    x, w, dy = normal(g, R, k, dtype=t), normal(g, 4, n, k, dtype=t, size=0.1), normal(g, R, n, dtype=t)
    arena = torch.full((4, n, k), 7.0, device="cuda")
    mask = None if bits is None else torch.tensor(bits, dtype=torch.uint8, device="cuda")
    fixed = None if bits is None else (*products.quantize_rows(w), *products.quantize_columns(w))
    x.requires_grad_()
    y = expert_linear(products, x, w, off, mask, arena)
    dx, = torch.autograd.grad(y, x, dy)
    y2 = expert_linear(products, x, w, off, mask, None, codes=fixed)
    assert torch.equal(y, y2)
    w2 = w.clone().requires_grad_()
    dx2, dw2 = torch.autograd.grad(expert_linear(products, x, w2, off, mask), (x, w2), dy)
    assert torch.equal(dx, dx2)
    x = x.detach()
    (xq, xs), (dq, ds), (wq, ws), (vq, vs) = (codes_oracle(a) for a in (x, dy, w, w.transpose(1, 2)))
    for e, at in spans(counts):
        X, D, W = x[at].double(), dy[at].double(), w[e].double()
        if bits is None or bits[e]:
            check(y[at], X @ W.T, X.abs() @ W.abs().T, k, "bf16")
            check(dx[at], D @ W, D.abs() @ W.abs(), n, "bf16")
        else:
            for got, a, s, b, u in ((y, xq, xs, wq, ws), (dx, dq, ds, vq, vs)):
                want = (a[at].astype(float) @ b[e].astype(float).T) * s[at].astype(float)[:, None] * u[e].astype(float)
                err = np.abs(got[at].detach().double().cpu().numpy() - want)
                assert (err <= np.abs(want) * (ROUND["bf16"] + 2.0 ** -21)).all()
        check(arena[e], D.T @ X, D.abs().T @ X.abs(), counts[e], "f32")
        check(dw2[e], D.T @ X, D.abs().T @ X.abs(), counts[e], "bf16")


@pytest.mark.parametrize("bit", [0, 1])
def test_expert_linear_of_one_dense_unit(products, bit):
    g, t = gen(18), torch.bfloat16
    x, w, dy = normal(g, 90, 136, dtype=t), normal(g, 72, 136, dtype=t, size=0.1), normal(g, 90, 72, dtype=t)
    arena = torch.full((72, 136), 7.0, device="cuda")
    mask = torch.tensor([bit], dtype=torch.uint8, device="cuda")
    x.requires_grad_()
    y = expert_linear(products, x, w, None, mask, arena)
    dx, = torch.autograd.grad(y, x, dy.expand(90, 72))
    X, D, W = x.detach().double(), dy.double(), w.double()
    check(arena, D.T @ X, D.abs().T @ X.abs(), 90, "f32")
    if bit:
        check(y, X @ W.T, X.abs() @ W.abs().T, 136, "bf16")
        check(dx, D @ W, D.abs() @ W.abs(), 72, "bf16")
    else:
        (xq, xs), (dq, ds), (wq, ws), (vq, vs) = (codes_oracle(a) for a in (x.detach(), dy, w, w.T))
        for got, a, s, b, u in ((y, xq, xs, wq, ws), (dx, dq, ds, vq, vs)):
            want = (a.astype(float) @ b.astype(float).T) * s.astype(float)[:, None] * u.astype(float)
            err = np.abs(got.detach().double().cpu().numpy() - want)
            assert (err <= np.abs(want) * (ROUND["bf16"] + 2.0 ** -21)).all()
