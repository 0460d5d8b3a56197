"""Layer norm and its gradients against the definition in 64 bits: types, widths, strides, rows of equal or
non-finite values, parameters present or not, arenas written or added to.

Tolerances, u = 2^-24.  No sum over a row takes a value through more than D = 16 + cols / 32 additions, so a mean is off by at most
D u mean|x|; the mean of squares by (D + 6) u of itself (and the square of the mean's error), rstd by half that and three
roundings; y by what these leave and four roundings.  The backward pass is given mean and rstd; its row sums are
bounded likewise, its sums over rows with R + 8 additions for R rows (never more, mostly far fewer)."""
import pytest

from paper_2606_00539_gb300 import GnmrError, LayerNorm, layer_norm

pytestmark = pytest.mark.gpu

import torch  # noqa: E402

from tests.test_gpu_products import LEAST, ROUND, TYPES, gen, normal  # noqa: E402

U = 2.0 ** -24


@pytest.fixture(scope="module")
def norms():
    return LayerNorm(device=0)


def inside(got, want, tol, kind, what):
    got = got.double()
    tol = tol + ROUND[kind] * (want.abs() + tol) + LEAST[kind] + 2.0 ** -140
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} outside, first at {bad.nonzero()[0].tolist()}: "
                           f"{got[bad][0].item()} for {want[bad][0].item()}, tolerance {tol[bad][0].item()}")


def check_forward(y, mean, rstd, x, w, b, eps, kind):
    x = x.double()
    D = 16 + x.shape[1] / 32
    m = x.mean(1, keepdim=True)
    var = (x - m).square().mean(1, keepdim=True)
    r = (var + eps) ** -0.5
    dm = D * U * x.abs().mean(1, keepdim=True)
    # (x - m') is rounded too: u of itself; m' is dm off
    dv = (D + 6) * U * var + 2 * dm * dm + 2 * U * dm * x.abs().mean(1, keepdim=True)
    dr = r * (0.5 * dv / (var + eps) + 4 * U)
    assert mean.dtype == rstd.dtype == torch.float32
    inside(mean[:, None], m, dm + U * m.abs(), "f32", "mean")
    inside(rstd[:, None], r, dr, "f32", "rstd")
    W = 1.0 if w is None else w.double()
    B = torch.zeros((), device="cuda", dtype=torch.float64) if b is None else b.double()
    hat = (x - m) * r
    away = abs(W) * (r * (dm + U * (x - m).abs()) + (x - m).abs() * dr) + 4 * U * ((hat * W).abs() + B.abs())
    inside(y, hat * W + B, 1.01 * away, kind, "y")


def check_backward(dx, dw, db, dy, x, w, mean, rstd, kind, grad_kind, old=(0.0, 0.0)):
    x, dy, m, r = x.double(), dy.double(), mean.double()[:, None], rstd.double()[:, None]
    D, R = 16 + x.shape[1] / 32, len(x)
    W = torch.ones((), device="cuda", dtype=torch.float64) if w is None else w.double()
    hat, t = (x - m) * r, dy * W
    if dx is not None:
        m1, m2 = t.mean(1, keepdim=True), (t * hat).mean(1, keepdim=True)
        s1, s2 = t.abs().mean(1, keepdim=True), (t * hat).abs().mean(1, keepdim=True)
        away = r * ((D + 3) * U * s1 + hat.abs() * (D + 8) * U * s2 + 8 * U * (t.abs() + m1.abs() + (hat * m2).abs()))
        inside(dx, r * (t - m1 - hat * m2), 1.01 * away, kind, "dx")
    for got, terms, before, what in ((dw, dy * hat, old[0], "dw"), (db, dy, old[1], "db")):
        if got is not None:
            want = terms.sum(0) + before
            inside(got, want, (min(R, 600 + R / 100) + 8) * U * (terms.abs().sum(0) + abs(before)), grad_kind, what)


KINDS = [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32")]
# rows, cols: single values, odd widths, what fills a warp or a block of threads and one less or more, long rows
SIZES = [(1, 1), (3, 1), (2, 2), (5, 7), (1, 8), (9, 31), (4, 256), (33, 264), (7, 1000), (300, 512), (65, 1023), (3, 1024),
         (2, 1032), (130, 1371), (1, 5120), (257, 5120), (31, 2048), (2, 8192), (3, 8200), (5, 16384), (1, 30001), (2, 32768),
         (2, 40000), (1000, 64), (3000, 40), (1, 131072)]


@pytest.mark.parametrize("dtype,params", KINDS)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward_and_backward(norms, rows, cols, dtype, params):
    g, t, p = gen(rows * 7 + cols), TYPES[dtype], TYPES[params]
    x = (normal(g, rows, cols, dtype=torch.float32) * 1.5 + 0.7).to(t)
    w, b = 1 + normal(g, cols, dtype=p, size=0.2), normal(g, cols, dtype=p)
    y, mean, rstd = norms.forward(x, w, b, eps=1e-5)
    check_forward(y, mean, rstd, x, w, b, 1e-5, dtype)
    dy = normal(g, rows, cols, dtype=t)
    dw, db = torch.empty(2, cols, dtype=p, device="cuda").unbind()
    dx = norms.backward(dy, x, w, mean, rstd, weight_grad=dw, bias_grad=db)
    check_backward(dx, dw, db, dy, x, w, mean, rstd, dtype, params)
    again = norms.backward(dy, x, w, mean, rstd, weight_grad=dw.clone(), bias_grad=db.clone())
    assert torch.equal(dx, again)


@pytest.mark.parametrize("rows,cols", [(3000, 512), (5000, 1371), (2500, 5120), (40000, 16), (9, 24000)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows(norms, rows, cols, dtype):
    g, t = gen(rows), TYPES[dtype]
    x, dy = normal(g, rows, cols, dtype=t), normal(g, rows, cols, dtype=t)
    w, b = 1 + normal(g, cols, dtype=torch.float32, size=0.2), normal(g, cols, dtype=torch.float32)
    y, mean, rstd = norms.forward(x, w, b)
    check_forward(y, mean, rstd, x, w, b, 1e-5, dtype)
    dw, db = torch.empty(2, cols, device="cuda").unbind()
    dx = norms.backward(dy, x, w, mean, rstd, weight_grad=dw, bias_grad=db)
    check_backward(dx, dw, db, dy, x, w, mean, rstd, dtype, "f32")


@pytest.mark.parametrize("cols", [7, 520, 5120])
def test_parts_that_are_not_there(norms, cols):
    """No weight, no bias, no input gradient, one parameter's gradient alone."""
    g = gen(cols)
    x, dy = normal(g, 40, cols, dtype=torch.bfloat16), normal(g, 40, cols, dtype=torch.bfloat16)
    w, b = 1 + normal(g, cols, dtype=torch.bfloat16, size=0.2), normal(g, cols, dtype=torch.bfloat16)
    for W in (None, w):
        for B in (None, b):
            y, mean, rstd = norms.forward(x, W, B, eps=1e-3)
            check_forward(y, mean, rstd, x, W, B, 1e-3, "bf16")
        for want_w in (True, False):
            for want_b in (True, False):
                for want_x in (True, False):
                    dw = torch.empty(cols, device="cuda") if want_w else None
                    db = torch.empty(cols, device="cuda") if want_b else None
                    dx = norms.backward(dy, x, W, mean, rstd, weight_grad=dw, bias_grad=db, input_grad=want_x)
                    assert (dx is not None) == want_x
                    check_backward(dx, dw, db, dy, x, W, mean, rstd, "bf16", "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols,pad,lead", [(136, 0, 0), (136, 8, 8), (136, 1, 0), (1371, 2, 1), (520, 3, 5), (5120, 64, 16)])
def test_strides_and_arenas(norms, cols, pad, lead, dtype):
    """Rows inside wider ones, parameters and their gradients inside arenas at any start; nothing around is written; in place."""
    g, t, R = gen(cols + pad), TYPES[dtype], 57
    wide = cols + pad + lead
    x, dy = (normal(g, R, wide, dtype=t)[:, lead:lead + cols] for _ in range(2))
    flat = normal(g, 2 * wide, dtype=t, size=0.5)
    w, b = flat[lead:lead + cols], flat[wide + lead:wide + lead + cols]
    out = torch.full((R, wide), 7.0, dtype=t, device="cuda")
    y, mean, rstd = norms.forward(x, w, b, out=out[:, lead:lead + cols])
    check_forward(y, mean, rstd, x, w, b, 1e-5, dtype)
    for kind in ("f32", "bf16", "f16"):
        arena = normal(g, 2 * wide, dtype=TYPES[kind])
        old = arena.clone()
        dw, db = arena[lead:lead + cols], arena[wide + lead:wide + lead + cols]
        before = dw.double(), db.double()
        for add in (False, True):
            to = out.fill_(7.0)[:, lead:lead + cols]
            arena.copy_(old)
            dx = norms.backward(dy, x, w, mean, rstd, out=to, weight_grad=dw, bias_grad=db, add=add)
            check_backward(dx, dw, db, dy, x, w, mean, rstd, dtype, kind, before if add else (0.0, 0.0))
            assert (out[:, :lead] == 7).all() and (out[:, lead + cols:] == 7).all()
            for a, z in ((0, lead), (lead + cols, wide + lead), (wide + lead + cols, 2 * wide)):
                assert torch.equal(arena[a:z], old[a:z])
    # in place
    for a, b_ in ((dy, x), (dy.contiguous(), x.contiguous())):
        dw = torch.empty(cols, device="cuda")
        old = a.clone()
        check_backward(norms.backward(a, b_, w, mean, rstd, out=a, weight_grad=dw), dw, None, old, b_, w, mean, rstd, dtype, "f32")
        old = b_.clone()
        check_forward(*norms.forward(b_, w, b, out=b_), old, w, b, 1e-5, dtype)


def test_no_rows(norms):
    x = torch.empty(0, 40, dtype=torch.bfloat16, device="cuda")
    y, mean, rstd = norms.forward(x)
    assert y.shape == (0, 40) and mean.shape == rstd.shape == (0,)
    dw, db = torch.full((2, 40), 7.0, device="cuda").unbind()
    norms.backward(x, x, None, mean, rstd, weight_grad=dw, bias_grad=db, add=True)
    assert (dw == 7).all() and (db == 7).all()
    norms.backward(x, x, None, mean, rstd, weight_grad=dw, bias_grad=db)
    assert (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("cols", [33, 512, 5120, 40000])
def test_hard_rows(norms, cols):
    """Equal values (no variance), a mean 1,000 times the spread, tiny and huge values, NaN and infinities."""
    g = gen(cols)
    x = normal(g, 9, cols, dtype=torch.float32)
    x[0], x[1] = 0.0, 0.1
    x[2] = x[2] + 1000
    x[3] *= 1e-20
    x[4] *= 1e15
    clean = norms.forward(x, eps=1e-5)
    check_forward(*clean, x, None, None, 1e-5, "f32")
    assert (clean[0][0] == 0).all()
    x[6, cols // 2], x[7, cols - 1] = float("nan"), float("-inf")
    y, mean, rstd = norms.forward(x, eps=1e-5)
    rest = [0, 1, 2, 3, 4, 5, 8]
    assert y[6].isnan().all() and y[7].isnan().all() and mean[6].isnan() and rstd[7].isnan()
    assert torch.equal(y[rest], clean[0][rest]) and torch.equal(mean[rest], clean[1][rest])
    dy = normal(g, 9, cols, dtype=torch.float32)
    dw = torch.empty(cols, device="cuda")
    dx = norms.backward(dy, x, None, mean, rstd, weight_grad=dw)
    assert dx[6].isnan().all() and dx[7].isnan().all() and dx[rest].isfinite().all() and dw.isnan().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols,pad", [(33, 0), (1371, 0), (99, 2), (1000, 1), (64, 0), (2056, 0), (5120, 0), (8192, 0), (20480, 0)])
def test_rows_do_not_meet(norms, cols, pad, dtype):
    """Neighbours of a row, read with it where rows start at odd places, mean nothing: every other row, and the gaps, are NaN."""
    g, t, rows = gen(cols), TYPES[dtype], 1501
    x, dy = (torch.full((rows, cols + pad), float("nan"), dtype=t, device="cuda") for _ in range(2))
    x[::2, :cols], dy[::2, :cols] = normal(g, 751, cols, dtype=t), normal(g, 751, cols, dtype=t)
    x, dy = x[:, :cols], dy[:, :cols]
    y, mean, rstd = norms.forward(x, out=torch.empty_like(x) if pad == 0 else torch.empty(rows, cols + pad, dtype=t, device="cuda")[:, :cols])
    check_forward(y[::2], mean[::2], rstd[::2], x[::2], None, None, 1e-5, dtype)
    assert y[1::2].isnan().all() and mean[1::2].isnan().all()
    dx = norms.backward(dy, x, None, mean, rstd)
    check_backward(dx[::2], None, None, dy[::2], x[::2], None, mean[::2], rstd[::2], dtype, "f32")
    assert dx[1::2].isnan().all()


@pytest.mark.parametrize("rows,cols,dtype", [(3000, 512, "bf16"), (2000, 1371, "bf16"), (2000, 5120, "bf16"), (900, 8192, "f32"),
                                             (800, 16384, "bf16"), (41, 777, "f32")])
def test_statistics_are_optional_and_results_repeat(norms, rows, cols, dtype):
    """The same bits each time, and with the statistics left out (the C call allows either)."""
    import ctypes

    from paper_2606_00539_gb300 import _native as N
    g, t = gen(rows), TYPES[dtype]
    x, w, b = normal(g, rows, cols, dtype=t), normal(g, cols, dtype=t), normal(g, cols, dtype=t)
    y, mean, rstd = norms.forward(x, w, b)
    for _ in range(3):
        assert all(torch.equal(a, z) for a, z in zip(norms.forward(x, w, b), (y, mean, rstd)))
    out = torch.empty_like(y)
    p = N.gnmr_norm(rows, cols, N.GNMR_DTYPE_F32 if dtype == "f32" else N.GNMR_DTYPE_BF16, N.GNMR_DTYPE_F32 if dtype == "f32" else N.GNMR_DTYPE_BF16,
                    1e-5, x.data_ptr(), cols, w.data_ptr(), b.data_ptr(), None, None, out.data_ptr(), cols)
    assert N.load().gnmr_layer_norm(ctypes.addressof(p), torch.cuda.current_stream().cuda_stream) == N.GNMR_OK
    assert torch.equal(out, y)
    dw, db = torch.empty(2, cols, device="cuda").unbind()
    dx = norms.backward(x, x, w, mean, rstd, weight_grad=dw, bias_grad=db)
    first = dx.clone(), dw.clone(), db.clone()
    for _ in range(3):
        dx = norms.backward(x, x, w, mean, rstd, weight_grad=dw, bias_grad=db)
        assert all(torch.equal(a, z) for a, z in zip((dx, dw, db), first))


def test_offsets_past_31_bits_of_elements(norms):
    R, cols = (1 << 21) + 3, 1032
    x = torch.zeros(R, cols, dtype=torch.bfloat16, device="cuda")
    g = gen(2)
    x[-5:] = normal(g, 5, cols, dtype=torch.bfloat16)
    y, mean, rstd = norms.forward(x)
    check_forward(y[-5:], mean[-5:], rstd[-5:], x[-5:], None, None, 1e-5, "bf16")
    dw = torch.empty(cols, device="cuda")
    dx = norms.backward(x, x, None, mean, rstd, weight_grad=dw, out=y)
    check_backward(dx[-5:], dw, None, x[-5:], x[-5:], None, mean[-5:], rstd[-5:], "bf16", "f32")


def test_captured_and_on_other_streams(norms):
    g, t = gen(3), torch.bfloat16
    x, dy, w = normal(g, 700, 1040, dtype=t), normal(g, 700, 1040, dtype=t), 1 + normal(g, 1040, dtype=t, size=0.2)
    dw = torch.empty(1040, device="cuda")
    y, mean, rstd = norms.forward(x, w)
    want = y, norms.backward(dy, x, w, mean, rstd, weight_grad=dw), dw.clone()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    grads = [torch.empty(1040, device="cuda") for _ in streams]
    got = []
    for _ in range(10):                                              # at the same time, each with scratch of its own
        got = [(norms.forward(x, w, stream=s)[0], norms.backward(dy, x, w, mean, rstd, weight_grad=d, stream=s), d)
               for s, d in zip(streams, grads)]
    torch.cuda.synchronize()
    for one in got:
        assert all(torch.equal(a, b) for a, b in zip(one, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y2, mean2, rstd2 = norms.forward(x, w)
        dx2 = norms.backward(dy, x, w, mean2, rstd2, weight_grad=dw)
    x.mul_(-1)
    graph.replay()
    graph.replay()
    assert torch.equal(dw, -want[2]) and torch.equal(mean2, -mean) and dx2.isfinite().all()
    assert torch.equal(y2, norms.forward(x, w)[0])


def test_layer_against_torch(norms):
    """The autograd layer, three dimensions: gradients as torch's in 64 bits, or in the arena; second derivatives refused."""
    g = gen(4)
    x = normal(g, 3, 20, 72, dtype=torch.float32).requires_grad_()
    w, b = (normal(g, 72, dtype=torch.float32).requires_grad_() for _ in range(2))
    dy = normal(g, 3, 20, 72, dtype=torch.float32)
    y = layer_norm(norms, x, w, b)
    got = torch.autograd.grad(y, (x, w, b), dy)
    X, W, B = (t.detach().double().requires_grad_() for t in (x, w, b))
    Y = torch.nn.functional.layer_norm(X, (72,), W, B, 1e-5)
    want = torch.autograd.grad(Y, (X, W, B), dy.double())
    for a, z in zip((y, *got), (Y, *want)):
        # 1e-5 of the largest is some twenty times what the sums' bounds (D = 18, 60 rows) come to
        assert a.shape == z.shape and (a - z).abs().max() <= 1e-5 * z.abs().max()
    arena = torch.full((150,), 7.0, device="cuda")
    layer_norm(norms, x.detach(), w.detach(), b.detach(), (arena[:72], arena[76:148])).backward(dy)
    assert torch.equal(arena[:72], got[1]) and torch.equal(arena[76:148], got[2]) and (arena[72:76] == 7).all()
    layer_norm(norms, x, w, b, (arena[:72], None), add=True).backward(dy)
    assert torch.allclose(arena[:72], 2 * got[1]) and w.grad is None and torch.equal(x.grad, got[0])
    gx, = torch.autograd.grad(layer_norm(norms, x, w, b).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivatives"):
        gx.sum().backward()


def test_gradients_against_differences(norms):
    """Directional derivatives of a loss in fp32: a central difference is step^2 / 6 of third derivatives off (the rows' spread is
    1, the step 2^-7: 1e-4 at most) and 2 u |y c| / step by rounding."""
    g = gen(6)
    x, w, b = normal(g, 30, 50, dtype=torch.float32), normal(g, 50, dtype=torch.float32), normal(g, 50, dtype=torch.float32)
    c = normal(g, 30, 50, dtype=torch.float64)
    args = [v.clone().requires_grad_() for v in (x, w, b)]
    grads = torch.autograd.grad((layer_norm(norms, *args).double() * c).sum(), args)
    for i, v in enumerate((x, w, b)):
        way, step = normal(g, *v.shape, dtype=torch.float32), 2.0 ** -7
        ends = []
        for s in (1, -1):
            moved = [x, w, b]
            moved[i] = v + s * step * way
            ends.append((norms.forward(*moved)[0].double() * c).sum())
        got = (ends[0] - ends[1]) / (2 * step)
        want = (grads[i].double() * way.double()).sum()
        assert (got - want).abs() <= 1e-3 * (grads[i].double() * way.double()).norm() * 10


def test_refusals(norms):
    t = torch.bfloat16
    x, w = torch.zeros(6, 16, dtype=t, device="cuda"), torch.zeros(16, dtype=t, device="cuda")
    m = torch.zeros(6, device="cuda")
    f = torch.zeros(16, device="cuda")
    for call, why in [
        (lambda: norms.forward(x.double()), "must be"), (lambda: norms.forward(x.cpu()), "CUDA"), (lambda: norms.forward(x[0]), "dimensions"),
        (lambda: norms.forward(x.T.contiguous().T), "contiguous"), (lambda: norms.forward(x[:, :0]), "column"),
        (lambda: norms.forward(x, w[:8]), "entries"), (lambda: norms.forward(x, w.half()), "must be"), (lambda: norms.forward(x, w, f), "one type"),
        (lambda: norms.forward(x, out=x[:5]), "out must"), (lambda: norms.forward(x, out=x.float()), "out must"),
        (lambda: norms.forward(x.requires_grad_()), "autograd"),
        (lambda: norms.backward(x.detach()[:5], x.detach(), w, m, m), "dy must"), (lambda: norms.backward(x.detach(), x.detach(), w, m[:5], m), "mean must"),
        (lambda: norms.backward(x.detach(), x.detach(), w, m, None), "given"),
        (lambda: norms.backward(x.detach(), x.detach(), w, m, m, weight_grad=f, bias_grad=w), "one type"),
        (lambda: norms.backward(x.detach(), x.detach(), w, m, m, weight_grad=f[:4]), "entries"),
        (lambda: norms.backward(x.detach(), x.detach(), w, m, m, out=x.detach(), input_grad=False), "out is"),
        (lambda: layer_norm(norms, x, w, None, (f,)), "grad must"),
    ]:
        with pytest.raises(ValueError, match=why):
            call()
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(GnmrError, match="eps"):
            norms.forward(x.detach(), eps=eps)


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 7])
@pytest.mark.parametrize("cols", [777, 1371, 5120, 9001, 16384, 40001])
def test_scratch_of_few_rows(norms, rows, cols):
    """Scratch for so many rows' parts: it is enough, and nothing behind it is written."""
    import ctypes

    from paper_2606_00539_gb300 import _native as N
    g = gen(rows + cols)
    x, dy = (normal(g, rows, cols, dtype=torch.bfloat16) for _ in range(2))
    _, mean, rstd = norms.forward(x)
    dw, db = torch.empty(2, cols, device="cuda").unbind()
    dx = torch.empty_like(x)
    p = N.gnmr_norm(rows, cols, N.GNMR_DTYPE_BF16, N.GNMR_DTYPE_F32, 0.0, x.data_ptr(), cols, None, None, mean.data_ptr(), rstd.data_ptr(), None, 0,
                    dy.data_ptr(), cols, dx.data_ptr(), cols, dw.data_ptr(), db.data_ptr(), N.GNMR_DTYPE_F32, 0)
    need = N.gnmr_layer_norm_scratch_bytes(p)
    scratch = torch.full((need + (1 << 20),), 77, dtype=torch.uint8, device="cuda")
    p.d_scratch, p.scratch_bytes = scratch.data_ptr(), need
    assert N.load().gnmr_layer_norm_grad(ctypes.addressof(p), torch.cuda.current_stream().cuda_stream) == N.GNMR_OK
    check_backward(dx, dw, db, dy, x, None, mean, rstd, "bf16", "f32")
    assert (scratch[need:] == 77).all()


def test_a_row_of_millions_of_columns(norms):
    """The backward pass of a few very wide rows takes memory by the rows: 4 KB a column would be 69 GB here."""
    rows, cols = 3, 1 << 24
    g = gen(11)
    x, dy = (normal(g, rows, cols, dtype=torch.bfloat16) for _ in range(2))
    xd = x.double()
    mean, rstd = xd.mean(1).float(), (xd.var(1, unbiased=False) + 1e-5).rsqrt().float()
    dw, db = torch.empty(2, cols, device="cuda").unbind()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    dx = norms.backward(dy, x, None, mean, rstd, weight_grad=dw, bias_grad=db)
    assert torch.cuda.max_memory_allocated() - before <= rows * cols * 2 + 2 * (rows + 1) * cols * 4 + (4 << 20)
    check_backward(dx, dw, db, dy, x, None, mean, rstd, "bf16", "f32")
