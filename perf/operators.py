"""Performance cases of the expert products: the linear units that the recovery mask chooses
a path for, in 16 bits and in 8-bit integers, grouped by expert over ragged rows.

Each case is one pass of ``run`` through one operator:

* ``forward``      y[r] = W_g x[r] for the rows r of every group (expert) g;
* ``input_grad``   dx[r] = W_g^T dy[r];
* ``weight_grad``  dW_g = sum over the group's rows of dy[r] x[r]^T, written (or added) into
                   a gradient arena, a group without rows included;
* ``rows_i8``      8-bit codes and one scale for every row (a token, an output channel);
* ``columns_i8``   8-bit codes, transposed, and one scale for every column (an input channel);
* ``forward_i8``   y[r] = xs[r] * ws_g * (Wq_g xq[r]) on such codes;
* ``layer``        a training step of one expert layer: forward and backward, every expert on
                   the path that the mask gives it, and its gradient in the arena.

Rows lie group by group: group g has the rows offsets[g] up to offsets[g+1].
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_products = []


def listed():
    return [
        # One token in serving: six of an MoE layer's 64 experts, their weights read once.
        dict(name="forward-token", op="forward", groups=64, n=1408, k=2048, rows=6, dtype="bf16", out="bf16",
             skew=0.5, unrouted=0.0),
        # A batch of 47 sequences being answered, through the experts' down projection.
        dict(name="forward-decode", op="forward", groups=64, n=2048, k=1408, rows=282, dtype="f16", out="f16",
             skew=0.5, unrouted=0.0),
        # A training batch of 8,192 tokens, each to six experts.
        dict(name="forward-train", op="forward", groups=64, n=1408, k=2048, rows=49152, dtype="bf16", out="bf16",
             skew=0.5, unrouted=0.0),
        # Its backward pass to the layer's input, with an odd number of tokens left.
        dict(name="input-grad-train", op="input_grad", groups=64, n=1408, k=2048, rows=24571, dtype="bf16", out="bf16",
             skew=0.5, unrouted=0.1),
        # The gradient of the experts' weights, 30 % of them unrouted, written into a bf16 arena.
        dict(name="weight-grad-train", op="weight_grad", groups=64, n=1408, k=2048, rows=24571, dtype="bf16", out="bf16",
             skew=0.5, unrouted=0.3, add=False),
        # Adding a further micro-batch's gradient to an fp32 arena: a dense 2048 x 5504 linear.
        dict(name="weight-grad-add", op="weight_grad", groups=1, n=2048, k=5504, rows=2047, dtype="bf16", out="f32",
             skew=0.0, unrouted=0.0, add=True),
        # A batch's activations at hidden size 5120 to codes.
        dict(name="rows-i8", op="rows_i8", groups=1, n=0, k=5120, rows=4096, dtype="bf16", skew=0.0, unrouted=0.0),
        # The weights of an MoE layer's experts to codes for the backward product.
        dict(name="columns-i8", op="columns_i8", groups=64, n=1408, k=2048, rows=0, dtype="bf16", skew=0.0, unrouted=0.0),
        # One token through a dense 5120 -> 13824 linear whose weights are held in 8 bits.
        dict(name="i8-token", op="forward_i8", groups=1, n=13824, k=5120, rows=1, dtype="bf16", out="bf16",
             skew=0.0, unrouted=0.0),
        # A prompt of 4,001 tokens through the same: the largest product.
        dict(name="i8-prompt", op="forward_i8", groups=1, n=13824, k=5120, rows=4001, dtype="bf16", out="bf16",
             skew=0.0, unrouted=0.0),
        # Experts of odd sizes, fp32 results.
        dict(name="i8-experts-odd", op="forward_i8", groups=24, n=1003, k=1371, rows=5003, dtype="f16", out="f32",
             skew=0.8, unrouted=0.2),
        # A training step of one expert layer, a fifth of the experts on the recovery path.
        dict(name="layer-train", op="layer", groups=64, n=1408, k=2048, rows=12288, dtype="bf16", out="f32",
             skew=0.5, unrouted=0.1, recovery=0.2),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["forward", "forward", "input_grad", "weight_grad", "rows_i8", "columns_i8", "forward_i8", "forward_i8",
                     "layer"])
    c = dict(op=op, groups=rng.choice([1, 1, _log(rng, 2, 96)]), dtype=rng.choice(["bf16", "f16"]))
    # widths mostly in whole 16-byte rows, one in six of any size
    step = rng.choice([1, 8, 16, 64, 64, 64])
    most = 13824 if c["groups"] == 1 else 2600
    c["n"], c["k"] = (max(1, _log(rng, 96, most) // step) * step for _ in range(2))
    room = min(50000, int(3e11 / (c["n"] * c["k"])))
    c["rows"] = _log(rng, 1, room)
    c["skew"] = rng.choice([0.0, 0.5, 0.8]) if c["groups"] > 1 else 0.0
    c["unrouted"] = rng.choice([0.0, 0.3]) if c["groups"] > 1 else 0.0
    if op in ("forward", "input_grad"):
        c["out"] = c["dtype"]
    elif op == "weight_grad":
        c.update(out=rng.choice(["f32", c["dtype"]]), add=rng.random() < 0.5)
    elif op == "forward_i8":
        c["out"] = rng.choice([c["dtype"], "f32"])
    elif op == "rows_i8":
        c.update(groups=1, n=0, skew=0.0, unrouted=0.0, rows=min(c["rows"], 16384))
    elif op == "columns_i8":
        c.update(rows=0, skew=0.0, unrouted=0.0)
    else:
        c.update(out=rng.choice(["f32", c["dtype"]]), recovery=0.2, rows=min(c["rows"], 12288))
    for f in ("n", "k", "rows"):
        if c[f] == 3 << 10:
            c[f] -= step
    return c


# -- inputs -------------------------------------------------------------------

def _counts(case, seed):
    """Rows of each group: an uneven router, some experts without any."""
    rng = np.random.default_rng([seed, 17])
    p = np.exp(case["skew"] * rng.standard_normal(case["groups"]))
    p[rng.random(case["groups"]) < case["unrouted"]] = 0.0
    if not p.any():
        p[0] = 1.0
    return rng.multinomial(case["rows"], p / p.sum())


def _codes(x, dim):
    """8-bit codes of x and their scales over `dim`: the inverse of the scale in 32 bits, halves to even."""
    amax = x.float().abs().amax(dim, keepdim=True)
    tiny = amax < 127.0 / torch.finfo(torch.float32).max
    q = torch.round(x.float() * torch.where(tiny, 0.0, 127.0 / amax)).to(torch.int8)
    return q, torch.where(tiny, 0.0, amax / 127.0).squeeze(dim)


def _room16(q):
    """The codes with every row starting at a multiple of 16 bytes, as the quantizing calls hand them out."""
    k = q.shape[-1]
    held = torch.zeros(*q.shape[:-1], (k + 15) // 16 * 16, dtype=torch.int8, device=q.device)
    held[..., :k] = q
    return held[..., :k]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 11)
    op, G, N, K, R = (case[f] for f in ("op", "groups", "n", "k", "rows"))
    t = TYPES[case["dtype"]]
    s = dict(case=case)

    def acts(rows, cols):
        # activations: every token with a magnitude of its own
        size = torch.exp(0.5 * torch.randn(rows, 1, device=DEV, generator=g))
        return (torch.randn(rows, cols, device=DEV, generator=g) * size).to(t)

    def weights():
        w = torch.empty(G, N, K, dtype=t, device=DEV)
        w.normal_(0.0, 1.0 / math.sqrt(K), generator=g)
        return w

    if op == "rows_i8":
        s["x"] = acts(R, K)
        return s
    if op == "columns_i8":
        s["w"] = weights()
        return s
    counts = _counts(case, seed)
    s["most"] = max(1, int(counts.max()))
    s["offsets"] = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)])).to(DEV)
    if op in ("forward", "weight_grad", "layer", "forward_i8"):
        s["x"] = acts(R, K)
    if op in ("input_grad", "weight_grad", "layer"):
        s["dy"] = acts(R, N) * 2.0 ** -7
    if op != "weight_grad":
        s["w"] = weights()
    if op == "forward_i8":
        (s["xq"], s["xs"]), (s["wq"], s["ws"]) = _codes(s.pop("x"), -1), _codes(s.pop("w"), -1)
        s["xq"], s["wq"] = _room16(s["xq"]), _room16(s["wq"])
    if op in ("weight_grad", "layer"):
        s["arena"] = torch.empty(G, N, K, dtype=TYPES[case["out"]], device=DEV)
        s["arena"].normal_(0.0, 2.0 ** -7, generator=g)
        s["start"] = s["arena"].clone() if case.get("add") else None
    if op == "layer":
        s["mask"] = (torch.rand(G, device=DEV, generator=g) < case["recovery"]).to(torch.uint8)
    return s


# -- one pass -----------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2606_00539_gb300 import ExpertProducts, expert_linear
    if not _products:
        _products.append(ExpertProducts(device=0))
    p, c = _products[0], s["case"]
    op = c["op"]
    if op == "forward":
        return p.forward(s["x"], s["w"], s["offsets"])
    if op == "input_grad":
        return p.input_grad(s["dy"], s["w"], s["offsets"])
    if op == "weight_grad":
        if c["add"]:
            s["arena"].copy_(s["start"])
        return p.weight_grad(s["dy"], s["x"], s["offsets"], out=s["arena"], add=c["add"])
    if op == "rows_i8":
        return p.quantize_rows(s["x"])
    if op == "columns_i8":
        return p.quantize_columns(s["w"])
    if op == "forward_i8":
        return p.forward_i8(s["xq"], s["xs"], s["wq"], s["ws"], s["offsets"], out_dtype=c["out"])
    x = s["x"].requires_grad_()
    y = expert_linear(p, x, s["w"], s["offsets"], s["mask"], s["arena"])
    dx, = torch.autograd.grad(y, x, s["dy"])
    return y.detach(), dx, s["arena"]


def _padded(s, x):
    """The rows of x by group, [groups, most, width] in 32 bits, zeros after a group's last."""
    off = s["offsets"]
    at = torch.arange(s["most"], device=DEV) + off[:-1, None]
    x = x[at.clamp(max=len(x) - 1)].float()
    return x.masked_fill_((at >= off[1:, None])[..., None], 0.0)


def _ragged(s, y):
    """The inverse: [rows, width] from [groups, most, width]."""
    off = s["offsets"]
    r = torch.arange(s["case"]["rows"], device=DEV)
    g = torch.searchsorted(off[1:].contiguous(), r, right=True)
    return y[g, r - off[g]], g


def _run_plain(s):
    c = s["case"]
    op = c["op"]
    if op == "rows_i8":
        return _codes(s["x"], -1)
    if op == "columns_i8":
        q, scale = _codes(s["w"], -2)
        return q.transpose(1, 2).contiguous(), scale
    t, o = TYPES[c["dtype"]], TYPES.get(c.get("out"))
    if op == "forward":
        return _ragged(s, torch.bmm(_padded(s, s["x"]), s["w"].float().transpose(1, 2)))[0].to(o)
    if op == "input_grad":
        return _ragged(s, torch.bmm(_padded(s, s["dy"]), s["w"].float()))[0].to(o)
    if op == "weight_grad":
        dw = torch.bmm(_padded(s, s["dy"]).transpose(1, 2), _padded(s, s["x"]))
        s["arena"].copy_(dw + s["start"].float() if c["add"] else dw)
        return s["arena"]
    if op == "forward_i8":
        y, g = _ragged(s, torch.bmm(_padded(s, s["xq"]), s["wq"].float().transpose(1, 2)))
        return (y * s["xs"][:, None] * s["ws"][g]).to(o)
    # the layer: both paths everywhere, then each row takes its expert's
    with torch.no_grad():
        x, dy, w = s["x"], s["dy"], s["w"]
        (xq, xs), (dq, ds) = _codes(x, -1), _codes(dy, -1)
        (wq, ws), (vq, vs) = _codes(w, -1), _codes(w, -2)
        xp, dp = _padded(s, x), _padded(s, dy)
        y, g = _ragged(s, torch.bmm(xp, w.float().transpose(1, 2)))
        low = _ragged(s, torch.bmm(_padded(s, xq), wq.float().transpose(1, 2)))[0] * xs[:, None] * ws[g]
        high = s["mask"].bool()[g][:, None]
        y = torch.where(high, y, low).to(t)
        dx = _ragged(s, torch.bmm(dp, w.float()))[0]
        low = _ragged(s, torch.bmm(_padded(s, dq), vq.float()))[0] * ds[:, None] * vs[g]
        dx = torch.where(high, dx, low).to(t)
        s["arena"].copy_(torch.bmm(dp.transpose(1, 2), xp))
    return y, dx, s["arena"]


# -- what a pass cannot do without ----------------------------------------------

def work(case):
    op, G, N, K, R = (case[f] for f in ("op", "groups", "n", "k", "rows"))
    if op == "rows_i8":
        return {"bytes": 3 * R * K + 4 * R, "flops": 2 * R * K}
    if op == "columns_i8":
        return {"bytes": 3 * G * N * K + 4 * G * K, "flops": 2 * G * N * K}
    o = 4 if case["out"] == "f32" else 2
    routed = int((_counts(case, 0) > 0).sum())
    product = 2 * R * N * K
    if op in ("forward", "input_grad"):
        return {"bytes": 2 * R * (N + K) + 2 * routed * N * K, "flops": product}
    if op == "weight_grad":
        touched = 2 * routed if case["add"] else G
        return {"bytes": 2 * R * (N + K) + o * touched * N * K, "flops": product}
    if op == "forward_i8":
        return {"bytes": R * (K + o * N + 4) + routed * N * (K + 4), "flops": product}
    return {"bytes": 4 * R * (N + K) + (2 * routed + o * G) * N * K, "flops": 3 * product}


# -- the definition in 64 bits ----------------------------------------------------

def _exact_codes(x, dim):
    """(codes, scales): both factors are 32-bit numbers by definition, and so is each scaled value before it is rounded."""
    top = x.double().abs().amax(dim, keepdim=True)
    up = (127.0 / top).float().double()
    dead = top < 127.0 / float(np.finfo(np.float32).max)
    code = (x.double() * up.masked_fill(dead, 0.0)).float().double().round()
    return code, (top / 127.0).float().double().masked_fill(dead, 0.0).squeeze(dim)


def exact(case, seed):
    s = prepare(case, seed)
    op, G = case["op"], case["groups"]
    if op == "rows_i8":
        q, scale = _exact_codes(s["x"], 1)
        return q.to(torch.int8), scale
    if op == "columns_i8":
        q, scale = _exact_codes(s["w"], 1)
        return q.permute(0, 2, 1).to(torch.int8).contiguous(), scale
    cut = s["offsets"].tolist()
    spans = [(e, slice(cut[e], cut[e + 1])) for e in range(G)]
    f8 = dict(dtype=torch.float64, device=DEV)
    rows = case["rows"]

    def by_group(a, w, side):
        """Rows of a through w[e] (side "out": along its inputs, "in": along its outputs)."""
        y = torch.zeros(rows, w.shape[1] if side == "out" else w.shape[2], **f8)
        for e, at in spans:
            if at.stop > at.start:
                m = w[e].double()
                y[at] = a[at].double() @ (m.T if side == "out" else m)
        return y

    def outer(a, b, start=None):
        d = torch.zeros(G, a.shape[1], b.shape[1], **f8)
        for e, at in spans:
            d[e] = a[at].double().T @ b[at].double()
        return d if start is None else d + start.double()

    if op == "forward":
        return by_group(s["x"], s["w"], "out")
    if op == "input_grad":
        return by_group(s["dy"], s["w"], "in")
    if op == "weight_grad":
        return outer(s["dy"], s["x"], s["start"])
    of_row = torch.repeat_interleave(torch.arange(G, device=DEV), s["offsets"].diff())
    if op == "forward_i8":
        return by_group(s["xq"], s["wq"], "out") * s["xs"].double()[:, None] * s["ws"].double()[of_row]
    high = (s["mask"] != 0)[of_row][:, None]
    xq, xs = _exact_codes(s["x"], 1)
    wq, ws = _exact_codes(s["w"], 2)
    dq, ds = _exact_codes(s["dy"], 1)
    vq, vs = _exact_codes(s["w"], 1)
    y = torch.where(high, by_group(s["x"], s["w"], "out"), by_group(xq, wq, "out") * xs[:, None] * ws[of_row])
    dx = torch.where(high, by_group(s["dy"], s["w"], "in"), by_group(dq, vq, "in") * ds[:, None] * vs[of_row])
    return y, dx, outer(s["dy"], s["x"])
