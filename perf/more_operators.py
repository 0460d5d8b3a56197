"""Performance cases of a feed-forward layer's other operators, as they are trained beside the monitor:

* ``gated``      h[r] = act(g) * u with [g, u] = W_e x[r] for the rows r of every group (expert) e, W_e holding the
                 gate's rows and then the other projection's; a training pass keeps [g, u] too, in the operands' type;
* ``gate_grad``  the gradient of [g, u] from that of h and from what was kept;
* ``gated_step`` forward and backward of such a layer, every expert on the path that the mask gives it (16 bits, or
                 8-bit codes), its weights' gradient in the arena.  [g, u] and its gradient are tensors of the operands'
                 type: the products, the codes and the backward pass take them as they are held;
* ``norm``       layer norm by row, and the rows' statistics;
* ``norm_grad``  its gradients: the input's, the weight's and the bias's;
* ``clip``       the norm over many tensors' gradients, and the gradients scaled down to a limit, where they lie
                 (``inplace``) or into other memory.

Rows lie group by group: group g has the rows offsets[g] up to offsets[g+1].
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_handles = {}


def listed():
    return [
        # One token in serving: six of an MoE layer's 64 experts, both projections' weights read once.
        dict(name="gated-token", op="gated", groups=64, n=1408, k=2048, rows=6, dtype="bf16", act="silu", keep=False,
             skew=0.5, unrouted=0.0),
        # A batch of 47 sequences being answered, through a dense 5120 -> 13824 layer.
        dict(name="gated-decode", op="gated", groups=1, n=13824, k=5120, rows=47, dtype="f16", act="silu", keep=False,
             skew=0.0, unrouted=0.0),
        # A training batch of 8,192 tokens, each to six experts: the largest product.
        dict(name="gated-train", op="gated", groups=64, n=1408, k=2048, rows=49152, dtype="bf16", act="silu", keep=True,
             skew=0.5, unrouted=0.1),
        # The same batch on its way back.
        dict(name="gate-grad-train", op="gate_grad", n=1408, rows=49152, dtype="bf16", act="silu"),
        # A training step of the layer, a fifth of the experts on the recovery path.
        dict(name="gated-step", op="gated_step", groups=64, n=1408, k=2048, rows=12288, dtype="bf16", act="silu",
             skew=0.5, unrouted=0.1, recovery=0.2),
        # One sequence's newest token at hidden size 5120.
        dict(name="norm-token", op="norm", rows=1, cols=5120, dtype="bf16", params="bf16", eps=1e-5),
        # A training batch of 16,384 tokens.
        dict(name="norm-train", op="norm", rows=16384, cols=5120, dtype="bf16", params="f32", eps=1e-5),
        # Its backward pass, the parameters' gradients in fp32.
        dict(name="norm-grad-train", op="norm_grad", rows=16384, cols=5120, dtype="bf16", params="f32"),
        # Rows of an odd width in fp32: no two of them start alike.
        dict(name="norm-grad-odd", op="norm_grad", rows=2047, cols=1371, dtype="f32", params="f32"),
        # A small model's 64 fp32 gradients, 4 MB: nothing but latency.
        dict(name="clip-tiny", op="clip", tensors=64, elements=1 << 20, spread=0.5, dtype="f32", mixed=False, inplace=False,
             limit=0.37, norms=False),
        # Two thousand tensors of 16 and 32 bits, from a few elements up, below the limit: only read.
        dict(name="clip-many", op="clip", tensors=2000, elements=60000000, spread=2.0, dtype="bf16", mixed=True, inplace=True,
             limit=2.0, norms=False),
        # The gradients of 24 layers of seven matrices, 2.4 GB of bf16, above the limit.
        dict(name="clip-train", op="clip", tensors=168, elements=1214251008, spread=0.4, dtype="bf16", mixed=False,
             inplace=False, limit=0.37, norms=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["gated", "gated", "gated", "gate_grad", "gated_step", "norm", "norm", "norm_grad", "norm_grad", "clip",
                     "clip"])
    c = dict(op=op, dtype=rng.choice(["bf16", "f16"]))
    if op == "clip":
        tensors = _log(rng, 1, 3000)
        elements = max(tensors, _log(rng, 1 << 12, 1 << 29))
        c.update(dtype=rng.choice(["bf16", "f16", "f32"]), tensors=tensors, elements=elements, spread=rng.choice([0.0, 0.5, 2.0]),
                 mixed=rng.random() < 0.3, limit=rng.choice([0.1, 0.7, 2.0]), norms=rng.random() < 0.2)
        c["inplace"] = c["limit"] > 1 and rng.random() < 0.5
        return c
    if op in ("norm", "norm_grad"):
        step = rng.choice([1, 1, 8, 64, 256])
        c["dtype"] = rng.choice(["bf16", "f16", "f32"])
        c["cols"] = max(1, _log(rng, 16, 20000) // step) * step
        c["rows"] = _log(rng, 1, min(60000, (80 << 20) // c["cols"]))
        c["params"] = rng.choice([c["dtype"], "f32"])
        if op == "norm":
            c["eps"] = rng.choice([1e-5, 1e-6])
        return c
    c["act"] = rng.choice(["silu", "silu", "gelu"])
    # widths mostly in whole 16-byte rows, one in six of any size
    step = rng.choice([1, 8, 16, 64, 64, 64])
    if op == "gate_grad":
        c["n"] = max(1, _log(rng, 96, 13824) // step) * step
        c["rows"] = _log(rng, 1, min(60000, int(7e7 / c["n"])))
        return c
    c["groups"] = rng.choice([1, 1, _log(rng, 2, 96)])
    most = 13824 if c["groups"] == 1 else 2600
    c["n"], c["k"] = (max(1, _log(rng, 96, most) // step) * step for _ in range(2))
    room = min(49000, int(1.4e11 / (c["n"] * c["k"])))
    c["rows"] = _log(rng, 1, room)
    c["skew"] = rng.choice([0.0, 0.5, 0.8]) if c["groups"] > 1 else 0.0
    c["unrouted"] = rng.choice([0.0, 0.3]) if c["groups"] > 1 else 0.0
    if op == "gated":
        c["keep"] = rng.random() < 0.5
    else:
        c.update(recovery=rng.choice([0.0, 0.2, 1.0]), rows=min(c["rows"], 12288))
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


def _layout(case):
    """(type, first element, length) of every tensor in the flat memory of its type, and that memory's sizes: starts at
    multiples of 16 bytes, and one in eight behind a neighbour of odd size."""
    rng = np.random.default_rng([case["tensors"], case["elements"], 29])
    size = np.exp(case["spread"] * rng.standard_normal(case["tensors"]))
    size = np.maximum((size * (case["elements"] / size.sum())).astype(np.int64), 1)
    kinds = ["bf16", "f16", "f32"] if case["mixed"] else [case["dtype"]]
    at, tensors = dict.fromkeys(kinds, 0), []
    for n, kind, packed in zip(size.tolist(), rng.integers(0, len(kinds), len(size)), rng.random(len(size)) < 0.125):
        kind = kinds[kind]
        first = at[kind] if packed else (at[kind] + 7) // 8 * 8
        tensors.append((kind, first, n))
        at[kind] = first + n
    return tensors, {kind: (n + 7) // 8 * 8 for kind, n in at.items()}


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 11)
    op, t = case["op"], TYPES[case["dtype"]]
    s = dict(case=case)

    def acts(rows, cols):
        # activations: every token with a magnitude of its own
        size = torch.exp(0.5 * torch.randn(rows, 1, device=DEV, generator=g))
        return (torch.randn(rows, cols, device=DEV, generator=g) * size).to(t)

    if op == "clip":
        return _prepare_clip(case, g, s)
    if op in ("norm", "norm_grad"):
        R, C, p = case["rows"], case["cols"], TYPES[case["params"]]
        # a residual stream: every channel with an offset of its own
        s["x"] = (acts(R, C).float() + 0.3 * torch.randn(C, device=DEV, generator=g)).to(t)
        s["w"] = (1 + 0.2 * torch.randn(C, device=DEV, generator=g)).to(p)
        s["b"] = (0.2 * torch.randn(C, device=DEV, generator=g)).to(p)
        if op == "norm_grad":
            s["dy"] = acts(R, C) * 2.0 ** -7
            x = s["x"].double()
            mean = x.mean(1)
            s["mean"], s["rstd"] = mean.float(), (x.var(1, unbiased=False) + 1e-5).rsqrt().float()
            s["dw"], s["db"] = (torch.empty(C, dtype=p, device=DEV) for _ in range(2))
        return s
    R, N = case["rows"], case["n"]
    if op == "gate_grad":
        s["gu"], s["dh"] = acts(R, 2 * N), acts(R, N) * 2.0 ** -7
        return s
    G, K = case["groups"], case["k"]
    counts = _counts(case, seed)
    s["most"] = max(1, int(counts.max()))
    s["offsets"] = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)])).to(DEV)
    s["x"] = acts(R, K)
    s["w"] = torch.empty(G, 2 * N, K, dtype=t, device=DEV).normal_(0.0, 1.0 / math.sqrt(K), generator=g)
    if op == "gated_step":
        s["dh"] = acts(R, N) * 2.0 ** -7
        s["arena"] = torch.empty(G, 2 * N, K, dtype=t, device=DEV).normal_(0.0, 2.0 ** -7, generator=g)
        s["mask"] = (torch.rand(G, device=DEV, generator=g) < case["recovery"]).to(torch.uint8)
    elif case["keep"]:
        s["keep"] = torch.empty(R, 2 * N, dtype=t, device=DEV)
    return s


def _prepare_clip(case, g, s):
    tensors, sizes = _layout(case)
    flat = {k: torch.zeros(n, dtype=TYPES[k], device=DEV) for k, n in sizes.items()}
    s["grads"] = [flat[k][at:at + n] for k, at, n in tensors]
    # gradients: every tensor with a scale of its own
    scales = torch.exp(torch.randn(len(tensors), device=DEV, generator=g)) * 2.0 ** -9
    if len(tensors) > 64 and case["spread"] > 1:
        for k, f in flat.items():
            f.normal_(0.0, 2.0 ** -9, generator=g)
            inside = torch.zeros(len(f) + 1, dtype=torch.int32, device=DEV)
            ends = torch.tensor([(at, at + n) for q, at, n in tensors if q == k], device=DEV).reshape(-1, 2)
            one = torch.ones(len(ends), dtype=torch.int32, device=DEV)
            inside.index_add_(0, ends[:, 0], one).index_add_(0, ends[:, 1], -one)
            f.mul_(inside.cumsum(0)[:-1].to(f.dtype))
    else:
        for x, scale in zip(s["grads"], scales.tolist()):
            x.normal_(0.0, scale, generator=g)
    s["flat"] = [flat[k] for k in sorted(flat)]
    out = flat if case["inplace"] else {k: torch.zeros_like(f) for k, f in flat.items()}
    s["out"] = [out[k] for k in sorted(out)]
    s["outs"] = None if case["inplace"] else [out[k][at:at + n] for k, at, n in tensors]
    norms = torch.stack([x.double().square().sum() for x in s["flat"]]).sqrt()
    s["max_norm"] = case["limit"] * float(norms.square().sum().sqrt())
    # the monitor's norms of its units, here one for each type's memory
    s["norms"] = norms if case["norms"] else None
    return s


# -- one pass -----------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _handle(kind):
    if kind not in _handles:
        _handles[kind] = kind(device=0)
    return _handles[kind]


def _run_own(s):
    import paper_2606_00539_gb300 as gnmr
    c = s["case"]
    op = c["op"]
    if op == "clip":
        if "clip" not in s:                        # the plan that a program keeps for its gradients
            plan = gnmr.GradientClip(s["grads"])
            s["clip"] = plan.prepare_clip(s["grads"], s["max_norm"], out=s["outs"], unit_norms=s["norms"])
        return s["clip"](), *s["out"]
    if op == "norm":
        return _handle(gnmr.LayerNorm).forward(s["x"], s["w"], s["b"], eps=c["eps"])
    if op == "norm_grad":
        dx = _handle(gnmr.LayerNorm).backward(s["dy"], s["x"], s["w"], s["mean"], s["rstd"], weight_grad=s["dw"],
                                              bias_grad=s["db"])
        return dx, s["dw"], s["db"]
    p = _handle(gnmr.ExpertProducts)
    if op == "gated":
        h = p.gated(s["x"], s["w"], s["offsets"], keep=s.get("keep"), activation=c["act"])
        return (h, s["keep"]) if c["keep"] else h
    if op == "gate_grad":
        return p.gate_grad(s["dh"], s["gu"], activation=c["act"])
    x = s["x"].requires_grad_()
    h = gnmr.expert_gated(p, x, s["w"], s["offsets"], s["mask"], s["arena"], activation=c["act"])
    dx, = torch.autograd.grad(h, x, s["dh"])
    return h.detach(), dx, s["arena"]


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


def _codes(x, dim):
    """8-bit codes of x and their scales over `dim`: the inverse of the scale in 32 bits, halves to even."""
    amax = x.float().abs().amax(dim, keepdim=True)
    tiny = amax < 127.0 / torch.finfo(torch.float32).max
    q = torch.round(x.float() * torch.where(tiny, 0.0, 127.0 * (1 / amax)))
    return q, torch.where(tiny, 0.0, amax / 127.0).squeeze(dim)


def _act(g, act):
    """The activation and its derivative."""
    if act == "silu":
        sig = 1 / (1 + torch.exp(-g))
        return g * sig, sig * (1 + g * (1 - sig))
    up = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
    return g * up, up + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))


def _gate(gu, act):
    g, u = gu.chunk(2, -1)
    return _act(g, act)[0] * u


def _gate_grad(dh, gu, act):
    g, u = gu.chunk(2, -1)
    a, d = _act(g, act)
    return torch.cat([dh * u * d, dh * a], -1)


def _run_plain(s):
    c = s["case"]
    op, t = c["op"], TYPES[c["dtype"]]
    if op == "clip":
        return _clip_plain(s)
    if op == "norm":
        x = s["x"].float()
        mean = x.mean(1)
        x = x - mean[:, None]
        rstd = 1 / torch.sqrt(x.square().mean(1) + c["eps"])
        return (x * rstd[:, None] * s["w"].float() + s["b"].float()).to(t), mean, rstd
    if op == "norm_grad":
        xh = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        dy = s["dy"].float()
        s["dw"].copy_((dy * xh).sum(0))
        s["db"].copy_(dy.sum(0))
        d = dy * s["w"].float()
        dx = s["rstd"][:, None] * (d - d.mean(1, keepdim=True) - xh * (d * xh).mean(1, keepdim=True))
        return dx.to(t), s["dw"], s["db"]
    if op == "gate_grad":
        return _gate_grad(s["dh"].float(), s["gu"].float(), c["act"]).to(t)
    x, w = s["x"].detach(), s["w"]
    gu, g = _ragged(s, torch.bmm(_padded(s, x), w.float().transpose(1, 2)))
    if op == "gated":
        h = _gate(gu, c["act"]).to(t)
        return (h, s["keep"].copy_(gu)) if c["keep"] else h
    # the step: both paths everywhere, then each row takes its expert's
    (xq, xs), (wq, ws), (vq, vs) = _codes(x, -1), _codes(w, -1), _codes(w, -2)
    high = s["mask"].bool()[g][:, None]
    low = (_ragged(s, torch.bmm(_padded(s, xq), wq.transpose(1, 2)))[0] * xs[:, None] * ws[g]).to(t).float()
    h = torch.where(high, _gate(gu, c["act"]), _gate(low, c["act"])).to(t)
    dgu = _gate_grad(s["dh"].float(), torch.where(high, gu.to(t).float(), low), c["act"]).to(t)
    dq, ds = _codes(dgu, -1)
    dx = _ragged(s, torch.bmm(_padded(s, dgu), w.float()))[0]
    low = _ragged(s, torch.bmm(_padded(s, dq), vq))[0] * ds[:, None] * vs[g]
    s["arena"].copy_(torch.bmm(_padded(s, dgu).transpose(1, 2), _padded(s, x)))
    return h, torch.where(high, dx, low).to(t), s["arena"]


def _clip_plain(s):
    """All tensors lie in one flat memory for each type, zeros between them."""
    if s["norms"] is not None:
        norm = s["norms"].square().sum().sqrt()
    else:
        norm = torch.stack([f.float().square().sum(dtype=torch.float64) for f in s["flat"]]).sum().sqrt()
    scale = (s["max_norm"] / norm).clamp(max=1.0).float()
    return norm.float(), *[o.copy_(f.float() * scale) for o, f in zip(s["out"], s["flat"])]


# -- what a pass cannot do without ----------------------------------------------

def work(case):
    op, size = case["op"], {"bf16": 2, "f16": 2, "f32": 4}
    if op == "clip":
        bytes_, count = sum(size[k] * n for k, _, n in _layout(case)[0]), sum(n for _, _, n in _layout(case)[0])
        moved = 2 * bytes_ if not case["inplace"] else 0 if case["norms"] else bytes_
        return {"bytes": moved + 4 + (8 if case["norms"] else 0), "flops": 2 * count}
    e = size[case["dtype"]]
    if op in ("norm", "norm_grad"):
        R, C, p = case["rows"], case["cols"], size[case["params"]]
        if op == "norm":
            return {"bytes": 2 * e * R * C + 2 * p * C + 8 * R, "flops": 8 * R * C}
        return {"bytes": 3 * e * R * C + 3 * p * C + 8 * R, "flops": 14 * R * C}
    R, N = case["rows"], case["n"]
    if op == "gate_grad":
        return {"bytes": 10 * R * N, "flops": 12 * R * N}
    G, K = case["groups"], case["k"]
    routed = int((_counts(case, 0) > 0).sum())
    product = 4 * R * N * K
    if op == "gated":
        return {"bytes": 2 * R * (K + N) + (4 * R * N if case["keep"] else 0) + 4 * routed * N * K, "flops": product}
    return {"bytes": 4 * R * (N + K) + 4 * (routed + G) * N * K, "flops": 3 * product}


# -- the definition in 64 bits ----------------------------------------------------

def _exact_act(g, act):
    """act(g), act'(g)."""
    if act == "silu":
        sig = torch.sigmoid(g)
        return g * sig, sig + g * sig * torch.sigmoid(-g)
    cdf = 0.5 * torch.erfc(-g / math.sqrt(2.0))
    return g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def _exact_codes(x, dim):
    """(codes, scales): the inverse, the factor and each scaled value are 32-bit numbers by definition."""
    top = x.double().abs().amax(dim, keepdim=True)
    up = (127.0 * (1.0 / top).float().double()).float().double()
    dead = top < 127.0 / float(np.finfo(np.float32).max)
    code = (x.double() * up.masked_fill(dead, 0.0)).float().double().round()
    return code, (top / 127.0).float().double().masked_fill(dead, 0.0).squeeze(dim)


def _exact_gate_grad(dh, gu, act):
    n = dh.shape[1]
    a, d = _exact_act(gu[:, :n], act)
    return torch.cat([dh * gu[:, n:] * d, dh * a], 1)


def exact(case, seed):
    s = prepare(case, seed)
    op, t = case["op"], TYPES[case["dtype"]]
    if op == "clip":
        total = 0.0
        for f in s["flat"]:
            for part in f.split(1 << 27):
                total += float(part.double().norm()) ** 2
        if s["norms"] is not None:
            total = float((s["norms"] ** 2).sum())
        scale = min(1.0, s["max_norm"] / math.sqrt(total))
        return torch.tensor(math.sqrt(total), dtype=torch.float64, device=DEV), *[f.double() * scale for f in s["flat"]]
    if op == "norm":
        x = s["x"].double()
        mean, var = x.mean(1), x.var(1, unbiased=False)
        rstd = (var + case["eps"]) ** -0.5
        return torch.addcmul(s["b"].double(), (x - mean[:, None]) * rstd[:, None], s["w"].double()), mean, rstd
    if op == "norm_grad":
        r, dy = s["rstd"].double()[:, None], s["dy"].double()
        hat = (s["x"].double() - s["mean"].double()[:, None]) * r
        pull = dy * s["w"].double()
        C = case["cols"]
        along = (pull * hat).sum(1, keepdim=True) / C
        return r * (pull - pull.sum(1, keepdim=True) / C - hat * along), (dy * hat).sum(0), dy.sum(0)
    if op == "gate_grad":
        return _exact_gate_grad(s["dh"].double(), s["gu"].double(), case["act"])
    cut = s["offsets"].tolist()
    spans = [(e, slice(cut[e], cut[e + 1])) for e in range(case["groups"])]

    def by_group(a, w, side):
        """Rows of a through w[e] (side "out": along its inputs, "in": along its outputs)."""
        y = torch.zeros(case["rows"], w.shape[1] if side == "out" else w.shape[2], dtype=torch.float64, device=DEV)
        for e, at in spans:
            if at.stop > at.start:
                m = w[e].double()
                y[at] = a[at].double() @ (m.T if side == "out" else m)
        return y

    n = case["n"]
    gu = by_group(s["x"], s["w"], "out")
    if op == "gated":
        h = _exact_act(gu[:, :n], case["act"])[0] * gu[:, n:]
        return (h, gu) if case["keep"] else h
    of_row = torch.repeat_interleave(torch.arange(case["groups"], device=DEV), s["offsets"].diff())
    high = (s["mask"] != 0)[of_row][:, None]
    (xq, xs), (wq, ws), (vq, vs) = _exact_codes(s["x"], 1), _exact_codes(s["w"], 2), _exact_codes(s["w"], 1)
    low = (by_group(xq, wq, "out") * xs[:, None] * ws[of_row]).to(t).double()
    from_gu = torch.where(high, gu, low)
    h = _exact_act(from_gu[:, :n], case["act"])[0] * from_gu[:, n:]
    dgu = _exact_gate_grad(s["dh"].double(), from_gu.to(t).double(), case["act"]).to(t)
    dq, ds = _exact_codes(dgu, 1)
    dx = torch.where(high, by_group(dgu, s["w"], "in"), by_group(dq, vq, "in") * ds[:, None] * vs[of_row])
    dw = torch.zeros(s["w"].shape, dtype=torch.float64, device=DEV)
    for e, at in spans:
        dw[e] = dgu[at].double().T @ s["x"][at].double()
    return h, dx, dw
