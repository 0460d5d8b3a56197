"""The expert products in a training loop with the monitor: a small mixture of experts whose
weight gradients are written straight into the arena that the monitor reads, one unit per
expert, and whose experts take the path that the previous step's mask gives them.

Every step: the monitor's norms against the norms of the gradients that autograd gets in fp32 for
the same path, and outputs of unselected experts against the definition on 8-bit
codes."""
import numpy as np
import pytest

from paper_2606_00539_gb300 import ExpertProducts, Monitor, expert_linear

pytestmark = pytest.mark.gpu

EXPERTS, HIDDEN, FFN, TOKENS, TOP, STEPS = 12, 136, 72, 200, 2, 8


def route(torch, logits):
    """Each token to its TOP experts: the tokens' copies by expert, and the offsets."""
    chosen = logits.topk(TOP, dim=1).indices.flatten()
    order = torch.argsort(chosen, stable=True)
    counts = torch.bincount(chosen, minlength=EXPERTS)
    offsets = torch.zeros(EXPERTS + 1, dtype=torch.int64, device=logits.device)
    offsets[1:] = counts.cumsum(0)
    return order // TOP, offsets


def codes(x, dim):
    top = x.float().abs().amax(dim, keepdim=True)
    up = 127 * (1 / top)
    return (x.float() * up).round().double() * (top / 127).double()


def test_monitored_experts(cuda_device):
    import torch
    torch.manual_seed(0)
    dev, t = cuda_device, torch.bfloat16
    up = (torch.randn(EXPERTS, FFN, HIDDEN, device=dev) * HIDDEN ** -0.5).to(t)
    down = (torch.randn(EXPERTS, HIDDEN, FFN, device=dev) * FFN ** -0.5).to(t)
    # the arena: for each expert its up and its down matrix
    size = 2 * FFN * HIDDEN
    arena = torch.zeros(EXPERTS * size, device=dev)
    g_up = torch.as_strided(arena, (EXPERTS, FFN, HIDDEN), (size, HIDDEN, 1), 0)
    g_down = torch.as_strided(arena, (EXPERTS, HIDDEN, FFN), (size, FFN, 1), FFN * HIDDEN)
    offsets = [e * size + i * FFN * HIDDEN for e in range(EXPERTS) for i in range(2)]
    mon = Monitor(offsets, [FFN * HIDDEN] * (2 * EXPERTS), dtype="f32", segment_unit=np.repeat(np.arange(EXPERTS), 2),
                  num_units=EXPERTS, window=2, max_o=3, lock_len=2, alpha=0.9, beta=1.5)
    stats = mon.new_stats()
    selected = 0
    with ExpertProducts(device=0) as products:
        mask = torch.zeros(EXPERTS, dtype=torch.uint8, device=dev)
        for step in range(STEPS):
            tokens = torch.randn(TOKENS, HIDDEN, device=dev).to(t)
            bias = torch.zeros(EXPERTS, device=dev)
            bias[step % EXPERTS] = -100.0                        # an expert without tokens
            rows, off = route(torch, torch.randn(TOKENS, EXPERTS, device=dev) + bias)
            x = tokens[rows].requires_grad_()
            h = expert_linear(products, x, up, off, mask, g_up)
            y = expert_linear(products, torch.relu(h), down, off, mask, g_down)
            (y.float().square().sum() / TOKENS).backward()
            low = (mask == 0).cpu()
            cut = off.tolist()
            # the path's own gradients, and the low path's outputs
            dy = (y.detach().float() * (2 / TOKENS)).to(t)
            hr = torch.relu(h.detach())
            want = torch.zeros(EXPERTS, dtype=torch.float64)
            for e in range(EXPERTS):
                at = slice(cut[e], cut[e + 1])
                X, H, D = x.detach()[at], hr[at], dy[at]
                if cut[e] == cut[e + 1]:
                    assert not g_up[e].any() and not g_down[e].any()
                    continue
                if low[e]:
                    exact = codes(X, 1) @ codes(up[e], 1).T
                    assert (h.detach()[at].double() - exact).abs().max() <= 2.0 ** -7 * exact.abs().max()
                    dh = codes(D, 1) @ codes(down[e], 0)
                else:
                    dh = D.double() @ down[e].double()
                dh = (dh.float().to(t) * (h.detach()[at] > 0)).double()
                want[e] = ((dh.T @ X.double()).square().sum() + (D.double().T @ H.double()).square().sum()).sqrt().item()
            mask = mon.step(arena, stats=stats)
            got = stats["norm"].cpu()
            # dh is rounded to bf16 once on both sides; a value that rounds the other way is 2^-8 off
            assert torch.allclose(got, want, rtol=2e-3, atol=1e-12)
            assert int(mask.sum()) <= 3
            selected += int(mask.sum())
            x.grad = None
    mon.close()
    assert selected > 0                                          # both paths ran
