"""The classifier of paper_2609_01956_amd.train: the operators together, against the same model
in float64 torch with autograd, and over a few steps."""
import math

import pytest

from gpu_common import device, say, torch

pytestmark = pytest.mark.gpu


def kan64(x, coef, base_w, G, lo, hi):
    """The layer from its definition: clamped truncated powers of the normalised coordinate."""
    j = torch.arange(G + 3, dtype=torch.float64, device=x.device)
    u = ((x.unsqueeze(-1) - lo) * (G / (hi - lo)) + 3 - j).clamp(0, 4)
    n = sum((-1) ** m * math.comb(4, m) * (u - m).clamp(min=0) ** 3 for m in range(5)) / 6
    return torch.einsum("bij,oij->bo", n, coef) + torch.nn.functional.silu(x) @ base_w.t()


def model64(params, x, targets, grid, bonus):
    stream, out = None, x
    for w, b, coef, base_w in params:
        h = out + stream if stream is not None and stream.shape == out.shape else out
        c = h - h.mean(1, keepdim=True)
        z = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * w + b
        stream, out = h, kan64(z, coef, base_w, *grid)
    lp = torch.log_softmax(out, 1)
    logp = lp.gather(1, targets[:, None])[:, 0].mean()
    return logp, -logp + bonus * (lp.exp() * lp).sum(1).mean()


@pytest.mark.parametrize("sizes", [(12, 16, 16, 16, 5), (33, 7, 7, 3)])
def test_gradients_against_autograd(sizes):
    """fp32 against float64: the sums of a few hundred terms in fp32 at each of four layers,
    1e-4 of a parameter's largest gradient."""
    from paper_2609_01956_amd.train import KanClassifier
    g = torch.Generator(device=device())
    g.manual_seed(1)
    model = KanClassifier(sizes, grid_size=6, dtype=torch.float32, device=device())
    for layer in model.params:
        layer[0].add_(torch.randn(layer[0].shape, device=device(), generator=g), alpha=0.2)
        layer[1].add_(torch.randn(layer[1].shape, device=device(), generator=g), alpha=0.2)
    x = torch.randn(130, sizes[0], device=device(), generator=g)
    t = torch.randint(0, sizes[-1], (130,), device=device(), generator=g)
    say(f"train gradients {sizes}")
    logp, grads = model.gradients(x, t, entropy_bonus=0.3)
    params = [[p.double().requires_grad_() for p in layer] for layer in model.params]
    want, loss = model64(params, x.double(), t, model.grid, 0.3)
    loss.backward()
    assert abs(float(logp) - float(want.detach())) < 1e-5
    flat = [p for layer in params for p in layer]
    assert len(grads) == len(flat)
    for a, p in zip(grads, flat):
        assert float((a.double() - p.grad).abs().max()) <= 1e-4 * float(p.grad.abs().max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_training_learns(dtype):
    from paper_2609_01956_amd.train import KanClassifier
    g = torch.Generator(device=device())
    g.manual_seed(2)
    teacher = torch.randn(20, 5, device=device(), generator=g)
    x = torch.randn(2048, 20, device=device(), generator=g)
    t = (x @ teacher).argmax(1)
    model = KanClassifier((20, 32, 32, 5), grid_size=5, dtype=dtype, device=device())
    say(f"train steps {dtype}")
    first = None
    for _ in range(60):
        logp, norm = model.step(x.to(dtype), t)
        first = float(logp) if first is None else first
        assert math.isfinite(float(norm))
    assert float(logp) > first / 2  # (the loss halved)
    lp, top, idx = model.alternatives(x[:7].to(dtype), t[:7], top_k=2)
    assert lp.shape == (7,) and top.shape == idx.shape == (7, 2)
    assert bool((top[:, 0] >= lp).all())
