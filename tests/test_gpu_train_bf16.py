"""The classifier's gradients in bf16 against float64 autograd."""
import pytest

from gpu_common import device, say, torch
from test_gpu_train import model64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sizes", [(12, 16, 16, 16, 5), (33, 7, 7, 3)])
def test_gradients_against_autograd(sizes):
    """Per layer the norm's output, the layer's, their gradients and the stored weights' products
    are rounded to bf16, forward and backward: six roundings of 2^-9 in each of at most four
    layers, each passed on with a factor of about 2 (the splines' slopes at unit spacing), 24 x 2 x
    2^-9 = 0.094 of a parameter's gradient if all lay one way; 0.1 of its 2-norm."""
    from paper_2609_01956_amd.train import KanClassifier
    g = torch.Generator(device=device())
    g.manual_seed(3)
    model = KanClassifier(sizes, grid_size=6, dtype=torch.bfloat16, device=device())
    for layer in model.params:
        layer[0].add_(torch.randn(layer[0].shape, device=device(), generator=g), alpha=0.2)
        layer[1].add_(torch.randn(layer[1].shape, device=device(), generator=g), alpha=0.2)
    x = torch.randn(520, sizes[0], device=device(), generator=g).to(torch.bfloat16)
    t = torch.randint(0, sizes[-1], (520,), device=device(), generator=g)
    say(f"train gradients bf16 {sizes}")
    logp, grads = model.gradients(x, t, entropy_bonus=0.3)
    params = [[p.double().requires_grad_() for p in layer] for layer in model.params]
    want, loss = model64(params, x.double(), t, model.grid, 0.3)
    loss.backward()
    assert abs(float(logp) - float(want.detach())) < 0.1 * abs(float(want.detach()))
    flat = [p for layer in params for p in layer]
    assert len(grads) == len(flat)
    for a, p, like in zip(grads, flat, [p for layer in model.params for p in layer]):
        assert a.dtype == like.dtype and a.shape == like.shape
        assert float((a.double() - p.grad).norm()) <= 0.1 * float(p.grad.norm())
