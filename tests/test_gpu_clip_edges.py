"""Clipping of gradients at the edges: bounds and norms that are infinite."""
import math

import pytest

from paper_2609_01956_amd import binding as kb
from gpu_common import device, say, torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dt", [F32, BF16])
def test_no_bound_keeps_infinite_gradients(dt):
    """max_norm infinite is no bound, also where a gradient, and with it the norm, is infinite;
    a NaN still reaches all."""
    g = [torch.linspace(-1, 1, 100, device=device()).to(dt), torch.ones(7, device=device(), dtype=dt)]
    g[1][3] = math.inf
    keep, out = [v.clone() for v in g], [torch.zeros_like(v) for v in g]
    say(f"clip_grad_norm without bound {dt}")
    assert math.isinf(float(kb.clip_grad_norm(g, math.inf, out=out)))
    assert all(torch.equal(a, b) for a, b in zip(out, keep))
    assert math.isinf(float(kb.clip_grad_norm(g, math.inf)))
    assert all(torch.equal(a, b) for a, b in zip(g, keep))
    g[1][3] = math.nan
    assert math.isnan(float(kb.clip_grad_norm(g, math.inf, out=out)))
    assert all(bool(torch.isnan(v).all()) for v in out)
