"""Clipping of gradients at the edges: bounds and norms that are infinite, lists that fill launches
exactly, and long lists in any order."""
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


@pytest.mark.parametrize("count", [175, 176, 177, 271, 272, 273, 352, 353, 544, 545])
def test_lists_that_fill_launches(count):
    """A launch takes 272 tensors, 176 with outputs elsewhere: counts on both sides of one and two
    of them, of mixed types and sizes (parts of a unit, whole chunks and their edges), with empty
    tensors at the edges, against float64.  The norm carries one rounding to fp32 (2^-23), the
    product two (2^-22; bf16 2^-8)."""
    g = torch.Generator(device=device())
    g.manual_seed(count)
    sizes = [(1, 16384, 7, 300, 16385, 8)[i % 6] + i % 5 for i in range(count)]
    grads = [torch.randn(n, device=device(), generator=g).to(BF16 if i % 3 == 1 else F32)
             for i, n in enumerate(sizes)]
    empty = torch.empty(0, device=device())
    for at in (544, 272, 176, 1, 0):
        if at <= len(grads):
            grads.insert(at, empty)
    n64 = math.sqrt(sum(float((v.double() ** 2).sum()) for v in grads))
    say(f"clip_grad_norm launches filled by {count} tensors")
    out = [torch.full_like(v, 9.0) for v in grads]
    for got in (kb.grad_norm(grads), kb.clip_grad_norm(grads, n64 / 2, eps=0.0, out=out)):
        assert abs(float(got) - n64) <= 2.0 ** -23 * n64
    for a, v in zip(out, grads):
        want = v.double() / 2
        tol = 2.0 ** -22 if v.dtype == F32 else 2.0 ** -8
        assert bool(((a.double() - want).abs() <= tol * want.abs()).all())
    kb.clip_grad_norm(grads, n64 / 2, eps=0.0)
    assert all(torch.equal(a, b) for a, b in zip(grads, out))


@pytest.mark.parametrize("count", [3000, 16384])
def test_thousands_of_neighbours_in_any_order(count):
    """Views that lie side by side in one buffer, in no order: none overlaps another, and every
    one is scaled once."""
    g = torch.Generator()
    g.manual_seed(count)
    cuts = torch.cat([torch.zeros(1, dtype=torch.int64),
                      torch.randint(1, 40, (count,), generator=g).cumsum(0)]).tolist()
    order = torch.randperm(count, generator=g).tolist()
    flat = torch.ones(cuts[-1], device=device())
    other = torch.zeros_like(flat)
    views = lambda t: [t[cuts[i]:cuts[i + 1]] for i in order]
    total = math.sqrt(cuts[-1])
    say(f"clip_grad_norm {count} neighbours")
    n = kb.clip_grad_norm(views(flat), total / 4, eps=0.0, out=views(other))
    assert abs(float(n) - total) <= 2.0 ** -23 * total
    assert bool(((other - 0.25).abs() <= 2.0 ** -22 * 0.25).all())
    kb.clip_grad_norm(views(flat), total / 4, eps=0.0)
    assert torch.equal(flat, other)
    late = views(other)
    late[-1] = other[cuts[order[0]] + (1 if late[0].numel() > 1 else 0):][:late[-1].numel()]
    with pytest.raises(ValueError):
        kb.clip_grad_norm(views(flat), 1.0, out=late)
