"""Token operators where values are far from each other, on the GPU against the formulas in float64:
targets nearly certain, logits far from 0 and out of range.

In the first two, rows of the identity make the logits the weights, and dz the weights' gradient;
the logits are exact in either type, and so are the stats' m.  u = 2^-24; bf16 rounds a gradient once
(2^-8 of it)."""
import math

import pytest

from paper_2609_01956_amd import binding as kb
from gpu_common import device, say, torch
from test_gpu_head import below, U

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 0.0, BF16: 2.0 ** -8}


def head_of(rows, V, n, dt, m, other, base=0.0):
    """x, weight, targets, stats and dlogp of logits `base` + m for the targets and + other elsewhere,
    the logits' distance from m, and logs."""
    g = torch.Generator(device=device())
    g.manual_seed(rows + V)
    at = torch.arange(rows, device=device())
    x = torch.zeros(rows, n, dtype=dt, device=device())
    x[at, at] = 1.0
    x[:, rows] = 1.0
    t = torch.randperm(V, device=device(), generator=g)[:rows]
    w = torch.zeros(V, n, dtype=dt, device=device())
    w[:, :rows] = other
    w[t, at] = m
    w[:, rows] = base
    logs = float(torch.tensor(math.log1p((V - 1) * math.exp(other - m)), dtype=F32))
    stats = torch.tensor([[base + m, logs]], device=device()).expand(rows, 2).contiguous()
    d = -torch.rand(rows, device=device(), generator=g) - 0.1
    return x, w, t, stats, d, other - m, logs


# few rows, tiles of both sizes, sums over parts of n
SIZES = [(6, 10, 7), (16, 20, 17), (40, 300, 41), (16, 1000, 4096), (600, 4000, 601),
         (2000, 20000, 2001)]


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("m,other", [(14.0, 0.0), (30.0, 10.0), (30.0, 9.0)])
@pytest.mark.parametrize("rows,V,n", SIZES)
def test_targets_nearly_certain(rows, V, n, m, other, dt):
    """1 - p of a target with p nearly 1, for given stats, to its own size (2^-22 of the series, two
    roundings of dz and as many of its terms and sum; in bf16 the gradient's), not to that of p."""
    x, w, t, stats, d, _, logs = head_of(rows, V, n, dt, m, other)
    say(f"linear head targets nearly certain {rows} {V} {n} {m} {other} {dt}")
    _, dw = kb.linear_logprobs_backward(x, w, t, stats, d, need_dx=False)
    want = -math.expm1(-logs) * d.double()
    got = dw[t, torch.arange(rows, device=device())].double()
    below((got - want).abs(), want.abs() * (HALF[dt] + 2.0 ** -22 + 6 * U))


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("base", [0.0, 2.0 ** 20, -(2.0 ** 20)])
@pytest.mark.parametrize("rows,V,n", SIZES)
def test_logits_far_from_zero(rows, V, n, base, dt):
    """p of logits near a large m: it depends on their distances t alone.  t is exact; t - logs, its
    product with log2 e and the exponential are off by 3 u (|t| + logs) + 4 u; 2^-22 for the fp32 form's,
    and 6 roundings of dz, its terms and their sums."""
    x, w, t, stats, d, far, logs = head_of(rows, V, n, dt, 14.0, 12.0, base)
    say(f"linear head far from zero {rows} {V} {n} {base} {dt}")
    _, dw = kb.linear_logprobs_backward(x, w, t, stats, d, need_dx=False)
    at = torch.arange(rows, device=device())
    want = (-math.exp(far - logs) * d.double()).expand(V, rows).clone()
    want[t, at] = -math.expm1(-logs) * d.double()
    below((dw[:, :rows].double() - want).abs(),
          want.abs() * (HALF[dt] + 2.0 ** -22 + (3 * (abs(far) + logs) + 10) * U))


# tiles of both sizes throughout (whole ones), sums over parts of n, few rows
WHOLE = [(2048, 16384, 16), (100, 1024, 16), (600, 4096, 16), (64, 256, 4096), (128, 512, 2048),
         (5, 1024, 16), (40, 1024, 16)]


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("rows,V,n", WHOLE)
def test_logits_that_the_scale_takes_out_of_range(rows, V, n, dt):
    """Finite sums whose scaled logits overflow: +infinity among them makes a row's logp and logs NaN,
    and its dx and all of dweight; -infinity takes no part."""
    g = torch.Generator(device=device())
    g.manual_seed(31)
    x = torch.zeros(rows, n, dtype=dt, device=device())
    x[:, 1] = 1.0
    x[2, 0], x[3, 0] = 2.0 ** 63, -(2.0 ** 63)
    w = torch.zeros(V, n, dtype=dt, device=device())
    w[:, 1] = torch.randint(-8, 9, (V,), device=device(), generator=g) / 8
    w[V - 1, 0] = 2.0 ** 63
    t = torch.randint(0, V - 1, (rows,), device=device(), generator=g)
    say(f"linear head out of range {rows} {V} {n} {dt}")
    logp, stats, _ = kb.linear_logprobs(x, w, t, scale=8.0)
    assert bool(logp[2].isnan()) and bool(stats[2, 1].isnan())
    keep = torch.arange(rows, device=device()) != 2
    z = x.double() @ w.double().t() * 8.0
    z[3, V - 1] = -math.inf
    lp = torch.log_softmax(z, 1).gather(1, t[:, None])[:, 0]
    # (the logits are exact: the sum of exponentials and its logarithm)
    below((logp.double() - lp)[keep].abs(), 4e-6 + 4 * U * lp[keep].abs())
    dx, dw = kb.linear_logprobs_backward(x, w, t, stats, -torch.ones_like(logp), scale=8.0)
    assert bool(dx[2].isnan().all()) and bool(dw.isnan().all()) and not bool(dx[keep].isnan().any())


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("logs", [-math.inf, 0.0, 1.0, math.nan])
@pytest.mark.parametrize("rows,V,n", WHOLE)
def test_stats_of_infinite_logits(rows, V, n, logs, dt):
    """m = +infinity in the stats, whatever logs is beside it: the row's dx and all of dweight are NaN,
    the other rows' dx as without it."""
    g = torch.Generator(device=device())
    g.manual_seed(32)
    x = torch.randn(rows, n, device=device(), generator=g).to(dt)
    w = torch.randn(V, n, device=device(), generator=g).to(dt)
    t = torch.randint(0, V, (rows,), device=device(), generator=g)
    say(f"linear head stats of infinite logits {rows} {V} {n} {logs} {dt}")
    logp, stats, _ = kb.linear_logprobs(x, w, t, scale=0.1)
    d = -torch.ones_like(logp)
    want, _ = kb.linear_logprobs_backward(x, w, t, stats, d, scale=0.1)
    stats[2, 0], stats[2, 1] = math.inf, logs
    dx, dw = kb.linear_logprobs_backward(x, w, t, stats, d, scale=0.1)
    keep = torch.arange(rows, device=device()) != 2
    assert bool(dx[2].isnan().all()) and bool(dw.isnan().all()) and torch.equal(dx[keep], want[keep])
