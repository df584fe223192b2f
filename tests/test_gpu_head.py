"""Log probabilities under a linear head and their gradients on the GPU, against the definitions in
float64, and against differences.

Tolerances (u = 2^-24, inputs exact in both).  A logit is a sum of n products in fp32: its partial
sums are about as large as the largest logits, and roundings of either sign add up as their root:
6 u sqrt(n) max(1, max |z|) bounds it at six standard deviations (ZTOL).  logp and stats take it
twice (the target's and the sum's), and 4e-6 for the sum of exponentials and its logarithm, as the
log probabilities of given logits do.  p is off by e = 2 ZTOL + 1e-6 relative, dz by e |dlogp|, and
a product's sum by the sizes of its terms, A = |dz| |W| (or |dz|^T |X|), times u for each of its
roundings, of which 6 sqrt(k) count, plus e |dlogp| times the other operand's terms.  bf16 rounds dz
(2^-8 of A) and the result (2^-8 of it)."""
import math

import pytest

from paper_2609_01956_amd import binding as kb
from gpu_common import device, say, torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24

# rows, classes, n, padding of x's rows, of the weights', first column of x: few rows (groups of 16,
# 32, 64), tiles of 128 and 256, odd sizes, rows that have to be copied
SIZES = [(1, 1, 1, 0, 0, 0), (1, 1000, 256, 0, 0, 0), (2, 17, 7, 1, 0, 0), (15, 130, 64, 0, 8, 0),
         (16, 5000, 33, 0, 0, 1), (17, 300, 100, 3, 1, 0), (33, 257, 1001, 15, 0, 0),
         (64, 100, 264, 0, 0, 8), (13, 500, 2500, 0, 0, 0), (64, 70, 5003, 1, 1, 1),
         (65, 10, 8, 0, 0, 0), (128, 128, 64, 8, 8, 0), (129, 255, 72, 0, 0, 0),
         (300, 1000, 100, 0, 0, 0), (131, 129, 131, 5, 3, 2), (1000, 2, 40, 0, 0, 0),
         (70, 4099, 16, 0, 0, 0), (2100, 9000, 48, 0, 0, 0), (2049, 8200, 37, 1, 0, 0),
         # (few rows: k over a workgroup's waves, and x in slices of k)
         (1, 10, 4096, 0, 0, 0), (20, 100, 1500, 1, 0, 0), (64, 33, 1023, 0, 0, 0),
         (3, 9001, 5000, 0, 0, 0), (50, 8300, 1300, 0, 1, 0), (31, 8200, 2052, 4, 0, 0),
         # (fp32 as bf16 terms: a few rows of many classes, the reverse, one piece and splits of k)
         (600, 4001, 70, 0, 0, 0), (5000, 1100, 130, 1, 3, 1), (1030, 1030, 1000, 0, 0, 4),
         (300, 6000, 9, 0, 0, 0)]


def make(rows, classes, n, xpad, wpad, first, dt, seed, std=2.0):
    g = torch.Generator(device=device())
    g.manual_seed(seed)
    x = torch.randn(rows, first + n + xpad, device=device(), generator=g).to(dt)
    w = (torch.randn(classes, n + wpad, device=device(), generator=g) * std).to(dt)
    x[:, :first] = float("nan")  # (what lies between the rows is not read)
    x[:, first + n:] = float("nan")
    w[:, n:] = float("nan")
    t = torch.randint(0, classes, (rows,), device=device(), generator=g)
    d = -torch.rand(rows, device=device(), generator=g)
    return x[:, first:first + n], w[:, :n], t, d


def forward64(x, w, t, scale):
    z = (x.double() * scale) @ w.double().t()
    lse = torch.logsumexp(z, 1)
    m, best = z.max(1)
    return z, z.gather(1, t[:, None])[:, 0] - lse, m, lse - m, best


def ztol(z, n):
    return 6 * U * math.sqrt(n) * max(1.0, float(z.abs().max()))


def below(err, bound):
    assert bool((err <= bound).all()), float((err - bound).max())


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("size", SIZES)
def test_forward(dt, size):
    rows, classes, n = size[:3]
    x, w, t, _ = make(*size, dt, 7)
    scale = n ** -0.5
    say(f"linear_logprobs {dt} {size}")
    logp, stats, best = kb.linear_logprobs(x, w, t, scale=scale, best=True)
    z, lp, m, logs, at = forward64(x, w, t, scale)
    tol = ztol(z, n)
    below((logp.double() - lp).abs(), 2 * tol + 4e-6 + 4 * U * lp.abs())
    below((stats[:, 0].double() - m).abs(), tol + U * m.abs())
    below((stats[:, 1].double() - logs).abs(), 2 * tol + 4e-6 + 4 * U * logs.abs())
    # the class itself where no other comes within the logits' error, one as good elsewhere
    got = z.gather(1, best[:, None])[:, 0]
    below(m - got, 2 * tol)
    clear = (z >= (m - 2 * tol)[:, None]).sum(1) == 1
    assert torch.equal(best[clear], at[clear])
    again = kb.linear_logprobs(x, w, t, scale=scale)
    assert again[2] is None and torch.equal(again[0], logp) and torch.equal(again[1], stats)


def gradient64(x, w, t, stats, d, scale):
    z = (x.double() * scale) @ w.double().t()
    p = torch.exp(z - stats.double().sum(1, keepdim=True))
    dz = -p * d.double()[:, None]
    dz.scatter_add_(1, t[:, None], d.double()[:, None])
    return z, dz


def check_gradients(x, w, dx, dw, z, dz, d, scale, dt):
    n, (rows, classes) = x.shape[1], dz.shape
    e = (2 * ztol(z, n) + 1e-6) * d.double().abs()[:, None]  # of dz
    half = 2.0 ** -8 if dt == BF16 else 0.0
    out = 2.0 ** -8 if dt == BF16 else U
    xd, wd, s = x.double(), w.double(), abs(scale)
    for got, want, terms, other, k in (
            (dx, dz @ wd * scale, dz.abs() @ wd.abs() * s, e * wd.abs().sum(0) * s, classes),
            (dw, dz.t() @ xd * scale, dz.abs().t() @ xd.abs() * s, (e * xd.abs()).sum(0) * s, rows)):
        if got is not None:
            assert got.dtype == dt and got.shape == want.shape
            below((got.double() - want).abs(),
                  terms * (half + 6 * U * math.sqrt(k) + 4 * U) + other * (1 + half) +
                  out * want.abs())


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("size", SIZES)
def test_gradients(dt, size):
    rows, classes, n = size[:3]
    x, w, t, d = make(*size, dt, 8)
    scale = 0.7 * n ** -0.5
    say(f"linear_logprobs_backward {dt} {size}")
    _, stats, _ = kb.linear_logprobs(x, w, t, scale=scale)
    dx, dw = kb.linear_logprobs_backward(x, w, t, stats, d, scale=scale)
    z, dz = gradient64(x, w, t, stats, d, scale)
    check_gradients(x, w, dx, dw, z, dz, d, scale, dt)
    # each alone, and into tensors at hand
    one, none = kb.linear_logprobs_backward(x, w, t, stats, d, scale=scale, need_dw=False)
    assert none is None and torch.equal(one, dx)
    out = (torch.empty_like(dx), torch.empty_like(dw))
    none, two = kb.linear_logprobs_backward(x, w, t, stats, d, scale=scale, need_dx=False, out=out)
    assert none is None and two is out[1] and torch.equal(two, dw)


@pytest.mark.parametrize("dt", [F32, BF16])
def test_vocabulary_in_pieces(dt):
    """Enough rows and classes that the gradient goes through several pieces, the last one short."""
    rows, classes, n = 3000, 50001, 24
    x, w, t, d = make(rows, classes, n, 0, 0, 0, dt, 9)
    say(f"linear_logprobs_backward pieces {dt}")
    _, stats, _ = kb.linear_logprobs(x, w, t, scale=0.2)
    dx, dw = kb.linear_logprobs_backward(x, w, t, stats, d, scale=0.2)
    z, dz = gradient64(x, w, t, stats, d, 0.2)
    check_gradients(x, w, dx, dw, z, dz, d, 0.2, dt)


@pytest.mark.parametrize("rows", [5, 90, 300])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_ignored_and_invalid_targets(rows, dt):
    """An ignored row counts for nothing, whatever it holds; a target that is no class shows."""
    x, w, t, d = make(rows, 77, 40, 0, 0, 0, dt, 10)
    say(f"linear head targets {rows} {dt}")
    skip = torch.arange(rows, device=device()) % 3 == 1
    t2 = torch.where(skip, -100, t)
    logp, stats, _ = kb.linear_logprobs(x, w, t2)
    full = kb.linear_logprobs(x, w, t)
    assert torch.equal(logp, torch.where(skip, 0.0, full[0])) and torch.equal(stats, full[1])
    x2 = torch.where(skip[:, None], float("nan"), x)
    d2 = torch.where(skip, float("nan"), d)
    for xx, dd in ((x, d), (x2, d2)):
        lp, st, _ = kb.linear_logprobs(xx, w, t2)
        assert torch.equal(lp, logp) and torch.equal(st[~skip], stats[~skip])
        dx, dw = kb.linear_logprobs_backward(xx, w, t2, st, dd)
        assert float(dx[skip].abs().max()) == 0.0
        z, dz = gradient64(x[~skip], w, t[~skip], stats[~skip], d[~skip], 1.0)
        check_gradients(x[~skip], w, dx[~skip], dw, z, dz, d[~skip], 1.0, dt)
    t3 = t.clone()
    t3[1], t3[2] = 77, -1
    lp, st, _ = kb.linear_logprobs(x, w, t3)
    assert bool(lp[1:3].isnan().all()) and torch.equal(st, full[1])
    assert torch.equal(lp[3:], full[0][3:]) and lp[0] == full[0][0]
    dx, dw = kb.linear_logprobs_backward(x, w, t3, st, d)
    assert bool(dx[1:3].isnan().all()) and bool(dw.isnan().all())
    assert not bool(dx[3:].isnan().any()) and not bool(dx[0].isnan().any())


@pytest.mark.parametrize("rows,classes", [(5, 300), (90, 300), (700, 3000), (300, 3000)])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_not_finite(rows, classes, dt):
    x, w, t, d = make(rows, classes, 16, 0, 0, 0, dt, 11)
    clean = kb.linear_logprobs(x, w, t, best=True)
    x[2, 3] = float("nan")
    x[3, 5] = float("inf")   # (weights of either sign: +infinity among the logits)
    say(f"linear head not finite {rows} {classes} {dt}")
    logp, stats, best = kb.linear_logprobs(x, w, t, best=True)
    assert bool(logp[2:4].isnan().all()) and bool(stats[2:4, 1].isnan().all())
    keep = torch.ones(rows, dtype=torch.bool, device=device())
    keep[2:4] = False
    for a, b in zip((logp, stats, best), clean):
        assert torch.equal(a[keep], b[keep])
    assert int(best[2]) == 0  # (no number to prefer)
    dx, dw = kb.linear_logprobs_backward(x, w, t, stats, d)
    assert bool(dx[2:4].isnan().all()) and not bool(dx[keep].isnan().any())
    assert bool(dw.isnan().all())
    # a class of -infinity logits takes no part
    x, w, t, d = make(rows, classes, 16, 0, 0, 0, dt, 12)
    x[:, 0] = x[:, 0].abs() + 0.5
    w[9] = 0
    w[9, 0] = float("-inf")
    w[9, 1:] = 1.0
    t[t == 9] = 10
    logp, stats, best = kb.linear_logprobs(x, w, t, best=True)
    z = (x.double() @ w.double().t())
    assert bool((z[:, 9] == float("-inf")).all())
    lp = torch.log_softmax(z, 1).gather(1, t[:, None])[:, 0]
    below((logp.double() - lp).abs(), 2 * ztol(z[:, :9], 16) * 2 + 4e-6 + 4 * U * lp.abs())
    t[0] = 9
    assert float(kb.linear_logprobs(x, w, t)[0][0]) == float("-inf")
    # no class left
    w[:] = w[9]
    logp, stats, best = kb.linear_logprobs(x, w, t, best=True)
    assert bool((logp == float("-inf")).all()) and bool((best == 0).all())


@pytest.mark.parametrize("rows", [3, 100])
def test_ties_go_to_the_lowest(rows):
    w = torch.ones(1000, 32, device=device(), dtype=BF16)
    w[:17] = 0.5
    x = torch.ones(rows, 32, device=device(), dtype=BF16)
    t = torch.full((rows,), 999, device=device())
    say(f"linear head ties {rows}")
    _, stats, best = kb.linear_logprobs(x, w, t, best=True)
    assert bool((best == 17).all()) and bool((stats[:, 0] == 32).all())


@pytest.mark.parametrize("scale", [1e-30, 1e30, 3e36])
def test_values_far_from_one(scale):
    """fp32 inputs of any size whose sums before the scale stay in range: the logits' relative error
    stays that of their sums."""
    x, w, t, d = make(600, 2000, 40, 0, 0, 0, F32, 14, std=1.0)
    say(f"linear head at {scale}")
    x, s = x.clamp(-4, 4) * scale, 0.2 / scale
    logp, stats, _ = kb.linear_logprobs(x, w, t, scale=s)
    z, lp, m, logs, _ = forward64(x, w, t, s)
    tol = ztol(z, 40) + 4 * U * float(z.abs().max())
    below((logp.double() - lp).abs(), 2 * tol + 4e-6 + 4 * U * lp.abs())
    dx, dw = kb.linear_logprobs_backward(x, w, t, stats, d, scale=s)
    z, dz = gradient64(x, w, t, stats, d, s)
    e = (2 * tol + 1e-6) * d.double().abs()[:, None]
    want, terms = dz.t() @ x.double() * s, dz.abs().t() @ x.double().abs() * s
    below((dw.double() - want).abs(),
          terms * (6 * U * math.sqrt(600) + 4 * U) + (e * x.double().abs()).sum(0) * s +
          U * want.abs())


def test_gradient_against_differences():
    """Central differences of the loss in fp32: with step h = 2^-6 the third derivative leaves
    h^2 / 6 of its size, a few 1e-5, and the loss's own error 4e-6 (rows) over 2 h, 3e-3 of one row's
    gradient; 1e-2 of the largest is asked."""
    rows, classes, n = 6, 40, 12
    x, w, t, d = make(rows, classes, n, 0, 0, 0, F32, 13, std=0.5)
    say("linear head differences")

    def loss(xx, ww):
        return float((kb.linear_logprobs(xx, ww, t, scale=0.6)[0].double() * d.double()).sum())
    _, stats, _ = kb.linear_logprobs(x, w, t, scale=0.6)
    dx, dw = kb.linear_logprobs_backward(x, w, t, stats, d, scale=0.6)
    h = 2.0 ** -6
    for a, grad, which in ((x, dx, 0), (w, dw, 1)):
        for i, j in ((0, 0), (3, 7), (5, 11)):
            up, down = a.clone(), a.clone()
            up[i, j] += h
            down[i, j] -= h
            args = ((up, w), (down, w)) if which == 0 else ((x, up), (x, down))
            diff = (loss(*args[0]) - loss(*args[1])) / (2 * h)
            assert abs(diff - float(grad[i, j])) <= 1e-2 * float(grad.abs().max())


def test_empty_batch():
    x = torch.empty(0, 40, device=device())
    w = torch.randn(30, 40, device=device())
    t = torch.empty(0, dtype=torch.int64, device=device())
    say("linear head empty")
    logp, stats, best = kb.linear_logprobs(x, w, t, best=True)
    assert logp.shape == best.shape == (0,) and stats.shape == (0, 2)
    dx, dw = kb.linear_logprobs_backward(x, w, t, stats, logp)
    assert dx.shape == (0, 40) and float(dw.abs().max()) == 0.0
