"""Layer norm at the edges of its range, against the definition in float64."""
import pytest

from paper_2609_01956_amd import binding as kb
from gpu_common import device, say, torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("n", [10, 300, 900, 2050, 9000, 16500])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_subnormal_variance(n, dt):
    """Without eps, rows whose variance is below 2^-126 keep their statistics.  Spread 2^-64:
    the squares are multiples of 2^-149 near 2^-128, each off by 2^-150 at most, their sum in
    that range exact and the mean off by 2^-150 again, so the variance is good to 2^-21 and
    rstd to 2^-22; 1e-5 as elsewhere (bf16: a rounding of the result on top)."""
    g = torch.Generator(device=device())
    g.manual_seed(n)
    x = (torch.randn(5, n, device=device(), generator=g) * 2.0 ** -64).to(dt)
    say(f"layer_norm subnormal variance n={n} {dt}")
    y, _, mean, rstd = kb.layer_norm(x, eps=0.0)
    h = x.double()
    var, m64 = torch.var_mean(h, 1, correction=0)
    r64 = 1 / var.sqrt()
    assert bool(((rstd.double() - r64).abs() <= 1e-5 * r64).all())
    want = (h - m64[:, None]) * r64[:, None]
    tol = 1e-5 if dt == F32 else 2.0 ** -8
    assert bool(((y.double() - want).abs() <= tol * want.abs().amax(1, keepdim=True)).all())


@pytest.mark.parametrize("n", [10, 300, 900, 2050, 9000, 16500])
def test_edges_of_the_range_as_documented(n):
    """Without eps a row whose squared differences all vanish has no finite y, and a row whose
    sum leaves binary32 is NaN; the others do not notice."""
    g = torch.Generator(device=device())
    g.manual_seed(n)
    x = torch.randn(4, n, device=device(), generator=g)
    say(f"layer_norm edges of the range n={n}")
    ref = kb.layer_norm(x, eps=0.0)[0]
    x[1] *= 2.0 ** -90
    x[2] = 3e38
    y = kb.layer_norm(x, eps=0.0)[0]
    assert torch.equal(y[0], ref[0]) and torch.equal(y[3], ref[3])
    assert not bool(torch.isfinite(y[1]).any()) and bool(torch.isnan(y[2]).all())


@pytest.mark.parametrize("rows,n", [(60, 7), (60, 100), (60, 300), (60, 784), (60, 1001),
                                    (60, 2500), (60, 9001), (60, 17000)])
def test_each_row_by_its_own_size(rows, n):
    """Rows whose spread runs from 2^-20 to 2^20, each held to its own largest value, forward and
    backward, in fp32.  Without a bias y is xh w: a few roundings, the mean's and rstd's errors
    (sums of 41 steps at most: 41 u) of the row's largest |xh w|, 1e-5 of it in all; the input's
    own centre is 0, so its rounding adds nothing.  dx has three such terms, rstd |g| (2 + |xh|)
    at most."""
    g = torch.Generator(device=device())
    g.manual_seed(n)
    r = lambda *s: torch.randn(*s, device=device(), generator=g)
    spread = 2.0 ** torch.linspace(-20, 20, rows, device=device())[:, None]
    x, dy = r(rows, n) * spread, r(rows, n) * spread.flip(0)
    w = 1 + 0.3 * r(n)
    say(f"layer_norm rows by their own size n={n}")
    y, _, mean, rstd = kb.layer_norm(x, w, None)
    dx, _, _ = kb.layer_norm_backward(x, mean, rstd, w, dy)
    h, w64 = x.double(), w.double()
    var, m64 = torch.var_mean(h, 1, correction=0, keepdim=True)
    r64 = 1 / torch.sqrt(var + 1e-5)
    xh = (h - m64) * r64
    want = xh * w64
    assert bool(((y.double() - want).abs() <= 1e-5 * want.abs().amax(1, keepdim=True)).all())
    gr = dy.double() * w64
    terms = r64 * gr.abs().amax(1, keepdim=True) * (2 + xh.abs().amax(1, keepdim=True))
    want = r64 * (gr - gr.mean(1, keepdim=True) - xh * (gr * xh).mean(1, keepdim=True))
    assert bool(((dx.double() - want).abs() <= 1e-5 * terms).all())
