"""Layer norm and its gradient on the GPU against the definitions in float64, and against
differences of the float64 forward.

Tolerances.  fp32: u = 2^-24.  y is (h - mean) rstd w + b: the mean's error is a rounding of
the mean, corrected (a few u |mean|, plus u |h| of the input's own rounding in h - mean), and
rstd, the products and the sum add a few u of |xh w| each; a sum over n terms in a tree of at
most 32 sequential steps and 9 joins adds at most 41 u of the mean absolute value.  With |h| at
most 64 times the row's spread below, 64 u 64 < 2.5e-4 of the spread bounds an offset row; rows
near their centre stay under 1e-5.  dx, dw, db are sums of the same kind; dw and db run over the
rows (at most 2048 sequential additions in a lane at these sizes): 1e-5 of the largest absolute
sum.  bf16: one rounding (2^-9 of the value) on top, and h's own rounding where the residual
sum is formed: 2^-8 of the largest value."""
import numpy as np
import pytest

from paper_2609_01956_amd import binding as kb
from gpu_common import device, say, torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
COMBOS = [(F32, F32), (BF16, BF16), (BF16, F32)]
TOL = {F32: 1e-5, BF16: 2.0 ** -8}

# rows, n: one lane, part of a unit, whole and ragged units, every count of lanes and units,
# four and eight waves a row, more rows than workgroups, and rows that do not fit in registers
SIZES = [(1, 1), (5, 2), (3, 3), (70, 7), (9, 8), (130, 9), (33, 31), (4, 64), (3, 65), (17, 100),
         (3, 127), (2, 256), (40, 257), (3, 511), (2, 512), (5, 513), (3, 784), (2, 1024), (7, 1025),
         (3, 1537), (2, 2048), (5, 2049), (3, 4095), (2, 4097), (3, 6145), (2, 8192), (3, 8193),
         (2, 12289), (3, 16384), (2, 16385), (3, 20011), (9000, 24), (3001, 333), (2100, 1200),
         (1400, 2500), (600, 9001)]


def make(rows, n, dt, pt, seed, centre=1.0):
    g = torch.Generator(device=device())
    g.manual_seed(seed)
    r = lambda *s: torch.randn(*s, device=device(), generator=g)
    x = (r(rows, n) * (r(rows, 1).abs() + 0.25) + centre * r(rows, 1)).to(dt)
    return dict(x=x, res=r(rows, n).to(dt), w=(1 + 0.3 * r(n)).to(pt), b=(0.3 * r(n)).to(pt),
                dy=r(rows, n).to(dt), dh=r(rows, n).to(dt))


def forward64(h, w, b, eps):
    mean = h.mean(-1, keepdim=True)
    var = ((h - mean) ** 2).mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    return (h - mean) * rstd * w + b, mean[..., 0], rstd[..., 0]


def backward64(h, mean, rstd, w, dy, dh):
    xh = (h - mean[:, None]) * rstd[:, None]
    g = dy * w
    dx = rstd[:, None] * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    return dx + dh, (dy * xh).sum(0), dy.sum(0), (dy * xh).abs().sum(0), dy.abs().sum(0)


def close(got, want, tol, scale=None):
    scale = want.abs().max() if scale is None else scale
    assert got.shape == want.shape
    err = (got.double() - want).abs()
    assert bool((err <= tol * scale + 1e-30).all()), float((err / (scale + 1e-30)).max())


@pytest.mark.parametrize("dt,pt", COMBOS)
@pytest.mark.parametrize("residual", [False, True])
def test_forward(dt, pt, residual):
    for i, (rows, n) in enumerate(SIZES):
        d = make(rows, n, dt, pt, 100 + i)
        say(f"layer_norm {dt} {pt} rows={rows} n={n} residual={residual}")
        res = d["res"] if residual else None
        y, h, mean, rstd = kb.layer_norm(d["x"], d["w"], d["b"], 1e-5, residual=res)
        h64 = d["x"].double() + (d["res"].double() if residual else 0)
        want, m64, r64 = forward64(h64, d["w"].double(), d["b"].double(), 1e-5)
        # (short rows can lie close together: rstd raises the rounding of x + residual)
        lift = 2.0 ** -21 * h64.abs().max() * d["w"].double().abs().max() * r64[:, None]
        close(y, want, TOL[dt], want.abs().max() + lift / TOL[dt])
        if n > 1:
            close(rstd, r64, 1e-5, r64 * (1 + 2.0 ** -3 * h64.abs().max() * r64))
        close(mean, m64, 1e-6, h64.abs().max())
        if residual:
            assert torch.equal(h, h64.to(F32).to(dt))
        else:
            assert h is d["x"]


@pytest.mark.parametrize("dt,pt", COMBOS)
@pytest.mark.parametrize("residual", [False, True])
def test_backward(dt, pt, residual):
    for i, (rows, n) in enumerate(SIZES):
        d = make(rows, n, dt, pt, 300 + i)
        _, mean, rstd = forward64(d["x"].double(), d["w"].double(), d["b"].double(), 1e-5)
        mean, rstd = mean.float(), rstd.float()
        say(f"layer_norm_backward {dt} {pt} rows={rows} n={n} dh={residual}")
        dh = d["dh"] if residual else None
        dx, dw, db = kb.layer_norm_backward(d["x"], mean, rstd, d["w"], d["dy"], dh=dh)
        want = backward64(d["x"].double(), mean.double(), rstd.double(), d["w"].double(),
                          d["dy"].double(), d["dh"].double() if residual else 0.0)
        # (the three terms of a short row cancel: what is left is good to their size)
        g = (d["dy"].double() * d["w"].double()).abs().amax(1)
        xh = ((d["x"].double() - mean[:, None]) * rstd[:, None]).abs().amax(1)
        terms = (rstd.double() * g * (2 + xh))[:, None]
        close(dx, want[0], TOL[dt], want[0].abs().max() + terms * (1e-5 / TOL[dt]))
        tol = 1e-5 if pt == F32 else 2.0 ** -8
        assert dw.dtype == pt and db.dtype == pt
        close(dw, want[1], tol, want[3] + 1e-3)
        close(db, want[2], tol, want[4])


def test_backward_against_differences():
    """dx, dw and db against central differences of the float64 forward: truncation error
    of a step of 1e-5 stays below 1e-8, so the fp32 gradients' 1e-5 decides."""
    rows, n = 3, 45
    d = make(rows, n, F32, F32, 5)
    h, w, b, dy = (d[k].double().cpu() for k in ("x", "w", "b", "dy"))
    y, _, mean, rstd = kb.layer_norm(d["x"], d["w"], d["b"], 1e-5)
    dx, dw, db = kb.layer_norm_backward(d["x"], mean, rstd, d["w"], d["dy"])
    loss = lambda h, w, b: float((forward64(h, w, b, 1e-5)[0] * dy).sum())
    for got, k in ((dx, 0), (dw, 1), (db, 2)):
        base = [h, w, b]
        num = torch.zeros_like(base[k])
        for j in range(num.numel()):
            ends = []
            for s in (1e-5, -1e-5):
                t = [v.clone() for v in base]
                t[k].view(-1)[j] += s
                ends.append(loss(*t))
            num.view(-1)[j] = (ends[0] - ends[1]) / 2e-5
        close(got.cpu(), num, 2e-5, num.abs().max())


@pytest.mark.parametrize("n", [5, 200, 1000, 3000, 10000, 17000])
def test_rows_far_from_zero(n):
    """A row whose centre is 4096 times its spread: the mean is corrected and the variance
    is of differences, so what is left is the input's own rounding (exact here: the inputs
    are multiples of 2^-9) and the last few roundings."""
    g = torch.Generator(device=device())
    g.manual_seed(n)
    x = torch.randn(6, n, device=device(), generator=g).mul_(512).round_().div_(512) + 4096.0
    say(f"layer_norm offset n={n}")
    y, _, mean, rstd = kb.layer_norm(x)
    want, m64, r64 = forward64(x.double(), 1.0, 0.0, 1e-5)
    close(y, want, 1e-5)
    close(rstd, r64, 1e-5, r64)


@pytest.mark.parametrize("n", [10, 300, 900, 2050, 9000, 16500])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_special_values(n, dt):
    """A NaN or infinity stays in its row; a constant row gives its bias (rstd = 1/sqrt(eps));
    large finite rows whose squares stay finite are exact to the tolerance."""
    d = make(7, n, dt, dt, n)
    x = d["x"].clone()
    x[1, n // 2] = float("nan")
    x[2, n - 1] = float("inf")
    x[3, 0] = -float("inf")
    x[4] = 3.0
    x[5] *= 2.0 ** 50
    x[6] *= 2.0 ** -30
    say(f"layer_norm special n={n} {dt}")
    y, _, mean, rstd = kb.layer_norm(x, d["w"], d["b"], 1e-5)
    want, m64, r64 = forward64(x.double(), d["w"].double(), d["b"].double(), 1e-5)
    for r in (1, 2, 3):
        assert bool(torch.isnan(y[r]).all())
    for r in (0, 4, 5, 6):
        close(y[r], want[r], TOL[dt])
    assert abs(float(rstd[4]) - 1e-5 ** -0.5) < 1e-3
    # the gradient: other rows are as without the odd ones, and so are sums that leave them out
    ok = torch.tensor([0, 4, 5, 6], device=device())
    dx, dw, db = kb.layer_norm_backward(x, mean, rstd, d["w"], d["dy"])
    dx2, dw2, db2 = kb.layer_norm_backward(x[ok].contiguous(), mean[ok].contiguous(),
                                           rstd[ok].contiguous(), d["w"],
                                           d["dy"][ok].contiguous())
    assert torch.equal(dx[ok], dx2)
    assert bool(torch.isnan(dx[1:4]).any(1).all()) and bool(torch.isnan(dw).any())
    assert bool(torch.isfinite(db).all()) and bool(torch.isfinite(dw2).all())


def test_without_parameters_statistics_or_outputs():
    for n in (33, 1500, 5000, 17000):
        d = make(12, n, BF16, F32, n)
        full = kb.layer_norm(d["x"], None, None, 1e-5, residual=d["res"])
        one = torch.ones(n, device=device())
        same = kb.layer_norm(d["x"], one, 0 * one, 1e-5, residual=d["res"], need_stats=False)
        assert torch.equal(full[0], same[0]) and same[2] is None and same[3] is None
        out = (torch.empty_like(d["x"]), torch.empty_like(d["x"]))
        y, h, _, _ = kb.layer_norm(d["x"], eps=1e-5, residual=d["res"], out=out)
        assert y is out[0] and h is out[1] and torch.equal(y, full[0]) and torch.equal(h, full[1])
        _, _, mean, rstd = full
        a = kb.layer_norm_backward(h, mean, rstd, one, d["dy"], dh=d["dh"])
        b = kb.layer_norm_backward(h, mean, rstd, one, d["dy"], dh=d["dh"], need_dw=False)
        c = kb.layer_norm_backward(h, mean, rstd, one, d["dy"], need_dx=False)
        e = kb.layer_norm_backward(h, mean, rstd, None, d["dy"], dh=d["dh"])
        assert torch.equal(a[0], b[0]) and b[1] is None and b[2] is None
        assert c[0] is None and torch.equal(a[1], c[1]) and torch.equal(a[2], c[2])
        assert torch.equal(a[0], e[0]) and e[1].dtype == BF16
        assert torch.equal(a[1].to(BF16), e[1])
        outs = (torch.empty_like(h), torch.empty_like(one), torch.empty_like(one))
        ws = torch.empty(1 << 24, dtype=torch.uint8, device=device())
        f = kb.layer_norm_backward(h, mean, rstd, one, d["dy"], dh=d["dh"], workspace=ws, out=outs)
        assert all(p is q and torch.equal(p, r) for p, q, r in zip(f, outs, a))


def test_shapes_of_more_dimensions_and_empty():
    d = make(24, 40, F32, F32, 1)
    y, h, mean, rstd = kb.layer_norm(d["x"].view(2, 3, 4, 40), d["w"], d["b"])
    assert y.shape == (2, 3, 4, 40) and mean.shape == (2, 3, 4)
    assert torch.equal(y.view(24, 40), kb.layer_norm(d["x"], d["w"], d["b"])[0])
    row = kb.layer_norm(d["x"][0], d["w"], d["b"])
    assert row[0].shape == (40,) and row[2].shape == () and torch.equal(row[0], y[0, 0, 0])
    e = torch.empty(0, 40, device=device())
    y, h, mean, rstd = kb.layer_norm(e, d["w"], d["b"])
    assert y.shape == (0, 40) and mean.shape == (0,)
    dx, dw, db = kb.layer_norm_backward(e, mean, rstd, d["w"], e)
    assert dx.shape == (0, 40) and not bool(dw.any()) and not bool(db.any())
    assert dw.shape == (40,)


def test_repeats_bitwise_on_another_stream():
    d = make(3001, 333, BF16, F32, 9)
    y, h, mean, rstd = kb.layer_norm(d["x"], d["w"], d["b"])
    ref = kb.layer_norm_backward(h, mean, rstd, d["w"], d["dy"])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y2, _, m2, r2 = kb.layer_norm(d["x"], d["w"], d["b"])
        again = kb.layer_norm_backward(h, m2, r2, d["w"], d["dy"])
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y, y2) and all(torch.equal(a, b) for a, b in zip(ref, again))


def test_refusals():
    d = make(4, 16, F32, F32, 1)
    x, w, b = d["x"], d["w"], d["b"]
    m = torch.zeros(4, device=device())
    bad = [lambda: kb.layer_norm(x.cpu()), lambda: kb.layer_norm(x.t()),
           lambda: kb.layer_norm(x, w[:8]), lambda: kb.layer_norm(x, w, b.to(BF16)),
           lambda: kb.layer_norm(x, w, b.cpu()), lambda: kb.layer_norm(x, residual=x[:2]),
           lambda: kb.layer_norm(x, residual=x.to(BF16)), lambda: kb.layer_norm(x, eps=-1.0),
           lambda: kb.layer_norm(x, eps=float("nan")), lambda: kb.layer_norm(x, out=(x, None)),
           lambda: kb.layer_norm(x, out=(torch.empty_like(x), torch.empty_like(x))),
           lambda: kb.layer_norm(torch.empty(4, 0, device=device())),
           lambda: kb.layer_norm_backward(x, m[:3], m, w, x),
           lambda: kb.layer_norm_backward(x, m, m.to(BF16), w, x),
           lambda: kb.layer_norm_backward(x, m, m, w, x[:, :8]),
           lambda: kb.layer_norm_backward(x, m, m, w, x, need_dx=False, need_dw=False),
           lambda: kb.layer_norm_backward(x, m, m, w, d["dy"], out=(x, None, None)),
           lambda: kb.layer_norm_backward(x, m, m, w, d["dy"], dh=x[:2])]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: kb.layer_norm(x.half()), lambda: kb.layer_norm(x, w.to(BF16), b.to(BF16))):
        with pytest.raises(NotImplementedError):
            f()


def test_offsets_past_32_bits():
    """More than 2^31 elements: the last rows as in a call of their own, forward and backward,
    and the weight gradients of rows that are 0 but for those."""
    rows, n = 140000, 16000
    small = make(5, n, BF16, F32, 3)
    say("layer_norm offsets past 2^31")
    x = torch.zeros(rows, n, dtype=BF16, device=device())
    x[-5:] = small["x"]
    y, _, mean, rstd = kb.layer_norm(x, small["w"], small["b"])
    y5, _, m5, r5 = kb.layer_norm(small["x"], small["w"], small["b"])
    assert torch.equal(y[-5:], y5) and torch.equal(mean[-5:], m5) and torch.equal(rstd[-5:], r5)
    del y
    dy = torch.zeros_like(x)
    dy[-5:] = small["dy"]
    dx, dw, db = kb.layer_norm_backward(x, mean, rstd, small["w"], dy)
    dx5, dw5, db5 = kb.layer_norm_backward(small["x"], m5, r5, small["w"], small["dy"])
    assert torch.equal(dx[-5:], dx5) and not bool(dx[: rows - 5].any())
    close(dw, dw5.double(), 1e-5, (small["dy"].double().abs() * 5).amax(0) + 1e-3)
    close(db, db5.double(), 1e-5, small["dy"].double().abs().sum(0) + 1e-3)


@pytest.mark.parametrize("rows,n", [(3, 300), (700, 784), (40, 5000)])
def test_in_a_graph(rows, n):
    """Captured with its gradient, and replayed with other inputs between eager calls."""
    d = make(rows, n, BF16, F32, 11)
    x, dy = d["x"].clone(), d["dy"].clone()
    run = lambda: kb.layer_norm(x, d["w"], d["b"], residual=d["res"])
    back = lambda o: kb.layer_norm_backward(o[1], o[2], o[3], d["w"], dy, dh=d["dh"])
    back(run())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = run()
        g = back(o)
    for turn in range(3):
        e = make(rows, n, BF16, F32, 20 + turn)
        x.copy_(e["x"])
        dy.copy_(e["dy"])
        torch.cuda.synchronize()
        say(f"layer_norm graph rows={rows} n={n} replay {turn}")
        graph.replay()
        torch.cuda.synchronize()
        o2 = run()
        g2 = back(o2)
        assert all(torch.equal(a, b) for a, b in zip(o, o2))
        assert all(torch.equal(a, b) for a, b in zip(g, g2))


@pytest.mark.parametrize("n", [10, 300, 900, 2050, 9000, 16500])
def test_squares_past_fp32(n):
    """Differences whose squares overflow: rstd 0 and y the bias, in that row alone; a constant
    row of large values keeps the variance 0."""
    d = make(3, n, F32, F32, n)
    x = d["x"].clone()
    x[1] *= 2.0 ** 100
    x[2] = 3.0e6
    say(f"layer_norm squares past fp32 n={n}")
    y, _, mean, rstd = kb.layer_norm(x, d["w"], d["b"], 1e-5)
    assert float(rstd[1]) == 0 and torch.equal(y[1], d["b"])
    want, _, r64 = forward64(x.double(), d["w"].double(), d["b"].double(), 1e-5)
    close(y[0], want[0], 1e-5)
    close(y[2], d["b"].double(), 1e-5, 1.0)
    # (the mean of equal values is off by a rounding at most, 0.25 here, squared and taken back
    # to 2^-22 of it)
    assert abs(float(rstd[2]) ** -2 - 1e-5) <= 2.0 ** -22 * 0.25 ** 2 + 1e-9
