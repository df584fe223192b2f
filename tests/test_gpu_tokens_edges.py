"""Token operators at the edges of what their calls allow: scales of either sign and 0, tensors past 4
GiB, strided inputs, workspaces and graphs that share them, outputs at hand."""
import math

import pytest

from paper_2609_01956_amd import binding as kb
from gpu_common import device, say, torch
from test_gpu_head import check_gradients, forward64, gradient64, make, ztol, below, U

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("scale", [-0.3, 0.0])
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("rows,classes,n", [(3, 200, 40), (40, 300, 40), (300, 400, 900),
                                            (900, 3000, 40)])
def test_scales(rows, classes, n, dt, scale):
    x, w, t, d = make(rows, classes, n, 0, 0, 0, dt, 20, std=1.0)
    say(f"linear head scale {scale} {rows} {classes} {n} {dt}")
    logp, stats, best = kb.linear_logprobs(x, w, t, scale=scale, best=True)
    z, lp, m, logs, _ = forward64(x, w, t, scale)
    tol = ztol(z / scale if scale else z, n) * max(abs(scale), 1e-9)
    below((logp.double() - lp).abs(), 2 * tol + 4e-6 + 4 * U * (lp.abs() + z.abs().amax(1)))
    below(m - z.gather(1, best[:, None])[:, 0], 2 * tol + 4 * U * m.abs())
    if scale == 0:
        assert bool((best == 0).all()) and bool((stats[:, 0] == 0).all())
    dx, dw = kb.linear_logprobs_backward(x, w, t, stats, d, scale=scale)
    z, dz = gradient64(x, w, t, stats, d, scale)
    check_gradients(x, w, dx, dw, z, dz, d, scale, dt)


def test_tables_past_4_gib():
    """A table, its gradient and a head's weights of 4.4 GiB: the last rows."""
    V, n = 72000, 32768
    say("token tables past 4 GiB")
    table = torch.zeros(V, n, dtype=BF16, device=device())
    g = torch.Generator(device=device())
    g.manual_seed(21)
    last = torch.randn(50, n, device=device(), generator=g).to(BF16)
    table[-50:] = last
    t = torch.arange(V - 50, V, device=device())
    t[0] = 0
    y = kb.embedding(t, table, scale=2.0)
    assert float(y[0].abs().max()) == 0.0
    assert torch.equal(y[1:], (last[1:].float() * 2).to(BF16))
    grad = kb.embedding_backward(t, y, V, scale=0.5)
    assert torch.equal(grad[-49:], last[1:]) and float(grad[:-49].abs().max()) == 0.0
    del grad
    for rows in (2, 20, 40):
        x = last[1:1 + rows]
        targets = t[1:1 + rows]
        logp, stats, best = kb.linear_logprobs(x, table, targets, scale=n ** -0.5, best=True)
        assert torch.equal(best, targets)  # (its own weight's square against products of others)
        z = torch.zeros(rows, V, dtype=torch.float64, device=device())
        z[:, -50:] = x.double() @ last.double().t() * n ** -0.5
        lp = torch.log_softmax(z, 1).gather(1, targets[:, None])[:, 0]
        below((logp.double() - lp).abs(), 2 * ztol(z, n) + 4e-6 + 4 * U * z.abs().amax(1))
        dx, dw = kb.linear_logprobs_backward(x, table, targets, stats, -torch.ones_like(logp),
                                             scale=n ** -0.5)
        dz = torch.exp(z - stats.double().sum(1, keepdim=True))
        dz[torch.arange(rows), targets] -= 1
        want = dz.t()[-60:] @ x.double() * n ** -0.5
        size = dz.t().abs()[-60:] @ x.double().abs() * n ** -0.5
        p = torch.exp(z - stats.double().sum(1, keepdim=True)).t()[-60:]
        e = (2 * ztol(z, n) + 1e-6) * (p @ x.double().abs()) * n ** -0.5
        below((dw[-60:].double() - want).abs(), size * (2.0 ** -8 + 8 * U) + e * 1.01 +
              2.0 ** -8 * want.abs() + 1e-12)
        assert dx.shape == (rows, n) and not bool(dx.isnan().any())
        del dw


def test_strided_inputs():
    """Rows of wider tensors, at odd offsets: as their copies."""
    g = torch.Generator(device=device())
    g.manual_seed(22)
    for dt in (F32, BF16):
        wide = torch.randn(700, 333, device=device(), generator=g).to(dt)
        table = torch.randn(900, 301, device=device(), generator=g).to(dt)
        t = torch.randint(0, 900, (700,), device=device(), generator=g)
        x, w = wide[:, 7:7 + 200], table[:, 3:3 + 200]
        say(f"token operators strided {dt}")
        for rows in (1, 12, 50, 700):
            a, b = x[:rows], t[:rows]
            one = kb.linear_logprobs(a, w, b, scale=0.1, best=True)
            two = kb.linear_logprobs(a.contiguous(), w.contiguous(), b, scale=0.1, best=True)
            z = (a.double() * 0.1) @ w.double().t()
            # (other kernels may take copies: as close as each is to the logits)
            assert float((one[0] - two[0]).abs().max()) <= 4 * ztol(z, 200) + 8e-6
            d = torch.ones(rows, device=device())
            ga = kb.linear_logprobs_backward(a, w, b, one[1], d, scale=0.1)
            gb = kb.linear_logprobs_backward(a.contiguous(), w.contiguous(), b, one[1], d, scale=0.1)
            for p, q in zip(ga, gb):
                assert torch.equal(p, q)
        assert torch.equal(kb.embedding(t, w), kb.embedding(t, w.contiguous()))
        assert torch.equal(kb.embedding_backward(t, x, 900),
                           kb.embedding_backward(t, x.contiguous(), 900))


def test_workspaces_and_outputs_at_hand():
    """One workspace for all calls, filled with NaN before each; expanded ones are left alone; rows
    past the last are left as they were."""
    g = torch.Generator(device=device())
    g.manual_seed(23)
    x = torch.randn(300, 96, device=device(), generator=g).to(BF16)
    w = torch.randn(4000, 96, device=device(), generator=g).to(BF16)
    t = torch.randint(0, 4000, (300,), device=device(), generator=g)
    d = torch.ones(300, device=device())
    stats = kb.linear_logprobs(x, w, t)[1]
    ws = torch.empty(1 << 28, dtype=torch.uint8, device=device())
    small = torch.full((4096,), 77, dtype=torch.uint8, device=device())
    calls = {
        "linear_logprobs": lambda **k: kb.linear_logprobs(x, w, t, best=True, **k),
        "linear_logprobs_backward": lambda **k: kb.linear_logprobs_backward(x, w, t, stats, d, **k),
        "backward of few": lambda **k: kb.linear_logprobs_backward(x[:3], w, t[:3], stats[:3], d[:3],
                                                                    **k),
        "embedding_backward": lambda **k: [kb.embedding_backward(t, x, 4000, **k)],
        "embedding_backward of many": lambda **k: [kb.embedding_backward(
            t.repeat(40), x.repeat(40, 1), 4000, **k)],
    }
    for name, call in calls.items():
        say(f"{name} with a workspace")
        want = call()
        for k in (ws, small[:1].expand(1 << 28)):
            if k is ws:
                ws.view(F32).fill_(float("nan"))
            for a, b in zip(call(workspace=k), want):
                assert torch.equal(a, b), name
        assert bool((small == 77).all()), name
    full = torch.full((310, 96), 5.0, dtype=BF16, device=device())
    kb.embedding(t, w, out=full[:300])
    assert torch.equal(full[:300], w[t]) and bool((full[300:] == 5).all())
    dx = torch.full((310, 96), 5.0, dtype=BF16, device=device())
    dw = torch.full((4010, 96), 5.0, dtype=BF16, device=device())
    want = kb.linear_logprobs_backward(x, w, t, stats, d)
    kb.linear_logprobs_backward(x, w, t, stats, d, out=(dx[:300], dw[:4000]))
    assert torch.equal(dx[:300], want[0]) and torch.equal(dw[:4000], want[1])
    assert bool((dx[300:] == 5).all()) and bool((dw[4000:] == 5).all())


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("rows", [5, 700])
def test_two_graphs_on_one_workspace(rows, dt):
    """Captured with one workspace between them and replayed in turn with eager work between: each
    replay as the eager call."""
    V, n = 3001, 77
    g = torch.Generator(device=device())
    g.manual_seed(24)
    x = torch.randn(rows, n, device=device(), generator=g).to(dt)
    w = torch.randn(V, n, device=device(), generator=g).to(dt)
    t = torch.randint(0, V, (rows,), device=device(), generator=g)
    d = torch.full((rows,), -1.0 / rows, device=device())
    ws = torch.empty(1 << 28, dtype=torch.uint8, device=device())

    def one():
        logp, stats, _ = kb.linear_logprobs(x, w, t, scale=0.1, workspace=ws)
        return (logp, stats) + kb.linear_logprobs_backward(x, w, t, stats, d, scale=0.1, workspace=ws)

    def two():
        return (kb.embedding_backward(t, x, V, workspace=ws),)
    say(f"token operators in two graphs {rows} {dt}")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one(), two()
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for f in (one, two):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(f())
        graphs.append(graph)
    for turn in range(3):
        x.copy_(torch.randn(rows, n, device=device(), generator=g))
        t.copy_(torch.randint(0, V, (rows,), device=device(), generator=g))
        want = [one(), two()]
        for graph in graphs + graphs[::-1]:
            graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            for p, q in zip(a, b):
                assert torch.equal(p, q), turn


def test_refusals():
    g = torch.Generator(device=device())
    g.manual_seed(25)
    x = torch.randn(20, 16, device=device(), generator=g)
    w = torch.randn(30, 16, device=device(), generator=g)
    t = torch.randint(0, 30, (20,), device=device(), generator=g)
    logp, stats, _ = kb.linear_logprobs(x, w, t)
    say("token operators refusals")
    bad = [lambda: kb.embedding(t.int(), w), lambda: kb.embedding(t[::2], w),
           lambda: kb.embedding(t, w.t()), lambda: kb.embedding(t, w[0]),
           lambda: kb.embedding(t, w.cpu()), lambda: kb.embedding(t, w, scale=math.inf),
           lambda: kb.embedding(t, w, out=torch.empty(20, 15, device=device())),
           lambda: kb.embedding(t, w, out=w[:20]),
           lambda: kb.embedding_backward(t, x[:19], 30), lambda: kb.embedding_backward(t, x, 0),
           lambda: kb.embedding_backward(t, x, 30, base=w[:29]),
           lambda: kb.embedding_backward(t, x, 30, base=w, out=w.to(BF16)),
           lambda: kb.embedding_backward(t, x, 20, out=x),
           lambda: kb.linear_logprobs(x, w[:, :15], t), lambda: kb.linear_logprobs(x, w.to(BF16), t),
           lambda: kb.linear_logprobs(x, w, t[:19]), lambda: kb.linear_logprobs(x.t(), w, t),
           lambda: kb.linear_logprobs(x, w, t, scale=math.nan),
           lambda: kb.linear_logprobs(x.expand(20, 16)[:1].expand(20, 16), w, t),
           lambda: kb.linear_logprobs_backward(x, w, t, stats[:, :1], logp),
           lambda: kb.linear_logprobs_backward(x, w, t, stats, None),
           lambda: kb.linear_logprobs_backward(x, w, t, stats, logp, need_dx=False, need_dw=False),
           lambda: kb.linear_logprobs_backward(x, w, t, stats, logp, out=(x, w)),
           lambda: kb.linear_logprobs_backward(x, w, t, stats, logp, out=(w[:20], None))]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was taken")
    for call in (lambda: kb.embedding(t, w.half()), lambda: kb.linear_logprobs(x.half(), w.half(), t),
                 lambda: kb.embedding(t, w.to(BF16), dtype=F32),
                 lambda: kb.embedding_backward(t, x, 30, dtype=BF16)):
        with pytest.raises(NotImplementedError):
            call()


def test_sizes_past_32_bits():
    """Sizes that a call's 32 bits do not hold are refused, not wrapped to small ones."""
    t = torch.zeros(4, dtype=torch.int64, device=device())
    dy = torch.ones(4, 1, dtype=BF16, device=device())
    say("token operators past 32 bits")
    for classes in (2 ** 32 + 3, 2 ** 31, 0, -1):
        with pytest.raises(ValueError):
            kb.embedding_backward(t, dy, classes)
    table = torch.empty(2 ** 32 + 3, 1, dtype=BF16, device=device())
    with pytest.raises(ValueError):
        kb.embedding(t, table)
    with pytest.raises(ValueError):
        kb.linear_logprobs(dy, table, t)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("rows,classes,n", [(1 << 20, 300, 16), (3, (1 << 24) + 5, 8),
                                            (70, (1 << 22) + 5, 8), (5, 21, 1 << 20),
                                            (100, 21, 1 << 20)])
def test_longest(rows, classes, n, dt):
    """The most rows and columns, and many classes."""
    x, w, t, d = make(rows, classes, n, 0, 0, 0, dt, 26)
    scale = 0.5 * n ** -0.5
    say(f"linear head of the longest {rows} {classes} {n} {dt}")
    logp, stats, best = kb.linear_logprobs(x, w, t, scale=scale, best=True)
    z, lp, m, _, _ = forward64(x, w, t, scale)
    tol = ztol(z, n)
    below((logp.double() - lp).abs(), 2 * tol + 4e-6 + 4 * U * lp.abs())
    below(m - z.gather(1, best[:, None])[:, 0], 2 * tol)
    del z
    dx, dw = kb.linear_logprobs_backward(x, w, t, stats, d, scale=scale)
    z, dz = gradient64(x, w, t, stats, d, scale)
    check_gradients(x, w, dx, dw, z, dz, d, scale, dt)


def test_rows_past_32_bits():
    """Rows of more than 2^32 elements in all, and their sums, which are whole numbers."""
    rows, V, n = 300000, 1000, 16384
    say("embedding rows past 2^32 elements")
    table = (torch.arange(V, device=device())[:, None] % 7 +
             torch.arange(n, device=device()) % 11).to(BF16)
    t = torch.arange(rows, device=device()) * 7 % V
    y = kb.embedding(t, table)
    for first in (0, rows // 2, rows - 100):
        assert torch.equal(y[first:first + 100], table[t[first:first + 100]])
    grad = kb.embedding_backward(t, y, V, dtype=F32)
    assert torch.equal(grad, table.float() * (rows // V))


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("rows,V,n", [(7, 5, 3), (100, 90001, 700), (5000, 2000, 33),
                                      (9000, 90001, 701)])
def test_gradients_at_odd_places(rows, V, n, dt):
    """The gradient and its base one element past an aligned place: as at aligned ones, and nothing
    around it; a row without tokens is its base or 0 wherever in the table it is."""
    g = torch.Generator(device=device())
    g.manual_seed(27)
    t = torch.randint(0, V, (rows,), device=device(), generator=g)
    dy = torch.randn(rows, n, device=device(), generator=g).to(dt)
    base = torch.randn(V, n, device=device(), generator=g).to(dt)
    odd = torch.full((V * n + 2,), 9.0, dtype=dt, device=device())
    odd_base = torch.empty(V * n + 3, dtype=dt, device=device())[3:].view(V, n).copy_(base)
    say(f"embedding_backward at odd places {rows} {V} {n} {dt}")
    absent = torch.ones(V, dtype=torch.bool, device=device())
    absent[t] = False
    for b, ob in ((None, None), (base, odd_base)):
        want = kb.embedding_backward(t, dy, V, base=b)
        assert torch.equal(want[absent], (torch.zeros_like(base) if b is None else b)[absent])
        kb.embedding_backward(t, dy, V, base=ob, out=odd[1:-1].view(V, n))
        assert torch.equal(odd[1:-1].view(V, n), want)
        assert float(odd[0]) == 9.0 and float(odd[-1]) == 9.0


@pytest.mark.parametrize("rows,V", [(6, 10), (16, 3000), (40, 300), (600, 4000)])
def test_targets_nearly_certain(rows, V):
    """1 - p of a target with p nearly 1, in fp32, for given stats: to its own size (2^-22 of the series,
    two roundings of dz and as many of its terms and sum), not to that of p.  Rows of the identity make
    the logits the weights, and dz the weights' gradient."""
    x = torch.eye(rows, device=device())
    t = torch.randperm(V, device=device())[:rows]
    w = torch.zeros(V, rows, device=device())
    w[t, torch.arange(rows, device=device())] = 14.0
    logs = torch.log1p(torch.tensor((V - 1) * math.exp(-14.0), dtype=torch.float64)).float()
    stats = torch.stack([torch.full((rows,), 14.0), logs.expand(rows)], 1).to(device())
    d = -torch.rand(rows, device=device()) - 0.1
    say(f"linear head targets nearly certain {rows} {V}")
    _, dw = kb.linear_logprobs_backward(x, w, t, stats, d, need_dx=False)
    want = -torch.expm1(-logs.double()).to(device()) * d.double()
    got = dw[t, torch.arange(rows, device=device())].double()
    below((got - want).abs(), want.abs() * (2.0 ** -22 + 6 * U))


@pytest.mark.parametrize("rows,classes,n,dt",
                         [(200, 45000, 40, F32),  # big tiles on the fp32 instruction
                          (300, 20000, 1000, F32), (300, 20000, 1000, BF16),  # dW by both tiles
                          (17000, 200, 1000, F32), (17000, 200, 1000, BF16),  # dx by both
                          (17000, 40000, 1000, BF16)])  # added up over pieces
def test_both_tiles(rows, classes, n, dt):
    """More big tiles than fill the GPU a whole number of turns: the rest by small ones."""
    x, w, t, d = make(rows, classes, n, 0, 0, 0, dt, 28)
    scale = 0.5 * n ** -0.5
    say(f"linear head by both tiles {rows} {classes} {n} {dt}")
    logp, stats, _ = kb.linear_logprobs(x, w, t, scale=scale)
    _, lp, _, _, _ = forward64(x, w, t, scale)
    z, dz = gradient64(x, w, t, stats, d, scale)
    below((logp.double() - lp).abs(), 2 * ztol(z, n) + 4e-6 + 4 * U * lp.abs())
    dx, dw = kb.linear_logprobs_backward(x, w, t, stats, d, scale=scale)
    check_gradients(x, w, dx, dw, z, dz, d, scale, dt)


@pytest.mark.parametrize("rows,classes,n", [(65, 3001, 33), (156, 9001, 135), (250, 700, 1001)])
def test_few_rows_in_groups(rows, classes, n):
    """fp32 rows past one group of 64 with weights at odd addresses."""
    x, w, t, _ = make(rows, classes, n, 0, 0, 0, F32, 29)
    scale = n ** -0.5
    say(f"linear head in groups of rows {rows} {classes} {n}")
    logp, stats, best = kb.linear_logprobs(x, w, t, scale=scale, best=True)
    z, lp, m, logs, _ = forward64(x, w, t, scale)
    tol = ztol(z, n)
    below((logp.double() - lp).abs(), 2 * tol + 4e-6 + 4 * U * lp.abs())
    below((stats[:, 0].double() - m).abs(), tol + U * m.abs())
    below((stats[:, 1].double() - logs).abs(), 2 * tol + 4e-6 + 4 * U * logs.abs())
    below(m - z.gather(1, best[:, None])[:, 0], 2 * tol)
