"""Log probabilities of given classes, entropy, the most probable classes and the gradient
on the GPU against the definitions in float64, and against differences.

Tolerances (u = 2^-24, inputs exact in both).  exp(z - m) has the rounding of z - m (at most
u |z - m|, where the weight is at least 1e-7 for |z - m| < 16) and of the exponential's argument
and result, a few u each: a term is good to 32 u.  A sum of positive terms keeps that, and adds
one u per step of a lane (at most 32 per tile, then per tile) and of the joins: 200 u = 1.2e-5
bounds s, relative, so log s, absolute, to 1.2e-5 in the worst case; 4e-6 is asked (the roundings
do not all lie one way), plus 4 u of the value for logp and top_logp and for the entropy.  The
gradient d ([v = t] - p) - dH p (log p + H): p to the same bound, and the rounding of the
result: 1e-5 of the row's largest factor.  bf16 gradients: a rounding (2^-9) on top."""
import math

import pytest

from paper_2609_01956_amd import binding as kb
from gpu_common import device, say, torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16

# rows, classes, padding: one lane to half a wave, one wave, four waves, parts of a row
SIZES = [(1, 1, 0), (3, 2, 0), (70, 5, 3), (300, 10, 0), (65, 16, 1), (40, 33, 0), (9, 100, 7),
         (5, 128, 0), (6, 129, 0), (4, 255, 1), (3, 256, 0), (7, 257, 0), (5, 512, 0), (3, 513, 2),
         (3, 1000, 0), (2, 2047, 0), (2, 2049, 1), (1, 5000, 0), (3, 8192, 0), (1, 50001, 15),
         (2, 131072, 0), (1, 200003, 1), (1100, 8200, 1), (1030, 6145, 0), (4100, 2100, 0),
         (70, 9000, 0)]


def make(rows, classes, pad, dt, seed, std=3.0, shift=0.0):
    g = torch.Generator(device=device())
    g.manual_seed(seed)
    z = torch.randn(rows, classes + pad, device=device(), generator=g) * std + shift
    z = z.to(dt)
    z[:, classes:] = float("nan")  # (what lies between the rows is not read)
    t = torch.randint(0, classes, (rows,), device=device(), generator=g)
    return z[:, :classes], t


def forward64(z, t, k):
    z = z.double()
    m = z.amax(1)
    w = torch.exp(z - m[:, None])
    s = w.sum(1)
    logs = torch.log(s)
    lp = z - m[:, None] - logs[:, None]
    p = w / s[:, None]
    ent = -(p * torch.where(p > 0, lp, 0.0)).sum(1)
    idx = torch.sort(z, dim=1, descending=True, stable=True)[1][:, :k]
    return lp, p, m, logs, ent, idx


def near(got, want, tol, scale=0.0):
    err = (got.double() - want).abs()
    bound = tol + 4 * 2.0 ** -24 * want.abs() + scale
    assert bool((err <= bound).all()), float((err - bound).max())


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("k", [0, 1, 5, 20, 64])
def test_forward(dt, k):
    for i, (rows, classes, pad) in enumerate(SIZES):
        kk = min(k, classes)
        z, t = make(rows, classes, pad, dt, 40 + i)
        say(f"token_logprobs {dt} rows={rows} classes={classes} pad={pad} k={kk}")
        logp, stats, ent, top, idx = kb.token_logprobs(z, t, top_k=kk, entropy=True)
        lp, _, m, logs, e64, i64 = forward64(z, t, kk)
        near(logp, lp.gather(1, t[:, None])[:, 0], 4e-6)
        assert torch.equal(stats[:, 0].double(), m)
        near(stats[:, 1], logs, 4e-6)
        near(ent, e64, 4e-6)
        if kk:
            assert torch.equal(idx, i64)
            near(top, lp.gather(1, i64), 4e-6)
        else:
            assert top is None and idx is None
        again = kb.token_logprobs(z, t, top_k=kk)
        assert torch.equal(again[0], logp) and torch.equal(again[1], stats) and again[2] is None
        if kk:
            assert torch.equal(again[3], top) and torch.equal(again[4], idx)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("order", ["rising", "falling", "constant", "few values", "zeros"])
def test_top_classes_of_awkward_orders(dt, order):
    """Rows that fill the list again and again, and ties that the index has to break (among
    them 0 and -0)."""
    for rows, classes in [(3, 20), (2, 200), (3, 700), (2, 5000), (1, 40000), (1030, 8300)]:
        a = torch.arange(classes, device=device(), dtype=F32)
        z = {"rising": a, "falling": -a, "constant": 0 * a + 2.5,
             "few values": (a * 7919 % 3), "zeros": torch.where(a % 2 == 0, -0.0, 0.0)}[order]
        z = (z / (classes if order in ("rising", "falling") else 1)).to(dt)
        z = z[None, :].repeat(rows, 1)
        t = torch.zeros(rows, dtype=torch.int64, device=device())
        for k in (1, 7, 20):
            say(f"token_logprobs {order} {dt} rows={rows} classes={classes} k={k}")
            _, _, _, top, idx = kb.token_logprobs(z, t, top_k=k)
            lp, _, _, _, _, i64 = forward64(z[:1] + 0.0, t[:1], k)
            assert torch.equal(idx, i64.expand(rows, k))
            near(top, lp.gather(1, i64).expand(rows, k), 4e-6)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("classes", [10, 300, 3000, 70000])
def test_masked_and_special_rows(dt, classes):
    ninf, low = -math.inf, torch.finfo(dt).min
    rows, k = 12, 4
    z, t = make(rows, classes, 5, dt, classes)
    t[:] = classes // 2
    z[0] = ninf                       # no class left
    z[1] = low                        # all masked by the type's lowest value: uniform
    z[2, : classes // 2] = ninf       # masked in part
    z[3, : classes // 2] = low
    z[4] = ninf
    z[4, classes // 2] = 1.5          # one class left
    z[5, 3] = float("nan")
    z[6, classes - 1] = math.inf
    z[7] = ninf
    z[7, classes // 2 + 1] = 0.0      # the target itself is masked
    z[8] += 20000.0 if dt == F32 else 256.0
    z[9, 1] = -low                    # the largest value over ordinary ones
    t[10] = -100
    t[11] = classes                   # outside
    say(f"token_logprobs special {dt} classes={classes}")
    logp, stats, ent, top, idx = kb.token_logprobs(z, t, top_k=k, entropy=True)
    lp, p, m, logs, e64, i64 = forward64(z, t.clamp(0, classes - 1), k)
    assert float(logp[0]) == ninf and float(ent[0]) == 0 and bool((top[0] == ninf).all())
    assert float(stats[0, 0]) == ninf
    assert idx[0].tolist() == list(range(k)) and idx[1].tolist() == list(range(k))
    near(logp[1], torch.tensor(-math.log(classes), dtype=torch.float64), 4e-6)
    near(ent[1], torch.tensor(math.log(classes), dtype=torch.float64), 4e-6)
    for r in (2, 3, 8, 9, 10, 11):
        near(ent[r], e64[r], 4e-6)
        near(top[r], lp[r].gather(0, i64[r]), 4e-6)
        assert torch.equal(idx[r], i64[r])
        if r < 10:
            near(logp[r], lp[r, int(t[r])], 4e-6)
    assert float(logp[4]) == 0 and float(ent[4]) == 0 and int(idx[4, 0]) == classes // 2
    assert float(top[4, 0]) == 0 and bool((top[4, 1:] == ninf).all())
    assert idx[4, 1:].tolist() == [v for v in range(k) if v != classes // 2][:k - 1]
    for r in (5, 6):
        assert math.isnan(float(logp[r])) and math.isnan(float(ent[r]))
        assert bool(torch.isnan(top[r]).all())
    assert int(idx[6, 0]) == classes - 1 and 3 not in idx[5].tolist()
    assert float(logp[7]) == ninf and float(ent[7]) == 0
    assert float(logp[10]) == 0 and math.isnan(float(logp[11]))
    # the gradient
    d = torch.linspace(-1, 1, rows, device=device())
    dh = torch.linspace(0.5, -0.5, rows, device=device())
    dz = kb.token_logprobs_backward(z, t, stats, d, entropy=ent, dentropy=dh)
    assert not bool(dz[0].any())
    for r in (1, 2, 3, 8, 9, 10):
        want = -p[r] * float(d[r] if r != 10 else 0)
        want[int(t[r]) if r != 10 else 0] += float(d[r] if r != 10 else 0)
        lpz = torch.where(p[r] > 0, lp[r], 0.0)
        want = want - float(dh[r]) * p[r] * (lpz + e64[r])
        near(dz[r], want, 1e-5, want.abs() * 2.0 ** -8 if dt == BF16 else 0.0)
    assert not bool(dz[2, : classes // 2].any())
    for r in (5, 6, 11):
        assert bool(torch.isnan(dz[r]).all())


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("entropy", [False, True])
def test_backward(dt, entropy):
    for i, (rows, classes, pad) in enumerate(SIZES):
        z, t = make(rows, classes, pad, dt, 70 + i)
        g = torch.Generator(device=device())
        g.manual_seed(i)
        t[torch.rand(rows, device=device(), generator=g) < 0.2] = 7777777
        d = torch.randn(rows, device=device(), generator=g)
        dh = torch.randn(rows, device=device(), generator=g) if entropy else None
        lp, p, m, logs, e64, _ = forward64(z, t, 1)
        stats = torch.stack([m, logs], 1).float()
        ent = e64.float() if entropy else None
        say(f"token_logprobs_backward {dt} rows={rows} classes={classes} entropy={entropy}")
        dz = kb.token_logprobs_backward(z, t, stats, d, entropy=ent, dentropy=dh,
                                        ignore_index=7777777)
        d64 = torch.where(t == 7777777, 0.0, d.double())
        want = -p * d64[:, None]
        want.scatter_add_(1, torch.where(t == 7777777, 0, t)[:, None], d64[:, None])
        scale = d64.abs()
        if entropy:
            want = want - dh.double()[:, None] * p * (lp + e64[:, None])
            scale = scale + dh.double().abs() * (1 + e64)
        bound = 1e-5 * scale[:, None] + (want.abs() * 2.0 ** -8 if dt == BF16 else 0.0)
        near(dz, want, 0.0, bound)
        # into padded rows, whose padding stays, and over the logits themselves
        pads = torch.full((rows, classes + 3), 7.0, dtype=dt, device=device())
        out = kb.token_logprobs_backward(z, t, stats, d, entropy=ent, dentropy=dh,
                                         ignore_index=7777777, out=pads[:, :classes])
        assert torch.equal(out, dz) and bool((pads[:, classes:] == 7.0).all())
        same = kb.token_logprobs_backward(z, t, stats, d, entropy=ent, dentropy=dh,
                                          ignore_index=7777777, out=z)
        assert same is z and torch.equal(z, dz)


def test_backward_against_differences():
    """dlogits against central differences of the float64 loss (steps of 1e-5: truncation
    below 1e-9, rounding below 1e-9)."""
    z, t = make(3, 37, 0, F32, 3, std=1.0)
    d = torch.tensor([0.7, -1.1, 0.4], device=device())
    dh = torch.tensor([0.3, 0.9, -0.6], device=device())
    _, stats, ent, _, _ = kb.token_logprobs(z, t, entropy=True)
    dz = kb.token_logprobs_backward(z, t, stats, d, entropy=ent, dentropy=dh).cpu()
    z64, tc, dc, hc = z.double().cpu(), t.cpu(), d.double().cpu(), dh.double().cpu()

    def loss(v):
        lp = torch.log_softmax(v, 1)
        return float((dc * lp.gather(1, tc[:, None])[:, 0]).sum() -
                     (hc * (lp.exp() * lp).sum(1)).sum())
    for j in range(z64.numel()):
        ends = []
        for s in (1e-5, -1e-5):
            v = z64.clone()
            v.view(-1)[j] += s
            ends.append(loss(v))
        assert abs(float(dz.view(-1)[j]) - (ends[0] - ends[1]) / 2e-5) < 1e-5


def test_offsets_past_32_bits():
    """Rows whose offset passes 2^31 elements."""
    classes, stride = 5000, 1 << 28
    buf = torch.empty(9 * stride + classes, dtype=BF16, device=device())
    z = buf.as_strided((10, classes), (stride, 1))
    small, t = make(10, classes, 0, BF16, 1)
    z.copy_(small)
    say("token_logprobs offsets past 2^31")
    a = kb.token_logprobs(z, t, top_k=3, entropy=True)
    b = kb.token_logprobs(small, t, top_k=3, entropy=True)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    d = torch.ones(10, device=device())
    want = kb.token_logprobs_backward(small, t, b[1], d)
    assert torch.equal(kb.token_logprobs_backward(z, t, a[1], d, out=z), want)


def test_empty_workspace_and_stream():
    z, t = make(2, 90000, 0, F32, 1)
    ref = kb.token_logprobs(z, t, top_k=9, entropy=True)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=device())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = kb.token_logprobs(z, t, top_k=9, entropy=True, workspace=ws)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(ref, got))
    e, te = z[:0], t[:0]
    logp, stats, ent, top, idx = kb.token_logprobs(e, te, top_k=3, entropy=True)
    assert logp.shape == (0,) and stats.shape == (0, 2) and top.shape == idx.shape == (0, 3)
    assert kb.token_logprobs_backward(e, te, stats, logp).shape == (0, 90000)


def test_refusals():
    z, t = make(4, 16, 0, F32, 1)
    _, stats, ent, _, _ = kb.token_logprobs(z, t, entropy=True)
    d = torch.ones(4, device=device())
    bad = [lambda: kb.token_logprobs(z.cpu(), t.cpu()), lambda: kb.token_logprobs(z.t(), t),
           lambda: kb.token_logprobs(z[0], t), lambda: kb.token_logprobs(z, t[:3]),
           lambda: kb.token_logprobs(z, t.int()), lambda: kb.token_logprobs(z, t.cpu()),
           lambda: kb.token_logprobs(z, t, top_k=17), lambda: kb.token_logprobs(z, t, top_k=-1),
           lambda: kb.token_logprobs(z[:1].expand(4, 16), t),
           lambda: kb.token_logprobs(z[:, :0], t),
           lambda: kb.token_logprobs_backward(z, t, stats[:, :1], d),
           lambda: kb.token_logprobs_backward(z, t, stats, d[:2]),
           lambda: kb.token_logprobs_backward(z, t, stats, d.double()),
           lambda: kb.token_logprobs_backward(z, t, stats, d, entropy=ent),
           lambda: kb.token_logprobs_backward(z, t, stats, d, dentropy=d),
           lambda: kb.token_logprobs_backward(z, t, stats, d, out=z[:2]),
           lambda: kb.token_logprobs_backward(z, t, stats, d, out=z.to(BF16))]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    wide, tw = make(2, 100, 0, F32, 1)
    with pytest.raises(ValueError):
        kb.token_logprobs(wide, tw, top_k=65)
    with pytest.raises(NotImplementedError):
        kb.token_logprobs(z.half(), t)


@pytest.mark.parametrize("rows,classes", [(100, 10), (2, 60000), (1100, 3000)])
def test_in_a_graph(rows, classes):
    """Captured with its gradient, and replayed with other inputs between eager calls."""
    z, t = make(rows, classes, 0, BF16, 1)
    z = z.clone()
    d = torch.randn(rows, device=device())
    run = lambda: kb.token_logprobs(z, t, top_k=7, entropy=True)
    back = lambda o: kb.token_logprobs_backward(z, t, o[1], d, entropy=o[2], dentropy=d)
    back(run())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = run()
        g = back(o)
    for turn in range(3):
        z.copy_(make(rows, classes, 0, BF16, 50 + turn)[0])
        torch.cuda.synchronize()
        say(f"token_logprobs graph rows={rows} classes={classes} replay {turn}")
        graph.replay()
        torch.cuda.synchronize()
        o2 = run()
        assert all(torch.equal(a, b) for a, b in zip(o, o2))
        assert torch.equal(g, back(o2))


@pytest.mark.parametrize("dt", [F32, BF16])
def test_fewer_numbers_than_alternatives(dt):
    """Rows that are NaN or masked but for a few classes: numbers first, then the masked, then
    NaN, each by rising index, in one tile, several, and parts of a row."""
    for rows, classes in [(2, 12), (3, 200), (2, 700), (2, 9000), (1030, 5000)]:
        z = torch.full((rows, classes), float("nan"), dtype=dt, device=device())
        t = torch.zeros(rows, dtype=torch.int64, device=device())
        z[:, classes - 1] = 1.0
        z[:, 5] = 1.0
        z[:, 7] = 2.0
        z[:, 9] = -math.inf
        say(f"token_logprobs few numbers {dt} rows={rows} classes={classes}")
        _, _, _, top, idx = kb.token_logprobs(z, t, top_k=8)
        want = [7, 5, classes - 1, 9] + [i for i in range(classes) if i not in (5, 7, 9)][:4]
        assert idx.tolist() == [want] * rows and bool(torch.isnan(top).all())
