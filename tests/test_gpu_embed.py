"""The embedding of tokens and its table's gradient on the GPU, against the definitions in float64.

Tolerances: the forward is one fp32 product (half a step) and its rounding.  The gradient is a sum of c
terms in fp32 (c - 1 roundings of partial sums, each within the sum of the terms' sizes A: c u A
bounds them), a product with the scale and the base's addition as one operation (u), and the
rounding to the table's type; u = 2^-24, in bf16 2^-8."""
import pytest

from paper_2609_01956_amd import binding as kb
from gpu_common import device, say, torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
TYPES = [(F32, F32), (BF16, BF16), (BF16, F32)]  # of the rows, of the table
HALF = {F32: U, BF16: 2.0 ** -8}


def make_tokens(rows, classes, seed, common=0.5):
    """Half of them one of a few, as in a text; some to be left out, some that are no class."""
    g = torch.Generator(device=device())
    g.manual_seed(seed)
    t = torch.randint(0, classes, (rows,), device=device(), generator=g)
    few = torch.randint(0, min(classes, 5), (rows,), device=device(), generator=g)
    t = torch.where(torch.rand(rows, device=device(), generator=g) < common, few, t)
    t[torch.rand(rows, device=device(), generator=g) < 0.1] = -100
    t[torch.rand(rows, device=device(), generator=g) < 0.02] = classes
    return t, g


@pytest.mark.parametrize("dt,tt", TYPES)
@pytest.mark.parametrize("rows,classes,n,pad", [
    (1, 1, 1, 0), (1, 50001, 256, 0), (7, 10, 3, 1), (100, 30, 8, 0), (33, 100, 9, 7),
    (1000, 257, 100, 0), (5, 20, 4096, 8), (300, 40, 1001, 1), (4097, 999, 17, 0)])
def test_forward(dt, tt, rows, classes, n, pad):
    t, g = make_tokens(rows, classes, 1)
    table = torch.randn(classes, n + pad, device=device(), generator=g).to(tt)
    table[:, n:] = float("nan")
    table = table[:, :n]
    say(f"embedding {dt} {tt} {rows} {classes} {n} {pad}")
    y = kb.embedding(t, table, scale=1.7, dtype=dt)
    assert y.shape == (rows, n) and y.dtype == dt
    ok = (t >= 0) & (t < classes)
    want = table[t.clamp(0, classes - 1)].double() * 1.7
    assert bool((y[t == -100] == 0).all()) and bool(y[t == classes].isnan().all())
    # (1.7 itself is rounded to fp32: one more u)
    err, bound = (y.double() - want).abs(), (HALF[dt] + 2 * U) * 1.01 * want.abs()
    assert bool((err[ok] <= bound[ok]).all())
    assert torch.equal(kb.embedding(t.view(1, rows), table, scale=1.7, dtype=dt)[0].nan_to_num(9.0),
                       y.nan_to_num(9.0))


GRAD_SIZES = [  # one workgroup's sort, one pass, two, three; rows of a unit and of many
    (1, 1, 1), (1, 50001, 256), (31, 2, 8), (32, 1, 8), (33, 1, 9), (64, 3, 4), (100, 7, 100),
    (1000, 300000, 12), (4096, 511, 33), (4097, 512, 40), (5000, 20, 7), (20000, 70000, 16),
    (9000, 300, 1001), (66000, 1000, 8), (300000, 400, 4), (270000, 300000, 3)]


@pytest.mark.parametrize("dt,tt", TYPES)
@pytest.mark.parametrize("rows,classes,n", GRAD_SIZES)
def test_gradient(dt, tt, rows, classes, n):
    t, g = make_tokens(rows, classes, 2)
    dy = torch.randn(rows, n + 3, device=device(), generator=g).to(dt)
    dy[:, n:] = float("nan")
    dy = dy[:, :n]
    dy[t == -100] = float("nan")  # (not read, or read and dropped)
    base = torch.randn(classes, n, device=device(), generator=g).to(tt)
    say(f"embedding_backward {dt} {tt} {rows} {classes} {n}")
    got = kb.embedding_backward(t, dy, classes, scale=0.3, dtype=tt)
    ok = (t >= 0) & (t < classes)
    terms = torch.zeros(classes, n, dtype=torch.float64, device=device())
    want = terms.clone()
    want.index_add_(0, t[ok], dy[ok].double() * 0.3)
    terms.index_add_(0, t[ok], dy[ok].double().abs() * 0.3)
    count = torch.bincount(t[ok], minlength=classes)[:, None]

    def check(got, want):
        bound = (count * U + 2 * U) * terms * 1.01 + (HALF[tt] + U) * want.abs() * 1.01
        err = (got.double() - want).abs()
        assert bool((err <= bound).all()), float((err - bound).max())
    assert got.shape == (classes, n) and got.dtype == tt
    check(got, want)
    again = kb.embedding_backward(t, dy, classes, scale=0.3, dtype=tt)
    assert torch.equal(got, again)
    added = kb.embedding_backward(t, dy, classes, scale=0.3, base=base)
    check(added, want + base.double())
    inside = base.clone()
    assert kb.embedding_backward(t, dy, classes, scale=0.3, base=inside, out=inside) is inside
    assert torch.equal(inside, added)


@pytest.mark.parametrize("rows", [40, 4096, 5000, 100000])
def test_sum_is_in_the_batch_s_order(rows):
    """One token throughout, and integers that fp32 sums exactly: every entry is in, once."""
    t = torch.full((rows,), 3, device=device())
    dy = torch.arange(rows, device=device(), dtype=F32)[:, None] % 64
    say(f"embedding_backward one token {rows}")
    g = kb.embedding_backward(t, dy, 5)
    assert float(g[3, 0]) == float(dy.double().sum()) and float(g.abs().sum()) == float(g[3, 0])


def test_runs_across_chunks():
    """Runs of every length around the chunk of 32 sorted entries, at every offset from it."""
    for lead in range(0, 34, 3):
        counts = [lead, 31, 32, 33, 1, 64, 65, 0, 2, 96, 40, 7, 33, 33, 100]
        t = torch.repeat_interleave(torch.arange(len(counts)), torch.tensor(counts)).to(device())
        g = torch.Generator(device=device())
        g.manual_seed(lead)
        t = t[torch.randperm(t.numel(), device=device(), generator=g)]
        dy = torch.randint(-8, 9, (t.numel(), 5), device=device(), generator=g).to(F32)
        if lead == 0:
            say("embedding_backward runs")
        got = kb.embedding_backward(t, dy, len(counts))
        want = torch.zeros(len(counts), 5, device=device()).index_add_(0, t, dy)
        assert torch.equal(got, want), lead


def test_empty_batch_and_absent_tokens():
    t = torch.empty(0, dtype=torch.int64, device=device())
    base = torch.randn(9, 6, device=device())
    say("embedding empty")
    assert kb.embedding(t, base).shape == (0, 6)
    dy = torch.empty(0, 6, device=device())
    assert float(kb.embedding_backward(t, dy, 9).abs().max()) == 0.0
    assert torch.equal(kb.embedding_backward(t, dy, 9, base=base), base)
    t = torch.full((50,), -100, device=device())
    dy = torch.full((50, 6), float("nan"), device=device())
    assert float(kb.embedding_backward(t, dy, 9).abs().max()) == 0.0
