"""Log probabilities and their gradient at the edges of what a row can hold, and of how many rows
there are."""
import math

import pytest

from paper_2609_01956_amd import binding as kb
from gpu_common import device, say, torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("classes", [10, 300, 3000, 70000])
@pytest.mark.parametrize("rows", [7, 1100])
def test_gradient_of_rows_without_numbers_or_classes(dt, classes, rows):
    """A row that is NaN throughout, or NaN and masked, has NaN statistics: its gradient is NaN,
    as its log probability is.  A row with no class left has none (0), unless its target is
    invalid, which shows as NaN in every row."""
    g = torch.Generator(device=device())
    g.manual_seed(classes)
    z = torch.randn(rows, classes, device=device(), generator=g).to(dt)
    t = torch.full((rows,), classes // 2, device=device())
    z[0] = math.nan
    z[1] = -math.inf
    z[1, classes // 3] = math.nan
    z[2:5] = -math.inf
    t[3] = classes
    t[4] = -100
    t[5] = -7
    say(f"token_logprobs rows without numbers {dt} rows={rows} classes={classes}")
    logp, stats, ent, _, _ = kb.token_logprobs(z, t, entropy=True)
    assert bool(torch.isnan(logp[:2]).all()) and bool(torch.isnan(ent[:2]).all())
    assert float(logp[2]) == -math.inf and bool(torch.isnan(logp[3])) and float(logp[4]) == 0
    d = torch.ones(rows, device=device())
    for dh in (None, d):
        dz = kb.token_logprobs_backward(z, t, stats, d, entropy=None if dh is None else ent,
                                        dentropy=dh)
        for r in (0, 1, 3, 5):
            assert bool(torch.isnan(dz[r]).all()), r
        for r in (2, 4):
            assert not bool(dz[r].any()), r
        assert bool(torch.isfinite(dz[6:]).all()) and bool(dz[6].any())


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("classes", [20, 900, 5000])
def test_gradient_of_improbable_classes(dt, classes):
    """p = exp(z - m - log s) down to exp(-85): with m = log s = 0 the exponent is exact, so what
    is left is the exponential: an instruction good to a unit in the last place (2^-23), its
    argument's rounding taken back, and one rounding more: 2^-22 (bf16: the result's rounding)."""
    z = (-85 * torch.rand(3, classes, device=device())).to(dt)
    t = torch.zeros(3, dtype=torch.int64, device=device())
    stats = torch.zeros(3, 2, device=device())
    d = torch.full((3,), -1.0, device=device())
    say(f"token_logprobs_backward improbable classes {dt} classes={classes}")
    dz = kb.token_logprobs_backward(z, t, stats, d)[:, 1:].double()
    want = torch.exp(z.double())[:, 1:]
    assert bool(((dz - want).abs() <= (2.0 ** -22 if dt == F32 else 2.0 ** -8) * want).all())


def test_more_rows_than_a_launch():
    """2^26 rows and some: 257 classes of bf16; the last 1000, on both sides of a launch's
    4 (2^24 - 1) tiles, as in a call of their own, forward and (in place) backward."""
    rows, classes = (1 << 26) + 301, 257
    g = torch.Generator(device=device())
    g.manual_seed(1)
    small = torch.randn(1000, classes, device=device(), generator=g).to(BF16)
    ts = torch.randint(0, classes, (1000,), device=device(), generator=g)
    say("token_logprobs more rows than a launch")
    z = torch.zeros(rows, classes, dtype=BF16, device=device())
    z[-1000:] = small
    t = torch.zeros(rows, dtype=torch.int64, device=device())
    t[-1000:] = ts
    logp, stats, ent, _, _ = kb.token_logprobs(z, t, entropy=True)
    want = kb.token_logprobs(small, ts, entropy=True)
    assert torch.equal(logp[-1000:], want[0]) and torch.equal(stats[-1000:], want[1])
    assert torch.equal(ent[-1000:], want[2]) and bool((logp[:-1000] == logp[0]).all())
    d = torch.linspace(-1, 1, rows, device=device())
    kb.token_logprobs_backward(z, t, stats, d, entropy=ent, dentropy=d, out=z)
    dz = kb.token_logprobs_backward(small, ts, want[1], d[-1000:].clone(), entropy=want[2],
                                    dentropy=d[-1000:].clone())
    assert torch.equal(z[-1000:], dz)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("classes", [10, 300, 5000])
def test_gradient_of_a_masked_target(dt, classes):
    """Masked classes have no gradient but the target itself, which keeps the formula's dlogp
    ([v = target] - 0); the others share -dlogp p.  Sums over them to 1e-5, as elsewhere (bf16: a
    rounding of each, 2^-8 of the total at most)."""
    g = torch.Generator(device=device())
    g.manual_seed(classes)
    z = torch.randn(4, classes, device=device(), generator=g).to(dt)
    t = torch.full((4,), classes // 2, device=device())
    z[:, ::2] = -math.inf
    z[:, classes // 2] = -math.inf
    say(f"token_logprobs_backward masked target {dt} classes={classes}")
    logp, stats, _, _, _ = kb.token_logprobs(z, t)
    d = torch.tensor([1.0, -0.5, 2.0, -1.0], device=device())
    dz = kb.token_logprobs_backward(z, t, stats, d).double()
    assert bool((logp == -math.inf).all())
    assert torch.equal(dz[:, classes // 2], d.double())
    masked = torch.isinf(z)
    masked[:, classes // 2] = False
    assert not bool(dz[masked].any())
    rest = dz.sum(1) - d.double()
    assert bool(((rest + d.double()).abs() <= (1e-5 if dt == F32 else 2.0 ** -8) * d.abs()).all())
