"""Log probabilities and their gradient at the edges of what a row can hold."""
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
