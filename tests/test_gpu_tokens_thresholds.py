"""Token operators at the sizes at which their kernels go another way, on the GPU against the formulas
in float64: fp32 gradients of few rows over a vocabulary in several pieces."""
import pytest

from paper_2609_01956_amd import binding as kb
from gpu_common import device, say, torch
from test_gpu_head import check_gradients, gradient64

pytestmark = pytest.mark.gpu

F32 = torch.float32



def head_inputs(rows, classes, n, seed):
    """x, weight, targets in every part of the vocabulary, and dlogp, in fp32."""
    g = torch.Generator(device=device())
    g.manual_seed(seed)
    x = torch.randn(rows, n, device=device(), generator=g)
    w = torch.randn(classes, n, device=device(), generator=g)
    t = torch.arange(rows, device=device()) * (classes - 1) // (rows - 1)
    return x, w, t, -torch.rand(rows, device=device(), generator=g)


@pytest.mark.parametrize("rows,classes,n", [(20, 50001, 4096), (40, 131072, 1024), (64, 60001, 4001)])
def test_few_rows_in_pieces(rows, classes, n):
    """fp32 gradients of 17 to 64 rows whose vocabulary goes through several pieces, each alone as
    both together."""
    x, w, t, d = head_inputs(rows, classes, n, 41)
    scale = 0.7 * n ** -0.5
    say(f"linear_logprobs_backward of few rows in pieces {rows} {classes} {n}")
    _, stats, _ = kb.linear_logprobs(x, w, t, scale=scale)
    dx, dw = kb.linear_logprobs_backward(x, w, t, stats, d, scale=scale)
    z, dz = gradient64(x, w, t, stats, d, scale)
    check_gradients(x, w, dx, dw, z, dz, d, scale, F32)
    del z, dz
    one, _ = kb.linear_logprobs_backward(x, w, t, stats, d, scale=scale, need_dw=False)
    assert torch.equal(one, dx)
    _, two = kb.linear_logprobs_backward(x, w, t, stats, d, scale=scale, need_dx=False)
    assert torch.equal(two, dw)


@pytest.mark.parametrize("rows,classes,n", [(20, 9001, 1024), (64, 20000, 100)])
def test_few_rows_leave_out_what_nothing_reads(rows, classes, n):
    """The weights' gradient alone has no use for the weights laid out anew (two bytes a value and
    term): less of the workspace is written."""
    x, w, t, d = head_inputs(rows, classes, n, 42)
    say(f"linear_logprobs_backward of few rows, dweight alone {rows} {classes} {n}")
    _, stats, _ = kb.linear_logprobs(x, w, t)
    ws = torch.full((1 << 28,), 0xa5, dtype=torch.uint8, device=device())
    _, dw = kb.linear_logprobs_backward(x, w, t, stats, d, need_dx=False, workspace=ws)
    _, want = kb.linear_logprobs_backward(x, w, t, stats, d)
    assert torch.equal(dw, want)
    # (z in fp32 for whole groups of 16 rows, dz's terms, those of x)
    most = classes * (64 * 4 + 6 * 64) + rows * (n + 8) * 8 + (1 << 20)
    assert int((ws != 0xa5).sum()) <= most
