"""Token operators at the sizes at which their kernels go another way, on the GPU against the formulas
in float64: runs of tokens around a chunk of sorted entries and around a group of chunks, and fp32
gradients of few rows over a vocabulary in several pieces."""
import pytest

from paper_2609_01956_amd import binding as kb
from gpu_common import device, say, torch
from test_gpu_head import check_gradients, gradient64

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
TYPES = [(F32, F32), (BF16, BF16), (BF16, F32)]  # of the rows, of the table


def check_runs(counts, n, dt, tt, seed):
    """Tokens 0, 1, .. so many times each, shuffled, with whole numbers, which fp32 adds exactly in any
    order: equal to the definition's, rounded once; with a base, in place too."""
    g = torch.Generator(device=device())
    g.manual_seed(seed)
    counts = torch.tensor(counts, device=device())
    t = torch.repeat_interleave(torch.arange(counts.numel(), device=device()), counts)
    t = t[torch.randperm(t.numel(), device=device(), generator=g)]
    dy = torch.randint(-4, 5, (t.numel(), n), device=device(), generator=g).to(dt)
    base = torch.randint(-4, 5, (counts.numel(), n), device=device(), generator=g).to(tt)
    want = torch.zeros(counts.numel(), n, dtype=torch.float64, device=device())
    want.index_add_(0, t, dy.double())
    got = kb.embedding_backward(t, dy, counts.numel(), dtype=tt)
    assert torch.equal(got, want.to(tt))
    total = (want + base.double()).to(tt)
    assert torch.equal(kb.embedding_backward(t, dy, counts.numel(), base=base), total)
    inside = base.clone()
    kb.embedding_backward(t, dy, counts.numel(), base=inside, out=inside)
    assert torch.equal(inside, total)


@pytest.mark.parametrize("dt,tt", TYPES)
@pytest.mark.parametrize("n", [1, 5, 8, 40])
def test_runs_around_a_chunk(dt, tt, n):
    """Runs of 15, 16 and 17 entries (the most that one chunk sums, and the fewest that it does not)
    and of about two chunks, at every offset from a chunk's first entry."""
    say(f"embedding_backward runs around a chunk {dt} {tt} {n}")
    for lead in range(17):
        check_runs([lead, 15, 16, 17, 1, 31, 32, 33, 0, 16, 17, 15, 2, 48, 17, 17, 16, 16, 15], n, dt,
                   tt, lead)


@pytest.mark.parametrize("dt,tt", TYPES)
@pytest.mark.parametrize("n", [3, 264])
def test_runs_around_a_group_of_chunks(dt, tt, n):
    """The same around 1024 entries, from which on a token's sums are themselves summed."""
    say(f"embedding_backward runs around a group of chunks {dt} {tt} {n}")
    for lead in (0, 1, 15, 16, 17, 1023):
        check_runs([lead, 1023, 1024, 1025, 1, 1024, 2047, 2048, 2049, 16, 1024], n, dt, tt, lead)


@pytest.mark.parametrize("dt,tt", TYPES)
@pytest.mark.parametrize("rows", [15, 16, 17])
def test_batches_around_a_chunk(dt, tt, rows):
    """A batch of a chunk, and one token less and more: all of one token, and of two."""
    say(f"embedding_backward batches around a chunk {dt} {tt} {rows}")
    for first in (rows, 1, rows - 1, rows // 2):
        check_runs([0, first, 0, rows - first], 9, dt, tt, first)


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
