"""The global norm of many tensors and their clipping on the GPU against float64.

Tolerances.  The sum of squares is in 64 bits, so norm carries one rounding to fp32: 2^-23 of
it.  The factor is rounded once, the product once: 2^-22 of each fp32 gradient, and a bf16
rounding (2^-8 of each) on top."""
import math

import pytest

from paper_2609_01956_amd import binding as kb
from gpu_common import device, say, torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def make(sizes, dtypes, seed=0, std=1.0):
    g = torch.Generator(device=device())
    g.manual_seed(seed)
    return [(torch.randn(n, device=device(), generator=g) * std).to(dt)
            for n, dt in zip(sizes, dtypes)]


def norm64(grads):
    return math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))


def check_scaled(got, grads, c):
    for a, g in zip(got, grads):
        want = g.double() * c
        tol = 2.0 ** -22 if g.dtype == F32 else 2.0 ** -8
        assert a.dtype == g.dtype and bool(((a.double() - want).abs() <= tol * want.abs() +
                                            1e-44).all())


# one element, parts of a 16-byte unit, one chunk and its edges, several, and more tensors
# than one launch takes
LISTS = {
    "one": ([1], [F32]),
    "small": ([3, 8, 1, 17, 64], [F32, BF16, BF16, F32, BF16]),
    "empty among them": ([0, 5, 0, 9], [F32, BF16, BF16, F32]),
    "chunk": ([16383, 16384, 16385, 32768], [BF16, F32, BF16, F32]),
    "large": ([3000017, 5, 1 << 22], [F32, F32, BF16]),
    "many": ([(i * 37) % 300 + 1 for i in range(700)],
             [F32 if i % 3 else BF16 for i in range(700)]),
    "launch edges": ([2] * 257, [F32] * 257),
}


@pytest.mark.parametrize("name", LISTS)
def test_norm_and_clip(name):
    sizes, dtypes = LISTS[name]
    grads = make(sizes, dtypes, seed=len(sizes))
    n64 = norm64(grads)
    say(f"grad_norm {name}")
    n = kb.grad_norm(grads)
    assert n.shape == () and n.dtype == F32 and abs(float(n) - n64) <= 2.0 ** -23 * n64
    for share in (0.37, 3.0):
        c = min(1.0, share * n64 / (n64 + 1e-6))
        keep = [g.clone() for g in grads]
        out = [torch.full_like(g, 9.0) for g in grads]
        say(f"clip_grad_norm {name} share={share}")
        n = kb.clip_grad_norm(grads, share * n64, out=out)
        assert abs(float(n) - n64) <= 2.0 ** -23 * n64
        assert all(torch.equal(a, b) for a, b in zip(grads, keep))
        check_scaled(out, keep, c)
        n = kb.clip_grad_norm(keep, share * n64)
        assert all(torch.equal(a, b) for a, b in zip(keep, out))


def test_views_of_one_buffer_keep_their_neighbours():
    """Odd-sized views side by side, every other one clipped in place."""
    for dt in (F32, BF16):
        flat = torch.ones(10007, dtype=dt, device=device())
        cuts = [0, 1, 4, 11, 100, 1001, 5000, 10007]
        views = [flat[a:b] for a, b in zip(cuts, cuts[1:])]
        kb.clip_grad_norm(views[1::2], 0.5, eps=0.0)
        total = math.sqrt(sum(v.numel() for v in views[1::2]))
        for i, v in enumerate(views):
            want = 1.0 if i % 2 == 0 else 0.5 / total
            assert bool(((v.double() - want).abs() <= 2.0 ** -8 * want).all())
            assert i % 2 or bool((v == 1).all())


def test_range_of_values():
    """No overflow and no underflow: squares of the largest and of the smallest gradients."""
    big = [torch.full((1000,), 1e38, device=device()), torch.full((9,), -2e38, device=device())]
    assert abs(float(kb.grad_norm([big[0][:4]])) - 2e38) <= 2e31
    assert math.isinf(float(kb.grad_norm(big)))  # (3.2e39 itself is past fp32)
    out = [torch.empty_like(b) for b in big]
    kb.clip_grad_norm(big, 1.0, out=out)
    check_scaled(out, big, 1.0 / norm64(big))
    tiny = [torch.full((100,), 1e-40, device=device())]
    assert abs(float(kb.grad_norm(tiny)) / norm64(tiny) - 1) <= 1e-4  # (a subnormal's own rounding)
    zero = [torch.zeros(50, device=device())]
    for m in (0.0, 1.0):
        assert float(kb.clip_grad_norm(zero, m, eps=0.0)) == 0 and not bool(zero[0].any())
    some = make([40], [F32])
    kb.clip_grad_norm(some, 0.0)
    assert not bool(some[0].any())
    some = make([40], [F32])
    keep = some[0].clone()
    kb.clip_grad_norm(some, math.inf)
    assert torch.equal(some[0], keep)


def test_nan_and_infinity():
    g = make([100, 7], [F32, BF16])
    g[1][3] = float("nan")
    out = [torch.empty_like(v) for v in g]
    assert math.isnan(float(kb.clip_grad_norm(g, 1.0, out=out)))
    assert all(bool(torch.isnan(v).all()) for v in out)
    g[1][3] = math.inf
    assert math.isinf(float(kb.clip_grad_norm(g, 1.0, out=out)))
    assert not bool(out[0].any()) and math.isnan(float(out[1][3]))


def test_repeats_bitwise_on_another_stream_and_in_a_graph():
    sizes, dtypes = LISTS["many"]
    grads = make(sizes, dtypes, seed=5)
    out = [torch.empty_like(g) for g in grads]
    n = kb.clip_grad_norm(grads, 2.0, out=out)
    ref = [n.clone()] + [o.clone() for o in out]
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=device())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        n2 = kb.clip_grad_norm(grads, 2.0, out=out, workspace=ws)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(n2, ref[0]) and all(torch.equal(a, b) for a, b in zip(out, ref[1:]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        n3 = kb.clip_grad_norm(grads, 2.0, out=out, workspace=ws)
    for turn in range(3):
        for o in out:
            o.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        say(f"clip graph replay {turn}")
        assert torch.equal(n3, ref[0]) and all(torch.equal(a, b) for a, b in zip(out, ref[1:]))


def test_refusals():
    g = make([8, 8], [F32, BF16])
    o = [torch.empty_like(v) for v in g]
    m = torch.zeros(4, 4, device=device())
    bad = [lambda: kb.grad_norm([]), lambda: kb.clip_grad_norm([], 1.0),
           lambda: kb.grad_norm([v.cpu() for v in g]), lambda: kb.grad_norm([g[0], g[1].cpu()]),
           lambda: kb.grad_norm([m.t()[1:]]), lambda: kb.clip_grad_norm(g, -1.0),
           lambda: kb.clip_grad_norm(g, math.nan), lambda: kb.clip_grad_norm(g, 1.0, eps=-1.0),
           lambda: kb.clip_grad_norm(g, 1.0, out=o[:1]),
           lambda: kb.clip_grad_norm(g, 1.0, out=[o[1], o[0]]),
           lambda: kb.clip_grad_norm(g, 1.0, out=[v.cpu() for v in o]),
           lambda: kb.clip_grad_norm([g[0], g[0]], 1.0),
           lambda: kb.clip_grad_norm([m[0], m[1]], 1.0, out=[m[1], m[2]])]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    with pytest.raises(NotImplementedError):
        kb.grad_norm([g[0].half()])
    with pytest.raises(NotImplementedError):
        kb.grad_norm([g[0].double()])


def test_offsets_past_32_bits():
    """A tensor of more than 2^31 elements, 0 but for its ends."""
    n = (1 << 31) + 12345
    g = torch.zeros(n, dtype=BF16, device=device())
    g[:3] = 2.0
    g[-7:] = 3.0
    total = math.sqrt(3 * 4 + 7 * 9)
    say("clip_grad_norm offsets past 2^31")
    got = float(kb.clip_grad_norm([g], total / 2, eps=0.0))
    assert abs(got - total) <= 2.0 ** -22 * total
    assert bool((g[:3] == 1.0).all()) and bool((g[-7:] == 1.5).all())
    assert int((g != 0).sum()) == 10
