"""The token model of paper_2609_01956_amd.train: embedding, KAN layers and the head on one table,
against the same model in float64 torch with autograd; and a run of the operators in a graph."""
import math

import pytest

from paper_2609_01956_amd import binding as kb
from gpu_common import device, say, torch
from test_gpu_train import kan64

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def model64(table, params, tokens, targets, grid, scale, pad):
    keep = (tokens != pad)[..., None]
    x = torch.where(keep, table[tokens.clamp(min=0)] * scale, 0.0).flatten(1)
    stream, out = None, x
    for w, b, coef, base_w in params:
        h = out + stream if stream is not None and stream.shape == out.shape else out
        c = h - h.mean(1, keepdim=True)
        z = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * w + b
        stream, out = h, kan64(z, coef, base_w, *grid)
    lp = torch.log_softmax(out @ table.t(), 1)
    ok = targets != pad
    return lp[ok].gather(1, targets[ok][:, None]).mean()


@pytest.mark.parametrize("dt,tol", [(F32, 1e-4), (BF16, 0.1)])
@pytest.mark.parametrize("classes,width,context,hidden", [(50, 16, 2, (16,)), (301, 24, 3, (40, 24))])
def test_gradients_against_autograd(dt, tol, classes, width, context, hidden):
    """fp32: the sums of a few hundred terms at each of four layers, 1e-4 of a parameter's largest
    gradient.  bf16: six roundings of 2^-8 per layer, forward and backward, of either sign and
    passed on with a factor of about 2: sqrt(24) 2 2^-8 = 0.04 of a parameter's gradient, the head's
    and the embedding's four more (0.016 of it); 0.1 of its 2-norm is asked."""
    from paper_2609_01956_amd.train import KanTokenModel
    g = torch.Generator(device=device())
    g.manual_seed(4)
    model = KanTokenModel(classes, width, context, hidden, grid_size=6, dtype=dt, device=device())
    tokens = torch.randint(0, classes, (200, context), device=device(), generator=g)
    tokens[torch.rand(200, context, device=device(), generator=g) < 0.3] = 7
    tokens[:20, 0] = -100
    targets = torch.randint(0, classes, (200,), device=device(), generator=g)
    targets[5:30] = -100
    say(f"token model gradients {dt} {classes} {width} {context} {hidden}")
    logp, grads = model.gradients(tokens, targets)
    table = model.table.double().requires_grad_()
    params = [[p.double().requires_grad_() for p in layer] for layer in model.body.params]
    want = model64(table, params, tokens, targets, model.body.grid, model.scale, -100)
    (-want).backward()
    assert abs(float(logp) - float(want.detach())) <= tol * abs(float(want.detach()))
    flat = [table] + [p for layer in params for p in layer]
    assert len(grads) == len(flat) == len(model.parameters())
    for a, p, like in zip(grads, flat, model.parameters()):
        assert a.dtype == like.dtype and a.shape == like.shape
        err = (a.double() - p.grad).abs()
        if dt == F32:
            assert float(err.max()) <= tol * float(p.grad.abs().max())
        else:
            assert float(err.norm()) <= tol * float(p.grad.norm())


@pytest.mark.parametrize("dt", [F32, BF16])
def test_steps_and_next_tokens(dt):
    from paper_2609_01956_amd.train import KanTokenModel
    g = torch.Generator(device=device())
    g.manual_seed(5)
    model = KanTokenModel(90, 32, dtype=dt, device=device())
    say(f"token model steps {dt}")
    for _ in range(3):
        tokens = torch.randint(0, 90, (256, 2), device=device(), generator=g)
        logp, norm = model.step(tokens, tokens[:, 0].contiguous())
        assert math.isfinite(float(logp)) and math.isfinite(float(norm))
    for rows in (1, 7, 200):
        best, lp = model.next_tokens(tokens[:rows])
        h, _ = model.forward(tokens[:rows], need_stats=False)
        z = torch.log_softmax(h.double() @ model.table.double().t(), 1)
        assert best.shape == lp.shape == (rows,)
        assert float((lp.double() - z.amax(1)).abs().max()) < 1e-4
        assert float((z.amax(1) - z.gather(1, best[:, None])[:, 0]).abs().max()) < 1e-4


def test_run_in_a_graph():
    """Embedding, head, their gradients and the update's sum captured once and replayed with other
    tokens and eager work between: each replay as the eager calls."""
    V, n, rows = 5000, 64, 6000
    g = torch.Generator(device=device())
    g.manual_seed(6)
    table = torch.randn(V, n, device=device(), generator=g).to(BF16)
    tokens = torch.randint(0, V, (rows,), device=device(), generator=g)
    targets = torch.randint(0, V, (rows,), device=device(), generator=g)
    d = torch.full((rows,), -1.0 / rows, device=device())

    def run():
        x = kb.embedding(tokens, table, scale=0.5)
        logp, stats, best = kb.linear_logprobs(x, table, targets, scale=0.25, best=True)
        dx, dw = kb.linear_logprobs_backward(x, table, targets, stats, d, scale=0.25)
        dw = kb.embedding_backward(tokens, dx, V, scale=0.5, base=dw, out=dw)
        return logp, stats, best, dx, dw
    say("token operators in a graph")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    for seed in range(4):
        tokens.copy_(torch.randint(0, V, (rows,), device=device(), generator=g) // (seed + 1))
        targets.copy_(torch.randint(0, V, (rows,), device=device(), generator=g))
        want = run()
        for t in captured:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, want):
            assert torch.equal(a, b), seed


def test_on_another_stream_and_two_at_once():
    """Calls on two streams, each with its own workspace: as one after the other."""
    g = torch.Generator(device=device())
    g.manual_seed(7)
    jobs = []
    for i in range(2):
        t = torch.randint(0, 700, (5000,), device=device(), generator=g)
        dy = torch.randn(5000, 40, device=device(), generator=g)
        x = torch.randn(300, 40, device=device(), generator=g)
        w = torch.randn(700, 40, device=device(), generator=g)
        jobs.append((t, dy, x, w))

    def run(t, dy, x, w):
        logp, stats, _ = kb.linear_logprobs(x, w, t[:300], scale=0.3)
        return (kb.embedding_backward(t, dy, 700), logp,
                *kb.linear_logprobs_backward(x, w, t[:300], stats, logp, scale=0.3))
    say("token operators on two streams")
    want = [run(*j) for j in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    got = []
    for s, j in zip(streams, jobs):
        with torch.cuda.stream(s):
            got.append(run(*j))
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        for p, q in zip(a, b):
            assert torch.equal(p, q)
