"""Workspaces and outputs that a wrapper must not write through."""
import pytest

from paper_2609_01956_amd import binding as kb
from gpu_common import device, say, torch

pytestmark = pytest.mark.gpu


def test_expanded_workspaces_are_left_alone():
    """One byte that counts as many: each call takes a workspace of its own, with the same
    results, and the byte and its neighbours stay."""
    g = torch.Generator(device=device())
    g.manual_seed(1)
    r = lambda *s: torch.randn(*s, device=device(), generator=g)
    buf = torch.full((1 << 16,), 77, dtype=torch.uint8, device=device())
    ws = buf[4096:4097].expand(1 << 28)
    x, dy, coef, base = r(40, 24), r(40, 12), r(12, 24, 8), r(12, 24)
    h, dh, z = r(3000, 300), r(3000, 300), r(2, 90000)
    t = torch.zeros(2, dtype=torch.int64, device=device())
    m, s = h.mean(1), r(3000).abs()
    grads = [r(100), r(30)]
    packed = kb.pack_layer(coef, base, 5)
    calls = {
        "layer_forward_packed": lambda **k: [kb.layer_forward_packed(x, packed, **k)],
        "layer_forward_span": lambda **k: [kb.layer_forward_span(x, coef, base, 5, **k)],
        "layer_backward": lambda **k: kb.layer_backward(x, coef, base, dy, 5, **k),
        "layer_norm_backward": lambda **k: kb.layer_norm_backward(h, m, s, None, dh, **k),
        "token_logprobs": lambda **k: kb.token_logprobs(z, t, top_k=3, entropy=True, **k),
        "grad_norm": lambda **k: [kb.grad_norm(grads, **k)],
        "clip_grad_norm": lambda **k: [kb.clip_grad_norm(grads, 1e9, **k)],
    }
    for name, call in calls.items():
        say(f"{name} with an expanded workspace")
        for a, b in zip(call(), call(workspace=ws)):
            assert torch.equal(a, b), name
        assert bool((buf == 77).all()), name


def test_span_forward_refuses_outputs_that_do_not_fit():
    x, coef, base = (torch.zeros(*s, device=device()) for s in ((40, 24), (12, 24, 8), (12, 24)))
    out = torch.zeros(40, 12, device=device())
    say("layer_forward_span outputs")
    assert kb.layer_forward_span(x, coef, base, 5, out=out) is out
    for bad in (out[:20], out.t(), out.to(torch.bfloat16), out.cpu(),
                torch.zeros(80, 12, device=device())[::2]):
        with pytest.raises(ValueError):
            kb.layer_forward_span(x, coef, base, 5, out=bad)


def test_gradients_refuse_missing_statistics():
    """A forward without statistics (need_stats=False) returns None for them."""
    x = torch.randn(4, 16, device=device())
    _, _, mean, rstd = kb.layer_norm(x)
    t = torch.zeros(4, dtype=torch.int64, device=device())
    for f in (lambda: kb.layer_norm_backward(x, None, None, None, x),
              lambda: kb.layer_norm_backward(x, mean, None, None, x),
              lambda: kb.layer_norm_backward(x, None, rstd, None, x),
              lambda: kb.token_logprobs_backward(x, t, None, mean)):
        with pytest.raises(ValueError):
            f()
