"""Host checks of the token operators, without a GPU: every invalid argument is rejected with the
documented status before the device is touched (fake addresses, never dereferenced)."""
import math

import pytest

from paper_2609_01956_amd import binding as kb

F32, BF16, BAD, OK = kb.KAN_F32, kb.KAN_BF16, kb.KAN_ERR_INVALID_ARG, kb.KAN_OK
UNSUPPORTED = kb.KAN_ERR_UNSUPPORTED
T, TAB, Y, DY, BASE, DT, WS, X, W, LP, ST, BEST, DL, DX, DW = (0x100000000 * (i + 1)
                                                               for i in range(15))


def test_embedding_host_checks():
    def call(dtype=F32, tdtype=F32, rows=10, classes=50, n=16, t=T, table=TAB, stride=20, scale=1.0,
             y=Y):
        return kb.kan_embedding(dtype, tdtype, rows, classes, n, t, -100, table, stride, scale, y)
    for kw in (dict(rows=-1), dict(rows=(1 << 30) + 1), dict(classes=0), dict(classes=(1 << 30) + 1),
               dict(n=0), dict(n=(1 << 24) + 1), dict(rows=1 << 28, n=1 << 22, stride=1 << 22),
               dict(stride=15), dict(stride=1 << 62), dict(scale=math.nan), dict(scale=math.inf),
               dict(t=0), dict(table=0), dict(y=0), dict(t=T + 4), dict(table=TAB + 2),
               dict(y=Y + 2), dict(y=T), dict(y=TAB + 64), dict(y=T - 16 * 4)):
        assert call(**kw) == BAD, kw
    for kw in (dict(dtype=2), dict(tdtype=-1), dict(tdtype=BF16)):
        assert call(**kw) == UNSUPPORTED, kw
    assert call(rows=0, t=0, table=0, y=0) == OK


def test_embedding_backward_host_checks():
    st, need = kb.kan_embedding_backward_workspace_bytes(10, 50, 16)
    assert st == OK and need > 0

    def call(dtype=F32, tdtype=F32, rows=10, classes=50, n=16, t=T, dy=DY, stride=20, scale=1.0,
             base=BASE, dt=DT, ws=WS, nb=need):
        return kb.kan_embedding_backward(dtype, tdtype, rows, classes, n, t, -100, dy, stride, scale,
                                         base, dt, ws, nb)
    for kw in (dict(rows=-1), dict(rows=(1 << 30) + 1), dict(classes=0), dict(n=0), dict(stride=15),
               dict(stride=1 << 62), dict(scale=math.nan), dict(t=0), dict(dy=0), dict(dt=0),
               dict(ws=0), dict(nb=need - 1), dict(ws=WS + 8), dict(t=T + 4), dict(dy=DY + 2),
               dict(base=BASE + 2), dict(dt=DT + 2), dict(dt=DY), dict(dt=T), dict(dt=BASE + 4),
               dict(ws=DY), dict(ws=T), dict(ws=DT), dict(ws=BASE - 16), dict(base=DT + 4)):
        assert call(**kw) == BAD, kw
    for kw in (dict(dtype=2), dict(tdtype=-1), dict(tdtype=BF16)):
        assert call(**kw) == UNSUPPORTED, kw
    for a in ((-1, 50, 16), (10, 0, 16), (10, 50, 0), ((1 << 30) + 1, 50, 16)):
        assert kb.kan_embedding_backward_workspace_bytes(*a)[0] == BAD
    assert kb.load_library().kan_embedding_backward_workspace_bytes(10, 50, 16, None) == BAD
    # what is kept beside the batch stays in proportion to it
    for rows, classes, n in [(1, 1, 1), (4096, 131072, 1024), (1 << 20, 50001, 4096),
                             (1 << 30, 1 << 30, 1)]:
        st, nb = kb.kan_embedding_backward_workspace_bytes(rows, classes, n)
        assert st == OK and nb <= 9 * classes + 32 * rows + rows * (n + 8) + (1 << 20)


def head(rows=10, classes=50, n=16, x=X, xs=20, w=W, ws=24, dtype=F32):
    return (dtype, rows, classes, n, x, xs, w, ws)


BAD_HEADS = (dict(rows=-1), dict(rows=(1 << 20) + 1), dict(classes=0), dict(classes=(1 << 30) + 1),
             dict(n=0), dict(n=(1 << 20) + 1, xs=1 << 21, ws=1 << 21), dict(xs=15), dict(ws=15),
             dict(xs=1 << 60), dict(ws=1 << 60))


def test_linear_logprobs_host_checks():
    st, need = kb.kan_linear_logprobs_workspace_bytes(*head())
    assert st == OK and need > 0

    def call(scale=1.0, t=T, lp=LP, stats=ST, best=BEST, ws_=WS, nb=need, **kw):
        return kb.kan_linear_logprobs(*head(**kw), scale, t, -100, lp, stats, best, ws_, nb)
    for kw in BAD_HEADS + (dict(scale=math.nan), dict(scale=-math.inf), dict(x=0), dict(w=0),
                           dict(t=0), dict(lp=0), dict(stats=0), dict(ws_=0), dict(nb=need - 1),
                           dict(ws_=WS + 8), dict(x=X + 2), dict(w=W + 2), dict(t=T + 4),
                           dict(best=BEST + 4), dict(lp=X), dict(stats=LP + 4), dict(best=T),
                           dict(ws_=W), dict(ws_=X - 16)):
        assert call(**kw) == BAD, kw
    assert call(dtype=2) == UNSUPPORTED
    assert call(rows=0, x=0, w=0, t=0, lp=0, stats=0, best=0, ws_=0, nb=0) == OK
    for kw in BAD_HEADS:
        assert kb.kan_linear_logprobs_workspace_bytes(*head(**kw))[0] == BAD, kw
        assert kb.kan_linear_logprobs_backward_workspace_bytes(*head(**kw))[0] == BAD, kw
    lib = kb.load_library()
    assert lib.kan_linear_logprobs_workspace_bytes(*head(), None) == BAD
    assert lib.kan_linear_logprobs_backward_workspace_bytes(*head(), None) == BAD


def test_linear_logprobs_backward_host_checks():
    st, need = kb.kan_linear_logprobs_backward_workspace_bytes(*head())
    assert st == OK and need > 0

    def call(scale=1.0, t=T, stats=ST, dl=DL, dx=DX, dw=DW, ws_=WS, nb=need, **kw):
        return kb.kan_linear_logprobs_backward(*head(**kw), scale, t, -100, stats, dl, dx, dw, ws_,
                                               nb)
    for kw in BAD_HEADS + (dict(scale=math.nan), dict(x=0), dict(w=0), dict(t=0), dict(stats=0),
                           dict(dl=0), dict(dx=0, dw=0), dict(ws_=0), dict(nb=need - 1),
                           dict(ws_=WS + 8), dict(dx=X), dict(dw=W), dict(dx=DW + 4), dict(dw=ST),
                           dict(dx=DL), dict(ws_=DX), dict(ws_=W), dict(dx=DX + 2)):
        assert call(**kw) == BAD, kw
    assert call(dtype=-1) == UNSUPPORTED
    # an empty batch that wants dx alone: nothing to do
    assert call(rows=0, x=0, w=0, t=0, stats=0, dl=0, dw=0, ws_=0, nb=0) == OK


def test_head_workspaces_hold_pieces_not_logits():
    """The gradient's workspace does not grow with the vocabulary past its pieces, the forward's
    only by its parts and, where rows have to be copied, a piece of them."""
    for dt, es in ((F32, 4), (BF16, 2)):
        for rows, n in ((8192, 2048), (2001, 1001), (65, 4096)):
            sizes = [kb.kan_linear_logprobs_backward_workspace_bytes(
                *head(rows, V, n, xs=n, ws=n, dtype=dt)) for V in (1 << 17, 1 << 20)]
            assert all(st == OK for st, _ in sizes)
            assert sizes[1][1] <= 6 * (1 << 30)
            st, nb = kb.kan_linear_logprobs_workspace_bytes(
                *head(rows, 1 << 17, n, xs=n, ws=n, dtype=dt))
            assert st == OK and nb < rows * (1 << 17) * es / 4 + (1 << 30)


def test_wrappers_refuse_without_a_gpu():
    torch = pytest.importorskip("torch")
    t = torch.zeros(3, dtype=torch.int64)
    x = torch.zeros(3, 4)
    with pytest.raises(ValueError):
        kb.embedding(t, x)
    with pytest.raises(ValueError):
        kb.embedding_backward(t, x, 5)
    with pytest.raises(ValueError):
        kb.linear_logprobs(x, x, t)
    with pytest.raises(ValueError):
        kb.linear_logprobs_backward(x, x, t, x, x)
