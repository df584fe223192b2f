"""Host checks of the operators around the layer, without a GPU: every invalid argument is
rejected with the documented status before the device is touched (fake addresses, never
dereferenced)."""
import math

import pytest

from paper_2609_01956_amd import binding as kb

F32, BF16, BAD, OK = kb.KAN_F32, kb.KAN_BF16, kb.KAN_ERR_INVALID_ARG, kb.KAN_OK
X, R, W, B, H, Y, M, S = (0x100000000 * (i + 1) for i in range(8))
DY, DH, DX, DW, DB, WS = (0x100000000 * (i + 16) for i in range(6))


def test_layer_norm_host_checks():
    def call(dtype=F32, pdtype=F32, rows=16, n=32, x=X, res=R, w=W, b=B, eps=1e-5, h=H, y=Y, m=M,
             s=S):
        return kb.kan_layer_norm(dtype, pdtype, rows, n, x, res, w, b, eps, h, y, m, s)
    for kw in (dict(rows=-1), dict(n=0), dict(n=(1 << 24) + 1), dict(rows=1 << 48), dict(eps=-1e-9),
               dict(eps=math.nan), dict(eps=math.inf), dict(x=0), dict(y=0), dict(res=0),
               dict(m=0), dict(s=0), dict(x=X + 2), dict(w=W + 1), dict(m=M + 2), dict(y=X + 64),
               dict(y=R), dict(y=W - 4), dict(h=X), dict(h=Y + 8), dict(m=Y), dict(s=M + 4),
               dict(m=B + 4)):
        assert call(**kw) == BAD, kw
    for kw in (dict(dtype=2), dict(pdtype=-1), dict(pdtype=BF16)):
        assert call(**kw) == kb.KAN_ERR_UNSUPPORTED, kw
    assert call(dtype=BF16, y=Y + 1) == BAD
    # an empty problem: pointers unchecked, nothing launched
    assert call(rows=0, x=0, res=0, w=0, b=0, h=0, y=0, m=0, s=0) == OK


def test_layer_norm_backward_host_checks():
    st, need = kb.kan_layer_norm_backward_workspace_bytes(F32, 16, 32)
    assert st == OK and need > 0 and need % (2 * 32 * 4) == 0

    def call(dtype=F32, pdtype=F32, rows=16, n=32, h=H, m=M, s=S, w=W, dy=DY, dh=DH, dx=DX, dw=DW,
             db=DB, ws=WS, nb=need):
        return kb.kan_layer_norm_backward(dtype, pdtype, rows, n, h, m, s, w, dy, dh, dx, dw, db,
                                          ws, nb)
    for kw in (dict(rows=-1), dict(n=0), dict(h=0), dict(m=0), dict(s=0), dict(dy=0), dict(dx=0),
               dict(dx=0, dh=0, dw=0, db=0), dict(ws=0), dict(nb=need - 1), dict(ws=WS + 8),
               dict(ws=DX - 16), dict(dx=H), dict(dx=DY + 4), dict(dw=W), dict(db=DW + 4),
               dict(dw=DX), dict(h=H + 2), dict(dw=DW + 2)):
        assert call(**kw) == BAD, kw
    assert call(pdtype=BF16) == kb.KAN_ERR_UNSUPPORTED
    # an empty batch that wants dx alone: nothing to do
    assert call(rows=0, h=0, m=0, s=0, dy=0, dh=0, dw=0, db=0, ws=0, nb=0) == OK
    assert kb.kan_layer_norm_backward_workspace_bytes(F32, -1, 32)[0] == BAD
    assert kb.kan_layer_norm_backward_workspace_bytes(F32, 16, 0)[0] == BAD
    assert kb.kan_layer_norm_backward_workspace_bytes(3, 16, 4)[0] == kb.KAN_ERR_UNSUPPORTED
    assert kb.load_library().kan_layer_norm_backward_workspace_bytes(F32, 16, 32, None) == BAD
    assert kb.kan_layer_norm_backward_workspace_bytes(F32, 0, 32) == (OK, 0)
    for rows, n in [(1, 1), (65536, 784), (16384, 8192), (100, 20000)]:
        for dt in (F32, BF16):
            st, nb = kb.kan_layer_norm_backward_workspace_bytes(dt, rows, n)
            assert st == OK and 8 * n <= nb <= 8 * n * min(rows, 1024)


Z, T, L, ST, E, TL, TI, DZ = (0x100000000 * (i + 32) for i in range(8))


def test_token_logprobs_host_checks():
    st, need = kb.kan_token_logprobs_workspace_bytes(F32, 2, 100000, 5)
    assert st == OK and need > 0  # (few long rows are split)
    assert kb.kan_token_logprobs_workspace_bytes(F32, 65536, 10, 5) == (OK, 0)

    def call(dtype=F32, rows=2, classes=100000, z=Z, stride=100000, t=T, k=5, logp=L, stats=ST,
             ent=E, top=TL, idx=TI, ws=WS, nb=need):
        return kb.kan_token_logprobs(dtype, rows, classes, z, stride, t, -100, k, logp, stats, ent,
                                     top, idx, ws, nb)
    for kw in (dict(rows=-1), dict(classes=0), dict(classes=(1 << 30) + 1), dict(stride=99999),
               dict(stride=1 << 62), dict(k=-1), dict(k=65), dict(classes=4, k=5), dict(z=0),
               dict(t=0), dict(logp=0), dict(stats=0), dict(top=0), dict(idx=0), dict(k=0),
               dict(ws=0), dict(nb=need - 1), dict(ws=WS + 8), dict(z=Z + 2), dict(t=T + 4),
               dict(idx=TI + 4), dict(logp=Z + 4), dict(stats=L + 4), dict(ent=T), dict(ws=Z),
               dict(top=E + 4)):
        assert call(**kw) == BAD, kw
    assert call(dtype=2) == kb.KAN_ERR_UNSUPPORTED
    assert call(rows=0, z=0, t=0, logp=0, stats=0, ent=0, top=0, idx=0, ws=0, nb=0) == OK
    assert kb.kan_token_logprobs_workspace_bytes(F32, 2, 4, 5)[0] == BAD
    assert kb.kan_token_logprobs_workspace_bytes(F32, 2, 100, 65)[0] == BAD
    assert kb.kan_token_logprobs_workspace_bytes(F32, -1, 4, 0)[0] == BAD
    assert kb.kan_token_logprobs_workspace_bytes(7, 1, 4, 0)[0] == kb.KAN_ERR_UNSUPPORTED
    assert kb.load_library().kan_token_logprobs_workspace_bytes(F32, 2, 4, 0, None) == BAD


def test_token_logprobs_backward_host_checks():
    def call(dtype=F32, rows=16, classes=100, z=Z, stride=104, t=T, stats=ST, dl=L, ent=E, de=TL,
             dz=DZ, ds=100):
        return kb.kan_token_logprobs_backward(dtype, rows, classes, z, stride, t, -100, stats, dl,
                                              ent, de, dz, ds)
    for kw in (dict(rows=-1), dict(classes=0), dict(stride=99), dict(ds=99), dict(z=0), dict(t=0),
               dict(stats=0), dict(dl=0), dict(ent=0), dict(de=0), dict(dz=0), dict(dz=DZ + 2),
               dict(dz=Z), dict(dz=Z + 4, ds=104), dict(dz=T), dict(dz=ST - 4), dict(dz=E)):
        assert call(**kw) == BAD, kw
    assert call(dtype=-1) == kb.KAN_ERR_UNSUPPORTED
    assert call(rows=0, z=0, t=0, stats=0, dl=0, ent=0, de=0, dz=0) == OK


G0, G1, O0, O1, NM = (0x100000000 * (i + 48) for i in range(5))


def test_clip_grad_norm_host_checks():
    st, need = kb.kan_grad_norm_workspace_bytes(2)
    assert st == OK and need > 0

    def call(g=(G0, G1), n=(100, 7), d=(F32, BF16), mx=1.0, eps=1e-6, o=(O0, O1), ws=WS, nb=need,
             nm=NM):
        return kb.kan_clip_grad_norm(g, n, d, mx, eps, o, ws, nb, nm)
    for kw in (dict(g=(0, G1)), dict(o=(0, O1)), dict(n=(-1, 7)), dict(n=(1 << 40, 1)),
               dict(mx=-1.0), dict(mx=math.nan), dict(eps=-1.0), dict(eps=math.inf), dict(o=None),
               dict(ws=0), dict(ws=WS + 8), dict(nb=need - 1), dict(nm=0), dict(nm=NM + 2),
               dict(nm=WS + 4), dict(nm=G0 + 4), dict(nm=O1), dict(ws=G1), dict(ws=O0),
               dict(g=(G0 + 2, G1)), dict(g=(G0, G1 + 1)), dict(o=(O0, O1 + 1)),
               dict(o=(G0 + 4, O1)), dict(o=(G1, O1)), dict(o=(O0, O0)), dict(o=(O0, O0 + 396)),
               dict(o=(O0, G0)), dict(g=(G0, G0), d=(F32, F32), o=(G0, G0)),
               dict(g=(G0, G0 + 396), d=(F32, F32), o=(G0, G0 + 396))):
        assert call(**kw) == BAD, kw
    assert call(d=(F32, 2)) == kb.KAN_ERR_UNSUPPORTED
    def norm(g=(G0, G1), n=(100, 7), d=(F32, BF16), ws=WS, nb=need, nm=NM):
        return kb.kan_grad_norm(g, n, d, ws, nb, nm)
    for kw in (dict(g=(0, G1)), dict(n=(100, -7)), dict(ws=0), dict(nb=need - 1), dict(nm=0),
               dict(nm=G1), dict(ws=G0 - 16)):
        assert norm(**kw) == BAD, kw
    assert norm(d=(-1, F32)) == kb.KAN_ERR_UNSUPPORTED
    assert kb.kan_grad_norm_workspace_bytes(-1)[0] == BAD
    assert kb.kan_grad_norm_workspace_bytes(16385)[0] == BAD
    assert kb.load_library().kan_grad_norm_workspace_bytes(1, None) == BAD


def test_clip_outputs_of_many_tensors():
    """The overlap check over thousands of tensors in any order (no device: an invalid dtype
    is found first, an overlap last, so both orders of 5000 end in the code asked for)."""
    count = 5000
    st, need = kb.kan_grad_norm_workspace_bytes(count)
    order = [(i * 1237) % count for i in range(count)]
    g = [G0 + 64 * i for i in order]
    bad = g[:-1] + [g[0] + 4]
    assert kb.kan_clip_grad_norm(bad, [16] * count, [F32] * count, 1.0, 1e-6, bad, WS, need,
                                 NM) == BAD
