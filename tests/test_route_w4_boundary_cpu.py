"""The router's and the 4-bit weights' entry points refuse bad arguments on the host, before anything touches a GPU."""
import ctypes

import numpy as np
import pytest

from paper_2511_21089_amd import binding as mm

vp = ctypes.c_void_p
P = vp(0x1000)


def topk(f, logits=P, ld=8, act=None, tok=None, T=4, B=8, k=2, elem=2, route=P, probs=P, counts=P, loss=P, tail=(None,)):
    return f(logits, ld, act, tok, T, B, k, elem, route, probs, counts, loss, *tail)


def test_route_topk_refusals():
    f, g = mm.lib.mlpmoe_route_topk, mm.lib.mlpmoe_route_topk_ws
    for call in (lambda **kw: topk(f, **kw), lambda **kw: topk(g, tail=(P, 1 << 20, None), **kw)):
        for kw in (dict(B=0), dict(B=65, ld=65), dict(T=-1), dict(T=(1 << 24) + 1), dict(k=0), dict(k=9), dict(ld=7)):
            assert call(**kw) == mm.ERR_SHAPE, kw
        for elem in (1, 3, 8):
            assert call(elem=elem) == mm.ERR_UNSUPPORTED
        assert call(logits=None) == mm.ERR_NULL and call(route=None) == mm.ERR_NULL
        assert call(logits=vp(0x1001)) == mm.ERR_ALIGN and call(logits=vp(0x1002), elem=4) == mm.ERR_ALIGN
        assert call(probs=vp(0x1002)) == mm.ERR_ALIGN and call(counts=vp(0x1002)) == mm.ERR_ALIGN
        assert call(loss=vp(0x1001)) == mm.ERR_ALIGN
        # no token and no sums asked for: nothing to do
        assert call(T=0, logits=None, route=None, probs=None, counts=None, loss=None) == mm.OK
    need = mm.mlpmoe_route_workspace_bytes(1 << 20, 8)
    assert need >= 2 * 4 * 9
    for ws, n in ((None, need), (P, need - 1), (vp(0x1010), need)):
        assert topk(g, T=1 << 20, tail=(ws, n, None)) == mm.ERR_WORKSPACE


def test_route_workspace_bytes():
    f = mm.mlpmoe_route_workspace_bytes
    assert f(-1, 8) == 0 and f(4, 0) == 0 and f(4, 65) == 0 and f((1 << 24) + 1, 8) == 0
    assert 0 < f(0, 1) <= f(1 << 24, 64) <= 1 << 20


def test_route_backward_refusals():
    def call(probs=P, counts=P, dp=P, dl=P, act=None, T=4, B=8, elem=2, out=P):
        return mm.lib.mlpmoe_route_backward(probs, counts, dp, dl, act, T, B, elem, out, None)

    for kw in (dict(B=0), dict(B=65), dict(T=-1), dict(T=(1 << 24) + 1)):
        assert call(**kw) == mm.ERR_SHAPE, kw
    assert call(elem=1) == mm.ERR_UNSUPPORTED
    assert call(probs=None) == mm.ERR_NULL and call(out=None) == mm.ERR_NULL and call(counts=None) == mm.ERR_NULL
    for kw in (dict(probs=vp(0x1002)), dict(dp=vp(0x1002)), dict(dl=vp(0x1002)), dict(counts=vp(0x1002)), dict(out=vp(0x1001)),
               dict(out=vp(0x1002), elem=4)):
        assert call(**kw) == mm.ERR_ALIGN, kw
    assert call(T=0, probs=None, out=None) == mm.OK


@pytest.mark.parametrize("name", ["mlpmoe_w4_quantize", "mlpmoe_w4_dequantize"])
def test_conversion_refusals(name):
    f = getattr(mm.lib, name)

    def call(a=P, b=P, c=P, rows=4, cols=64, elem=2):
        return f(a, rows, cols, elem, b, c, None) if name.endswith("_quantize") else f(a, b, rows, cols, elem, c, None)

    if name.endswith("_quantize"):
        assert f is mm.lib.mlpmoe_w4_quantize
    for kw in (dict(rows=-1), dict(cols=0), dict(rows=(1 << 22) + 1), dict(cols=(1 << 22) + 32), dict(rows=1 << 22, cols=1 << 22)):
        assert call(**kw) == mm.ERR_SHAPE, kw
    for kw in (dict(elem=1), dict(cols=48), dict(cols=31)):
        assert call(**kw) == mm.ERR_UNSUPPORTED, kw
    for which in "abc":
        assert call(**{which: None}) == mm.ERR_NULL
        assert call(**{which: vp(0x1008)}) == mm.ERR_ALIGN
    assert call(a=None, b=None, c=None, rows=0) == mm.OK


def test_forward_w4_refusals():
    off = np.array([0, 60, 128], np.int32)
    al, mk = np.ones(2, np.float32), np.ones(2, np.uint8)
    f, g = mm.lib.mlpmoe_forward_w4, mm.lib.mlpmoe_forward_w4_ws

    def call(x=P, w=(P,) * 6, offs=off, alpha=al, mask=mk, route=None, T=4, d_model=64, d_inter=128, B=2, ob=2, out=P, ws=None):
        a = [x, *w, offs.ctypes.data, None if alpha is None else alpha.ctypes.data, mask.ctypes.data, route, T, d_model, d_inter, B, ob, out]
        return f(*a, None) if ws is None else g(*a, *ws, None)

    for kw in (dict(B=0), dict(B=65), dict(T=-1), dict(d_model=0), dict(T=65535 * 16 + 1)):
        assert call(**kw) == mm.ERR_SHAPE, kw
    assert call(d_inter=96) == mm.ERR_OFFSETS and call(offs=np.array([0, 130, 128], np.int32)) == mm.ERR_OFFSETS
    for kw in (dict(ob=3), dict(d_model=48), dict(offs=np.array([0, 60, 120], np.int32), d_inter=120)):
        assert call(**kw) == mm.ERR_UNSUPPORTED, kw
    assert call(x=None) == mm.ERR_NULL and call(out=None) == mm.ERR_NULL and call(alpha=None) == mm.ERR_NULL
    for i in range(6):
        w = [P] * 6
        w[i] = None
        assert call(w=w) == mm.ERR_NULL, i
        w[i] = vp(0x1004)
        assert call(w=w) == mm.ERR_ALIGN, i
    assert call(x=vp(0x1008)) == mm.ERR_ALIGN and call(out=vp(0x1008)) == mm.ERR_ALIGN
    need = mm.mlpmoe_w4_workspace_bytes(4, 64, 128, 2)
    for ws in ((None, need), (P, need - 1), (vp(0x1010), need)):
        assert call(ws=ws) == mm.ERR_WORKSPACE
    assert call(T=0, x=None, out=None) == mm.OK and call(T=0, ws=(None, 0)) == mm.OK


def test_w4_workspace_bytes():
    f = mm.mlpmoe_w4_workspace_bytes
    assert f(-1, 64, 128, 2) == 0 and f(1, 0, 128, 2) == 0 and f(1, 64, -1, 2) == 0 and f(1, 64, 128, 65) == 0
    assert f(0, 64, 128, 2) > 0 and f(16, 4096, 14336, 16) >= 16 * 14336 * 2


@pytest.mark.parametrize("d_model,d_inter", [(4096, 14336), (896, 4864), (64, 32), (32, 131072), (131072, 1024)])
def test_a_workspace_for_more_tokens_serves_fewer(d_model, d_inter):
    tokens = [*range(200), 255, 256, 257, 500, 1000, 1600, 4000, 100000, 65535 * 16]
    sizes = [mm.mlpmoe_w4_workspace_bytes(T, d_model, d_inter, 8) for T in tokens]
    assert sizes == sorted(sizes)
    for B in (1, 5, 64):
        sizes = [mm.mlpmoe_route_workspace_bytes(T, B) for T in [*tokens, 1 << 24]]
        assert sizes == sorted(sizes)


def test_forward_w4_refuses_longer_rows():
    f = mm.lib.mlpmoe_forward_w4
    al, mk = np.ones(1, np.float32), np.ones(1, np.uint8)
    for d_model, d_inter in ((131072 + 32, 64), (64, 131072 + 32)):
        off = np.array([0, d_inter], np.int32)
        assert f(P, P, P, P, P, P, P, off.ctypes.data, al.ctypes.data, mk.ctypes.data, None, 1, d_model, d_inter, 1, 2, P,
                 None) == mm.ERR_UNSUPPORTED


def test_binding_refuses_what_is_not_on_the_gpu_or_has_another_form():
    torch = pytest.importorskip("torch")
    cpu = torch.zeros((4, 8))
    with pytest.raises(ValueError):
        mm.mlpmoe_route_topk(cpu, 2)
    with pytest.raises(ValueError):
        mm.mlpmoe_route_topk(cpu.double(), 2)
    with pytest.raises(ValueError):
        mm.mlpmoe_route_topk(cpu[0], 2)
    with pytest.raises(ValueError):
        mm.mlpmoe_route_backward(cpu.double(), None)
    with pytest.raises(ValueError):
        mm.mlpmoe_route_backward(cpu, torch.zeros(8, dtype=torch.int32))
    with pytest.raises(ValueError):
        mm.mlpmoe_w4_quantize(torch.zeros((4, 32), dtype=torch.float16))
    with pytest.raises(ValueError):
        mm.mlpmoe_w4_dequantize(torch.zeros((4, 16), dtype=torch.uint8), torch.zeros((4, 2), dtype=torch.uint8))
