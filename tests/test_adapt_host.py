"""Validation of the adapter and orthogonalisation entry points on the host: nothing reaches the device."""
import ctypes
import os

import pytest

from paper_2608_13144_amd import _lib as L

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="liblipcache.so not built")
FAKE = ctypes.c_void_p(0x100000)  # never dereferenced: validation fails first


def _ad(**kw):
    a = L.LipcacheAdapters(FAKE.value, FAKE.value, FAKE.value, FAKE.value, FAKE.value, 3, 8, 4)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def test_adapter_forward_validation():
    lib = L.load()
    base = dict(x=FAKE, ldx=64, T=10, W=FAKE, ldw=64, bias=FAKE, K=64, N=48, ad=_ad(), dtype=L.BF16, y=FAKE, ldy=48,
                v=None, ws=FAKE, wsb=1 << 30)

    def call(**over):
        a = dict(base, **over)
        ad = None if a["ad"] is None else ctypes.byref(a["ad"])
        return lib.lipcache_adapter_forward(a["x"], a["ldx"], a["T"], a["W"], a["ldw"], a["bias"], a["K"], a["N"], ad,
                                            a["dtype"], a["y"], a["ldy"], a["v"], a["ws"], a["wsb"], None)
    assert call(ad=None) == L.EINVAL
    for bad in (dict(T=-1), dict(K=0), dict(N=0), dict(dtype=3), dict(dtype=-1), dict(ldx=63), dict(ldw=63), dict(ldy=47),
                dict(x=None), dict(W=None), dict(y=None), dict(x=ctypes.c_void_p(0x100001)),
                dict(bias=ctypes.c_void_p(0x100002)), dict(v=ctypes.c_void_p(0x100002)),
                dict(dtype=L.F32, x=ctypes.c_void_p(0x100002))):
        assert call(**bad) == L.EINVAL, bad
    for bad in (dict(S=-1), dict(R=-1), dict(r=0), dict(A=None), dict(B=None), dict(scale=None), dict(offsets=None),
                dict(adapter=None), dict(A=0x100001), dict(offsets=0x100002)):
        assert call(ad=_ad(**bad)) == L.EINVAL, bad
    for bad in (dict(r=129), dict(S=65536)):
        assert call(ad=_ad(**bad)) == L.EUNSUPPORTED, bad
    assert call(T=1 << 31) == L.EUNSUPPORTED
    assert call(K=(1 << 20) + 1, ldx=1 << 21, ldw=1 << 21) == L.EUNSUPPORTED
    assert call(ws=None) == L.EWORKSPACE
    assert call(ws=ctypes.c_void_p(0x100040)) == L.EWORKSPACE
    need = lib.lipcache_adapter_forward_workspace_bytes(10, 64, 48, 8, 3, L.BF16)
    assert need > 0 and call(wsb=need - 1) == L.EWORKSPACE
    assert call(T=0, x=None, y=None) == L.OK
    assert call(T=0, ad=_ad(S=0, A=None, B=None, scale=None)) == L.OK


def test_adapter_backward_validation():
    lib = L.load()
    base = dict(dy=FAKE, lddy=48, x=FAKE, ldx=64, T=10, W=FAKE, ldw=64, K=64, N=48, ad=_ad(), dtype=L.F16, v=None,
                dx=FAKE, lddx=64, dA=FAKE, dB=FAKE, ws=FAKE, wsb=1 << 30)

    def call(**over):
        a = dict(base, **over)
        return lib.lipcache_adapter_backward(a["dy"], a["lddy"], a["x"], a["ldx"], a["T"], a["W"], a["ldw"], a["K"],
                                             a["N"], ctypes.byref(a["ad"]), a["dtype"], a["v"], a["dx"], a["lddx"],
                                             a["dA"], a["dB"], a["ws"], a["wsb"], None)
    for bad in (dict(T=-1), dict(K=0), dict(N=0), dict(dtype=7), dict(lddy=47), dict(ldx=63), dict(ldw=63),
                dict(lddx=63), dict(dy=None), dict(x=None), dict(W=None), dict(dA=None), dict(dB=None),
                dict(dx=ctypes.c_void_p(0x100001)), dict(v=ctypes.c_void_p(0x100002)), dict(ad=_ad(r=0)),
                dict(ad=_ad(A=None))):
        assert call(**bad) == L.EINVAL, bad
    assert call(ad=_ad(r=200)) == L.EUNSUPPORTED
    assert call(ws=None) == L.EWORKSPACE
    need = lib.lipcache_adapter_backward_workspace_bytes(10, 64, 48, 8, 3, L.F16)
    assert need > 0 and call(wsb=need - 1) == L.EWORKSPACE


def test_orthogonalise_and_step_validation():
    lib = L.load()
    coef = (ctypes.c_float * 15)(*([3.4445, -4.775, 2.0315] * 5))

    def ortho(G=FAKE, batch=2, m=64, n=96, dtype=L.F32, steps=5, coef=coef, eps=1e-7, out=FAKE, ws=FAKE, wsb=1 << 30):
        return lib.lipcache_orthogonalise(G, batch, m, n, dtype, steps, coef, eps, out, ws, wsb, None)

    def step(W=FAKE, G=FAKE, M=FAKE, batch=2, m=64, n=96, dtype=L.BF16, ws=FAKE, wsb=1 << 30, opt=True, **kw):
        o = L.LipcacheMuon(0.1, 0.9, 0.0, 1.0, 1e-7, 1, 5, ctypes.cast(coef, ctypes.POINTER(ctypes.c_float)))
        for k, v in kw.items():
            setattr(o, k, v)
        return lib.lipcache_muon_step(W, G, M, batch, m, n, dtype, ctypes.byref(o) if opt else None, ws, wsb, None)
    for bad in (dict(batch=-1), dict(m=0), dict(n=0), dict(dtype=3), dict(steps=-1), dict(steps=33), dict(eps=-1.0),
                dict(eps=float("nan")), dict(eps=float("inf")), dict(coef=None), dict(G=None), dict(out=None),
                dict(G=ctypes.c_void_p(0x100002))):
        assert ortho(**bad) == L.EINVAL, bad
    for bad in (dict(batch=65536), dict(m=16385, n=16385), dict(m=1, n=(1 << 30) + 1)):
        assert ortho(**bad) == L.EUNSUPPORTED, bad
    for rows in ([30.0, 5.0, 5.0], [3.4445, -4.775, 2.0315] * 4 + [20.0, 0.0, 0.0]):
        c = (ctypes.c_float * len(rows))(*rows)
        assert ortho(steps=len(rows) // 3, coef=c) == L.EUNSUPPORTED
    nan = (ctypes.c_float * 3)(1.0, float("nan"), 0.0)
    assert ortho(steps=1, coef=nan) == L.EINVAL
    assert ortho(ws=None) == L.EWORKSPACE
    need = lib.lipcache_orthogonalise_workspace_bytes(2, 64, 96, L.F32)
    assert need > 0 and ortho(wsb=need - 1) == L.EWORKSPACE
    assert ortho(batch=0, G=None, out=None) == L.OK
    assert step(opt=False) == L.EINVAL
    for bad in (dict(W=None), dict(G=None), dict(M=None), dict(M=ctypes.c_void_p(0x100002)), dict(lr=float("nan")),
                dict(momentum=float("inf")), dict(weight_decay=float("nan")), dict(scale=float("inf")), dict(steps=40),
                dict(eps=-1.0)):
        assert step(**bad) == L.EINVAL, bad
    assert step(m=20000, n=20000) == L.EUNSUPPORTED
    need = lib.lipcache_muon_step_workspace_bytes(2, 64, 96, L.BF16)
    assert need > 0 and step(wsb=need - 1) == L.EWORKSPACE
    assert step(batch=0) == L.OK
