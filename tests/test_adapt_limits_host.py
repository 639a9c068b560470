"""Limits and options of the adapter and orthogonalisation entry points, on the host: nothing reaches the device."""
import ctypes
import os

import pytest

from paper_2608_13144_amd import _lib as L

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="liblipcache.so not built")
FAKE = ctypes.c_void_p(0x100000)  # never dereferenced: validation fails first, or there is nothing to do


def _step(batch=0, m=96, n=128, dtype=L.BF16, nesterov=1, steps=5, ws=FAKE, wsb=1 << 40):
    coef = (ctypes.c_float * 96)(*([3.4445, -4.775, 2.0315] * 32))
    opt = L.LipcacheMuon(0.1, 0.9, 0.0, 1.0, 1e-7, nesterov, steps, ctypes.cast(coef, ctypes.POINTER(ctypes.c_float)))
    return L.load().lipcache_muon_step(FAKE, FAKE, FAKE, batch, m, n, dtype, ctypes.byref(opt), ws, wsb, None)


def test_operands_of_a_step():
    for flags in (0, 1, L.MUON_SHORT_OPERANDS, 1 | L.MUON_SHORT_OPERANDS):
        assert _step(nesterov=flags) == L.OK
        assert _step(nesterov=flags, dtype=L.F16) == L.OK
        assert _step(nesterov=flags, dtype=L.F32) == (L.OK if flags < 2 else L.EINVAL), flags
    for flags in (4, 8, -1):
        assert _step(nesterov=flags) == L.EINVAL
    lib = L.load()
    need = lib.lipcache_muon_step_workspace_bytes(2, 96, 128, L.BF16)
    for flags in (1, 1 | L.MUON_SHORT_OPERANDS):
        assert need > 0 and _step(batch=2, nesterov=flags, wsb=need - 1) == L.EWORKSPACE


def test_requests_have_a_limit():
    lib = L.load()
    for requests, expect in ((1 << 30, L.EWORKSPACE), ((1 << 30) + 1, L.EUNSUPPORTED), ((1 << 31) - 1, L.EUNSUPPORTED)):
        ad = L.LipcacheAdapters(FAKE.value, FAKE.value, FAKE.value, FAKE.value, FAKE.value, 3, 8, requests)
        assert lib.lipcache_adapter_forward(FAKE, 64, 10, FAKE, 64, None, 64, 48, ctypes.byref(ad), L.BF16, FAKE, 48, None,
                                            None, 0, None) == expect
        assert lib.lipcache_adapter_backward(FAKE, 48, FAKE, 64, 10, FAKE, 64, 64, 48, ctypes.byref(ad), L.BF16, None, FAKE, 64,
                                             FAKE, FAKE, None, 0, None) == expect
