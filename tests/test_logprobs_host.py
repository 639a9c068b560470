"""Validation of the scoring and distillation entry points on the host: nothing reaches the device."""
import ctypes
import os

import pytest
import torch

from paper_2608_13144_amd import _lib as L
from paper_2608_13144_amd import api

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="liblipcache.so not built")
FAKE = ctypes.c_void_p(0x100000)  # never dereferenced: validation fails first
ODD, HALF = ctypes.c_void_p(0x100001), ctypes.c_void_p(0x100002)
NAN, INF = float("nan"), float("inf")


def test_logprobs_validation():
    lib = L.load()
    base = dict(x=FAKE, ldx=64, T=10, C=64, dtype=L.BF16, t=1.0, label=FAKE, k=4, logp=FAKE, lse=FAKE, ent=FAKE, at=FAKE,
                top=FAKE, ws=None, wsb=0)

    def call(**over):
        return lib.lipcache_logprobs(*dict(base, **over).values(), None)
    for bad in (dict(T=-1), dict(C=0), dict(C=-3), dict(ldx=63), dict(dtype=3), dict(dtype=-1), dict(x=None), dict(x=ODD),
                dict(dtype=L.F32, x=HALF), dict(t=0.0), dict(t=-1.0), dict(t=NAN), dict(t=INF), dict(t=1e-9), dict(k=-1),
                dict(at=None), dict(top=None), dict(label=HALF), dict(logp=HALF), dict(lse=HALF), dict(ent=HALF),
                dict(at=HALF), dict(top=HALF)):
        assert call(**bad) == L.EINVAL, bad
    assert call(k=65) == L.EUNSUPPORTED and call(T=1 << 31) == L.EUNSUPPORTED
    assert call(C=(1 << 20) + 1, ldx=1 << 21) == L.EUNSUPPORTED
    assert call(T=0, x=None, at=None, top=None) == L.OK


def test_logprobs_backward_validation():
    lib = L.load()
    base = dict(x=FAKE, ldx=64, T=10, C=64, dtype=L.F16, t=1.0, label=FAKE, gl=FAKE, gs=FAKE, ge=FAKE, k=4, at=FAKE, gt=FAKE,
                dx=FAKE, ldd=64, ws=None, wsb=0)

    def call(**over):
        return lib.lipcache_logprobs_backward(*dict(base, **over).values(), None)
    for bad in (dict(T=-1), dict(C=0), dict(ldx=63), dict(ldd=63), dict(dtype=9), dict(x=None), dict(dx=None), dict(dx=ODD),
                dict(t=0.0), dict(t=NAN), dict(k=-1), dict(at=None), dict(gt=None), dict(label=None), dict(gl=HALF),
                dict(gs=HALF), dict(ge=HALF), dict(at=HALF), dict(gt=HALF), dict(label=HALF)):
        assert call(**bad) == L.EINVAL, bad
    assert call(k=1025) == L.EUNSUPPORTED and call(T=1 << 31) == L.EUNSUPPORTED
    assert call(C=(1 << 20) + 1, ldx=1 << 21, ldd=1 << 21) == L.EUNSUPPORTED
    assert call(T=0, x=None, dx=None) == L.OK


def test_distill_validation():
    lib = L.load()
    base = dict(x=FAKE, ldx=64, T=10, C=64, dtype=L.F32, t=2.0, hard=0.5, soft=1.0, k=4, teacher=FAKE, index=FAKE, label=FAKE,
                weight=FAKE, ce=FAKE, kl=FAKE, dx=FAKE, ldd=64, ws=None, wsb=0)

    def call(**over):
        return lib.lipcache_distill(*dict(base, **over).values(), None)
    for bad in (dict(T=-1), dict(C=0), dict(ldx=63), dict(ldd=63), dict(dtype=4), dict(x=None), dict(x=HALF), dict(dx=HALF),
                dict(t=0.0), dict(t=INF), dict(hard=NAN), dict(soft=INF), dict(k=-1), dict(teacher=None), dict(index=None),
                dict(teacher=HALF), dict(index=HALF), dict(label=HALF), dict(weight=HALF), dict(ce=HALF), dict(kl=HALF)):
        assert call(**bad) == L.EINVAL, bad
    assert call(k=1025) == L.EUNSUPPORTED and call(T=1 << 31) == L.EUNSUPPORTED
    assert call(T=0, x=None, dx=None, teacher=None, index=None) == L.OK


def test_few_rows_of_many_classes_need_a_workspace():
    lib = L.load()
    C = 1 << 17
    for name, k in (("logprobs", 4), ("logprobs_backward", 4), ("distill", 4)):
        bytes_of = getattr(lib, f"lipcache_{name}_workspace_bytes")
        assert bytes_of(3, C, k, L.BF16) > 0 and bytes_of(L.FEW_ROWS, C, k, L.BF16) > 0
        assert bytes_of(L.FEW_ROWS + 1, C, k, L.BF16) == 0 and bytes_of(3, 1000, k, L.BF16) == 0 and bytes_of(0, C, k, L.BF16) == 0
        assert bytes_of(-1, C, k, L.BF16) == 0 and bytes_of(3, 0, k, L.BF16) == 0 and bytes_of(3, C, k, 9) == 0

    def calls(ws, size):
        yield lib.lipcache_logprobs(FAKE, C, 3, C, L.BF16, 1.0, FAKE, 4, FAKE, FAKE, FAKE, FAKE, FAKE, ws, size, None)
        yield lib.lipcache_logprobs_backward(FAKE, C, 3, C, L.BF16, 1.0, FAKE, FAKE, FAKE, FAKE, 4, FAKE, FAKE, FAKE, C, ws,
                                             size, None)
        yield lib.lipcache_distill(FAKE, C, 3, C, L.BF16, 2.0, 0.5, 1.0, 4, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, C, ws,
                                   size, None)
    for ws, size in ((None, 0), (FAKE, 64), (ctypes.c_void_p(0x100040), 1 << 20)):
        assert list(calls(ws, size)) == [L.EWORKSPACE] * 3, (ws, size)


def test_head_logprobs_validation():
    lib = L.load()
    base = dict(x=FAKE, ldx=64, T=10, W=FAKE, ldw=64, bias=FAKE, K=64, C=48, dtype=L.BF16, t=1.0, label=FAKE, logp=FAKE, lse=FAKE,
                ent=FAKE, ws=FAKE, wsb=1 << 30)

    def call(**over):
        return lib.lipcache_head_logprobs(*dict(base, **over).values(), None)
    for bad in (dict(T=-1), dict(K=0), dict(C=0), dict(ldx=63), dict(ldw=63), dict(dtype=3), dict(x=None), dict(W=None),
                dict(x=ODD), dict(W=ODD), dict(bias=HALF), dict(label=HALF), dict(logp=HALF), dict(lse=HALF), dict(ent=HALF),
                dict(t=0.0), dict(t=NAN)):
        assert call(**bad) == L.EINVAL, bad
    assert call(T=1 << 31) == L.EUNSUPPORTED
    assert call(K=(1 << 20) + 1, ldx=1 << 21, ldw=1 << 21) == L.EUNSUPPORTED
    assert call(C=(1 << 20) + 1) == L.EUNSUPPORTED
    assert call(ws=None) == L.EWORKSPACE and call(ws=ctypes.c_void_p(0x100040)) == L.EWORKSPACE
    bytes_of = lib.lipcache_head_logprobs_workspace_bytes
    need = bytes_of(FAKE, 64, 10, FAKE, 64, 64, 48, L.BF16)
    assert need > 0 and call(wsb=need - 1) == L.EWORKSPACE
    assert bytes_of(FAKE, 64, 10, FAKE, 64, 0, 48, L.BF16) == 0
    # room for a copy of each matrix whose rows are not whole vectors, and for no other
    copies = [bytes_of(FAKE, 64, 10, FAKE, 68, 64, 48, L.BF16), bytes_of(ctypes.c_void_p(0x100002), 64, 10, FAKE, 64, 64, 48, L.BF16),
              bytes_of(FAKE, 64, 10, FAKE, 64, 62, 48, L.BF16)]
    assert copies[0] >= need + 48 * 64 * 2 and copies[1] >= need + 10 * 64 * 2 and copies[2] >= need + 58 * 64 * 2
    assert call(ldw=68, wsb=copies[0] - 1) == L.EWORKSPACE
    assert call(T=0, x=None) == L.OK


def test_the_binding_refuses_host_tensors():
    x = torch.zeros(3, 8)
    for call in (lambda: api.logprobs(x), lambda: api.logprobs_backward(x), lambda: api.distill(x, None, None),
                 lambda: api.head_logprobs(x, x, None)):
        with pytest.raises(ValueError, match="device tensor"):
            call()
