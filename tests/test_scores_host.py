"""How the scoring and distillation calls take their arguments, on the host."""
import os

import pytest
import torch

from paper_2608_13144_amd import _lib as L
from paper_2608_13144_amd import api

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="liblipcache.so not built")
CALLS = [("logprobs", "logits", {}), ("logprobs_backward", "logits", {}), ("distill", "logits", dict(teacher=None, index=None)),
         ("head_logprobs", "x", dict(W=torch.zeros(3, 8), bias=None))]


@pytest.mark.parametrize("name,first,more", CALLS)
def test_every_argument_by_name(name, first, more):
    with pytest.raises(ValueError, match=f"{first} must be a device tensor"):
        getattr(api, name)(**{first: torch.zeros(3, 8)}, **more)


@pytest.mark.parametrize("name,first,more", CALLS)
def test_a_call_without_its_first_argument_names_it(name, first, more):
    with pytest.raises(TypeError, match=rf"{name}\(\) missing 1 required positional argument: '{first}'"):
        getattr(api, name)(**more)


def test_no_rows_need_no_workspace():
    """T = 0 does nothing, whatever the operands' alignment, with as much workspace as the query says: none."""
    lib, some = L.load(), 0x100000
    for ldw, K in ((64, 64), (62, 62), (1, 1)):
        assert lib.lipcache_head_logprobs_workspace_bytes(some, 64, 0, some, ldw, K, 48, L.BF16) == 0, (ldw, K)
        assert lib.lipcache_head_logprobs(some, 64, 0, some, ldw, None, K, 48, L.BF16, 1.0, None, None, None, None, None, 0,
                                          None) == L.OK, (ldw, K)
    assert lib.lipcache_head_logprobs(some, 64, 1, some, 64, None, 64, 48, L.BF16, 1.0, None, None, None, None, None, 0,
                                      None) == L.EWORKSPACE
    assert lib.lipcache_head_logprobs(some, 63, 0, some, 64, None, 64, 48, L.BF16, 1.0, None, None, None, None, None, 0,
                                      None) == L.EINVAL
