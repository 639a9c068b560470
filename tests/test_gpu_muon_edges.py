"""Orthogonalisation and the momentum step at their edges, against float64."""
import numpy as np
import pytest
import torch

import adapt_ref as R
from gpu_helpers import say
from paper_2608_13144_amd import api
from test_gpu_muon import DEV, NS5, far, matrices, n64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", [(1, 200, 256), (2, 260, 130), (5, 1100, 1030), (1, 2050, 2080), (40, 520, 500), (8, 1030, 1100),
                                   (60, 500, 470)], ids=lambda s: "x".join(map(str, s)))
def test_steps_on_16_bits_lose_only_the_rounding_of_the_result(shape, dtype):
    """W = 0 and a step of the direction itself: it is off by its own rounding and by float32's error alone.

    With ``short_operands`` by what 11-bit operands cost besides (worked out for adapt_ref.NS_TOL)."""
    G = matrices(31, *shape, dtype, "strong")
    ref = -R.newton_schulz(1.5 * n64(G), 5, NS5, 1e-7)
    own = {"f16": 2.0 ** -11, "bf16": 2.0 ** -9}[dtype]  # of the rounding, in the 2-norm
    for short in (False, True):
        say("step on 16 bits", shape, dtype, short)
        W, M = torch.zeros_like(G), torch.zeros(shape, device=DEV)
        api.muon_step(W, G, M, lr=1.0, momentum=0.5, scale=1.0, short_operands=short)
        tol = own + (2.6e-3 if short else R.NS_TOL["f32"])
        assert far(W, ref) <= tol, (shape, dtype, short, far(W, ref))
        assert float(np.max(np.abs(n64(W) - ref)) / np.sqrt(np.mean(ref * ref))) <= 40 * tol
        assert np.array_equal(n64(M), n64(G))
        again = torch.zeros_like(G)
        api.muon_step(again, G, torch.zeros(shape, device=DEV), lr=1.0, momentum=0.5, scale=1.0, short_operands=short)
        assert torch.equal(W, again), "two calls differ"
