"""The example that trains, serves and certifies with the adapters, at a small size."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))

pytestmark = pytest.mark.gpu


def test_adapt_sites():
    import adapt_sites
    out = adapt_sites.run(sites=5, d=96, C=30, r=4, rows=40, steps=40)
    assert out["last"] < 0.7 * out["first"], (out["first"], out["last"])
    # the single queries' logits are each site's own head's: sums of d + r float32 products of numbers of order 10
    for s in range(5):
        Ws = out["W"].double() + float(out["scale"][s]) * out["B"][s].double() @ out["A"][s].double()
        ref = Ws @ out["queries"][s].double()
        size = Ws.abs() @ out["queries"][s].double().abs()
        assert bool(((out["logits"][s].double() - ref).abs() <= 2.0 ** -24 * (96 + 4 + 16) * size).all())
    assert out["hits"] == out["agree"] == out["certified"] > 0
    assert out["moved"] <= out["bound"] + 1e-4
    assert torch.isfinite(out["A"]).all() and torch.isfinite(out["B"]).all()
