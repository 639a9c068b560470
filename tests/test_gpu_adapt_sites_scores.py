"""What the example of many sites says of its answers: likelihoods that its own logits and head give."""
import os
import sys

import pytest
import torch

import score_ref as ref

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))

pytestmark = pytest.mark.gpu


def test_likelihoods_of_the_answers():
    import adapt_sites
    out = adapt_sites.run(sites=4, d=64, C=20, r=4, rows=32, steps=8)
    r = ref.Rows(out["logits"], 1.0)
    top = ref.top(out["logits"], 3)
    assert torch.equal(out["answers"].top_index, top)
    ref.near(out["answers"].top_logp, r.logp.gather(1, top.long()), r.logp_off().gather(1, top.long()))
    # the certified labels' likelihoods: sums of 64 float32 products move a logit by (64 + 3) u sum |w x| at most
    logits = out["z"].double() @ out["W0"].double().t() + out["bias"].double()
    moved = 67 * ref.U * (out["z"].double().abs() @ out["W0"].double().abs().t()).amax(1)
    r = ref.Rows(logits, 1.0)
    assert torch.equal(out["label"].long(), logits.argmax(1))
    ref.near(out["sure"].logp, ref.pick(r.logp, out["label"], 0.0), ref.pick(r.logp_off(), out["label"], 0.0) + 2 * moved)
