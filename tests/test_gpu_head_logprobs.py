"""Log probabilities straight from features and a head against float64."""
import math

import pytest
import torch

import score_ref as ref
from test_gpu_logprobs import BF16, DEV, F16, F32, INF, _labels

pytestmark = pytest.mark.gpu


def _api():
    from paper_2608_13144_amd import api
    return api


def _case(T, K, C, dtype, seed, strided=False):
    g = torch.Generator(device=DEV).manual_seed(seed)
    more = 19 if strided else 0
    x = torch.randn(T, K + more, generator=g, device=DEV).to(dtype)[:, more:]
    W = (3.0 * torch.randn(C, K + 2 * more, generator=g, device=DEV) / math.sqrt(K)).to(dtype)[:, 2 * more:]
    return x, W, torch.randn(C, generator=g, device=DEV), _labels(T, C, g)


def _check(x, W, bias, y, t, out):
    """The scores' bounds, and what float32 sums of K products move them by: a logit by at most (K + 3) u sum |w x|, a
    log probability by twice the largest of a row, an entropy by that times the spread of the logits."""
    logits = x.double() @ W.double().t()
    size = (x.double().abs() @ W.double().abs().t()).amax(1)
    if bias is not None:
        logits = logits + bias.double()
        size = size + torch.where(bias > -INF, bias, torch.zeros_like(bias)).double().abs().amax()
    moved = (x.shape[1] + 3) * ref.U * size / t
    r = ref.Rows(logits, t)
    ref.near(out.logp, ref.pick(r.logp, y, 0.0), ref.pick(r.logp_off(), y, 0.0) + 2 * moved, "logp")
    ref.near(out.lse, r.lse[:, 0], r.lse_off()[:, 0] + moved, "lse")
    ref.near(out.entropy, r.entropy[:, 0], r.entropy_off()[:, 0] + 2 * moved * (1 + r.A[:, 0] + r.A2[:, 0]), "entropy")


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T,K,C", [(1, 1, 1), (1, 64, 10), (3, 33, 7), (1, 4096, 4099), (32, 64, 257), (33, 250, 130), (64, 256, 200),
                                   (129, 100, 1000), (257, 72, 513), (300, 264, 5003), (1000, 40, 3001), (40, 512, 40000),
                                   (2049, 64, 128), (520, 1024, 9000), (171, 60, 33000), (3, 1359, 16600), (300, 33, 32800)])
def test_head(T, K, C, dtype):
    x, W, bias, y = _case(T, K, C, dtype, T + K + C, strided=(T + K + C) % 3 == 0)
    _check(x, W, bias, y, 1.0, _api().head_logprobs(x, W, bias, y))
    _check(x, W, None, y, 2.5, _api().head_logprobs(x, W, None, y, temperature=2.5))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_tiles(dtype):
    x, W, bias, y = _case(3000, 128, 6000, dtype, 5)
    _check(x, W, bias, y, 1.0, _api().head_logprobs(x, W, bias, y))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("C", [1, 31, 33, 64, 90, 128, 130, 170, 200, 225, 256, 257])
@pytest.mark.parametrize("T,K", [(8200, 72), (24700, 33), (25000, 200)])
def test_whole_heads(T, K, C, dtype):
    """Heads of up to 256 classes and many rows, which one tile finishes (and one class more, which none does)."""
    x, W, bias, y = _case(T, K, C, dtype, T + C)
    out = _api().head_logprobs(x, W, bias, y, temperature=1.2)
    _check(x, W, bias, y, 1.2, out)
    if C > 40:
        bias[3::4] = -INF
        _check(x, W, bias, y, 1.0, _api().head_logprobs(x, W, bias, y))


def test_rows_in_passes():
    """So many classes that the parts of all rows pass 256 MiB: 1024 rows at a time."""
    T, K, C = 1300, 32, 1 << 20
    x, W, bias, y = _case(T, K, C, BF16, 9)
    out = _api().head_logprobs(x, W, bias, y)
    for r in (slice(0, 20), slice(1010, 1040), slice(1280, 1300)):
        part = _api().LogProbs(out.logp[r], out.lse[r], out.entropy[r], None, None)
        _check(x[r], W, bias, y[r], 1.0, part)


@pytest.mark.parametrize("T", [3, 70, 700])
def test_masked_classes(T):
    """A bias of -inf or of the type's lowest value; a head of which nothing is left."""
    x, W, bias, y = _case(T, 64, 700, F32, 2)
    bias[::3] = -INF
    bias[1::3] = torch.finfo(F32).min
    y[:2] = torch.tensor([3, 2], dtype=torch.int32)
    out = _api().head_logprobs(x, W, bias, y)
    _check(x, W, torch.where(bias < -1e38, torch.full_like(bias, -INF), bias), y,
           1.0, _api().LogProbs(torch.where(out.logp < -1e38, torch.full_like(out.logp, -INF), out.logp), out.lse, out.entropy, None, None))
    assert out.logp[0] == -INF
    none = _api().head_logprobs(x, W, torch.full_like(bias, -INF), y)
    inside = (y >= 0) & (y < 700)
    assert bool((none.lse == -INF).all()) and bool((none.entropy == 0).all())
    assert bool((none.logp[inside] == -INF).all()) and bool((none.logp[~inside] == 0).all())


@pytest.mark.parametrize("T", [5, 300])
def test_not_finite(T):
    """A row's NaN stays with the row."""
    x, W, bias, y = _case(T, 96, 500, BF16, 3)
    was = _api().head_logprobs(x, W, bias, y)
    x[2, 7] = math.nan
    x[4] = INF
    y[2], y[4] = 5, 6
    out = _api().head_logprobs(x, W, bias, y)
    keep = [t for t in range(T) if t not in (2, 4)]
    for name in ("logp", "lse", "entropy"):
        assert torch.equal(getattr(out, name)[keep], getattr(was, name)[keep]), name
        assert bool(getattr(out, name)[[2, 4]].isnan().all()), name


def test_no_rows_and_another_stream():
    api = _api()
    x, W, bias, y = _case(200, 128, 3001, F16, 4)
    assert api.head_logprobs(x[:0], W, bias, y[:0]).logp.shape == (0,)
    want = api.head_logprobs(x, W, bias, y)
    torch.cuda.synchronize()
    found = []
    for s in [torch.cuda.Stream() for _ in range(2)] * 2:
        with torch.cuda.stream(s):
            found.append(api.head_logprobs(x, W, bias, y))
    torch.cuda.synchronize()
    for out in found:
        assert torch.equal(out.logp, want.logp) and torch.equal(out.lse, want.lse) and torch.equal(out.entropy, want.entropy)


def test_as_the_logits_score():
    """The same as scoring the projection's own logits, up to the rounding of float32 products."""
    api = _api()
    x, W, bias, y = _case(64, 256, 200, F32, 6)
    none = torch.zeros(2, dtype=torch.int32, device=DEV)
    none[1] = 64
    logits = api.adapter_forward(x, W, bias, torch.zeros(1, 4, 256, device=DEV), torch.zeros(1, 200, 4, device=DEV),
                                 torch.ones(1, device=DEV), none, torch.full((1,), -1, dtype=torch.int32, device=DEV)).y
    a, b = api.head_logprobs(x, W, bias, y), api.logprobs(logits, y)
    size = (x.abs() @ W.abs().t()).amax(1) + bias.abs().amax()
    off = 4 * (256 + 3 + ref.chain(200)) * ref.U * (1 + size)
    for name in ("logp", "lse"):
        assert bool(((getattr(a, name) - getattr(b, name)).abs() <= off).all()), name
