"""Log probabilities of rows of logits and their gradient against float64, row by row and value by value."""
import math

import pytest
import torch

import score_ref as ref

pytestmark = pytest.mark.gpu

INF = math.inf
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
DEV = "cuda"


def _api():
    from paper_2608_13144_amd import api
    return api


def _logits(T, C, dtype, seed, masked=0.0, strided=False, spread=3.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    room = C + 37 if strided else C
    x = spread * torch.randn(T, room, generator=g, device=DEV)
    if masked:
        x[torch.rand(T, room, generator=g, device=DEV) < masked] = -INF
    return x.to(dtype)[:, room - C:], g


def _labels(T, C, g):
    y = torch.randint(0, C, (T,), generator=g, device=DEV, dtype=torch.int32)
    y[::5] = -1
    if T > 3:
        y[3] = C  # outside: none
    return y


def _check_scores(x, y, k, t, out):
    r = ref.Rows(x, t)
    if y is not None:
        ref.near(out.logp, ref.pick(r.logp, y, 0.0), ref.pick(r.logp_off(), y, 0.0), "logp")
    else:
        assert bool((out.logp == 0).all())
    ref.near(out.lse, r.lse[:, 0], r.lse_off()[:, 0], "lse")
    ref.near(out.entropy, r.entropy[:, 0], r.entropy_off()[:, 0], "entropy")
    if k:
        at = ref.top(x, k)
        assert torch.equal(out.top_index, at)
        there = at >= 0
        safe = at.clamp(min=0).long()
        nothing = torch.full_like(safe, -INF, dtype=torch.float64)
        exact = torch.where(there, r.logp.gather(1, safe), nothing)
        ref.near(out.top_logp, exact, torch.where(there, r.logp_off().gather(1, safe), torch.zeros_like(exact)), "top")


SHAPES = [(1, 1), (5, 2), (4, 7), (300, 10), (9, 64), (70, 200), (5, 257), (6, 1000), (130, 1024), (3, 1031), (4, 4099),
          (3, 5003), (2, 16384), (2, 32767), (3, 50021), (2, 65536), (1, 131072), (2, 131075), (1, 262147), (1, 1 << 20),
          # more rows, which other numbers of threads take
          (2100, 1300), (2601, 2500), (2600, 5003), (801, 9001), (800, 20000), (101, 20000), (65, 60000), (66, 131072), (65, 200001)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T,C", SHAPES)
def test_scores(T, C, dtype):
    x, g = _logits(T, C, dtype, 7 * C + T, strided=C % 2 == 1)
    y = _labels(T, C, g)
    k = min(64, C) if T % 2 else min(8, C)
    _check_scores(x, y, k, 0.7, _api().logprobs(x, y, top=k, temperature=0.7))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("k", [0, 1, 2, 5, 8, 9, 20, 32, 33, 63, 64])
@pytest.mark.parametrize("C", [33, 200, 3000, 40000, 70001])
def test_alternatives(C, k, dtype):
    x, g = _logits(12, C, dtype, C + k, masked=0.3)
    x[1] = -INF                      # nothing left
    x[2] = -INF
    x[2, C - 1] = 1.0                # one class left
    x[3] = 0.5                       # all alike: by index
    x[4] = torch.finfo(dtype).min    # masked by the lowest value throughout
    x[5] = torch.linspace(-4, 4, C, device=DEV).to(dtype)  # the largest ones last, next to each other
    x[6] = torch.linspace(4, -4, C, device=DEV).to(dtype)
    x[7] = 0.0
    x[7, ::2] = -0.0                 # equal to the others
    x[8, : C // 2] = 3.0             # a long run of equal ones
    y = _labels(12, C, g)
    _check_scores(x, y, k, 1.0, _api().logprobs(x, y, top=k))


@pytest.mark.parametrize("C", [12, 500, 9000, 70001])
def test_more_alternatives_than_classes(C):
    x = torch.full((3, C), -INF, device=DEV)
    x[1, 3] = 2.0
    x[2, :9] = torch.arange(9.0, device=DEV)
    out = _api().logprobs(x, top=20)
    _check_scores(x, None, 20, 1.0, out)
    assert out.top_index[0].tolist() == [-1] * 20 and out.top_index[1].tolist() == [3] + [-1] * 19


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("C", [30, 700, 20000, 70001])
@pytest.mark.parametrize("t", [0.25, 1.0, 8.0])
def test_lowest_and_largest_values(C, t, dtype):
    """Logits of the type's lowest value are logits like others; differences past float32 are p = 0."""
    low, high = torch.finfo(dtype).min, torch.finfo(dtype).max
    x = torch.full((4, C), low, device=DEV, dtype=dtype)
    x[1, 5] = 1.0
    x[2] = high
    x[3, 2::3] = high
    y = torch.tensor([4, 5, 6, 2], dtype=torch.int32, device=DEV)
    out = _api().logprobs(x, y, temperature=t)
    r = ref.Rows(x, t)
    assert torch.isfinite(out.logp).all() and torch.isfinite(out.entropy).all()
    ref.near(out.logp, ref.pick(r.logp, y, 0.0), ref.pick(r.logp_off(), y, 0.0))
    n = torch.tensor([C, 1, C, len(range(2, C, 3))], device=DEV).double()
    ref.near(out.entropy, n.log(), 64 * ref.U * (n.log() + 1) + ref.chain(C) * ref.U)
    lse = r.lse[:, 0]
    lse = torch.where(lse.abs() > torch.finfo(F32).max * (1 + 2.0 ** -24), INF * lse.sign(), lse)  # past float32
    ref.near(out.lse, lse, r.lse_off()[:, 0])


@pytest.mark.parametrize("C", [30, 700, 20000, 70001])
def test_not_finite(C):
    """NaN and +inf make their own row's numbers NaN, and nobody else's."""
    x, g = _logits(7, C, F32, C)
    clean = x.clone()
    x[1, C // 2] = math.nan
    x[3, C - 1] = INF
    x[5] = math.nan
    y = torch.arange(7, dtype=torch.int32, device=DEV)
    y[5] = -1
    out, was = _api().logprobs(x, y, top=3), _api().logprobs(clean, y, top=3)
    for name in ("logp", "lse", "entropy", "top_logp"):
        got, other = getattr(out, name), getattr(was, name)
        for t in (0, 2, 4, 6):
            assert torch.equal(got[t], other[t]), (name, t)
        for t in (1, 3):
            assert bool(got[t].isnan().all()), (name, t)
    assert out.logp[5] == 0 and out.lse[5].isnan() and out.top_index[5].tolist() == [-1] * 3
    assert int(out.top_index[3, 0]) == C - 1 and torch.equal(out.top_index[1], ref.top(x[1:2], 3)[0])


@pytest.mark.parametrize("C", [60, 300, 1500, 3001, 20000, 70001])
@pytest.mark.parametrize("k", [3, 9, 20, 32, 64])
def test_alternatives_among_nan(C, k):
    """A NaN is no alternative and hides none, however many there are and wherever."""
    x, g = _logits(8, C, F32, C + k)
    x[1, : C // 2] = math.nan
    x[2, C // 2:] = math.nan
    x[3, ::2] = math.nan
    x[4, -1] = math.nan
    x[5, : C - 2] = math.nan
    x[6] = math.nan
    x[7, C - C % 8:] = math.nan
    out = _api().logprobs(x, top=k)
    at = ref.top(x, k)
    assert torch.equal(out.top_index, at)
    assert bool((out.top_logp.isnan() == ((at >= 0) & x.isnan().any(1, keepdim=True))).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,C", [(64, 40000), (65, 40000), (3, 300000), (2000, 5000), (40, 5000)])
def test_classes_allowed_in_a_run(T, C, dtype):
    """What is allowed lies in one run somewhere, or rises to the end: the first part of a row tells nothing of its largest."""
    x, g = _logits(T, C, dtype, T + C)
    first = torch.randint(0, C - 700, (T, 1), generator=g, device=DEV)
    j = torch.arange(C, device=DEV)
    x = torch.where((j >= first) & (j < first + 600), x, torch.full_like(x, -INF))
    x[::3] = torch.linspace(-9, 9, C, device=DEV).to(dtype)
    y = _labels(T, C, g)
    for k in (1, 8, 20, 64):
        _check_scores(x, y, k, 1.0, _api().logprobs(x, y, top=k))


def test_no_rows_and_parts_of_the_output():
    api = _api()
    out = api.logprobs(torch.empty(0, 50, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV), top=4)
    assert out.logp.shape == (0,) and out.top_index.shape == (0, 4)
    assert api.logprobs_backward(torch.empty(0, 50, device=DEV), g_lse=torch.empty(0, device=DEV)).shape == (0, 50)
    x, g = _logits(6, 90, F32, 3)
    mine = api.LogProbs(None, torch.full((6,), 9.0, device=DEV), None, None, None)
    assert api.logprobs(x, out=mine) is mine
    assert torch.equal(mine.lse, api.logprobs(x).lse)


def _gradients(T, C, g, k):
    def randn(*s):
        return torch.randn(*s, generator=g, device=DEV)
    index = torch.randint(0, C, (T, k), generator=g, device=DEV, dtype=torch.int32)  # the same class twice among them
    if k > 1:
        index[::3, 0] = -1
        index[1::3, 1] = C + 5
    return dict(g_logp=randn(T), g_lse=randn(T), g_entropy=randn(T), top_index=index, g_top=randn(T, k))


def _check_backward(x, y, t, grads, got):
    exact, off = ref.backward(x, t, y, grads.get("g_logp"), grads.get("g_lse"), grads.get("g_entropy"),
                              grads.get("top_index"), grads.get("g_top"))
    ref.near(got, exact, ref.rounded(off, exact, x.dtype), "dx")


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T,C", SHAPES)
def test_gradient(T, C, dtype):
    x, g = _logits(T, C, dtype, 5 * C + T, masked=0.2 if T > 2 else 0.0, strided=C % 2 == 1)
    y, grads = _labels(T, C, g), _gradients(T, C, g, 3)
    _check_backward(x, y, 1.3, grads, _api().logprobs_backward(x, y, temperature=1.3, **grads))


@pytest.mark.parametrize("which", ["g_logp", "g_lse", "g_entropy", "g_top"])
@pytest.mark.parametrize("C", [40, 3000])
def test_gradient_of_each_output(C, which):
    x, g = _logits(20, C, F32, C)
    y, grads = _labels(20, C, g), _gradients(20, C, g, 7)
    grads = {n: v for n, v in grads.items() if n == which or (n == "top_index" and which == "g_top")}
    _check_backward(x, y, 1.0, grads, _api().logprobs_backward(x, y, **grads))


def test_gradient_against_differences():
    """Central differences of the float64 definition, step 1e-5: off by h^2 / 6 times the third derivative (order one)."""
    T, C, t = 4, 9, 0.8
    x, g = _logits(T, C, F32, 1, spread=1.0)
    y, grads = _labels(T, C, g), _gradients(T, C, g, 4)
    grads["top_index"] = torch.randint(0, C, (T, 4), generator=g, device=DEV, dtype=torch.int32)

    def value(z):
        r = ref.Rows(z, t)
        some = (y >= 0) & (y < C)
        return (torch.where(some, ref.pick(r.logp, y, 0.0) * grads["g_logp"].double(), 0.0) +
                r.lse[:, 0] * grads["g_lse"].double() + r.entropy[:, 0] * grads["g_entropy"].double() +
                (r.logp.gather(1, grads["top_index"].long()) * grads["g_top"].double()).sum(1))
    got, h = _api().logprobs_backward(x, y, temperature=t, **grads).double(), 1e-5
    for j in range(C):
        step = torch.zeros(T, C, dtype=torch.float64, device=DEV)
        step[:, j] = h
        slope = (value(x.double() + step) - value(x.double() - step)) / (2 * h)
        assert bool(((slope - got[:, j]).abs() < 1e-5).all()), (j, slope, got[:, j])


@pytest.mark.parametrize("C", [40, 600, 30000, 70001])
def test_rows_without_a_gradient(C):
    """Zero gradients give zero rows whatever they hold; so does a row that is masked throughout."""
    x, g = _logits(8, C, F32, C)
    x[1] = math.nan
    x[2, 3] = INF
    x[4] = -INF
    y = torch.arange(8, dtype=torch.int32, device=DEV)
    y[1] = -1
    g_logp = torch.randn(8, generator=g, device=DEV)
    g_logp[2] = 0.0
    dx = _api().logprobs_backward(x, y, g_logp=g_logp)
    assert bool((dx[[1, 2, 4]] == 0).all())
    assert torch.equal(dx[[0, 3, 5, 6, 7]], _api().logprobs_backward(x[[0, 3, 5, 6, 7]], y[[0, 3, 5, 6, 7]], g_logp=g_logp[[0, 3, 5, 6, 7]]))
    # gradients that cancel in their sum still count
    index = torch.tensor([[3, 7]] * 8, dtype=torch.int32, device=DEV)
    both = torch.tensor([[1.0, -1.0]] * 8, device=DEV)
    keep = [0, 3, 5, 6, 7]
    dx = _api().logprobs_backward(x[keep], top_index=index[keep], g_top=both[keep])
    exact, off = ref.backward(x[keep], 1.0, index=index[keep], g_top=both[keep])
    ref.near(dx, exact, ref.rounded(off, exact, F32))
    assert bool((dx[:, 3] == 1).all()) and bool((dx[:, 7] == -1).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,C,k", [(3, 50, 1024), (5, 200, 200), (2, 7000, 1000), (2, 70, 65), (70, 130, 33),
                                   (16400, 40, 224), (16385, 200, 65), (16384, 300, 225)])
def test_many_entries(T, C, k, dtype):
    """More entries than threads of a row, most of them several times."""
    x, g = _logits(T, C, dtype, C)
    grads = _gradients(T, C, g, k)
    grads["top_index"][0] = 5 % C
    _check_backward(x, None, 1.0, dict(top_index=grads["top_index"], g_top=grads["g_top"]),
                    _api().logprobs_backward(x, top_index=grads["top_index"], g_top=grads["g_top"]))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("C", [48, 201, 5003, 140001])
def test_gradient_in_place_and_beside(C, dtype):
    """dx may be x; rows inside a wider buffer leave what lies between them as it was."""
    api = _api()
    x, g = _logits(3, C, dtype, C)
    y, grads = _labels(3, C, g), _gradients(3, C, g, 3)
    want = api.logprobs_backward(x, y, **grads)
    wide = torch.full((3, C + 9), 7.0, dtype=dtype, device=DEV)
    assert torch.equal(api.logprobs_backward(x, y, out=wide[:, 4:4 + C], **grads), want)
    assert bool((wide[:, :4] == 7).all()) and bool((wide[:, 4 + C:] == 7).all())
    mine = x.clone()
    assert api.logprobs_backward(mine, y, out=mine, **grads) is mine
    assert torch.equal(mine, want)


def test_offsets_past_32_bits():
    """More than 2^32 logits: the last rows come out as they do alone."""
    T, C = 33000, 131072
    x = torch.empty(T, C, dtype=BF16, device=DEV)
    for part in x.split(4096):
        part.copy_(torch.randn(C, device=DEV).roll(len(part))[None, :] * 3)
    part = _logits(6, C, BF16, 1)[0]
    rows = torch.tensor([0, 1, 16384, 32767, T - 2, T - 1], device=DEV)
    x[rows] = part
    y = torch.arange(T, dtype=torch.int32, device=DEV)
    g = torch.randn(T, device=DEV)
    api = _api()
    out, alone = api.logprobs(x, y, top=3), api.logprobs(torch.cat([part] * 12), y[rows].repeat(12), top=3)  # not in shares
    for name in ("logp", "lse", "entropy"):
        assert torch.allclose(getattr(out, name)[rows], getattr(alone, name)[:6], rtol=1e-5, atol=1e-5), name
    assert torch.equal(out.top_index[rows], alone.top_index[:6])
    dx = api.logprobs_backward(x, y, g_logp=g, out=x)
    want = api.logprobs_backward(torch.cat([part] * 12), y[rows].repeat(12), g_logp=g[rows].repeat(12))
    assert dx is x and torch.equal(dx[rows], want[:6])


def test_another_stream_and_twice():
    api = _api()
    x, g = _logits(500, 3001, BF16, 4)
    y, grads = _labels(500, 3001, g), _gradients(500, 3001, g, 3)
    want, d = api.logprobs(x, y, top=5), api.logprobs_backward(x, y, **grads)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    found = []
    for s in streams * 2:
        with torch.cuda.stream(s):
            found.append((api.logprobs(x, y, top=5), api.logprobs_backward(x, y, **grads)))
    torch.cuda.synchronize()
    for out, dx in found:
        for name in ("logp", "lse", "entropy", "top_index", "top_logp"):
            assert torch.equal(getattr(out, name), getattr(want, name)), name
        assert torch.equal(dx, d)
