"""Distillation from a teacher's top logits against float64, and the operators together as a training step uses them."""
import math

import pytest
import torch

import score_ref as ref
from test_gpu_logprobs import BF16, DEV, F16, F32, INF, SHAPES, _labels, _logits

pytestmark = pytest.mark.gpu


def _api():
    from paper_2608_13144_amd import api
    return api


def _teacher(x, k, g, short=0.2):
    """k distinct classes near the row's largest ones where there are as many, some of them left out."""
    T, C = x.shape
    noisy = torch.where(x.float() > -INF, x.float(), torch.full((), -30.0, device=DEV)) + torch.randn(T, C, generator=g, device=DEV)
    found = torch.topk(noisy, k, dim=1)
    index = found.indices.to(torch.int32)
    index[torch.rand(T, k, generator=g, device=DEV) < short] = -1
    return found.values, index


def _check(x, teacher, index, y, w, hard, soft, t, out):
    ce, ce_off, kl, kl_off, grad, off = ref.distill(x, teacher, index, y, w, hard, soft, t)
    ref.near(out.ce, ce, ce_off, "ce")
    ref.near(out.kl, kl, kl_off, "kl")
    if out.grad is not None:
        ref.near(out.grad, grad, ref.rounded(off, grad, x.dtype), "grad")


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T,C", SHAPES)
def test_distill(T, C, dtype):
    x, g = _logits(T, C, dtype, 3 * C + T, strided=C % 2 == 1)
    y = _labels(T, C, g)
    teacher, index = _teacher(x, min(C, 16), g)
    w = torch.rand(T, generator=g, device=DEV)
    for hard, soft, t in ((0.4, 2.4, 2.0), (0.5, 0.5, 1.0)):
        _check(x, teacher, index, y, w, hard, soft, t,
               _api().distill(x, teacher, index, y, weight=w, hard=hard, soft=soft, temperature=t))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k", [0, 1, 2, 17, 63, 64, 65, 200, 1000])
@pytest.mark.parametrize("C", [200, 3000, 70001])
def test_entries(C, k, dtype):
    """Numbers of entries around a wave's and a workgroup's; every class of a small head; classes named twice."""
    x, g = _logits(9, C, dtype, C + k)
    n = min(k, C)
    teacher, index = _teacher(x, n, g, short=0.0)
    if k > n:
        teacher = torch.cat([teacher, torch.randn(9, k - n, generator=g, device=DEV)], 1)
        index = torch.cat([index, torch.randint(-1, C + 1, (9, k - n), generator=g, device=DEV, dtype=torch.int32)], 1)
    if k > 1:
        index[2, :] = 4          # one class alone
        index[3, 1] = index[3, 0]
    out = _api().distill(x, teacher.contiguous(), index.contiguous(), soft=1.5, temperature=3.0)
    _check(x, teacher, index, None, None, 0.0, 1.5, 3.0, out)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("C,k", [(40, 224), (200, 65), (250, 200), (200, 225)])
def test_entries_of_many_short_rows(C, k, dtype):
    x, g = _logits(16390, C, dtype, C + k)
    n = min(k, C)
    teacher, index = _teacher(x, n, g)
    if k > n:
        teacher = torch.cat([teacher, torch.randn(16390, k - n, generator=g, device=DEV)], 1)
        index = torch.cat([index, torch.randint(-1, C + 1, (16390, k - n), generator=g, device=DEV, dtype=torch.int32)], 1)
    y = _labels(16390, C, g)
    out = _api().distill(x, teacher, index, y, hard=0.3, soft=1.5, temperature=3.0)
    _check(x, teacher, index, y, None, 0.3, 1.5, 3.0, out)


@pytest.mark.parametrize("C", [40, 600, 30000, 70001])
def test_edges(C):
    """Rows without entries, labels or weight; -inf and NaN on either side."""
    api = _api()
    x, g = _logits(12, C, F32, C)
    teacher, index = _teacher(x, 6, g, short=0.0)
    y = torch.randint(0, C, (12,), generator=g, device=DEV, dtype=torch.int32)
    w = torch.rand(12, generator=g, device=DEV) + 0.1
    index[1] = -1                                 # no entry: ce alone
    y[2] = -1                                     # no label: kl alone
    index[3], y[3] = -1, -1                       # neither
    x[3, 0] = math.nan
    w[4], x[4, 1] = 0.0, math.nan                 # no weight
    x[5] = -INF                                   # nothing left
    teacher[6, 2] = -INF                          # an entry without mass
    teacher[7] = -INF                             # none with mass
    x[8, int(index[8, 0])] = -INF                 # mass where the row has none
    teacher[9, 1] = math.nan
    x[10, 5] = math.nan
    x[11] = torch.finfo(F32).min
    out = api.distill(x, teacher, index, y, weight=w, hard=0.7, soft=1.2, temperature=2.0)
    rows = [0, 1, 2, 5, 6, 7, 8, 11]
    at = torch.tensor(rows, device=DEV)
    part = api.Distilled(out.ce[at], out.kl[at], out.grad[at])
    _check(x[at], teacher[at], index[at], y[at], w[at], 0.7, 1.2, 2.0, part)
    assert out.ce[3] == 0 and out.kl[3] == 0 and bool((out.grad[3] == 0).all())
    assert bool((out.grad[4] == 0).all()) and bool((out.grad[5] == 0).all())
    assert out.kl[7] == 0 and out.kl[8] == INF and out.ce[5] == INF and out.kl[5] == INF
    assert out.kl[9].isnan() and bool(out.grad[9].isnan().any()) and torch.isfinite(out.ce[9])
    assert out.kl[10].isnan() and out.ce[10].isnan() and bool(out.grad[10].isnan().any())
    # hard = 0 leaves rows without entries alone, soft = 0 rows without a label
    only = api.distill(x, teacher, index, y, weight=w, hard=0.0, soft=1.0)
    assert bool((only.grad[1] == 0).all()) and bool((only.grad[7] == 0).all())
    only = api.distill(x, teacher, index, y, weight=w, hard=1.0, soft=0.0)
    assert bool((only.grad[2] == 0).all()) and torch.equal(only.ce[at], out.ce[at])


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("C", [48, 201, 5003, 140001])
def test_in_place_beside_and_without_a_gradient(C, dtype):
    api = _api()
    x, g = _logits(3, C, dtype, C)
    y = _labels(3, C, g)
    teacher, index = _teacher(x, 12, g)
    args = dict(hard=0.5, soft=1.0, temperature=1.5)
    want = api.distill(x, teacher, index, y, **args)
    wide = torch.full((3, C + 9), 7.0, dtype=dtype, device=DEV)
    got = api.distill(x, teacher, index, y, out=wide[:, 5:5 + C], **args)
    assert torch.equal(got.grad, want.grad) and bool((wide[:, :5] == 7).all()) and bool((wide[:, 5 + C:] == 7).all())
    without = api.distill(x, teacher, index, y, want_grad=False, **args)
    assert without.grad is None and torch.equal(without.ce, want.ce) and torch.equal(without.kl, want.kl)
    mine = x.clone()
    got = api.distill(mine, teacher, index, y, out=mine, **args)
    assert got.grad is mine and torch.equal(mine, want.grad) and torch.equal(got.kl, want.kl)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,C", [(65, 140001), (700, 33000), (66, 65537)])
def test_losses_alone(T, C, dtype):
    """Without a gradient long rows go through in other shares, as far as they need no registers for it."""
    x, g = _logits(T, C, dtype, C + T)
    y = _labels(T, C, g)
    teacher, index = _teacher(x, 70, g)
    for hard, t in ((0.4, 2.0), (0.0, 0.7)):
        out = _api().distill(x, teacher, index, y, hard=hard, temperature=t, want_grad=False)
        assert out.grad is None
        _check(x, teacher, index, y, None, hard, 1.0, t, out)


def test_against_differences():
    """Central differences of the float64 definition, step 1e-5: off by h^2 / 6 times the third derivative (order one)."""
    T, C, t, hard, soft = 5, 11, 1.7, 0.6, 2.3
    x, g = _logits(T, C, F32, 2, spread=1.0)
    y = _labels(T, C, g)
    teacher, index = _teacher(x, 4, g)
    w = torch.rand(T, generator=g, device=DEV)
    got, h = _api().distill(x, teacher, index, y, weight=w, hard=hard, soft=soft, temperature=t).grad.double(), 1e-5

    def value(z):
        ce, _, kl, _, _, _ = ref.distill(z, teacher, index, y, w, hard, soft, t)
        return (hard * ce + soft * kl) * w.double()
    for j in range(C):
        step = torch.zeros(T, C, dtype=torch.float64, device=DEV)
        step[:, j] = h
        slope = (value(x.double() + step) - value(x.double() - step)) / (2 * h)
        assert bool(((slope - got[:, j]).abs() < 1e-5).all()), (j, slope, got[:, j])


def test_equal_bits_every_time():
    x, g = _logits(700, 5003, BF16, 8)
    y = _labels(700, 5003, g)
    teacher, index = _teacher(x, 64, g)
    index[::2, 10] = index[::2, 3]
    first = _api().distill(x, teacher, index, y, hard=0.3, soft=1.0, temperature=2.0)
    for _ in range(4):
        again = _api().distill(x, teacher, index, y, hard=0.3, soft=1.0, temperature=2.0)
        assert torch.equal(first.ce, again.ce) and torch.equal(first.kl, again.kl) and torch.equal(first.grad, again.grad)


def test_a_training_step_of_the_sites():
    """Teacher's alternatives -> adapted logits -> losses and gradient -> the pairs' gradients -> their step."""
    api = _api()
    g = torch.Generator(device=DEV).manual_seed(11)

    def randn(*s):
        return torch.randn(*s, generator=g, device=DEV)
    T, K, C, S, r, k, t = 96, 64, 40, 3, 4, 8, 2.0
    x, W, bias = randn(T, K), randn(C, K) / 8, 0.1 * randn(C)
    A, B, scale = randn(S, r, K) / 8, 0.3 * randn(S, C, r), torch.ones(S, device=DEV)
    offsets = torch.tensor([0, 30, 31, 96], dtype=torch.int32, device=DEV)
    adapter = torch.tensor([2, -1, 0], dtype=torch.int32, device=DEV)
    y = _labels(T, C, g)
    main = 2.0 * randn(T, C)                                     # the main model's logits
    best = api.logprobs(main, top=k)
    out = api.adapter_forward(x, W, bias, A, B, scale, offsets, adapter, keep=True)
    loss = api.distill(out.y, best.top_logp, best.top_index, y, weight=torch.full((T,), 1 / T, device=DEV), hard=0.5,
                       soft=0.5 * t * t, temperature=t, out=out.y)
    grad = api.adapter_backward(loss.grad, x, W, A, B, scale, offsets, adapter, v=out.v)
    # the same in float64 by automatic differentiation (float32 logits: sums of 64 products, gradients of order 1/T)
    Ad, Bd = A.double().requires_grad_(), B.double().requires_grad_()
    logits = x.double() @ W.double().t() + bias.double()
    for lo, hi, a in ((0, 30, 2), (31, 96, 0)):
        logits = torch.cat([logits[:lo], logits[lo:hi] + x[lo:hi].double() @ Ad[a].t() @ Bd[a].t(), logits[hi:]])
    some = (y >= 0) & (y < C)
    q = torch.softmax(best.top_logp.double() / t, 1)
    logp, hot = torch.log_softmax(logits, 1), torch.log_softmax(logits / t, 1)
    ce = -(logp.gather(1, y.clamp(0, C - 1).long()[:, None])[:, 0] * some)
    kl = (q * (q.log() - hot.gather(1, best.top_index.long()))).sum(1)
    (0.5 * ce + 0.5 * t * t * kl).mean().backward()
    # relative: 64 + 96 additions of float32 and the score's own 50 or so
    assert bool(((loss.ce - ce).abs() <= 300 * ref.U * (1 + ce.abs())).all())
    assert bool(((loss.kl - kl).abs() <= 300 * ref.U * (1 + kl.abs())).all())
    for got, want in ((grad.dA, Ad.grad), (grad.dB, Bd.grad)):
        assert bool(((got - want).abs() <= 600 * ref.U * want.abs().amax()).all())
    before = A.clone()
    api.muon_step(A, grad.dA, torch.zeros_like(A), 0.05)
    assert torch.isfinite(A).all() and not torch.equal(A, before)


def test_few_rows_captured_and_replayed():
    """Rows that go in shares, two graphs of them replayed in turn: each has its own workspace."""
    api = _api()
    T, C, k = 3, 70001, 8
    graphs = []
    for seed in (1, 2):
        x, g = _logits(T, C, BF16, seed)
        teacher, index = _teacher(x, k, g)
        y = _labels(T, C, g)

        def work(x=x, y=y, teacher=teacher, index=index):
            return api.logprobs(x, y, top=k), api.distill(x, teacher, index, y, hard=0.5, soft=1.0, temperature=2.0)
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            work()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            found = work()
        graphs.append((graph, found, x, work))
    for turn in range(3):
        for i, (graph, found, x, work) in enumerate(graphs):
            x.copy_(_logits(T, C, BF16, 10 * turn + i)[0])
        for graph, _, _, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, (s, loss), _, work in graphs:
            es, eloss = work()
            for got, want in ((s.logp, es.logp), (s.entropy, es.entropy), (s.top_index, es.top_index), (s.top_logp, es.top_logp),
                              (loss.ce, eloss.ce), (loss.kl, eloss.kl), (loss.grad, eloss.grad)):
                assert torch.equal(got, want), turn


def test_captured_and_replayed():
    """One graph of scores, gradient and distillation, replayed on new inputs with eager work between."""
    api = _api()
    T, C, k = 37, 1501, 8
    x, g = _logits(T, C, BF16, 6)
    y = _labels(T, C, g)
    teacher, index = _teacher(x, k, g)
    g_logp = torch.randn(T, generator=g, device=DEV)
    W, z = torch.randn(C, 64, generator=g, device=DEV).to(BF16), torch.randn(T, 64, generator=g, device=DEV).to(BF16)

    def work():
        return (api.logprobs(x, y, top=k), api.logprobs_backward(x, y, g_logp=g_logp),
                api.distill(x, teacher, index, y, hard=0.5, soft=1.0, temperature=2.0), api.head_logprobs(z, W, None, y))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s, d, loss, head = work()
    for seed in range(3):
        x.copy_(_logits(T, C, BF16, 50 + seed)[0])
        z.copy_(torch.randn(T, 64, generator=g, device=DEV))
        teacher.add_(0.1)
        graph.replay()
        torch.cuda.synchronize()
        es, ed, eloss, ehead = work()
        for got, want in ((s.logp, es.logp), (s.lse, es.lse), (s.entropy, es.entropy), (s.top_index, es.top_index),
                          (s.top_logp, es.top_logp), (d, ed), (loss.ce, eloss.ce), (loss.kl, eloss.kl),
                          (loss.grad, eloss.grad), (head.logp, ehead.logp), (head.entropy, ehead.entropy)):
            assert torch.equal(got, want), seed
