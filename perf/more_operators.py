"""The measured cases of the operators that score a head's answers and train it: log probabilities and distillation.

A proxy's head gives logits.  A site that takes its answers asks how likely they are
(the log probability of an answer, the entropy, the most likely alternatives) and
leaves unlikely ones to the main model.  The head and its sites' pairs learn from the
main model: from its labels, and from the few largest logits that it sends with them.

Kinds of case (``case["kind"]``):

  score      log probabilities of given labels, log of the sum of exponentials, entropy
             and top alternatives of rows of logits (``api.logprobs``)
  gradient   the gradient of the same with regard to the logits (``api.logprobs_backward``)
  distill    cross entropy with labels and the divergence from a teacher's top logits at
             a temperature, and their gradient, in one call (``api.distill``)
  head       log probabilities, sums and entropies straight from features and a head, no
             logits in memory (``api.head_logprobs``)

Sizes: 256 features, 200 classes and 32768 queries are this library's headline head and
batch; 32768 to 131072 classes are generic vocabularies of a language model's head.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
NONE = -1  # a label that is none, a teacher's entry or an alternative that is not there
INF = math.inf


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # The headline head's logits of a batch of queries, float32 as certified, with five alternatives.
        dict(name="score-queries", kind="score", dtype="f32", T=32768, C=200, top=5, temperature=1.0, masked=0.0,
             strided=False),
        # The smallest call: one token of a decode step over a large vocabulary; latency.
        dict(name="score-token", kind="score", dtype="bf16", T=1, C=131072, top=20, temperature=0.7, masked=0.0,
             strided=False),
        # Odd sizes inside a wider buffer, most classes masked (some rows altogether), no alternatives.
        dict(name="score-masked", kind="score", dtype="f16", T=1001, C=50021, top=0, temperature=1.0, masked=0.6,
             strided=True),
        # Scoring the tokens of prompts, with alternatives.
        dict(name="score-prompts", kind="score", dtype="bf16", T=4096, C=32768, top=8, temperature=1.0, masked=0.0,
             strided=False),
        # Training the headline head on labels, with an entropy term.
        dict(name="gradient-queries", kind="gradient", dtype="f32", T=32768, C=200, top=0, temperature=1.0, masked=0.0,
             strided=False),
        # Training on sampled tokens: gradients of the labels', the entropy's and the alternatives' terms.
        dict(name="gradient-prompts", kind="gradient", dtype="bf16", T=4096, C=32768, top=8, temperature=1.0,
             masked=0.0, strided=False),
        # The guard's own recipe: labels and all 200 logits of the main model, at a temperature.
        dict(name="distill-queries", kind="distill", dtype="f32", T=4096, C=200, k=200, temperature=4.0, hard=0.5,
             soft=8.0, short=0.0, strided=False),
        # A ragged batch of moderate width, 16 logits of the teacher, some rows with fewer.
        dict(name="distill-ragged", kind="distill", dtype="f16", T=1777, C=5003, k=16, temperature=2.0, hard=0.3,
             soft=2.8, short=0.3, strided=True),
        # The largest training call: a large vocabulary, 64 logits of the teacher, no labels.
        dict(name="distill-large", kind="distill", dtype="bf16", T=4096, C=131072, k=64, temperature=1.0, hard=0.0,
             soft=1.0, short=0.0, strided=False),
        # The headline head and batch from features: confidence beside the certified label.
        dict(name="head-queries", kind="head", dtype="f32", T=32768, K=256, C=200, temperature=1.0),
        # One token through a wide head: reads the head once.
        dict(name="head-token", kind="head", dtype="bf16", T=1, K=4096, C=131072, temperature=1.0),
        # Scoring prompts through a wide head.
        dict(name="head-prompts", kind="head", dtype="bf16", T=4096, K=4096, C=32768, temperature=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _width(rng, lo, hi):
    """A width: two times in three a multiple of eight, else any number."""
    w = _log_int(rng, lo, hi)
    return w if rng.random() < 1 / 3 else max(8, 8 * (w // 8))


def draw(rng):
    """One more case of the ranges above."""
    kind = rng.choice(["score", "gradient", "distill", "head"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    temperature = rng.choice([1.0, 1.0, 0.7, 2.0, 4.0])
    if kind == "head":
        K = _width(rng, 32, 4096)
        C = _width(rng, 10, 131072)
        most = (1 << 34) if dtype == "f32" else (1 << 37)  # T K C
        T = _log_int(rng, 1, max(4, min(32768, most // (K * C))))
        return dict(kind=kind, dtype=dtype, T=T, K=K, C=C, temperature=temperature)
    C = _width(rng, 8, 262144)
    T = _log_int(rng, 1, min(32768, (1 << 28) // C))
    c = dict(kind=kind, dtype=dtype, T=T, C=C, temperature=temperature, strided=rng.random() < 0.3)
    if kind == "distill":
        c["k"] = min(C, rng.choice([1, 5, 8, 16, 20, 64, 200]))
        c["hard"], c["soft"] = rng.choice([(0.0, 1.0), (0.5, 0.5), (0.1, 3.0), (1.0, 0.0)])
        c["short"] = rng.choice([0.0, 0.0, 0.3])
    else:
        c["top"] = min(C, rng.choice([0, 1, 5, 8, 20, 64]))
        c["masked"] = rng.choice([0.0, 0.0, 0.3, 0.9])
    return c


# ------------------------------------------------------------------ inputs
def _logits(g, case):
    """[T, C] rows: a few classes stand out; in masked cases others are -inf, a row in 97 altogether."""
    T, C, dtype = case["T"], case["C"], DTYPES[case["dtype"]]
    room = C + (-C) % 8 + 64 if case["strided"] else C
    x = torch.randn(T, room, generator=g, device=DEV)
    x += 0.5 * x * x.abs()  # a longer tail than the normal distribution's
    if case.get("masked"):
        x[torch.rand(T, room, generator=g, device=DEV) < case["masked"]] = -INF
        x[50::97] = -INF
    return x.to(dtype)[:, :C]


def _labels(g, T, C, x=None):
    """One label a row, none for a row in ten; likely ones among them."""
    label = torch.randint(0, C, (T,), generator=g, device=DEV)
    if x is not None:
        likely = x[:, :4096].float().argmax(1)
        label = torch.where(torch.rand(T, generator=g, device=DEV) < 0.6, likely, label)
    label[torch.rand(T, generator=g, device=DEV) < 0.1] = NONE
    return label.to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    kind, T, C = case["kind"], case["T"], case["C"]
    s = dict(case=case)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device=DEV)
    if kind == "head":
        K, dtype = case["K"], DTYPES[case["dtype"]]
        s["W"] = (randn(C, K) / math.sqrt(K)).to(dtype)
        s["bias"] = 0.1 * randn(C)
        s["label"] = _labels(g, T, C)
        # features lean towards their label's row
        s["x"] = (randn(T, K) + 4.0 * s["W"][s["label"].clamp(min=0).long()].float()).to(dtype)
        return s
    # float16 gradients come from a loss scaled to order one, others from a mean over the rows
    unit = 16.0 if case["dtype"] == "f16" else 1.0 / T
    x = s["x"] = _logits(g, case)
    s["label"] = _labels(g, T, C, x)
    if kind == "distill":
        k = case["k"]
        rows = max(1, (1 << 28) // C)
        parts = [torch.topk(x[i:i + rows].float() + randn(min(rows, T - i), C), k, dim=1) for i in range(0, T, rows)]
        s["teacher"] = torch.cat([p.values for p in parts])
        index = torch.cat([p.indices for p in parts]).to(torch.int32)
        if case["short"]:  # rows with fewer entries, some with none
            index[torch.rand(T, k, generator=g, device=DEV) < case["short"]] = NONE
            index[20::41] = NONE
        s["index"] = index
        s["weight"] = unit * torch.rand(T, generator=g, device=DEV)
    elif kind == "gradient":
        s["g_logp"], s["g_entropy"] = unit * randn(T), 0.01 * unit * randn(T)
        if case["top"]:
            s["index"] = torch.topk(x[:, :8 * case["top"]].float(), case["top"], dim=1).indices.to(torch.int32) \
                if 8 * case["top"] <= C else torch.arange(case["top"], device=DEV, dtype=torch.int32).repeat(T, 1)
            s["g_top"] = 0.1 * unit * randn(T, case["top"])
    return s


# ------------------------------------------------------------------ plain forms
def _sums(x, temperature):
    """Exponents a = (x - max) / temperature, e = exp(a), their sum and the row's largest value."""
    m = x.amax(1, keepdim=True)
    m = torch.where(m == -INF, torch.zeros_like(m), m)  # a row that is masked altogether
    a = (x - m) / temperature
    e = a.exp()
    return a, e, e.sum(1, keepdim=True), m


def _at(a, s, label):
    """Log probability of the labels, 0 where there is none."""
    none = label < 0
    at = a.gather(1, label.clamp(min=0).long()[:, None])
    logp = torch.where(s > 0, at - s.log(), torch.full_like(s, -INF))[:, 0]
    return torch.where(none, torch.zeros_like(logp), logp)


def _entropy(a, e, s):
    mean = torch.where(e > 0, a * e, torch.zeros_like(a)).sum(1, keepdim=True) / s
    return torch.where(s > 0, s.log() - mean, torch.zeros_like(s))


def _top(x, a, s, k):
    """The k largest, ties to the lowest index; masked classes are none."""
    T, C = x.shape
    bits = (x + 0.0).view(torch.int32)  # -0 counts as 0
    order = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long()
    key = (order << 32) + (C - 1 - torch.arange(C, device=DEV))
    at = C - 1 - (torch.topk(key, k, dim=1).values & 0xffffffff)
    there = x.gather(1, at) > -INF
    logp = torch.where(there, a.gather(1, at) - s.log(), torch.full((T, k), -INF, device=DEV))
    return torch.where(there, at, torch.full_like(at, NONE)).to(torch.int32), logp


def _plain_score(s):
    case, x = s["case"], s["x"].float()
    a, e, total, m = _sums(x, case["temperature"])
    out = dict(logp=_at(a, total, s["label"]), lse=(m / case["temperature"] + total.log())[:, 0],
               entropy=_entropy(a, e, total)[:, 0])
    if case["top"]:
        out["index"], out["top"] = _top(x, a, total, case["top"])
    return out


def _plain_gradient(s):
    case, x = s["case"], s["x"].float()
    a, e, total, _ = _sums(x, case["temperature"])
    some = total > 0
    p = torch.where(some, e / total, torch.zeros_like(e))
    label = s["label"].clamp(min=0).long()[:, None]
    g = torch.where(s["label"] >= 0, s["g_logp"], torch.zeros_like(s["g_logp"]))[:, None]
    mass = g + s["g_top"].sum(1, keepdim=True) if case["top"] else g
    surprise = torch.where(e > 0, a - total.log() + _entropy(a, e, total), torch.zeros_like(a))
    d = -p * (mass + s["g_entropy"][:, None] * surprise)
    d.scatter_add_(1, label, g)
    if case["top"]:
        d.scatter_add_(1, s["index"].long(), s["g_top"])
    return torch.where(some, d / case["temperature"], torch.zeros_like(d)).to(s["x"].dtype)


def _plain_distill(s):
    case, x = s["case"], s["x"].float()
    tau, hard, soft = case["temperature"], case["hard"], case["soft"]
    there, at = s["index"] >= 0, s["index"].clamp(min=0).long()
    t = torch.where(there, s["teacher"] / tau, torch.full_like(s["teacher"], -INF))
    b, w, w_sum, _ = _sums(t, 1.0)
    some = w_sum > 0
    q = torch.where(some, w / w_sum, torch.zeros_like(w))
    a, e, total, _ = _sums(x, tau)
    kl = torch.where(q > 0, q * ((b - w_sum.log()) - (a.gather(1, at) - total.log())), torch.zeros_like(q)).sum(1)
    grad = torch.where(some, e / total, torch.zeros_like(e))
    grad.scatter_add_(1, at, -q)
    grad *= soft / tau
    a, e, total, _ = _sums(x, 1.0)
    ce = -_at(a, total, s["label"])
    label = (s["label"] >= 0)[:, None]
    grad += hard * torch.where(label, e / total, torch.zeros_like(e))
    grad.scatter_add_(1, s["label"].clamp(min=0).long()[:, None], -hard * label.float())
    return dict(ce=ce, kl=kl, grad=(grad * s["weight"][:, None]).to(s["x"].dtype))


def _plain_head(s):
    x = s["x"].float() @ s["W"].float().t() + s["bias"]
    a, e, total, m = _sums(x, s["case"]["temperature"])
    return dict(logp=_at(a, total, s["label"]), lse=(m / s["case"]["temperature"] + total.log())[:, 0],
                entropy=_entropy(a, e, total)[:, 0])


def run(state):
    s, case = state, state["case"]
    kind = case["kind"]
    if not own:
        if kind == "score":
            return _plain_score(s)
        if kind == "gradient":
            return _plain_gradient(s)
        if kind == "distill":
            return _plain_distill(s)
        return _plain_head(s)
    from paper_2608_13144_amd import api
    if kind == "score":
        out = api.logprobs(s["x"], s["label"], top=case["top"], temperature=case["temperature"])
        found = dict(logp=out.logp, lse=out.lse, entropy=out.entropy)
        return dict(found, index=out.top_index, top=out.top_logp) if case["top"] else found
    if kind == "gradient":
        return api.logprobs_backward(s["x"], s["label"], g_logp=s["g_logp"], g_entropy=s["g_entropy"],
                                     top_index=s.get("index"), g_top=s.get("g_top"), temperature=case["temperature"])
    if kind == "distill":
        out = api.distill(s["x"], s["teacher"], s["index"], s["label"], weight=s["weight"], hard=case["hard"],
                          soft=case["soft"], temperature=case["temperature"])
        return dict(ce=out.ce, kl=out.kl, grad=out.grad)
    out = api.head_logprobs(s["x"], s["W"], s["bias"], s["label"], temperature=case["temperature"])
    return dict(logp=out.logp, lse=out.lse, entropy=out.entropy)


# ------------------------------------------------------------------ work and the definition in 64 bits
def work(case):
    """Bytes of the inputs and outputs, and operations: an exponential, a sum and a product with its sum for each logit."""
    kind, T, C, e = case["kind"], case["T"], case["C"], SIZE[case["dtype"]]
    if kind == "head":
        K = case["K"]
        return {"bytes": (T + C) * K * e + 4 * C + 16 * T, "flops": 2.0 * T * K * C + 4.0 * T * C}
    size = T * C
    if kind == "score":
        return {"bytes": size * e + 16 * T + 8 * T * case["top"], "flops": 4.0 * size}
    if kind == "gradient":
        return {"bytes": 2 * size * e + 12 * T + 8 * T * case["top"], "flops": 6.0 * size}
    return {"bytes": 2 * size * e + 16 * T + 8 * T * case["k"], "flops": 6.0 * size}


def _rows_of(T, C):
    """Rows of 64-bit numbers that are worked on at a time."""
    step = max(1, (1 << 27) // C)
    return [slice(i, min(T, i + step)) for i in range(0, T, step)]


def _exact_score(logits, label, tau, top):
    y = logits.double() / tau
    lse = torch.logsumexp(y, 1)
    z = y - torch.where(lse == -INF, torch.zeros_like(lse), lse)[:, None]
    p = z.exp()
    rows = torch.arange(len(y), device=DEV)
    logp = torch.where(label >= 0, z[rows, label.clamp(min=0).long()], torch.zeros_like(lse))
    out = dict(logp=logp, lse=lse, entropy=-torch.special.xlogy(p, p).sum(1))
    if top:
        value, at = torch.sort(logits.double(), dim=1, descending=True, stable=True)
        value, at = value[:, :top], at[:, :top]
        out["index"] = torch.where(value > -INF, at, torch.full_like(at, NONE)).to(torch.int32)
        out["top"] = z.gather(1, at)
    return out


def _exact_gradient(s, r):
    case = s["case"]
    y = s["x"][r].double() / case["temperature"]
    empty = (y == -INF).all(1)
    y[empty] = 0.0
    p = torch.softmax(y, 1)
    total = torch.zeros_like(p)  # the gradient with regard to log p_j, as far as it goes through labels and alternatives
    rows = torch.arange(len(p), device=DEV)
    has = s["label"][r] >= 0
    total[rows[has], s["label"][r][has].long()] += s["g_logp"][r][has].double()
    if case["top"]:
        total.scatter_add_(1, s["index"][r].long(), s["g_top"][r].double())
    grad = total - p * total.sum(1, keepdim=True)
    plogp = torch.special.xlogy(p, p)
    entropy = -plogp.sum(1, keepdim=True)
    grad -= s["g_entropy"][r].double()[:, None] * (plogp + p * entropy)
    grad[empty] = 0.0
    return grad / case["temperature"]


def _exact_distill(s, r):
    case = s["case"]
    x, tau = s["x"][r].double(), case["temperature"]
    index = s["index"][r].long()
    there = index >= 0
    some = there.any(1)
    t = (s["teacher"][r].double() / tau).masked_fill(~there, -INF)
    q = torch.softmax(torch.where(some[:, None], t, torch.zeros_like(t)), 1) * there
    full = torch.zeros_like(x).scatter_add_(1, index.clamp(min=0), q)
    logp = torch.log_softmax(x / tau, 1)
    kl = (torch.special.xlogy(full, full) - full * logp).sum(1)
    grad = (case["soft"] / tau) * (logp.exp() * some[:, None] - full)
    logp = torch.log_softmax(x, 1)
    has = s["label"][r] >= 0
    hit = torch.zeros_like(x)
    hit[torch.arange(len(x), device=DEV)[has], s["label"][r][has].long()] = 1.0
    ce = -(hit * logp).sum(1)
    grad += case["hard"] * (logp.exp() * has[:, None] - hit)
    return dict(ce=ce, kl=kl, grad=grad * s["weight"][r].double()[:, None])


def exact(case, seed):
    s = prepare(case, seed)
    kind, T, C = case["kind"], case["T"], case["C"]
    found = []
    for r in _rows_of(T, C):
        if kind == "gradient":
            found.append(dict(grad=_exact_gradient(s, r)))
        elif kind == "distill":
            found.append(_exact_distill(s, r))
        elif kind == "score":
            found.append(_exact_score(s["x"][r], s["label"][r], case["temperature"], case["top"]))
        else:
            logits = torch.addmm(s["bias"].double(), s["x"][r].double(), s["W"].double().t())
            found.append(_exact_score(logits, s["label"][r], case["temperature"], 0))
    out = {name: torch.cat([f[name] for f in found]) for name in found[0]}
    return out["grad"] if kind == "gradient" else out
