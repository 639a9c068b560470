"""The measured cases of the operators that adapt a shared head: low-rank adapters and orthogonalised updates.

A proxy that serves many sites keeps one shared projection W and, for each site, a
low-rank pair (A_s, B_s).  A batch mixes requests of many sites, some without an
adapter.  Their training takes the gradients of the pairs and steps along an
orthogonalised momentum, whose singular values are near 1, so a step moves the
projection's spectral norm (which divides every certified radius) by a known amount.

Kinds of case (``case["kind"]``):

  forward        y = W x + bias + s_a B_a (A_a x) for every row x of a batch, with the
                 request's adapter a (``api.adapter_forward``)
  backward       gradients of the rows and of every adapter's pair
                 (``api.adapter_backward``; W and bias are frozen)
  orthogonalise  Newton-Schulz products of a stack of matrices (``api.orthogonalise``)
  step           momentum, orthogonalisation and the update of a stack of parameters
                 (``api.muon_step``, in place)

Sizes: rows of d = 256 features and C = 200 classes are this library's headline
head; 1024 to 8192 are generic projection widths.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
STEPS = 5
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
EPS = 1e-7
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.01


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # Logits of the headline head for single queries of 64 sites: one row a request, float32 as certified.
        dict(name="logits-sites", kind="forward", dtype="f32", T=1024, K=256, N=200, S=64, r=8, requests=1024,
             none=0.1, keep=False, strided=False),
        # The smallest serving call: one row through a wide projection and one adapter; latency.
        dict(name="decode-one", kind="forward", dtype="bf16", T=1, K=4096, N=4096, S=32, r=16, requests=1,
             none=0.0, keep=False, strided=False),
        # A decode batch: 64 requests of one row each, nearly all with adapters of their own.
        dict(name="decode-batch", kind="forward", dtype="bf16", T=64, K=4096, N=4096, S=64, r=16, requests=64,
             none=0.1, keep=False, strided=False),
        # Mixed lengths (empty requests and single rows among them), odd row count and output width, rows inside a
        # wider buffer.
        dict(name="mixed-ragged", kind="forward", dtype="f16", T=3001, K=2000, N=5003, S=12, r=24, requests=29,
             none=0.2, keep=True, strided=True),
        # The largest serving call: long prompts of a few sites.
        dict(name="prefill", kind="forward", dtype="bf16", T=8192, K=4096, N=8192, S=4, r=64, requests=5,
             none=0.0, keep=False, strided=False),
        # Training the sites' pairs on the headline head, float32.
        dict(name="train-sites", kind="backward", dtype="f32", T=4096, K=256, N=200, S=16, r=8, requests=64,
             none=0.0, strided=False),
        # A ragged training batch of moderate width.
        dict(name="train-ragged", kind="backward", dtype="f16", T=1777, K=1024, N=1536, S=7, r=16, requests=19,
             none=0.1, strided=True),
        # The largest training call: 8192 rows of four sites through a square projection.
        dict(name="train-wide", kind="backward", dtype="bf16", T=8192, K=4096, N=4096, S=4, r=32, requests=8,
             none=0.0, strided=False),
        # Orthogonalising the headline head itself, float32.
        dict(name="ortho-head", kind="orthogonalise", dtype="f32", b=1, m=200, n=256),
        # Tall float16 matrices of odd sizes.
        dict(name="ortho-odd", kind="orthogonalise", dtype="f16", b=3, m=1000, n=777),
        # A step on the A factors of 64 sites: many small wide matrices.
        dict(name="step-factors", kind="step", dtype="bf16", b=64, m=16, n=4096),
        # A step on a wide projection: the largest matrices.
        dict(name="step-projection", kind="step", dtype="bf16", b=1, m=4096, n=4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: three times in four a multiple of eight, else any number."""
    w = _log_int(rng, lo, hi)
    return w if rng.random() < 0.25 else max(8, 8 * (w // 8))


def draw(rng):
    """One more case of the ranges above."""
    kind = rng.choice(["forward", "forward", "backward", "orthogonalise", "step"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if kind in ("forward", "backward"):
        most = (1 << 34) if dtype == "f32" else (1 << 37)  # T K N
        K = _width(rng, 64, 4096)
        N = _width(rng, 10, 8192 if kind == "forward" else 4096)
        T = _log_int(rng, 1 if kind == "forward" else 16, max(32, min(8192, most // (K * N))))
        r = rng.choice([1, 4, 8, 16, 16, 24, 32, 64])
        S = _log_int(rng, 1, max(2, min(64, 1024 // r)))
        requests = T if rng.random() < 0.3 and T <= 1024 else min(max(1, T), _log_int(rng, 1, 64))
        c = dict(kind=kind, dtype=dtype, T=T, K=K, N=N, S=S, r=r, requests=requests,
                 none=rng.choice([0.0, 0.1, 0.3]), strided=rng.random() < 0.3)
        if kind == "forward":
            c["keep"] = rng.random() < 0.4
        return c
    m, n = _width(rng, 8, 4096), _width(rng, 8, 4096)
    b = _log_int(rng, 1, max(2, min(64, (1 << 24) // (m * n), (1 << 34) // (min(m, n) ** 2 * max(m, n)))))
    return dict(kind=kind, dtype=dtype, b=b, m=m, n=n)


# ------------------------------------------------------------------ inputs
def _generators(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    h = torch.Generator()
    h.manual_seed(seed)
    return g, h


def _requests(case, h):
    """Request borders (empty requests among them where there are fewer requests than rows) and their adapters."""
    T, R = case["T"], case["requests"]
    if R == T:
        cuts = torch.arange(T + 1)
    else:
        inner = torch.randint(0, T + 1, (R - 1,), generator=h).sort().values
        cuts = torch.cat([torch.zeros(1, dtype=torch.int64), inner, torch.full((1,), T)])
    adapter = torch.randint(0, case["S"], (R,), generator=h)
    adapter[torch.rand(R, generator=h) < case["none"]] = -1
    return cuts.to(torch.int32), adapter.to(torch.int32)


def _gradient(g, b, m, n):
    """Gradient-like: a few strong directions over noise, small in size."""
    k = min(8, m, n)
    strong = torch.randn(b, m, k, generator=g, device=DEV) @ torch.randn(b, k, n, generator=g, device=DEV)
    return 1e-3 * (strong / math.sqrt(k) + torch.randn(b, m, n, generator=g, device=DEV))


def _rows(g, case, width, dtype):
    """[T, width] rows, inside a wider buffer where the case says so."""
    room = width + (-width) % 8 + 64 if case["strided"] else width
    return torch.randn(case["T"], room, generator=g, device=DEV).to(dtype)[:, :width]


def prepare(case, seed):
    g, h = _generators(seed)
    dtype = DTYPES[case["dtype"]]
    s = dict(case=case)
    if case["kind"] in ("orthogonalise", "step"):
        b, m, n = case["b"], case["m"], case["n"]
        s["G"] = _gradient(g, b, m, n).to(dtype)
        if case["kind"] == "step":
            s["W"] = (torch.randn(b, m, n, generator=g, device=DEV) / math.sqrt(n)).to(dtype)
            s["M"] = 5.0 * _gradient(g, b, m, n)
        return s
    K, N, S, r = case["K"], case["N"], case["S"], case["r"]
    s["x"] = _rows(g, case, K, dtype)
    s["W"] = (torch.randn(N, K, generator=g, device=DEV) / math.sqrt(K)).to(dtype)
    s["bias"] = 0.1 * torch.randn(N, generator=g, device=DEV)
    s["A"] = (torch.randn(S, r, K, generator=g, device=DEV) / math.sqrt(K)).to(dtype)
    s["B"] = (0.3 * torch.randn(S, N, r, generator=g, device=DEV) / math.sqrt(r)).to(dtype)
    s["scale"] = torch.rand(S, generator=g, device=DEV) + 0.5
    offsets, adapter = _requests(case, h)
    s["offsets"], s["adapter"] = offsets.to(DEV), adapter.to(DEV)
    if case["kind"] == "backward":
        s["dy"] = (_rows(g, case, N, torch.float32) / math.sqrt(case["T"])).to(dtype)
        # what the forward pass keeps: A_a x of every row
        s["v"] = _shrink(s["x"].float(), s["A"].float(), _pick(s)).sum(1)
    return s


# ------------------------------------------------------------------ plain forms
def _pick(s):
    """[T, S] of 0 and 1: the adapter of each row (none: a row of zeros)."""
    T, S = s["x"].shape[0], s["A"].shape[0]
    row = torch.arange(T, device=DEV, dtype=s["offsets"].dtype)
    request = torch.searchsorted(s["offsets"], row, right=True) - 1
    return (s["adapter"][request][:, None] == torch.arange(S, device=DEV)).float()


def _shrink(x, A, pick):
    """[T, S, r]: A_s x where s is the row's adapter, zero elsewhere."""
    S, r, K = A.shape
    return (x @ A.reshape(S * r, K).t()).view(-1, S, r) * pick[:, :, None]


def _plain_forward(s):
    x, W, A, B = s["x"].float(), s["W"].float(), s["A"].float(), s["B"].float()
    S, r, _ = A.shape
    v = _shrink(x, A, _pick(s))
    y = x @ W.t() + s["bias"]
    y += (v * s["scale"][:, None]).view(-1, S * r) @ B.permute(0, 2, 1).reshape(S * r, -1)
    y = y.to(s["x"].dtype)
    return dict(y=y, v=v.sum(1)) if s["case"]["keep"] else dict(y=y)


def _plain_backward(s):
    x, W, A, B, dy = s["x"].float(), s["W"].float(), s["A"].float(), s["B"].float(), s["dy"].float()
    S, r, K = A.shape
    N = W.shape[0]
    pick = _pick(s) * s["scale"]
    u = ((dy @ B.permute(1, 0, 2).reshape(N, S * r)).view(-1, S, r) * pick[:, :, None]).view(-1, S * r)
    dx = dy @ W + u @ A.view(S * r, K)
    dA = (u.t() @ x).view(S, r, K)
    v = (s["v"][:, None, :] * pick[:, :, None]).view(-1, S * r)
    dB = (dy.t() @ v).view(N, S, r).permute(1, 0, 2)
    return dict(dx=dx.to(s["x"].dtype), dA=dA.to(s["A"].dtype), dB=dB.to(s["B"].dtype))


def _plain_orthogonalise(G):
    a, b, c = COEFFICIENTS
    X = G.float()
    X = X / (X.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    tall = X.shape[1] > X.shape[2]
    X = X.transpose(1, 2).contiguous() if tall else X
    for _ in range(STEPS):
        P = X @ X.transpose(1, 2)
        X = a * X + (b * P + c * (P @ P)) @ X
    return X.transpose(1, 2) if tall else X


def _plain_step(s):
    W, M, G = s["W"], s["M"], s["G"].float()
    M.mul_(MOMENTUM).add_(G)
    O = _plain_orthogonalise(MOMENTUM * M + G)
    m, n = W.shape[1:]
    W.copy_((1.0 - LR * DECAY) * W.float() - LR * math.sqrt(max(1.0, m / n)) * O)
    return dict(W=W, M=M)


def run(state):
    s, kind = state, state["case"]["kind"]
    if not own:
        if kind == "forward":
            return _plain_forward(s)
        if kind == "backward":
            return _plain_backward(s)
        if kind == "orthogonalise":
            return _plain_orthogonalise(s["G"]).to(s["G"].dtype)
        return _plain_step(s)
    from paper_2608_13144_amd import api
    if kind == "forward":
        out = api.adapter_forward(s["x"], s["W"], s["bias"], s["A"], s["B"], s["scale"], s["offsets"], s["adapter"],
                                  keep=s["case"]["keep"])
        return dict(y=out.y, v=out.v) if s["case"]["keep"] else dict(y=out.y)
    if kind == "backward":
        out = api.adapter_backward(s["dy"], s["x"], s["W"], s["A"], s["B"], s["scale"], s["offsets"], s["adapter"],
                                   v=s["v"])
        return dict(dx=out.dx, dA=out.dA, dB=out.dB)
    if kind == "orthogonalise":
        return api.orthogonalise(s["G"], steps=STEPS, coefficients=COEFFICIENTS, eps=EPS)
    api.muon_step(s["W"], s["G"], s["M"], lr=LR, momentum=MOMENTUM, weight_decay=DECAY, nesterov=True, steps=STEPS,
                  coefficients=COEFFICIENTS, eps=EPS)
    return dict(W=s["W"], M=s["M"])


# ------------------------------------------------------------------ work and the definition in 64 bits
def work(case):
    e = SIZE[case["dtype"]]
    if case["kind"] in ("orthogonalise", "step"):
        b, m, n = case["b"], case["m"], case["n"]
        p, q = min(m, n), max(m, n)
        # a symmetric product needs half its entries; powers of the p x p Gram matrix carry the iteration:
        # one Gram matrix, per step A^2 and the running product, the next A but for the last step, one application
        product = p * p * (p + 1.0)
        flops = b * (p * (p + 1.0) * q + STEPS * product + (STEPS - 1) * 3 * product + 2.0 * p * p * q)
        size = b * m * n
        return {"bytes": size * (2 * e if case["kind"] == "orthogonalise" else 3 * e + 8), "flops": flops}
    T, K, N, r = case["T"], case["K"], case["N"], case["r"]
    used = min(case["S"], case["requests"])
    pairs = used * r * (K + N) * e
    if case["kind"] == "forward":
        return {"bytes": (T * K + N * K + T * N) * e + pairs + 4 * N + (4 * T * r if case["keep"] else 0),
                "flops": 2.0 * T * K * N + 2.0 * T * r * (K + N)}
    return {"bytes": (2 * T * K + T * N + N * K) * e + pairs + case["S"] * r * (K + N) * e + 4 * T * r,
            "flops": 2.0 * T * K * N + 4.0 * T * r * (K + N)}


def _exact_orthogonalise(G):
    """The same iteration in float64, each step as X (a + b Z + c Z^2) with Z = X^T X on the smaller side."""
    a, b, c = COEFFICIENTS
    X = G.double()
    X = X / (torch.linalg.vector_norm(X, dim=(1, 2), keepdim=True) + EPS)
    wide = X.shape[2] > X.shape[1]
    X = X.mT.contiguous() if wide else X
    eye = torch.eye(X.shape[2], dtype=torch.float64, device=DEV)
    for _ in range(STEPS):
        Z = torch.matmul(X.mT.contiguous(), X)
        X = torch.matmul(X, a * eye + torch.matmul(Z, b * eye + c * Z))
    return X.mT if wide else X


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "orthogonalise":
        return _exact_orthogonalise(s["G"])
    if case["kind"] == "step":
        M = MOMENTUM * s["M"].double() + s["G"].double()
        O = _exact_orthogonalise(MOMENTUM * M + s["G"].double())
        W = s["W"].double()
        return dict(W=W - LR * DECAY * W - LR * max(1.0, case["m"] / case["n"]) ** 0.5 * O, M=M)
    x, W = s["x"].double(), s["W"].double()
    off, ids = s["offsets"].tolist(), s["adapter"].tolist()
    if case["kind"] == "forward":
        y = torch.addmm(s["bias"].double(), x, W.mT)
        v = torch.zeros(case["T"], case["r"], dtype=torch.float64, device=DEV)
        for i, a in enumerate(ids):
            lo, hi = off[i], off[i + 1]
            if a < 0 or hi == lo:
                continue
            v[lo:hi] = x[lo:hi] @ s["A"][a].double().mT
            y[lo:hi] += s["scale"][a].double() * (v[lo:hi] @ s["B"][a].double().mT)
        return dict(y=y, v=v) if case["keep"] else dict(y=y)
    dy, v = s["dy"].double(), s["v"].double()
    dx = dy @ W
    dA = torch.zeros(s["A"].shape, dtype=torch.float64, device=DEV)
    dB = torch.zeros(s["B"].shape, dtype=torch.float64, device=DEV)
    for i, a in enumerate(ids):
        lo, hi = off[i], off[i + 1]
        if a < 0 or hi == lo:
            continue
        u = s["scale"][a].double() * (dy[lo:hi] @ s["B"][a].double())
        dx[lo:hi] += u @ s["A"][a].double()
        dA[a] += u.mT @ x[lo:hi]
        dB[a] += s["scale"][a].double() * (dy[lo:hi].mT @ v[lo:hi])
    return dict(dx=dx, dA=dA, dB=dB)
