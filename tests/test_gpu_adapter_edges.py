"""Adapters at their edges: what the passes work out in between keeps float32's digits, requests keep apart."""
import numpy as np
import pytest
import torch

from gpu_helpers import say
from paper_2608_13144_amd import api
from test_gpu_adapter import DEV, DT, n64

pytestmark = pytest.mark.gpu


def ints(g, lo, hi, *shape):
    return torch.randint(lo, hi + 1, shape, generator=g).float()


def one_hot(width, at):
    return torch.nn.functional.one_hot(at % width, width).float()


def batch(T, S, g, dtype, x, W, A, B):
    cuts = torch.randint(0, T + 1, (6,), generator=g).sort().values
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), cuts, torch.full((1,), T)])
    adapter = torch.arange(7) % S
    cast = lambda t: t.to(DT[dtype]).to(DEV)  # noqa: E731
    for t in (x, W, A, B):
        assert torch.equal(t.to(DT[dtype]).float(), t)
    return dict(x=cast(x), W=cast(W), A=cast(A), B=cast(B), scale=torch.ones(S, device=DEV), offsets=offsets.int().to(DEV),
                adapter=adapter.int().to(DEV)), torch.repeat_interleave(adapter, offsets[1:] - offsets[:-1])


# Whole numbers whose sums stay below 2^24 are exact in float32, whatever the order.  A x and B^T dy take 17 to 21 bits here
# and nearly cancel against W's part, or in pairs of rows, so that a digit lost in between is whole units of the result.
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T", [50, 8300])
def test_forward_keeps_every_digit_of_what_lies_between(dtype, T):
    say("digits of v", T, dtype)
    g = torch.Generator().manual_seed(T)
    S, r, K, N = 2, 3, 64, 48
    A = ints(g, 0, 100, r, K).expand(S, r, K).contiguous()
    rho = torch.arange(N) % r
    B = one_hot(r, rho).expand(S, N, r).contiguous()
    keep = torch.arange(N) % K
    W = one_hot(K, keep) - A[0][rho]  # y = x[keep]
    x = ints(g, 0, 255, T, K)
    b, _ = batch(T, S, g, dtype, x, W, A, B)
    y = api.adapter_forward(b["x"], b["W"], None, b["A"], b["B"], b["scale"], b["offsets"], b["adapter"]).y
    assert torch.equal(y.float().cpu(), x[:, keep])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,r", [(50, 3), (700, 3), (700, 20), (700, 40), (700, 100)])
def test_backward_keeps_every_digit_of_what_lies_between(dtype, T, r):
    say("digits of u and v", T, r, dtype)
    g = torch.Generator().manual_seed(T + r)
    S, K, N = 2, 64, 512
    # ranks past the third are zeros in A and small in B, so that the sums stay exact
    A = torch.zeros(S, r, K)
    A[:, -3:] = ints(g, 0, 7, 3, K)
    rho = torch.arange(N) % 3
    B = torch.zeros(S, N, r)
    B[:, :, -3:] = one_hot(3, rho) * ints(g, 1, 15, N, 1)
    W = one_hot(K, torch.arange(N)) - B[0] @ A[0]  # dx: the sums of dy over the n of each column
    dy = ints(g, 0, 127, T, N)
    n0 = torch.randint(0, N, (T // 2,), generator=g)
    dy[1::2] = -dy[0::2]
    dy[1::2] += one_hot(N, n0)
    x = ints(g, 0, 3, T // 2, K).repeat_interleave(2, 0)
    v = ints(g, -(1 << 20), 1 << 20, T // 2, r).repeat_interleave(2, 0)
    b, pair = batch(T, S, g, dtype, x, W, A, B)
    b["offsets"] = (b["offsets"] // 2 * 2).int()  # pairs of rows stay in one request
    pair = torch.repeat_interleave(b["adapter"].cpu().long(), (b["offsets"][1:] - b["offsets"][:-1]).cpu().long())
    args = [b[k] for k in ("x", "W", "A", "B", "scale", "offsets", "adapter")]
    out = api.adapter_backward(dy.to(DT[dtype]).to(DEV), *args, v=v.to(DEV))
    exact = lambda t: t.to(DT[dtype]).double()  # noqa: E731  (rounded once)
    dx = dy.double() @ one_hot(K, torch.arange(N)).double()
    assert torch.equal(out.dx.double().cpu(), exact(dx))
    u = dy.double() @ B[0].double()
    dA = torch.stack([u[pair == a].T @ x[pair == a].double() for a in range(S)])
    assert torch.equal(out.dA.double().cpu(), exact(dA))
    # dB: a second row's v is minus the first's, and a little
    v[1::2] = -v[0::2] + ints(g, 0, 3, T // 2, r)
    dz = ints(g, -1, 1, T // 2, N).repeat_interleave(2, 0)
    out = api.adapter_backward(dz.to(DT[dtype]).to(DEV), *args, v=v.to(DEV), want_dx=False)
    dB = torch.stack([dz[pair == a].double().T @ v[pair == a].double() for a in range(S)])
    assert torch.equal(out.dB.double().cpu(), exact(dB))
    assert np.isfinite(n64(out.dB)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T", [64, 700, 8300])
def test_rows_of_other_requests_cost_no_digits(dtype, T):
    """Every fifth row's A x (B^T dy) is 2^35, the others' below 2^12 with eight digits after the point: none of them is lost."""
    say("rows of different size", T, dtype)
    g = torch.Generator().manual_seed(T)
    S, r, K, N = 1, 3, 64, 64
    rho = torch.arange(N) % r
    big = torch.zeros(T, dtype=torch.bool)
    big[::5] = True

    def rows(top):  # whole numbers / 256 in the first half of the columns, or 2^15 in the second
        x = torch.zeros(T, 64)
        x[:, :32] = ints(g, 0, top, T, 32) / 256
        x[big, :32] = 0
        x[big, 32:] = 32768
        return x
    half = torch.zeros(64)
    half[:32] = 1
    A = ints(g, 0, 100, S, r, K) * half + 32768 * (1 - half)
    B = one_hot(r, rho).expand(S, N, r).contiguous()
    keep = torch.arange(N) % 32
    W = one_hot(K, keep) - A[0][rho]  # y = x[keep]
    x = rows(255)
    b, _ = batch(T, S, g, dtype, x, W, A, B)
    y = api.adapter_forward(b["x"], b["W"], None, b["A"], b["B"], b["scale"], b["offsets"], b["adapter"]).y
    assert torch.equal(y.float().cpu(), x[:, keep])
    # backward: dx = dy in the first half, zero in the second
    A = ints(g, 0, 1, S, r, K)
    B = (one_hot(r, rho) * (ints(g, 1, 100, N, 1) * half[:, None] + 32768 * (1 - half[:, None]))).expand(S, N, r).contiguous()
    W = torch.diag(half) - B[0] @ A[0]
    dy = rows(255)
    b, _ = batch(T, S, g, dtype, x, W, A, B)
    out = api.adapter_backward(dy.to(DT[dtype]).to(DEV), *[b[k] for k in ("x", "W", "A", "B", "scale", "offsets", "adapter")])
    assert torch.equal(out.dx.float().cpu(), dy * half)


@pytest.mark.parametrize("T", [40, 300])
def test_keep_with_an_output_of_the_callers(T):
    g = torch.Generator().manual_seed(T)
    b, _ = batch(T, 2, g, "f32", ints(g, -9, 9, T, 96), ints(g, -9, 9, 40, 96), ints(g, -9, 9, 2, 4, 96), ints(g, -9, 9, 2, 40, 4))
    args = [b["x"], b["W"], None] + [b[k] for k in ("A", "B", "scale", "offsets", "adapter")]
    ref = api.adapter_forward(*args, keep=True)
    out = api.AdapterOutput(torch.empty_like(ref.y), None)
    y = out.y
    assert api.adapter_forward(*args, keep=True, out=out) is out and out.y is y
    assert out.v is not None and torch.equal(out.v, ref.v) and torch.equal(out.y, ref.y)
    out = api.AdapterOutput(torch.empty_like(ref.y), None)
    assert api.adapter_forward(*args, out=out).v is None and torch.equal(out.y, ref.y)
    out = api.AdapterOutput(torch.empty_like(ref.y), torch.empty_like(ref.v))
    v = out.v
    assert api.adapter_forward(*args, out=out).v is v and torch.equal(v, ref.v)


# Sizes whose kernels have more workgroups than a launch takes (2^32 threads).
def test_copies_of_more_workgroups_than_a_launch_takes():
    T, K = (1 << 28) + 100, 33
    say("copies", T, K)
    x = torch.empty(T, K, dtype=torch.bfloat16, device=DEV).random_(-4, 5)
    W = torch.ones(1, K, dtype=torch.bfloat16, device=DEV)
    none = torch.empty(0, 1, K, dtype=torch.bfloat16, device=DEV)
    y = api.adapter_forward(x, W, None, none, torch.empty(0, 1, 1, dtype=torch.bfloat16, device=DEV), torch.empty(0, device=DEV),
                            torch.tensor([0, T], dtype=torch.int32, device=DEV), torch.tensor([-1], dtype=torch.int32, device=DEV)).y
    for t in range(0, T, 1 << 25):
        assert torch.equal(y[t:t + (1 << 25), 0], x[t:t + (1 << 25)].float().sum(1).bfloat16()), t


def test_rows_of_more_workgroups_than_a_launch_takes():
    T, K, N = (1 << 29) + 64, 8, 8
    say("rows", T)
    g = torch.Generator().manual_seed(1)
    at = torch.cat([torch.randint(0, T, (2000,), generator=g), torch.tensor([0, T - 1])]).unique()
    n = at.numel()
    sx, sdy, sv, B = ints(g, -3, 3, n, K), ints(g, -3, 3, n, N), ints(g, -9, 9, n, 1), ints(g, -3, 3, 1, N, 1)
    x, dy = (torch.zeros(T, 8, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    v = torch.zeros(T, 1, device=DEV)
    for full, some in ((x, sx), (dy, sdy), (v, sv)):
        full[at.to(DEV)] = some.to(full.dtype).to(DEV)
    out = api.adapter_backward(dy, x, torch.zeros(N, K, dtype=torch.bfloat16, device=DEV),
                               torch.zeros(1, 1, K, dtype=torch.bfloat16, device=DEV), B.bfloat16().to(DEV), torch.ones(1, device=DEV),
                               torch.tensor([0, 5, T], dtype=torch.int32, device=DEV),
                               torch.tensor([0, 0], dtype=torch.int32, device=DEV), v=v, want_dx=False)
    u = sdy @ B[0]
    assert torch.equal(out.dA[0].cpu(), (u.t() @ sx).bfloat16())
    assert torch.equal(out.dB[0].cpu(), (sdy.t() @ sv).bfloat16())


def test_pairs_of_more_workgroups_than_a_launch_takes():
    T, K, N, S = 6, 1 << 17, 1 << 17, 8192
    say("pairs", S, K, N)
    g = torch.Generator().manual_seed(2)
    x, dy, v = ints(g, -3, 3, T, K), ints(g, -1, 1, T, N), ints(g, -9, 9, T, 1)
    B = torch.empty(S, N, 1, dtype=torch.bfloat16, device=DEV).random_(-1, 2)
    adapter = torch.tensor([5, S - 1, 0, -1, 4097, 5])
    out = api.adapter_backward(dy.bfloat16().to(DEV), x.bfloat16().to(DEV), torch.zeros(N, K, dtype=torch.bfloat16, device=DEV),
                               torch.empty(S, 1, K, dtype=torch.bfloat16, device=DEV), B, torch.ones(S, device=DEV),
                               torch.arange(T + 1, dtype=torch.int32, device=DEV), adapter.int().to(DEV), v=v.to(DEV), want_dx=False)
    used = sorted(set(adapter.tolist()) - {-1})
    for grad in (out.dA, out.dB):
        assert set((grad != 0).flatten(1).any(1).nonzero().flatten().tolist()) <= set(used)
    for a in used:
        t = adapter == a
        assert torch.equal(out.dA[a].cpu(), ((dy[t] @ B[a].float().cpu()).t() @ x[t]).bfloat16())
        assert torch.equal(out.dB[a].cpu(), (dy[t].t() @ v[t]).bfloat16())
