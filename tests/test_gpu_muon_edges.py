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


CUBIC = (15 / 8, -10 / 8, 3 / 8)


def deficient(seed, kind, b, m, n, dtype):
    """Matrices of whole numbers with an exact null space: rank 1, rank 4, equal halves, rows of zero; or full rank."""
    g = torch.Generator().manual_seed(seed)
    p = min(m, n)
    ints = lambda *s: torch.randint(-3, 4, s, generator=g).float()  # noqa: E731
    if kind in ("rank 1", "rank 4"):
        k = min(1 if kind == "rank 1" else 4, p)
        G = ints(b, m, k) @ ints(b, k, n)
    else:
        G = ints(b, p, max(m, n)) + torch.eye(p, max(m, n))
        if kind == "halves":
            G[:, p // 2:2 * (p // 2)] = G[:, :p // 2]
        elif kind == "zeros":
            G[:, 1::3] = 0
        G = G if m <= n else G.transpose(1, 2).contiguous()
    out = G.to({"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype])
    assert torch.equal(out.float(), G) and bool((G.abs().sum((1, 2)) > 0).all())
    return out.to(DEV)


def by_singular_values(G, coefficients, eps):
    """The iteration on the singular values, in float64: what is zero stays zero.  Also the projector on G's columns."""
    u, s, vt = np.linalg.svd(G, full_matrices=False)
    s = np.where(s > 1e-9 * s[:, :1], s, 0.0)
    t = s / (np.sqrt(np.sum(s * s, axis=1, keepdims=True)) + eps)
    for a, b, c in coefficients:
        t = t * (a + t * t * (b + c * t * t))
    u1 = u * (s > 0)[:, None, :]
    return (u * t[:, None, :]) @ vt, u1 @ u1.transpose(0, 2, 1)


def amplified(coefficients):
    """What the steps make of float64's rounding, 2^-53, in directions that G does not have."""
    return 2.0 ** -53 * float(np.prod([max(1.0, abs(c[0])) for c in coefficients]))


@pytest.mark.parametrize("kind", ["rank 1", "rank 4", "halves", "zeros", "full"])
@pytest.mark.parametrize("shape", [(2, 8, 256), (3, 16, 40), (1, 300, 30), (2, 33, 500), (1, 64, 256), (1, 256, 64), (1, 1, 9)],
                         ids=lambda s: "x".join(map(str, s)))
def test_short_matrices_and_many_steps(shape, kind):
    """Singular values stay below the last step's bound, and the result is the float64 one, also on a null space."""
    for dtype in ("f32", "bf16"):
        G = deficient(sum(shape), kind, *shape, dtype)
        for name, one, counts in (("usual", api.NEWTON_SCHULZ, (7, 8, 12, 16, 20, 32)), ("cubic", CUBIC, (12, 24, 32))):
            one = tuple(float(np.float32(c)) for c in one)
            for steps in counts:
                say("many steps", shape, kind, dtype, name, steps)
                O = n64(api.orthogonalise(G, steps=steps, coefficients=one))
                assert np.isfinite(O).all()
                # rounding to bfloat16 moves a singular value by at most 2^-8 of the Frobenius norm
                slack = 1e-5 + (2.0 ** -8 * np.sqrt(min(shape[1:])) if dtype == "bf16" else 0.0)
                assert np.linalg.svd(O, compute_uv=False).max() <= 1.21 + slack
                ref, columns = by_singular_values(n64(G), [one] * steps, float(np.float32(1e-7)))
                grown = 64 * amplified([one] * steps)
                off = O - ref if grown < 1e-5 else columns @ (O - ref)  # what rounding makes of nothing is no error
                tol = R.NS_TOL["f32"] + (R.U["bf16"] if dtype == "bf16" else 0.0) + min(1e-5, grown)
                assert np.linalg.norm(off) <= tol * np.linalg.norm(ref), np.linalg.norm(off) / np.linalg.norm(ref)
        G = deficient(sum(shape), kind, *shape, dtype)
        W, M = torch.zeros_like(G), torch.zeros(shape, device=DEV)
        api.muon_step(W, G, M, lr=1.0, momentum=0.5, nesterov=False, scale=1.0, steps=16)
        assert np.array_equal(n64(M), n64(G))
        ref, _ = by_singular_values(n64(G), [tuple(float(np.float32(c)) for c in api.NEWTON_SCHULZ)] * 16, float(np.float32(1e-7)))
        assert far(W, -ref) <= R.NS_TOL["f32"] + (R.U["bf16"] if dtype == "bf16" else 0.0) + 1e-5


@pytest.mark.parametrize("kind", ["rank 1", "halves", "full"])
@pytest.mark.parametrize("shape", [(2, 72, 200), (1, 150, 70)], ids=lambda s: "x".join(map(str, s)))
def test_other_matrices_and_many_steps(shape, kind):
    """Shorter sides above 64 iterate on X itself: singular values stay bounded whatever the steps."""
    for dtype in ("f32", "f16"):
        G = deficient(sum(shape), kind, *shape, dtype)
        for steps in (8, 16, 32):
            say("many steps", shape, kind, dtype, steps)
            s = np.linalg.svd(n64(api.orthogonalise(G, steps=steps)), compute_uv=False)
            assert s.max() <= 1.21 + 1e-3  # float16: 2^-11 of a norm of at most 9 at random angles


@pytest.mark.parametrize("n,what", [(8_600_000, "f32"), (16_519_104, "bf16"), (16_519_104, "step"), (16_519_104, "short step")])
def test_rows_past_31_bits(n, what):
    """65 rows so long that a tile of 64 of them passes 2^31 bytes; one step, against float64 in pieces."""
    m, coef = 65, tuple(float(np.float32(c)) for c in api.NEWTON_SCHULZ)
    say("long rows", n, what)
    g = torch.Generator(device=DEV).manual_seed(n)
    G = torch.randn(m, n, generator=g, device=DEV, dtype=torch.float32 if what == "f32" else torch.bfloat16)
    if what in ("f32", "bf16"):
        O = api.orthogonalise(G, steps=1, eps=0.0)
        sign = 1.0
    else:
        O, M, sign = torch.zeros_like(G), torch.zeros(m, n, device=DEV), -1.0
        api.muon_step(O, G, M, lr=1.0, momentum=0.5, nesterov=False, scale=1.0, steps=1, eps=0.0, short_operands=what == "short step")
        del M
    pieces = [slice(c, min(c + (1 << 20), n)) for c in range(0, n, 1 << 20)]
    P = torch.zeros(m, m, dtype=torch.float64, device=DEV)
    for c in pieces:
        x = G[:, c].double()
        P += x @ x.t().contiguous()
    size = P.trace()
    P /= size
    B = coef[0] * torch.eye(m, dtype=torch.float64, device=DEV) + coef[1] * P + coef[2] * (P @ P)
    wrong = ref2 = 0.0
    for c in pieces:
        ref = sign * (B @ (G[:, c].double() / size.sqrt()))
        wrong += float(((O[:, c].double() - ref) ** 2).sum())
        ref2 += float((ref ** 2).sum())
    # one step: float32's error is below a step's share of five; 11-bit operands as in NS_TOL
    own = 0.0 if what == "f32" else R.U["bf16"]
    assert (wrong / ref2) ** 0.5 <= own + R.NS_TOL["f32"] + (2.6e-3 if what == "short step" else 0.0)


@pytest.mark.parametrize("shape", [(2, 12, 50), (2, 150, 140), (1, 90, 300)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype,size", [("f32", 1e-37), ("f32", 3e-41), ("f32", 6e37), ("bf16", 1e-37), ("bf16", 6e37), ("f16", 1e-6)])
def test_matrices_near_the_ends_of_the_range(shape, dtype, size):
    """No eps: 1 / ||G|| and its multiples pass float32's range, the result does not."""
    say("ends of the range", shape, dtype, size)
    H = matrices(50, *shape, dtype, size=size)
    assert bool(H.isfinite().all()) and bool((H != 0).any())
    ref = R.newton_schulz(n64(H), 5, NS5, 0.0)
    O = api.orthogonalise(H, eps=0.0)
    assert far(O, ref) <= R.NS_TOL[dtype], far(O, ref)
    W, M = torch.zeros_like(H), H.float() / 4
    api.muon_step(W, torch.zeros_like(H), M, lr=1.0, momentum=2.0, nesterov=False, scale=1.0, eps=0.0)
    ref = R.newton_schulz(n64(M), 5, NS5, 0.0)
    assert far(W, -ref) <= R.NS_TOL[dtype], far(W, -ref)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("lr,decay", [(0.05, 0.0), (0.05, 2.0), (1e-4, 0.5)])
def test_how_far_a_step_moves_the_spectral_norm(dtype, lr, decay):
    """By 1.21 lr scale, the decay and the rounding of W, step after step."""
    W = matrices(60, 1, 200, 256, dtype, size=256 ** -0.5)[0].contiguous()
    M = torch.zeros(W.shape, device=DEV)
    sigma = api.spectral_norm(W.float()).sigma
    for step in range(6):
        G = matrices(61 + step, 1, 200, 256, dtype, "strong")[0].contiguous()
        api.muon_step(W, G, M, lr=lr, weight_decay=decay, short_operands=dtype != "f32" and step % 2 == 1)
        new = api.spectral_norm(W.float()).sigma
        short = 4e-3 * 1.21 * 200 ** 0.5 if dtype != "f32" and step % 2 == 1 else 0.0
        most = (1.21 + short) * lr + lr * decay * sigma + R.U[dtype] * float(W.double().norm())
        assert abs(new - sigma) <= most, (step, new, sigma, most)
        sigma = new
