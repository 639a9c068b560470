"""Newton-Schulz orthogonalisation and the momentum step, against float64 on the CPU."""
import numpy as np
import pytest
import torch

import adapt_ref as R
from gpu_helpers import say
from paper_2608_13144_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
NS5 = [api.NEWTON_SCHULZ] * 5


def n64(t):
    return t.detach().cpu().double().numpy()


def matrices(seed, b, m, n, dtype, kind="random", size=1.0):
    g = torch.Generator().manual_seed(seed)
    G = torch.randn(b, m, n, generator=g)
    if kind == "strong":  # a few strong directions over noise
        G = torch.randn(b, m, 2, generator=g) @ torch.randn(b, 2, n, generator=g) + 0.05 * G
    return (size * G).to(DT[dtype]).to(DEV)


def far(got, ref):
    return float(np.linalg.norm(n64(got) - ref) / np.linalg.norm(ref))


SHAPES = [(1, 1, 1), (2, 1, 37), (3, 16, 16), (2, 8, 300), (5, 33, 17), (1, 64, 64), (2, 65, 130), (1, 200, 256),
          (2, 128, 1000), (1, 129, 128), (1, 300, 140), (1, 257, 511), (1, 700, 390), (1, 384, 1100)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_orthogonalise(shape, dtype):
    for kind in ("random", "strong"):
        say("orthogonalise", shape, dtype, kind)
        G = matrices(sum(shape), *shape, dtype, kind)
        before = G.clone()
        O = api.orthogonalise(G)
        assert torch.equal(G, before) and O.dtype == G.dtype and O.shape == G.shape
        ref = R.newton_schulz(n64(G), 5, NS5, 1e-7)
        assert far(O, ref) <= R.NS_TOL[dtype], (shape, dtype, kind, far(O, ref))
        worst = float(np.max(np.abs(n64(O) - ref)) / np.sqrt(np.mean(ref * ref)))
        assert worst <= 40 * R.NS_TOL[dtype], (shape, dtype, kind, worst)
        assert torch.equal(O, api.orthogonalise(G)), "two calls differ"
        inplace = G.clone()
        assert api.orthogonalise(inplace, out=inplace) is inplace and torch.equal(inplace, O)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_a_matrix_and_a_stack_agree(dtype):
    G = matrices(3, 4, 40, 96, dtype)
    O = api.orthogonalise(G)
    for i in range(4):
        assert torch.equal(api.orthogonalise(G[i].contiguous()), O[i])


@pytest.mark.parametrize("m,n", [(24, 100), (160, 150), (300, 400)])
def test_singular_values_and_other_coefficients(m, n):
    """(15/8, -10/8, 3/8) converges to the polar factor; per-step coefficients are taken in order."""
    G = matrices(4, 1, m, n, "f32")
    cubic = (15 / 8, -10 / 8, 3 / 8)
    O = api.orthogonalise(G, steps=24, coefficients=cubic)
    u, s, vt = np.linalg.svd(n64(G)[0], full_matrices=False)
    # 24 steps at slope 15/8 bring every s > 1e-4 to 1; rounding 2^-22 on singular values away from 0
    assert far(O[0], u @ vt) <= 1e-4
    mixed = [api.NEWTON_SCHULZ] * 3 + [cubic] * 4
    O = api.orthogonalise(G, steps=7, coefficients=mixed)
    assert far(O, R.newton_schulz(n64(G), 7, mixed, 1e-7)) <= 2 * R.NS_TOL["f32"]
    s = np.linalg.svd(n64(api.orthogonalise(G))[0], compute_uv=False)
    assert s.max() <= 1.21


@pytest.mark.parametrize("shape", [(1, 30, 60), (1, 200, 180)])
def test_steps_none_and_one(shape):
    G = matrices(5, *shape, "f32")
    for steps in (0, 1):
        O = api.orthogonalise(G, steps=steps)
        assert far(O, R.newton_schulz(n64(G), steps, NS5, 1e-7)) <= 1e-6


@pytest.mark.parametrize("shape", [(3, 12, 50), (3, 150, 140)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_zero_huge_tiny_and_not_finite(shape, dtype):
    G = matrices(6, *shape, dtype)
    clean = api.orthogonalise(G)
    G[1].zero_()
    O = api.orthogonalise(G)
    assert bool((O[1] == 0).all()) and torch.equal(O[0], clean[0]) and torch.equal(O[2], clean[2])
    for bad in (float("nan"), float("inf")):
        G[1, 3, 4] = bad
        O = api.orthogonalise(G)
        assert bool(O[1].isnan().all()), bad
        assert torch.equal(O[0], clean[0]) and torch.equal(O[2], clean[2])
    for size in (1e-6, 1e3) if dtype == "f16" else (1e-30, 1e30):
        H = matrices(6, *shape, dtype, size=size)
        ref = R.newton_schulz(n64(H), 5, NS5, 0.0)
        assert far(api.orthogonalise(H, eps=0.0), ref) <= R.NS_TOL[dtype], size
    # eps weighs in where the norm is small
    H = matrices(7, *shape, "f32", size=1e-8)
    O = api.orthogonalise(H, eps=1e-6)
    assert far(O, R.newton_schulz(n64(H), 5, NS5, float(np.float32(1e-6)))) <= R.NS_TOL["f32"]


STEP_SHAPES = [(1, 1, 5), (4, 16, 300), (3, 40, 24), (1, 200, 256), (1, 300, 130), (2, 260, 260)]


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", STEP_SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_muon_step(shape, dtype, nesterov):
    b, m, n = shape
    say("muon step", shape, dtype, nesterov)
    W = matrices(8, *shape, dtype, size=n ** -0.5)
    G = matrices(9, *shape, dtype, "strong", size=1e-2)
    M = matrices(10, *shape, "f32", size=3e-2)
    W0, G0, M0 = n64(W), n64(G), n64(M)
    lr, mu, wd = 0.02, 0.95, 0.1
    api.muon_step(W, G, M, lr=lr, momentum=mu, weight_decay=wd, nesterov=nesterov)
    f = lambda v: float(np.float32(v))  # noqa: E731  (the options are float32)
    M1 = f(mu) * M0 + G0
    assert np.array_equal(n64(G), G0)
    assert np.all(np.abs(n64(M) - M1) <= 2.0 ** -23 * (np.abs(M0) + np.abs(G0)))
    O = R.newton_schulz(f(mu) * M1 + G0 if nesterov else M1, 5, NS5, 1e-7)
    gain = f(lr) * f(max(1.0, m / n) ** 0.5)
    ref = (1 - f(lr) * f(wd)) * W0 - gain * O
    lim = 2 * R.U[dtype] * np.linalg.norm(ref) + gain * R.NS_TOL[dtype] * np.linalg.norm(O)
    assert np.linalg.norm(n64(W) - ref) <= lim, (shape, dtype)


@pytest.mark.parametrize("shape", [(1, 3, 70000), (1, 66000, 5), (3, 64, 5000), (2, 4099, 50), (300, 16, 24), (2, 33, 2048),
                                   (70, 48, 520)], ids=lambda s: "x".join(map(str, s)))
def test_short_matrices_with_long_sides(shape):
    for dtype in ("f32", "bf16"):
        say("short", shape, dtype)
        for kind in ("random", "strong"):
            G = matrices(40, *shape, dtype, kind)
            assert far(api.orthogonalise(G), R.newton_schulz(n64(G), 5, NS5, 1e-7)) <= R.NS_TOL[dtype]
        W, M = torch.zeros_like(G), matrices(41, *shape, "f32")
        U = 0.25 * n64(M) + 1.5 * n64(G)
        api.muon_step(W, G, M, lr=1.0, momentum=0.5, scale=1.0)
        assert far(W, -R.newton_schulz(U, 5, NS5, 1e-7)) <= R.NS_TOL[dtype]


# Large and many matrices: every tile size of the products, wide and tall.
LARGE = [("ortho", (1, 2080, 2050), "f32"), ("ortho", (1, 2050, 2080), "f16"), ("ortho", (5, 1100, 1030), "f32"),
         ("ortho", (5, 1030, 1100), "bf16"), ("ortho", (40, 500, 520), "f32"), ("ortho", (40, 520, 500), "f16"),
         ("step", (40, 500, 520), "bf16"), ("step", (40, 520, 500), "f16"), ("step", (60, 500, 470), "bf16"),
         ("step", (60, 470, 500), "f16"), ("step", (5, 1100, 1030), "bf16"), ("step", (1, 2050, 2080), "bf16"),
         ("step", (8, 1030, 1100), "bf16"), ("step", (5, 1030, 1100), "f32")]


@pytest.mark.parametrize("what,shape,dtype", LARGE, ids=lambda v: "x".join(map(str, v)) if isinstance(v, tuple) else v)
def test_large_and_many(what, shape, dtype):
    say("large", what, shape, dtype)
    b, m, n = shape
    G = matrices(30, *shape, dtype, "strong")
    if what == "ortho":
        ref = R.newton_schulz(n64(G), 5, NS5, 1e-7)
        O = api.orthogonalise(G)
        assert far(O, ref) <= R.NS_TOL[dtype], far(O, ref)
        assert float(np.max(np.abs(n64(O) - ref)) / np.sqrt(np.mean(ref * ref))) <= 40 * R.NS_TOL[dtype]
        return
    W = torch.zeros_like(G)  # so that W's rounding hides nothing of the step's
    M = torch.zeros(shape, device=DEV)
    api.muon_step(W, G, M, lr=1.0, momentum=0.5, scale=1.0)
    ref = -R.newton_schulz(1.5 * n64(G), 5, NS5, 1e-7)
    tol = R.NS_TOL["f32" if dtype == "f32" else "bf16"]  # 16-bit steps take 11-bit operands
    assert far(W, ref) <= tol, far(W, ref)
    assert float(np.max(np.abs(n64(W) - ref)) / np.sqrt(np.mean(ref * ref))) <= 40 * tol
    assert np.array_equal(n64(M), n64(G))


def test_a_step_bounds_the_spectral_norm():
    """sigma_max moves by at most 1.21 lr scale: what certified radii are divided by stays known."""
    W = matrices(11, 1, 200, 256, "f32", size=256 ** -0.5)[0].contiguous()
    G = matrices(12, 1, 200, 256, "f32", "strong")[0].contiguous()
    M = torch.zeros_like(W)
    before = api.spectral_norm(W).sigma
    api.muon_step(W, G, M, lr=0.05)
    after = api.spectral_norm(W).sigma
    assert abs(after - before) <= 1.21 * 0.05


@pytest.mark.parametrize("shape,dtype", [((4, 16, 200), "bf16"), ((1, 200, 256), "f32"), ((1, 300, 200), "f16")])
def test_graph_replays_and_side_stream(shape, dtype):
    W = matrices(13, *shape, dtype)
    G, M = matrices(14, *shape, dtype), matrices(15, *shape, "f32")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        O_side = api.orthogonalise(G)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(O_side, api.orthogonalise(G))
    Wg, Mg = W.clone(), M.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        O = api.orthogonalise(G)
        api.muon_step(Wg, G, Mg, lr=0.1)
    for k in range(3):
        G.copy_(matrices(20 + k, *shape, dtype))
        ref = api.orthogonalise(G)
        api.muon_step(W, G, M, lr=0.1)
        torch.cuda.synchronize()
        O.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, ref) and torch.equal(Wg, W) and torch.equal(Mg, M), k
    del graph


def test_empty_stack_and_binding_refuses():
    G = torch.zeros(0, 8, 9, device=DEV)
    assert api.orthogonalise(G).shape == (0, 8, 9)
    api.muon_step(G, G.clone(), G.clone(), lr=0.1)
    G = matrices(16, 2, 8, 9, "f32")
    for bad in (G.cpu(), G.double(), G.transpose(1, 2), G[0, 0]):
        with pytest.raises(ValueError):
            api.orthogonalise(bad)
    with pytest.raises(ValueError):
        api.orthogonalise(G, coefficients=[(1.0, 0.0, 0.0)] * 4)
    with pytest.raises(ValueError):
        api.orthogonalise(G, out=torch.empty(2, 9, 8, device=DEV))
    with pytest.raises(ValueError):
        api.muon_step(G, G.bfloat16(), torch.zeros_like(G), lr=0.1)
    with pytest.raises(ValueError):
        api.muon_step(G, G.clone(), torch.zeros_like(G).bfloat16(), lr=0.1)
    with pytest.raises(api.L.LipcacheError):  # singular values that no bound holds
        api.orthogonalise(G, coefficients=(30.0, 5.0, 5.0))
    with pytest.raises(api.L.LipcacheError):
        api.orthogonalise(G, coefficients=(float("nan"), 0.0, 0.0))
