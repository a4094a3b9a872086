"""GPU parity of the orthogonalised update against its factor by singular
values in 64 bits: square, wide, tall, one row, odd sides, groups, both operand
types, other coefficients, zero and non-finite matrices, extreme sizes of the
gradient, momentum policies and the weight step, replays."""

import numpy as np
import pytest

import ops_ref as R
from gpu_util import log, to_dev, to_host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    from paper_2102_10424_amd import gist
    return gist


@pytest.fixture(scope="module")
def ctx(G):
    return G.Context(0)


def matrices(g, r, c, rng):
    """A few strong directions over noise, as gradients have."""
    k = max(1, min(r, c) // 8)
    low = rng.standard_normal((g, r, k)) @ rng.standard_normal((g, k, c)) / np.sqrt(k)
    return ((low + rng.standard_normal((g, r, c))) * 1e-3).astype(np.float32)


def dtype_of(G, name):
    return G.GIST_DTYPE_F32 if name == "f32" else G.GIST_DTYPE_F16_IN


def workspace(G, d):
    import torch
    return torch.empty(G.gist_muon_workspace_size(d), dtype=torch.uint8, device="cuda")


def orthogonalize(G, ctx, U, dtype, **kw):
    """The result as float64, with a guard behind it."""
    import torch
    g, r, c = U.shape
    d = G.muon_desc(r, c, groups=g, dtype=dtype_of(G, dtype), **kw)
    O = torch.full((g * r * c + 8,), 3.0, device="cuda",
                   dtype=torch.float32 if dtype == "f32" else torch.float16)
    G.gist_orthogonalize(ctx, d, to_dev(U), O, workspace(G, d))
    h = to_host(O.float()).astype(np.float64)
    assert (h[g * r * c:] == 3).all()
    return h[:g * r * c].reshape(g, r, c)


def store_slack(want, dtype):
    """2-norm of the last rounding: fp32, or fp16 with its smallest step."""
    return np.linalg.norm(want) * R.HALF[dtype if dtype == "f32" else "f16"] + \
        (2.0 ** -25 * np.sqrt(want.size) if dtype != "f32" else 0.0)


SHAPES = [(1, 1, 1), (1, 1, 9), (1, 9, 1), (1, 2, 3), (2, 16, 16), (1, 31, 33), (1, 64, 64), (3, 41, 64),
          (1, 65, 63), (1, 100, 700), (2, 700, 100), (1, 128, 128), (1, 129, 257), (4, 257, 130),
          (1, 512, 512), (1, 1433, 128), (2, 300, 1024), (1, 1000, 640), (1, 64, 128), (1, 129, 128),
          (2, 65, 128), (2, 128, 66), (1, 3, 1000), (3, 127, 127), (1, 33, 8300), (1, 2047, 100), (1, 100, 2050),
          (70, 40, 300), (1, 640, 64)]


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("g,r,c", SHAPES)
def test_orthogonalize(G, ctx, dtype, g, r, c):
    rng = np.random.default_rng(g * 1000 + r * 7 + c)
    U = matrices(g, r, c, rng)
    got = orthogonalize(G, ctx, U, dtype)
    for i in range(0, g, max(1, g // 4)):
        want = R.orthogonal(U[i])
        tol = R.muon_tolerance(U[i], dtype) + store_slack(want, dtype)
        err = np.linalg.norm(got[i] - want)
        log(f"orthogonalize {dtype} {r}x{c}: error {err / np.linalg.norm(want):.2e} of norm, "
            f"{err / tol:.2f} of the bound")
        assert err <= tol


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("g,r,c", [(9, 300, 600), (9, 513, 260), (16, 600, 700), (15, 770, 512), (1, 3000, 2900)])
def test_orthogonalize_many_tiles(G, ctx, dtype, g, r, c):
    """Sizes whose products take the larger tiles; first, middle and last group checked."""
    rng = np.random.default_rng(g * 1000 + r * 7 + c)
    U = matrices(g, r, c, rng)
    got = orthogonalize(G, ctx, U, dtype)
    if r > 1024:      # the iteration itself in 64 bits on the GPU; errors as at the smaller sizes
        import torch
        X = to_dev(U[0]).double()
        X = X.t() if r > c else X
        X = X / torch.linalg.vector_norm(X)
        a, b, q = (float(np.float32(x)) for x in R.COEF)
        for _ in range(5):
            A = X @ X.t()
            X = a * X + (b * A + q * (A @ A)) @ X
        want = to_host(X.t() if r > c else X)
        rel = 2.0 ** -22 if dtype == "f32" else 2.0 ** -11
        # the bound at 512 x 512 is 14 roundings of this size
        assert np.linalg.norm(got[0] - want) <= 14 * rel * np.linalg.norm(want)
        return
    for i in sorted({0, g // 2, g - 1}):
        want = R.orthogonal(U[i])
        tol = R.muon_tolerance(U[i], dtype) + store_slack(want, dtype)
        err = np.linalg.norm(got[i] - want)
        log(f"orthogonalize {dtype} {r}x{c} group {i}: {err / tol:.2f} of the bound")
        assert err <= tol


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("steps,coef", [(1, R.COEF), (3, R.COEF), (8, (1.5, -0.5, 0.0)),
                                        (6, (15 / 8, -10 / 8, 3 / 8)), (2, (1.0, 0.0, 0.0))])
def test_steps_and_coefficients(G, ctx, dtype, steps, coef):
    rng = np.random.default_rng(steps)
    U = matrices(1, 70, 150, rng)
    got = orthogonalize(G, ctx, U, dtype, steps=steps, coef=coef)[0]
    want = R.orthogonal(U[0], steps, coef)
    tol = R.muon_tolerance(U[0], dtype, steps, coef) + store_slack(want, dtype)
    assert np.linalg.norm(got - want) <= tol


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_scale_of_the_gradient_does_not_matter(G, ctx, dtype):
    """Entries near the ends of the fp32 range, and one dominant entry."""
    rng = np.random.default_rng(9)
    U = matrices(1, 40, 60, rng)
    for f in (2.0 ** -20, 2.0 ** 40, 2.0 ** 135):
        V = (U.astype(np.float64) * f).astype(np.float32)
        assert np.isfinite(V).all()
        eps = 1e-30
        got = orthogonalize(G, ctx, V, dtype, eps=eps)[0]
        want = R.orthogonal(V[0], eps=eps)
        tol = R.muon_tolerance(V[0].astype(np.float64) / f, dtype) + store_slack(want, dtype)
        assert np.linalg.norm(got - want) <= tol, f
    spike = U * 1e-6
    spike[0, 3, 5] = 1.0
    got = orthogonalize(G, ctx, spike, dtype)[0]
    want = R.orthogonal(spike[0])
    assert np.linalg.norm(got - want) <= R.muon_tolerance(spike[0], dtype) + store_slack(want, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_eps_zero_and_nonfinite(G, ctx, dtype):
    """A zero matrix gives zero, a norm below eps divides by eps, a NaN or Inf makes its own
    group NaN and leaves the others as they are without it."""
    rng = np.random.default_rng(10)
    U = matrices(4, 50, 30, rng)
    ref = orthogonalize(G, ctx, U, dtype)
    V = U.copy()
    V[0], V[1, 7, 7], V[2, 0, 29] = 0, np.nan, -np.inf
    got = orthogonalize(G, ctx, V, dtype)
    assert (got[0] == 0).all()
    assert np.isnan(got[1]).all() and np.isnan(got[2]).all()
    assert np.array_equal(got[3], ref[3])
    small = orthogonalize(G, ctx, U, dtype, eps=float(np.linalg.norm(U[0])) * 4)
    want = R.orthogonal(U[0], eps=float(np.float32(np.linalg.norm(U[0]) * 4)))
    assert np.linalg.norm(small[0] - want) <= R.muon_tolerance(U[0], dtype) + store_slack(want, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("g,r,c", [(1, 1, 1), (2, 48, 100), (1, 130, 70), (1, 333, 333), (2, 602, 64), (3, 128, 100)])
def test_update(G, ctx, dtype, nesterov, g, r, c):
    """Three steps, the first with fresh momentum over garbage.  M: two products and a sum,
    three roundings of its terms a step.  W: the factor's bound times lr scale, and three
    roundings (keep, product, sum) of |W| and of the step."""
    import torch
    rng = np.random.default_rng(r + c + g)
    lr, mu, wd, scale = 0.02, 0.95, 0.1, 0.2 * np.sqrt(max(r, c))
    W0 = (rng.standard_normal((g, r, c)) / np.sqrt(r)).astype(np.float32)
    W, M = to_dev(W0), torch.full((g, r, c), float("nan"), device="cuda")
    muf, lrf, wdf, sf = (float(np.float32(x)) for x in (mu, lr, wd, scale))
    w, m, mb = W0.astype(np.float64), np.zeros((g, r, c)), np.zeros((g, r, c))
    tolw = np.zeros(g)
    for k in range(3):
        dW = matrices(g, r, c, rng)
        flags = (G.GIST_MUON_NESTEROV if nesterov else 0) | (G.GIST_MUON_FRESH if k == 0 else 0)
        d = G.muon_desc(r, c, groups=g, dtype=dtype_of(G, dtype), flags=flags)
        G.gist_muon_update(ctx, d, W, to_dev(dW), M, lr, mu, wd, scale, workspace(G, d))
        old = m
        m = muf * old + (1 - muf) * dW
        mb = muf * mb + 3 * R.U32 * (np.abs(muf * old) + np.abs((1 - muf) * dW))
        u = (1 - muf) * dW + muf * m if nesterov else m
        assert (np.abs(to_host(M) - m) <= mb).all()
        for i in range(g):
            f = R.orthogonal(u[i])
            tol = R.muon_tolerance(u[i], dtype, seed=k)
            # the direction itself is off by mb and three roundings: relative to its norm,
            # times the iteration's largest slope (a^5)
            du = np.linalg.norm(mb[i] + 3 * R.U32 * np.abs(u[i])) / np.linalg.norm(u[i])
            tol += R.COEF[0] ** 5 * 2 * du
            step = lrf * sf
            tolw[i] += step * tol + 3 * R.U32 * (np.linalg.norm(w[i]) + step * np.linalg.norm(f))
            w[i] = (1 - lrf * wdf) * w[i] - step * f
    got = to_host(W)
    for i in range(g):
        err = np.linalg.norm(got[i] - w[i])
        log(f"muon_update {dtype} {r}x{c} nesterov={nesterov}: {err / tolw[i]:.2f} of the bound")
        assert err <= tolw[i]


def test_workspace_contents_do_not_matter(G, ctx):
    """Workspace and outputs full of NaN before the call; the same bits again."""
    import torch
    rng = np.random.default_rng(12)
    for r, c in ((100, 200), (65, 64), (300, 30), (100, 100), (500, 200)):
        U = to_dev(matrices(1, r, c, rng))
        d = G.muon_desc(r, c)
        ws = workspace(G, d)
        a, b = (torch.full((r, c), float("nan"), device="cuda") for _ in range(2))
        ws.fill_(255)
        G.gist_orthogonalize(ctx, d, U, a, ws)
        ws.fill_(126)
        G.gist_orthogonalize(ctx, d, U, b, ws)
        assert torch.equal(a, b) and bool(torch.isfinite(a).all())


@pytest.mark.parametrize("g,r,c", [(2, 20, 30), (2, 40, 300), (1, 130, 200), (2, 300, 140)])
def test_in_place(G, ctx, g, r, c):
    """The fp32 factor in its gradient's place: the bits of one written elsewhere."""
    import torch
    U = to_dev(matrices(g, r, c, np.random.default_rng(r)))
    d = G.muon_desc(r, c, groups=g)
    ws = torch.empty(G.gist_muon_workspace_size(d), dtype=torch.uint8, device="cuda")
    O = torch.empty_like(U)
    G.gist_orthogonalize(ctx, d, U, O, ws)
    G.gist_orthogonalize(ctx, d, U, U, ws)
    torch.cuda.synchronize()
    assert torch.equal(U, O)


def test_empty(G, ctx):
    for r, c in ((0, 5), (5, 0)):
        d = G.muon_desc(r, c)
        assert G.gist_muon_workspace_size(d) == 0
        G.gist_orthogonalize(ctx, d, None, None, None)
        G.gist_muon_update(ctx, d, None, None, None, 0.1, 0.9, 0.0, 1.0, None)


@pytest.mark.parametrize("r,c", [(96, 200), (1500, 40), (64, 64), (200, 180)])
def test_replays(G, r, c):
    """An update recorded once and replayed with new gradients equals the eager updates."""
    import torch
    st = torch.cuda.Stream()
    cctx, ectx = G.Context(0, stream=st.cuda_stream), G.Context(0)
    rng = np.random.default_rng(13)
    d = G.muon_desc(r, c, groups=2, flags=G.GIST_MUON_NESTEROV)
    W = to_dev(rng.standard_normal((2, r, c)).astype(np.float32))
    M = torch.zeros_like(W)
    W2, M2, dW = W.clone(), M.clone(), torch.empty_like(W)
    ws, ws2 = workspace(G, d), workspace(G, d)
    torch.cuda.synchronize()
    G.gist_capture_begin(cctx)
    G.gist_muon_update(cctx, d, W, dW, M, 0.02, 0.9, 0.01, 1.0, ws)
    rep = G.gist_capture_end(cctx)
    for k in range(4):
        dW.copy_(torch.from_numpy(matrices(2, r, c, rng)))
        G.gist_muon_update(ectx, d, W2, dW, M2, 0.02, 0.9, 0.01, 1.0, ws2)
        G.gist_replay_launch(ectx, rep)
        torch.cuda.synchronize()
        assert torch.equal(W, W2) and torch.equal(M, M2), k
