"""Arrays of more than 2^31 elements (for AdamW 2^32): norm and gradients, class-table loss, AdamW, at the
places behind the border, against the same rows in a small call or 64 bits."""

import numpy as np
import pytest

import more_ref as R
from gpu_util import to_dev, to_host

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module")
def G():
    from paper_2102_10424_amd import gist
    return gist


@pytest.fixture(scope="module")
def ctx(G):
    return G.Context(0)


@pytest.fixture(autouse=True)
def free():
    import torch
    yield
    torch.cuda.empty_cache()


def test_norm(G, ctx):
    """The last 2,000 of 540,000 rows of 4,096: bitwise as a call of their own."""
    import torch
    n, d, k, b, e = 540_000, 4096, 2000, G.GIST_STORE_BF16, G.GIST_STORE_E4M3
    x = torch.empty(n, d, dtype=torch.bfloat16, device="cuda").normal_()
    gain = 1 + 0.1 * torch.randn(d, device="cuda")
    assert n * d > 2 ** 31

    def run(X):
        m = len(X)
        h, y8 = torch.empty_like(X), torch.empty(m, d, dtype=torch.uint8, device="cuda")
        s, rs = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
        G.gist_rms_norm(ctx, m, d, X, d, X, d, b, gain, EPS, h, d, y8, d, e, s, rs)
        dx = torch.empty_like(X)
        G.gist_rms_norm_bwd(ctx, m, d, X, d, b, h, d, b, gain, rs, X, d, dx, d, None, None)
        return h[-k:].clone(), y8[-k:].clone(), s[-k:].clone(), rs[-k:].clone(), dx[-k:].clone()

    for a, w in zip(run(x), run(x[-k:].clone())):
        assert torch.equal(a, w)


@pytest.mark.parametrize("store", ["bf16", "e4m3"])
def test_class_table(G, ctx, store):
    """3 rows against 2,200,000 classes of 1,024."""
    import torch
    n, C, d, scale = 3, 2_200_000, 1024, 0.5
    assert C * d > 2 ** 31
    grad = store == "bf16"
    H = (torch.randn(n, d, device="cuda") / 16).bfloat16()
    T = torch.empty(C, d, dtype=torch.bfloat16, device="cuda").normal_()
    y = torch.tensor([C - 1, 5, 2_150_000], dtype=torch.int32, device="cuda")
    hs = ts = None
    Hd, Td = H, T
    if not grad:
        Hd, Td = (torch.empty(k, d, dtype=torch.uint8, device="cuda") for k in (n, C))
        hs, ts = torch.empty(n, device="cuda"), torch.empty(C, device="cuda")
        G.gist_quantize_rows(ctx, n, d, H, d, G.GIST_STORE_BF16, Hd, d, hs)
        G.gist_quantize_rows(ctx, C, d, T, d, G.GIST_STORE_BF16, Td, d, ts)
    D = G.table_xent_desc(n, C, d, R.store_of(G, store), 0, scale, 1.0)
    ws = torch.empty(G.gist_table_xent_workspace(D, grad), dtype=torch.uint8, device="cuda")
    loss, logp, lse = torch.empty(1, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    dH, dT = (torch.empty_like(H), torch.empty_like(T)) if grad else (None, None)
    G.gist_table_xent(ctx, D, Hd, hs, Td, ts, y, None, loss, logp, lse, dH, dT, ws)

    def part(a, b):          # classes a .. b in 64 bits
        if grad:
            return T[a:b].double()
        return Td[a:b].view(torch.float8_e4m3fn).double() * ts[a:b, None].double()

    h = H.double() if grad else Hd.view(torch.float8_e4m3fn).double() * hs[:, None].double()
    cuts = [(a, min(a + 100_000, C)) for a in range(0, C, 100_000)]
    z = torch.cat([scale * (part(a, b) @ h.t().contiguous()) for a, b in cuts]).t().contiguous()
    far = max(float(scale * (part(a, b).abs() @ h.abs().t().contiguous()).max()) for a, b in cuts)
    want = torch.logsumexp(z, 1)
    # a logit: 2 u a sum of d terms; the sums of the classes' exponentials, in parts
    ez = 2 * R.U32 * (d + 16) * far + R.U32 * 4 * 16
    e = ez + R.U32 * (C / 64 + 300)
    assert float((lse - want).abs().max()) <= e
    zy = z[torch.arange(n), y.long()]
    assert float((logp - (zy - want)).abs().max()) <= 2 * e
    if not grad:
        return
    f = scale / n
    g = torch.exp(z - want[:, None])
    g[torch.arange(n), y.long()] -= 1
    # E and the factored rows of H in bf16; e^(z - lse) off by the logit's error and the lse's
    rel = 2 * R.HALF["bf16"] * (1 + R.HALF["bf16"]) + 2 * e
    for c in (slice(0, 1000), slice(2_096_900, 2_097_400), slice(2_149_900, 2_150_100), slice(C - 1000, C)):
        w = f * (g[:, c].t() @ h)
        b = f * (g[:, c].abs().t() @ h.abs()) * rel
        b = b + R.HALF["bf16"] * (w.abs() + b) + 2.0 ** -126
        assert bool(((dT[c].double() - w).abs() <= b).all()), c
    # dH: a matrix instruction adds 32 terms to a sum: 2 u (C / 32 + 32) of all magnitudes
    w = f * sum(g[:, a:b] @ part(a, b) for a, b in cuts)
    m = f * sum(g[:, a:b].abs() @ part(a, b).abs() for a, b in cuts)
    b = m * (rel + 2 * R.U32 * (C / 32 + 100))
    assert bool(((dH.double() - w).abs() <= b + R.HALF["bf16"] * (w.abs() + b)).all())


def test_adamw(G, ctx):
    """One tensor of 2^32 + 1,000 weights with 8-bit moments: the elements behind 2^32 and some before them."""
    import torch
    n = 2 ** 32 + 1000
    W = torch.ones(n, device="cuda")
    g = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    nb = -(-n // G.GIST_ADAMW_BLOCK)
    ms, vs = (torch.zeros(nb, device="cuda") for _ in range(2))
    t = G.adamw_tensors([G.adamw_tensor(W, g, m, v, n, 0.0, G.GIST_STORE_BF16, ms, vs, None, G.GIST_STORE_BF16)])
    G.gist_adamw_update(ctx, t, 2.0 ** -5, 1, 0.9, 0.999, 0.0, 0, 1.0, 1)
    for s in (slice(0, 600), slice(2 ** 31 - 300, 2 ** 31 + 300), slice(2 ** 32 - 600, n)):
        w = to_host(W[s]).astype(np.float64)
        # m / (1 - beta1) = g and v / (1 - beta2) = g^2: a step of lr, within the few roundings of
        # moments, corrections, root, quotient and product (each u), and of the difference
        assert (np.abs(w - (1 - 2.0 ** -5)) <= 2.0 ** -5 * 16 * R.U32 + R.U32).all()
        # all alike: the block's largest, code 448, or the one below where no random bit is set
        assert bool(((m[s] == 0x7e) | (m[s] == 0x7d)).all()) and bool(((v[s] == 0x7e) | (v[s] == 0x7d)).all())
    assert float(ms.min()) > 0 and float(vs.min()) > 0
    assert float(ms.max() - ms.min()) == 0 and float(vs.max() - vs.min()) == 0
