"""Class-table loss in bf16 over several pieces of rows whose table gradient is cut over workgroups as
well: parts that a shorter last piece adds to, and rows far from their reference in any piece."""

import numpy as np
import pytest

import more_ref as R
from gpu_util import log, to_host
from test_gpu_table_xent import inputs, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    from paper_2102_10424_amd import gist
    return gist


def reference(Hv, Tv, y, scale, gscale, half, d, rows=1024):
    """lse, dH, dT in 64 bits on the GPU, and bounds: a logit's error (as in more_ref) and that of lse, by
    the row; relative to the exponentials those, their rounding and that of the scaled rows, and the
    sums'."""
    import torch
    H, T, yd = torch.from_numpy(Hv).cuda(), torch.from_numpy(Tv).cuda(), torch.from_numpy(y).cuda().long()
    n, C = len(y), len(Tv)
    aH, aT = H.abs(), T.abs()
    Tt, aTt = T.t().contiguous(), aT.t().contiguous()
    f = gscale * scale / int((y >= 0).sum())
    lse, ez = (torch.empty(n, dtype=torch.float64, device="cuda") for _ in range(2))
    dH, bH = torch.zeros_like(H), torch.zeros_like(H)
    dT, bT = torch.zeros_like(T), torch.zeros_like(T)
    u = R.U32
    for a in range(0, n, rows):
        s = slice(a, a + rows)
        z = scale * (H[s] @ Tt)
        lse[s] = torch.logsumexp(z, 1)
        far = scale * (aH[s] @ aTt).amax(1)
        ez[s] = 4 * u * (d + 16) * far + u * (C / 64 + 28 + 4 * np.log2(C) + 8 * far + 200)
        g = torch.exp(z - lse[s, None])
        at, c = torch.arange(len(g), device="cuda"), yd[s].clamp(min=0)
        A = g.clone()
        g[at, c] -= 1
        A[at, c] += g[at, c].abs()
        g[yd[s] < 0] = 0
        A[yd[s] < 0] = 0
        dH[s] = f * (g @ T)
        dT += f * (g.t().contiguous() @ H[s])
        bH[s] = f * (ez[s, None] + 1.1 * half + 2 * u * (C + 24)) * (A @ aT)
        w = f * (ez[s, None] + 2.1 * half + 2 * u * (n + 24)) * A
        bT += w.t().contiguous() @ aH[s]
    bH += half * dH.abs()
    bT += half * dT.abs()
    return [t.cpu().numpy() for t in (lse, ez, dH, bH + 2.0 ** -120, dT, bT + 2.0 ** -120)]


@pytest.mark.parametrize("store,dtype", [("bf16", None), ("f32", "bf16")])
@pytest.mark.parametrize("far", [False, True])
def test_cut_pieces(G, store, dtype, far):
    """Pieces of 10,496 and 5,888 rows, the table's gradient in 5 slices."""
    rng = np.random.default_rng(3)
    n, C, d = 16384, 50001, 64
    H, T, y = inputs(n, C, d, rng)
    if far:
        H[100:103] *= 60
        H[12000:12011] *= 60
        H[n - 1] *= 60
        y[n - 1] = 5
    ctx = G.Context(0)
    out, Hv, Tv, args = run(G, ctx, H, T, y, store, dtype)
    scale = float(np.float32(0.7))
    half = R.HALF["bf16"]
    lse, ez, dH, bH, dT, bT = reference(Hv, Tv, y, scale, 3.0, half, d)
    for k, want, b in (("lse", lse, ez), ("dH", dH, bH), ("dT", dT, bT)):
        e = np.abs(out[k] - want) / b
        log(f"{k}: {e.max():.2g} of the bound")
        assert (e <= 1).all(), k
    # again: the same bits
    before = [args[k].clone() for k in (11, 12)]
    G.gist_table_xent(*args)
    for a, k, m in zip(before, (11, 12), (n, C)):
        assert np.array_equal(to_host(a.float())[:m], to_host(args[k].float())[:m])
