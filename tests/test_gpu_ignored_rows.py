"""Rows that take no part in a step -- without a label, or behind a padded batch's last -- leave
nothing in any gradient, whatever they hold: the norm's backward pass with the loss's labels, and
the whole end of a step behind it."""

import numpy as np
import pytest

import more_ref as R
from gpu_util import BF16_TOL, FP32_TOL, log, relerr, to_dev, to_host
from test_gpu_table_head import reference, runner, setup

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    from paper_2102_10424_amd import gist
    return gist


@pytest.mark.parametrize("kind", ["gcn", "sage"])
@pytest.mark.parametrize("mode", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("fill", [float("nan"), float("inf")])
def test_step(G, kind, mode, fill):
    """Non-finite output rows that have no label or lie behind n_dev: every gradient of the step
    as if they were not there, the rows' own zero."""
    import torch
    data = setup(kind, 11)
    csr, n, widths, W, X, T, gain, y = data
    nv = n - 33
    dtype = dict(bf16=torch.bfloat16, f16=torch.float16).get(mode, torch.float32)
    gs = 1024.0 if mode == "f16" else 1.0
    b, run, params, head = runner(G, G.Context(0), kind, data, dtype, gscale=gs)
    b.n_dev = torch.tensor([nv], dtype=torch.int32, device="cuda")
    out = (y < 0) | (np.arange(n) >= nv)
    assert 0 < (y[:nv] < 0).sum() < nv
    for residual in (True, False):
        run.forward(b, params)
        run.H[2][:n][to_dev(out)] = fill
        head.loss_and_grad(run, b, b.X if residual else None)
        run.backward(b, params)
        loss, logp, dout, dT, dg = reference(kind, csr, n, widths, W, X, T, gain, y, residual, nv)
        mine = to_host(run.dlogits)[:n]
        assert (mine[out] == 0).all()
        got = [relerr(float(head.loss), loss), relerr(to_host(head.logp), logp), relerr(mine, dout),
               relerr(to_host(head.dT.float()) / gs, dT), relerr(to_host(head.dgain) / gs, dg)]
        dW = reference(kind, csr, n, widths, W, X, T, gain, y, residual, dout=mine)
        exact = [relerr(to_host(run.dW[l]), dW[l]) for l in range(2)]
        log(f"{kind} {mode}: " + ", ".join("%.1e" % e for e in got + exact))
        assert max(got) < (FP32_TOL if mode == "f32" else BF16_TOL), got
        assert max(exact) < FP32_TOL, exact


@pytest.mark.parametrize("n,d", [(300, 7), (100, 16), (4097, 41), (77, 128), (33, 130), (600, 512), (70, 519),
                                 (40, 1025), (9, 4104), (5, 16384), (4, 16385), (3, 20011)])
@pytest.mark.parametrize("store,dys", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f32", "bf16")])
def test_norm_backward(G, n, d, store, dys):
    """dx and dgain have the bits of the call without the rows that take no part (their dy zero, h
    finite: terms of exact zeros), whatever dy, h and rstd hold there."""
    import torch
    ctx = G.Context(0)
    rng = np.random.default_rng(n + 31 * d)
    t = lambda name, s: torch.from_numpy(rng.standard_normal((n, d)).astype(np.float32) * s).to(R.torch_type(name)).cuda()
    h, dy, ds = t(store, 1.0), t(dys, 0.3), t(store, 0.3)
    gain = to_dev((1 + 0.3 * rng.standard_normal(d)).astype(np.float32))
    rstd = to_dev((0.5 + rng.random(n)).astype(np.float32))
    y = rng.integers(-1, 3, n).astype(np.int32)
    y[0] = 0
    ws = torch.empty(G.gist_rms_norm_bwd_workspace(n, d), dtype=torch.uint8, device="cuda")
    st, dst = R.store_of(G, store), R.store_of(G, dys)
    for nv in (None, n + 5, max(1, n - n // 3), 0, -2):
        out = to_dev((y < 0) | (np.arange(n) >= (n if nv is None else nv)))
        n_dev = None if nv is None else torch.tensor([nv], dtype=torch.int32, device="cuda")
        clean, bad = dy.clone(), [dy.clone(), h.clone(), rstd.clone()]
        clean[out] = 0
        for a in bad:
            a[out] = float("nan")
        for dsum in (ds, None):
            want, wg = torch.empty_like(h), torch.empty(d, device="cuda")
            G.gist_rms_norm_bwd(ctx, n, d, clean, d, dst, h, d, st, gain, rstd, dsum, d, want, d, wg, ws)
            want[out] = 0 if dsum is None else dsum[out]
            got, gg = torch.full_like(h, 7), torch.full((d,), 7.0, device="cuda")
            args = (ctx, n, d, bad[0], d, dst, bad[1], d, st, gain, bad[2], dsum, d)
            G.gist_rms_norm_bwd(*args, got, d, gg, ws, to_dev(y), n_dev)
            assert torch.equal(got, want) and torch.equal(gg, wg), (nv, dsum is None)
            # in place of h, and dx alone
            G.gist_rms_norm_bwd(*args, bad[1], d, None, None, to_dev(y), n_dev)
            assert torch.equal(bad[1], want)
            bad[1] = h.clone()
            bad[1][out] = float("nan")
    # without labels: the valid rows' count alone
    dy[n - 1], n_dev = float("nan"), torch.tensor([n - 1], dtype=torch.int32, device="cuda")
    G.gist_rms_norm_bwd(ctx, n, d, dy, d, dst, h, d, st, gain, rstd, None, d, got, d, gg, ws, None, n_dev)
    assert bool((got[n - 1] == 0).all()) and bool(torch.isfinite(got).all() & torch.isfinite(gg).all())


@pytest.mark.parametrize("d", [24, 700])
def test_replayed(G, d):
    """Recorded once, the labels and the valid rows' count changed between three replays."""
    import torch
    n = 200
    side = torch.cuda.Stream()
    ctx, cap = G.Context(0), G.Context(0, stream=side.cuda_stream)
    torch.manual_seed(d)
    h, dy = torch.randn(n, d, device="cuda"), torch.randn(n, d, device="cuda")
    dy[50:60] = float("nan")
    gain, rstd = torch.ones(d, device="cuda"), torch.ones(n, device="cuda")
    y = torch.zeros(n, dtype=torch.int32, device="cuda")
    nv = torch.zeros(1, dtype=torch.int32, device="cuda")
    dx, dg = [torch.empty(n, d, device="cuda") for _ in range(2)], [torch.empty(d, device="cuda") for _ in range(2)]
    ws = [torch.empty(G.gist_rms_norm_bwd_workspace(n, d), dtype=torch.uint8, device="cuda") for _ in range(2)]
    call = lambda c, k: G.gist_rms_norm_bwd(c, n, d, dy, d, 0, h, d, 0, gain, rstd, None, d, dx[k], d, dg[k], ws[k], y, nv)
    torch.cuda.synchronize()
    G.gist_capture_begin(cap)
    try:
        call(cap, 0)
    finally:
        rep = G.gist_capture_end(cap)
    for k in range(3):
        y.zero_()
        y[50:60] = -1
        y[k::7] = -1
        nv.fill_(n - 40 * k)
        G.gist_replay_launch(ctx, rep, None, None, 0)
        call(ctx, 1)
        torch.cuda.synchronize()
        assert torch.equal(dx[0], dx[1]) and torch.equal(dg[0], dg[1]) and bool(torch.isfinite(dg[0]).all()), k
