"""GPU parity of the log probabilities, entropy, best classes and their
gradient against 64 bits, at one class and many, one row and many, masked
rows and classes, missing and wrong tokens, non-finite logits, ties, strides
and offsets, within bounds derived in ops_ref."""

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


def logits(n, C, store, rng, kind="plain"):
    """Values as stored (float32 array of them) and the padded device tensor's source."""
    import torch
    z = (rng.standard_normal((n, C)) * 3).astype(np.float32)
    if kind == "masked":
        z[rng.random((n, C)) < 0.4] = -np.inf
        z[::3] = -np.inf
        if n > 4:
            z[4, C // 2] = 1.5            # one class left
    elif kind == "lowest":
        low = dict(f32=np.finfo(np.float32).min, bf16=-3.3895e38, f16=-65504.0)[store]
        z[rng.random((n, C)) < 0.5] = low
        z[::4] = low
    elif kind == "offset":
        z += np.float32(400.0) * np.where(np.arange(n) % 2, 1, -1)[:, None].astype(np.float32)
    elif kind == "ties":
        z = np.round(z)
        z[z == 0] = np.where(rng.random((n, C)) < 0.5, -0.0, 0.0).astype(np.float32)[z == 0]
    elif kind == "ascending":
        z = np.sort(z, axis=1)
    return torch.from_numpy(z).to(R.torch_type(store))


def forward(G, ctx, t, store, y, K, ldz=None, want_all=True):
    import torch
    n, C = t.shape
    ldz = ldz or C
    dev = torch.full((n, ldz), float("nan"), dtype=t.dtype, device="cuda")
    dev[:, :C] = t.cuda()
    o = lambda *s: torch.full(s, 9.0, device="cuda")
    lp, H, l, top = o(n + 1), o(n + 1), o(n + 1), o(n + 1, max(K, 1))
    idx = torch.full((n + 1, max(K, 1)), 77, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(16, G.gist_log_probs_workspace(n, C, K)), dtype=torch.uint8, device="cuda")
    G.gist_log_probs(ctx, n, C, dev, ldz, R.store_of(G, store), to_dev(y), lp, H, l, K,
                     top if K else None, idx if K else None, ws)
    for x in (lp, H, l, top):
        assert (to_host(x)[n:] == 9).all()       # nothing behind the rows
    assert (to_host(idx)[n:] == 77).all()
    return dev, lp[:n], H[:n], l[:n], top[:n, :K], idx[:n, :K]


def close(got, want, bound):
    """Equal where not finite, else within the bound."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    fin = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[~fin & ~np.isnan(want)], want[~fin & ~np.isnan(want)])
    err = np.where(fin, np.abs(np.where(fin, got, 0) - np.where(fin, want, 0)), 0)
    bound = np.broadcast_to(bound, err.shape)
    worst = float(np.max(err / bound)) if err.size else 0.0
    assert (err <= bound).all(), worst
    return worst


SHAPES = [(1, 1, 1), (5, 2, 2), (7, 7, 3), (300, 41, 5), (64, 47, 47), (33, 64, 64), (20, 65, 20),
          (9, 130, 0), (6, 1000, 32), (3, 4096, 8), (2, 5003, 20), (1, 32000, 20), (1, 100003, 64),
          (2, 131072, 5), (1100, 129, 4), (40, 8192, 1), (2000, 16, 2)]


@pytest.mark.parametrize("store", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,C,K", SHAPES)
def test_forward(G, ctx, store, n, C, K):
    rng = np.random.default_rng(n * 13 + C + K)
    kinds = ["plain", "masked", "lowest", "offset", "ties", "ascending"] if C <= 8192 else \
        ["plain", "masked", "ties"]
    for kind in kinds:
        t = logits(n, C, store, rng, kind)
        z = t.float().numpy()
        y = rng.integers(-1, C, n).astype(np.int32)
        y[0] = C - 1
        ldz = C + (n + C) % 3 * 4
        _, lp, H, l, top, idx = forward(G, ctx, t, store, y, K, ldz)
        wl, wlp, wH = R.log_probs(z, y)
        lb = R.lse_bound(z)
        a = close(to_host(l), wl, lb)
        b = close(to_host(lp), wlp, lb + R.U32 * np.abs(np.where(np.isfinite(wlp), wlp, 0)))
        c = close(to_host(H), wH, R.entropy_bound(z))
        wi = R.top_classes(z, K)
        assert np.array_equal(to_host(idx), wi), kind
        if K:
            zt = np.take_along_axis(z.astype(np.float64), wi.astype(np.int64), 1)
            with np.errstate(invalid="ignore"):
                wt = np.where(zt == -np.inf, -np.inf, zt - wl[:, None])
            close(to_host(top), wt, lb[:, None] + R.U32 * np.abs(np.where(np.isfinite(wt), wt, 0)))
        log(f"log_probs {store} n={n} C={C} K={K} {kind}: error / bound lse {a:.2f} logp {b:.2f} H {c:.2f}")


@pytest.mark.parametrize("store", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,C,K", [(8, 5, 5), (9, 47, 4), (4, 300, 8), (2, 20000, 6), (8, 16, 3)])
def test_nonfinite_and_wrong_tokens(G, ctx, store, n, C, K):
    rng = np.random.default_rng(C)
    t = logits(n, C, store, rng)
    t[0, C // 2] = float("nan")
    t[1, C - 1] = float("inf")
    if n > 5:
        t[2] = -float("inf")
        t[2, 0] = float("nan")
        t[5] = -float("inf")
        t[5, C - 1] = float("inf")
    y = rng.integers(0, C, n).astype(np.int32)
    y[n - 1] = C                       # the caller's mistake
    y[n - 2] = -5                      # no given class
    _, lp, H, l, top, idx = forward(G, ctx, t, store, y, K)
    z = t.float().numpy()
    wl, wlp, wH = R.log_probs(z, y)
    close(to_host(l), wl, R.lse_bound(z))
    close(to_host(lp), wlp, R.lse_bound(z) * 2)
    close(to_host(H), wH, R.entropy_bound(z))
    assert np.array_equal(to_host(idx), R.top_classes(z, K))
    assert np.isnan(to_host(top)[:2]).all() and np.isfinite(to_host(top)[3:4]).all()


def test_outputs_not_wanted(G, ctx):
    """Any output may be left out; the others are what they are with all."""
    import torch
    n, C, K = 50, 77, 3
    rng = np.random.default_rng(1)
    t = logits(n, C, "f32", rng)
    y = rng.integers(0, C, n).astype(np.int32)
    dev, lp, H, l, top, idx = forward(G, ctx, t, "f32", y, K)
    ws = torch.empty(16, dtype=torch.uint8, device="cuda")
    e = torch.empty(n, device="cuda")
    G.gist_log_probs(ctx, n, C, dev, C, 0, None, None, e, None, 0, None, None, ws)
    assert torch.equal(e, H)
    G.gist_log_probs(ctx, n, C, dev, C, 0, None, None, None, e, 0, None, None, None)
    assert torch.equal(e, l)
    G.gist_log_probs(ctx, n, C, dev, C, 0, to_dev(y), e, None, None, 0, None, None, ws)
    assert torch.equal(e, lp)
    i2, t2 = torch.empty_like(idx), torch.empty_like(top)
    t2, i2 = t2.contiguous(), i2.contiguous()
    G.gist_log_probs(ctx, n, C, dev, C, 0, None, None, None, None, K, t2, i2, ws)
    assert torch.equal(i2, idx) and torch.equal(t2, top)
    G.gist_log_probs(ctx, n, C, dev, C, 0, None, None, None, None, 0, None, None, ws)
    G.gist_log_probs(ctx, 0, C, None, C, 0, None, None, None, None, 0, None, None, ws)


@pytest.mark.parametrize("store", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,C", [(1, 1), (5, 2), (300, 41), (64, 47), (33, 64), (20, 130), (6, 1000),
                                 (2, 5003), (1, 32000), (1, 100003), (3, 16384), (1500, 12)])
def test_backward(G, ctx, store, n, C):
    import torch
    rng = np.random.default_rng(n + C)
    for kind in ("plain", "masked", "lowest", "offset"):
        t = logits(n, C, store, rng, kind)
        z = t.float().numpy()
        y = rng.integers(-1, C, n).astype(np.int32)
        y[0] = C - 1
        ldz = C + (n + C) % 3 * 4
        dev, _, H, l, _, _ = forward(G, ctx, t, store, y, 0, ldz)
        glh, ghh = (rng.standard_normal(n).astype(np.float32) for _ in range(2))
        for gl, gh in ((glh, ghh), (glh, None), (None, ghh)):
            ldd = C + 3
            dz = torch.full((n + 1, ldd), 5.0, dtype=t.dtype, device="cuda")
            G.gist_log_probs_bwd(ctx, n, C, dev, ldz, R.store_of(G, store), to_dev(y), l, H,
                                 None if gl is None else to_dev(gl),
                                 None if gh is None else to_dev(gh), dz, ldd)
            got = to_host(dz.float())
            want = R.log_probs_grad(z, y, gl, gh)
            w = close(got[:n, :C], want, R.grad_bound(z, y, gl, gh, store) + 1e-45)
            assert (got[n:] == 5).all() and (got[:, C:] == 5).all()
        log(f"log_probs_bwd {store} n={n} C={C} {kind}: error / bound {w:.2f}")


@pytest.mark.parametrize("C", [40, 3000])
def test_backward_special_rows(G, ctx, C):
    """In place; a masked row has gradient 0, a row with a NaN or a token past the classes
    NaN, a row without a token no log-probability term."""
    n = 6
    rng = np.random.default_rng(C)
    t = logits(n, C, "f32", rng)
    t[0], t[1, 3] = -float("inf"), float("nan")
    y = rng.integers(0, C, n).astype(np.int32)
    y[2], y[3] = C, -1
    dev, _, H, l, _, _ = forward(G, ctx, t, "f32", y, 0)
    gl, gh = (rng.standard_normal(n).astype(np.float32) for _ in range(2))
    G.gist_log_probs_bwd(ctx, n, C, dev, C, 0, to_dev(y), l, H, to_dev(gl), to_dev(gh), dev, C)
    z = t.numpy()
    close(to_host(dev), R.log_probs_grad(z, y, gl, gh),
          np.nan_to_num(R.grad_bound(z, y, gl, gh, "f32")) + 1e-45)


@pytest.mark.parametrize("store", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("C,K", [(1, 1), (2, 2), (3, 0), (5, 3), (16, 8), (24, 6), (33, 4), (41, 5), (42, 7)])
def test_many_short_rows(G, ctx, store, C, K):
    """Many rows one after another take a lane each; the same rows a column further apart take
    several.  The same classes and, where both are within the bound of the 64-bit values, at
    most two bounds between them; some rows against those values."""
    import torch
    n = 98304 + 37
    rng = np.random.default_rng(C * 10 + K)
    for kind in ("plain", "masked", "ties", "lowest", "offset"):
        t = logits(n, C, store, rng, kind)
        y = rng.integers(-1, C + 1, n).astype(np.int32)
        t[n // 2, C // 2], t[n - 1, 0], t[7] = float("nan"), float("inf"), -float("inf")
        a = [to_host(x) for x in forward(G, ctx, t, store, y, K, C)[1:]]
        b = [to_host(x) for x in forward(G, ctx, t, store, y, K, C + 1)[1:]]
        z = t.float().numpy()
        lb = R.lse_bound(z) * 2
        assert np.array_equal(a[4], b[4])
        with np.errstate(invalid="ignore"):
            close(a[2], b[2], lb)
            close(a[1], b[1], 2 * R.entropy_bound(z))
            for i in (0, 3):
                bound = lb if i == 0 else lb[:, None]
                close(a[i], b[i], bound + 2 * R.U32 * np.abs(np.where(np.isfinite(b[i]), b[i], 0)))
        some = np.unique(np.concatenate([np.arange(0, n, 991), [7, n // 2, n - 1]]))
        z = z[some]
        wl, wlp, wH = R.log_probs(z, y[some])
        lb = R.lse_bound(z)
        close(a[2][some], wl, lb)
        close(a[0][some], wlp, lb + R.U32 * np.abs(np.where(np.isfinite(wlp), wlp, 0)))
        close(a[1][some], wH, R.entropy_bound(z))
        if K:
            wi = np.where(np.isnan(wl)[:, None], -1, R.top_classes(z, K))
            assert np.array_equal(a[4][some], wi)


FAR = dict(f32=[1e5, -3e7, 2e30], bf16=[1e4, -3e7, 2e30], f16=[3e4, -6e4])


@pytest.mark.parametrize("store", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,C,K", [(3, 1, 1), (40, 47, 5), (9, 130, 3), (5, 400, 2), (6, 1000, 8), (3, 20011, 4),
                                   (1100, 1100, 2), (1, 100003, 20)])
def test_far_rows(G, ctx, store, n, C, K):
    """Rows whose offset swallows log s in an fp32 lse: whole rows of the type's lowest value,
    and offsets of up to 2e30.  Log probabilities and gradients are those of the row without
    its offset (an exact subtraction in 64 bits), in place too.  Bounds: (z - m) is rounded
    once (u of |logp| + log C), log s errs as an lse without maximum.  The gradient's exponents
    (z - l) - log s' take two roundings more, and s' as many errors as s: twice grad_bound."""
    import torch
    rng = np.random.default_rng(n + C)
    low = dict(f32=float(np.finfo(np.float32).min), bf16=-3.3895e38, f16=-65504.0)[store]
    for far in FAR[store] + ["lowest"]:
        z = (rng.standard_normal((n, C)) * 3).astype(np.float32)
        if far == "lowest":
            z[:] = low
            if n > 2:
                z[2, ::2] = np.float32(low / 2)
        else:
            z = np.float32(far) + z
            z[rng.random((n, C)) < 0.2] = -np.inf
            z[:, C // 2] = np.float32(far)
        t = torch.from_numpy(z).to(R.torch_type(store))
        z = t.double().numpy()
        z = z - z.max(1, keepdims=True)
        y = rng.integers(0, C, n).astype(np.int32)
        dev, lp, H, l, top, idx = forward(G, ctx, t, store, y, K)
        _, wlp, wH = R.log_probs(z, y)
        near = R.lse_bound(z) + 4 * R.U32 * np.log(C + 1)
        close(to_host(lp), wlp, near + 4 * R.U32 * np.abs(np.where(np.isfinite(wlp), wlp, 0)))
        close(to_host(H), wH, R.entropy_bound(z))
        wi = R.top_classes(z, K)
        assert np.array_equal(to_host(idx), wi)
        wt = np.stack([R.log_probs(z, wi[:, k])[1] for k in range(K)], 1)
        close(to_host(top), wt, near[:, None] + 4 * R.U32 * np.abs(np.where(np.isfinite(wt), wt, 0)))
        gl, gh = (rng.standard_normal(n).astype(np.float32) for _ in range(2))
        want = R.log_probs_grad(z, y, gl, gh)
        bound = 2 * R.grad_bound(z, y, gl, gh, store) + 1e-45
        dz = torch.full_like(dev, 5.0)
        G.gist_log_probs_bwd(ctx, n, C, dev, C, R.store_of(G, store), to_dev(y), l, H, to_dev(gl), to_dev(gh), dz, C)
        w = close(to_host(dz.float()), want, bound)
        G.gist_log_probs_bwd(ctx, n, C, dev, C, R.store_of(G, store), to_dev(y), l, H, to_dev(gl), to_dev(gh), dev, C)
        assert torch.equal(dev.float().isnan(), dz.float().isnan())
        close(to_host(dev.float()), want, bound)
        log(f"far rows {store} n={n} C={C} {far}: error / bound {w:.2f}")


@pytest.mark.parametrize("store,n,C", [("f32", 600, 16400), ("f32", 200, 70000), ("f32", 70, 65536), ("f32", 520, 32768),
                                       ("bf16", 1100, 32000), ("f16", 530, 65537), ("bf16", 90, 131072), ("f32", 3, 300000),
                                       ("f32", 513, 16384 + 8192)])
def test_far_rows_among_near_ones(G, ctx, store, n, C):
    """Rows of several column slabs, every third far: those go to fewer groups than the others.
    Rows at every place of a round of workgroups against 64 bits, within the bounds of
    test_far_rows; all rows within two of them of the gradient in place, which has one group a row
    (its sum of exp(z - lse) and its rounding differ)."""
    import torch
    rng = np.random.default_rng(n + C)
    g = torch.Generator(device="cuda").manual_seed(n + C)
    dev = torch.randn(n, C, generator=g, device="cuda") * 3
    dev[::3] += 1000.0
    dev[1::5, : C // 3] = -float("inf")
    dev = dev.to(R.torch_type(store))
    y = rng.integers(0, C, n).astype(np.int32)
    o = lambda: torch.empty(n, device="cuda")
    lp, H, l, ws = o(), o(), o(), torch.empty(max(16, G.gist_log_probs_workspace(n, C, 0)), dtype=torch.uint8, device="cuda")
    s = R.store_of(G, store)
    G.gist_log_probs(ctx, n, C, dev, C, s, to_dev(y), lp, H, l, 0, None, None, ws)
    glh, ghh = (rng.standard_normal(n).astype(np.float32) for _ in range(2))
    gl, gh = to_dev(glh), to_dev(ghh)
    dz = torch.full((n + 1, C), 5.0, dtype=dev.dtype, device="cuda")
    G.gist_log_probs_bwd(ctx, n, C, dev, C, s, to_dev(y), l, H, gl, gh, dz, C)
    assert bool((dz[n].float() == 5).all())
    some = np.unique(np.concatenate([np.arange(0, min(n, 66), 3), [1, 2, n // 2, n - 1], np.arange(n % 3, n, 96)]))
    some = some[some < n][:40]
    bound = np.empty((len(some), C))
    for i, v in enumerate(some):
        z = dev[v:v + 1].double().cpu().numpy()
        z = z - z.max()
        w = slice(v, v + 1)
        bound[i] = 2 * R.grad_bound(z, y[w], glh[w], ghh[w], store) + 1e-45
        close(to_host(dz[w].float()), R.log_probs_grad(z, y[w], glh[w], ghh[w]), bound[i])
    G.gist_log_probs_bwd(ctx, n, C, dev, C, s, to_dev(y), l, H, gl, gh, dev, C)
    assert not bool((dz[:n].float() - dev.float()).isnan().any())
    got, inp = to_host(dz[torch.from_numpy(some).cuda()].float()), to_host(dev[torch.from_numpy(some).cuda()].float())
    assert (np.abs(got.astype(np.float64) - inp) <= 2 * bound).all()
    # an element left unwritten or written by the wrong row would be off by whole probabilities
    assert float((dz[:n].float() - dev.float()).abs().max()) <= float(2 * bound.max())


def test_far_rows_cost_no_more_with_more_columns(G, ctx):
    """An offset of the logits makes a row's gradient read it twice, not once per slab: 300
    rows of 123 slabs take about twice the time of rows without one, not tens of times."""
    import torch
    n, C = 300, 1000003
    z = torch.randn(n, C, device="cuda")
    y = torch.zeros(n, dtype=torch.int32, device="cuda")
    gl = torch.ones(n, device="cuda")
    lp, H, l = (torch.empty(n, device="cuda") for _ in range(3))
    ws = torch.empty(G.gist_log_probs_workspace(n, C, 0), dtype=torch.uint8, device="cuda")
    dz = torch.empty_like(z)
    us = []
    for offset in (0.0, 1000.0):
        z += offset
        G.gist_log_probs(ctx, n, C, z, C, 0, y, lp, H, l, 0, None, None, ws)
        times = []
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            G.gist_log_probs_bwd(ctx, n, C, z, C, 0, y, l, H, gl, gl, dz, C)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b) * 1e3)
        us.append(sorted(times)[2])
    log(f"far rows: {us[0]:.0f} us without an offset, {us[1]:.0f} with one")
    assert us[1] < 8 * us[0]


def test_gradient_against_differences(G, ctx):
    """The gradient against differences of the library's own values: a change h of one logit
    changes logp and entropy by h g + O(h^2); with h = 2^-6 the second-order term is below
    h^2 (curvatures below 2 for these logits), the values' errors two bounds over h."""
    import torch
    n, C = 4, 50
    rng = np.random.default_rng(2)
    t = logits(n, C, "f32", rng)
    y = rng.integers(0, C, n).astype(np.int32)
    dev, _, H, l, _, _ = forward(G, ctx, t, "f32", y, 0)
    one = to_dev(np.ones(n, np.float32))
    h = 2.0 ** -6
    for gl, gh, pick in ((one, None, 0), (None, one, 1)):
        dz = torch.empty(n, C, device="cuda")
        G.gist_log_probs_bwd(ctx, n, C, dev, C, 0, to_dev(y), l, H, gl, gh, dz, C)
        got = to_host(dz)
        for j in range(0, C, 7):
            f = []
            for s in (h, -h):
                u = t.clone()
                u[:, j] += s
                f.append(to_host(forward(G, ctx, u, "f32", y, 0)[1 + pick]).astype(np.float64))
            diff = (f[0] - f[1]) / (2 * h)
            tol = h * h + (R.lse_bound(t.numpy()) + R.entropy_bound(t.numpy())) / h
            assert (np.abs(diff - got[:, j]) <= tol).all()


def test_logits_beyond_32_bit_offsets(G, ctx):
    """Rows whose elements lie past 2^31."""
    import torch
    n, C = 17000, 131072            # 2.2e9 elements, 4.5 GB
    dev = torch.zeros(n, C, dtype=torch.bfloat16, device="cuda")
    dev[n - 1, 70000] = 20.0
    y = torch.zeros(n, dtype=torch.int32, device="cuda")
    y[n - 1] = 70000
    o = lambda *s: torch.empty(*s, device="cuda")
    lp, H, l, top = o(n), o(n), o(n), o(n, 1)
    idx = torch.empty(n, 1, dtype=torch.int32, device="cuda")
    G.gist_log_probs(ctx, n, C, dev, C, G.GIST_STORE_BF16, y, lp, H, l, 1, top, idx, None)
    want = -np.log1p((C - 1) * np.exp(-20.0))
    assert abs(to_host(lp)[-1] - want) < 1e-5 and to_host(idx)[-1, 0] == 70000
    assert np.allclose(to_host(lp)[:-1], -np.log(C), rtol=1e-6) and (to_host(idx)[:-1] == 0).all()
    g = torch.ones(n, device="cuda")
    G.gist_log_probs_bwd(ctx, n, C, dev, C, G.GIST_STORE_BF16, y, l, None, g, None, dev, C)
    assert abs(float(dev[n - 1, 70000]) - (1 - np.exp(want))) < 2 ** -8
    assert abs(float(dev[n - 2, 0]) - 1) < 2 ** -8 and float(dev[n - 2, 1]) < 0


@pytest.mark.parametrize("n,C,K", [(200, 47, 5), (2, 40000, 20)])
def test_replays(G, n, C, K):
    """Forward and gradient recorded once; every replay on new logits equals the eager
    calls."""
    import torch
    st = torch.cuda.Stream()
    cctx, ectx = G.Context(0, stream=st.cuda_stream), G.Context(0)
    rng = np.random.default_rng(3)
    z = torch.empty(n, C, device="cuda")
    y = to_dev(rng.integers(0, C, n).astype(np.int32))
    gl = to_dev(rng.standard_normal(n).astype(np.float32))
    sets = []
    for _ in range(2):
        o = lambda *s: torch.zeros(*s, device="cuda")
        sets.append((o(n), o(n), o(n), o(n, K), torch.zeros(n, K, dtype=torch.int32, device="cuda"),
                     torch.empty(max(16, G.gist_log_probs_workspace(n, C, K)), dtype=torch.uint8,
                                 device="cuda"), o(n, C)))

    def calls(c, s):
        G.gist_log_probs(c, n, C, z, C, 0, y, s[0], s[1], s[2], K, s[3], s[4], s[5])
        G.gist_log_probs_bwd(c, n, C, z, C, 0, y, s[2], s[1], gl, gl, s[6], C)

    torch.cuda.synchronize()
    G.gist_capture_begin(cctx)
    calls(cctx, sets[0])
    r = G.gist_capture_end(cctx)
    for k in range(4):
        z.copy_(logits(n, C, "f32", rng, "masked" if k % 2 else "plain"))
        calls(ectx, sets[1])
        G.gist_replay_launch(ectx, r)
        torch.cuda.synchronize()
        for a, b in zip(sets[0][:5] + sets[0][6:], sets[1][:5] + sets[1][6:]):
            assert torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)), k
