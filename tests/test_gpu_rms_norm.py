"""GPU parity of the root-mean-square norm with the residual's addition, its 8-bit rows and its
gradients against 64 bits: every store, widths around the register and workgroup sizes, strides,
shared arrays, rows of zeros, non-finite rows, within bounds derived in more_ref."""

import numpy as np
import pytest

import more_ref as R
from gpu_util import to_dev, to_host

pytestmark = pytest.mark.gpu
EPS = float(np.float32(1e-6))


@pytest.fixture(scope="module")
def G():
    from paper_2102_10424_amd import gist
    return gist


@pytest.fixture(scope="module")
def ctx(G):
    return G.Context(0)


def padded(t, ld, fill=float("nan")):
    """t in rows of ld elements, one more row behind, all else `fill`."""
    import torch
    out = torch.full((t.shape[0] + 1, ld), fill, dtype=torch.float32).to(t.dtype)
    out[:-1, :t.shape[1]] = t
    return out.cuda()


def rows(n, d, store, rng, spread=1.0):
    import torch
    x = rng.standard_normal((n, d)) * np.exp(spread * rng.standard_normal((n, 1)))
    return torch.from_numpy(x.astype(np.float32)).to(R.torch_type(store))


def forward(G, ctx, x, r, gain, store, out, pad=0):
    """Runs with every array in rows of d + pad; returns h, y, y_scale, rstd on the host and the
    device arrays."""
    import torch
    n, d = x.shape
    ld = d + pad
    X, Rr = padded(x, ld), None if r is None else padded(r, ld)
    Hh = torch.full((n + 1, ld), 7.0, device="cuda").to(R.torch_type(store))
    Y = torch.full((n + 1, ld), 7.0, device="cuda").to(R.torch_type(out))
    s = torch.full((n + 1,), 7.0, device="cuda") if out == "e4m3" else None
    rstd = torch.full((n + 1,), 7.0, device="cuda")
    G.gist_rms_norm(ctx, n, d, X, ld, Rr, ld, R.store_of(G, store), to_dev(gain), EPS, Hh, ld, Y, ld,
                    R.store_of(G, out), s, rstd)
    h, y = to_host(Hh.float()), to_host(Y.float())
    for a in (h, y):                      # nothing beside or behind the rows
        assert (a[n:] == 7).all() and (a[:, d:] == 7).all()
    assert float(rstd[n]) == 7 and (s is None or float(s[n]) == 7)
    return h[:n, :d], y[:n, :d], None if s is None else to_host(s)[:n], to_host(rstd)[:n], Hh, rstd


SHAPES = [(1, 1), (3, 2), (5, 7), (2, 63), (9, 64), (4, 255), (300, 256), (7, 513), (1030, 600),
          (2, 1024), (33, 1500), (1025, 2048), (3, 2049), (1, 4096), (5, 8191), (2, 8192), (3, 8200),
          (2, 20011)]


@pytest.mark.parametrize("n,d", SHAPES)
@pytest.mark.parametrize("store,out", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"),
                                       ("f32", "bf16"), ("bf16", "f32"), ("f16", "e4m3"),
                                       ("f32", "e4m3"), ("bf16", "e4m3")])
def test_forward(G, ctx, n, d, store, out):
    rng = np.random.default_rng(n * 100003 + d)
    x = rows(n, d, store, rng)
    r = rows(n, d, store, rng) if d % 2 else None
    if n > 4:
        x[2] = 0
        if r is not None:
            r[2] = 0
    gain = (1 + 0.3 * rng.standard_normal(d)).astype(np.float32)
    h, y, s, rstd, _, _ = forward(G, ctx, x, r, gain, store, out, pad=(3 if n % 2 else 0))
    hw = x.float().numpy() if r is None else (x.float() + r.float()).to(x.dtype).float().numpy()
    assert np.array_equal(h, hw)
    want_rstd, want = R.rms(hw, gain, EPS)
    assert (np.abs(rstd - want_rstd) <= want_rstd * R.rstd_rel(d)).all()
    if out != "e4m3":
        assert (np.abs(y - want) <= R.rms_bound(hw, gain, EPS, out)).all()
        return
    top = np.abs(want).max(1)
    rel = R.rstd_rel(d) + 4 * R.U32
    assert (np.abs(s * R.TOP - top) <= top * (rel + 2 * R.U32)).all()
    a = want * np.where(top > 0, R.TOP / np.where(top > 0, top, 1), 0)[:, None]
    # half a step of the code, and the value's own error
    assert (np.abs(y - a) <= R.step_of(a) / 2 + np.abs(a) * 2 * rel).all()
    assert (np.abs(y).max(1)[top > 0] == R.TOP).all()


@pytest.mark.parametrize("n,d", SHAPES + [(4099, 96), (2500, 1040)])
@pytest.mark.parametrize("store,dys", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"),
                                       ("f32", "bf16"), ("bf16", "f32"), ("f16", "f32")])
def test_backward(G, ctx, n, d, store, dys):
    import torch
    rng = np.random.default_rng(n * 7 + d)
    h, dy = rows(n, d, store, rng, 0.3), rows(n, d, dys, rng, 0.3)
    ds = rows(n, d, store, rng, 0.3) if (n + d) % 2 else None
    gain = (1 + 0.3 * rng.standard_normal(d)).astype(np.float32)
    rstd, _ = R.rms(h.float().numpy(), gain, EPS)
    pad = 5 if d % 3 == 0 else 0
    ld = d + pad
    dx = torch.full((n + 1, ld), 7.0, device="cuda").to(h.dtype)
    dg = torch.full((d + 1,), 7.0, device="cuda")
    ws = torch.empty(G.gist_rms_norm_bwd_workspace(n, d), dtype=torch.uint8, device="cuda")
    args = (ctx, n, d, padded(dy, ld), ld, R.store_of(G, dys), padded(h, ld), ld,
            R.store_of(G, store), to_dev(gain), to_dev(rstd.astype(np.float32)),
            None if ds is None else padded(ds, ld), ld)
    G.gist_rms_norm_bwd(*args, dx, ld, dg, ws)
    x, bx, g, bg = R.rms_grad(dy.float().numpy(), h.float().numpy(), gain, EPS,
                              None if ds is None else ds.float().numpy())
    got = to_host(dx.float())
    assert (got[n:] == 7).all() and (got[:, d:] == 7).all() and float(dg[d]) == 7
    b = bx + R.HALF[store] * (np.abs(x) + bx) + (2.0 ** -25 if store == "f16" else 0)
    assert (np.abs(got[:n, :d] - x) <= b).all()
    assert (np.abs(to_host(dg)[:d] - g) <= bg).all()
    # either alone, and again: the same bits
    dx2, dg2 = torch.zeros_like(dx), torch.zeros_like(dg)
    G.gist_rms_norm_bwd(*args, dx2, ld, None, None)
    G.gist_rms_norm_bwd(*args, None, ld, dg2, ws)
    assert torch.equal(dx2[:n, :d], dx[:n, :d]) and torch.equal(dg2[:d], dg[:d])


def test_gradient_against_differences(G, ctx):
    """dx and dgain of sum(c y) by central differences of the library's own forward pass in fp32: step
    2^-5 loses 2^-10 / 6 of third derivatives of order one; fp32's rounding of y (2^-24 of
    values of up to 4) over 2^-4 adds 4 u 2^5 a term, of 40."""
    import torch
    n, d = 3, 40
    rng = np.random.default_rng(4)
    x = rng.standard_normal((n, d)).astype(np.float32)
    gain = (1 + 0.3 * rng.standard_normal(d)).astype(np.float32)
    c = rng.standard_normal((n, d)).astype(np.float32)

    def f(xx, gg):
        y = forward(G, ctx, torch.from_numpy(xx), None, gg, "f32", "f32")[1]
        return (c.astype(np.float64) * y).sum(1)

    _, _, _, rstd, H, rs = forward(G, ctx, torch.from_numpy(x), None, gain, "f32", "f32")
    dx, dg = torch.empty(n, d, device="cuda"), torch.empty(d, device="cuda")
    ws = torch.empty(G.gist_rms_norm_bwd_workspace(n, d), dtype=torch.uint8, device="cuda")
    G.gist_rms_norm_bwd(ctx, n, d, to_dev(c), d, 0, H, d, 0, to_dev(gain), rs, None, d, dx, d, dg, ws)
    dx, dg = to_host(dx), to_host(dg)
    s = 2.0 ** -5
    for j in range(d):
        e = np.zeros((n, d), np.float32)
        e[:, j] = s
        assert (np.abs((f(x + e, gain) - f(x - e, gain)) / (2 * s) - dx[:, j]) < 8e-3).all()
        eg = gain.copy()
        eg[j] += s
        em = gain.copy()
        em[j] -= s
        assert abs((f(x, eg) - f(x, em)).sum() / (2 * s) - dg[j]) < 1e-3


@pytest.mark.parametrize("d", [40, 300, 9000])
def test_shared_arrays(G, ctx, d):
    """h in x's or the residual's place, y in the other's; dx in dsum's, h's or dy's."""
    import torch
    n = 6
    rng = np.random.default_rng(d)
    x, r = rows(n, d, "bf16", rng), rows(n, d, "bf16", rng)
    gain = to_dev((1 + 0.3 * rng.standard_normal(d)).astype(np.float32))
    b = G.GIST_STORE_BF16
    new = lambda: torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
    h, y, rs = new(), new(), torch.empty(n, device="cuda")
    G.gist_rms_norm(ctx, n, d, x.cuda(), d, r.cuda(), d, b, gain, EPS, h, d, y, d, b, None, rs)
    for k in range(2):
        X, Rr = x.cuda(), r.cuda()
        hh, yy = (X, Rr) if k == 0 else (Rr, X)
        G.gist_rms_norm(ctx, n, d, X, d, Rr, d, b, gain, EPS, hh, d, yy, d, b, None, None)
        assert torch.equal(hh, h) and torch.equal(yy, y)
    dy, ds, dx = rows(n, d, "bf16", rng).cuda(), rows(n, d, "bf16", rng).cuda(), new()
    G.gist_rms_norm_bwd(ctx, n, d, dy, d, b, h, d, b, gain, rs, ds, d, dx, d, None, None)
    for k in range(3):
        a = [dy.clone(), h.clone(), ds.clone()]
        G.gist_rms_norm_bwd(ctx, n, d, a[0], d, b, a[1], d, b, gain, rs, a[2], d, a[k], d, None, None)
        assert torch.equal(a[k], dx)


@pytest.mark.parametrize("d", [40, 300, 2500, 9000])
def test_non_finite_rows(G, ctx, d):
    import torch
    n = 7
    rng = np.random.default_rng(d)
    x = rows(n, d, "f32", rng, 0.0)
    x[1, d // 2], x[3, 0], x[5, d - 1] = float("nan"), float("inf"), float("-inf")
    gain = np.ones(d, np.float32)
    _, y8, s, rstd, _, _ = forward(G, ctx, x, None, gain, "f32", "e4m3")
    bad = [1, 3, 5]
    good = [0, 2, 4, 6]
    assert np.isnan(s[bad]).all() and np.isnan(y8[bad]).all()
    assert np.isfinite(s[good]).all() and np.isfinite(y8[good]).all()
    _, y, _, _, _, _ = forward(G, ctx, x, None, gain, "f32", "f32")
    assert np.isnan(y[1]).all() and np.isfinite(y[good]).all()
    q, sc = torch.empty(n, d, dtype=torch.uint8, device="cuda"), torch.empty(n, device="cuda")
    G.gist_quantize_rows(ctx, n, d, to_dev(x.numpy()), d, 0, q, d, sc)
    v = to_host(q.view(torch.float8_e4m3fn).float())
    assert np.isnan(v[bad]).all() and np.isnan(to_host(sc)[bad]).all()
    assert np.isfinite(v[good]).all()


@pytest.mark.parametrize("n,d", [(1, 1), (5, 7), (300, 41), (3, 1000), (2, 9001)])
@pytest.mark.parametrize("store", ["f32", "bf16", "f16"])
def test_quantize_rows(G, ctx, n, d, store):
    import torch
    rng = np.random.default_rng(n + d)
    x = rows(n, d, store, rng)
    x[0, 0] = 0
    if n > 2:
        x[1] = 0
        x[2] = 2.0 ** -120 if store != "f16" else 0    # below 2^-100: zero
    q = torch.full((n + 1, d + 2), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.full((n + 1,), 7.0, device="cuda")
    G.gist_quantize_rows(ctx, n, d, padded(x, d + 1), d + 1, R.store_of(G, store), q, d + 2, s)
    raw = to_host(q)
    assert (raw[n] == 0x55).all() and (raw[:, d:] == 0x55).all() and float(s[n]) == 7
    v = to_host(q.view(torch.float8_e4m3fn).float())[:n, :d]
    xs, s = x.double().numpy(), to_host(s)[:n]
    top = np.abs(xs).max(1)
    zero = top < 2.0 ** -100
    assert (s[zero] == 0).all() and (v[zero] == 0).all()
    a = xs[~zero] * (R.TOP / top[~zero])[:, None]
    assert (np.abs(s[~zero] * R.TOP - top[~zero]) <= 2 * R.U32 * top[~zero]).all()
    assert (np.abs(v[~zero] - a) <= R.step_of(a) / 2 + np.abs(a) * 4 * R.U32).all()


def test_no_rows(G, ctx):
    import torch
    dg = torch.full((5,), 3.0, device="cuda")
    e = torch.empty(0, 5, device="cuda")
    G.gist_rms_norm(ctx, 0, 5, e, 5, None, 5, 0, dg, EPS, None, 5, e, 5, 0, None, None)
    G.gist_rms_norm_bwd(ctx, 0, 5, e, 5, 0, e, 5, 0, dg.clone(), None, None, 5, e, 5, dg, None)
    assert (to_host(dg) == 0).all()       # the sum over no rows


# Where the number of threads and of elements a row changes, and rows that no workgroup holds.
EDGES = [(50, 16), (4097, 41), (33, 128), (17, 129), (1000, 130), (600, 512), (70, 516), (5, 520),
         (40, 1025), (3, 4104), (2, 16384), (2, 16385), (3, 32768), (2, 32769), (2, 40003)]


@pytest.mark.parametrize("n,d", EDGES)
@pytest.mark.parametrize("store,out", [("f32", "f32"), ("bf16", "bf16"), ("f16", "e4m3"),
                                       ("f32", "e4m3")])
def test_forward_at_edges(G, ctx, n, d, store, out):
    test_forward(G, ctx, n, d, store, out)


@pytest.mark.parametrize("n,d", EDGES)
@pytest.mark.parametrize("store,dys", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32"),
                                       ("f32", "bf16")])
def test_backward_at_edges(G, ctx, n, d, store, dys):
    test_backward(G, ctx, n, d, store, dys)


@pytest.mark.parametrize("d", [16, 130, 17000, 40000])
def test_shared_arrays_at_edges(G, ctx, d):
    test_shared_arrays(G, ctx, d)


@pytest.mark.parametrize("d", [16, 100, 130, 17000, 40001])
def test_non_finite_rows_at_edges(G, ctx, d):
    test_non_finite_rows(G, ctx, d)


@pytest.mark.parametrize("n,d", [(40, 16), (300, 128), (9, 512), (2, 40003)])
@pytest.mark.parametrize("store", ["f32", "bf16", "f16"])
def test_quantize_rows_at_edges(G, ctx, n, d, store):
    test_quantize_rows(G, ctx, n, d, store)


def codes_in_64_bits(v):
    """Nearest codes (ties to even) of rows whose largest magnitude is 448; |code| < 2^-6 are left out."""
    v = to_host(v)
    a = v * (R.TOP / np.abs(v).max(1, keepdims=True))
    return R.e4m3(a), np.abs(a) >= 2.0 ** -6


@pytest.mark.parametrize("n,d", [(60000, 40), (30000, 130), (3000, 2048), (1500, 4099), (800, 4096), (150, 20000),
                                 (60, 40001)])
@pytest.mark.parametrize("store", ["f32", "bf16"])
def test_codes_are_exact(G, ctx, n, d, store):
    """Every code is the nearest of the 64-bit value, whichever side of a middle 32 bits would put it."""
    import torch
    torch.manual_seed(d)
    t = R.torch_type(store)
    x, r = torch.randn(n, d, device="cuda").to(t), torch.randn(n, d, device="cuda").to(t)
    gain = 1 + 0.2 * torch.randn(d, device="cuda")
    y, s = torch.empty(n, d, dtype=torch.uint8, device="cuda"), torch.empty(n, device="cuda")
    st = R.store_of(G, store)
    value = lambda: to_host(y.view(torch.float8_e4m3fn).double())
    for res in (r, None):
        h = x if res is None else (x.float() + r.float()).to(t)
        want, counts = codes_in_64_bits(h.double() * gain.double())
        into = torch.empty_like(x)
        for hh in (into, None):
            G.gist_rms_norm(ctx, n, d, x, d, res, d, st, gain, EPS, hh, d, y, d, G.GIST_STORE_E4M3, s, None)
            assert np.array_equal(value()[counts], want[counts])
    G.gist_quantize_rows(ctx, n, d, x, d, st, y, d, s)
    want, counts = codes_in_64_bits(x.double())
    assert np.array_equal(value()[counts], want[counts])
    # h in x's place
    z = x.clone()
    G.gist_rms_norm(ctx, n, d, z, d, r, d, st, gain, EPS, z, d, y, d, G.GIST_STORE_E4M3, s, None)
    want, counts = codes_in_64_bits((x.float() + r.float()).to(t).double() * gain.double())
    assert np.array_equal(value()[counts], want[counts])


@pytest.mark.parametrize("d", [16, 449, 2000, 9000, 40000])
def test_codes_of_exact_middles(G, ctx, d):
    """Whole numbers up to 448, of which many lie in the middle between two codes: to the even one."""
    import torch
    torch.manual_seed(d)
    x = torch.randint(-447, 448, (20, d), device="cuda").float()
    x[:, d // 2] = 448
    y, s = torch.empty(20, d, dtype=torch.uint8, device="cuda"), torch.empty(20, device="cuda")
    G.gist_quantize_rows(ctx, 20, d, x, d, G.GIST_STORE_F32, y, d, s)
    want, _ = codes_in_64_bits(x.double())
    assert np.array_equal(to_host(y.view(torch.float8_e4m3fn).double()), want) and bool((s == 1).all())
