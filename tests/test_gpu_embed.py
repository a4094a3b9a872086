"""GPU parity of the learned rows: lookup (bit-exact), the table's gradient by
sorted ids and its fused SGD step, at the sizes and ids where they can go
wrong: nothing to look up, one row, all rows alike, padding, ids outside the
table, chunk and tile borders, odd widths, strides, offsets."""

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


def make_ids(kind, n, V, rng):
    if kind == "same":
        return np.full(n, V // 2, np.int32)
    if kind == "padding":
        return np.where(rng.random(n) < 0.5, -1, V).astype(np.int32)
    if kind == "distinct":
        return rng.permutation(max(n, V))[:n].astype(np.int32) % V if n <= V else \
            (np.arange(n) % V).astype(np.int32)
    if kind == "ascending":
        return np.sort(rng.integers(0, V, n)).astype(np.int32)
    ids = (np.exp(rng.random(n) * np.log(V + 1)) - 1).astype(np.int64).clip(0, V - 1)
    ids = rng.permutation(V)[ids].astype(np.int32)      # power law
    if kind == "mixed":
        ids[rng.random(n) < 0.1] = -1
        ids[rng.random(n) < 0.05] = V
        if n > 4:
            ids[1], ids[3] = np.iinfo(np.int32).min, np.iinfo(np.int32).max
    return ids


@pytest.mark.parametrize("store", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,V,d,pad", [
    (0, 5, 4, 0), (1, 1, 1, 0), (3, 2, 7, 0), (257, 300, 100, 0), (40, 70000, 602, 0),
    (9, 50, 4096, 0), (5, 20, 1030, 2), (33, 20, 96, 8), (70, 11, 8, 1), (2, 3, 5000, 0),
    (1000, 17, 1, 0), (300, 0, 12, 0)])
def test_lookup(G, ctx, store, n, V, d, pad):
    import torch
    log(f"lookup {store} n={n} V={V} d={d} pad={pad}")
    rng = np.random.default_rng(n + V + d)
    full = torch.from_numpy(rng.standard_normal((max(V, 1), d + pad)).astype(np.float32))
    full = full.to(R.torch_type(store)).cuda()
    ids = make_ids("mixed", n, V, rng) if V else np.zeros(n, np.int32)
    out = torch.full((n + 2, d + pad), 7.0, device="cuda")
    scale = 0.37
    G.gist_embed_lookup(ctx, n, V, d, full if V else None, d + pad, R.store_of(G, store),
                        to_dev(ids), scale, out, d + pad)
    got = to_host(out)
    t = to_host(full.float())
    ok = (ids >= 0) & (ids < V)
    want = np.zeros((n, d), np.float32)
    want[ok] = t[ids[ok], :d] * np.float32(scale)
    assert np.array_equal(got[:n, :d], want)
    assert (got[n:] == 7).all() and (got[:, d:] == 7).all()    # nothing behind the rows


@pytest.mark.parametrize("store,shift", [("f32", 1), ("f32", 2), ("bf16", 1), ("bf16", 4), ("f16", 2)])
def test_lookup_offset_table(G, ctx, store, shift):
    """A table and an output that begin inside an allocation, off the vector alignment."""
    import torch
    V, d, n = 30, 64, 50
    rng = np.random.default_rng(shift)
    flat = torch.from_numpy(rng.standard_normal(V * d + shift).astype(np.float32))
    flat = flat.to(R.torch_type(store)).cuda()
    ids = rng.integers(0, V, n).astype(np.int32)
    out = torch.zeros(n * d + shift, device="cuda")
    G.gist_embed_lookup(ctx, n, V, d, flat[shift:], d, R.store_of(G, store), to_dev(ids), 2.0,
                        out[shift:], d)
    want = 2 * to_host(flat.float())[shift:].reshape(V, d)[ids]
    assert np.array_equal(to_host(out)[shift:].reshape(n, d), want)


CASES = [(1, 1, 1, "same"), (1, 1000, 6, "distinct"), (31, 5, 4, "mixed"), (32, 5, 4, "same"),
         (33, 7, 100, "same"), (64, 255, 260, "distinct"), (200, 256, 8, "padding"),
         (4096, 257, 12, "mixed"), (4097, 65535, 36, "mixed"), (10000, 70000, 100, "zipf"),
         (9000, 3, 64, "mixed"), (9000, 1, 33, "same"), (5000, 300000, 7, "ascending"),
         (700, 900, 1030, "mixed"), (100, 40, 4096, "zipf"), (20000, 20000000, 1, "distinct"),
         (12345, 65536, 2, "zipf"), (8192, 16384, 5, "distinct"), (8193, 16385, 16, "zipf")]


def run_grad(G, ctx, n, V, d, ids, dY, scale, ldy, ldg, fill=7.0):
    import torch
    ws = torch.empty(G.gist_embed_grad_workspace(n, V, d), dtype=torch.uint8, device="cuda")
    g = torch.full((V, ldg), fill, device="cuda")
    G.gist_embed_grad(ctx, n, V, d, ids, scale, dY, ldy, g, ldg, ws)
    return g


@pytest.mark.parametrize("n,V,d,kind", CASES)
def test_grad(G, ctx, n, V, d, kind):
    import torch
    log(f"embed_grad n={n} V={V} d={d} {kind}")
    rng = np.random.default_rng(n * 7 + V + d)
    ids = make_ids(kind, n, V, rng)
    pad = (n + d) % 3
    dYh = rng.standard_normal((n, d + pad)).astype(np.float32)
    dY, idd, scale = to_dev(dYh), to_dev(ids), -1.7
    g = run_grad(G, ctx, n, V, d, idd, dY, scale, d + pad, d + pad)
    want, bound = R.embed_grad(ids, V, dYh[:, :d], float(np.float32(scale)))
    got = to_host(g)
    err = np.abs(got[:, :d] - want)
    log(f"  worst error over bound {np.max(err / (bound + 1e-45)):.3f}")
    assert (err <= bound).all()
    assert (got[:, d:] == 7).all()
    # again, the same bits
    g2 = run_grad(G, ctx, n, V, d, idd, dY, scale, d + pad, d + pad, fill=-3.0)
    assert np.array_equal(to_host(g2)[:, :d], got[:, :d])
    # fused SGD: bitwise the gradient and then gist_sgd_update, other rows untouched
    T0 = rng.standard_normal((V, d + pad)).astype(np.float32)
    T, lr = to_dev(T0), 0.3
    ws = torch.empty(G.gist_embed_grad_workspace(n, V, d), dtype=torch.uint8, device="cuda")
    G.gist_embed_grad_sgd(ctx, n, V, d, idd, scale, dY, d + pad, lr, T, d + pad, ws)
    ref = to_dev(np.ascontiguousarray(T0[:, :d]))
    gd = to_dev(np.ascontiguousarray(got[:, :d]))
    G.gist_sgd_update(ctx, ref, gd, V * d, lr)
    named = np.zeros(V, bool)
    named[ids[(ids >= 0) & (ids < V)]] = True
    Th, Rh = to_host(T), to_host(ref)
    assert np.array_equal(Th[named][:, :d], Rh[named])
    assert np.array_equal(Th[~named], T0[~named])
    assert np.array_equal(Th[:, d:], T0[:, d:])


@pytest.mark.parametrize("n,V,d,kind", [(262144, 300, 2, "mixed"), (262145, 70000, 3, "zipf"),
                                        (300000, 20000000, 1, "distinct"), (1050001, 65537, 1, "zipf"),
                                        (270000, 1, 5, "same"), (2200000, 100000, 1, "zipf"),
                                        (8400000, 3000, 1, "mixed"), (140000, 9000, 60, "zipf"), (30, 23673, 107, "zipf"), (9, 1063, 563, "mixed"),
                                        (40, 4464, 16, "padding"), (3, 500000, 9, "distinct")])
def test_grad_many_and_few(G, ctx, n, V, d, kind):
    """Ids of more tiles than a workgroup adds up itself; few ids of a long table."""
    test_grad(G, ctx, n, V, d, kind)


def test_grad_of_nothing(G, ctx):
    """No rows: the dense gradient is zero and the fused step leaves the table alone."""
    import torch
    V, d = 300, 20
    g = run_grad(G, ctx, 0, V, d, None, None, 1.0, d, d)
    assert (to_host(g) == 0).all()
    T = torch.full((V, d), 2.5, device="cuda")
    ws = torch.empty(max(1, G.gist_embed_grad_workspace(0, V, d)), dtype=torch.uint8, device="cuda")
    G.gist_embed_grad_sgd(ctx, 0, V, d, None, 1.0, None, d, 0.1, T, d, ws)
    assert (to_host(T) == 2.5).all()
    G.gist_embed_grad(ctx, 4, 0, d, to_dev(np.zeros(4, np.int32)), 1.0, T, d, None, d, ws)


def test_nonfinite_rows_stay_with_their_id(G, ctx):
    """A NaN or Inf in a row of dY reaches its own id's row alone; in a padding row, none."""
    n, V, d = 500, 40, 24
    rng = np.random.default_rng(8)
    ids = make_ids("mixed", n, V, rng)
    dY = rng.standard_normal((n, d)).astype(np.float32)
    ids[10], ids[200], ids[300] = 5, 9, -1
    dY[10, 3], dY[200, 0], dY[300] = np.nan, np.inf, np.nan
    got = to_host(run_grad(G, ctx, n, V, d, to_dev(ids), to_dev(dY), 1.0, d, d))
    bad = ~np.isfinite(got)
    want = np.zeros((V, d), bool)
    want[5, 3] = want[9, 0] = True
    assert np.array_equal(bad, want)


def test_lookup_beyond_32_bit_offsets(G, ctx):
    """A table whose last rows lie past 2^31 (and 2^32 bytes) elements."""
    import torch
    V, d = 300000, 8192            # 2.46e9 elements
    T = torch.zeros(V, d, dtype=torch.bfloat16, device="cuda")
    ids = np.array([0, V - 1, 262143, 262144, V, -1], np.int32)
    for r in (0, V - 1, 262143, 262144):
        T[r] = (r % 97) + 1
    out = torch.full((len(ids), d), 3.0, device="cuda")
    G.gist_embed_lookup(ctx, len(ids), V, d, T, d, G.GIST_STORE_BF16, to_dev(ids), 1.0, out, d)
    got = to_host(out)
    for i, r in enumerate(ids):
        assert (got[i] == ((r % 97) + 1 if 0 <= r < V else 0)).all()


def test_replays(G):
    """Lookup and fused step recorded once: each replay works on the ids its buffer then
    holds, between other work, as the eager calls do."""
    import torch
    n, V, d = 3000, 5000, 36
    st = torch.cuda.Stream()
    cctx, ectx = G.Context(0, stream=st.cuda_stream), G.Context(0)
    rng = np.random.default_rng(4)
    ids = to_dev(np.zeros(n, np.int32))
    T = to_dev(rng.standard_normal((V, d)).astype(np.float32))
    E = T.clone()
    dY = to_dev(rng.standard_normal((n, d)).astype(np.float32))
    X, XE = torch.empty(n, d, device="cuda"), torch.empty(n, d, device="cuda")
    ws = torch.empty(G.gist_embed_grad_workspace(n, V, d), dtype=torch.uint8, device="cuda")
    wse = torch.empty_like(ws)
    torch.cuda.synchronize()
    G.gist_capture_begin(cctx)
    G.gist_embed_lookup(cctx, n, V, d, T, d, 0, ids, 0.5, X, d)
    G.gist_embed_grad_sgd(cctx, n, V, d, ids, 0.5, dY, d, 0.1, T, d, ws)
    r = G.gist_capture_end(cctx)
    for k in range(4):
        ids.copy_(torch.from_numpy(make_ids("mixed" if k % 2 else "ascending", n, V, rng)))
        G.gist_embed_lookup(ectx, n, V, d, E, d, 0, ids, 0.5, XE, d)
        G.gist_embed_grad_sgd(ectx, n, V, d, ids, 0.5, dY, d, 0.1, E, d, wse)
        G.gist_replay_launch(ectx, r)
        torch.cuda.synchronize()
        assert torch.equal(X, XE) and torch.equal(T, E), k


def test_two_streams(G):
    """Two gradients at once on two streams, each with its own workspace."""
    import torch
    rng = np.random.default_rng(6)
    jobs = []
    for k, (n, V, d) in enumerate([(60000, 30000, 128), (50000, 200, 128)]):
        st = torch.cuda.Stream()
        jobs.append((n, V, d, make_ids("zipf", n, V, rng), rng.standard_normal((n, d)).astype(np.float32), st))
    dev = [(to_dev(j[3]), to_dev(j[4]), torch.empty(j[1], j[2], device="cuda"),
            torch.empty(G.gist_embed_grad_workspace(*j[:3]), dtype=torch.uint8, device="cuda")) for j in jobs]
    torch.cuda.synchronize()
    for _ in range(3):
        for j, (i, y, g, w) in zip(jobs, dev):
            c = G.Context(0, stream=j[5].cuda_stream)
            G.gist_embed_grad(c, *j[:3], i, 1.0, y, j[2], g, j[2], w)
    torch.cuda.synchronize()
    for j, (i, y, g, w) in zip(jobs, dev):
        want, bound = R.embed_grad(j[3], j[1], j[4], 1.0)
        assert (np.abs(to_host(g) - want) <= bound).all()
