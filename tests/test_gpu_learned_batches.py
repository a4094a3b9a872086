"""Learned rows, log probabilities and Muon on the batches that the runners take: layer-sampled
ones (rectangular layers), batches padded to a fixed layout, recorded steps over batches of
different sizes; the input gradient beside the fused SGD step; two of the calls at once on two
streams."""

import numpy as np
import pytest

import ops_ref as R
from gist_synth.graphs import sbm
from gpu_util import FP32_TOL, log, relerr, to_dev, to_host
from test_gpu_ladies import _Workload
from test_gpu_learned_step import LR, LR_TABLE, MU, SCALE, device_state, setup

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    from paper_2102_10424_amd import gist
    return gist


def weights(n, pad, rng):
    """Weights of the log probabilities and the entropies: 0 for padding rows."""
    gl, gh = np.zeros(n + pad, np.float32), np.zeros(n + pad, np.float32)
    gl[:n], gh[:n] = -rng.random(n) / n, -0.05 / n
    return gl, gh


def learned_step(run, rows, view, ids, n_ids, params, M, gl, gh):
    rows.lookup(ids, n_ids, view.X)
    run.forward(view, params)
    run.log_probs(view, 2)
    run.log_probs_grad(view, gl, gh)
    run.backward(view, params)
    run.muon(params, M, LR, momentum=MU)
    rows.sgd(ids, n_ids, run.dH[0], LR_TABLE)


def test_ladies_batch(G):
    """A layer-sampled batch (each layer its own rows) against the step in 64 bits: dense
    rectangular matrices, automatic differentiation through the device's ReLU decisions."""
    import torch
    from paper_2102_10424_amd import step as S
    ctx = G.Context(0)
    w = _Workload(2000, 20, (24, 40, 9), 50, 200)
    key = 11
    slot = S.LadiesSlot(ctx, w.L, w.b, w.s, w.max_degree, 24)
    batch = slot.load(G.CsrHandle(w.A), w.batch_nodes(key), key, to_dev(w.X), w.y)
    from oracle import ladies as LD
    sampled = LD.sample(w.A, w.batch_nodes(key), w.L, w.s, seed=key)
    ids = np.asarray(sampled["nodes"][0], dtype=np.int32)
    y = w.y[sampled["nodes"][w.L]]
    n0, n = batch.rows(0), batch.rows(w.L)
    assert n0 == len(ids) and n == len(y) and n0 > n
    rng = np.random.default_rng(5)
    T = rng.standard_normal((2000, 24)).astype(np.float32)
    M = [(rng.standard_normal(t.shape) * 1e-3).astype(np.float32) for t in w.theta]
    gl, gh = weights(n, 0, rng)
    run = S.SubGCN(ctx, "gcn", w.widths, 1, input_grad=True)
    rows = S.LearnedRows(ctx, to_dev(T), SCALE)
    params, Md = [to_dev(t) for t in w.theta], [to_dev(m) for m in M]
    learned_step(run, rows, batch, to_dev(ids), n0, params, Md, to_dev(gl), to_dev(gh))
    f = lambda a: torch.from_numpy(np.asarray(a, dtype=np.float64))
    Tt, Wt = f(T).requires_grad_(), [f(t).requires_grad_() for t in w.theta]
    H = SCALE * Tt[torch.from_numpy(ids.astype(np.int64))]
    for l, lay in enumerate(sampled["layers"]):
        A = np.zeros((lay["n"], lay["n_in"]))
        for i in range(lay["n"]):
            s = slice(lay["rowptr"][i], lay["rowptr"][i + 1])
            A[i, lay["col"][s]] = lay["val"][s]
        H = f(A) @ H @ Wt[l]
        if l + 1 < w.L:
            H = H * f(to_host(run.H[l + 1])[:lay["n"]] > 0)
    lp = torch.log_softmax(H, 1)
    logp, ent = lp[torch.arange(n), torch.from_numpy(y.astype(np.int64))], -(lp.exp() * lp).sum(1)
    (f(gl) * logp + f(gh) * ent).sum().backward()
    assert relerr(to_host(run.H[w.L])[:n], H.detach().numpy()) <= FP32_TOL
    assert relerr(to_host(run.lp["logp"])[:n], logp.detach().numpy()) <= FP32_TOL
    assert relerr(to_host(run.lp["entropy"])[:n], ent.detach().numpy()) <= FP32_TOL
    mu, lr = float(np.float32(MU)), float(np.float32(LR))
    for l in range(w.L):
        g = Wt[l].grad.numpy()
        assert relerr(to_host(run.dW[l]), g) <= FP32_TOL
        m = mu * M[l].astype(np.float64) + (1 - mu) * g
        want = w.theta[l] - lr * 0.2 * max(g.shape) ** 0.5 * R.orthogonal((1 - mu) * g + mu * m)
        assert relerr(to_host(Md[l]), m) <= FP32_TOL and relerr(to_host(params[l]), want) <= FP32_TOL
    assert relerr(to_host(rows.table), T - LR_TABLE * Tt.grad.numpy()) <= FP32_TOL
    other = np.ones(2000, bool)
    other[ids] = False
    assert np.array_equal(to_host(rows.table)[other], T[other])


@pytest.mark.parametrize("kind", ["gcn", "sage", "gat", "ladies"])
def test_padded_batches_replayed(G, kind):
    """A whole step on a batch padded to a fixed layout (padding rows: node 0, no edges,
    weight 0), recorded once and replayed on batches of different sizes: the unpadded batches'
    results, up to the order of sums, and a table whose other rows, node 0's among them, stay
    as they were."""
    import torch
    from paper_2102_10424_amd import step as S
    st = torch.cuda.Stream()
    cctx, ctx = G.Context(0, stream=st.cuda_stream), G.Context(0)
    rng = np.random.default_rng(17)
    ladies = kind == "ladies"
    widths = [24, 40, 9]
    if ladies:
        w = _Workload(2000, 20, widths, 50, 200)
        g, y, A = w.g, w.y, G.CsrHandle(w.A)
        fixed = S.LadiesSlot(ctx, 2, 50, 200, w.max_degree, 24, fixed=True, fixed_nnz_per_row=40)
        plain = S.LadiesSlot(ctx, 2, 50, 200, w.max_degree, 24)
    else:
        g = sbm(2000, 40, 15.0, 0.9, seed=31)
        y = rng.integers(0, 9, g.n).astype(np.int32)
        norm = "sage" if kind == "sage" else "gcn"
        cap_n = int(np.sort(np.diff(g.cluster_ptr))[-4:].sum())
        cap_nnz = int(np.sort(np.diff(g.rowptr))[-cap_n:].sum()) + cap_n
        gh_ = G.GraphHandle(g)
        fixed = S.FixedBatchSlot(ctx, norm, cap_n, cap_nnz, 24)
        plain = S.BatchSlot(ctx, norm, cap_n, cap_nnz, 24)
    X = to_dev(np.zeros((g.n, 24), np.float32))
    T = rng.standard_normal((g.n, 24)).astype(np.float32)
    wr = lambda l: widths[l] + 2 if kind == "gat" else (2 if kind == "sage" else 1) * widths[l]
    theta = [(rng.standard_normal((wr(l), widths[l + 1])) * 0.3).astype(np.float32) for l in range(2)]
    if ladies:
        runner = S.LadiesGraphRunner(cctx, widths, 2, 50, 200, 24, X, fixed_nnz_per_row=40)
        ids, cap = runner.nodes0, runner.n0
    else:
        runner = S.ClusterGraphRunner(cctx, kind, widths, cap_n, cap_nnz, 24, X)
        ids, cap = runner.node_map, cap_n
    view, cap_out = runner.view, runner.view.rows(2)
    k = "gcn" if ladies else kind
    run, eager = S.SubGCN(cctx, k, widths, cap, input_grad=True), S.SubGCN(ctx, k, widths, 1, input_grad=True)
    rows, erows = S.LearnedRows(cctx, to_dev(T), SCALE), S.LearnedRows(ctx, to_dev(T), SCALE)
    p, pe = ([to_dev(t) for t in theta] for _ in range(2))
    M, Me = ([to_dev(np.zeros_like(t)) for t in theta] for _ in range(2))
    gl, gh = (torch.zeros(cap_out, device="cuda") for _ in range(2))
    run.prepare(view)
    run.prepare_muon()
    rows._reserve(cap)
    run._log_probs_buffers(cap_out, 2)
    torch.cuda.synchronize()
    G.gist_capture_begin(cctx)
    learned_step(run, rows, view, ids, cap, p, M, gl, gh)
    r = G.gist_capture_end(cctx)
    touched, ns = np.zeros(g.n, bool), set()
    cluster0 = 0 if ladies else int(np.searchsorted(g.cluster_ptr, np.flatnonzero(g.cluster_nodes == 0)[0], "right") - 1)
    for step in range(4):
        if ladies:
            out = np.sort(rng.choice(np.arange(1, g.n), 50, replace=False)).astype(np.int32)
            fixed.build(A, out, 90 + step, y)
            assert fixed.fits_fixed()
            b = plain.load(A, out, 90 + step, X, y)
            lay = plain.built[2][0]["nodes"]
            eids = plain.packed_d[lay:lay + b.rows(0)]
        else:
            clusters = np.sort(rng.choice(np.setdiff1d(np.arange(g.n_clusters), [cluster0]), 1 + step % 3,
                                          replace=False)).astype(np.int32)
            fixed.build(gh_, clusters, y)
            b = plain.load(gh_, clusters, X, y)
            eids = plain.d["node_map"][:b.rows(0)]
        n = b.rows(2)
        glh, ghh = weights(n, cap_out - n, rng)
        gl.copy_(torch.from_numpy(glh))
        gh.copy_(torch.from_numpy(ghh))
        runner.dev.copy_(fixed.packed_h[:runner.dev.numel()])
        G.gist_replay_launch(ctx, r)
        learned_step(eager, erows, b, eids, b.rows(0), pe, Me, to_dev(glh[:n]), to_dev(ghh[:n]))
        torch.cuda.synchronize()
        touched[to_host(eids)] = True
        ns.add(b.rows(0))
        log(f"padded {kind} step {step}: {b.rows(0)} of {cap} rows")
        assert relerr(to_host(run.lp["logp"])[:n], to_host(eager.lp["logp"])[:n]) <= 1e-5
        assert relerr(to_host(run.lp["entropy"])[:n], to_host(eager.lp["entropy"])[:n]) <= 1e-5
        for a, c in zip(run.dW + p + M + [rows.table], eager.dW + pe + Me + [erows.table]):
            assert relerr(to_host(a), to_host(c)) <= FP32_TOL
        for t in (rows.table, erows.table):
            assert np.array_equal(to_host(t)[~touched], T[~touched])
    assert len(ns) > 1 and max(ns) < cap and (ladies or not touched[0])


@pytest.mark.parametrize("kind", ["gcn", "sage", "gat"])
def test_input_gradient_beside_the_fused_step(G, kind):
    """With the SGD step inside the backward pass the input gradient is still that of the
    weights before it: the bits of a backward pass followed by the step."""
    import torch
    from paper_2102_10424_amd import step as S
    ctx = G.Context(0)
    inp = setup(kind, 36)
    a, b = device_state(S, ctx, kind, *inp), device_state(S, ctx, kind, *inp)
    for s in (a, b):
        s[1].lookup(s[3], s[2].n, s[2].X)
        s[0].forward(s[2], s[4])
        s[0].log_probs(s[2])
        s[0].log_probs_grad(s[2], s[6], s[7])
    a[0].backward(a[2], a[4], sgd_lr=LR)
    b[0].backward(b[2], b[4])
    b[0].sgd(b[4], LR)
    torch.cuda.synchronize()
    n = inp[1]
    assert torch.equal(a[0].dH[0][:n], b[0].dH[0][:n]) and bool((a[0].dH[0][:n] != 0).any())
    for x, y in zip(a[4], b[4]):
        assert torch.equal(x, y)


def test_updates_on_two_streams(G):
    """Two Muon updates at once, each with its own workspace: the bits of one after the other."""
    import torch
    rng = np.random.default_rng(8)
    cases = [(1, 700, 900, "f32"), (3, 64, 1000, "f32"), (2, 520, 260, "f16"), (4, 128, 100, "f32")]
    for first, second in ((cases[0], cases[1]), (cases[2], cases[0]), (cases[1], cases[3])):
        results = []
        for streams in (1, 2):
            rng = np.random.default_rng(8)
            st = [torch.cuda.Stream() for _ in range(streams)]
            jobs = []
            for k, (g, r, c, dt) in enumerate((first, second)):
                d = G.muon_desc(r, c, groups=g, flags=G.GIST_MUON_NESTEROV,
                                dtype=G.GIST_DTYPE_F32 if dt == "f32" else G.GIST_DTYPE_F16_IN)
                t = [to_dev(rng.standard_normal((g, r, c)).astype(np.float32)) for _ in range(3)]
                ws = torch.empty(G.gist_muon_workspace_size(d), dtype=torch.uint8, device="cuda")
                jobs.append((G.Context(0, stream=st[k % streams].cuda_stream), d, t, ws))
            torch.cuda.synchronize()
            for _ in range(4):
                for c, d, t, ws in jobs:
                    G.gist_muon_update(c, d, t[0], t[1], t[2], 0.02, 0.9, 0.01, 1.0, ws)
            torch.cuda.synchronize()
            results.append([x.clone() for j in jobs for x in j[2]])
        for x, y in zip(*results):
            assert torch.equal(x, y) and bool(torch.isfinite(x).all())


def test_log_probs_on_two_streams(G):
    """Forward and gradient of two sets of rows at once: the bits of one after the other."""
    import torch
    results = []
    for streams in (1, 2):
        gen = torch.Generator(device="cuda").manual_seed(3)
        st = [torch.cuda.Stream() for _ in range(streams)]
        jobs = []
        for k, (n, C, K) in enumerate([(2, 131072, 20), (3000, 2000, 5), (100000, 41, 5), (70, 33000, 0)]):
            z = torch.randn(n, C, generator=gen, device="cuda") + (500.0 if k == 3 else 0.0)
            y = torch.randint(0, C, (n,), generator=gen, device="cuda", dtype=torch.int32)
            o = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t, device="cuda")
            ws = torch.empty(max(16, G.gist_log_probs_workspace(n, C, K)), dtype=torch.uint8, device="cuda")
            jobs.append((G.Context(0, stream=st[k % streams].cuda_stream), n, C, K, z, y, o(n), o(n), o(n),
                         o(n, K) if K else None, o(n, K, t=torch.int32) if K else None, ws, torch.zeros_like(z),
                         torch.ones(n, device="cuda")))
        torch.cuda.synchronize()
        for _ in range(3):
            for c, n, C, K, z, y, lp, H, l, top, idx, ws, dz, one in jobs:
                G.gist_log_probs(c, n, C, z, C, 0, y, lp, H, l, K, top, idx, ws)
                G.gist_log_probs_bwd(c, n, C, z, C, 0, y, l, H, one, one, dz, C)
        torch.cuda.synchronize()
        results.append([t for j in jobs for t in j[6:11] + j[12:13] if t is not None])
    for x, y in zip(*results):
        assert torch.equal(x, y) and bool((x != 0).any())
