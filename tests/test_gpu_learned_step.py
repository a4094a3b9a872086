"""Learned rows, log probabilities and Muon in one training step, as they are used
together: rows of a learned table through GCN, GraphSAGE and GAT sub-GCNs, a weighted
log-likelihood with an entropy bonus, the layers' backward pass down to the rows, Muon on
the weights and SGD on the table, against the same step in 64 bits (dense matrices,
automatic differentiation on the CPU, the orthogonal factor by singular values); the step
recorded and replayed."""

import numpy as np
import pytest

import ops_ref as R
from gist_synth.graphs import erdos_renyi
from gpu_util import FP32_TOL, csr_to_dev, log, relerr, to_dev, to_host
from oracle import minibatch as OM

pytestmark = pytest.mark.gpu

SCALE, LR, LR_TABLE, MU = 0.5, 0.02, 0.3, 0.95


@pytest.fixture(scope="module")
def G():
    from paper_2102_10424_amd import gist
    return gist


def setup(kind, seed):
    g = erdos_renyi(300, 1500, seed=seed, clusters=5)
    csr = OM.build(g, [0, 2, 3], "sage" if kind == "sage" else "gcn")
    for k in csr:      # as the library's own builder returns them
        if k.endswith(("rowptr", "col", "map")):
            csr[k] = np.asarray(csr[k], dtype=np.int32)
        elif k.endswith("val"):
            csr[k] = np.asarray(csr[k], dtype=np.float32)
    rng = np.random.default_rng(seed)
    n, widths = int(csr["n"]), [24, 40, 7]
    T = (rng.standard_normal((300, 24)) * 2).astype(np.float32)
    rows = lambda l: (2 * widths[l] if kind == "sage" else widths[l] + 2 if kind == "gat" else widths[l])
    W = [(rng.standard_normal((rows(l), widths[l + 1])) / np.sqrt(widths[l])).astype(np.float32) for l in range(2)]
    M = [(rng.standard_normal(w.shape) * 1e-3).astype(np.float32) for w in W]
    y = rng.integers(0, 7, n).astype(np.int32)
    gl = (-rng.random(n) / n).astype(np.float32)
    gh = np.full(n, -0.05 / n, np.float32)
    return csr, n, widths, T, W, M, y, gl, gh


def dense(csr):
    n = int(csr["n"])
    A = np.zeros((n, n))
    for i in range(n):
        s = slice(csr["rowptr"][i], csr["rowptr"][i + 1])
        A[i, csr["col"][s]] = csr["val"][s]
    return A


def reference(kind, csr, n, widths, T, W, M, y, gl, gh):
    """The step in 64 bits: logits, log probabilities, gradients, updated state."""
    import torch
    f = lambda a: torch.from_numpy(np.asarray(a, dtype=np.float64))
    A = f(dense(csr))
    ids = np.asarray(csr["node_map"])[:n]
    Tt = f(T).requires_grad_()
    Wt = [f(w).requires_grad_() for w in W]
    H = SCALE * Tt[torch.from_numpy(ids.astype(np.int64))]
    for l in range(2):
        s = widths[l]
        if kind == "sage":
            Z = H @ Wt[l][:s] + (A @ H) @ Wt[l][s:]
        elif kind == "gcn":
            Z = A @ H @ Wt[l]
        else:
            P = H @ Wt[l][:s]
            e = torch.nn.functional.leaky_relu((P @ Wt[l][s])[:, None] + (P @ Wt[l][s + 1])[None, :], 0.2)
            e = e.masked_fill(A == 0, -np.inf)
            Z = torch.softmax(e, 1) @ P
        H = torch.relu(Z) if l == 0 else Z
    lp = torch.log_softmax(H, 1)
    logp = lp[torch.arange(n), torch.from_numpy(y.astype(np.int64))]
    ent = -(lp.exp() * lp).sum(1)
    (f(gl) * logp + f(gh) * ent).sum().backward()
    out = dict(logits=H, logp=logp, entropy=ent, dT=Tt.grad, dW=[w.grad for w in Wt])
    out = {k: ([x.detach().numpy() for x in v] if isinstance(v, list) else v.detach().numpy()) for k, v in out.items()}
    mu, lr = float(np.float32(MU)), float(np.float32(LR))
    newW, newM = [], []
    for l in range(2):
        s, c = widths[l], widths[l + 1]
        g = out["dW"][l]
        m = mu * M[l].astype(np.float64) + (1 - mu) * g
        u = (1 - mu) * g + mu * m
        w = W[l].astype(np.float64).copy()
        for k in range(2 if kind == "sage" else 1):
            w[k * s:(k + 1) * s] -= lr * 0.2 * max(s, c) ** 0.5 * R.orthogonal(u[k * s:(k + 1) * s])
        if kind == "gat":
            w[s:] -= lr * g[s:]
            m[s:] = M[l][s:]            # the attention vectors have no momentum
        newW.append(w)
        newM.append(m)
    out.update(W=newW, M=newM, T=T - LR_TABLE * out["dT"])
    return out


def run_step(G, S, ctx, run, rows, batch, ids, params, M, gl, gh):
    rows.lookup(ids, batch.n, batch.X)
    run.forward(batch, params)
    run.log_probs(batch, 3)
    run.log_probs_grad(batch, gl, gh)
    run.backward(batch, params)
    run.muon(params, M, LR, momentum=MU)
    rows.sgd(ids, batch.n, run.dH[0], LR_TABLE)


def device_state(S, ctx, kind, csr, n, widths, T, W, M, y, gl, gh):
    import torch
    batch = S.DeviceBatch(csr, torch.zeros(n, widths[0], device="cuda"), to_dev(y), "cuda")
    rows = S.LearnedRows(ctx, to_dev(T), SCALE, n)
    run = S.SubGCN(ctx, kind, widths, n, input_grad=True)
    run.prepare(batch)
    run.prepare_muon()
    ids = to_dev(np.asarray(csr["node_map"])[:n].astype(np.int32))
    return run, rows, batch, ids, [to_dev(w) for w in W], [to_dev(m) for m in M], to_dev(gl), to_dev(gh)


@pytest.mark.parametrize("kind", ["gcn", "sage", "gat"])
def test_step(G, kind):
    from paper_2102_10424_amd import step as S
    ctx = G.Context(0)
    inp = setup(kind, 31)
    csr, n, widths, T, W, M = inp[:6]
    want = reference(kind, *inp)
    run, rows, batch, ids, Wd, Md, gl, gh = device_state(S, ctx, kind, *inp)
    run_step(G, S, ctx, run, rows, batch, ids, Wd, Md, gl, gh)
    p = run.lp
    log(f"{kind}: logits {relerr(to_host(run.H[2])[:n], want['logits']):.1e}")
    assert relerr(to_host(run.H[2])[:n], want["logits"]) <= FP32_TOL
    assert relerr(to_host(p["logp"]), want["logp"]) <= FP32_TOL
    assert relerr(to_host(p["entropy"]), want["entropy"]) <= FP32_TOL
    assert np.array_equal(to_host(p["top_idx"]), R.top_classes(to_host(run.H[2])[:n], 3))
    for l in range(2):
        assert relerr(to_host(run.dW[l]), want["dW"][l]) <= FP32_TOL
        assert relerr(to_host(Wd[l]), want["W"][l]) <= FP32_TOL
        assert relerr(to_host(Md[l]), want["M"][l]) <= FP32_TOL
    nm = np.asarray(csr["node_map"])[:n]
    assert relerr(to_host(run.dH[0])[:n], want["dT"][nm] / SCALE) <= FP32_TOL
    assert relerr(to_host(rows.table), want["T"]) <= FP32_TOL
    other = np.ones(300, bool)
    other[nm] = False
    assert other.any() and np.array_equal(to_host(rows.table)[other], T[other])


@pytest.mark.parametrize("kind", ["gcn", "sage"])
def test_step_replayed(G, kind):
    """The whole step recorded; replays, between eager steps on other buffers, give the
    eager steps' bits."""
    import torch
    from paper_2102_10424_amd import step as S
    inp = setup(kind, 32)
    st = torch.cuda.Stream()
    cctx, ectx = G.Context(0, stream=st.cuda_stream), G.Context(0)
    a, b = device_state(S, cctx, kind, *inp), device_state(S, ectx, kind, *inp)
    a[0].forward(a[2], a[4])
    a[0].log_probs(a[2], 3)        # allocates
    torch.cuda.synchronize()
    G.gist_capture_begin(cctx)
    run_step(G, S, cctx, *a)
    r = G.gist_capture_end(cctx)
    for k in range(4):
        run_step(G, S, ectx, *b)
        G.gist_replay_launch(ectx, r)
        torch.cuda.synchronize()
        for x, y in zip(a[4] + a[5] + [a[1].table, a[0].lp["logp"], a[0].lp["top_idx"]],
                        b[4] + b[5] + [b[1].table, b[0].lp["logp"], b[0].lp["top_idx"]]):
            assert torch.equal(x, y), k


def test_muon_step_trains(G):
    """``SubGCN.step`` with Muon: three steps equal its parts called one by one, the first
    with fresh momentum over garbage."""
    import torch
    from paper_2102_10424_amd import step as S
    ctx = G.Context(0)
    inp = setup("gcn", 33)
    a, b = device_state(S, ctx, "gcn", *inp), device_state(S, ctx, "gcn", *inp)
    for s in (a, b):
        s[1].lookup(s[3], s[2].n, s[2].X)
        for m in s[5]:
            m.fill_(float("nan"))
    for k in range(3):
        a[0].step(a[2], a[4], LR, muon=(a[5], k == 0))
        b[0].forward(b[2], b[4])
        b[0].loss_and_grad(b[2])
        b[0].backward(b[2], b[4])
        b[0].muon(b[4], b[5], LR, fresh=k == 0)
    torch.cuda.synchronize()
    for x, y in zip(a[4] + a[5], b[4] + b[5]):
        assert torch.equal(x, y) and bool(torch.isfinite(x).all())


@pytest.mark.parametrize("kind", ["gcn", "sage", "gat"])
def test_replay_after_a_larger_batch(G, kind):
    """A recorded step works on the buffers it was recorded with after its runner has seen a
    larger batch, whatever is allocated since: the bits of a runner that saw none."""
    import torch
    from paper_2102_10424_amd import step as S
    inp = setup(kind, 34)
    st = torch.cuda.Stream()
    cctx, ectx = G.Context(0, stream=st.cuda_stream), G.Context(0)
    a, b = device_state(S, cctx, kind, *inp), device_state(S, ectx, kind, *inp)
    a[0].log_probs(a[2], 3)        # allocates
    torch.cuda.synchronize()
    G.gist_capture_begin(cctx)
    run_step(G, S, cctx, *a)
    r = G.gist_capture_end(cctx)
    g = erdos_renyi(900, 6000, seed=35, clusters=3)
    csr = OM.build(g, [0, 1, 2], "sage" if kind == "sage" else "gcn")
    csr = {k: np.asarray(v, dtype=np.float32 if k.endswith("val") else np.int32) if np.ndim(v) else v
           for k, v in csr.items()}
    n, w = int(csr["n"]), inp[2]
    big = S.DeviceBatch(csr, torch.ones(n, w[0], device="cuda"), to_dev(np.zeros(n, np.int32)), "cuda")
    params, ones = [p.clone() for p in a[4]], torch.ones(n, device="cuda")
    torch.cuda.synchronize()
    a[0].forward(big, params)
    lp = a[0].log_probs(big, 3)
    a[0].log_probs_grad(big, ones)
    a[0].backward(big, params)
    torch.cuda.synchronize()
    assert n > inp[1] and bool(torch.isfinite(lp["logp"]).all())
    junk = [torch.full((k, inp[1]), float("nan"), device="cuda") for k in (w + [1]) * 4]
    for k in range(3):
        run_step(G, S, ectx, *b)
        G.gist_replay_launch(ectx, r)
        torch.cuda.synchronize()
        for x, y in zip(a[4] + a[5] + [a[1].table], b[4] + b[5] + [b[1].table]):
            assert torch.equal(x, y), k
    assert all(bool(torch.isnan(j).all()) for j in junk)
