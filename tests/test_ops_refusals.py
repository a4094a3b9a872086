"""Arguments that the learned-row, log-probability and orthogonalised-update
calls refuse, and their workspace sizes.  No GPU needed: every check runs on
the host before anything touches the device."""

import ctypes

import numpy as np
import pytest

import ops_ref as R

G = pytest.importorskip("paper_2102_10424_amd.gist",
                        reason="libgist.so not built (python -m paper_2102_10424_amd.build)")


class NoDevice:
    """A context handle over zeroed memory: device 0, the default stream.  A refused call
    reads no more of it."""

    def __init__(self):
        self.mem = ctypes.create_string_buffer(256)
        self.handle = ctypes.cast(self.mem, ctypes.c_void_p)


ctx = NoDevice()
A = np.zeros(64, dtype=np.float32)     # stands for device memory; never read
I = np.zeros(64, dtype=np.int32)
INVAL, NOMEM, UNSUP = G.GIST_E_INVAL, G.GIST_E_NOMEM, G.GIST_E_UNSUPPORTED


class Ws:
    def __init__(self, nbytes, addr=None):
        self.n, self.a = nbytes, addr if addr is not None else 4096

    def numel(self):
        return self.n

    def element_size(self):
        return 1

    def data_ptr(self):
        return self.a


def refused(status, fn, *args, **kw):
    with pytest.raises(G.GistError) as e:
        fn(*args, **kw)
    assert e.value.status == status, e.value


def test_null_context():
    class Null:
        handle = None
    refused(INVAL, G.gist_embed_lookup, Null, 1, 1, 1, A, 1, 0, I, 1.0, A, 1)
    refused(INVAL, G.gist_embed_grad, Null, 1, 1, 1, I, 1.0, A, 1, A, 1, Ws(1 << 20))
    refused(INVAL, G.gist_embed_grad_sgd, Null, 1, 1, 1, I, 1.0, A, 1, 0.1, A, 1, Ws(1 << 20))
    refused(INVAL, G.gist_log_probs, Null, 1, 1, A, 1, 0, I, A, A, A, 0, None, None, None)
    refused(INVAL, G.gist_log_probs_bwd, Null, 1, 1, A, 1, 0, I, A, A, A, A, A, 1)
    d = G.muon_desc(4, 4)
    refused(INVAL, G.gist_orthogonalize, Null, d, A, A, Ws(1 << 20))
    refused(INVAL, G.gist_muon_update, Null, d, A, A, A, 0.1, 0.9, 0.0, 1.0, Ws(1 << 20))


@pytest.mark.parametrize("change,status", [
    (dict(n=-1), INVAL), (dict(V=-1), INVAL), (dict(d=0), INVAL), (dict(d=(1 << 22) + 1, ldt=1 << 23, ldo=1 << 23), UNSUP),
    (dict(n=2**31 - 1), UNSUP), (dict(V=2**31 - 1), UNSUP), (dict(ldt=3), INVAL),
    (dict(ldo=3), INVAL), (dict(store=3), INVAL), (dict(store=-1), INVAL),
    (dict(scale=float("nan")), INVAL), (dict(scale=float("inf")), INVAL),
    (dict(table=None), INVAL), (dict(ids=None), INVAL), (dict(out=None), INVAL)])
def test_embed_lookup(change, status):
    a = dict(n=2, V=5, d=4, table=A, ldt=4, store=0, ids=I, scale=1.0, out=A, ldo=4)
    refused(status, G.gist_embed_lookup, ctx, **{**a, **change})


@pytest.mark.parametrize("sgd", [False, True])
@pytest.mark.parametrize("change,status", [
    (dict(n=-1), INVAL), (dict(V=-1), INVAL), (dict(d=0), INVAL),
    (dict(n=2**31 - 1), UNSUP), (dict(V=2**31 - 1), UNSUP),
    (dict(ldy=3), INVAL), (dict(ldt=3), INVAL), (dict(scale=float("nan")), INVAL),
    (dict(ids=None), INVAL), (dict(dY=None), INVAL), (dict(out=None), INVAL),
    (dict(ws=None), NOMEM), (dict(ws="small"), NOMEM), (dict(ws="odd"), INVAL),
    (dict(lr=float("inf")), INVAL)])
def test_embed_grad(sgd, change, status):
    a = dict(n=2, V=5, d=4, ids=I, scale=1.0, dY=A, ldy=4, out=A, ldt=4, lr=0.1,
             ws=Ws(G.gist_embed_grad_workspace(2, 5, 4)))
    a.update(change)
    if a["ws"] == "small":
        a["ws"] = Ws(G.gist_embed_grad_workspace(2, 5, 4) - 1)
    if a["ws"] == "odd":
        a["ws"] = Ws(1 << 20, 4100)
    if sgd:
        refused(status, G.gist_embed_grad_sgd, ctx, a["n"], a["V"], a["d"], a["ids"], a["scale"],
                a["dY"], a["ldy"], a["lr"], a["out"], a["ldt"], a["ws"])
    elif "lr" not in change:
        refused(status, G.gist_embed_grad, ctx, a["n"], a["V"], a["d"], a["ids"], a["scale"],
                a["dY"], a["ldy"], a["out"], a["ldt"], a["ws"])


@pytest.mark.parametrize("change,status", [
    (dict(n=-1), INVAL), (dict(C_=0), INVAL), (dict(ldz=6), INVAL), (dict(store=7), INVAL),
    (dict(n=2**31 - 1), UNSUP), (dict(C_=2**31 - 1, ldz=2**31), UNSUP),
    (dict(logits=None), INVAL), (dict(K=-1), INVAL), (dict(K=8), INVAL),
    (dict(C_=100, ldz=100, K=65), INVAL), (dict(K=2, top_logp=None), INVAL),
    (dict(K=2, top_idx=None), INVAL), (dict(tokens=None), INVAL)])
def test_log_probs(change, status):
    a = dict(n=2, C_=7, logits=A, ldz=7, store=0, tokens=I, logp=A, entropy=A, lse=A, K=0,
             top_logp=A, top_idx=I, ws=Ws(1 << 20))
    refused(status, G.gist_log_probs, ctx, **{**a, **change})


def test_log_probs_workspace():
    assert G.gist_log_probs_workspace(0, 5, 0) >= 0
    need = G.gist_log_probs_workspace(1, 1 << 20, 8)     # one long row is split
    assert need > 0
    a = dict(n=1, C_=1 << 20, logits=A, ldz=1 << 20, store=0, tokens=I, logp=A, entropy=A, lse=A,
             K=8, top_logp=A, top_idx=I)
    refused(NOMEM, G.gist_log_probs, ctx, **a, ws=Ws(need - 1))
    refused(NOMEM, G.gist_log_probs, ctx, **a, ws=None)
    refused(INVAL, G.gist_log_probs, ctx, **a, ws=Ws(need, 4104))
    for bad in ((-1, 5, 0), (2, 0, 0), (2, 5, 6), (2, 100, 65), (2, 5, -1), (2**31, 5, 0)):
        assert G.gist_log_probs_workspace(*bad) == 0


@pytest.mark.parametrize("change,status", [
    (dict(n=-1), INVAL), (dict(C_=0), INVAL), (dict(ldz=6), INVAL), (dict(ldd=6), INVAL),
    (dict(store=3), INVAL), (dict(logits=None), INVAL), (dict(lse=None), INVAL),
    (dict(dlogits=None), INVAL), (dict(tokens=None), INVAL), (dict(entropy=None), INVAL),
    (dict(dlogits=A, ldd=8), INVAL)])
def test_log_probs_bwd(change, status):
    a = dict(n=2, C_=7, logits=A, ldz=7, store=0, tokens=I, lse=A, entropy=A, g_logp=A,
             g_entropy=A, dlogits=A.copy(), ldd=7)
    refused(status, G.gist_log_probs_bwd, ctx, **{**a, **change})


DESC = [(dict(rows=-1), INVAL), (dict(cols=-1), INVAL), (dict(groups=-1), INVAL),
        (dict(rows=65537), UNSUP), (dict(cols=65537), UNSUP), (dict(groups=65536), UNSUP),
        (dict(dtype=G.GIST_DTYPE_BF16_IN), INVAL), (dict(dtype=9), INVAL), (dict(flags=4), INVAL),
        (dict(steps=0), INVAL), (dict(steps=33), INVAL), (dict(eps=0.0), INVAL),
        (dict(eps=float("nan")), INVAL), (dict(eps=-1.0), INVAL),
        (dict(coef=(float("nan"), 0, 0)), INVAL), (dict(coef=(9.0, 0, 0)), INVAL),
        (dict(coef=(3.0, 1.0, 1.0)), INVAL), (dict(coef=(1.5, 10.0, -10.0)), INVAL),
        (dict(coef=(2.0, 0.0, 0.0), steps=4), INVAL)]


@pytest.mark.parametrize("change,status", DESC)
def test_muon_desc(change, status):
    d = G.muon_desc(**{**dict(rows=8, cols=6), **change})
    refused(status, G.gist_muon_workspace_size, d)
    refused(status, G.gist_orthogonalize, ctx, d, A, A, Ws(1 << 30))
    refused(status, G.gist_muon_update, ctx, d, A, A, A, 0.1, 0.9, 0.0, 1.0, Ws(1 << 30))


@pytest.mark.parametrize("coef", [R.COEF, (1.5, -0.5, 0.0), (15 / 8, -10 / 8, 3 / 8), (1.0, 0, 0)])
def test_muon_coefficients_in_use_are_accepted(coef):
    for steps in (1, 5, 32):
        assert G.gist_muon_workspace_size(G.muon_desc(8, 6, coef=coef, steps=steps)) > 0


def test_muon_calls():
    d = G.muon_desc(8, 6)
    need = G.gist_muon_workspace_size(d)
    w = Ws(need)
    refused(INVAL, G.gist_orthogonalize, ctx, d, None, A, w)
    refused(INVAL, G.gist_orthogonalize, ctx, d, A, None, w)
    refused(NOMEM, G.gist_orthogonalize, ctx, d, A, A, Ws(need - 1))
    refused(NOMEM, G.gist_orthogonalize, ctx, d, A, A, None)
    refused(INVAL, G.gist_orthogonalize, ctx, d, A, A, Ws(need, 4097))
    ok = dict(W=A, dW=A, M=A, lr=0.1, momentum=0.9, weight_decay=0.0, scale=1.0, ws=w)
    for change in (dict(W=None), dict(dW=None), dict(M=None), dict(lr=float("nan")),
                   dict(momentum=1.0), dict(momentum=-0.1), dict(momentum=float("nan")),
                   dict(weight_decay=float("inf")), dict(scale=float("nan"))):
        refused(INVAL, G.gist_muon_update, ctx, d, **{**ok, **change})
    refused(NOMEM, G.gist_muon_update, ctx, d, **{**ok, "ws": Ws(need - 1)})


def test_embed_workspace_serves_fewer_ids():
    """A runner allocates for its largest batch and passes the same workspace for every other."""
    sizes = sorted({n + k for n in (1, 8, 32, 64, 2048, 8192, 32768, 1 << 17, 1 << 20, 1 << 22) for k in (-1, 0, 1, 7)})
    for d in (1, 30, 1024):
        need = [G.gist_embed_grad_workspace(n, 1000, d) for n in sizes]
        assert need == sorted(need)


def test_embed_grad_ids_that_chunks_would_carry_past_int32():
    """The gradient's kernels round n up to whole chunks (of 128 for this many ids) in int32:
    an n that this carries past 2^31 - 1 is refused, and has no workspace."""
    w = Ws(1 << 62)
    for n in (2**31 - 127, 2**31 - 8, 2**31 - 2):
        refused(UNSUP, G.gist_embed_grad, ctx, n, 5, 1, I, 1.0, A, 1, A, 1, w)
        refused(UNSUP, G.gist_embed_grad_sgd, ctx, n, 5, 1, I, 1.0, A, 1, 0.1, A, 1, w)
        assert G.gist_embed_grad_workspace(n, 5, 1) == 0
    need = G.gist_embed_grad_workspace(2**31 - 128, 5, 1)     # the largest accepted: on to the next check
    assert need > 4 * 4 * (2**31 - 128)
    refused(NOMEM, G.gist_embed_grad, ctx, 2**31 - 128, 5, 1, I, 1.0, A, 1, A, 1, Ws(need - 1))


def test_muon_arrays_that_overlap():
    """An update reads dW again after M is written and W is the last to be: three arrays.  The
    factor may take its gradient's place where both are fp32."""
    B, D = np.zeros(64, dtype=np.float32), np.zeros(64, dtype=np.float32)
    d = G.muon_desc(8, 6)
    w = Ws(G.gist_muon_workspace_size(d))
    for W, dW, M in ((A, A, B), (A, B, A), (B, A, A)):
        refused(INVAL, G.gist_muon_update, ctx, d, W, dW, M, 0.1, 0.9, 0.0, 1.0, w)
    h = G.muon_desc(8, 6, dtype=G.GIST_DTYPE_F16_IN)
    refused(INVAL, G.gist_orthogonalize, ctx, h, D, D, Ws(G.gist_muon_workspace_size(h)))


def test_outgrown_buffers_live_on():
    """A recorded step keeps the addresses of the buffers it was recorded with, so none of them
    is freed when a later call needs a larger one, or one for another K."""
    import weakref
    import torch
    from paper_2102_10424_amd import step as S
    rows = S.LearnedRows(None, torch.zeros(50, 4), n_cap=10, device="cpu")
    first = weakref.ref(rows.ws)
    for n in (11, 40, 300, 5000):
        rows._reserve(n)
        assert rows.ws.numel() >= G.gist_embed_grad_workspace(n, 50, 4)
    assert first() is not None and first() is not rows.ws
    run = S.SubGCN(None, "gcn", [8, 300, 5000], 16, device="cpu")
    run.prepare_muon(G.GIST_DTYPE_F16_IN)
    ws = weakref.ref(run.muon_ws)
    run.prepare_muon(G.GIST_DTYPE_F32)
    assert ws() is not None and ws() is not run.muon_ws
    three = run._log_probs_buffers(16, 3)
    refs = [weakref.ref(t) for k, t in three.items() if k != "n"]
    run._log_probs_buffers(16, 0)
    assert run.lp is not three
    assert run._log_probs_buffers(12, 3) is three and run.lp is three
    assert run._log_probs_buffers(40, 3)["n"] >= 40     # a larger batch
    del three
    assert all(r() is not None for r in refs)


def test_layers_refuse_fp16_operands():
    refused(INVAL, G.gist_layer_workspace_size,
            G.layer_desc(G.GIST_LAYER_GCN, G.GIST_ACT_NONE, 8, 4, 4, G.GIST_DTYPE_F16_IN))
    refused(INVAL, G.gist_gat_workspace_size,
            G.gat_desc(8, 8, 4, 4, G.GIST_ACT_NONE, G.GIST_DTYPE_F16_IN))


# ---- the references ---------------------------------------------------------------
def test_log_probs_grad_reference_against_differences():
    """The gradient formula against central differences of the 64-bit objective: with step
    h the difference is off by h^2 / 6 of the third derivative (below 10 here) and 2^-52 / h
    of the value."""
    rng = np.random.default_rng(3)
    z = rng.standard_normal((4, 9))
    z[1, 3] = -np.inf
    y = np.array([2, 0, -1, 8])
    gl, gh = rng.standard_normal(4), rng.standard_normal(4)

    def f(zz):
        lse, lp, H = R.log_probs(zz, y)
        return float((gl * np.where(y >= 0, lp, 0.0) + gh * H).sum())

    d = R.log_probs_grad(z, y, gl, gh)
    h = 1e-4
    for v in range(4):
        for j in range(9):
            if z[v, j] == -np.inf:
                assert d[v, j] == 0
                continue
            a, b = z.copy(), z.copy()
            a[v, j] += h
            b[v, j] -= h
            assert abs((f(a) - f(b)) / (2 * h) - d[v, j]) < 10 * h * h + 1e-10


def test_orthogonal_reference_forms_agree():
    """The factor by singular values and by the iteration without noise."""
    rng = np.random.default_rng(5)
    for shape in ((5, 9), (9, 5), (1, 7), (6, 6)):
        a = rng.standard_normal(shape)
        w = R.orthogonal(a)
        x = R.orthogonal_noisy(a, 0.0, 0.0, rng)
        # coefficients differ by their rounding to fp32 in the first
        assert np.linalg.norm(w - x) < 1e-5 * np.linalg.norm(w)


# ---- the runners' own checks ---------------------------------------------------------
def no_library(monkeypatch, *names):
    """Library calls replaced by a count: a refused call makes none."""
    from paper_2102_10424_amd import step as S
    calls = []
    for name in names:
        monkeypatch.setattr(S.G, name, lambda *a, name=name: calls.append(name))
    return S, calls


def test_learned_rows_check_their_arrays(monkeypatch):
    """Types, gaps and lengths that the kernels, which see addresses, cannot check."""
    import torch
    S, calls = no_library(monkeypatch, "gist_embed_lookup", "gist_embed_grad_sgd")
    T = torch.zeros(50, 4)
    for bad in (T.double(), T.half(), T[:, :3], T.t(), torch.zeros(50), torch.zeros(2, 25, 4)):
        with pytest.raises(ValueError):
            S.LearnedRows(None, bad, device="cpu")
    rows = S.LearnedRows(None, T, n_cap=10, device="cpu")
    ids, X = torch.zeros(10, dtype=torch.int32), torch.zeros(10, 4)
    bad_ids = (ids.long(), ids.short(), torch.zeros(20, dtype=torch.int32)[::2], ids[:9], ids[:1].expand(10))
    bad_X = (X.double(), X[:9], torch.zeros(10, 5), torch.zeros(10, 5)[:, :4], torch.zeros(40), X[:1].expand(10, 4))
    for call in (lambda i, x: rows.lookup(i, 10, x), lambda i, x: rows.sgd(i, 10, x, 0.1)):
        for i in bad_ids:
            with pytest.raises(ValueError):
                call(i, X)
        for x in bad_X:
            with pytest.raises(ValueError):
                call(ids, x)
    with pytest.raises(ValueError):
        rows.lookup(ids, -1, X)
    assert not calls
    rows.lookup(ids, 10, X)
    rows.sgd(torch.zeros(64, dtype=torch.int32), 10, torch.zeros(16, 4), 0.1)   # longer ones serve
    rows.lookup(ids[:0], 0, X[:0])
    assert calls == ["gist_embed_lookup", "gist_embed_grad_sgd", "gist_embed_lookup"]


class CpuBatch:
    """Sizes and labels of a mini-batch without matrices: no library call is made on it."""

    def __init__(self, n):
        import torch
        self.n, self.nnz, self.X = n, n, torch.zeros(n, 8)
        self.labels = torch.zeros(n, dtype=torch.int32)

    def rows(self, l):
        return self.n

    def adj(self, l):
        return None, None


def test_log_probs_grad_takes_the_last_forward_pass(monkeypatch):
    """The gradient needs the log-sum-exp of the logits as they are: after another forward
    pass, of another batch, or without log_probs, it is refused."""
    import torch
    S, calls = no_library(monkeypatch, "gist_gcn_layer_fwd", "gist_log_probs", "gist_log_probs_bwd")
    run = S.SubGCN(None, "gcn", [8, 24, 5], 16, device="cpu")
    a, b = CpuBatch(16), CpuBatch(16)
    g = torch.zeros(16)
    params = [torch.zeros(8, 24), torch.zeros(24, 5)]

    def refuse(batch, *grads):
        n = len(calls)
        with pytest.raises(ValueError):
            run.log_probs_grad(batch, *grads)
        assert len(calls) == n

    refuse(a, g)                       # no log_probs yet
    run.forward(a, params)
    refuse(a, g)
    run.log_probs(a)
    run.log_probs_grad(a, g)
    run.log_probs_grad(a, g, torch.zeros(20))
    run.log_probs_grad(a, None, g)
    run.log_probs_grad(a, g[:, None], g[None])   # any shape of so many in a row
    refuse(a, torch.tensor(1.0))
    refuse(b, g)                       # another batch's labels
    refuse(CpuBatch(9), g)
    for bad in (g.double(), g[:15], g[:1].expand(16), torch.zeros(32)[::2]):
        refuse(a, bad)
        refuse(a, g, bad)
    run.log_probs(a, K=3)              # another K, the same logits
    run.log_probs_grad(a, g)
    run.forward(b, params)
    refuse(a, g)
    refuse(b, g)
    run.log_probs(b)
    run.log_probs_grad(b, g)
    n = len(calls)
    with pytest.raises(ValueError):
        run.log_probs(CpuBatch(17))    # more rows than the logits have
    assert len(calls) == n


def test_muon_checks_its_momenta(monkeypatch):
    import torch
    S, calls = no_library(monkeypatch, "gist_muon_update")
    run = S.SubGCN(None, "sage", [8, 24, 5], 16, device="cpu")
    params = [torch.zeros(16, 24), torch.zeros(48, 5)]
    ok = [torch.zeros(16, 24), torch.zeros(48, 5)]
    run.muon(params, ok, 0.1)
    assert len(calls) == 2
    for bad in (ok[0].double(), torch.zeros(8, 24), torch.zeros(16, 25)[:, :24], torch.zeros(16 * 24)):
        with pytest.raises(ValueError):
            run.muon(params, [bad, ok[1]], 0.1)
    assert len(calls) == 2


def test_one_optimizer_a_step(monkeypatch):
    import torch
    S, calls = no_library(monkeypatch, "gist_gcn_layer_fwd")
    run = S.SubGCN(None, "gcn", [8, 24, 5], 16, device="cpu")
    params = [torch.zeros(8, 24), torch.zeros(24, 5)]
    with pytest.raises(ValueError):
        run.step(CpuBatch(16), params, 0.1, adam=(params, params, 1, True), muon=(params, True))
    assert not calls


@pytest.mark.parametrize("change,message", [
    (dict(K=0, top_logp=A), "K == 0 takes no"), (dict(K=0, top_idx=I), "K == 0 takes no"),
    (dict(K=0, top_logp=A, top_idx=I), "K == 0 takes no"),
    (dict(K=2), "K > 0 needs"), (dict(K=2, top_logp=A), "K > 0 needs"), (dict(K=2, top_idx=I), "K > 0 needs"),
    (dict(K=8, top_logp=A, top_idx=I), "K outside"), (dict(K=-1), "K outside"), (dict(tokens=None), "logp needs tokens"),
    (dict(logits=None), "NULL logits"), (dict(store=3), "unknown store"), (dict(ldz=6), "bad sizes")])
def test_log_probs_top_outputs_match_K(change, message):
    """From a call that is right but for the change, each refusal by its own message."""
    a = dict(n=2, C_=7, logits=A, ldz=7, store=0, tokens=I, logp=A, entropy=A, lse=A, K=0,
             top_logp=None, top_idx=None, ws=None)
    with pytest.raises(G.GistError) as e:
        G.gist_log_probs(ctx, **{**a, **change})
    assert e.value.status == INVAL and message in str(e.value)


@pytest.mark.parametrize("C", [5, 1025, 4096, 8191, 8192, 20011, 131072, 1 << 20, 1 << 22])
def test_log_probs_workspace_serves_fewer_rows(C):
    """Fewer rows are cut into more parts each: a workspace sized for the largest batch serves
    every other.  A call's own need is no more than what is reported for it."""
    sizes = sorted({max(0, n + k) for n in (0, 1, 2, 3, 7, 32, 63, 128, 341, 512, 1000, 1024, 5000, 1 << 20) for k in (-1, 0, 1)})
    for K in (0, 5):
        need = [G.gist_log_probs_workspace(n, C, K) for n in sizes]
        assert need == sorted(need)
        assert need[-1] < (1 << 17)     # 2,047 parts at most
        a = dict(C_=C, logits=A, ldz=C, store=0, tokens=I, logp=A, entropy=A, lse=A, K=K,
                 top_logp=A if K else None, top_idx=I if K else None)
        for n, w in zip(sizes, need):      # past the size check, on to that of the address
            if 0 < n < 1024 and w:         # (more rows need no workspace: nothing would be refused)
                with pytest.raises(G.GistError) as e:
                    G.gist_log_probs(ctx, n=n, **a, ws=Ws(w, 4104))
                assert "aligned" in str(e.value), (n, str(e.value))
