"""Arguments that the norm, 8-bit rows, class-table loss and AdamW calls refuse, and their workspace
sizes.  No GPU needed: every check runs on the host before anything touches the device."""

import ctypes

import numpy as np
import pytest

import more_ref as R

G = pytest.importorskip("paper_2102_10424_amd.gist",
                        reason="libgist.so not built (python -m paper_2102_10424_amd.build)")


class NoDevice:
    """A context handle over zeroed memory: device 0, the default stream.  A refused call
    reads no more of it."""

    def __init__(self):
        self.mem = ctypes.create_string_buffer(256)
        self.handle = ctypes.cast(self.mem, ctypes.c_void_p)


class Null:
    handle = None


class Ws:
    def __init__(self, nbytes, addr=4096):
        self.n, self.a = nbytes, addr

    def numel(self):
        return self.n

    def element_size(self):
        return 1

    def data_ptr(self):
        return self.a


ctx = NoDevice()
arr = lambda: np.zeros(64, dtype=np.float32)     # stand for device memory; never read
A, B, D, E, F, H = (arr() for _ in range(6))
I = np.zeros(64, dtype=np.int32)
INVAL, NOMEM, UNSUP = G.GIST_E_INVAL, G.GIST_E_NOMEM, G.GIST_E_UNSUPPORTED
NAN, INF = float("nan"), float("inf")


def refused(status, fn, *args, **kw):
    with pytest.raises(G.GistError) as e:
        fn(*args, **kw)
    assert e.value.status == status, e.value


@pytest.mark.parametrize("change,status", [
    (dict(n=-1), INVAL), (dict(d=0), INVAL), (dict(n=2**31 - 1), UNSUP),
    (dict(d=(1 << 22) + 1, ldx=1 << 23, ldr=1 << 23, ldh=1 << 23, ldy=1 << 23), UNSUP),
    (dict(ldx=3), INVAL), (dict(ldr=3), INVAL), (dict(ldh=3), INVAL), (dict(ldy=3), INVAL),
    (dict(store=3), INVAL), (dict(store=-1), INVAL), (dict(out_store=4), INVAL),
    (dict(eps=-1.0), INVAL), (dict(eps=NAN), INVAL), (dict(eps=INF), INVAL),
    (dict(x=None), INVAL), (dict(gain=None), INVAL), (dict(y=None), INVAL),
    (dict(out_store=3), INVAL), (dict(y_scale=F), INVAL), (dict(h=A, ldh=5), INVAL),
    (dict(h=B, ldh=5), INVAL), (dict(y=A, out_store=1), INVAL), (dict(y=A, ldy=5), INVAL),
    (dict(y=B, out_store=3, y_scale=F), INVAL), (dict(y=E), INVAL)])
def test_rms_norm(change, status):
    a = dict(n=2, d=4, x=A, ldx=4, residual=B, ldr=4, store=0, gain=D, eps=1e-6, h=E, ldh=4, y=F,
             ldy=4, out_store=0, y_scale=None, rstd=None)
    refused(status, G.gist_rms_norm, ctx, **{**a, **change})
    refused(INVAL, G.gist_rms_norm, Null, **a)


@pytest.mark.parametrize("change,status", [
    (dict(n=-1), INVAL), (dict(d=0), INVAL), (dict(n=2**31 - 1), UNSUP), (dict(lddy=3), INVAL),
    (dict(ldh=3), INVAL), (dict(ldds=3), INVAL), (dict(lddx=3), INVAL), (dict(store=3), INVAL),
    (dict(dy_store=3), INVAL), (dict(dy=None), INVAL), (dict(h=None), INVAL),
    (dict(gain=None), INVAL), (dict(rstd=None), INVAL), (dict(dx=A, lddx=5), INVAL),
    (dict(dx=A, dy_store=1), INVAL), (dict(dx=B, lddx=6), INVAL), (dict(dx=E, lddx=6), INVAL),
    (dict(ws=None), NOMEM), (dict(ws="small"), NOMEM), (dict(ws="odd"), INVAL)])
def test_rms_norm_bwd(change, status):
    need = G.gist_rms_norm_bwd_workspace(2, 4)
    a = dict(n=2, d=4, dy=A, lddy=4, dy_store=0, h=B, ldh=4, store=0, gain=D, rstd=D, dsum=E, ldds=4,
             dx=F, lddx=4, dgain=H, ws=Ws(need))
    a.update(change)
    if a["ws"] == "small":
        a["ws"] = Ws(need - 1)
    if a["ws"] == "odd":
        a["ws"] = Ws(need, 4100)
    refused(status, G.gist_rms_norm_bwd, ctx, **a)
    refused(INVAL, G.gist_rms_norm_bwd, Null, **a)


def test_rms_norm_bwd_workspace():
    for bad in ((-1, 4), (2, 0), (2**31, 4), (2, (1 << 22) + 1)):
        assert G.gist_rms_norm_bwd_workspace(*bad) == 0
    for d in (1, 64, 1024, 1025, 5000):
        need = [G.gist_rms_norm_bwd_workspace(n, d) for n in (1, 3, 4, 5, 1000, 4096, 10**6)]
        assert need == sorted(need) and need[0] >= 4 * d


@pytest.mark.parametrize("change,status", [
    (dict(n=-1), INVAL), (dict(d=0), INVAL), (dict(n=2**31 - 1), UNSUP), (dict(ldx=3), INVAL),
    (dict(ldy=3), INVAL), (dict(store=3), INVAL), (dict(x=None), INVAL), (dict(y=None), INVAL),
    (dict(scale=None), INVAL), (dict(y=A), INVAL)])
def test_quantize_rows(change, status):
    a = dict(n=2, d=4, x=A, ldx=4, store=0, y=B, ldy=4, scale=D)
    refused(status, G.gist_quantize_rows, ctx, **{**a, **change})
    refused(INVAL, G.gist_quantize_rows, Null, **a)


DESC = [(dict(n=-1), INVAL), (dict(C_=0), INVAL), (dict(d=0), INVAL), (dict(ldh=3), INVAL),
        (dict(ldt=3), INVAL), (dict(lddh=3), INVAL), (dict(lddt=-1), INVAL), (dict(store=4), INVAL),
        (dict(store=-1), INVAL), (dict(store=0, dtype=G.GIST_DTYPE_F16_IN), INVAL),
        (dict(scale=NAN), INVAL), (dict(grad_scale=INF), INVAL), (dict(n=2**30 + 1), UNSUP),
        (dict(C_=2**30 + 1), UNSUP), (dict(d=65537), UNSUP)]


@pytest.mark.parametrize("change,status", DESC)
def test_table_xent_desc(change, status):
    d = G.table_xent_desc(**{**dict(n=2, C_=3, d=4, store=1), **change})
    refused(status, G.gist_table_xent_workspace, d, False)
    refused(status, G.gist_table_xent, ctx, d, A, None, B, None, I, None, D, None, None, None, None,
            Ws(1 << 40))


def test_table_xent_calls():
    d = G.table_xent_desc(2, 3, 4, G.GIST_STORE_BF16)
    need = G.gist_table_xent_workspace(d, True)
    ok = dict(H=A, h_scale=None, T=B, t_scale=None, labels=I, n_valid_dev=None, loss_dev=D, logp=None,
              lse=None, dH=E, dT=F, ws=Ws(need))
    call = lambda desc=d, c=ctx, **ch: (c, desc) + tuple({**ok, **ch}.values())
    for ch in (dict(H=None), dict(T=None), dict(labels=None), dict(loss_dev=None), dict(dH=None),
               dict(dT=None), dict(h_scale=D), dict(t_scale=D), dict(dH=A), dict(dT=B), dict(dH=B),
               dict(dT=A), dict(dT=E), dict(ws=Ws(need, 4104))):
        refused(INVAL, G.gist_table_xent, *call(**ch))
    refused(INVAL, G.gist_table_xent, *call(c=Null))
    refused(NOMEM, G.gist_table_xent, *call(ws=Ws(64)))
    refused(NOMEM, G.gist_table_xent, *call(ws=None))
    e = G.table_xent_desc(2, 3, 4, G.GIST_STORE_E4M3)
    refused(INVAL, G.gist_table_xent_workspace, e, True)
    refused(INVAL, G.gist_table_xent, *call(e, h_scale=D, t_scale=D))
    for ch in (dict(h_scale=D), dict(t_scale=D), dict()):
        refused(INVAL, G.gist_table_xent, *call(e, dH=None, dT=None, **ch))


@pytest.mark.parametrize("store,dtype", [(0, 0), (0, 1), (1, 0), (2, 0), (3, 0)])
def test_table_xent_workspace_holds_no_logits(store, dtype):
    """Far below n C values where these are many, whatever the shape."""
    for n, C, d in ((1, 1, 1), (1, 1 << 20, 64), (8192, 131072, 1024), (1 << 20, 50000, 256), (33, 7, 5000)):
        D = G.table_xent_desc(n, C, d, store, dtype)
        for grad in (False, True) if store != 3 else (False,):
            need = G.gist_table_xent_workspace(D, grad)
            operands = 8 * (n + 64) * (d + 128) + 4 * (C + 64) * (d + 128)
            parts = 4 * 4 * max(n, 1) * (d + 4) + 4 * 4 * (1 << 20) * 64
            assert 0 < need < (2 << 30) + operands + parts
    assert G.gist_table_xent_workspace(G.table_xent_desc(0, 5, 4, 1), True) == 0


TENSOR = dict(W=A, dW=B, m=D, v=E, n=64)


def tensors(**change):
    return G.adamw_tensors([G.adamw_tensor(**TENSOR), G.adamw_tensor(**{**TENSOR, **change})])


@pytest.mark.parametrize("change,status", [
    (dict(n=-1), INVAL), (dict(n=2**34), UNSUP), (dict(W=None), INVAL), (dict(dW=None), INVAL),
    (dict(m=None), INVAL), (dict(v=None), INVAL), (dict(grad_store=3), INVAL),
    (dict(grad_store=-1), INVAL), (dict(copy=F, copy_store=0), INVAL), (dict(copy=F, copy_store=3), INVAL),
    (dict(weight_decay=NAN), INVAL), (dict(m_scale=F), INVAL), (dict(v_scale=F), INVAL),
    (dict(m_scale=F, v_scale=F), INVAL), (dict(dW=A), INVAL), (dict(m=A), INVAL), (dict(v=D), INVAL),
    (dict(copy=A), INVAL), (dict(m_scale=D, v_scale=F), INVAL)])
def test_adamw_tensors(change, status):
    refused(status, G.gist_adamw_update, ctx, tensors(**change), 0.1, 1)
    refused(status, G.gist_adamw_update_dev, ctx, tensors(**change), F)


@pytest.mark.parametrize("change", [
    dict(lr=NAN), dict(step=0), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(eps=-1.0),
    dict(eps=INF), dict(flags=2), dict(grad_scale=NAN)])
def test_adamw_arguments(change):
    a = dict(lr=0.1, step=1)
    refused(INVAL, G.gist_adamw_update, ctx, tensors(), **{**a, **change})
    refused(INVAL, G.gist_adamw_coefficients, **{**a, **change})
    refused(INVAL, G.gist_adamw_update, Null, tensors(), **a)
    refused(INVAL, G.gist_adamw_update_dev, Null, tensors(), F)
    refused(INVAL, G.gist_adamw_update_dev, ctx, tensors(), None)
    for k in ("beta1", "beta2", "eps"):
        if k in change:
            refused(INVAL, G.gist_adamw_update_dev, ctx, tensors(), F, **change)


def test_adamw_coefficients():
    c = G.gist_adamw_coefficients(1e-3, 7, 0.9, 0.99, flags=G.GIST_ADAM_FRESH, grad_scale=0.5, seed=0xfedcba98)
    assert c[0] == np.float32(float(np.float32(1e-3)) / (1 - float(np.float32(0.9)) ** 7))
    assert c[2] == 1 and c[3] == np.float32(1e-3) and c[4] == 0.5
    assert c[5:].view(np.uint32)[0] == 0xfedcba98
    assert np.array_equal(c[:3], G.gist_adam_coefficients(1e-3, 7, 0.9, 0.99, flags=G.GIST_ADAM_FRESH))


# ---- the references ---------------------------------------------------------------
def test_table_xent_reference_against_differences():
    """The gradient formula against central differences in 64 bits: step 1e-4 loses 1e-8 of third
    derivatives below 10 and 2^-52 / 1e-4 of the value."""
    rng = np.random.default_rng(0)
    H, T = rng.standard_normal((4, 5)), rng.standard_normal((6, 5))
    y = np.array([2, -1, 0, 5])
    r = R.table_xent(H, T, y, 0.8, 1.0)
    f = lambda a, b: R.table_xent(a, b, y, 0.8, 1.0)["loss"]
    for name, x in (("dH", H), ("dT", T)):
        for i in range(x.shape[0]):
            for j in range(5):
                p, q = x.copy(), x.copy()
                p[i, j] += 1e-4
                q[i, j] -= 1e-4
                d = (f(p, T) - f(q, T)) if name == "dH" else (f(H, p) - f(H, q))
                assert abs(d / 2e-4 - r[name][i, j]) < 1e-7


def test_rms_reference_against_differences():
    rng = np.random.default_rng(1)
    h, dy, ds = (rng.standard_normal((3, 6)) for _ in range(3))
    g = rng.standard_normal(6)
    dx, _, dg, _ = R.rms_grad(dy, h, g, 1e-3, ds)
    f = lambda a, b: float((dy * R.rms(a, b, 1e-3)[1]).sum() + (ds * a).sum())
    for j in range(6):
        for i in range(3):
            p, q = h.copy(), h.copy()
            p[i, j] += 1e-5
            q[i, j] -= 1e-5
            assert abs((f(p, g) - f(q, g)) / 2e-5 - dx[i, j]) < 1e-7
        p, q = g.copy(), g.copy()
        p[j] += 1e-5
        q[j] -= 1e-5
        assert abs((f(h, p) - f(h, q)) / 2e-5 - dg[j]) < 1e-7


def test_random_bits_are_uniform():
    """Mean and deviation of 2^16 draws, within six standard errors, and no link between the two."""
    a, b = R.random_bits(1 << 16, 3, 12345)
    for x in (a, b):
        assert 0 <= x.min() and x.max() < 65536
        assert abs(x.mean() - 32767.5) < 6 * 65536 / np.sqrt(12 * 65536)
    assert abs(np.corrcoef(a, b)[0, 1]) < 6 / 256
    assert abs(np.corrcoef(a[1:], a[:-1])[0, 1]) < 6 / 256


# ---- the runners' own checks ---------------------------------------------------------
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


def test_adamw_checks_its_arrays():
    import torch
    from paper_2102_10424_amd import step as S
    W, g = torch.zeros(6, 4), torch.zeros(6, 4)
    for bad in (dict(W=W.double()), dict(W=W[:, :3]), dict(W=W.t()), dict(dW=g.double()),
                dict(dW=g[:5]), dict(dW=torch.zeros(6, 8)[:, :4]), dict(copy=torch.zeros(6, 4)),
                dict(copy=torch.zeros(5, 4, dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            S.AdamW(None, [dict(dict(W=W, dW=g), **bad)], device="cpu")
    o = S.AdamW(None, [dict(W=W, dW=g.half(), copy=torch.zeros(24, dtype=torch.float16))], eight=True, device="cpu")
    assert [t.numel() for t in o.state[0]] == [24, 24, 1, 1]
    assert S.AdamW(None, [], device="cpu").step is not None


def test_table_head_checks_its_arrays(monkeypatch):
    import torch
    from paper_2102_10424_amd import step as S
    calls = []
    for name in ("gist_rms_norm", "gist_rms_norm_bwd", "gist_table_xent", "gist_quantize_rows", "gist_gcn_layer_fwd"):
        monkeypatch.setattr(S.G, name, lambda *a, name=name: calls.append(name))
    T = torch.zeros(50, 5)
    for bad in (T.double(), T[:, :4], T.t(), torch.zeros(250)):
        with pytest.raises(ValueError):
            S.TableHead(None, bad, device="cpu")
    for kw in (dict(dtype=torch.float64), dict(grad_scale=0.0), dict(grad_scale=float("nan"))):
        with pytest.raises(ValueError):
            S.TableHead(None, T, device="cpu", **kw)
    head = S.TableHead(None, T, device="cpu")
    run, other = S.SubGCN(None, "gcn", [8, 24, 5], 16, device="cpu"), S.SubGCN(None, "gcn", [8, 24, 6], 16, device="cpu")
    b = CpuBatch(16)
    run.forward(b, [torch.zeros(8, 24), torch.zeros(24, 5)])
    calls.clear()
    with pytest.raises(ValueError):
        head.loss_and_grad(other, b)
    for res in (torch.zeros(16, 4), torch.zeros(15, 5), torch.zeros(16, 5).double(), torch.zeros(16, 10)[:, :5]):
        with pytest.raises(ValueError):
            head.loss_and_grad(run, b, res)
    with pytest.raises(ValueError):
        head.score(run, b, eight=True)
    b.labels = b.labels.long()
    with pytest.raises(ValueError):
        head.loss_and_grad(run, b)
    assert not calls
    b.labels = b.labels.int()
    head.loss_and_grad(run, b, torch.zeros(16, 5))
    head.quantise()
    head.score(run, b, eight=True)
    assert calls == ["gist_rms_norm", "gist_table_xent", "gist_rms_norm_bwd", "gist_quantize_rows", "gist_rms_norm", "gist_table_xent"]
    with pytest.raises(ValueError):
        run.step(b, [], 0.1, adam=(1, 2, 3, 4), adamw=(None, 1))
    with pytest.raises(ValueError):
        run.step(b, [torch.zeros(8, 24), torch.zeros(24, 5)], 0.1, residual=b.X)


def test_table_head_keeps_outgrown_buffers():
    """A recorded step keeps the addresses of the buffers it was recorded with."""
    import weakref
    import torch
    from paper_2102_10424_amd import step as S
    head = S.TableHead(None, torch.zeros(50, 5), n_cap=16, device="cpu")
    head.prepare(16)
    refs = [weakref.ref(t) for t in head.b.values()] + [weakref.ref(head.ws[True])]
    head.prepare(17)
    head.prepare(5000)
    assert all(r() is not None for r in refs) and head.n_cap >= 5000
    assert head.ws[True].numel() >= S.G.gist_table_xent_workspace(head._desc(5000, head.store), True)


def test_table_xent_most_classes():
    """bf16 products' gradients address 256 rows of exponentials in 32 bits."""
    for store, dtype, limit in ((1, 0, 23), (0, G.GIST_DTYPE_BF16_IN, 23), (2, 0, 29), (0, 0, 29)):
        d = lambda C: G.table_xent_desc(1, C, 4, store, dtype)
        assert G.gist_table_xent_workspace(d(1 << limit), True) > 0
        refused(UNSUP, G.gist_table_xent_workspace, d((1 << limit) + 1), True)
        refused(UNSUP, G.gist_table_xent, ctx, d((1 << limit) + 1), A, None, B, None, I, None, D, None, None,
                E, F, Ws(1 << 50))
        assert G.gist_table_xent_workspace(d(1 << 29), False) > 0
        refused(UNSUP, G.gist_table_xent_workspace, d((1 << 29) + 1), False)


def test_table_head_replaces_outgrown_buffers_without_a_recording():
    import types
    import weakref
    import torch
    from paper_2102_10424_amd import step as S
    head = S.TableHead(types.SimpleNamespace(captures=0), torch.zeros(50, 5), n_cap=16, device="cpu")
    head.prepare(16)
    refs = [weakref.ref(t) for t in head.b.values()] + [weakref.ref(head.ws[True])]
    head.prepare(5000)
    assert all(r() is None for r in refs) and head.n_cap == 5000 and not head._kept


def test_table_head_of_an_empty_batch(monkeypatch):
    import torch
    from paper_2102_10424_amd import step as S
    calls = []
    for name in ("gist_rms_norm", "gist_rms_norm_bwd", "gist_table_xent", "gist_gcn_layer_fwd"):
        monkeypatch.setattr(S.G, name, lambda *a, name=name: calls.append(name))
    head = S.TableHead(None, torch.zeros(50, 5), device="cpu")
    run, b = S.SubGCN(None, "gcn", [8, 24, 5], 16, device="cpu"), CpuBatch(0)
    head.loss_and_grad(run, b)
    head.score(run, b)
    assert calls == ["gist_rms_norm", "gist_table_xent", "gist_rms_norm_bwd", "gist_rms_norm", "gist_table_xent"]


def test_adamw_belongs_to_its_runner_and_weights(monkeypatch):
    import torch
    from paper_2102_10424_amd import step as S
    calls = []
    for name in ("gist_gcn_layer_fwd", "gist_gcn_layer_bwd", "gist_rms_norm", "gist_rms_norm_bwd",
                 "gist_table_xent", "gist_softmax_xent", "gist_adamw_update"):
        monkeypatch.setattr(S.G, name, lambda *a, name=name: calls.append(name))
    run, b = S.SubGCN(None, "gcn", [8, 24, 5], 16, device="cpu"), CpuBatch(16)
    weights = lambda: [torch.zeros(8, 24), torch.zeros(24, 5)]
    params = weights()
    for gs in (2.0, 0.5):
        with pytest.raises(ValueError):
            run.adamw(params, S.TableHead(None, torch.zeros(50, 5), grad_scale=gs, device="cpu"))
    head = S.TableHead(None, torch.zeros(50, 5), device="cpu")
    opt = run.adamw(params, head)
    twin = S.SubGCN(None, "gcn", [8, 24, 5], 16, device="cpu")
    for r, p, o in ((run, weights(), opt), (twin, params, opt), (run, params[::-1], opt),
                    (run, params, S.AdamW(None, head.items(), device="cpu"))):
        with pytest.raises(ValueError):
            r.step(b, p, 0.1, adamw=(o, 1), head=head)
    assert not calls
    run.step(b, params, 0.1, adamw=(opt, 1), head=head)
    assert calls[-1] == "gist_adamw_update"
