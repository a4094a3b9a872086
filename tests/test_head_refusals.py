"""What the end of a step refuses beyond its arrays: the norm's backward pass with labels,
optimizers of another head, batches that the runner has no rows for, learned rows of another
table; and that the table's copy follows them.  No GPU needed: every check runs on the host
before anything touches the device."""

import pytest

from test_more_refusals import (A, B, D, E, F, G, H, I, INVAL, NOMEM, UNSUP, CpuBatch, Null, Ws, ctx,
                                refused)


@pytest.fixture
def calls(monkeypatch):
    """The library's device calls, by name, in place of being made."""
    from paper_2102_10424_amd import step as S
    made = []
    for name in ("gist_gcn_layer_fwd", "gist_gcn_layer_bwd", "gist_rms_norm", "gist_rms_norm_bwd",
                 "gist_table_xent", "gist_softmax_xent", "gist_quantize_rows", "gist_adamw_update",
                 "gist_embed_lookup"):
        monkeypatch.setattr(S.G, name, lambda *a, name=name: made.append(name))
    return made


@pytest.mark.parametrize("change,status", [
    (dict(n=-1), INVAL), (dict(d=0), INVAL), (dict(n=2**31 - 1), UNSUP), (dict(lddy=3), INVAL),
    (dict(ldds=3), INVAL), (dict(dy_store=3), INVAL), (dict(dy=None), INVAL), (dict(rstd=None), INVAL),
    (dict(dx=A, lddx=5), INVAL), (dict(ws=None), NOMEM), (dict(ws=Ws(1 << 20, 4100)), INVAL)])
@pytest.mark.parametrize("labels,n_dev", [(I, None), (None, I), (I, I)])
def test_rms_norm_bwd_padded(change, status, labels, n_dev):
    need = G.gist_rms_norm_bwd_workspace(2, 4)
    a = dict(n=2, d=4, dy=A, lddy=4, dy_store=0, h=B, ldh=4, store=0, gain=D, rstd=D, dsum=E, ldds=4,
             dx=F, lddx=4, dgain=H, ws=Ws(need), labels=labels, n_valid_dev=n_dev)
    refused(status, G.gist_rms_norm_bwd, ctx, **{**a, **change})
    refused(INVAL, G.gist_rms_norm_bwd, Null, **a)


def test_adamw_belongs_to_its_head(calls):
    import torch
    from paper_2102_10424_amd import step as S
    run, b = S.SubGCN(None, "gcn", [8, 24, 5], 16, device="cpu"), CpuBatch(16)
    params = [torch.zeros(8, 24), torch.zeros(24, 5)]
    head, other = (S.TableHead(None, torch.zeros(50, 5), device="cpu") for _ in range(2))
    with_head, without = run.adamw(params, head), run.adamw(params)
    scaled = S.TableHead(None, torch.zeros(50, 5), grad_scale=8.0, device="cpu")   # has an AdamW of its own
    for opt, h in ((with_head, None), (with_head, other), (without, head), (with_head, scaled)):
        with pytest.raises(ValueError):
            run.step(b, params, 0.1, adamw=(opt, 1), head=h)
        assert not calls
    for opt, h in ((with_head, head), (without, None), (without, scaled)):
        run.step(b, params, 0.1, adamw=(opt, 1), head=h)
        assert calls.pop() == "gist_adamw_update"
        calls.clear()


@pytest.mark.parametrize("n", [17, 1000])
def test_more_rows_than_the_runner_has(calls, n):
    """Its outputs and their gradient end at its capacity."""
    import torch
    from paper_2102_10424_amd import step as S
    run, head = S.SubGCN(None, "gcn", [8, 24, 5], 16, device="cpu"), S.TableHead(None, torch.zeros(50, 5), device="cpu")
    params, big = [torch.zeros(8, 24), torch.zeros(24, 5)], CpuBatch(n)
    head.quantise()
    calls.clear()
    for f in (lambda: head.score(run, big), lambda: head.score(run, big, eight=True),
              lambda: head.loss_and_grad(run, big)):
        with pytest.raises(ValueError):
            f()
    assert not calls
    run.forward(big, params)
    head.loss_and_grad(run, big)
    head.score(run, big)
    assert calls[-1] == "gist_table_xent" and run.dlogits.shape[0] >= n


def test_learned_rows_of_another_table():
    import torch
    from paper_2102_10424_amd import step as S
    T = torch.zeros(50, 5)
    head = S.TableHead(None, T, dtype=torch.bfloat16, device="cpu")
    for other in (torch.zeros(50, 5), T[:40], T[1:]):
        with pytest.raises(ValueError):
            S.LearnedRows(None, other, head=head, device="cpu")
    assert S.LearnedRows(None, T, head=head, device="cpu").head is head


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_table_copy_follows(monkeypatch, dtype):
    """After round_table, and after the learned rows' step, the copy is the table's."""
    import torch
    from paper_2102_10424_amd import step as S
    T = torch.randn(50, 5)
    head = S.TableHead(None, T, dtype=getattr(torch, dtype), device="cpu")
    same = lambda: head.table16 is None or torch.equal(head.table16, T.to(head.dtype))
    T += 1
    head.round_table()
    assert same()
    monkeypatch.setattr(S.G, "gist_embed_grad_sgd", lambda *a: T.mul_(2))
    rows = S.LearnedRows(None, T, device="cpu", head=head)
    rows.sgd(torch.zeros(3, dtype=torch.int32), 3, torch.zeros(3, 5), 0.1)
    assert same()
