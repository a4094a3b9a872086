"""What the end of a step refuses beyond its arrays: the norm's backward pass with labels.  No GPU
needed: every check runs on the host before anything touches the device."""

import pytest

from test_more_refusals import A, B, D, E, F, G, H, I, INVAL, NOMEM, UNSUP, Null, Ws, ctx, refused


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
