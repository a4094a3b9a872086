"""One table as learned input rows and as a 16-bit head's classes: what the head scores after the
rows' step is the table as it is then, eager, on two streams and in a recorded step; heads and
optimizers made while torch's own stream still has work."""

import numpy as np
import pytest

from gpu_util import to_dev
from test_gpu_table_head import C, D, EPS, SCALE, setup

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    from paper_2102_10424_amd import gist
    return gist


def make(G, ctx, dtype, seed):
    """A batch whose inputs are rows of the table that the head scores against."""
    import torch
    from paper_2102_10424_amd.step import DeviceBatch, LearnedRows, SubGCN, TableHead
    csr, n, widths, W, X, T, gain, y = setup("gcn", seed)
    b = DeviceBatch(csr, to_dev(X), to_dev(y), "cuda")
    run = SubGCN(ctx, "gcn", widths, n, input_grad=True)
    head = TableHead(ctx, to_dev(T.copy()), n_cap=n, dtype=dtype, scale=SCALE, eps=EPS)
    rows = LearnedRows(ctx, head.table, n_cap=n, head=head)
    ids = to_dev(np.random.default_rng(seed).integers(0, C, n).astype(np.int32))
    run.prepare(b)
    head.prepare(n)
    head.prepare(n, False)
    return b, run, [to_dev(w.copy()) for w in W], head, rows, ids


def step(b, run, params, head, rows, ids):
    n = b.n
    rows.lookup(ids, n, b.X)
    run.forward(b, params)
    head.loss_and_grad(run, b, b.X)
    run.backward(b, params)
    rows.sgd(ids, n, run.dH[0], 0.5)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_score_after_the_rows_step(G, dtype):
    import torch
    from paper_2102_10424_amd.step import TableHead
    side = torch.cuda.Stream()
    for ctx in (G.Context(0), G.Context(0, stream=side.cuda_stream)):
        b, run, params, head, rows, ids = made = make(G, ctx, getattr(torch, dtype), 21)
        torch.cuda.synchronize()
        before = head.table.clone()
        for k in range(3):
            if k == 2:                      # weights from elsewhere
                torch.cuda.synchronize()
                head.table.mul_(1.5)
                torch.cuda.synchronize()
                head.round_table()
            step(*made)
            got = head.score(run, b, b.X)
            torch.cuda.synchronize()
            got = {q: v.clone() for q, v in got.items()}
            fresh = TableHead(ctx, head.table, n_cap=b.n, dtype=getattr(torch, dtype), scale=SCALE, eps=EPS)
            torch.cuda.synchronize()
            want = fresh.score(run, b, b.X)
            torch.cuda.synchronize()
            assert not torch.equal(head.table, before)
            if head.table16 is not None:
                assert torch.equal(head.table16, head.table.to(head.dtype)), (k, ctx.stream)
                assert torch.equal(head.table16, fresh.table16), (k, ctx.stream)
            for q in got:
                same = got[q] == want[q]
                assert bool(same.all()), (q, k, ctx.stream, got[q][~same][:4], want[q][~same][:4], int((~same).sum()))


def test_recorded(G):
    """Recorded once, replayed three times beside eager steps of a twin: the same bits."""
    import torch
    side = torch.cuda.Stream()
    ctx, cap = G.Context(0), G.Context(0, stream=side.cuda_stream)
    twins = [make(G, c, torch.bfloat16, 22) for c in (cap, ctx)]
    torch.cuda.synchronize()
    G.gist_capture_begin(cap)
    try:
        step(*twins[0])
    finally:
        rep = G.gist_capture_end(cap)
    for k in range(3):
        G.gist_replay_launch(ctx, rep)
        step(*twins[1])
        torch.cuda.synchronize()
        for a, b in zip(*[(t[3].loss, t[3].table, t[3].table16, t[3].dT) for t in twins]):
            assert torch.equal(a, b), k
        assert torch.equal(twins[0][3].table16, twins[0][3].table.bfloat16()), k


@pytest.mark.parametrize("own_stream", [False, True])
@pytest.mark.parametrize("current", [False, True])
def test_rounded_behind_the_streams_work(G, own_stream, current):
    """The copy is made on the context's stream, behind a change of the table that is still to come there,
    whichever stream is torch's current one."""
    import torch
    from paper_2102_10424_amd.step import TableHead
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    ctx = G.Context(0, stream=side.cuda_stream) if own_stream else G.Context(0)
    on = side if own_stream else torch.cuda.default_stream()
    head = TableHead(ctx, torch.randn(3000, 24, device="cuda"), dtype=torch.bfloat16)
    torch.cuda.synchronize()
    for k in range(3):
        with torch.cuda.stream(on):
            torch.cuda._sleep(20_000_000)      # some 10 ms
            head.table.add_(1.0)
        with torch.cuda.stream(other if current else torch.cuda.default_stream()):
            head.round_table()
        torch.cuda.synchronize()
        assert torch.equal(head.table16, head.table.bfloat16()), k


def test_made_while_the_current_stream_works(G):
    """A head and an AdamW of a context on another stream, used right after they were made: what
    torch filled for them is there."""
    import torch
    from paper_2102_10424_amd.step import AdamW, TableHead
    side = torch.cuda.Stream()
    ctx = G.Context(0, stream=side.cuda_stream)
    table, W, dW = torch.randn(300, 24, device="cuda"), torch.ones(5000, device="cuda"), torch.ones(5000, device="cuda")
    ids, copy = torch.arange(300, dtype=torch.int32, device="cuda"), torch.empty(300, 24, device="cuda")
    torch.empty(1 << 22, device="cuda").fill_(float("nan"))      # what is allocated next is not zero
    torch.cuda.synchronize()
    for k in range(3):
        torch.cuda._sleep(20_000_000)      # some 10 ms
        opt = AdamW(ctx, [dict(W=W, dW=dW)])
        head = TableHead(ctx, table, dtype=torch.bfloat16)
        opt.step(0.0, 1)
        G.gist_embed_lookup(ctx, 300, 300, 24, head.table16, 24, G.GIST_STORE_BF16, ids, 1.0, copy, 24)
        torch.cuda.synchronize()
        m, v = opt.state[0]
        assert bool((m == 1 - torch.tensor(0.9).float().cuda()).all()) and bool((v > 0).all()), k
        assert torch.equal(copy, table.bfloat16().float()), k
