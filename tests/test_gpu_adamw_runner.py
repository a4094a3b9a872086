"""AdamW as a runner with a head steps it: several steps in a row, each against the 64-bit update of
the weights, gradients and moments that were there before it, the 8-bit ones code by code."""

import numpy as np
import pytest

import more_ref as R
from gpu_util import to_host
from test_gpu_table_head import runner, setup

pytestmark = pytest.mark.gpu
LR, BETAS, EPS = 1e-2, (0.9, 0.999), 1e-8


@pytest.fixture(scope="module")
def G():
    from paper_2102_10424_amd import gist
    return gist


def moments(st, eight):
    """m, v in 64 bits as they are stored (8 bits: codes, scales; sqrt v)."""
    import torch
    if not eight:
        return [to_host(t).astype(np.float64) for t in st]
    q = [to_host(t.view(torch.float8_e4m3fn).float()).astype(np.float64) for t in st[:2]]
    s = [np.repeat(to_host(t).astype(np.float64), 256)[:len(q[0])] for t in st[2:]]
    return q[0] * s[0], (q[1] * s[1]) ** 2


@pytest.mark.parametrize("kind", ["gcn", "sage", "gat"])
@pytest.mark.parametrize("eight", [False, True])
def test_steps(G, kind, eight):
    import torch
    ctx = G.Context(0)
    b, run, params, head = runner(G, ctx, kind, setup(kind, 13), torch.bfloat16)
    opt = run.adamw(params, head, weight_decay=0.1, eight=eight)
    decays = [0.1] * 2 if kind != "gat" else [0.1, 0, 0.1, 0]
    loss = torch.zeros(1, device="cuda")
    for k in range(1, 5):
        before = [(to_host(W).ravel().astype(np.float64), *moments(st, eight))
                  for (W, _, _), st in zip(opt._keep, opt.state)]
        run.step(b, params, LR, adamw=(opt, k), head=head, residual=b.X, loss_out=loss)
        for i, ((W, dW, _), st, wd, (w0, m0, v0)) in enumerate(zip(opt._keep, opt.state, decays + [0.1, 0], before)):
            g = to_host(dW.float()).ravel()
            assert np.abs(g).max() > 0
            w, m, v, bW, bm, bv = R.adamw(w0, g, m0, v0, LR, k, *BETAS, EPS, wd, 1.0)
            # 8-bit moments are read as code times scale: one more rounding, squared for v
            assert (np.abs(to_host(W).ravel() - w) <= bW * (2 if eight else 1)).all(), (k, i)
            if not eight:
                assert (np.abs(to_host(st[0]) - m) <= bm).all() and (np.abs(to_host(st[1]) - v) <= bv).all()
                continue
            bits = R.random_bits(len(g), i + 1, k)
            code = lambda t: to_host(t.view(torch.float8_e4m3fn).float())
            R.check_codes(code(st[0]), to_host(st[2]), m, bits[0], False, bm + R.U32 * np.abs(m0))
            root = np.sqrt(v)
            R.check_codes(code(st[1]), to_host(st[3]), root, bits[1], True,
                          (bv + 3 * R.U32 * v0) / (2 * np.maximum(root, 1e-300)) + R.U32 * root)
        assert torch.equal(head.table16, head.table.bfloat16())
