"""Rows of the class-table loss whose given class is far from the others, on either side, in bf16:
its logit is the reference of the exponentials that the gradients are made of."""

import numpy as np
import pytest

import more_ref as R
from gpu_util import log, to_dev, to_host
from test_gpu_table_xent import inputs, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    from paper_2102_10424_amd import gist
    return gist


@pytest.mark.parametrize("store,dtype", [("bf16", None), ("f32", "bf16"), ("f16", None), ("f32", "f32")])
@pytest.mark.parametrize("level", [-1, -40, -100, -200, 50, 200])
def test_class_out_of_the_question(G, store, dtype, level):
    """A class whose vector makes its logit no usable reference (-1e32; -3e4 times 64 in fp16),
    given in some rows, and all other logits about `level`: the gradients are finite, and right where
    that class is not concerned."""
    ctx = G.Context(0)
    rng = np.random.default_rng(abs(level))
    n, C, d = 300, 90, 64
    H, T, y = inputs(n, C, d, rng, 0.1)
    H[:, 0] = 1.0
    T[:, 0] = level / 0.7
    T[7, 0] = -3e4 if store == "f16" else -1e32
    y[5:280:11] = 7
    y[3] = 1
    out, Hv, Tv, _ = run(G, ctx, H, T, y, store, dtype)
    assert np.isfinite(out["dH"]).all() and np.isfinite(out["dT"]).all()
    scale = float(np.float32(0.7))
    r = R.table_xent(Hv, Tv, y, scale, 3.0)
    op = "bf16" if store == "f32" and dtype == "bf16" else store
    # the class has no probability: bounds without it, of the rows that are not its
    Tz = Tv.copy()
    Tz[7] = 0
    b = R.table_xent_bounds(Hv, Tz, y, scale, r, op, store)
    other = y != 7
    keep = np.arange(C) != 7
    for k, got, want, bound in (("lse", out["lse"], r["lse"], b["lse"]),
                                ("logp", out["logp"][other], r["logp"][other], b["logp"][other]),
                                ("dH", out["dH"][other], r["dH"][other], b["dH"][other]),
                                ("dT", out["dT"][keep], r["dT"][keep], b["dT"][keep])):
        assert (np.abs(got - want) <= bound).all(), (k, float(np.max(np.abs(got - want) / bound)))
    # its rows: (p - 1) is -1 but for rounding
    mine = y == 7
    assert (np.abs(out["logp"][mine] / r["logp"][mine] - 1) < 1e-5).all()
    assert (np.abs(out["dH"][mine, 0] / r["dH"][mine, 0] - 1) < 2.0 ** -7).all()
