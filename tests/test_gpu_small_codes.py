"""8-bit codes below 2^-6, whose steps are all 2^-9: nearest even as the larger ones, on either side
of a middle and on it."""

import numpy as np
import pytest

import more_ref as R
from gpu_util import to_host

pytestmark = pytest.mark.gpu
EPS = float(np.float32(1e-6))


@pytest.fixture(scope="module")
def G():
    from paper_2102_10424_amd import gist
    return gist


SHAPES = [(80000, 40), (30000, 130), (2000, 2047), (1000, 4099), (1500, 2048), (250, 16001), (100, 40001)]


def wanted(v):
    """Nearest codes of 64-bit rows, their largest magnitude at 448."""
    v = to_host(v)
    a = v * (R.TOP / np.abs(v).max(1, keepdims=True))
    want = R.e4m3(a)
    assert (np.abs(a) < 2.0 ** -6).mean() > 0.9      # what is tested
    return want


@pytest.mark.parametrize("n,d", SHAPES)
@pytest.mark.parametrize("store", ["f32", "bf16", "f16"])
def test_small_codes_are_exact(G, n, d, store):
    """Rows of which all but one element are small: every code is that of exact arithmetic."""
    import torch
    ctx = G.Context(0)
    torch.manual_seed(d)
    t = R.torch_type(store)
    x = (2 * torch.rand(n, d, device="cuda") - 1) * 2.0 ** -6 / 448
    x[:, d // 3] = 1 + torch.rand(n, device="cuda")
    x = (x * 8).to(t)
    gain = 1 + 0.01 * torch.rand(d, device="cuda")
    y, s = torch.empty(n, d, dtype=torch.uint8, device="cuda"), torch.empty(n, device="cuda")
    st = R.store_of(G, store)
    value = lambda: to_host(y.view(torch.float8_e4m3fn).double())
    G.gist_quantize_rows(ctx, n, d, x, d, st, y, d, s)
    assert np.array_equal(value(), wanted(x.double()))
    G.gist_rms_norm(ctx, n, d, x, d, None, d, st, gain, EPS, None, d, y, d, G.GIST_STORE_E4M3, s, None)
    assert np.array_equal(value(), wanted(x.double() * gain.double()))


@pytest.mark.parametrize("d", [16, 449, 2000, 9000, 40000])
@pytest.mark.parametrize("power", [0, -11, 30])
def test_small_codes_of_exact_middles(G, d, power):
    """Multiples of 2^-10 up to 2^-5 beside a 448 (times a power of two): half of them lie in the
    middle between two codes, and go to the even one."""
    import torch
    ctx = G.Context(0)
    torch.manual_seed(d)
    x = torch.randint(-32, 33, (20, d), device="cuda").float() * 2.0 ** -10
    x[:, d // 2] = 448
    y, s = torch.empty(20, d, dtype=torch.uint8, device="cuda"), torch.empty(20, device="cuda")
    G.gist_quantize_rows(ctx, 20, d, x * 2.0 ** power, d, G.GIST_STORE_F32, y, d, s)
    a = to_host(x.double())
    assert np.array_equal(to_host(y.view(torch.float8_e4m3fn).double()), R.e4m3(a)) and bool((s == 2.0 ** power).all())
