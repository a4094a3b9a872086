"""64-bit references of the root-mean-square norm, the loss against a class table and the
AdamW step, and the rounding bounds their tests hold the library to.

u = 2^-24 is half a unit in the last place of fp32, relative to the value; HALF the same for
every store."""

import numpy as np

from ops_ref import HALF, U32, lse_bound

TOP = 448.0          # largest e4m3 value


def torch_type(name):
    import torch
    return dict(f32=torch.float32, bf16=torch.bfloat16, f16=torch.float16,
                e4m3=torch.float8_e4m3fn)[name]


def store_of(G, name):
    return dict(f32=G.GIST_STORE_F32, bf16=G.GIST_STORE_BF16, f16=G.GIST_STORE_F16,
                e4m3=G.GIST_STORE_E4M3)[name]


def e4m3(a):
    """Nearest e4m3 value (ties to even) of 64-bit values of at most 448."""
    _, e = np.frexp(np.abs(a))
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.rint(a / step) * step


def step_of(a):
    """Distance of e4m3 values around a."""
    _, e = np.frexp(np.abs(a))
    return np.ldexp(1.0, np.maximum(e - 1, -6) - 3)


# ---- root-mean-square norm ---------------------------------------------------------
def rms(h, gain, eps):
    """(rstd, y) of rows h in 64 bits."""
    h = np.asarray(h, np.float64)
    rstd = 1 / np.sqrt((h * h).mean(1) + eps)
    return rstd, h * rstd[:, None] * np.asarray(gain, np.float64)


def chain(d):
    """Additions a term of a row's sum meets: at most 32 in its thread (or one per 1,024 values of a
    long row), the lanes', the waves' and the mean's product."""
    return 32 + d / 256 + 24


def rstd_rel(d):
    """The sum's relative error halves under the root; eps, root and quotient add 3 u."""
    return U32 * (chain(d) / 2 + 4)


def rms_bound(h, gain, eps, out):
    rstd, y = rms(h, gain, eps)
    e = np.abs(y) * (rstd_rel(h.shape[1]) + 2 * U32)
    # fp16's smallest step is 2^-24
    return e + HALF[out] * (np.abs(y) + e) + (2.0 ** -25 if out == "f16" else 0.0)


def rms_grad(dy, h, gain, eps, dsum):
    """dx, dgain and their bounds (fp32, before dx is rounded to its store)."""
    dy, h, gain = (np.asarray(t, np.float64) for t in (dy, h, gain))
    n, d = h.shape
    rstd, _ = rms(h, np.ones(d), eps)
    m = h * rstd[:, None]
    u = dy * gain
    dx = rstd[:, None] * (u - m * (u * m).mean(1, keepdims=True))
    r = rstd_rel(d)
    mag = rstd[:, None] * (np.abs(u) + np.abs(m) * np.abs(u * m).mean(1, keepdims=True))
    # m carries r, its product with the dot (three roundings, the dot's own chain) twice r more
    bx = mag * (4 * r + U32 * (chain(d) + 10))
    if dsum is not None:
        dx = dx + dsum
        bx = bx + 2 * U32 * (np.abs(dsum) + np.abs(dx))
    dg = (dy * m).sum(0)
    # a workgroup's rows one after another (n / 1,024 of them, or the waves of 4), then 1,024 sums
    bg = np.abs(dy * m).sum(0) * (r + U32 * (n / 1024 + 1024 / 16 + 40))
    return dx, bx, dg, bg


# ---- loss against a class table ------------------------------------------------------
def table_xent(H, T, y, scale, gscale, n_valid=None):
    """loss, logp, lse, G (n x C), dH, dT in 64 bits; rows without a label give zeros, whatever
    they hold."""
    H, T = np.asarray(H, np.float64), np.asarray(T, np.float64)
    n, C = H.shape[0], T.shape[0]
    nv = n if n_valid is None else min(max(n_valid, 0), n)
    real = (y >= 0) & (np.arange(n) < nv)
    with np.errstate(all="ignore"):
        z = scale * (H @ T.T)
        m = z.max(1, keepdims=True)
        lse = (m + np.log(np.exp(z - m).sum(1, keepdims=True)))[:, 0]
    logp = np.zeros(n)
    G = np.zeros((n, C))
    for v in np.flatnonzero(real):
        logp[v] = np.nan if y[v] >= C else z[v, y[v]] - lse[v]
        G[v] = np.exp(z[v] - lse[v])
        if y[v] < C:
            G[v, y[v]] -= 1.0
    count = int(real.sum())
    f = gscale * scale / count if count else 0.0
    loss = -logp[real].sum() / count if count else 0.0
    Hz = np.where(real[:, None], H, 0.0)
    return dict(loss=loss, logp=logp, lse=lse, z=z, G=G, f=f, dH=f * (G @ T), dT=f * (G.T @ Hz),
                real=real, Hz=Hz)


def table_xent_bounds(H, T, y, scale, r, op, store):
    """Bounds of lse, logp, loss, dH and dT.  op: the products' operands; store: the gradients'.

    A logit: products of two 16-bit values are exact in fp32 (those of fp32 values carry 2^-22
    each), every one of d additions loses at most 2 u (a matrix instruction may cut instead of
    rounding) of the terms' magnitudes.  8-bit values are widened exactly; their scales are
    fp32 factors (2 u more)."""
    H, T = np.asarray(H, np.float64), np.asarray(T, np.float64)
    n, C, d = H.shape[0], T.shape[0], H.shape[1]
    mag = abs(scale) * (np.abs(H) @ np.abs(T).T)
    ez = mag * 2 * U32 * (d + 16)
    lse = ez.max(1) + lse_bound(r["z"]) + 4 * U32 * np.abs(r["lse"])
    yy = np.clip(y, 0, C - 1)
    at = np.arange(n)
    logp = ez[at, yy] + lse + 4 * U32 * (np.abs(r["z"][at, yy]) + np.abs(r["lse"]))
    loss = (logp[r["real"]].mean() if r["real"].any() else 0.0) + 4 * U32 * abs(r["loss"])
    if op == "e4m3":      # no gradients
        return dict(lse=lse, logp=logp, loss=loss)
    p = np.where(r["real"][:, None], np.exp(np.minimum(r["z"] - r["lse"][:, None], 0.0)), 0.0)
    eg = p * (ez + lse[:, None] + U32 * (np.abs(r["z"] - r["lse"][:, None]) + 6)) + U32 * np.abs(r["G"])
    # bf16: e^(z - r) e^(r - lse), r about the given class's logit
    eg = eg + p * U32 * 2 * (np.abs(r["z"][at, yy] - r["lse"])[:, None] + 4)
    # G's rounding: fp16 holds it times 2^15
    eg = eg + HALF[op] * (np.abs(r["G"]) + eg) + (2.0 ** -25 / 32768 if op == "f16" else 0.0)
    f = abs(r["f"])
    # an exponential below 2^-126, fp32's least normal number, is zero; so is its product with f
    eg = eg + 2.0 ** -126 * (1 + 1 / max(f, 2.0 ** -60))
    aG = np.abs(r["G"]) + eg
    out = {}
    for name, a, b, k in (("dH", aG, np.abs(T), C), ("dT", aG.T, np.abs(r["Hz"]), n)):
        # dT in bf16: the rows of H times their factors are rounded as well
        more = HALF[op] * (a @ b) if name == "dT" and op == "bf16" else 0.0
        e = f * (more + (eg if name == "dH" else eg.T) @ b + 2 * U32 * (k + 24) * (a @ b)) + 2.0 ** -126
        out[name] = e + HALF[store] * (np.abs(r[name]) + e) + (2.0 ** -25 if store == "f16" else 0.0)
    return dict(lse=lse, logp=logp, loss=loss, **out)


# ---- AdamW --------------------------------------------------------------------------
def mix(x):
    x = np.asarray(x, np.uint64) & 0xffffffff
    x ^= x >> np.uint64(16)
    x = (x * np.uint64(0x7feb352d)) & np.uint64(0xffffffff)
    x ^= x >> np.uint64(15)
    x = (x * np.uint64(0x846ca68b)) & np.uint64(0xffffffff)
    return x ^ (x >> np.uint64(16))


def random_bits(n, place, seed):
    """(bits of m, bits of sqrt v) of a tensor's n elements; place counts from 1."""
    key = int(mix((seed ^ (place * 0x9e3779b9)) & 0xffffffff))
    h = mix((np.arange(n, dtype=np.uint64) + np.uint64(key)) & np.uint64(0xffffffff))
    return (h >> np.uint64(16)).astype(np.int64), (h & np.uint64(0xffff)).astype(np.int64)


def adamw(W, g, m, v, lr, k, b1, b2, eps, wd, gscale):
    """One step in 64 bits: W, m, v and the bounds of their rounding."""
    f = lambda t: np.asarray(t, np.float64)
    b1, b2, lr, eps, wd, gscale = (float(np.float32(t)) for t in (b1, b2, lr, eps, wd, gscale))
    W, g, m, v = f(W), f(g) * gscale, f(m), f(v)
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    bm = 4 * U32 * (np.abs(b1 * m) + np.abs((1 - b1) * g))
    bv = 6 * U32 * v1
    upd = lr / (1 - b1 ** k) * m1 / (np.sqrt(v1 / (1 - b2 ** k)) + eps)
    W1 = (1 - lr * wd) * W - upd
    scale = lr / (1 - b1 ** k) / (np.sqrt(v1 / (1 - b2 ** k)) + eps)
    bW = U32 * (4 * np.abs(W) + np.abs(W1) + 14 * np.abs(upd)) + scale * bm
    return W1, m1, v1, bW, bm, bv


def check_codes(codes, scales, x, bits, root, err):
    """8-bit blocks against 64-bit values x that the library has to within err: scales to 8 u,
    every code x / step + r rounded down, or its neighbour where that lies within its error of
    a whole number.  The error of t = x (448 / top) / step + r: x's own, err (448 / top) / step (where
    a sum cancels it is many u of x); the quotient, product and top's u each, 4 u of a / step;
    and the addition of r, u of at most 17."""
    n = len(x)
    nb = -(-n // 256)
    blocks = lambda t: np.pad(np.asarray(t, np.float64), (0, 256 * nb - n)).reshape(nb, 256)
    xb, q, bits = blocks(x), blocks(codes), blocks(bits)
    top = np.abs(xb).max(1)
    zero = top < 2.0 ** -100
    assert (scales[zero] == 0).all() and (q[zero] == 0).all()
    err = blocks(err)[~zero]
    xb, q, bits, top = xb[~zero], q[~zero], bits[~zero], top[~zero]
    assert (np.abs(scales[~zero] * TOP - top) <= 8 * U32 * top).all()
    a = np.abs(xb) * (TOP / top)[:, None]
    step = step_of(a)
    t = a / step + bits / 65536.0
    k = np.floor(t)
    if root:
        k = np.where((k == 0) & (xb > 0), 1, k)
    near = np.abs(t - np.rint(t)) <= (err * (TOP / top)[:, None] + 8 * U32 * a) / step + 17 * U32
    # at a power of two the fp32 value may lie on the other side, where the step is another
    e = np.log2(np.maximum(a, 1e-300))
    edge = np.abs(e - np.rint(e)) < 1e-5
    off = np.abs(np.abs(q) - k * step)
    ok = (off == 0) | ((near | edge) & (off <= step))
    assert ok.all(), (np.argwhere(~ok)[:5], q[~ok][:5], (k * step)[~ok][:5])
    assert (np.sign(q) * np.sign(xb) >= 0).all()
