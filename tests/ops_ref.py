"""64-bit references of the learned rows, the log probabilities and the
orthogonalised update, and the rounding bounds their tests hold the library to.

u = 2^-24 is half a unit in the last place of fp32, relative to the value."""

import numpy as np

U32 = 2.0 ** -24
HALF = dict(f32=2.0 ** -24, bf16=2.0 ** -8, f16=2.0 ** -11)   # relative rounding of a store


def store_of(G, name):
    return dict(f32=G.GIST_STORE_F32, bf16=G.GIST_STORE_BF16, f16=G.GIST_STORE_F16)[name]


def torch_type(name):
    import torch
    return dict(f32=torch.float32, bf16=torch.bfloat16, f16=torch.float16)[name]


# ---- learned rows ----------------------------------------------------------------
def embed_grad(ids, V, dY, scale):
    """(gradient, bound): a row of k terms takes k - 1 additions in any order and one
    product, each rounding relative to a partial sum of magnitudes."""
    dY = np.asarray(dY, dtype=np.float64)
    g, mag = np.zeros((V, dY.shape[1])), np.zeros((V, dY.shape[1]))
    k = np.zeros(V)
    ok = (ids >= 0) & (ids < V)
    np.add.at(g, ids[ok], dY[ok])
    np.add.at(mag, ids[ok], np.abs(dY[ok]))
    np.add.at(k, ids[ok], 1.0)
    return scale * g, (k[:, None] + 1) * U32 * abs(scale) * mag


# ---- log probabilities ---------------------------------------------------------------
def log_probs(z, y):
    """lse, logp, entropy in 64 bits, by the documented rules for masked rows, missing
    tokens and non-finite logits."""
    z = np.asarray(z, dtype=np.float64)
    n, C = z.shape
    bad = np.isnan(z).any(1) | (z == np.inf).any(1)
    lse, logp, H = np.empty(n), np.zeros(n), np.empty(n)
    for v in range(n):
        if bad[v]:
            lse[v] = logp[v] = H[v] = np.nan
            continue
        m = z[v].max()
        if m == -np.inf:
            lse[v], H[v] = -np.inf, 0.0
        else:
            x = z[v] - m
            e = np.exp(x)
            S = e.sum()
            lse[v] = m + np.log(S)
            keep = e > 0
            H[v] = np.log(S) - (e[keep] * x[keep]).sum() / S
        if y is not None and y[v] >= 0:
            if y[v] >= C:
                logp[v] = np.nan
            else:
                zy = z[v, y[v]]
                logp[v] = -np.inf if zy == -np.inf else zy - lse[v]
    return lse, logp, H


def top_classes(z, K):
    """The K best classes: value descending, then class ascending; -1 in a row holding NaN
    or +Inf."""
    z = np.asarray(z, dtype=np.float64)
    out = np.empty((z.shape[0], K), dtype=np.int32)
    for v in range(z.shape[0]):
        if np.isnan(z[v]).any() or (z[v] == np.inf).any():
            out[v] = -1
        else:
            out[v] = np.argsort(-z[v], kind="stable")[:K]
    return out


def lse_bound(z):
    """Error of a row's log-sum-exp.  With y = (z - m) log2 e: the terms' relative errors
    are 3 u |y| ln 2 (y's two roundings, log2 e's) + 2 u (the exponential's unit), at most 4 u
    after weighting with 2^y (2^y |y| <= 0.54); the sum adds a rounding per addition of a thread
    (C / 64 at most) and 20 for the joins; log2 and the final fma 2 u each of their value."""
    z = np.asarray(z, dtype=np.float64)
    C = z.shape[1]
    m = np.max(np.where(np.isfinite(z), z, -1e4), axis=1)
    return U32 * (C / 64 + 28 + 4 * np.log2(C + 1) + 4 * np.abs(m))


def entropy_bound(z):
    """log s as above without the maximum; t = sum 2^y y has the same relative errors on
    each term, whose magnitudes over s sum to at most log2 C + 1."""
    C = np.asarray(z).shape[1]
    return U32 * (C / 64 + 32) * (3 * np.log2(C + 1) + 4)


def log_probs_grad(z, y, gl, gh):
    """Gradient of sum(gl logp + gh entropy) in 64 bits."""
    z = np.asarray(z, dtype=np.float64)
    n, C = z.shape
    lse, _, H = log_probs(z, None)
    d = np.zeros((n, C))
    for v in range(n):
        if np.isnan(lse[v]) or (y is not None and y[v] >= C and gl is not None):
            d[v] = np.nan
            continue
        if lse[v] == -np.inf:
            continue
        with np.errstate(invalid="ignore"):
            lp = z[v] - lse[v]
        p = np.exp(lp)
        lp = np.where(p > 0, lp, 0.0)
        has = gl is not None and y[v] >= 0
        a = gl[v] if has else 0.0
        b = gh[v] if gh is not None else 0.0
        d[v] = -p * (a + b * (lp + H[v]))
        if has:
            d[v, y[v]] += a
    return d


def grad_bound(z, y, gl, gh, store):
    """p = exp(x), x = z - lse: relative error lse_bound + u (|x| + |x| + 4), and the
    weight a + b (x + H) takes three roundings of its terms' magnitudes and lse_bound and
    entropy_bound of b; then one rounding to the store (fp16: at least half its smallest
    step, 2^-25)."""
    z = np.asarray(z, dtype=np.float64)
    n, C = z.shape
    lse, _, H = log_probs(z, None)
    lb, eb = lse_bound(z)[:, None], entropy_bound(z)
    with np.errstate(invalid="ignore"):
        x = np.where(np.isfinite(z), z - lse[:, None], 0.0)
        p = np.where(np.isfinite(z), np.exp(x), 0.0)
    a = np.abs(gl)[:, None] if gl is not None else 0.0
    b = np.abs(gh)[:, None] if gh is not None else 0.0
    w = a + b * (np.abs(x) + H[:, None])
    e = p * (w * (lb + U32 * (2 * np.abs(x) + 10)) + b * (lb + eb)) + U32 * 2 * a
    d = np.abs(log_probs_grad(z, y, gl, gh))
    return e + HALF[store] * (d + e) + (2.0 ** -25 if store == "f16" else 0.0)


# ---- orthogonalised update -----------------------------------------------------------
COEF = (3.4445, -4.7750, 2.0315)


def polynomial(s, steps, coef):
    a, b, c = coef
    for _ in range(steps):
        s = a * s + b * s ** 3 + c * s ** 5
    return s


def orthogonal(Umat, steps=5, coef=COEF, eps=1e-7):
    """The factor by its singular values: P f(S / norm) Q^T."""
    Umat = np.asarray(Umat, dtype=np.float64)
    coef = tuple(float(np.float32(x)) for x in coef)
    norm = np.sqrt((Umat ** 2).sum())
    p, s, qt = np.linalg.svd(Umat, full_matrices=False)
    return (p * polynomial(s / max(norm, eps), steps, coef)) @ qt


def orthogonal_noisy(Umat, rel, absolute, rng, steps=5, coef=COEF, eps=1e-7):
    """The iteration in 64 bits with every stored matrix (X, A, B) rounded like the
    library's: a uniform relative error of up to ``rel`` and an absolute one up to
    ``absolute`` on each entry."""
    a, b, c = coef

    def noise(t):
        return t * (1 + rel * rng.uniform(-1, 1, t.shape)) + absolute * rng.uniform(-1, 1, t.shape)

    Umat = np.asarray(Umat, dtype=np.float64)
    flip = Umat.shape[0] > Umat.shape[1]
    X = Umat.T if flip else Umat
    X = noise(X / max(np.sqrt((X ** 2).sum()), eps))
    for _ in range(steps):
        A = X @ X.T
        A = noise((A + A.T) / 2)
        B = b * A + c * (A @ A)
        B = noise((B + B.T) / 2)
        X = noise(a * X + B @ X)
    return X.T if flip else X


def muon_tolerance(Umat, dtype, steps=5, coef=COEF, seed=0):
    """2-norm bound of the factor's error: what roundings of the library's size do to the
    64-bit iteration, largest of three runs, times 4 (the runs' own spread, and the fp32
    sums of the products).  Two fp16 parts leave 2^-22 relative and 2^-25 / 2^12 absolute
    (the lowest part's smallest step, halved, unscaled), and a dropped lo lo' term and fp32
    sums of the same order; one part 2^-11 and 2^-37."""
    rel = 2.0 ** -22 if dtype == "f32" else 2.0 ** -11
    rng = np.random.default_rng(seed)
    want = orthogonal(Umat, steps, coef)
    return 4 * max(np.linalg.norm(orthogonal_noisy(Umat, rel, 2.0 ** -37, rng, steps, coef) - want)
                   for _ in range(3))
