"""Rotary positions over three axes, group norm with an activation over packed scans and rows in 8 bits, in float64 on
the CPU from their definitions, with the gradients in closed form and the error bounds that the GPU tests hold the
kernels to.

The bounds follow the kernels' roundings: inputs are exact, steps are float32 (half a unit, 2^-24, each), every output
is rounded once to its type (half a step of it)."""
import numpy as np

EPS = 2.0 ** -24
UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # half a step at 24, 8 and 11 bits
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -24}  # below it a type's values are absolute steps


# -- rotary positions ------------------------------------------------------------

def rope(x, coords, freqs, sections, halves=False, inverse=False):
    """x [n][heads][D], coords [n][4] whole numbers; the rotated rows and their error bounds but for the last rounding."""
    P = sum(sections)
    axis = [1 + a for a, s in enumerate(sections) for _ in range(s)]
    theta = np.clip(coords[:, axis], -32767, 32766).astype(np.float64) * freqs.astype(np.float64)
    c, s = np.cos(theta)[:, None], np.sin(theta)[:, None] * (-1.0 if inverse else 1.0)
    i = np.arange(P) if halves else 2 * np.arange(P)
    j = np.arange(P) + P if halves else 2 * np.arange(P) + 1
    y, e = x.copy(), np.zeros_like(x)
    u, w = x[..., i], x[..., j]
    y[..., i], y[..., j] = u * c - w * s, u * s + w * c
    # sine and cosine: an angle of at most pi / 4 rounded to float32, some steps of their sums, and theta's own
    # 2^-50; the rotation: two products and a sum
    own = 4 * EPS + 2.0 ** -50 * np.abs(theta)[:, None]
    e[..., i] = e[..., j] = (np.abs(u) + np.abs(w)) * (own + 2 * EPS)
    return y, e


def rounded(y, e, dtype):
    """The bound with the last rounding."""
    return e + UNIT[dtype] * (np.abs(y) + e) + TINY[dtype]


# -- rows in 8 bits ----------------------------------------------------------------

def codes(x, dtype):
    """(codes [m][C], exponent bytes [m][blocks], what is read back) of x [m][C]."""
    m, C = x.shape
    nb = (C + 31) // 32
    f = np.zeros((m, nb * 32))
    f[:, :C] = x
    f = f.reshape(m, nb, 32)
    ok = np.isfinite(f)
    top = np.where(ok, np.abs(f), 0.0).max(2, keepdims=True)
    _, k = np.frexp(top)  # top < 2^k
    e = np.where(top > 0, k - 7, -1000)
    e = np.maximum(e, -24 if dtype == "f16" else -126)
    q = np.clip(np.rint(np.ldexp(np.where(ok, f, 0.0), -e)), -127, 127)
    read = np.where(ok, np.ldexp(q, e), np.nan).reshape(m, nb * 32)[:, :C]
    return np.where(ok, q, -128).reshape(m, nb * 32)[:, :C].astype(np.int8), (e[..., 0] + 127).astype(np.uint8), read


def wgrad_bound(x, da, dW):
    """A sum over m rows in float32 steps of a workgroup's rows, at most 4096 of them in any order (twice that: products
    are added in groups whose own sums may be cut), then in 64 bits."""
    return EPS * (2 * min(len(x), 4096) + 16) * (np.abs(x).T @ np.abs(da)) + EPS * np.abs(dW)


# -- group norm ------------------------------------------------------------------

def act(z, kind):
    """(value, slope) of the activation."""
    if kind == "relu":
        return np.maximum(z, 0.0), (z > 0).astype(np.float64)
    if kind == "silu":
        s = 0.5 * (1.0 + np.tanh(0.5 * z))
        return z * s, s * (1.0 + z * (1.0 - s))
    return z, np.ones_like(z)


def group_norm(x, off, G, gamma, beta, eps, kind, dtype, dy=None, dres=None, saved=None):
    """x [m][C] float64: a dict of y, mu and r [B][G] and, with dy, dx, dgamma, dbeta (the rows' values there are
    `saved` where given), each with its bound under the name + "_tol".  Rows of no scan are NaN."""
    m, C = x.shape
    B, w, u = len(off) - 1, x.shape[1] // G, UNIT[dtype]
    R = dict(y=np.full(x.shape, np.nan), y_tol=np.zeros(x.shape), mu=np.zeros((B, G)), r=np.zeros((B, G)),
             mu_tol=np.zeros((B, G)), r_tol=np.zeros((B, G)))
    if dy is not None:
        R.update(dx=np.full(x.shape, np.nan), dx_tol=np.zeros(x.shape))
        for n in ("dgamma", "dbeta", "dgamma_tol", "dbeta_tol"):
            R[n] = np.zeros(C)
    for b in range(B):
        rows = slice(max(0, min(m, off[b])), max(0, min(m, off[b + 1])))
        n = rows.stop - rows.start
        if n <= 0:
            continue

        def grouped(t):
            return t[rows].reshape(n, G, w)

        def mean(t):
            return t.mean((0, 2), keepdims=True)
        X = grouped(x)
        mu = mean(X)
        var = mean((X - mu) ** 2)
        r = 1.0 / np.sqrt(var + eps)
        # a lane's running mean takes a rounding or three a row, of at most 1024 rows; what joins them is in 64 bits
        steps = 3 * min(n, 1024) + 16
        e_mu = EPS * steps * np.abs(X).max((0, 2), keepdims=True)
        rel_r = EPS * steps + (e_mu * r) ** 2  # of r: half of the variance's
        R["mu"][b], R["r"][b] = mu.ravel(), r.ravel()
        R["mu_tol"][b], R["r_tol"][b] = e_mu.ravel(), (r * rel_r).ravel()
        ga, be = gamma.reshape(1, G, w), beta.reshape(1, G, w)

        def normed(t):
            xh = (t - mu) * r
            e_xh = r * (e_mu + EPS * np.abs(t - mu)) + np.abs(xh) * (rel_r + 2 * EPS)
            z = xh * ga + be
            return xh, e_xh, z, np.abs(ga) * e_xh + EPS * (2 * np.abs(xh * ga) + np.abs(be) + np.abs(z))
        xh, e_xh, z, e_z = normed(X)
        y, _ = act(z, kind)
        # the activations' slopes are at most 1.1; the exponential's argument in float32, 16 bits' at their size
        e_y = 1.1 * e_z + np.abs(y) * EPS * (8 + 2 * np.abs(z)) * (kind == "silu")
        R["y"][rows] = y.reshape(n, C)
        R["y_tol"][rows] = (e_y + u * (np.abs(y) + e_y) + TINY[dtype]).reshape(n, C)
        if dy is None:
            continue
        if saved is not None:
            xh, e_xh, z, e_z = normed(grouped(saved))
        dY = grouped(dy)
        _, slope = act(z, kind)
        gz = dY * slope
        e_gz = np.abs(dY) * ((0.5 * e_z + EPS * (8 + 2 * np.abs(z))) if kind == "silu" else 0.0) + EPS * np.abs(gz)
        if kind == "relu":  # z's sign is not known within its error
            e_gz = e_gz + np.abs(dY) * (np.abs(z) <= e_z)
        h, e_h = gz * ga, np.abs(ga) * e_gz + EPS * np.abs(gz * ga)
        m1, m2 = mean(h), mean(h * xh)
        e_m1 = mean(e_h) + EPS * steps * mean(np.abs(h))
        e_m2 = mean(e_h * np.abs(xh) + np.abs(h) * e_xh) + EPS * steps * mean(np.abs(h * xh))
        d = r * (h - m1 - xh * m2)
        e_d = r * (e_h + e_m1 + e_xh * np.abs(m2) + np.abs(xh) * e_m2 +
                   4 * EPS * (np.abs(h) + np.abs(m1) + np.abs(xh * m2))) + np.abs(d) * (rel_r + EPS)
        if dres is not None:
            d = d + grouped(dres)
            e_d = e_d + EPS * np.abs(d)
        R["dx"][rows] = d.reshape(n, C)
        R["dx_tol"][rows] = (e_d + u * (np.abs(d) + e_d) + TINY[dtype]).reshape(n, C)

        def cols(t):
            return t.sum(0).reshape(C)
        R["dgamma"] += cols(gz * xh)
        R["dbeta"] += cols(gz)
        R["dgamma_tol"] += cols(e_gz * np.abs(xh) + np.abs(gz) * e_xh + EPS * steps * np.abs(gz * xh))
        R["dbeta_tol"] += cols(e_gz + EPS * steps * np.abs(gz))
    if dy is not None:
        for n in ("dgamma", "dbeta"):
            R[n + "_tol"] += EPS * np.abs(R[n]) + TINY["f32"]
    return R
