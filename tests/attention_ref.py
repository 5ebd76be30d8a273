"""Layer norm and attention over packed scans in float64 on the CPU, from their definitions, with the gradients
in closed form, and the error bounds that the GPU tests hold the kernels to.

The bounds follow the kernels' roundings: inputs are exact, products and sums are float32 (unit 2^-24 a step),
the softmax weights and the scores' gradients are rounded to the storage type before they are multiplied
(unit u), and every output is rounded to it once."""
import numpy as np

EPS = 2.0 ** -24
UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # half a step at 24, 8 and 11 bits
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -24}  # below it a type's values are absolute steps


# -- layer norm ----------------------------------------------------------------

def norm(x, gamma, beta, eps):
    mu = x.mean(1, keepdims=True)
    r = 1.0 / np.sqrt(((x - mu) ** 2).mean(1, keepdims=True) + eps)
    return (x - mu) * r, r, (x - mu) * r * gamma + beta


def norm_backward(dy, x, gamma, eps, dres=None):
    xh, r, _ = norm(x, gamma, 0.0, eps)
    h = dy * gamma
    dx = r * (h - h.mean(1, keepdims=True) - xh * (h * xh).mean(1, keepdims=True))
    return dx + (0.0 if dres is None else dres), (dy * xh).sum(0), dy.sum(0)


def norm_bounds(dy, x, gamma, beta, eps, dres, dtype):
    """(y, dx, dgamma, dbeta): a mean of C float32 terms is off by at most (C / 64 + 8) roundings of the
    largest |x| on the way through 64 lanes, and xh by that, over the deviation, plus its own steps."""
    u, C = UNIT[dtype], x.shape[1]
    xh, r, y = norm(x, gamma, beta, eps)
    steps = C / 64 + 12
    e_xh = EPS * steps * (r * np.abs(x).max(1, keepdims=True) + np.abs(xh).max(1, keepdims=True) + 1.0)
    b_y = u * np.abs(y) + 2 * (np.abs(gamma) * e_xh + EPS * (np.abs(gamma * xh) + np.abs(beta))) + TINY[dtype]
    h = dy * gamma
    dx, dg, db = norm_backward(dy, x, gamma, eps, dres)
    hm, xm = np.abs(h).max(1, keepdims=True), np.abs(xh).max(1, keepdims=True)
    # d(r) / r is at most e_xh * |xh| on average; every product of dx sees it once or twice
    e_dx = r * (EPS * steps * hm * (1 + xm * xm) + 4 * e_xh * hm * (1 + xm))
    b_dx = u * np.abs(dx) + 2 * e_dx + 4 * EPS * np.abs(0.0 if dres is None else dres) + TINY[dtype]
    # column sums: float32 within a workgroup's rows, in 64 bits beyond: at most the rows' count of roundings
    n = min(len(x), 512) + 8
    b_dg = (np.abs(dy) * (2 * e_xh + EPS * n * np.abs(xh))).sum(0) + EPS * np.abs(dg)
    b_db = (EPS * n * np.abs(dy)).sum(0) + EPS * np.abs(db)
    return b_y, b_dx, b_dg, b_db


# -- attention -------------------------------------------------------------------

def attention(q, k, v, q_off, k_off, scale, cap=0.0, qc=None, kc=None, slopes=None, dout=None, dtype="f32"):
    """q [nq][H][D], k, v [nk][K][D] float64, coordinates [n][4].  A dict of out, lse and, with dout, dq, dk, dv,
    each with its error bound under the name + "_tol"; rows of no scan are NaN."""
    nq, H, D = q.shape
    nk, K, _ = k.shape
    u = UNIT[dtype]
    up = u if dtype != "f32" else EPS
    R = dict(out=np.full(q.shape, np.nan), lse=np.full((nq, H), np.nan))
    if dout is not None:
        R.update(dq=np.full(q.shape, np.nan), dk=np.full(k.shape, np.nan), dv=np.full(v.shape, np.nan))
    for n in list(R):
        R[n + "_tol"] = np.zeros(R[n].shape)
    for b in range(len(q_off) - 1):
        i, j = slice(q_off[b], q_off[b + 1]), slice(k_off[b], k_off[b + 1])
        if dout is not None:
            for n in ("dk", "dv", "dk_tol", "dv_tol"):
                R[n][j] = 0.0
        if i.start == i.stop:
            continue
        if j.start == j.stop:
            R["out"][i], R["lse"][i] = 0.0, -np.inf
            if dout is not None:
                R["dq"][i] = 0.0
            continue
        dist = 0.0
        if slopes is not None:
            dist = np.abs(qc[i, None, 1:].astype(np.float64) - kc[None, j, 1:]).sum(-1)
        for h in range(H):
            g = h // (H // K)
            Q, Kk, V = q[i, h], k[j, g], v[j, g]
            z = scale * (Q @ Kk.T)
            t = cap * np.tanh(z / cap) if cap else z
            sl = 0.0 if slopes is None else slopes[h]
            s = t - sl * dist
            m = s.max(1, keepdims=True)
            lse = m + np.log(np.exp(s - m).sum(1, keepdims=True))
            p = np.exp(s - lse)
            o = p @ V
            # a score's absolute error: the product's D steps, the cap's and the bias's own, the maximum and lse
            ds_ = EPS * ((D + 8) * scale * (np.abs(Q) @ np.abs(Kk).T) + 8 * (cap + np.abs(sl) * dist + np.abs(m) +
                                                                            np.abs(lse)) + 16)
            ep = up + 2 * ds_ + EPS * (len(V) / 16 + 64)  # relative error of a weight, sums of many among it
            pl = p + TINY[dtype]
            R["out"][i, h], R["lse"][i, h] = o, lse[:, 0]
            R["out_tol"][i, h] = 2 * ((pl * ep) @ np.abs(V)) + u * np.abs(o) + TINY[dtype]
            R["lse_tol"][i, h] = 2 * ((p * ds_).sum(1) + (up + EPS * (len(V) / 16 + 64)) + EPS * np.abs(lse[:, 0]))
            if dout is None:
                continue
            dO = dout[i, h]
            dp = dO @ V.T
            delta = (dO * o).sum(1, keepdims=True)
            bend = 1 - np.tanh(z / cap) ** 2 if cap else np.ones_like(z)
            dz = p * (dp - delta) * bend
            R["dv"][j, g] += p.T @ dO
            R["dq"][i, h] = scale * (dz @ Kk)
            R["dk"][j, g] += scale * (dz.T @ Q)
            # delta is formed from the rounded out; dp and delta are sums of D products
            e_o = R["out_tol"][i, h]
            e_d = (np.abs(dO) * (e_o + EPS * (D + 8) * np.abs(o))).sum(1, keepdims=True)
            e_z = np.abs(dz) * (ep + 8 * EPS) + pl * bend * (e_d + EPS * (D + 8) * (np.abs(dO) @ np.abs(V).T)) + \
                p * np.abs(dp - delta) * (16 * EPS + 2 * ds_ / max(cap, 1e-30) * (cap > 0)) + TINY[dtype]
            R["dv_tol"][j, g] += 2 * (pl * ep).T @ np.abs(dO)
            R["dq_tol"][i, h] = 2 * scale * (e_z @ np.abs(Kk))
            R["dk_tol"][j, g] += 2 * scale * (e_z.T @ np.abs(Q))
    if dout is not None:
        for n in ("dq", "dk", "dv"):
            R[n + "_tol"] += u * np.abs(np.nan_to_num(R[n])) + TINY[dtype] + EPS * R[n + "_tol"]
    return R
