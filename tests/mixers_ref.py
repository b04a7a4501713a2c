"""The token mixers in 64 bits, from their formulas (numpy, no library code), with
the magnitudes that the tests' error bounds are made of."""
import numpy as np


def bf16(a):
    """Rounded to bf16 (to nearest even), as float64."""
    u = np.ascontiguousarray(a, dtype=np.float32).view(np.uint32).astype(np.uint64)
    u = (u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000
    return u.astype(np.uint32).view(np.float32).astype(np.float64)


def store(a, dtype):
    return bf16(a) if dtype == "bf16" else np.asarray(a, np.float32).astype(np.float64)


def turn(x, cos, sin, adjacent, sign=1.0):
    """x [B][T][H][D], cos and sin [B][T][R/2]: its first R entries turned."""
    n = cos.shape[-1]
    y = x.copy()
    i = np.arange(n)
    a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + n)
    c, s = cos[:, :, None, :], sign * sin[:, :, None, :]
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y


def norm_rotate(x, w, cos, sin, adjacent, eps):
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return turn(x * r * w, cos, sin, adjacent)


def norm_rotate_grad(x, w, dy, cos, sin, adjacent, eps):
    """dx, dw and the sums of the absolute terms of either."""
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r
    t = turn(dy, cos, sin, adjacent, -1.0)
    m = (t * w * n).mean(-1, keepdims=True)
    dx = r * (t * w - n * m)
    # |t| is at most |a| + |b| of its pair, whatever the rounding
    mag_dx = r * (np.abs(t * w) + np.abs(n) * np.abs(t * w * n).mean(-1, keepdims=True))
    return dx, (t * n).sum((0, 1, 2)), mag_dx, np.abs(t * n).sum((0, 1, 2))


def visible(n, p, Tk, left, right, sinks):
    """[len(p)][Tk]: whether the query at position p sees key j of a sequence of n tokens."""
    p, j = np.asarray(p)[:, None], np.arange(Tk)[None]
    see = (j < n) & (p < n) & (p >= 0)
    if right >= 0:
        see &= j <= p + right
    if left >= 0:
        see &= (j >= p - left) | (j < sinks)
    return see


def attention(q, k, v, see, scale, do=None):
    """One head: q [n][D], k, v [m][D], see [n][m].  A dict of o, lse and, with
    do, dq, dk, dv, each with the sums of absolute terms that bound its errors
    (mag_*), and `s_mag`, the largest sum of absolute terms of a score."""
    k, v = np.where(see.any(0)[:, None], k, 0.0), np.where(see.any(0)[:, None], v, 0.0)
    q = np.where(see.any(1)[:, None], q, 0.0)
    s = np.where(see, scale * (q @ k.T), -np.inf)
    m = s.max(1, initial=-np.inf, keepdims=True)
    m = np.where(np.isfinite(m), m, 0.0)
    e = np.exp(s - m)
    z = e.sum(1, keepdims=True)
    p = e / np.where(z > 0, z, 1.0)
    with np.errstate(divide="ignore"):
        lse = (m + np.log(z))[:, 0]
    o = p @ v
    out = dict(o=o, lse=lse, mag_o=p @ np.abs(v), s_mag=float((scale * np.abs(q) @ np.abs(k).T).max(initial=0.0)))
    if do is None:
        return out
    do = np.where(see.any(1)[:, None], do, 0.0)
    dp = do @ v.T
    mag_dp = np.abs(do) @ np.abs(v).T
    d = (do * o).sum(1, keepdims=True)
    ds = p * (dp - d)
    # what ds can be off by where o is (mag_o + |o|) and a product its absolute terms
    mag_d = (np.abs(do) * (out["mag_o"] + np.abs(o))).sum(1, keepdims=True)
    out.update(dq=scale * ds @ k, dk=scale * ds.T @ q, dv=p.T @ do, mag_dv=p.T @ np.abs(do),
               mag_dq=scale * (np.abs(ds) + p * mag_d) @ np.abs(k),
               mag_dk=scale * (np.abs(ds) + p * mag_d).T @ np.abs(q),
               wide_dq=scale * (p * mag_dp) @ np.abs(k), wide_dk=scale * (p * mag_dp).T @ np.abs(q))
    return out


def delta_rule(q, k, v, g, beta, S, scale, do=None, dS=None):
    """One head, token by token: q, k [T][Dk], v [T][Dv], g, beta [T], S [Dk][Dv].
    A dict of o, state and, with do and dS, the gradients."""
    T = len(g)
    a, o, kept = np.exp(g), np.zeros_like(v), []
    for t in range(T):
        kept.append(S)
        S = a[t] * S
        S = S + np.outer(k[t], beta[t] * (v[t] - S.T @ k[t]))
        o[t] = scale * S.T @ q[t]
    out = dict(o=o, state=S)
    if do is None:
        return out
    dq, dk, dv, dg, db = (np.zeros_like(x) for x in (q, k, v, g, beta))
    for t in reversed(range(T)):
        before = a[t] * kept[t]
        z = v[t] - before.T @ k[t]
        S = before + np.outer(k[t], beta[t] * z)
        dq[t] = scale * S @ do[t]
        dS = dS + scale * np.outer(q[t], do[t])
        du = dS.T @ k[t]
        db[t] = du @ z
        dk[t] = dS @ (beta[t] * z) - before @ (beta[t] * du)
        dv[t] = beta[t] * du
        dS = dS - np.outer(k[t], beta[t] * du)
        dg[t] = (dS * before).sum()
        dS = a[t] * dS
    out.update(dq=dq, dk=dk, dv=dv, dg=dg, dbeta=db, dstate=dS)
    return out
