"""The state space sublayer's operators in 64 bits, from their formulas (numpy, no library
code), each result with a bound on what fp32 arithmetic may be off by.

Rounding: u = 2^-24 is half a step of fp32 relative to a value.  An exponential exp(-|x|),
formed as a power of 2, is off by (1.5 |x| + 2) u of itself: its argument's product and
constant (1.5 u |x|) and one step of the instruction (2 u).  So are, with three more
roundings, sigmoid(x) by (1.5 |x| + 5) u of itself and softplus(x) by (1.5 |x| + 8) u of
itself.  A sum of n terms in any order of depth m is off by m u of the sum of its absolute
terms.  A recurrence h = a h + b carries the errors of h with it: its bound is the same
recurrence on absolute values, err = a err + (what a and b are off by)."""
import numpy as np

U = 2.0 ** -24


def sigmoid(x):
    return 1 / (1 + np.exp(-x))


def silu(x, err=0.0):
    """x sigmoid(x) and what it may be off by, where x is off by err."""
    y = x * sigmoid(x)
    return y, np.abs(y) * (1.5 * np.abs(x) + 7) * U + 1.1 * err


def silu_grad(x, err=0.0):
    """The derivative s + x m, m = s (1 - s), and what it may be off by: s by m (1.5 |x| + 2) u
    + 3 s u; 1 - s by that and u; the sum by (1 + |x|) of it, and 4 roundings; its own
    derivative is below 0.5 in absolute value."""
    s = sigmoid(x)
    es = s * (1 - s) * (1.5 * np.abs(x) + 2) * U + 3 * s * U
    return s + x * s * (1 - s), (1 + np.abs(x)) * (es + U) + 4 * U + 0.5 * err


def conv(x, w, bias, state, n, act, dy=None, dend=None, depth=0):
    """One sequence: x [T][C], w [C][K], bias [C], state [K-1][C], n its length.  A dict of
    results and, under the same names with e_, their bounds."""
    T, C = x.shape
    K = w.shape[1]
    rows = np.concatenate((state, x[:n]))
    taps = np.stack([rows[j:j + n] for j in range(K)], -1)          # [n][C][K]
    u = bias + (taps * w).sum(-1)
    eu = (K + 1) * U * (np.abs(bias) + (np.abs(taps) * np.abs(w)).sum(-1))
    out = {"y": np.zeros((T, C)), "e_y": np.zeros((T, C)), "end": rows[n:]}
    out["y"][:n], out["e_y"][:n] = silu(u, eu) if act else (u, eu)
    if dy is None:
        return out
    f, ef = silu_grad(u, eu) if act else (np.ones_like(u), 0.0)
    du, edu = dy[:n] * f, np.abs(dy[:n]) * ef + np.abs(dy[:n] * f) * U
    back, eback = np.zeros_like(rows), np.zeros_like(rows)
    for j in range(K):
        back[j:j + n] += w[:, j] * du
        eback[j:j + n] += np.abs(w[:, j]) * (edu + (K + 1) * U * np.abs(du))
    back[n:] += dend
    eback[n:] += U * np.abs(dend)
    out.update(dx=np.zeros((T, C)), e_dx=np.zeros((T, C)), dstate=back[:K - 1], e_dstate=eback[:K - 1])
    out["dx"][:n], out["e_dx"][:n] = back[K - 1:], eback[K - 1:]
    out["dbias"], out["e_dbias"] = du.sum(0), (edu + depth * U * np.abs(du)).sum(0)
    out["dw"] = (taps * du[:, :, None]).sum(0)
    out["e_dw"] = (np.abs(taps) * (edu + depth * U * np.abs(du))[:, :, None]).sum(0)
    return out


def scan(x, dt, A, B, C, D, z, bias, h, n, soft, dy=None, dend=None, depth_t=0, depth_c=0):
    """One sequence: x, dt, z [T][c] (z may be None), A [c][N], B, C [T][c][N] (each channel its
    group's), D, bias [c], h [c][N], n its length."""
    T, c = x.shape
    raw = dt[:n] + bias
    d = np.logaddexp(0, raw) if soft else raw
    rd = (2.5 * np.abs(raw) + 8) * U if soft else U                # of d, relative
    x, B, C = x[:n], B[:n], C[:n]
    u = d * x
    dA = d[:, :, None] * A
    a = np.exp(dA)
    ra = np.abs(dA) * ((rd if np.isscalar(rd) else rd[:, :, None]) + 2 * U) + 4 * U   # of a step's decay and its sum, relative
    if z is None:
        gate, egate = np.ones_like(x), np.zeros_like(x)
    else:
        gate, egate = silu(z[:n])
    hs, ha, eh = np.zeros((n + 1, c, h.shape[1])), np.zeros((n + 1, c, h.shape[1])), np.zeros((n + 1, c, h.shape[1]))
    hs[0], ha[0] = h, np.abs(h)
    for t in range(n):
        add = np.abs(u[t])[:, None] * np.abs(B[t])
        hs[t + 1] = a[t] * hs[t] + u[t][:, None] * B[t]
        ha[t + 1] = a[t] * ha[t] + add
        eh[t + 1] = a[t] * (eh[t] + ra[t] * ha[t]) + add * ((rd if np.isscalar(rd) else rd[t][:, None]) + 4 * U)
    # chunks are joined by exponentials of sums of d, off by T u of the sum: with a decay of
    # exp(-s) that is T u s exp(-s), beyond what ra counts (4 u a token) at most 3e-3 T u
    eh += 3e-3 * T * U * ha.max(initial=0.0)
    core = (C * hs[1:]).sum(-1) + D * x
    m = (np.abs(C) * ha[1:]).sum(-1) + np.abs(D * x)
    ecore = (np.abs(C) * eh[1:]).sum(-1) + (A.shape[1] + 3) * U * m
    out = {"y": np.zeros((T, c)), "e_y": np.zeros((T, c)), "end": hs[n], "e_end": eh[n]}
    out["y"][:n] = core * gate
    out["e_y"][:n] = ecore * np.abs(gate) + np.abs(core) * (egate + U * np.abs(gate))
    if dy is None:
        return out
    up = dy[:n] * gate
    eup = np.abs(dy[:n]) * egate + U * np.abs(up)
    g, ga, eg = dend.copy(), np.abs(dend), np.zeros_like(dend)
    gs, gm, ge = (np.zeros((n, c, h.shape[1])) for _ in range(3))
    for t in reversed(range(n)):
        gs[t] = g + C[t] * up[t][:, None]
        gm[t] = ga + np.abs(C[t] * up[t][:, None])
        ge[t] = eg + np.abs(C[t]) * eup[t][:, None] + 2 * U * gm[t]
        g, ga, eg = a[t] * gs[t], a[t] * gm[t], a[t] * (ge[t] + ra[t] * gm[t])
    ge += 3e-3 * T * U * gm.max(initial=0.0)
    N = A.shape[1]
    w, wm = gs * a * hs[:-1], gm * a * ha[:-1]
    ew = ge * a * ha[:-1] + gm * a * eh[:-1] + wm * (ra + 3 * U)
    full = np.abs(u)[:, :, None]
    du, em = (gs * B).sum(-1), (gm * np.abs(B)).sum(-1)
    edu = (ge * np.abs(B)).sum(-1) + (N + 2) * U * em
    dd = (w * A).sum(-1) + du * x
    edd = (ew * np.abs(A)).sum(-1) + (N + 4) * U * (wm * np.abs(A)).sum(-1) + (edu + 2 * U * em) * np.abs(x)
    s = sigmoid(raw) if soft else np.ones_like(raw)
    es = s * (1.5 * np.abs(raw) + 6) * U if soft else 0.0
    full_t = {"dx": (du * d + D * up, edu * d + em * d * (rd + 2 * U) + np.abs(D) * (eup + 2 * U * np.abs(up))),
              "ddt": (dd * s, edd * s + np.abs(dd) * (es + U)),
              "dB": (gs * u[:, :, None], (ge + gm * ((rd if np.isscalar(rd) else rd[:, :, None]) + depth_c * U)) * full),
              "dC": (hs[1:] * up[:, :, None], eh[1:] * np.abs(up)[:, :, None] + ha[1:] * (eup + depth_c * U * np.abs(up))[:, :, None])}
    if z is not None:
        f, ef = silu_grad(z[:n])
        full_t["dz"] = (dy[:n] * core * f, np.abs(dy[:n]) * (ecore * np.abs(f) + np.abs(core) * (ef + 3 * U)))
    for k, (v, e) in full_t.items():     # per channel: the caller adds up groups
        out[k], out["e_" + k] = np.zeros((T, *v.shape[1:])), np.zeros((T, *v.shape[1:]))
        out[k][:n], out["e_" + k][:n] = v, e
    dcol = d[:, :, None]
    out["dA"] = (w * dcol).sum(0)
    out["e_dA"] = (ew * dcol + wm * dcol * ((rd if np.isscalar(rd) else rd[:, :, None]) + depth_t * U)).sum(0)
    out["dD"], out["e_dD"] = (up * x).sum(0), ((eup + depth_t * U * np.abs(up)) * np.abs(x)).sum(0)
    out["dbias"], out["e_dbias"] = (dd * s).sum(0), (out["e_ddt"][:n] + depth_t * U * np.abs(dd * s)).sum(0)
    out["dstate"], out["e_dstate"] = g, eg + 3e-3 * T * U * ga.max(initial=0.0)
    return out


def join(r, f, w, w_post, scale, gate, eps, dy=None, dro=None, depth=0):
    """r, f [B][T][C], gate [B][C] (any vector may be None).  A sum of squares of C terms is off by C u of itself at most, its inverse
    root by half of that and three roundings."""
    C = r.shape[-1]
    ri = (C / 2 + 4) * U
    one = np.ones(C)
    gs = (one if gate is None else gate[:, None]) * (one if scale is None else scale)
    out = {}
    if f is None:
        ro, ero = r, np.zeros_like(r)
        nf = enf = None
    else:
        nf, enf = f, np.zeros_like(f)
        if w_post is not None:
            i = 1 / np.sqrt((f * f).mean(-1, keepdims=True) + eps)
            nf, enf = f * i, np.abs(f) * i * (ri + U)
        k = gs * (one if w_post is None else w_post)
        ro = r + k * nf
        ero = np.abs(k) * (enf + 4 * U * np.abs(nf)) + U * np.abs(ro)
        out["r"], out["e_r"] = ro, ero
    i = 1 / np.sqrt((ro * ro).mean(-1, keepdims=True) + eps)
    # an error of ro moves n by at most i (ero + |n| rms(ero) ...): its own entry and the mean's
    n = ro * i
    en = i * ero + np.abs(n) * (ri + U + i * np.sqrt((ero * ero).mean(-1, keepdims=True)))
    ww = one if w is None else w
    out["y"], out["e_y"] = n * ww, np.abs(ww) * (en + U * np.abs(n))
    if dy is None:
        return out
    t = dy * ww
    m, am = (t * n).mean(-1, keepdims=True), np.abs(t * n).mean(-1, keepdims=True)
    em = (np.abs(t) * en).mean(-1, keepdims=True) + am * (C + 4) * U
    g = i * (t - n * m)
    rr = ri + 3 * U + i * np.sqrt((ero * ero).mean(-1, keepdims=True))      # of the inverse root, relative
    eg = i * (np.abs(t) * rr + en * am + np.abs(n) * (em + am * rr))
    if dro is not None:
        g, eg = g + dro, eg + U * np.abs(g + dro)
    ax = (0, 1)
    out.update(dr=g, e_dr=eg, dw=(dy * n).sum(ax), e_dw=(np.abs(dy) * (en + depth * U * np.abs(n))).sum(ax))
    if f is None:
        return out
    k = gs * (one if w_post is None else w_post)
    t, et = g * k, np.abs(k) * (eg + 3 * U * np.abs(g))
    if w_post is None:
        out["df"], out["e_df"] = t, et
    else:
        i = 1 / np.sqrt((f * f).mean(-1, keepdims=True) + eps)
        m, am = (t * nf).mean(-1, keepdims=True), np.abs(t * nf).mean(-1, keepdims=True)
        em = (et * np.abs(nf)).mean(-1, keepdims=True) + am * ((C + 4) * U + 2 * ri)
        out["df"] = i * (t - nf * m)
        out["e_df"] = i * (et + np.abs(t) * (ri + 3 * U) + np.abs(nf) * (em + am * (ri + 3 * U)))
    q = (g * nf).sum(1)
    eq = (eg * np.abs(nf) + np.abs(g) * (enf + depth * U * np.abs(nf))).sum(1)
    ga, sc, wp = one if gate is None else gate, one if scale is None else scale, one if w_post is None else w_post
    B = r.shape[0]
    aq = eq + (B + 3) * U * np.abs(g * nf).sum(1)
    if w_post is not None:
        out["dw_post"], out["e_dw_post"] = (ga * q).sum(0) * sc, (np.abs(ga) * aq).sum(0) * np.abs(sc)
    if scale is not None:
        out["dscale"], out["e_dscale"] = (ga * q).sum(0) * wp, (np.abs(ga) * aq).sum(0) * np.abs(wp)
    if gate is not None:
        out["dgate"], out["e_dgate"] = q * sc * wp, aq * np.abs(sc * wp)
    return out
