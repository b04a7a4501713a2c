"""Calls of the state space sublayer's operators, in the sizes and layouts in which they occur.

Beside attention and the delta rule stands the recurrence with a diagonal state, the
scan's nearest relative over a sequence of tokens.  The operators of its sublayer, in
the order in which they are called:

* residual_fwd / residual_train: what joins two sublayers.  The block's output f, normed
  where the norm behind a block has a weight, gated a sequence and scaled a channel, is
  added to the residual stream, and the sum is normed for the next block:
  p = w_post f / rms(f) (or f),  r' = r + scale gate p,  y = w r' / rms(r').
* conv_fwd / conv_train: the causal convolution of each channel with its own K taps,
  u_t = bias + sum_j w_j x_{t-K+1+j},  y = u sigmoid(u), from the K - 1 inputs before
  the first token and to those behind the last; one token a sequence is its serving form.
* scan_fwd / scan_train: the selective state space scan.  With d = softplus(dt + dt_bias),
  h_t = exp(d A) h_{t-1} + d x_t B_t,  y_t = (C_t . h_t + D x_t) z sigmoid(z)
  for every channel with N states (A [C][N], B and C [B][T][G][N] shared by groups of
  channels), from a state and to one (fp32 [B][C][N]).

The _train cases are the operator and its gradient, one step of training.  `plain` forms
are in 32 bits, rounded once at the end; `exact` is each operator's definition in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6


def listed():
    return [
        # one decoding step: the joint between two sublayers, 8 sequences, one token each
        dict(name="residual_fwd-token", op="residual_fwd", B=8, T=1, C=1152, post=True, gate=False, scale=True, wide=False, dtype="bf16"),
        # 74 x 74 tokens of 1152 channels, batch 32, behind a block with a residual scale
        dict(name="residual_fwd-74x74", op="residual_fwd", B=32, T=5476, C=1152, post=False, gate=False, scale=True, wide=False, dtype="bf16"),
        # the 64 x 64 training workload of 768 channels, batch 8: norms on both sides, a gate, the residual stream in fp32
        dict(name="residual_train-64x64", op="residual_train", B=8, T=4096, C=768, post=True, gate=True, scale=True, wide=True, dtype="bf16"),
        # 185 x 185 tokens in fp32
        dict(name="residual_train-185x185-f32", op="residual_train", B=1, T=34225, C=1152, post=False, gate=False, scale=True, wide=True, dtype="f32"),
        # one token each of 64 sequences, channels twice those of the 64 x 64 workload
        dict(name="conv_fwd-token", op="conv_fwd", B=64, T=1, C=1536, K=4, state=True, ragged=False, dtype="bf16"),
        # 74 x 74 tokens as sequences
        dict(name="conv_fwd-74x74", op="conv_fwd", B=32, T=5476, C=1152, K=4, state=False, ragged=False, dtype="bf16"),
        # the 64 x 64 training workload as sequences, channels doubled by the sublayer's projection
        dict(name="conv_train-64x64", op="conv_train", B=8, T=4096, C=1536, K=4, state=False, ragged=False, dtype="bf16"),
        # one token each of 64 sequences
        dict(name="scan_fwd-token", op="scan_fwd", B=64, T=1, C=1536, N=16, G=1, z=True, state=True, ragged=False, dtype="bf16"),
        # one sequence of 185 x 185 tokens: parallel over the tokens alone
        dict(name="scan_fwd-185x185", op="scan_fwd", B=1, T=34225, C=2304, N=16, G=1, z=True, state=False, ragged=False, dtype="bf16"),
        # long ragged sequences continued from a state, in fp32, 8 states
        dict(name="scan_fwd-8191-f32", op="scan_fwd", B=4, T=8191, C=768, N=8, G=2, z=False, state=True, ragged=True, dtype="f32"),
        # the 64 x 64 training workload as sequences
        dict(name="scan_train-64x64", op="scan_train", B=8, T=4096, C=1536, N=16, G=1, z=True, state=False, ragged=False, dtype="bf16"),
        # an odd short step in fp32, ragged, two groups that are no multiple of a wave
        dict(name="scan_train-777-f32", op="scan_train", B=2, T=777, C=400, N=16, G=2, z=True, state=True, ragged=True, dtype="f32"),
    ]


def _log(rng, lo, hi):
    """A size between lo and hi, spread over its logarithm; odd or a small multiple of an odd one."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))) | rng.choice((1, 2, 4))))


def draw(rng):
    top = max(_cost(c) for c in listed())
    op = rng.choice(["residual_fwd", "residual_train", "conv_fwd", "conv_train", "scan_fwd", "scan_fwd", "scan_train", "scan_train"])
    while True:
        c = dict(op=op, B=_log(rng, 1, 64), T=_log(rng, 1, 34225), C=8 * _log(rng, 2, 512), dtype=rng.choice(["bf16", "bf16", "f32"]))
        if op.startswith("residual"):
            c.update(post=rng.choice([False, True]), gate=rng.choice([False, True]), scale=rng.choice([False, True, True]))
            c.update(wide=rng.choice([False, True]) or c["dtype"] == "f32")
        else:
            if rng.random() < 0.25 and op.endswith("fwd"):
                c.update(T=rng.choice([1, 1, 1, 2, 5]))
            c.update(state=rng.choice([False, True]), ragged=rng.choice([False, True]))
            if op.startswith("conv"):
                c.update(K=rng.choice([2, 3, 4, 4]))
            else:
                G = rng.choice([1, 1, 2, 4])
                c.update(C=G * 8 * _log(rng, 1, 288 // G), N=rng.choice([1, 2, 4, 5, 8, 16, 16, 16, 24, 32]), G=G, z=rng.choice([False, True, True]))
        if op.startswith("scan") and c["B"] * c["T"] * c["C"] * c["N"] > 8 * 4096 * 1536 * 16:   # what the plain form's states take
            continue
        if _cost(c) <= top:
            return c


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _lens(c):
    """The sequences' lengths: whole, or ragged (the same for every seed)."""
    if not c.get("ragged"):
        return None
    return [max(1, c["T"] - (b * 769 + 767) % max(1, c["T"] // 2)) for b in range(c["B"])]


def work(case):
    c, s = case, 2 if case["dtype"] == "bf16" else 4
    n = c["B"] * c["T"] * c["C"]
    train = c["op"].endswith("train")
    if c["op"].startswith("residual"):
        rs = 4 if c["wide"] else s
        vectors = c["C"] * s * (1 + c["post"] + c["scale"] + c["B"] * c["gate"])
        if train:
            return {"bytes": 4 * n * s + 4 * n * rs + 2 * vectors, "flops": 40 * n}
        return {"bytes": 2 * n * s + 2 * n * rs + vectors, "flops": 12 * n}
    if c["op"].startswith("conv"):
        K = c["K"]
        ends = c["B"] * (K - 1) * c["C"] * s * (1 + c["state"])
        if train:
            return {"bytes": 4 * n * s + 2 * ends + 2 * (K + 1) * c["C"] * s, "flops": (8 * K + 20) * n}
        return {"bytes": 2 * n * s + ends + (K + 1) * c["C"] * s, "flops": (2 * K + 5) * n}
    N = c["N"]
    ends = 4 * c["B"] * c["C"] * N * (1 + c["state"])
    shared = 2 * c["B"] * c["T"] * c["G"] * N * s
    if train:
        return {"bytes": (6 + 2 * c["z"]) * n * s + 2 * shared + 2 * ends + 8 * c["C"] * (N + 2), "flops": 27 * n * N}
    return {"bytes": (3 + c["z"]) * n * s + shared + ends + 4 * c["C"] * (N + 2), "flops": 7 * n * N}


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def prepare(case, seed):
    c, dt = case, _dtype(case)
    B, T, C = c["B"], c["T"], c["C"]
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, device=DEV, generator=g)

    def rand(*shape):
        return torch.randn(*shape, device=DEV, dtype=dt, generator=g)

    st = {"case": c}
    lens = _lens(c)
    st["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV) if lens else None
    train = c["op"].endswith("train")
    if c["op"].startswith("residual"):
        rt = torch.float32 if c["wide"] else dt
        st.update(r=(2 * randn(B, T, C)).to(rt), f=rand(B, T, C), w=1 + 0.1 * rand(C))
        st["w_post"] = 1 + 0.1 * rand(C) if c["post"] else None
        st["scale"] = 0.5 + 0.1 * rand(C) if c["scale"] else None
        st["gate"] = 1 + 0.3 * rand(B, C) if c["gate"] else None
        if train:
            st.update(dy=rand(B, T, C), dr=randn(B, T, C).to(rt))
        return st
    if c["op"].startswith("conv"):
        K = c["K"]
        fused = rand(B, T, 2 * C)     # the projection's output: the scan's input and its gate
        st.update(x=fused[:, :, :C], w=rand(C, K) / math.sqrt(K), bias=0.1 * rand(C))
        st["state"] = rand(B, K - 1, C) if c["state"] else None
        if train:
            st.update(dy=rand(B, T, C), dend=rand(B, K - 1, C))
        return st
    N, G = c["N"], c["G"]
    fused = rand(B, T, 2 * C)
    small = rand(B, T, 8 + 2 * G * N)   # the projection that the steps, B and C come from
    st.update(x=rand(B, T, C), z=fused[:, :, C:] if c["z"] else None, dt=0.5 * rand(B, T, C))
    st["B"], st["C"] = (small[:, :, at:at + G * N].unflatten(2, (G, N)) for at in (8, 8 + G * N))
    # states that decay at rates of 1 to N, steps of 1/1000 to 1/10
    st["A"] = -torch.arange(1, N + 1, device=DEV) * torch.exp(0.1 * randn(C, N))
    step = torch.exp(torch.rand(C, device=DEV, generator=g) * math.log(100) + math.log(1e-3))
    st.update(dt_bias=step + torch.log(-torch.expm1(-step)), D=1 + 0.1 * randn(C))
    st["state"] = 0.1 * randn(B, C, N) if c["state"] else None
    if train:
        st.update(dy=rand(B, T, C), dend=0.1 * randn(B, C, N))
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    c = state["case"]
    return _run_own(c, state) if own else _run_plain(c, state)


def _run_own(c, s):
    import paper_2606_00746_amd as gspn
    if c["op"].startswith("residual"):
        weights = (s["w"], s["w_post"], s["scale"], s["gate"])
        y, r = gspn.residual_norm_fwd(s["r"], s["f"], *weights, eps=EPS)
        if c["op"] == "residual_fwd":
            return y, r
        return (y, r, *gspn.residual_norm_bwd(s["r"], s["f"], *weights, s["dy"], s["dr"], eps=EPS))
    if c["op"].startswith("conv"):
        y, end = gspn.short_conv_fwd(s["x"], s["w"], s["bias"], state=s["state"], lens=s["lens"])
        if c["op"] == "conv_fwd":
            return y, end
        return (y, end, *gspn.short_conv_bwd(s["x"], s["w"], s["bias"], s["dy"], dstate=s["dend"], state=s["state"], lens=s["lens"]))
    x = (s["x"], s["dt"], s["A"], s["B"], s["C"], s["D"], s["z"], s["dt_bias"])
    if c["op"] == "scan_fwd":
        return gspn.selective_scan_fwd(*x, state=s["state"], lens=s["lens"])
    y, end, reserve = gspn.selective_scan_fwd_train(*x, state=s["state"], lens=s["lens"])
    return (y, end, *gspn.selective_scan_bwd_reserve(*x, s["dy"], reserve, dstate=s["dend"], state=s["state"], lens=s["lens"]))


def _run_plain(c, s):
    op = {"res": _residual, "con": _conv, "sca": _scan}[c["op"][:3]]
    names = {"res": "r f w w_post scale gate", "con": "x w bias state", "sca": "x dt A B C D z dt_bias state"}[c["op"][:3]].split()
    x = {n: None if s[n] is None else s[n].float() for n in names}
    if not c["op"].endswith("train"):
        a, b = op(c, s["lens"], **x)
    else:
        there = [n for n in names if x[n] is not None]
        leaves = {n: x[n].detach().requires_grad_() for n in there}
        a, b = op(c, s["lens"], **{n: leaves.get(n) for n in names})
        up = (s["dy"], s["dr"]) if c["op"].startswith("res") else (s["dy"], s["dend"])
        grads = dict(zip(there, torch.autograd.grad((a, b), [leaves[n] for n in there], [u.float() for u in up])))
        grads = [grads[n].to(s[n].dtype) if n in grads else None for n in names]
        a, b = a.detach(), b.detach()
    # the second output: the residual stream, the last inputs, the last state
    first, second = (s["f"], s["r"]) if c["op"].startswith("res") else (s["x"], s["x"] if c["op"].startswith("conv") else s["A"])
    out = (a.to(first.dtype), b.to(second.dtype))
    return (*out, *grads) if c["op"].endswith("train") else out


def _rms(x):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)


def _residual(c, lens, r, f, w, w_post, scale, gate):
    p = f if w_post is None else _rms(f) * w_post
    if gate is not None:
        p = p * gate[:, None]
    if scale is not None:
        p = p * scale
    r = r + p
    return _rms(r) * w, r


def _ends(c, lens):
    return torch.full((c["B"],), c["T"], device=DEV) if lens is None else lens.long()


def _conv(c, lens, x, w, bias, state):
    B, T, C, K = c["B"], c["T"], c["C"], c["K"]
    n = _ends(c, lens)
    if state is None:
        state = torch.zeros(B, K - 1, C, device=DEV)
    live = (torch.arange(T, device=DEV) < n[:, None])[:, :, None]
    rows = torch.cat((state, x), 1)
    u = bias
    for j in range(K):
        u = u + w[:, j] * rows[:, j:j + T]
    y = u * torch.sigmoid(u) * live
    at = n[:, None] + torch.arange(K - 1, device=DEV)
    return y, rows[torch.arange(B, device=DEV)[:, None], at]


def _scan(c, lens, x, dt, A, B, C, D, z, dt_bias, state):
    """Parts of about sqrt(T) tokens side by side, each from zero; their ends joined; and again from where each begins."""
    b, T, ch, N, G = c["B"], c["T"], c["C"], c["N"], c["G"]
    L = max(1, math.isqrt(T))
    nc = -(-T // L)
    live = (torch.arange(T, device=DEV) < _ends(c, lens)[:, None])[:, :, None]
    d = dt + dt_bias
    d = (torch.clamp(d, min=0) + torch.log1p(torch.exp(-d.abs()))) * live

    def parts(t, *shape):   # [b][T]... as L tensors [b][nc][shape]
        t = torch.nn.functional.pad(t, (0, 0) * (t.dim() - 2) + (0, nc * L - T))
        return t.reshape(b, nc, L, *shape).unbind(2)

    dp, u = parts(d, G, ch // G, 1), parts(d * x, G, ch // G, 1)
    Bp, Cp = parts(B, G, 1, N), parts(C, G, 1, N)
    A = A.view(G, ch // G, N)
    h = torch.zeros(b, nc, G, ch // G, N, device=DEV)
    if nc > 1:
        for i in range(L):
            h = torch.exp(dp[i] * A) * h + u[i] * Bp[i]
    at = torch.zeros(b, G, ch // G, N, device=DEV) if state is None else state.view(b, G, ch // G, N)
    starts, whole = [at], torch.exp(sum(dp) * A)
    for k in range(nc - 1):
        at = whole[:, k] * at + h[:, k]
        starts.append(at)
    h, y = torch.stack(starts, 1), []
    for i in range(L):
        h = torch.exp(dp[i] * A) * h + u[i] * Bp[i]
        y.append((h * Cp[i]).sum(-1))
    y = torch.stack(y, 2).reshape(b, nc * L, ch)[:, :T] + D * x
    if z is not None:
        y = y * z * torch.sigmoid(z)
    return y * live, h[:, -1].reshape(b, ch, N)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    s = {n: t.double() if torch.is_tensor(t) and t.is_floating_point() else t for n, t in s.items()}
    return {"res": _exact_residual, "con": _exact_conv, "sca": _exact_scan}[case["op"][:3]](case, s)


def _exact_residual(c, s):
    """By the norms' own gradients: of n = x / s(x), s = sqrt(mean(x^2) + eps), dx = (t - n mean(t n)) / s."""
    one = torch.ones(c["C"], device=DEV, dtype=torch.float64)
    scale = one if s["scale"] is None else s["scale"]
    gate = one.expand(c["B"], -1) if s["gate"] is None else s["gate"]
    k = (gate * scale)[:, None]
    f, sf, nf = s["f"], None, s["f"]
    if s["w_post"] is not None:
        sf = (f.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
        nf = f / sf
        k = k * s["w_post"]
    r = s["r"] + k * nf
    sr = (r.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
    n = r / sr
    y = n * s["w"]
    if c["op"] == "residual_fwd":
        return y, r
    t = s["dy"] * s["w"]
    dr = s["dr"] + (t - n * (t * n).mean(-1, keepdim=True)) / sr
    dw = (s["dy"] * n).sum((0, 1))
    q = (dr * nf).sum(1)
    t = dr * k
    df = t if sf is None else (t - nf * (t * nf).mean(-1, keepdim=True)) / sf
    wp = one if s["w_post"] is None else s["w_post"]
    return (y, r, dr, df, dw, None if s["w_post"] is None else (gate * scale * q).sum(0),
            None if s["scale"] is None else (gate * wp * q).sum(0), None if s["gate"] is None else scale * wp * q)


def _exact_conv(c, s):
    """Sequence by sequence: its own tokens behind the state's."""
    B, T, C, K = c["B"], c["T"], c["C"], c["K"]
    train = c["op"] == "conv_train"
    kw = dict(device=DEV, dtype=torch.float64)
    y, end = torch.zeros(B, T, C, **kw), torch.zeros(B, K - 1, C, **kw)
    dx, dw, dbias, dstate = torch.zeros(B, T, C, **kw), torch.zeros(C, K, **kw), torch.zeros(C, **kw), torch.zeros(B, K - 1, C, **kw)
    for b, n in enumerate(_lens(c) or [T] * B):
        head = torch.zeros(K - 1, C, **kw) if s["state"] is None else s["state"][b]
        rows = torch.cat((head, s["x"][b, :n]))
        taps = rows.unfold(0, K, 1)                       # [n][C][K]
        u = s["bias"] + (taps * s["w"]).sum(-1)
        sig = 1 / (1 + torch.exp(-u))
        y[b, :n], end[b] = u * sig, rows[n:]
        if not train:
            continue
        du = s["dy"][b, :n] * (sig + u * sig * (1 - sig))
        dbias += du.sum(0)
        dw += (taps * du[:, :, None]).sum(0)
        back = torch.zeros_like(rows)
        for j in range(K):
            back[j:j + n] += s["w"][:, j] * du
        back[n:] += s["dend"][b]
        dstate[b], dx[b, :n] = back[:K - 1], back[K - 1:]
    if not train:
        return y, end
    return y, end, dx, dw, dbias, None if s["state"] is None else dstate


def _exact_scan(c, s):
    """Token by token, and for the gradient back again over the states that were kept."""
    B, T, ch, N, G = c["B"], c["T"], c["C"], c["N"], c["G"]
    train = c["op"] == "scan_train"
    if train and 8 * B * T * ch * N > 60e9:
        return None
    x, A, D = s["x"], s["A"], s["D"]
    live = torch.ones(B, T, 1, device=DEV, dtype=torch.float64)
    if s["lens"] is not None:
        live = (torch.arange(T, device=DEV) < s["lens"][:, None]).double()[:, :, None]
    raw = s["dt"] + s["dt_bias"]
    d = torch.where(raw > 30, raw, torch.log1p(torch.exp(torch.clamp(raw, max=30)))) * live
    gate = live if s["z"] is None else live * s["z"] / (1 + torch.exp(-s["z"]))
    rep = ch // G
    Bm, Cm = s["B"], s["C"]
    h = torch.zeros(B, ch, N, device=DEV, dtype=torch.float64) if s["state"] is None else s["state"]
    first, kept, core = h, [], torch.zeros(B, T, ch, device=DEV, dtype=torch.float64)

    def wide(m, t):
        return m[:, t].repeat_interleave(rep, 1)

    for t in range(T):
        h = torch.exp(d[:, t, :, None] * A) * h + (d[:, t] * x[:, t])[..., None] * wide(Bm, t)
        core[:, t] = (h * wide(Cm, t)).sum(-1)
        kept.append(h) if train else None
    core = core + D * x
    y = core * gate
    if not train:
        return y, h
    dy = s["dy"] * live
    dc = dy if s["z"] is None else dy * gate
    dx, dd, dA = D * dc, torch.zeros_like(d), torch.zeros_like(A)
    dB, dC = torch.zeros_like(Bm), torch.zeros_like(Cm)
    g = s["dend"]
    for t in reversed(range(T)):
        before = kept[t - 1] if t else first
        dC[:, t] = (kept[t] * dc[:, t, :, None]).unflatten(1, (G, rep)).sum(2)
        g = g + wide(Cm, t) * dc[:, t, :, None]
        dB[:, t] = (g * (d[:, t] * x[:, t])[..., None]).unflatten(1, (G, rep)).sum(2)
        gb = (g * wide(Bm, t)).sum(-1)
        dx[:, t] += gb * d[:, t]
        a = torch.exp(d[:, t, :, None] * A)
        q = g * a * before
        dd[:, t] = gb * x[:, t] + (q * A).sum(-1)
        dA += (q * d[:, t, :, None]).sum(0)
        g = a * g
    draw = dd * live / (1 + torch.exp(-raw))
    dz = None
    if s["z"] is not None:
        sig = 1 / (1 + torch.exp(-s["z"]))
        dz = dy * core * (sig + s["z"] * sig * (1 - sig))
    return y, h, dx, draw, dA, dB, dC, (dc * x).sum((0, 1)), dz, draw.sum((0, 1)), None if s["state"] is None else g
