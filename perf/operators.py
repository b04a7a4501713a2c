"""Calls of the token mixers that stand beside the scan, in the sizes and layouts in which they occur.

The encoders that the scan belongs to keep some attention sublayers between the
propagation ones, and the scan's counterpart over a sequence of tokens is a
linear recurrence with a matrix state.  Their operators, in the order in which a
sublayer calls them:

* norm_fwd / norm_bwd: the RMS norm of every query and key head, with the position
  rotation in the same pass, and its gradient.  q and k are slices of one fused
  projection [B][T][(Hq + 2 Hkv) D], as the projection leaves them.
* attn_fwd: attention with a window of `left` keys before and `right` keys behind
  the query's own position (-1: no bound) and the first `sinks` tokens, which no
  lower bound hides.  v is still the projection's slice.
* attn_train: the same and its gradient, one step of training.
* decode: one token (or a few) at the end of each sequence against its cache.
* delta_fwd: the gated delta rule, S_t = exp(g_t) (I - beta_t k_t k_t^T) S_{t-1} + beta_t k_t v_t^T
  with o_t = S_t^T q_t / sqrt(Dk), from a state and to one (fp32 [B][H][Dk][Dv]);
  one token a sequence is its serving form.
* delta_train: the same and its gradient.

`plain` forms are in 32 bits, rounded once at the end; `exact` is each operator's
definition in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6


def listed():
    return [
        # one decoding step's queries and keys: 8 sequences, one token each
        dict(name="norm_fwd-token", op="norm_fwd", B=8, T=1, Hq=16, Hkv=4, D=128, R=128, pairs="half", dtype="bf16"),
        # 74 x 74 tokens of 1152 channels, batch 32: the latent sublayer's second grid
        dict(name="norm_fwd-74x74", op="norm_fwd", B=32, T=5476, Hq=18, Hkv=18, D=64, R=64, pairs="half", dtype="bf16"),
        # the 64 x 64 training workload of 768 channels, batch 8
        dict(name="norm_bwd-64x64", op="norm_bwd", B=8, T=4096, Hq=12, Hkv=12, D=64, R=64, pairs="half", dtype="bf16"),
        # 185 x 185 tokens behind 4 register tokens of 1152 channels: 6 image rows either side
        dict(name="attn_fwd-185x185", op="attn_fwd", B=1, T=34229, Hq=18, Hkv=18, D=64, left=1110, right=1110, sinks=4, ragged=False, dtype="bf16"),
        # the 64 x 64 training workload behind 4 register tokens: 7 image rows either side
        dict(name="attn_train-64x64", op="attn_train", B=8, T=4100, Hq=12, Hkv=12, D=64, left=448, right=448, sinks=4, ragged=False, dtype="bf16"),
        # causal training on long sequences, four query heads to a key head, ragged lengths
        dict(name="attn_train-causal", op="attn_train", B=2, T=8192, Hq=16, Hkv=4, D=128, left=1023, right=0, sinks=4, ragged=True, dtype="bf16"),
        # an odd short step in fp32, heads of 72
        dict(name="attn_train-777-f32", op="attn_train", B=2, T=777, Hq=6, Hkv=6, D=72, left=100, right=60, sinks=1, ragged=False, dtype="f32"),
        # one token of one sequence with a window of 4096 in a cache of 32768: latency counts
        dict(name="decode-one", op="decode", B=1, T=1, Tk=32768, Hq=16, Hkv=4, D=128, left=4095, sinks=4, ragged=True, dtype="bf16"),
        # one token each of 64 sequences, the whole of ragged caches of up to 8192
        dict(name="decode-64", op="decode", B=64, T=1, Tk=8192, Hq=16, Hkv=4, D=128, left=-1, sinks=0, ragged=True, dtype="bf16"),
        # the 64 x 64 training workload as a sequence, 12 heads of 64
        dict(name="delta_train-64x64", op="delta_train", B=8, T=4096, Hq=12, Hv=12, D=64, Dv=64, ragged=False, dtype="bf16"),
        # long ragged sequences continued from a state, four value heads to a key head
        dict(name="delta_fwd-8191", op="delta_fwd", B=2, T=8191, Hq=4, Hv=16, D=128, Dv=128, ragged=True, dtype="bf16"),
        # one token each of 64 sequences
        dict(name="delta_fwd-token", op="delta_fwd", B=64, T=1, Hq=4, Hv=16, D=128, Dv=128, ragged=False, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    """A size between lo and hi, spread over its logarithm; odd or a small multiple of an odd one."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))) | rng.choice((1, 2, 4))))


def draw(rng):
    top = max(_cost(c) for c in listed())
    op = rng.choice(["norm_fwd", "norm_bwd", "attn_fwd", "attn_fwd", "attn_train", "attn_train", "decode", "decode", "delta_fwd", "delta_fwd", "delta_train"])
    while True:
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        Hkv = rng.choice([1, 2, 3, 4, 6, 8, 12, 16, 18])
        Hq = Hkv * rng.choice([1, 1, 2, 3, 4, 6, 8])
        if Hq > 32:
            continue
        D = rng.choice([32, 64, 64, 72, 80, 96, 104, 128, 128])
        c = dict(op=op, B=_log(rng, 1, 64), T=_log(rng, 1, 34225), Hq=Hq, Hkv=Hkv, D=D, dtype=dtype)
        if op.startswith("norm"):
            c.update(R=rng.choice([D, D, D // 2 // 4 * 4]), pairs=rng.choice(["half", "adjacent"]))
        elif op == "decode":
            c.update(T=rng.choice([1, 1, 1, 2, 5]), Tk=_log(rng, 16, 65536), sinks=rng.choice([0, 1, 4, 16]), ragged=True)
            c.update(left=rng.choice([-1, _log(rng, 16, 8192)]))
        elif op.startswith("delta"):
            c.update(B=_log(rng, 1, 16), T=min(c["T"], 8192), Hq=Hkv, Hv=Hq, D=rng.choice([32, 64, 96, 128]), Dv=rng.choice([32, 64, 96, 128]))
            c.update(T=1 if op == "delta_fwd" and rng.random() < 0.4 else c["T"], ragged=rng.choice([False, True]))
            c.pop("Hkv")
        else:
            c.update(left=rng.choice([-1, _log(rng, 16, 2048), _log(rng, 16, 2048)]), right=rng.choice([0, 0, -1, _log(rng, 16, 2048)]))
            c.update(sinks=rng.choice([0, 1, 4, 16]), ragged=rng.choice([False, True]))
        if dtype == "f32" and op.startswith("attn") and _cost(c) > top / 16:
            continue
        if op.startswith("delta") and c["B"] * c["T"] * c["Hv"] * c["D"] * c["Dv"] > 8 * 4096 * 12 * 64 * 64:
            continue
        if op.startswith("attn") and 4 * c["B"] * Hq * c["T"] * _span(c) > 12e9:   # what the plain form's scores take
            continue
        if _cost(c) <= top:
            return c


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _lens(c):
    """The sequences' lengths: whole, or ragged (the same for every seed)."""
    top = c["Tk"] if c["op"] == "decode" else c["T"]
    if not c.get("ragged"):
        return None
    return [max(1, top - (b * 769 + 767) % max(1, top // 2)) for b in range(c["B"])]


def _span(c):
    """Keys that the plain form looks at for one query."""
    if c["left"] < 0 or c["right"] < 0:
        return c["T"]
    return min(c["T"], 256 + c["left"] + c["right"]) + c["sinks"]


def _visible(c):
    """Pairs of a query and a key that it sees, over the batch, for one head."""
    total = 0
    Tk = c["Tk"] if c["op"] == "decode" else c["T"]
    right = 0 if c["op"] == "decode" else c["right"]
    for n in (_lens(c) or [Tk] * c["B"]):
        p = torch.arange(max(0, n - c["T"]), n) if c["op"] == "decode" else torch.arange(n)
        hi = torch.clamp(p + right, max=n - 1) if right >= 0 else torch.full_like(p, n - 1)
        lo = torch.clamp(p - c["left"], min=0) if c["left"] >= 0 else torch.zeros_like(p)
        sunk = torch.minimum(torch.clamp(lo, max=c["sinks"]), hi + 1)
        total += int((torch.clamp(hi - lo + 1, min=0) + sunk).sum())
    return total


def work(case):
    c, s = case, 2 if case["dtype"] == "bf16" else 4
    B, T, Hq, D = c["B"], c["T"], c["Hq"], c["D"]
    if c["op"].startswith("delta"):
        Hv, Dv = c["Hv"], c["Dv"]
        state, tokens = 8 * B * Hv * D * Dv, B * T * (2 * Hq * D + 2 * Hv * Dv + 2 * Hv) * s
        if c["op"] == "delta_fwd":
            return {"bytes": state + tokens, "flops": 6 * B * T * Hv * D * Dv}
        return {"bytes": 2 * state + 2 * tokens, "flops": 18 * B * T * Hv * D * Dv}
    Hkv = c["Hkv"]
    if c["op"].startswith("norm"):
        n = B * T * (Hq + Hkv) * D
        table = T * c["R"] * 4 + 2 * D * s
        if c["op"] == "norm_fwd":
            return {"bytes": 2 * n * s + table, "flops": 7 * n}
        return {"bytes": 3 * n * s + table + 2 * D * s, "flops": 16 * n}
    pairs = _visible(c) * Hq
    if c["op"] == "decode":
        keys = 0
        for n in _lens(c):
            seen = n if c["left"] < 0 else min(n, c["left"] + T) + min(c["sinks"], max(0, n - c["left"] - T))
            keys += seen
        return {"bytes": 2 * keys * Hkv * D * s + 2 * B * T * Hq * D * s, "flops": 4 * D * pairs}
    nq, nk = B * T * Hq * D * s, B * T * Hkv * D * s
    if c["op"] == "attn_fwd":
        return {"bytes": 2 * nq + 2 * nk + 4 * B * T * Hq, "flops": 4 * D * pairs}
    return {"bytes": 4 * nq + 4 * nk + 4 * B * T * Hq, "flops": 14 * D * pairs}


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def _table(T, R):
    """cos and sin of the rotation of R/2 pairs at T positions."""
    f = 10000.0 ** (-torch.arange(R // 2, device=DEV, dtype=torch.float64) * 2 / R)
    a = torch.arange(T, device=DEV, dtype=torch.float64)[:, None] * f
    return a.cos().float().contiguous(), a.sin().float().contiguous()


def prepare(case, seed):
    c, dt = case, _dtype(case)
    B, T, Hq, D = c["B"], c["T"], c["Hq"], c["D"]
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def rand(*shape):
        return torch.randn(*shape, device=DEV, dtype=dt, generator=g)

    st = {"case": c}
    lens = _lens(c)
    st["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV) if lens else None
    if c["op"].startswith("delta"):
        Hv, Dv = c["Hv"], c["Dv"]
        unit = torch.nn.functional.normalize
        st.update(q=unit(rand(B, T, Hq, D).float(), dim=-1).to(dt), k=unit(rand(B, T, Hq, D).float(), dim=-1).to(dt), v=rand(B, T, Hv, Dv))
        # decays whose memory is some ten to a thousand tokens, and how much of a value is written
        st["g"] = (-torch.exp(rand(B, T, Hv).float() - 4)).to(dt)
        st["beta"] = torch.sigmoid(rand(B, T, Hv).float()).to(dt)
        st["state"] = 0.1 * torch.randn(B, Hv, D, Dv, device=DEV, generator=g)
        if c["op"] == "delta_train":
            st["do"] = rand(B, T, Hv, Dv)
            st["dstate"] = 0.1 * torch.randn(B, Hv, D, Dv, device=DEV, generator=g)
        return st
    Hkv = c["Hkv"]
    if c["op"] == "decode":
        st.update(q=rand(B, T, Hq, D), k=rand(B, c["Tk"], Hkv, D), v=rand(B, c["Tk"], Hkv, D))
        return st
    fused = rand(B, T, Hq + 2 * Hkv, D)
    q, k, v = fused[:, :, :Hq], fused[:, :, Hq:Hq + Hkv], fused[:, :, Hq + Hkv:]
    if c["op"].startswith("norm"):
        st.update(q=q, k=k, wq=1 + 0.1 * rand(D), wk=1 + 0.1 * rand(D))
        st["cos"], st["sin"] = _table(T, c["R"])
        if c["op"] == "norm_bwd":
            st.update(dyq=rand(B, T, Hq, D), dyk=rand(B, T, Hkv, D))
        return st
    st.update(q=q.contiguous(), k=k.contiguous(), v=v)
    if c["op"] == "attn_train":
        st["do"] = rand(B, T, Hq, D)
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    c = state["case"]
    return _run_own(c, state) if own else _run_plain(c, state)


def _run_own(c, s):
    import paper_2606_00746_amd as gspn
    if c["op"] == "norm_fwd":
        return gspn.qk_norm_rotate_fwd(s["q"], s["k"], s["wq"], s["wk"], s["cos"], s["sin"], eps=EPS, pairs=c["pairs"])
    if c["op"] == "norm_bwd":
        return gspn.qk_norm_rotate_bwd(s["q"], s["k"], s["wq"], s["wk"], s["dyq"], s["dyk"], s["cos"], s["sin"], eps=EPS, pairs=c["pairs"])
    if c["op"] == "decode":
        return gspn.window_attn_decode(s["q"], s["k"], s["v"], s["lens"], left=c["left"], sinks=c["sinks"])
    if c["op"] == "delta_fwd":
        return gspn.delta_rule_fwd(s["q"], s["k"], s["v"], s["g"], s["beta"], state=s["state"], lens=s["lens"])
    if c["op"] == "delta_train":
        x = (s["q"], s["k"], s["v"], s["g"], s["beta"])
        o, end, reserve = gspn.delta_rule_fwd_train(*x, state=s["state"], lens=s["lens"])
        return (o, end, *gspn.delta_rule_bwd_reserve(*x, s["do"], reserve, dstate=s["dstate"], state=s["state"], lens=s["lens"]))
    mask = dict(left=c["left"], right=c["right"], sinks=c["sinks"], lens=s["lens"])
    o, lse = gspn.window_attn_fwd(s["q"], s["k"], s["v"], **mask)
    if c["op"] == "attn_fwd":
        return o, lse
    return (o, *gspn.window_attn_bwd(s["q"], s["k"], s["v"], o, lse, s["do"], **mask))


def _run_plain(c, s):
    if c["op"] == "norm_fwd":
        return tuple(_norm(s[x], s["w" + x], s["cos"], s["sin"], c["pairs"]) for x in "qk")
    if c["op"] == "norm_bwd":
        (dq, dwq), (dk, dwk) = (_norm_grad(s[x], s["w" + x], s["dy" + x], s["cos"], s["sin"], c["pairs"]) for x in "qk")
        return dq, dk, dwq, dwk
    if c["op"] == "decode":
        return _decode(c, s)
    if c["op"] == "delta_fwd":
        return _delta(c, s, *(s[x].float() for x in ("q", "k", "v", "g", "beta", "state")))
    if c["op"] == "delta_train":
        x = [s[n].float().requires_grad_() for n in ("q", "k", "v", "g", "beta", "state")]
        o, end = _delta(c, s, *x)
        grads = torch.autograd.grad((o, end), x, (s["do"], s["dstate"]))
        return (o.detach(), end.detach(), *(d.to(s[n].dtype) for d, n in zip(grads, ("q", "k", "v", "g", "beta", "state"))))
    return _attn(c, s)


def _turn(x, cos, sin, pairs):
    """x [B][T][H][D] with its first R entries rotated; R = 2 * cos.shape[1]."""
    r = cos.shape[1]
    cos, sin = cos[None, :, None], sin[None, :, None]
    part, rest = x[..., :2 * r], x[..., 2 * r:]
    a, b = (part[..., :r], part[..., r:]) if pairs == "half" else (part[..., 0::2], part[..., 1::2])
    a, b = a * cos - b * sin, a * sin + b * cos
    part = torch.cat((a, b), -1) if pairs == "half" else torch.stack((a, b), -1).flatten(-2)
    return torch.cat((part, rest), -1)


def _norm(x, w, cos, sin, pairs):
    f = x.float()
    f = f * torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS) * w.float()
    return _turn(f, cos, sin, pairs).to(x.dtype)


def _norm_grad(x, w, dy, cos, sin, pairs):
    f = x.float()
    r = torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS)
    f = f * r
    d = _turn(dy.float(), cos, -sin, pairs)
    dw = (d * f).sum((0, 1, 2))
    d = d * w.float()
    dx = r * (d - f * (d * f).mean(-1, keepdim=True))
    return dx.to(x.dtype), dw.to(w.dtype)


def _softmax(s):
    """exp(s - max), its sum and the log of the whole sum over the last axis; rows of -inf give zeros and -inf."""
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = (s - m).exp_()
    z = p.sum(-1, keepdim=True)
    return p / torch.where(z == 0, torch.ones_like(z), z), (m + z.log()).squeeze(-1)


def _attn(c, s):
    """The windowed form: blocks of `n` queries, each with the `span` keys that its window may reach, and the sinks beside them."""
    q, k, v = (s[x].float() for x in "qkv")
    B, T, Hq, D = q.shape
    Hkv, left, right, sinks = c["Hkv"], c["left"], c["right"], c["sinks"]
    whole = _span(c) >= T
    lo, hi = (T if left < 0 else left), (T if right < 0 else right)   # no bound: as far as the sequence
    n = T if whole else 256
    span, first = (T, 0) if whole else (n + left + right, left)
    nb = -(-T // n)
    sinks = 0 if whole else min(sinks, T)
    pad = torch.nn.functional.pad
    back = (nb - 1) * n + span - first - T
    q = pad(q, (0, 0, 0, 0, 0, nb * n - T)).view(B, nb, n, Hkv, Hq // Hkv, D).permute(0, 3, 4, 1, 2, 5)
    k, v = (x.permute(0, 2, 1, 3) for x in (k, v))
    kb, vb = (pad(x, (0, 0, first, max(0, back))).unfold(2, span, n)[:, :, :nb].transpose(-1, -2).unsqueeze(2) for x in (k, v))
    ks, vs = (x[:, :, None, None, :sinks] for x in (k, v))
    p = torch.arange(nb * n, device=DEV).view(nb, n, 1)
    j = (torch.arange(nb, device=DEV) * n - first)[:, None, None] + torch.arange(span, device=DEV)
    end = (s["lens"] if s["lens"] is not None else torch.full((B,), T, device=DEV)).view(B, 1, 1, 1, 1, 1)
    in_window = (j >= p - lo) if not whole else (j >= p - lo) | (j < c["sinks"])
    see = (in_window & (j >= 0) & (j <= p + hi))[None, None, None] & (j < end) & (p < end)
    sink = torch.arange(sinks, device=DEV)
    see_s = ((sink < p - lo) & (sink <= p + hi))[None, None, None] & (sink < end) & (p < end)
    see = torch.cat((see, see_s.expand(*see.shape[:-1], sinks)), -1)
    scale = 1 / math.sqrt(D)
    scores = torch.cat((q @ kb.transpose(-1, -2), q @ ks.transpose(-1, -2)), -1) * scale
    w, lse = _softmax(scores.masked_fill_(~see, -math.inf))
    del scores, see
    o = w[..., :span] @ vb + w[..., span:] @ vs

    def rows(x):   # [B][Hkv][g][nb][n][D] as [B][T][Hq][D]
        return x.permute(0, 3, 4, 1, 2, 5).reshape(B, nb * n, Hq, D)[:, :T].to(s["q"].dtype)

    if c["op"] == "attn_fwd":
        return rows(o), lse.reshape(B, Hq, nb * n)[..., :T].contiguous()
    d = pad(s["do"].float(), (0, 0, 0, 0, 0, nb * n - T)).view(B, nb, n, Hkv, Hq // Hkv, D).permute(0, 3, 4, 1, 2, 5)
    dp = torch.cat((d @ vb.transpose(-1, -2), d @ vs.transpose(-1, -2)), -1)
    ds = w * (dp - (d * o).sum(-1, keepdim=True)) * scale
    del dp
    dq = ds[..., :span] @ kb + ds[..., span:] @ ks
    at = (j + first).reshape(-1)

    def keys(x, y):   # x^T y, the blocks' and heads' shares of a key added up
        out = torch.zeros(B, Hkv, first + T + max(0, back), D, device=DEV)
        share = (x[..., :span].transpose(-1, -2) @ y).sum(2)
        out.index_add_(2, at, share.reshape(B, Hkv, nb * span, D))
        out = out[:, :, first:first + T]
        out[:, :, :sinks] += (x[..., span:].transpose(-1, -2) @ y).sum((2, 3))
        return out.permute(0, 2, 1, 3).to(s["q"].dtype)

    return rows(o), rows(dq), keys(ds, q), keys(w, d)


def _decode(c, s):
    B, T, Hq, D = s["q"].shape
    Tk, Hkv = c["Tk"], c["Hkv"]
    n = s["lens"].long()
    if c["left"] < 0 or c["left"] + T + c["sinks"] >= Tk:
        j = torch.arange(Tk, device=DEV).expand(B, Tk)
        k, v = s["k"].float(), s["v"].float()
        twice = torch.zeros_like(j, dtype=torch.bool)
    else:   # the sinks and the window's keys
        back = torch.arange(c["left"] + T, device=DEV)
        j = n[:, None] - (c["left"] + T) + back
        j = torch.cat((torch.arange(c["sinks"], device=DEV).expand(B, -1), j), 1)
        twice = (j < c["sinks"]) & (torch.arange(j.shape[1], device=DEV) >= c["sinks"])
        at = j.clamp(0, Tk - 1)
        b = torch.arange(B, device=DEV)[:, None]
        k, v = s["k"][b, at].float(), s["v"][b, at].float()
    p = (n[:, None] - T + torch.arange(T, device=DEV))[:, :, None]
    j, twice = j[:, None], twice[:, None]
    see = (j <= p) & (p >= 0) & (j >= 0) & ~twice & ((j < c["sinks"]) | ((j >= p - c["left"]) if c["left"] >= 0 else (j >= 0)))
    q = s["q"].float().view(B, T, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, Hq // Hkv * T, D)
    scores = q @ k.permute(0, 2, 3, 1) * (1 / math.sqrt(D))
    see = see[:, None, None].expand(B, Hkv, Hq // Hkv, T, -1).reshape(scores.shape)
    w, _ = _softmax(scores.masked_fill_(~see, -math.inf))
    o = w @ v.permute(0, 2, 1, 3)
    return o.view(B, Hkv, Hq // Hkv, T, D).permute(0, 3, 1, 2, 4).reshape(B, T, Hq, D).to(s["q"].dtype)


def _delta(c, s, q, k, v, g, beta, state):
    """The chunked form: within a chunk of n tokens U = (I + L)^-1 beta (V - exp(G) K S), L strictly lower
    triangular, and the state S once a chunk; (I + L)^-1 as a product of (I + (-L)^(2^i))."""
    B, T, Hv, Dv = v.shape
    D, rep = c["D"], Hv // c["Hq"]
    n = min(64, T)
    nc = -(-T // n)
    live = None
    if s["lens"] is not None:   # tokens past a sequence's end write nothing and decay nothing
        live = (torch.arange(T, device=DEV) < s["lens"][:, None])[:, :, None]
        g, beta = g * live, beta * live

    def chunks(x):   # [B][T][H]... as [B][H][nc][n]...
        x = torch.nn.functional.pad(x, (0, 0) * (x.dim() - 2) + (0, nc * n - T)).unflatten(1, (nc, n))
        return x.movedim(3, 1)

    q, k = (chunks(x).repeat_interleave(rep, 1) for x in (q, k))
    v, g, beta = chunks(v), chunks(g), chunks(beta)
    G = g.cumsum(-1)
    lower = torch.ones(n, n, device=DEV, dtype=torch.bool).tril()
    decay = torch.exp((G[..., :, None] - G[..., None, :]).masked_fill(~lower, -math.inf))
    m = -(k @ k.transpose(-1, -2)) * decay * beta[..., None]
    m = m.tril(-1)
    inv = torch.eye(n, device=DEV) + m
    for _ in range(max(0, (n - 1).bit_length() - 1)):
        m = m @ m
        inv = inv + inv @ m
    u0 = inv @ (beta[..., None] * v)
    w = inv @ ((beta * G.exp())[..., None] * k)
    a = (q @ k.transpose(-1, -2)) * decay / math.sqrt(D)
    qd = q * (G.exp() / math.sqrt(D))[..., None]
    kd = (k * (G[..., -1:] - G).exp()[..., None]).transpose(-1, -2)
    end = G[..., -1].exp()
    out = []
    for i in range(nc):
        u = u0[:, :, i] - w[:, :, i] @ state
        out.append(qd[:, :, i] @ state + a[:, :, i] @ u)
        state = end[:, :, i, None, None] * state + kd[:, :, i] @ u
    o = torch.stack(out, 2).flatten(2, 3)[:, :, :T].transpose(1, 2)
    if live is not None:
        o = o * live[..., None]
    return o.to(s["v"].dtype), state


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "norm_fwd":
        return tuple(_exact_norm(c, s, x)[0] for x in "qk")
    if c["op"] == "norm_bwd":
        a, b = _exact_norm(c, s, "q"), _exact_norm(c, s, "k")
        return a[1], b[1], a[2], b[2]
    if c["op"].startswith("delta"):
        return _exact_delta(c, s)
    return _exact_attn(c, s)


def _exact_delta(c, s):
    """Token by token, and for the gradient back again over the states that were kept."""
    B, T, Hv, Dv = s["v"].shape
    D, rep, train = c["D"], Hv // c["Hq"], c["op"] == "delta_train"
    if train and 8 * B * Hv * D * Dv * T > 60e9:
        return None
    q, k = (s[x].double().repeat_interleave(rep, 2) for x in "qk")
    v, g, beta, S = (s[x].double() for x in ("v", "g", "beta", "state"))
    live = torch.ones(B, T, device=DEV, dtype=torch.float64)
    if s["lens"] is not None:
        live = (torch.arange(T, device=DEV) < s["lens"][:, None]).double()
    a = torch.exp(g * live[..., None])
    beta = beta * live[..., None]
    q = q * live[..., None, None] / math.sqrt(D)
    o = torch.zeros(B, T, Hv, Dv, device=DEV, dtype=torch.float64)
    kept = []
    for t in range(T):
        kept.append(S) if train else None
        S = a[:, t, :, None, None] * S
        u = beta[:, t, :, None] * (v[:, t] - (S * k[:, t, :, :, None]).sum(2))
        S = S + k[:, t, :, :, None] * u[:, :, None]
        o[:, t] = (S * q[:, t, :, :, None]).sum(2)
    if not train:
        return o, S
    end, dS, do = S, s["dstate"].double(), s["do"].double()
    dq, dk, dv, dg, db = (torch.zeros_like(x) for x in (q, k, v, g, beta))
    for t in reversed(range(T)):
        kt = k[:, t, :, :, None]
        before = a[:, t, :, None, None] * kept[t]
        z = v[:, t] - (before * kt).sum(2)
        u = beta[:, t, :, None] * z
        S = before + kt * u[:, :, None]
        dq[:, t] = (S * do[:, t, :, None]).sum(-1)
        dS = dS + q[:, t, :, :, None] * do[:, t, :, None]
        du = (dS * kt).sum(2)
        dk[:, t] = (dS * u[:, :, None]).sum(-1)
        db[:, t] = (du * z).sum(-1)
        dz = beta[:, t, :, None] * du
        dv[:, t] = dz
        dk[:, t] -= (before * dz[:, :, None]).sum(-1)
        dS = dS - kt * dz[:, :, None]
        dg[:, t] = (dS * before).sum((-1, -2))
        dS = a[:, t, :, None, None] * dS
    dq = dq * live[..., None, None] / math.sqrt(D)
    dq, dk = (x.unflatten(2, (c["Hq"], rep)).sum(3) for x in (dq, dk))
    return o, end, dq, dk, dv, dg * live[..., None], db * live[..., None], dS


def _exact_norm(c, s, which):
    """y_r = R_t (w x / rms(x)) by a rotation matrix for each position; the gradient by the chain rule through it."""
    x, w = s[which].double(), s["w" + which].double()
    D, R = c["D"], c["R"]
    i = torch.arange(R // 2, device=DEV)
    a, b = (i, i + R // 2) if c["pairs"] == "half" else (2 * i, 2 * i + 1)
    cos, sin = s["cos"].double()[None, :, None], s["sin"].double()[None, :, None]
    rms = (x.pow(2).sum(-1, keepdim=True) / D + EPS).sqrt()
    n = x / rms
    y = n * w
    ya, yb = y[..., a], y[..., b]
    y = y.clone()
    y[..., a], y[..., b] = ya * cos - yb * sin, yb * cos + ya * sin
    if c["op"] == "norm_fwd":
        return y, None, None
    dy = s["dy" + which].double()
    da, db = dy[..., a], dy[..., b]
    t = dy.clone()
    t[..., a], t[..., b] = da * cos + db * sin, db * cos - da * sin
    dw = (t * n).flatten(0, 2).sum(0)
    t = t * w
    return y, t / rms - x * ((t * x).sum(-1, keepdim=True) / (D * rms.pow(3))), dw


def _exact_attn(c, s):
    """Query by query over all keys, in slices of the queries of one head."""
    B, T, Hq, D = s["q"].shape
    Tk = s["k"].shape[1]
    decode, train = c["op"] == "decode", c["op"] == "attn_train"
    lens = _lens(c) or [Tk] * B
    right = 0 if decode else c["right"]
    o = torch.zeros(B, T, Hq, D, dtype=torch.float64, device=DEV)
    lse = torch.full((B, Hq, T), -math.inf, dtype=torch.float64, device=DEV)
    if train:
        dq, dk, dv = (torch.zeros_like(s[x], dtype=torch.float64) for x in "qkv")
    j = torch.arange(Tk, device=DEV)
    step = max(1, 1 << 25) // max(Tk, 1) + 1
    for b in range(B):
        n = lens[b]
        for h in range(Hq):
            g = h // (Hq // c["Hkv"])
            k, v = s["k"][b, :n, g].double(), s["v"][b, :n, g].double()
            for t in range(0, T, step):
                at = torch.arange(t, min(T, t + step), device=DEV)
                p = at + (n - T if decode else 0)
                keep = (p >= 0) & (p < n)
                at, p = at[keep], p[keep][:, None]
                if not len(at):
                    continue
                see = torch.ones(len(at), n, dtype=torch.bool, device=DEV)
                if right >= 0:
                    see &= j[:n] <= p + right
                if c["left"] >= 0:
                    see &= (j[:n] >= p - c["left"]) | (j[:n] < c["sinks"])
                q = s["q"][b, at, h].double()
                x = (q @ k.T / math.sqrt(D)).masked_fill(~see, -math.inf)
                e = torch.logsumexp(x, -1)
                w = torch.exp(x - torch.where(e == -math.inf, 0.0, e)[:, None])
                out = w @ v
                o[b, at, h], lse[b, h, at] = out, e
                if train:
                    d = s["do"][b, at, h].double()
                    ds = w * (d @ v.T - (d * out).sum(-1, keepdim=True)) / math.sqrt(D)
                    dq[b, at, h] = ds @ k
                    dk[b, :n, g] += ds.T @ q
                    dv[b, :n, g] += w.T @ d
    if decode:
        return o
    return (o, dq, dk, dv) if train else (o, lse)
