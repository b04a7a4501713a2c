"""The gated delta rule (gspn_delta_rule_fwd, _fwd_train, _bwd_reserve) against the
recurrence in 64 bits, token by token, on inputs that are exact in the storage type.

Bounds, by the largest entry of an output: every output is one rounding (u = 2^-8 of
the entry itself for bf16, 2^-24 for fp32 and for states) of what fp32 arithmetic
gives.  That is off by the products' roundings, each 2^-24 of its absolute terms.  An
entry is a sum over at most 64 tokens of a chunk and 128 entries of a head, three
products deep, and what a chunk adds to the state's error decays as the state does
(|I - beta k k^T| <= 1): f = 2^-24 * 3 * (64 + 128) times the largest entry, for
forward outputs.  Gradients pass twice through it, and sum such terms over up to the
4 heads that share a key and, for dg, over the rest of the chunk, whose terms cancel:
16 f.  With keys of unit length, inverses of chunks of like keys stay below 2 in
every entry, which the last test drives at."""
import numpy as np
import pytest

import mixers_ref as ref
import paper_2606_00746_amd as gspn
from gpu_util import require_gpu, to_host
from test_attention_gpu import dev, within

pytestmark = pytest.mark.gpu

F = 2.0 ** -24 * 3 * (64 + 128)


def make(B, T, Hq, Hv, Dk, Dv, dtype, seed, decay=-3.0, alike=0.0):
    rng = np.random.default_rng(seed)
    unit = lambda x: x / np.linalg.norm(x, axis=-1, keepdims=True)
    x = {n: unit(rng.standard_normal((B, T, Hq, Dk)) + alike) for n in "qk"}
    x["v"] = rng.standard_normal((B, T, Hv, Dv))
    x["g"] = -np.exp(rng.standard_normal((B, T, Hv)) + decay)
    x["beta"] = 1 / (1 + np.exp(-rng.standard_normal((B, T, Hv))))
    x["do"] = rng.standard_normal((B, T, Hv, Dv))
    x = {n: ref.store(a, dtype) for n, a in x.items()}
    x["state"], x["dstate"] = (ref.store(rng.standard_normal((B, Hv, Dk, Dv)), "f32") for _ in range(2))
    return x


NAMES = ("dq", "dk", "dv", "dg", "dbeta", "dstate")


def expect(x, scale, lens=None, grads=True):
    B, T, Hv, Dv = x["v"].shape
    Hq = x["q"].shape[2]
    want = {"o": np.zeros_like(x["v"]), "state": np.zeros_like(x["state"])}
    if grads:
        want.update(dq=np.zeros_like(x["q"]), dk=np.zeros_like(x["k"]), dv=np.zeros_like(x["v"]),
                    dg=np.zeros_like(x["g"]), dbeta=np.zeros_like(x["g"]), dstate=np.zeros_like(x["state"]))
    for b in range(B):
        n = T if lens is None else min(max(lens[b], 0), T)
        for h in range(Hv):
            j = h // (Hv // Hq)
            r = ref.delta_rule(x["q"][b, :n, j], x["k"][b, :n, j], x["v"][b, :n, h], x["g"][b, :n, h],
                               x["beta"][b, :n, h], x["state"][b, h], scale,
                               x["do"][b, :n, h] if grads else None, x["dstate"][b, h] if grads else None)
            want["o"][b, :n, h], want["state"][b, h] = r["o"], r["state"]
            if grads:
                want["dq"][b, :n, j] += r["dq"]
                want["dk"][b, :n, j] += r["dk"]
                for m in ("dv", "dg", "dbeta"):
                    want[m][b, :n, h] = r[m]
                want["dstate"][b, h] = r["dstate"]
    return want


def check(got, want, dtype):
    for n, t in got.items():
        u = 2.0 ** -8 if dtype == "bf16" and n not in ("state", "dstate") else 2.0 ** -24
        f = F if n in ("o", "state") else 16 * F
        within(n, to_host(t), want[n], u * np.abs(want[n]) + f * np.abs(want[n]).max(initial=0.0) + 1e-37)


CASES = [
    # B, T, Hq, Hv, Dk, Dv, lens
    (1, 1, 1, 1, 64, 64, None),
    (2, 64, 2, 2, 64, 64, None),
    (1, 65, 1, 1, 64, 64, None),
    (2, 200, 2, 4, 128, 128, [200, 130]),
    (1, 333, 1, 3, 32, 96, None),
    (3, 130, 1, 2, 72, 40, [0, 1, 130]),
    (1, 77, 3, 3, 8, 8, None),
    (1, 100, 1, 4, 104, 16, None),
    (1, 300, 1, 1, 16, 120, [257]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[:6])))
def test_training_pair(case, dtype):
    torch = require_gpu()
    *sizes, lens = case
    x = make(*sizes, dtype, seed=sizes[1] + sizes[4])
    t = {n: dev(a, "f32" if "state" in n else dtype) for n, a in x.items()}
    ln = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    args = [t[n] for n in ("q", "k", "v", "g", "beta")]
    o, end, reserve = gspn.delta_rule_fwd_train(*args, state=t["state"], lens=ln)
    grads = gspn.delta_rule_bwd_reserve(*args, t["do"], reserve, dstate=t["dstate"], state=t["state"], lens=ln)
    want = expect(x, sizes[4] ** -0.5, lens)
    check({"o": o, "state": end, **dict(zip(NAMES, grads))}, want, dtype)
    if sizes[1] > 8:   # the same without a reserve, bit for bit
        a, b = gspn.delta_rule_fwd(*args, state=t["state"], lens=ln)
        assert torch.equal(a, o) and torch.equal(b, end)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_states(dtype):
    """From zeros, with no gradient of the last state."""
    x = make(1, 150, 2, 2, 64, 32, dtype, seed=6)
    x["state"][:], x["dstate"][:] = 0, 0
    args = [dev(x[n], dtype) for n in ("q", "k", "v", "g", "beta")]
    o, end, reserve = gspn.delta_rule_fwd_train(*args, scale=1.0)
    *grads, none = gspn.delta_rule_bwd_reserve(*args, dev(x["do"], dtype), reserve, scale=1.0)
    assert none is None
    check({"o": o, "state": end, **dict(zip(NAMES, grads))}, expect(x, 1.0), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [(2, 1, 2, 4, 128, 128, None), (3, 1, 1, 1, 72, 40, [1, 0, 1]),
                                  (1, 5, 1, 2, 64, 96, [3]), (2, 8, 3, 3, 8, 8, None)],
                         ids=lambda c: "x".join(map(str, c[:6])))
def test_single_tokens(case, dtype):
    torch = require_gpu()
    *sizes, lens = case
    x = make(*sizes, dtype, seed=3)
    t = {n: dev(a, "f32" if "state" in n else dtype) for n, a in x.items()}
    ln = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    args = [t[n] for n in ("q", "k", "v", "g", "beta")]
    o, end = gspn.delta_rule_fwd(*args, state=t["state"], lens=ln)
    check({"o": o, "state": end}, expect(x, sizes[4] ** -0.5, lens, grads=False), dtype)
    keep = t["state"].clone()   # in place
    o2, end2 = gspn.delta_rule_fwd(*args, state=keep, state_out=keep, lens=ln)
    assert end2 is keep and torch.equal(o, o2) and torch.equal(end, keep)


def test_tokens_one_by_one_meet_the_chunks():
    """A prefill in chunks, then single tokens, is the sequence at once."""
    torch = require_gpu()
    x = make(2, 140, 1, 2, 64, 64, "f32", seed=12)
    t = {n: dev(a, "f32") for n, a in x.items()}
    names = ("q", "k", "v", "g", "beta")
    parts, state = [], t["state"]
    for a, b in [(0, 100)] + [(i, i + 1) for i in range(100, 130)] + [(130, 140)]:
        o, state = gspn.delta_rule_fwd(*[t[n][:, a:b].contiguous() for n in names], state=state)
        parts.append(o)
    check({"o": torch.cat(parts, 1), "state": state}, expect(x, 0.125, grads=False), "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_padding_may_hold_anything(dtype):
    torch = require_gpu()
    got = []
    for bad in (0.0, float("nan"), float("inf")):
        x = make(2, 150, 1, 2, 64, 64, dtype, seed=2)
        t = {n: dev(a, "f32" if "state" in n else dtype) for n, a in x.items()}
        lens = [90, 3]
        for n in ("q", "k", "v", "g", "beta", "do"):
            for b in range(2):
                t[n][b, lens[b]:] = bad
        ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
        args = [t[n] for n in ("q", "k", "v", "g", "beta")]
        o, end, reserve = gspn.delta_rule_fwd_train(*args, state=t["state"], lens=ln)
        grads = gspn.delta_rule_bwd_reserve(*args, t["do"], reserve, dstate=t["dstate"], state=t["state"], lens=ln)
        s = gspn.delta_rule_fwd(*[a[:, :5].contiguous() for a in args], state=t["state"],
                                lens=torch.clamp(ln, max=5))
        got.append([o, end, *grads, *s])
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_hard_gates(dtype):
    """Tokens that forget everything (g = -inf and -1000), that keep everything (g = 0),
    and that write nothing (beta = 0) or everything (beta = 1)."""
    torch = require_gpu()
    x = make(1, 140, 1, 2, 64, 64, dtype, seed=15)
    x["g"][0, 5::17], x["g"][0, 9::17], x["g"][0, 11::17] = -np.inf, -1000.0, 0.0
    x["beta"][0, 3::11], x["beta"][0, 4::11] = 0.0, 1.0
    t = {n: dev(a, "f32" if "state" in n else dtype) for n, a in x.items()}
    args = [t[n] for n in ("q", "k", "v", "g", "beta")]
    o, end, reserve = gspn.delta_rule_fwd_train(*args, state=t["state"])
    grads = gspn.delta_rule_bwd_reserve(*args, t["do"], reserve, dstate=t["dstate"], state=t["state"])
    # some eight gates of -100 in a chunk take its running sum to 800, whose fp32 steps are
    # 2^-14: a decay after them is off by up to 2^-14 of itself, each way
    want = expect(x, 0.125)
    for n, a in {"o": o, "state": end, **dict(zip(NAMES, grads))}.items():
        u = 2.0 ** -8 if dtype == "bf16" and "state" not in n else 2.0 ** -24
        within(n, to_host(a), want[n], u * np.abs(want[n]) + (16 * F + 2.0 ** -12) * np.abs(want[n]).max() + 1e-37)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_like_keys(dtype):
    """Keys that all but repeat, written in full: the chunk's triangular system is as
    far from the identity as it gets."""
    x = make(1, 192, 1, 1, 64, 64, dtype, seed=17, decay=-9.0, alike=6.0)
    x["beta"][:] = 1.0
    t = {n: dev(a, "f32" if "state" in n else dtype) for n, a in x.items()}
    args = [t[n] for n in ("q", "k", "v", "g", "beta")]
    o, end, reserve = gspn.delta_rule_fwd_train(*args, state=t["state"])
    grads = gspn.delta_rule_bwd_reserve(*args, t["do"], reserve, dstate=t["dstate"], state=t["state"])
    check({"o": o, "state": end, **dict(zip(NAMES, grads))}, expect(x, 0.125), dtype)


def test_strides():
    torch = require_gpu()
    x = make(2, 100, 2, 2, 64, 64, "bf16", seed=5)
    t = {n: dev(a, "f32" if "state" in n else "bf16") for n, a in x.items()}
    args = [t[n] for n in ("q", "k", "v", "g", "beta")]
    fused = torch.cat(args[:3], 2)
    s = [fused[:, :, :2], fused[:, :, 2:4], fused[:, :, 4:]] + args[3:]
    o, end, reserve = gspn.delta_rule_fwd_train(*args)
    o2, end2, reserve2 = gspn.delta_rule_fwd_train(*s)
    assert torch.equal(o, o2) and torch.equal(end, end2)
    grads = gspn.delta_rule_bwd_reserve(*args, t["do"], reserve)
    df = torch.full_like(fused, float("nan"))
    out = (df[:, :, :2], df[:, :, 2:4], df[:, :, 4:], torch.empty_like(t["g"]), torch.empty_like(t["g"]), None)
    gspn.delta_rule_bwd_reserve(*s, t["do"], reserve2, out=out)
    for a, b in zip(grads[:5], out[:5]):
        assert torch.equal(a, b)


def test_gradient_against_differences():
    torch = require_gpu()
    x = make(1, 90, 1, 2, 32, 32, "f32", seed=31)
    t = {n: dev(a, "f32") for n, a in x.items()}
    names = ("q", "k", "v", "g", "beta", "state")
    o, end, reserve = gspn.delta_rule_fwd_train(*[t[n] for n in names])
    grads = gspn.delta_rule_bwd_reserve(*[t[n] for n in names[:5]], t["do"], reserve, dstate=t["dstate"],
                                        state=t["state"])
    h = 3e-3
    for i, n in enumerate(names):
        torch.manual_seed(i)
        d = torch.randn_like(t[n])
        d /= d.norm()
        sums = []
        for e in (h, -h):
            a = [t[m] + e * d if m == n else t[m] for m in names]
            o, end = gspn.delta_rule_fwd(*a)
            sums.append(float((o.double() * t["do"].double()).sum() + (end.double() * t["dstate"].double()).sum()))
        num, ana = (sums[0] - sums[1]) / (2 * h), float((grads[i].double() * d.double()).sum())
        assert abs(num - ana) <= 2e-2 * float(grads[i].double().norm()) + 1e-2, (n, num, ana)
