"""The selective state space scan (gspn_selective_scan_fwd, _fwd_train, _bwd_reserve) against
the recurrence in 64 bits, token by token, on inputs that are exact in the storage type.  An
output is one rounding (2^-8 of itself for bf16, 2^-24 for fp32, states and the gradients of
A, D and dt_bias) of what fp32 arithmetic gives, which is off by at most what sublayer_ref
counts.  Sums over channels: up to 2 in a lane, 16 rows of lanes of 4 waves by up to 16, the
workgroups' of a group (up to 3 here): a depth of 25 at most.  Sums over tokens: a lane's own (T), 3 of lanes,
64 rows of shares with 8 each: T + 75."""
import numpy as np
import pytest

import mixers_ref
import paper_2606_00746_amd as gspn
import sublayer_ref as ref
from gpu_util import require_gpu, to_host
from test_attention_gpu import dev, within

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
F32 = ("A", "D", "bias", "state", "dend")
WIDE = ("end", "dA", "dD", "dbias", "dstate")      # fp32 whatever the storage type
GRADS = ("dx", "ddt", "dA", "dB", "dC", "dD", "dz", "dbias", "dstate")


def make(b, T, C, G, N, dtype, seed, lo=1e-3, hi=0.3):
    rng = np.random.default_rng(seed)
    n = rng.standard_normal
    step = np.exp(rng.uniform(np.log(lo), np.log(hi), C))
    x = dict(x=n((b, T, C)), dt=0.5 * n((b, T, C)), A=-np.exp(0.7 * n((C, N))) * rng.uniform(0.5, N, (C, N)), B=n((b, T, G, N)),
             C=n((b, T, G, N)), D=n(C), z=n((b, T, C)), bias=np.log(np.expm1(step)), state=n((b, C, N)),
             dy=n((b, T, C)), dend=n((b, C, N)))
    return {k: mixers_ref.store(a, "f32" if k in F32 else dtype) for k, a in x.items()}


def expect(x, lens, without=(), soft=True, grads=True):
    b, T, C = x["x"].shape
    G = x["B"].shape[2]
    x = {k: np.zeros_like(a) if k in without else a for k, a in x.items()}
    out = {}
    for i in range(b):
        wide = [x[k][i].repeat(C // G, 1) for k in "BC"]
        r = ref.scan(x["x"][i], x["dt"][i], x["A"], *wide, x["D"], None if "z" in without else x["z"][i], x["bias"], x["state"][i],
                     T if lens is None else min(max(lens[i], 0), T), soft, x["dy"][i] if grads else None, x["dend"][i],
                     T + 75, 25)
        for k, v in r.items():
            if k.replace("e_", "") in ("dB", "dC"):
                v = v.reshape(T, G, C // G, -1).sum(2)
            out.setdefault(k, []).append(v)
    return {k: np.stack(v).sum(0) if k.replace("e_", "") in ("dA", "dD", "dbias") else np.stack(v) for k, v in out.items()}


def check(got, want, dtype):
    for n, t in got.items():
        if t is not None:
            u = HALF["f32" if n in WIDE else dtype]
            within(n, to_host(t), want[n], u * np.abs(want[n]) + (1 + u) * want["e_" + n] + 1e-37)


def tensors(x, dtype, without=()):
    return {k: None if k in without else dev(a, "f32" if k in F32 else dtype) for k, a in x.items()}


def lengths(lens):
    torch = require_gpu()
    return None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")


def args(t):
    return [t[n] for n in ("x", "dt", "A", "B", "C", "D", "z", "bias")]


CASES = [
    # b, T, C, G, N, lens
    (1, 1, 8, 1, 1, None),
    (2, 9, 24, 1, 4, [9, 4]),
    (1, 33, 64, 1, 16, None),
    (2, 100, 136, 1, 16, [100, 65]),
    (1, 257, 48, 2, 8, [250]),
    (3, 70, 144, 3, 16, [-1, 1, 99]),
    (1, 130, 16, 2, 5, None),
    (1, 90, 72, 1, 33, [81]),
    (2, 41, 40, 1, 64, None),
    (1, 64, 272, 1, 2, None),
    (1, 200, 32, 4, 24, [199]),
    (1, 600, 8, 1, 3, [555]),
    (2, 40, 40, 1, 24, [33, 40]),
    (2, 30, 24, 1, 8, [7, 30]),
    (1, 300, 40, 1, 4, None),
    (1, 333, 88, 1, 16, [300]),
    (2, 64, 48, 1, 1, [64, 50]),
    (9, 75, 256, 32, 16, [75, 1, 0, 40, 75, 75, 8, 9, 64]),
    (8, 100, 512, 64, 64, [100, 99, 3, 0, 100, 57, 8, 1]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[:5])))
def test_training_pair(case, dtype):
    torch = require_gpu()
    *sizes, lens = case
    x = make(*sizes, dtype, seed=sizes[1] + sizes[4])
    t, ln = tensors(x, dtype), lengths(lens)
    y, end, reserve = gspn.selective_scan_fwd_train(*args(t), state=t["state"], lens=ln)
    grads = gspn.selective_scan_bwd_reserve(*args(t), t["dy"], reserve, dstate=t["dend"], state=t["state"], lens=ln)
    check(dict(y=y, end=end, **dict(zip(GRADS, grads))), expect(x, lens), dtype)
    # the same without a reserve
    a, b = gspn.selective_scan_fwd(*args(t), state=t["state"], lens=ln)
    check(dict(y=a, end=b), expect(x, lens, grads=False), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("without", [("z",), ("D",), ("bias",), ("state",), ("z", "D", "bias", "state", "dend")], ids="-".join)
def test_without(without, dtype):
    require_gpu()
    x = make(2, 75, 56, 1, 16, dtype, seed=6)
    t = tensors(x, dtype, without)
    y, end, reserve = gspn.selective_scan_fwd_train(*args(t), state=t["state"])
    grads = dict(zip(GRADS, gspn.selective_scan_bwd_reserve(*args(t), t["dy"], reserve, dstate=t["dend"], state=t["state"])))
    for n, g in (("z", "dz"), ("D", "dD"), ("bias", "dbias"), ("state", "dstate")):
        assert (grads[g] is None) == (n in without)
    check(dict(y=y, end=end, **grads), expect(x, None, without), dtype)


def test_steps_as_they_are():
    """softplus=False: dt + dt_bias is the step."""
    require_gpu()
    x = make(1, 60, 40, 1, 16, "f32", seed=8)
    x["dt"], x["bias"] = np.abs(x["dt"]), mixers_ref.store(np.full(40, 0.01), "f32")
    t = tensors(x, "f32")
    y, end, reserve = gspn.selective_scan_fwd_train(*args(t), state=t["state"], softplus=False)
    grads = gspn.selective_scan_bwd_reserve(*args(t), t["dy"], reserve, dstate=t["dend"], state=t["state"], softplus=False)
    check(dict(y=y, end=end, **dict(zip(GRADS, grads))), expect(x, None, soft=False), "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [(2, 1, 40, 1, 16, None), (3, 1, 16, 2, 5, [1, 0, 1]), (1, 5, 72, 1, 64, [3]), (2, 8, 24, 3, 1, None),
                                  (1, 2, 8, 1, 2, None), (5, 3, 264, 1, 32, [3, 9, 2, -7, 1])],
                         ids=lambda c: "x".join(map(str, c[:5])))
def test_single_tokens(case, dtype):
    torch = require_gpu()
    *sizes, lens = case
    x = make(*sizes, dtype, seed=3)
    t, ln = tensors(x, dtype), lengths(lens)
    y, end = gspn.selective_scan_fwd(*args(t), state=t["state"], lens=ln)
    check(dict(y=y, end=end), expect(x, lens, grads=False), dtype)
    keep = t["state"].clone()   # in place
    y2, end2 = gspn.selective_scan_fwd(*args(t), state=keep, state_out=keep, lens=ln)
    assert end2 is keep and torch.equal(y, y2) and torch.equal(end, keep)


def test_tokens_one_by_one_meet_the_chunks():
    """A prompt in chunks, then single tokens, is the sequence at once; the state is continued
    in place, in chunks too."""
    torch = require_gpu()
    x = make(2, 140, 40, 1, 16, "f32", seed=12)
    t = tensors(x, "f32")
    parts, state = [], t["state"].clone()
    for a, b in [(0, 100)] + [(i, i + 1) for i in range(100, 120)] + [(120, 140)]:
        part = [t[n][:, a:b].contiguous() if n in ("x", "dt", "B", "C", "z") else t[n] for n in ("x", "dt", "A", "B", "C", "D", "z", "bias")]
        y, _ = gspn.selective_scan_fwd(*part, state=state, state_out=state)
        parts.append(y)
    check(dict(y=torch.cat(parts, 1), end=state), expect(x, None, grads=False), "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_padding_may_hold_anything(dtype):
    torch = require_gpu()
    got, lens = [], [90, 3, 0]
    for bad in (0.0, float("nan"), float("inf")):
        t = tensors(make(3, 150, 40, 1, 16, dtype, seed=2), dtype)
        for n in ("x", "dt", "B", "C", "z", "dy"):
            for b in range(3):
                t[n][b, lens[b]:] = bad
        ln = lengths(lens)
        y, end, reserve = gspn.selective_scan_fwd_train(*args(t), state=t["state"], lens=ln)
        grads = gspn.selective_scan_bwd_reserve(*args(t), t["dy"], reserve, dstate=t["dend"], state=t["state"], lens=ln)
        few = [a[:, :5].contiguous() if a.dim() > 2 else a for a in args(t)]
        got.append([y, end, *grads, *gspn.selective_scan_fwd(*few, state=t["state"], lens=torch.clamp(ln, max=5))])
        assert all(torch.isfinite(a).all() for a in got[-1])
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_hard_steps(dtype):
    """Steps that forget everything, that keep everything (exactly 0), and both at once; rates
    of 0."""
    require_gpu()
    x = make(1, 120, 24, 1, 16, dtype, seed=15)
    x["dt"][0, 5::17], x["dt"][0, 9::17], x["dt"][0, 11::17] = 200.0, -np.inf, 20.0
    x["A"][:, 3], x["A"][4] = 0.0, 0.0
    t = tensors(x, dtype)
    y, end, reserve = gspn.selective_scan_fwd_train(*args(t), state=t["state"])
    grads = gspn.selective_scan_bwd_reserve(*args(t), t["dy"], reserve, dstate=t["dend"], state=t["state"])
    x["dt"] = np.where(np.isinf(x["dt"]), -1e4, x["dt"])
    want = expect(x, None)
    for e in [k for k in want if k.startswith("e_")]:   # the bounds count |dt| u of a step that is 0
        want[e] = np.where(np.isnan(want[e]), 0, want[e])
    check(dict(y=y, end=end, **dict(zip(GRADS, grads))), want, dtype)


def test_strides():
    torch = require_gpu()
    x = make(2, 100, 48, 2, 5, "bf16", seed=5)
    t = tensors(x, "bf16")
    y, end, reserve = gspn.selective_scan_fwd_train(*args(t))
    grads = gspn.selective_scan_bwd_reserve(*args(t), t["dy"], reserve)
    wide = torch.cat([t[n] for n in ("x", "dt", "z", "dy")], 2)
    small = torch.cat([t["B"].flatten(2), t["C"].flatten(2)], 2)       # rows of 20, from entry 10 on: odd addresses
    s = dict(t, **{n: wide[:, :, i * 48:(i + 1) * 48] for i, n in enumerate(("x", "dt", "z", "dy"))})
    s["B"], s["C"] = (small[:, :, i * 10:(i + 1) * 10].unflatten(2, (2, 5)) for i in (0, 1))
    dw, ds = torch.full_like(wide, float("nan")), torch.full_like(small, float("nan"))
    y2, end2, reserve2 = gspn.selective_scan_fwd_train(*args(s), y=dw[:, :, 144:])
    assert torch.equal(y, y2) and torch.equal(end, end2)
    out = (dw[:, :, :48], dw[:, :, 48:96], torch.empty_like(t["A"]), ds[:, :, :10].unflatten(2, (2, 5)), ds[:, :, 10:].unflatten(2, (2, 5)),
           torch.empty_like(t["D"]), dw[:, :, 96:144], torch.empty_like(t["bias"]), None)
    gspn.selective_scan_bwd_reserve(*args(s), s["dy"], reserve2, out=out)
    for n, a, b in zip(GRADS[:8], grads, out):
        assert torch.equal(a, b), n
    one = [a[:1, :1].expand(2, *[100] + [-1] * (a.dim() - 2)) if a.dim() > 2 else a for a in args(t)]   # one token, again and again
    a, b = gspn.selective_scan_fwd(*one), gspn.selective_scan_fwd(*[o.contiguous() for o in one])
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_gradient_against_differences():
    torch = require_gpu()
    x = make(1, 50, 16, 1, 4, "f32", seed=31)
    t = tensors(x, "f32")
    names = ("x", "dt", "A", "B", "C", "D", "z", "bias", "state")
    y, end, reserve = gspn.selective_scan_fwd_train(*args(t), state=t["state"])
    grads = gspn.selective_scan_bwd_reserve(*args(t), t["dy"], reserve, dstate=t["dend"], state=t["state"])
    h = 3e-3
    for i, n in enumerate(names):
        torch.manual_seed(i)
        d = torch.randn_like(t[n])
        d /= d.norm()
        sums = []
        for e in (h, -h):
            a = {**t, n: t[n] + e * d}
            y, end = gspn.selective_scan_fwd(*args(a), state=a["state"])
            sums.append(float((y.double() * t["dy"].double()).sum() + (end.double() * t["dend"].double()).sum()))
        num, ana = (sums[0] - sums[1]) / (2 * h), float((grads[i].double() * d.double()).sum())
        assert abs(num - ana) <= 2e-2 * float(grads[i].double().norm()) + 1e-2, (n, num, ana)


ENDS = [(9, 75, 256, 32, 16, [75, 1, 0, 40, 75, 75, 8, 9, 64]), (1, 333, 88, 1, 16, [300]), (1, 600, 8, 1, 3, [555]),
        (2, 41, 40, 1, 64, None), (1, 30, 24, 1, 4, [27]), (2, 5, 24, 1, 16, [5, 3])]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", ENDS, ids=lambda c: "x".join(map(str, c[:5])))
def test_rates_down_to_the_lowest(case, dtype):
    """States that forget at once: exp(d A) is 0 at any of these rates, so that results are the
    same bits, also where tokens and whole chunks lie past a sequence's end."""
    torch = require_gpu()
    *sizes, lens = case
    x = make(*sizes, dtype, seed=21)
    ln, got = lengths(lens), []
    for rate in (-1e30, np.finfo(np.float32).min, -np.inf):
        x["A"][:, 1::2], x["A"][3] = rate, rate
        t = tensors(x, dtype)
        y, end, reserve = gspn.selective_scan_fwd_train(*args(t), state=t["state"], lens=ln)
        grads = gspn.selective_scan_bwd_reserve(*args(t), t["dy"], reserve, dstate=t["dend"], state=t["state"], lens=ln)
        a, b = gspn.selective_scan_fwd(*args(t), state=t["state"], lens=ln)
        got.append(dict(y=y, end=end, **dict(zip(GRADS, grads)), a=a, b=b))
        if rate == -1e30:
            want = expect(x, lens)
            check({k: v for k, v in got[0].items() if k not in "ab"}, want, dtype)
            check(dict(y=a, end=b), want, dtype)
    for other in got[1:]:
        for n, v in other.items():
            assert torch.equal(got[0][n], v), n


@pytest.mark.parametrize("case", ENDS, ids=lambda c: "x".join(map(str, c[:5])))
def test_an_infinite_last_token(case):
    """What a sequence's last token makes infinite stays so, its sign kept, and nothing else changes."""
    torch = require_gpu()
    *sizes, lens = case
    b, T = sizes[:2]
    lens = [T] * b if lens is None else lens
    x = make(*sizes, "f32", seed=22)
    t, ln = tensors(x, "f32"), lengths(lens)
    base = gspn.selective_scan_fwd(*args(t), state=t["state"], lens=ln)
    for i, n in enumerate(lens):
        if n > 0:
            t["B"][i, n - 1, :, 0] = float("inf")
    for y, end, *_ in (gspn.selective_scan_fwd(*args(t), state=t["state"], lens=ln),
                       gspn.selective_scan_fwd_train(*args(t), state=t["state"], lens=ln)):
        for i, n in enumerate(lens):
            if n > 0:
                assert torch.equal(end[i, :, 0], torch.sign(t["x"][i, n - 1]) * float("inf")), i
                torch.testing.assert_close(y[i, :n - 1], base[0][i, :n - 1], rtol=1e-4, atol=1e-4)
            torch.testing.assert_close(end[i, :, 1:], base[1][i, :, 1:], rtol=1e-4, atol=1e-4)
            assert (y[i, max(n, 0):] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [c for c in ENDS if c[5]], ids=lambda c: "x".join(map(str, c[:5])))
def test_gradients_past_the_end_of_infinite_states(case, dtype):
    torch = require_gpu()
    *sizes, lens = case
    t, ln = tensors(make(*sizes, dtype, seed=23), dtype), lengths(lens)
    for i, n in enumerate(lens):
        if n > 0:
            t["B"][i, n - 1, :, 0] = float("inf")
    y, end, reserve = gspn.selective_scan_fwd_train(*args(t), state=t["state"], lens=ln)
    grads = dict(zip(GRADS, gspn.selective_scan_bwd_reserve(*args(t), t["dy"], reserve, dstate=t["dend"], state=t["state"], lens=ln)))
    for n in ("dx", "ddt", "dB", "dC", "dz"):
        for i, k in enumerate(lens):
            assert (grads[n][i, k:] == 0).all(), (n, i)
