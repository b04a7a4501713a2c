"""The short causal convolution (gspn_short_conv_fwd, _bwd) against its formula in 64 bits, on
inputs that are exact in the storage type.  An output is one rounding (2^-8 of itself for
bf16, 2^-24 for fp32) of what fp32 arithmetic gives, which is off by at most what
sublayer_ref counts.  Sums of the weights' gradients: a thread's own tokens (up to 71), the
128 threads or fewer of a workgroup that share a channel, and 64 rows of shares, with 8 for
what a row of them adds up: a depth of 271."""
import numpy as np
import pytest

import mixers_ref
import paper_2606_00746_amd as gspn
import sublayer_ref as ref
from gpu_util import require_gpu, to_host
from test_attention_gpu import dev, within

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
DEPTH = 271


def make(B, T, C, K, dtype, seed):
    rng = np.random.default_rng(seed)
    x = dict(x=rng.standard_normal((B, T, C)), w=rng.standard_normal((C, K)), bias=rng.standard_normal(C),
             state=rng.standard_normal((B, K - 1, C)), dy=rng.standard_normal((B, T, C)), dend=rng.standard_normal((B, K - 1, C)))
    return {n: mixers_ref.store(a, dtype) for n, a in x.items()}


def expect(x, lens, act, state=True, bias=True, grads=True, dend=True):
    B, T, C = x["x"].shape
    zero = np.zeros_like(x["state"][0])
    rs = [ref.conv(x["x"][b], x["w"], x["bias"] if bias else np.zeros(C), x["state"][b] if state else zero,
                   T if lens is None else min(max(lens[b], 0), T), act, x["dy"][b] if grads else None,
                   x["dend"][b] if dend else zero, DEPTH) for b in range(B)]
    out = {}
    for n in rs[0]:
        add = np.stack([r[n] for r in rs])
        out[n] = add.sum(0) if n.replace("e_", "") in ("dw", "dbias") else add
    return out


def check(got, want, dtype):
    for n, t in got.items():
        within(n, to_host(t), want[n], HALF[dtype] * np.abs(want[n]) + (1 + HALF[dtype]) * want.get("e_" + n, 0.0) + 1e-37)


CASES = [
    # B, T, C, K, lens
    (1, 1, 8, 2, None),
    (2, 3, 24, 4, [3, 1]),
    (3, 2, 16, 8, [2, 0, 1]),
    (2, 65, 72, 4, [65, 2]),
    (1, 300, 520, 4, None),
    (2, 130, 40, 3, [130, 64]),
    (1, 77, 104, 5, [76]),
    (2, 70, 136, 7, None),
    (1, 200, 32, 8, [190]),
    (4, 515, 16, 6, [600, -1, 8, 512]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", [True, False])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[:4])))
def test_both_passes(case, act, dtype):
    torch = require_gpu()
    *sizes, lens = case
    x = make(*sizes, dtype, seed=sizes[1] + sizes[3])
    t = {n: dev(a, dtype) for n, a in x.items()}
    ln = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    kw = dict(state=t["state"], lens=ln, silu=act)
    y, end = gspn.short_conv_fwd(t["x"], t["w"], t["bias"], **kw)
    grads = gspn.short_conv_bwd(t["x"], t["w"], t["bias"], t["dy"], dstate=t["dend"], **kw)
    check(dict(zip(("y", "end", "dx", "dw", "dbias", "dstate"), (y, end, *grads))), expect(x, lens, act), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_states_and_bias(dtype):
    require_gpu()
    x = make(2, 90, 48, 4, dtype, seed=4)
    t = {n: dev(a, dtype) for n, a in x.items()}
    y, end = gspn.short_conv_fwd(t["x"], t["w"])
    dx, dw, dbias, din = gspn.short_conv_bwd(t["x"], t["w"], None, t["dy"])
    assert dbias is None and din is None
    check(dict(y=y, end=end, dx=dx, dw=dw), expect(x, None, True, state=False, bias=False, dend=False), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parts_meet(dtype):
    """A prompt, single tokens and a few more, the state continued in place, are the sequence
    at once, bit for bit."""
    torch = require_gpu()
    x = make(3, 120, 40, 4, dtype, seed=9)
    t = {n: dev(a, dtype) for n, a in x.items()}
    y, end = gspn.short_conv_fwd(t["x"], t["w"], t["bias"], state=t["state"])
    parts, state = [], t["state"].clone()
    for a, b in [(0, 100)] + [(i, i + 1) for i in range(100, 115)] + [(115, 117), (117, 120)]:
        out, same = gspn.short_conv_fwd(t["x"][:, a:b].contiguous(), t["w"], t["bias"], state=state, state_out=state)
        assert same is state
        parts.append(out)
    assert torch.equal(torch.cat(parts, 1), y) and torch.equal(state, end)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_padding_may_hold_anything(dtype):
    torch = require_gpu()
    got, lens = [], [70, 2, 0]
    for bad in (0.0, float("nan"), float("inf")):
        x = make(3, 100, 24, 4, dtype, seed=2)
        t = {n: dev(a, dtype) for n, a in x.items()}
        for b, n in enumerate(lens):
            t["x"][b, n:] = bad
            t["dy"][b, n:] = bad
        kw = dict(state=t["state"], lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
        got.append([*gspn.short_conv_fwd(t["x"], t["w"], t["bias"], **kw),
                    *gspn.short_conv_bwd(t["x"], t["w"], t["bias"], t["dy"], dstate=t["dend"], **kw)])
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(a, b)


def test_large_arguments():
    """Sums far from 0, to either side and at infinity: y and the gradient are what they tend to."""
    torch = require_gpu()
    C = 64
    x = torch.zeros(1, 1, C, device="cuda")
    x[0, 0] = torch.linspace(-300, 300, C, device="cuda")
    x[0, 0, 0], x[0, 0, -1] = float("-inf"), float("inf")
    w = torch.tensor([[0.0, 1.0]], device="cuda").repeat(C, 1)
    state = torch.zeros(1, 1, C, device="cuda")
    y, _ = gspn.short_conv_fwd(x, w, state=state)
    want = torch.nn.functional.silu(x.double())
    want[0, 0, 0], want[0, 0, -1] = 0.0, float("inf")
    torch.testing.assert_close(y.double(), want, rtol=(1.5 * 300 + 7) * 2.0 ** -24, atol=1e-36)
    dx = gspn.short_conv_bwd(x, w, None, torch.ones_like(x), state=state)[0]
    assert torch.isfinite(dx).all()
    assert (dx[0, 0, :20].abs() < 1e-30).all() and (dx[0, 0, -20:] == 1).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides(dtype):
    """Slices of a projection, broadcast tokens, gradients into slices of one buffer."""
    torch = require_gpu()
    x = make(2, 100, 32, 4, dtype, seed=5)
    t = {n: dev(a, dtype) for n, a in x.items()}
    fused = torch.cat((t["dy"], t["x"], t["dy"]), 2)
    s, sdy = fused[:, :, 32:64], fused[:, :, 64:]
    y, end = gspn.short_conv_fwd(t["x"], t["w"], t["bias"])
    wide = torch.full((2, 100, 96), float("nan"), dtype=y.dtype, device="cuda")
    y2, end2 = gspn.short_conv_fwd(s, t["w"], t["bias"], y=wide[:, :, 32:64])
    assert torch.equal(y, y2) and torch.equal(end, end2) and wide[:, :, :32].isnan().all() and wide[:, :, 64:].isnan().all()
    grads = gspn.short_conv_bwd(t["x"], t["w"], t["bias"], t["dy"])
    out = (wide[:, :, :32], torch.empty_like(t["w"]), torch.empty_like(t["bias"]), None)
    gspn.short_conv_bwd(s, t["w"], t["bias"], sdy, out=out)
    for a, b in zip(grads[:3], out[:3]):
        assert torch.equal(a, b)
    one = t["x"][:1, :1].expand(2, 100, 32)
    a, b = gspn.short_conv_fwd(one, t["w"])[0], gspn.short_conv_fwd(one.contiguous(), t["w"])[0]
    assert torch.equal(a, b)


def test_gradient_against_differences():
    torch = require_gpu()
    x = make(2, 40, 16, 4, "f32", seed=31)
    t = {n: dev(a, "f32") for n, a in x.items()}
    names = ("x", "w", "bias", "state")

    def call(a):
        return gspn.short_conv_fwd(a["x"], a["w"], a["bias"], state=a["state"])

    grads = gspn.short_conv_bwd(t["x"], t["w"], t["bias"], t["dy"], dstate=t["dend"], state=t["state"])
    h = 1e-2
    for i, n in enumerate(names):
        torch.manual_seed(i)
        d = torch.randn_like(t[n])
        d /= d.norm()
        sums = [sum(float((o.double() * g.double()).sum()) for o, g in zip(call({**t, n: t[n] + e * d}), (t["dy"], t["dend"])))
                for e in (h, -h)]
        num, ana = (sums[0] - sums[1]) / (2 * h), float((grads[i].double() * d.double()).sum())
        # the difference's own error, h^2 times a third derivative, and roundings over h
        assert abs(num - ana) <= 1e-2 * float(grads[i].double().norm()) + 1e-2, (n, num, ana)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [2, 4, 8])
def test_an_infinite_last_input(K, dtype):
    """It reaches the last tap's gradient alone: the other taps' pair it with tokens past the end."""
    torch = require_gpu()
    t = {n: dev(a, dtype) for n, a in make(2, 70, 40, K, dtype, seed=4).items()}
    lens, got = torch.tensor([50, 70], dtype=torch.int32, device="cuda"), []
    for _ in range(2):
        got.append(gspn.short_conv_bwd(t["x"], t["w"], t["bias"], t["dy"], lens=lens, silu=False))
        t["x"][0, 49] = float("inf")
    (dx, dw, db, _), (dx2, dw2, db2, _) = got
    assert torch.isinf(dw2[:, -1]).all()
    assert torch.equal(dx, dx2) and torch.equal(dw[:, :-1], dw2[:, :-1]) and torch.equal(db, db2)
