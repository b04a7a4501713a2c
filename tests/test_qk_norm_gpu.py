"""The norm of query and key heads with the position rotation
(gspn_qk_norm_rotate_fwd, _bwd) against its formulas in 64 bits.

Bounds, element by element, with u = 2^-8 (bf16: the one rounding of a result) or
2^-24 (fp32) and f = 2^-23 (D + 16), what sums over a head and the few products
after them can be off by: y: u |y| + f (|a| + |b|) of the pair it is turned from;
dx and dw: u of the value, f (dw: 2^-23 times the sum's length, at most) of the sums
of absolute terms."""
import numpy as np
import pytest

import mixers_ref as ref
import paper_2606_00746_amd as gspn
from gpu_util import require_gpu, to_host
from test_attention_gpu import dev, within

pytestmark = pytest.mark.gpu

EPS = 1e-6

CASES = [
    # B, T, Hq, Hk, D, R, pairs
    (1, 1, 1, 1, 64, 64, "half"),
    (2, 37, 6, 2, 64, 64, "half"),
    (2, 19, 5, 3, 128, 128, "adjacent"),
    (1, 50, 4, 4, 72, 36, "half"),        # pairs that cross runs of 8
    (1, 33, 3, 1, 72, 48, "half"),
    (3, 11, 2, 2, 80, 40, "adjacent"),
    (1, 9, 7, 1, 104, 52, "half"),
    (2, 13, 3, 2, 96, 0, "half"),         # no rotation
    (1, 21, 2, 1, 256, 256, "half"),
    (1, 17, 2, 2, 8, 8, "half"),
    (1, 5, 1, 1, 8, 2, "adjacent"),
    (1, 6, 2, 1, 256, 34, "half"),
    (4, 700, 9, 5, 64, 32, "half"),       # many rows: several heads a group
]


def make(B, T, Hq, Hk, D, R, dtype, seed, rows=None):
    rng = np.random.default_rng(seed)
    n = T if rows is None else rows
    x = {x: ref.store(rng.standard_normal((B, T, h, D)), dtype) for x, h in (("q", Hq), ("k", Hk))}
    x.update({"d" + n2: ref.store(rng.standard_normal(x[n2].shape), dtype) for n2 in ("q", "k")})
    x.update({"w" + n2: ref.store(1 + 0.3 * rng.standard_normal(D), dtype) for n2 in ("q", "k")})
    ang = rng.uniform(-7, 7, (n, R // 2))
    x["cos"], x["sin"] = (np.float32(f(ang)).astype(np.float64) for f in (np.cos, np.sin))
    return x


def run_case(case, dtype, positions=None, first=0, rows=None, weights=True):
    torch = require_gpu()
    B, T, Hq, Hk, D, R, pairs = case
    x = make(B, T, Hq, Hk, D, R, dtype, seed=T + D + R, rows=rows)
    t = {n: dev(a, dtype) for n, a in x.items() if n not in ("cos", "sin")}
    kw = dict(eps=EPS, pairs=pairs, first=first)
    if R:
        kw.update(cos=dev(x["cos"], "f32"), sin=dev(x["sin"], "f32"))
    if positions is not None:
        kw["positions"] = torch.tensor(positions, dtype=torch.int32, device="cuda")
    wq, wk = (t["wq"], t["wk"]) if weights else (None, None)
    y = gspn.qk_norm_rotate_fwd(t["q"], t["k"], wq, wk, **kw)
    g = gspn.qk_norm_rotate_bwd(t["q"], t["k"], wq, wk, t["dq"], t["dk"], **kw)
    at = np.broadcast_to(np.arange(T) + first, (B, T)) if positions is None else np.clip(positions, 0, len(x["cos"]) - 1)
    cos, sin = x["cos"][at], x["sin"][at]
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    f = 2.0 ** -23 * (D + 16)
    for i, n in enumerate("qk"):
        w = x["w" + n] if weights else np.ones(D)
        adj = pairs == "adjacent"
        want = ref.norm_rotate(x[n], w, cos, sin, adj, EPS)
        r = 1 / np.sqrt((x[n] ** 2).mean(-1, keepdims=True) + EPS)
        pair = ref.turn(np.abs(x[n] * r * w), np.ones_like(cos), np.ones_like(sin), adj, 0.0)
        mag = pair.copy()
        k = np.arange(R // 2)
        a, b = (2 * k, 2 * k + 1) if adj else (k, k + R // 2)
        mag[..., a] = mag[..., b] = pair[..., a] + pair[..., b]
        within(f"y{n}", to_host(y[i]), want, u * np.abs(want) + f * mag + 1e-37)
        dx, dw, mdx, mdw = ref.norm_rotate_grad(x[n], w, x["d" + n], cos, sin, adj, EPS)
        # a turned gradient is off by the absolute terms of its pair
        turned = np.abs(x["d" + n]).copy()
        turned[..., a] = turned[..., b] = turned[..., a] + turned[..., b]
        slack = r * np.abs(w) * turned + r * np.abs(x[n] * r) * (turned * np.abs(w * x[n] * r)).mean(-1, keepdims=True)
        within(f"d{n}", to_host(g[i]), dx, u * np.abs(dx) + f * (mdx + slack) + 1e-37)
        if weights:
            rows_ = x[n].shape[0] * x[n].shape[1] * x[n].shape[2]
            terms = (turned * np.abs(x[n] * r)).sum((0, 1, 2))
            within(f"dw{n}", to_host(g[2 + i]), dw, u * np.abs(dw) + 2.0 ** -23 * (rows_ + D + 16) * terms + 1e-37)
        else:
            assert g[2 + i] is None


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c)))
def test_norm_rotate(case, dtype):
    run_case(case, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_positions(dtype):
    """Rows by position (those outside the table take its ends) and rows from `first`."""
    rng = np.random.default_rng(1)
    run_case((2, 40, 4, 2, 64, 64, "half"), dtype, positions=rng.integers(-3, 60, (2, 40)), rows=50)
    run_case((2, 40, 4, 2, 64, 48, "half"), dtype, first=7, rows=47)
    run_case((2, 40, 4, 2, 72, 36, "adjacent"), dtype, weights=False)


def test_in_place_and_strides():
    torch = require_gpu()
    x = make(2, 90, 6, 2, 64, 64, "bf16", seed=8)
    q, k = dev(x["q"], "bf16"), dev(x["k"], "bf16")
    cos, sin = dev(x["cos"], "f32"), dev(x["sin"], "f32")
    want = gspn.qk_norm_rotate_fwd(q, k, None, None, cos, sin)
    fused = torch.cat((q, k, k), 2)
    a, b = fused[:, :, :6], fused[:, :, 6:8]
    out = gspn.qk_norm_rotate_fwd(a, b, None, None, cos, sin, out=(a, b))
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    assert torch.equal(fused[:, :, 8:], k)


def test_zero_rows():
    """A head of zeros: eps alone under the root, no NaN."""
    torch = require_gpu()
    z = torch.zeros(1, 3, 2, 64, device="cuda")
    y = gspn.qk_norm_rotate_fwd(z, z)
    g = gspn.qk_norm_rotate_bwd(z, z, None, None, torch.ones_like(z), z)
    assert float(y[0].abs().max()) == 0 and bool(torch.isfinite(g[0]).all())
    assert torch.allclose(g[0], torch.full_like(z, EPS ** -0.5), rtol=1e-5)


def test_gradient_against_differences():
    torch = require_gpu()
    x = make(1, 12, 2, 1, 72, 36, "f32", seed=4)
    t = {n: dev(a, "f32") for n, a in x.items()}
    kw = dict(cos=t["cos"], sin=t["sin"], eps=EPS)
    g = gspn.qk_norm_rotate_bwd(t["q"], t["k"], t["wq"], t["wk"], t["dq"], t["dk"], **kw)
    names = ("q", "k", "wq", "wk")
    h = 1e-2
    for i, n in enumerate(names):
        torch.manual_seed(i)
        d = torch.randn_like(t[n])
        d /= d.norm()
        sums = []
        for e in (h, -h):
            a = {m: t[m] + e * d if m == n else t[m] for m in names}
            yq, yk = gspn.qk_norm_rotate_fwd(a["q"], a["k"], a["wq"], a["wk"], **kw)
            sums.append(float((yq.double() * t["dq"].double()).sum() + (yk.double() * t["dk"].double()).sum()))
        num, ana = (sums[0] - sums[1]) / (2 * h), float((g[i].double() * d.double()).sum())
        assert abs(num - ana) <= 2e-2 * float(g[i].double().norm()) + 1e-3, (n, num, ana)
