"""The joint between two sublayers (gspn_residual_norm_fwd, _bwd) against its formula in 64
bits, on inputs that are exact in the storage types.  An output is one rounding of its type
of what fp32 arithmetic gives, which is off by at most what sublayer_ref counts.  Sums of
the vectors' gradients: a group of lanes' rows (all of them at most), the 32 groups of a
workgroup and 64 rows of shares with 8 each: T B + 104."""
import numpy as np
import pytest

import mixers_ref
import paper_2606_00746_amd as gspn
import sublayer_ref as ref
from gpu_util import require_gpu, to_host
from test_attention_gpu import dev, within

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
EPS = 1e-5
STREAM = ("r", "dro", "dr")    # of the residual stream's type
NAMES = ("dr", "df", "dw", "dw_post", "dscale", "dgate")
ALL = ("f", "w", "w_post", "scale", "gate", "dro")


def make(B, T, C, types, seed):
    rng = np.random.default_rng(seed)
    n = rng.standard_normal
    x = dict(r=2 * n((B, T, C)), f=n((B, T, C)) * np.exp(n((B, T, 1))), w=n(C), w_post=n(C), scale=n(C), gate=n((B, C)),
             dy=n((B, T, C)), dro=n((B, T, C)))
    return {k: mixers_ref.store(a, types[1] if k in STREAM else types[0]) for k, a in x.items()}


def run(x, types, given):
    """Both passes' outputs by name."""
    t = {k: dev(a, types[1] if k in STREAM else types[0]) if k in given or k in ("r", "dy") else None for k, a in x.items()}
    vectors = [t[k] for k in ("w", "w_post", "scale", "gate")]
    y, ro = gspn.residual_norm_fwd(t["r"], t["f"], *vectors, eps=EPS)
    if t["f"] is None and t["w"] is None and types[0] != types[1]:
        raise AssertionError("y's type is not given")
    grads = gspn.residual_norm_bwd(t["r"], t["f"], *vectors, t["dy"], t["dro"], eps=EPS)
    return dict(zip(("y", "r", *NAMES), (y, ro, *grads)))


def check(x, types, given):
    got = run(x, types, given)
    v = {k: x[k] if k in given else None for k in ALL}
    want = ref.join(x["r"], v["f"], v["w"], v["w_post"], v["scale"], v["gate"], EPS, x["dy"], v["dro"],
                    depth=x["r"].shape[0] * x["r"].shape[1] + 104)
    if v["f"] is None:
        want["r"], want["e_r"] = x["r"], np.zeros_like(x["r"])
    for n, t in got.items():
        if t is None:
            assert {"df": "f"}.get(n, n[1:]) not in given, n
            continue
        u = HALF[types[1] if n in STREAM else types[0]]
        within(n, to_host(t), want[n], u * np.abs(want[n]) + (1 + u) * want["e_" + n] + 1e-37)


TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]
# rows of part of a wave, of a wave with 1 to 3 runs a lane, of 256 and of 1024 threads
SIZES = [(1, 1, 8), (2, 3, 24), (3, 5, 72), (1, 40, 136), (2, 33, 256), (1, 9, 520), (2, 7, 1032), (1, 13, 1536), (3, 2, 1544),
         (2, 3, 4104), (1, 2, 6152), (1, 3, 16384)]


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_everything_given(sizes, types):
    require_gpu()
    check(make(*sizes, types, seed=sizes[2]), types, ALL)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("given", [("f",), ("f", "w"), ("f", "w_post"), ("f", "scale"), ("f", "gate"), ("f", "w", "scale", "dro"),
                                   ("w",), ("w", "dro")], ids="-".join)
def test_some_given(given, types):
    require_gpu()
    check(make(3, 37, 264, types, seed=len(given)), types, given)


@pytest.mark.parametrize("B,T", [(70, 2), (1100, 1), (1, 5000), (2, 2100)])
def test_many_rows(B, T):
    """More sequences than workgroups, more rows than a launch has groups."""
    require_gpu()
    check(make(B, T, 64, ("bf16", "f32"), seed=B), ("bf16", "f32"), ALL)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_in_place_and_strides(types):
    torch = require_gpu()
    x = make(2, 50, 96, types, seed=5)
    t = {k: dev(a, types[1] if k in STREAM else types[0]) for k, a in x.items()}
    vectors = [t[k] for k in ("w", "w_post", "scale", "gate")]
    y, ro = gspn.residual_norm_fwd(t["r"], t["f"], *vectors)
    grads = gspn.residual_norm_bwd(t["r"], t["f"], *vectors, t["dy"], t["dro"])
    wide, stream = torch.cat((t["f"], t["dy"], t["f"]), 2), torch.cat((t["r"], t["dro"]), 2)
    f, dy, r, dro = wide[:, :, :96], wide[:, :, 96:192], stream[:, :, :96], stream[:, :, 96:]
    out = (dro, wide[:, :, 192:], *(torch.empty_like(v) for v in vectors))
    gspn.residual_norm_bwd(r, f, *vectors, dy, dro, out=out)
    for n, a, b in zip(NAMES, grads, out):
        assert torch.equal(a, b), n
    y2, r2 = gspn.residual_norm_fwd(r, f, *vectors, out=(torch.empty_like(y), r))
    assert r2 is r and torch.equal(y, y2) and torch.equal(ro, r)


def test_rows_of_zeros_and_large_rows():
    """Rows whose squares all but overflow keep their norm; a row of zeros has one of 0."""
    torch = require_gpu()
    r = torch.zeros(1, 3, 64, device="cuda")
    r[0, 1], r[0, 2] = 1e18, 1e-18
    y, _ = gspn.residual_norm_fwd(r, eps=1e-6)
    assert torch.equal(y[0, 0], torch.zeros(64, device="cuda"))
    # 1e36 a square, 64 of them: below the largest fp32; the mean's root is off by (64 / 2 + 4) 2^-24
    assert (y[0, 1] - 1).abs().max() <= 36 * 2.0 ** -24 + 2.0 ** -23
    assert (y[0, 2] - 1e-15).abs().max() <= 1e-15 * 2.0 ** -20
    dr = gspn.residual_norm_bwd(r, None, None, None, None, None, torch.ones_like(r))[0]
    assert torch.isfinite(dr).all()


def test_gradient_against_differences():
    torch = require_gpu()
    x = make(2, 9, 40, ("f32", "f32"), seed=31)
    t = {k: dev(a, "f32") for k, a in x.items()}
    names = ("r", "f", "w", "w_post", "scale", "gate")

    def call(a):
        return gspn.residual_norm_fwd(*[a[n] for n in names], eps=EPS)

    y, ro = call(t)
    grads = gspn.residual_norm_bwd(*[t[n] for n in names], t["dy"], t["dro"], eps=EPS)
    h = 1e-2
    for i, n in enumerate(names):
        torch.manual_seed(i)
        d = torch.randn_like(t[n])
        d /= d.norm()
        sums = [sum(float((o.double() * g.double()).sum()) for o, g in zip(call({**t, n: t[n] + e * d}), (t["dy"], t["dro"])))
                for e in (h, -h)]
        num, ana = (sums[0] - sums[1]) / (2 * h), float((grads[i].double() * d.double()).sum())
        assert abs(num - ana) <= 1e-2 * float(grads[i].double().norm()) + 1e-2, (n, num, ana)
