"""Windowed attention (gspn_window_attn_fwd, _bwd, _decode) against its formulas in
64 bits, on inputs that are exact in the storage type.

Bounds, element by element, with u = 2^-8 for bf16 storage (half an ulp, relative)
and 0 for fp32, and f = 2^-23 (D s + n + 16), where s is the largest sum of absolute
terms of a score and n the number of keys: what fp32 products and sums of those
lengths, and an exponential of a score that is f off, can be off by.
* o: a softmax weight is rounded once for its product with v, the result once:
  (u + f) sum_j p |v| + u |o|.
* lse: f (1 + |lse|).
* dv: as o, with do.  dq, dk: ds is rounded once, and is off by what o is off by
  (its rounding and its weights'): 2 u times the absolute terms, and f times the
  products' own absolute terms; the result is rounded once.
"""
import numpy as np
import pytest

import mixers_ref as ref
import paper_2606_00746_amd as gspn
from gpu_util import require_gpu, to_host

pytestmark = pytest.mark.gpu


def dev(a, dtype):
    torch = require_gpu()
    return torch.tensor(np.ascontiguousarray(a), device="cuda").to(
        torch.bfloat16 if dtype == "bf16" else torch.float32)


def make(B, Tq, Tk, Hq, Hkv, D, dtype, seed, scale=1.0):
    rng = np.random.default_rng(seed)
    q = ref.store(scale * rng.standard_normal((B, Tq, Hq, D)), dtype)
    k, v = (ref.store(rng.standard_normal((B, Tk, Hkv, D)), dtype) for _ in range(2))
    return q, k, v, ref.store(rng.standard_normal((B, Tq, Hq, D)), dtype)


def within(tag, got, want, bound):
    assert got.shape == want.shape
    same = ~np.isfinite(want)
    assert np.array_equal(got[same], want[same]), f"{tag}: values that are not finite"
    off = np.abs(np.where(same, 0, got) - np.where(same, 0, want))
    worst = float((off / np.maximum(np.where(same, 1.0, bound), 1e-30)).max(initial=0.0))
    print(f"[err] {tag}: {worst:.3f} of the bound, largest {off.max(initial=0.0):.2e}", flush=True)
    assert worst <= 1.0, f"{tag}: {worst:.3f} of the bound"


def check(q, k, v, do, o, lse, grads, dtype, left, right, sinks, lens=None, offset=0, tail=False, scale=None):
    B, Tq, Hq, D = q.shape
    Tk, Hkv = k.shape[1], k.shape[2]
    scale = 1 / np.sqrt(D) if scale is None else scale
    u = 2.0 ** -8 if dtype == "bf16" else 0.0
    G = Hq // Hkv
    names = ["o"] + (["lse"] if lse is not None else []) + (["dq", "dk", "dv"] if grads else [])
    want = {n: np.zeros((B, Hq, Tq) if n == "lse" else (B, Tk, Hkv, D) if n in ("dk", "dv") else (B, Tq, Hq, D))
            for n in names}
    bound = {n: np.zeros_like(x) for n, x in want.items()}
    for b in range(B):
        n = Tk if lens is None else min(max(int(lens[b]), 0), Tk)
        p = np.arange(Tq) + (n - Tq if tail else offset)
        see = ref.visible(n, p, Tk, left, right, sinks)
        for h in range(Hq):
            r = ref.attention(q[b, :, h], k[b, :, h // G], v[b, :, h // G], see, scale, do[b, :, h] if grads else None)
            f = 2.0 ** -23 * (D * r["s_mag"] + Tk + 16)
            want["o"][b, :, h] = r["o"]
            bound["o"][b, :, h] = (u + f) * r["mag_o"] + u * np.abs(r["o"])
            if lse is not None:
                want["lse"][b, h] = r["lse"]
                bound["lse"][b, h] = f * (1 + np.abs(np.where(np.isfinite(r["lse"]), r["lse"], 0)))
            if grads:
                want["dq"][b, :, h] = r["dq"]
                bound["dq"][b, :, h] = (2 * u + 2 * f) * r["mag_dq"] + 2 * f * r["wide_dq"]
                want["dk"][b, :, h // G] += r["dk"]
                bound["dk"][b, :, h // G] += (2 * u + 2 * f) * r["mag_dk"] + 2 * f * r["wide_dk"]
                want["dv"][b, :, h // G] += r["dv"]
                bound["dv"][b, :, h // G] += (u + f) * r["mag_dv"]
    got = dict(zip(names, [o] + ([lse] if lse is not None else []) + list(grads or [])))
    for n in names:
        if n not in ("o", "lse"):
            bound[n] += u * np.abs(want[n])
        within(n, to_host(got[n]), want[n], bound[n] + 1e-37)


CASES = [
    # B, Tq, Tk, Hq, Hkv, D, left, right, sinks, lens, offset
    (1, 1, 1, 1, 1, 64, -1, -1, 0, None, 0),
    (2, 65, 65, 2, 2, 64, -1, -1, 0, None, 0),            # one row past a tile
    (1, 200, 200, 3, 3, 64, -1, 0, 0, None, 0),            # causal, no window
    (2, 333, 333, 4, 2, 64, 70, 0, 5, [333, 100], 0),      # causal window, sinks, ragged
    (1, 400, 400, 2, 1, 128, 33, 31, 3, None, 0),          # both sides
    (1, 300, 300, 2, 2, 72, 0, 0, 1, None, 0),             # each token itself and one sink
    (1, 129, 129, 6, 2, 96, 10, -1, 4, None, 0),           # no upper bound
    (2, 190, 190, 2, 2, 32, 64, 64, 130, [190, 64], 0),    # sinks over several tiles
    (1, 100, 357, 4, 4, 80, 90, 0, 2, None, 257),          # a chunk behind earlier keys
    (1, 70, 400, 2, 2, 104, -1, 0, 0, [390], 330),         # a chunk, no window, some queries past the end
    (3, 140, 140, 2, 1, 8, 20, 5, 0, [0, 1, 140], 0),      # an empty sequence, one of one token
    (1, 1100, 1100, 1, 1, 64, 100, 50, 16, [1000], 0),     # sinks whose queries are split
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[:6])) + f"-{c[6]}-{c[7]}-{c[8]}")
def test_forward_and_gradient(case, dtype):
    torch = require_gpu()
    B, Tq, Tk, Hq, Hkv, D, left, right, sinks, lens, offset = case
    q, k, v, do = make(B, Tq, Tk, Hq, Hkv, D, dtype, seed=Tq + D)
    x = [dev(a, dtype) for a in (q, k, v, do)]
    ln = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    mask = dict(left=left, right=right, sinks=sinks, lens=ln, offset=offset)
    o, lse = gspn.window_attn_fwd(*x[:3], **mask)
    grads = gspn.window_attn_bwd(*x[:3], o, lse, x[3], **mask)
    check(q, k, v, do, o, lse, grads, dtype, left, right, sinks, lens, offset)


# forwards of few queries take the split keys
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [
    (2, 3, 700, 4, 2, 64, -1, 0, 0, [700, 650], 690),
    (1, 5, 90, 6, 1, 128, 20, 3, 4, None, 80),
    (1, 17, 17, 1, 1, 72, -1, -1, 0, None, 0),
], ids=lambda c: "x".join(map(str, c[:6])))
def test_few_queries(case, dtype):
    test_forward_and_gradient(case, dtype)


DECODE = [
    # B, Tq, Tk, Hq, Hkv, D, left, sinks, lens
    (1, 1, 1, 1, 1, 64, -1, 0, None),
    (3, 1, 300, 8, 2, 128, -1, 0, [300, 1, 77]),
    (2, 1, 5000, 4, 1, 64, 999, 4, [5000, 300]),
    (2, 3, 600, 6, 2, 72, 100, 40, [600, 2]),     # more queries than tokens
    (1, 2, 64, 32, 1, 80, 31, 1, [40]),
    (2, 1, 129, 2, 2, 32, 0, 3, [0, 129]),        # an empty sequence
    (1, 9, 2100, 4, 4, 104, -1, 0, [2050]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", DECODE, ids=lambda c: "x".join(map(str, c[:6])))
def test_decode(case, dtype):
    torch = require_gpu()
    B, Tq, Tk, Hq, Hkv, D, left, sinks, lens = case
    q, k, v, _ = make(B, Tq, Tk, Hq, Hkv, D, dtype, seed=Tk + D)
    ln = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    o = gspn.window_attn_decode(dev(q, dtype), dev(k, dtype), dev(v, dtype), ln, left=left, sinks=sinks)
    check(q, k, v, None, o, None, None, dtype, left, 0, sinks, lens, tail=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(dtype):
    """Scores of some hundreds: one key carries a row, its weight next to 1."""
    q, k, v, do = make(1, 150, 150, 2, 2, 64, dtype, seed=3, scale=30.0)
    x = [dev(a, dtype) for a in (q, k, v, do)]
    o, lse = gspn.window_attn_fwd(*x[:3], left=40, right=20)
    grads = gspn.window_attn_bwd(*x[:3], o, lse, x[3], left=40, right=20)
    check(q, k, v, do, o, lse, grads, dtype, 40, 20, 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_padding_may_hold_anything(dtype):
    """NaN and infinities past a sequence's end reach nothing: the results are those
    with zeros there, bit for bit."""
    torch = require_gpu()
    B, T, H, D = 2, 230, 2, 64
    lens = torch.tensor([150, 30], dtype=torch.int32, device="cuda")
    got = []
    for bad in (0.0, float("nan"), float("inf")):
        x = [dev(a, dtype) for a in make(B, T, T, H, H, D, dtype, seed=11)]
        for t in x:
            for b in range(B):
                t[b, int(lens[b]):] = bad
        o, lse = gspn.window_attn_fwd(*x[:3], left=60, right=9, sinks=2, lens=lens)
        grads = gspn.window_attn_bwd(*x[:3], o, lse, x[3], left=60, right=9, sinks=2, lens=lens)
        d = gspn.window_attn_decode(x[0][:, :1].nan_to_num(1.0, 1.0, 1.0), x[1], x[2], lens, left=60, sinks=2)
        got.append([t.clone() for t in (o, lse, *grads, d)])
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(a, b)


def test_strides_and_fused_buffers():
    """Slices of a fused projection in, slices of a fused gradient out, a cache with
    heads outside tokens: the results of contiguous tensors, bit for bit."""
    torch = require_gpu()
    B, T, Hq, Hkv, D = 2, 210, 4, 2, 64
    q, k, v, do = make(B, T, T, Hq, Hkv, D, "bf16", seed=5)
    fused = dev(np.concatenate([q, k, v], 2), "bf16")
    c = [dev(a, "bf16") for a in (q, k, v, do)]
    s = [fused[:, :, :Hq], fused[:, :, Hq:Hq + Hkv], fused[:, :, Hq + Hkv:]]
    mask = dict(left=50, right=10, sinks=3)
    o, lse = gspn.window_attn_fwd(*c[:3], **mask)
    grads = gspn.window_attn_bwd(*c[:3], o, lse, c[3], **mask)
    o2, lse2 = gspn.window_attn_fwd(*s, **mask)
    df = torch.full_like(fused, float("nan"))
    out = (df[:, :, :Hq], df[:, :, Hq:Hq + Hkv], df[:, :, Hq + Hkv:])
    gspn.window_attn_bwd(*s, o2, lse2, c[3], out=out, **mask)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    for a, b in zip(grads, out):
        assert torch.equal(a, b)
    heads_first = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in c[1:3]]
    lens = torch.tensor([210, 33], dtype=torch.int32, device="cuda")
    a = gspn.window_attn_decode(c[0][:, :1], *c[1:3], lens, left=100, sinks=1)
    b = gspn.window_attn_decode(c[0][:, :1], *heads_first, lens, left=100, sinks=1)
    assert torch.equal(a, b)


def test_a_stream_of_its_own():
    torch = require_gpu()
    x = [dev(a, "bf16") for a in make(1, 300, 300, 2, 2, 64, "bf16", seed=9)]
    o, lse = gspn.window_attn_fwd(*x[:3], left=64, right=0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a, b = gspn.window_attn_fwd(*x[:3], left=64, right=0)
    side.synchronize()
    assert torch.equal(o, a) and torch.equal(lse, b)


@pytest.mark.parametrize("mask", [dict(left=40, right=0, sinks=2), dict(left=-1, right=-1)])
def test_gradient_against_differences(mask):
    """Central differences of sum(o do) in fp32 along random directions.  With steps of
    h the third derivative's share is below 1e-2 of the step's; the rounding of o
    (2^-24 of its terms) over 2 h stays below 1e-3."""
    torch = require_gpu()
    x = [dev(a, "f32") for a in make(1, 130, 130, 2, 1, 32, "f32", seed=21)]
    o, lse = gspn.window_attn_fwd(*x[:3], **mask)
    grads = gspn.window_attn_bwd(*x[:3], o, lse, x[3], **mask)
    h = 1e-2
    for i, g in enumerate(grads):
        torch.manual_seed(i)
        d = torch.randn_like(x[i])
        d /= d.norm()
        hi, lo = (gspn.window_attn_fwd(*[t + e * d if n == i else t for n, t in enumerate(x[:3])], **mask)[0].double()
                  for e in (h, -h))
        num = float(((hi - lo) * x[3].double()).sum() / (2 * h))
        ana = float((g.double() * d.double()).sum())
        assert abs(num - ana) <= 2e-2 * float(g.double().norm()) + 1e-3, (i, num, ana)
