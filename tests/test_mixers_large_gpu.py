"""The token mixers' kernels that large calls take, and the split over the keys as
forwards with windows take it, against the formulas in 64 bits within the bounds of
test_attention_gpu.py and test_qk_norm_gpu.py.  Which kernels a case takes is checked on
the CPU (test_mixers_host.py).  Of attention's large cases a sample of sequences and key
heads is compared, every query head that shares them included."""
import numpy as np
import pytest

import paper_2606_00746_amd as gspn
from gpu_util import require_gpu, to_host
from test_attention_gpu import check, dev
from test_attention_gpu import test_forward_and_gradient as forward_and_gradient
from test_qk_norm_gpu import make as make_norm
from test_qk_norm_gpu import run_case

pytestmark = pytest.mark.gpu

# B, Tq, Tk, Hq, Hkv, D, left, right, sinks, lens, offset
RAGGED8 = [530, 0, 1, 64, 65, 400, 529, 129]
WHOLE = [   # 128 rows a workgroup in all three kernels
    (8, 530, 530, 16, 8, 64, 70, 0, 5, RAGGED8, 0),              # causal window, sinks
    (8, 530, 530, 16, 16, 32, 64, 64, 130, None, 0),             # both sides, sinks over several tiles
    (8, 530, 530, 16, 16, 72, -1, -1, 0, RAGGED8, 0),            # no bounds
    (8, 600, 600, 16, 4, 128, -1, 0, 0, None, 0),                # causal
    (10, 515, 700, 12, 6, 96, 90, 20, 2, [700, 690, 300, 185, 186, 0, 650, 640, 630, 1], 185),   # behind earlier keys
    (4, 1100, 1100, 16, 4, 128, 200, 0, 7, [1100, 1037, 640, 1], 0),
    (8, 530, 530, 16, 8, 104, 33, 40, 1, None, 0),
]
PAIRS = [   # 64 rows a workgroup, without the longer sums of few keys
    (1, 600, 600, 2, 1, 128, 100, 50, 3, None, 0),
    (2, 530, 530, 2, 2, 32, 300, 0, 70, [530, 200], 0),
    (1, 520, 650, 4, 2, 72, -1, 0, 0, [640], 130),
    (1, 700, 700, 12, 4, 96, 64, -1, 2, None, 0),
]
SPLIT = [   # forwards over split keys
    (2, 5, 4000, 4, 2, 64, 1500, 200, 40, [4000, 2700], 2600),
    (1, 40, 4000, 8, 2, 128, 1500, -1, 40, [3900], 3000),
    (2, 33, 3000, 2, 2, 72, -1, 250, 0, [2500, 3000], 2480),
    (1, 17, 2600, 18, 1, 32, 700, 0, 3, None, 2583),             # 306 rows a key head
    (1, 7, 5000, 2, 1, 96, 60, 2000, 500, [4100], 1500),
]
# B, T, Hq, Hk, D, R, pairs
NORM = [    # four heads a group of lanes, the last group of a token not full
    (4, 3400, 9, 5, 64, 32, "half"),
    (2, 5600, 6, 3, 80, 40, "adjacent"),
    (2, 5600, 5, 2, 72, 36, "half"),          # pairs that cross runs of 8
    (2, 11000, 5, 2, 64, 0, "half"),          # no rotation
    (1, 5500, 6, 2, 256, 256, "half"),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", WHOLE, ids=lambda c: "x".join(map(str, c[:6])))
def test_attention_of_many_rows(case, dtype):
    torch = require_gpu()
    B, Tq, Tk, Hq, Hkv, D, left, right, sinks, lens, offset = case
    G = Hq // Hkv
    gen = torch.Generator(device="cuda").manual_seed(Tq + D)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q, k, v, do = (torch.randn(B, t, h, D, device="cuda", generator=gen).to(dt)
                   for t, h in ((Tq, Hq), (Tk, Hkv), (Tk, Hkv), (Tq, Hq)))
    ln = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    mask = dict(left=left, right=right, sinks=sinks, lens=ln, offset=offset)
    o, lse = gspn.window_attn_fwd(q, k, v, **mask)
    grads = gspn.window_attn_bwd(q, k, v, o, lse, do, **mask)
    for t in (o, *grads):
        assert torch.isfinite(t).all()
    for b in range(B):
        # every sequence once, and one of them twice
        for hk in {b * 5 % Hkv, Hkv - 1 if b == B // 2 else b * 5 % Hkv}:
            hs, one = slice(hk * G, hk * G + G), slice(hk, hk + 1)
            part = [to_host(t[b:b + 1, :, s]) for t, s in ((q, hs), (k, one), (v, one), (do, hs))]
            check(*part, o[b:b + 1, :, hs], lse[b:b + 1, hs], [t[b:b + 1, :, s] for t, s in zip(grads, (hs, one, one))], dtype,
                  left, right, sinks, None if lens is None else lens[b:b + 1], offset)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", PAIRS + SPLIT, ids=lambda c: "x".join(map(str, c[:6])))
def test_attention_of_few_rows(case, dtype):
    forward_and_gradient(case, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", NORM, ids=lambda c: "x".join(map(str, c)))
def test_norm_of_many_rows(case, dtype):
    run_case(case, dtype)


@pytest.mark.parametrize("case", NORM[:3], ids=lambda c: "x".join(map(str, c)))
def test_norm_of_many_rows_in_place(case):
    """On slices of a fused buffer: what it gives elsewhere, bit for bit."""
    torch = require_gpu()
    B, T, Hq, Hk, D, R, pairs = case
    x = make_norm(B, T, Hq, Hk, D, R, "bf16", seed=2)
    t = {n: dev(x[n], "bf16") for n in ("q", "k", "wq", "wk")}
    cos, sin = dev(x["cos"], "f32"), dev(x["sin"], "f32")
    want = gspn.qk_norm_rotate_fwd(t["q"], t["k"], t["wq"], t["wk"], cos, sin, pairs=pairs)
    fused = torch.cat((t["q"], t["k"], t["k"]), 2)
    a, b = fused[:, :, :Hq], fused[:, :, Hq:Hq + Hk]
    gspn.qk_norm_rotate_fwd(a, b, t["wq"], t["wk"], cos, sin, pairs=pairs, out=(a, b))
    assert bool(torch.equal(a, want[0])) and bool(torch.equal(b, want[1])) and bool(torch.equal(fused[:, :, Hq + Hk:], t["k"]))
