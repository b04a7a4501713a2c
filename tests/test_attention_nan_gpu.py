"""A NaN in a query or a key that counts (a run that has diverged) is seen in every
result that it is part of, and in no other."""
import pytest

import paper_2606_00746_amd as gspn
from gpu_util import require_gpu
from test_attention_gpu import dev, make

pytestmark = pytest.mark.gpu


# the forward proper, its pairs of waves, and the split over the keys with one part and several
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,Tq,Tk,Hq,Hkv,D,left", [(1, 200, 200, 2, 1, 64, 50), (4, 2100, 2100, 16, 8, 32, 20),
                                                    (1, 4, 60, 2, 1, 128, -1), (1, 4, 6000, 2, 1, 96, -1)])
def test_nan_rows(B, Tq, Tk, Hq, Hkv, D, left, dtype):
    torch = require_gpu()
    q, k, v, _ = (dev(a, dtype) for a in make(B, Tq, Tk, Hq, Hkv, D, dtype, seed=Tk))
    mask = dict(left=left, right=0, offset=Tk - Tq)
    o, lse = gspn.window_attn_fwd(q, k, v, **mask)
    bad = q.clone()
    bad[0, 1, 0, 3] = float("nan")
    o2, lse2 = gspn.window_attn_fwd(bad, k, v, **mask)
    assert torch.isnan(o2[0, 1, 0]).all() and torch.isnan(lse2[0, 0, 1])
    o2[0, 1, 0], lse2[0, 0, 1] = o[0, 1, 0], lse[0, 0, 1]
    assert bool(torch.equal(o, o2)) and bool(torch.equal(lse, lse2))
    # a key: every query that sees it
    bad = k.clone()
    j = Tk - 2
    bad[0, j, 0, 5] = float("nan")
    o2, lse2 = gspn.window_attn_fwd(q, bad, v, **mask)
    p = torch.arange(Tq, device="cuda") + Tk - Tq
    see = (p >= j) & ((p - j <= left) | (left < 0))
    G = Hq // Hkv
    assert torch.isnan(o2[0, see, :G]).all() and torch.isnan(lse2[0, :G, see]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1e-38, 3e-38, 1e-30])
def test_scales_next_to_nothing(scale, dtype):
    """Scores of all but 0: lse is the log of the number of keys seen (to the rounding of
    fp32: 2^-22 of logs below 8), o their values' mean."""
    torch = require_gpu()
    q, k, v, do = (dev(a, dtype) for a in make(1, 600, 600, 4, 4, 64, dtype, seed=1))
    o, lse = gspn.window_attn_fwd(q, k, v, left=-1, right=0, scale=scale)
    want = torch.arange(1, 601, device="cuda").double().log().float()
    assert ((lse - want).abs() <= 2.0 ** -22 * 8).all()
    mean = v.double().cumsum(1) / torch.arange(1, 601, device="cuda").view(1, -1, 1, 1)
    # a weight and the result are rounded once each (bf16: 2^-8), and summed in fp32
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23 * 600
    bound = u * (v.double().abs().cumsum(1) / torch.arange(1, 601, device="cuda").view(1, -1, 1, 1) + mean.abs()) + 1e-6
    assert ((o.double() - mean).abs() <= bound).all()
