"""Gates at the ends of their range in the delta rule's chunks: tokens that forget
everything among ordinary ones, in the bounds of test_delta_rule_gpu.py."""
import numpy as np
import pytest

import paper_2606_00746_amd as gspn
from gpu_util import require_gpu, to_host
from test_attention_gpu import dev
from test_delta_rule_gpu import NAMES, check, expect, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("resets", [1, 8, 40])
def test_digits_behind_resets(resets, dtype):
    """`resets` tokens of a chunk forget everything, the ones behind them decay as
    ordinary ones do: what is carried over tens of tokens keeps fp32's digits, however
    far the chunk's gates add up."""
    torch = require_gpu()
    B, T, Hq, Hv, D = 1, 250, 1, 2, 64
    x = make(B, T, Hq, Hv, D, D, dtype, seed=resets)
    at = np.arange(T) % 64
    x["g"][:, (at < 40) & (at % (40 // resets) == 0)] = -100.0
    assert (x["g"][0, :64, 0] == -100.0).sum() == resets
    t = {n: dev(a, "f32" if "state" in n else dtype) for n, a in x.items()}
    args = [t[n] for n in ("q", "k", "v", "g", "beta")]
    o, end, reserve = gspn.delta_rule_fwd_train(*args, state=t["state"])
    grads = gspn.delta_rule_bwd_reserve(*args, t["do"], reserve, dstate=t["dstate"], state=t["state"])
    check({"o": o, "state": end, **dict(zip(NAMES, grads))}, expect(x, D ** -0.5), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,bad", [(200, 70), (64, 0), (8, 3)])
def test_a_nan_gate_is_seen(T, bad, dtype):
    """A gate that is NaN (a run that has diverged) leaves NaN in its head from its token
    on and in the state, and nothing in the chunks ahead of it or in the other head."""
    torch = require_gpu()
    x = make(1, T, 1, 2, 64, 64, dtype, seed=T)
    t = {n: dev(a, "f32" if "state" in n else dtype) for n, a in x.items()}
    args = [t[n] for n in ("q", "k", "v", "g", "beta")]
    want = gspn.delta_rule_fwd(*args, state=t["state"])
    args[3] = t["g"].clone()
    args[3][0, bad, 1] = float("nan")
    calls = [gspn.delta_rule_fwd(*args, state=t["state"]), gspn.delta_rule_fwd_train(*args, state=t["state"])]
    for o, end, *reserve in calls:
        assert torch.isnan(o[0, bad:, 1]).all() and torch.isnan(end[0, 1]).all()
        ahead = bad if T <= 8 and not reserve else bad // 64 * 64
        assert torch.isfinite(o[0, :ahead, 1]).all()
        assert torch.isfinite(o[0, :, 0]).all() and torch.isfinite(end[0, 0]).all()
        if T > 8 or not reserve:
            assert torch.equal(o[:, :, 0], want[0][:, :, 0]) and torch.equal(o[0, :ahead, 1], want[0][0, :ahead, 1])
    dg = gspn.delta_rule_bwd_reserve(*args, t["do"], calls[1][2], state=t["state"])[3]
    assert torch.isnan(dg[0, bad, 1]) and torch.isfinite(dg[0, :, 0]).all()
