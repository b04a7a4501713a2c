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
