"""The selective scan's chain over many chunks: runs of them side by side, each of more chunks
than it holds at once, so that it reads them a second time."""
import numpy as np
import pytest

import paper_2606_00746_amd as gspn
from gpu_util import require_gpu
from test_selective_scan_gpu import GRADS, args, check, expect, lengths, make, tensors

pytestmark = pytest.mark.gpu

# b, T, C, G, N, lens; more than 256 chunks each (test_sublayer_chunks.py)
CASES = [(1, 6200, 8, 1, 3, [6187]), (2, 6161, 8, 1, 4, [6161, 3001]), (1, 6400, 16, 2, 16, None)]


def slow(case, dtype, seed):
    """Inputs whose states last over chunks: rates of 0.1 to 1, steps of 1/1000 to 1/50."""
    x = make(*case[:5], dtype, seed, lo=1e-3, hi=2e-2)
    x["A"] = np.asarray(-np.random.default_rng(seed).uniform(0.1, 1, x["A"].shape), np.float32).astype(np.float64)
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[:5])))
def test_training_pair(case, dtype):
    torch = require_gpu()
    lens = case[5]
    x = slow(case, dtype, case[1])
    t, ln = tensors(x, dtype), lengths(lens)
    y, end, reserve = gspn.selective_scan_fwd_train(*args(t), state=t["state"], lens=ln)
    grads = gspn.selective_scan_bwd_reserve(*args(t), t["dy"], reserve, dstate=t["dend"], state=t["state"], lens=ln)
    want = expect(x, lens)
    check(dict(y=y, end=end, **dict(zip(GRADS, grads))), want, dtype)
    a, b = gspn.selective_scan_fwd(*args(t), state=t["state"], lens=ln)
    check(dict(y=a, end=b), want, dtype)
    keep = t["state"].clone()      # in place
    a2, same = gspn.selective_scan_fwd(*args(t), state=keep, state_out=keep, lens=ln)
    assert same is keep and torch.equal(a, a2) and torch.equal(b, keep)
    keep = t["state"].clone()
    gspn.selective_scan_fwd_train(*args(t), state=keep, state_out=keep, lens=ln)
    assert torch.equal(end, keep)
