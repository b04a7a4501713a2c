"""What bf16 decoding, and forwards over split keys, are off by: little more than the one
rounding of a result.  Relative norms of the errors against the formulas in 64 bits and
against those results rounded once: weights of 16 bits (2^-17) and fp32 sums add some
1e-5, so 1.05 of the one rounding leaves its own luck over some thousand entries."""
import numpy as np
import pytest

import mixers_ref as ref
import paper_2606_00746_amd as gspn
from gpu_util import require_gpu, to_host
from test_attention_gpu import dev, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,Tq,Tk,Hq,Hkv,D,left,sinks", [
    (1, 1, 3000, 16, 4, 128, -1, 0), (4, 1, 900, 8, 8, 64, 500, 4), (1, 16, 4000, 4, 1, 72, -1, 0), (2, 3, 40, 32, 2, 128, -1, 0)])
def test_one_rounding(B, Tq, Tk, Hq, Hkv, D, left, sinks):
    require_gpu()
    q, k, v, _ = make(B, Tq, Tk, Hq, Hkv, D, "bf16", seed=Tk)
    x = [dev(t, "bf16") for t in (q, k, v)]
    got = [gspn.window_attn_decode(*x, left=left, sinks=sinks),
           gspn.window_attn_fwd(*x, left=left, right=0, sinks=sinks, offset=Tk - Tq)[0]]
    want = np.zeros(q.shape)
    see = ref.visible(Tk, np.arange(Tq) + Tk - Tq, Tk, left, 0, sinks)
    for b in range(B):
        for h in range(Hq):
            want[b, :, h] = ref.attention(q[b, :, h], k[b, :, h // (Hq // Hkv)], v[b, :, h // (Hq // Hkv)], see, 1 / np.sqrt(D))["o"]
    one = np.linalg.norm(ref.bf16(want) - want)
    for i, o in enumerate(got):
        off = np.linalg.norm(to_host(o) - want)
        print(f"[err] {i}: {off / np.linalg.norm(want):.2e}, rounded once {one / np.linalg.norm(want):.2e}", flush=True)
        if i == 0 or Tk > 2000:    # (shorter forwards are not split)
            assert off <= 1.05 * one, (i, off, one)
