"""Strides that the token mixers' C entry points take: those that are not read, and
outputs that share a buffer without meeting.  A call that gets as far as its workspace's
check has passed the checks of its tensors (no GPU is used)."""
import ctypes

import pytest

from paper_2606_00746_amd import _native as n
from test_mixers_abi import CALLS, HEADS, OUTPUTS, P, call

D = 64
TAKES_WORKSPACE = ["qk_norm_rotate_bwd", "window_attn_bwd", "delta_rule_fwd_train", "delta_rule_bwd_reserve"]


def strides(rows):
    flat = [x for r in rows for x in r]
    return (ctypes.c_int64 * len(flat))(*flat)


@pytest.mark.parametrize("name", TAKES_WORKSPACE)
def test_strides_of_one_are_not_read(name):
    """One token of a buffer with heads outside tokens: its heads are far apart, and its
    token and batch strides mean nothing."""
    sizes = {d: 1 for d in ("B", "T", "Tq", "Tk") if d in CALLS[name][1]}
    ptrs = {x: P(1000 * (i + 1)) for i, x in enumerate(HEADS[name].split())}
    for other in (1, 3, -8, 1 << 60):
        s = strides([(other, other, 1 << 22)] * len(ptrs))      # 65536 tokens
        assert call(name, strides=s, **sizes, **ptrs, ws=None, ws_bytes=0) == n.ERR_WORKSPACE, other
