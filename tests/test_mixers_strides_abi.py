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


def layouts(B, T, H, parts):
    """(strides, offsets of `parts` slices, all in entries) of slices of one buffer: by heads
    within a token, by entries within a head, by heads of a batch entry, by batch entries."""
    n = parts
    return {
        "heads of a token [B][T][n H][D]": ((T * n * H * D, n * H * D, D), [i * H * D for i in range(n)]),
        "beside each other in a head [B][T][H][n D]": ((T * n * H * D, n * H * D, n * D), [i * D for i in range(n)]),
        "heads outside tokens [B][n H][T][D]": ((n * H * T * D, D, T * D), [i * H * T * D for i in range(n)]),
        "tokens outside batch [T][B][n H][D]": ((n * H * D, B * n * H * D, D), [i * H * D for i in range(n)]),
        "interleaved tokens [B][T n][H][D]": ((T * n * H * D, n * H * D, D), [i * H * D for i in range(n)]),
        "interleaved batch [B n][T][H][D]": ((n * T * H * D, H * D, D), [i * T * H * D for i in range(n)]),
    }


# outputs of one head count each, so that any of them can share a buffer
SHARED = {"qk_norm_rotate_bwd": (dict(B=2, T=3, Hq=4, Hk=4), "dq dk"), "window_attn_bwd": (dict(B=2, Tq=6, Tk=6, Hq=4, Hkv=4), "dq dk dv"),
          "delta_rule_bwd_reserve": (dict(B=2, T=70, Hq=4, Hv=4, Dk=64, Dv=64), "dq dk dv")}


def shared(name, layout, moved=None):
    """The call whose gradients are slices of one buffer; `moved`: one of them by so many entries."""
    sizes, outs = SHARED[name]
    outs = outs.split()
    B, T, H = sizes["B"], sizes.get("T", sizes.get("Tq")), 4
    (sb, st, sh), offsets = layouts(B, T, H, len(outs))[layout]
    at = dict(zip(outs, offsets))
    if moved:
        at[moved[0]] += moved[1]
    rows = [(sb, st, sh) if x in at else (T * H * D, H * D, D) for x in HEADS[name].split()]
    ptrs = {x: P(10 * (i + 1)) for i, x in enumerate(CALLS[name][0])}
    ptrs.update({x: P(1000, 2 * o) for x, o in at.items()})
    return call(name, strides=strides(rows), **sizes, **ptrs, reserve_bytes=1 << 30, reserve=P(2000), ws=None, ws_bytes=0) \
        if "reserve" in CALLS[name][1] else call(name, strides=strides(rows), **sizes, **ptrs, ws=None, ws_bytes=0)


@pytest.mark.parametrize("layout", layouts(1, 1, 1, 1))
@pytest.mark.parametrize("name", SHARED)
def test_gradients_of_one_buffer(name, layout):
    """Gradients that are slices of one fused gradient, whichever way, are taken; one that
    reaches into another is refused."""
    assert shared(name, layout) == n.ERR_WORKSPACE
    outs = SHARED[name][1].split()
    for x in outs[:-1]:
        assert shared(name, layout, (x, 8)) == n.ERR_ALIAS, x
    for x in outs[1:]:
        assert shared(name, layout, (x, -8)) == n.ERR_ALIAS, x


def test_apart_is_what_addresses_say():
    """Two outputs of random strides in one buffer: refused where they have a byte in
    common, and taken, at least, in the layouts above."""
    import random
    rng = random.Random(5)
    B, T, H = 2, 3, 4
    seen = {n.ERR_ALIAS: 0, n.ERR_WORKSPACE: 0}
    for _ in range(4000):
        order = rng.sample(range(3), 3)
        steps, ext = [0, 0, 0], D
        for d in order:
            steps[d] = ext * rng.choice((1, 1, 2, 3)) + 8 * rng.choice((0, 0, 8))
            ext = steps[d] * (B, T, H)[d]
        off = 8 * rng.randrange(0, ext // 8 + 8)
        rows = [(T * H * D, H * D, D)] * 4 + [tuple(steps)] * 2
        ptrs = {x: P(10 * (i + 1)) for i, x in enumerate(CALLS["qk_norm_rotate_bwd"][0])}
        ptrs.update(dq=P(1000), dk=P(1000, 2 * off))
        got = call("qk_norm_rotate_bwd", strides=strides(rows), B=B, T=T, Hq=H, Hk=H, **ptrs, ws=None, ws_bytes=0)
        first = {b * steps[0] + t * steps[1] + h * steps[2] + e for b in range(B) for t in range(T) for h in range(H) for e in range(0, D, 8)}
        meet = any(off + i in first for i in first)
        if meet:
            assert got == n.ERR_ALIAS, (steps, off)
        seen[got] += 1
    assert min(seen.values()) > 500, seen
