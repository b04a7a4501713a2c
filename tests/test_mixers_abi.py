"""Refusals of the token mixers' C entry points: every invalid argument is found on the
host, before any HIP call (the addresses here are never read, and there is no GPU)."""
import ctypes

import pytest

import paper_2606_00746_amd as g
from paper_2606_00746_amd import _native as n
from paper_2606_00746_amd._mixers import (ATTN_BWD, DELTA_BWD_RESERVE, DELTA_FWD,
                                           DELTA_FWD_TRAIN)

BASE = 0x7F0000000000


def P(i, off=0):
    """Address i, 1 MiB from the next and aligned, plus an offset."""
    return BASE + i * (1 << 20) + off


NORM = dict(B=2, T=3, Hq=4, Hk=2, D=64, R=64, rows=8, first=1, pairs=0, eps=1e-6, dtype=g.BF16)
ATTN = dict(B=2, Tq=6, Tk=9, Hq=4, Hkv=2, D=64, left=5, right=0, sinks=1, offset=3, scale=0.1, dtype=g.BF16)
DECODE = {k: v for k, v in ATTN.items() if k not in ("right", "offset")}
DELTA = dict(B=2, T=70, Hq=2, Hv=4, Dk=64, Dv=32, scale=0.1, dtype=g.BF16)
WS = dict(ws=P(40), ws_bytes=1 << 20, stream=None)
RS = dict(reserve=P(30), reserve_bytes=1 << 20, **WS)


def pointers(names):
    return {name: P(i) for i, name in enumerate(names.split())}


# entry point: its pointers, and its other arguments in order behind `strides`
CALLS = {
    "qk_norm_rotate_fwd": (pointers("q k wq wk cos sin positions yq yk"), dict(NORM, stream=None)),
    "qk_norm_rotate_bwd": (pointers("q k wq wk cos sin positions dyq dyk dq dk dwq dwk"), dict(NORM, **WS)),
    "window_attn_fwd": (pointers("q k v lens o lse"), dict(ATTN, **WS)),
    "window_attn_bwd": (pointers("q k v o lse do lens dq dk dv"), dict(ATTN, **WS)),
    "window_attn_decode": (pointers("q k v lens o"), dict(DECODE, **WS)),
    "delta_rule_fwd": (pointers("q k v g beta state lens o state_out"), dict(DELTA, **WS)),
    "delta_rule_fwd_train": (pointers("q k v g beta state lens o state_out"), dict(DELTA, **RS)),
    "delta_rule_bwd_reserve": (pointers("q k v g beta do dstate_out lens dq dk dv dg dbeta dstate"), dict(DELTA, **RS)),
}
# NULL for these is a meaning of its own
OPTIONAL = {"wq", "wk", "positions", "lens", "lse", "state", "state_out", "dstate_out", "dstate"}
# aligned to their elements only
SMALL = {"lens", "positions", "lse", "g", "beta", "dg", "dbeta"}
HEADS = {"qk_norm_rotate_fwd": "q k yq yk", "qk_norm_rotate_bwd": "q k dyq dyk dq dk",
         "window_attn_fwd": "q k v o", "window_attn_bwd": "q k v o do dq dk dv", "window_attn_decode": "q k v o",
         "delta_rule_fwd": "q k v o", "delta_rule_fwd_train": "q k v o", "delta_rule_bwd_reserve": "q k v do dq dk dv"}
OUTPUTS = {"qk_norm_rotate_fwd": "yq yk", "qk_norm_rotate_bwd": "dq dk dwq dwk", "window_attn_fwd": "o lse",
           "window_attn_bwd": "dq dk dv", "window_attn_decode": "o", "delta_rule_fwd": "o state_out",
           "delta_rule_fwd_train": "o state_out", "delta_rule_bwd_reserve": "dq dk dv dg dbeta dstate"}


def call(name, strides=None, **kw):
    ptrs, rest = CALLS[name]
    assert not set(kw) - set(ptrs) - set(rest), kw
    p, r = {**ptrs, **kw}, {**rest, **kw}
    fn = getattr(g.load(), "gspn_" + name)
    return fn(*(p[x] for x in ptrs), strides, *(r[x] for x in rest))


@pytest.mark.parametrize("name", CALLS)
def test_pointers(name):
    ptrs, _ = CALLS[name]
    for x in ptrs:
        if x not in OPTIONAL and not (name == "window_attn_bwd" and x == "lse"):
            assert call(name, **{x: None}) == n.ERR_NULL, x
        off = 1 if x in SMALL else 8
        assert call(name, **{x: ptrs[x] + off}) == n.ERR_ALIGN, x
    if name == "window_attn_bwd":
        assert call(name, lse=None) == n.ERR_NULL
    for x in OUTPUTS[name].split():
        for y in ptrs:
            same = name == "qk_norm_rotate_fwd" and y == x[1:] or {x, y} == {"state", "state_out"}
            if y != x and not same:
                assert call(name, **{x: ptrs[y]}) == n.ERR_ALIAS, (x, y)


@pytest.mark.parametrize("name", CALLS)
def test_sizes_and_types(name):
    _, rest = CALLS[name]
    for d in ("B", "T", "Tq", "Tk", "Hq", "Hk", "Hkv", "Hv", "D", "Dk", "Dv"):
        if d in rest:
            for bad in (0, -4):
                assert call(name, **{d: bad}) == n.ERR_DIM, d
            assert call(name, **{d: (1 << 31) - 8}) == n.ERR_UNSUPPORTED, d
    for d in ("D", "Dk", "Dv"):
        if d in rest:
            for bad in (4, 60, 264):
                assert call(name, **{d: bad}) == n.ERR_UNSUPPORTED, d
    for bad in (-1, 2, 9):
        assert call(name, dtype=bad) == n.ERR_DTYPE
    if "scale" in rest:
        for bad in (float("nan"), float("inf")):
            assert call(name, scale=bad) == n.ERR_DIM


@pytest.mark.parametrize("name", [x for x in CALLS if x.startswith("window")])
def test_attention_arguments(name):
    for kw in (dict(Hq=3), dict(sinks=-1), dict(scale=0.0), dict(scale=-1.0)):
        assert call(name, **kw) == n.ERR_DIM, kw
    assert call(name, D=136) == n.ERR_UNSUPPORTED
    if name != "window_attn_decode":
        assert call(name, offset=-1) == n.ERR_DIM
        assert call(name, offset=(1 << 28) + 1) == n.ERR_UNSUPPORTED


@pytest.mark.parametrize("name", [x for x in CALLS if x.startswith("qk")])
def test_norm_arguments(name):
    bad_eps = (-1.0, float("nan"), float("inf"))
    for kw in (dict(R=3), dict(R=-2), dict(R=66), dict(rows=0), dict(pairs=2), dict(pairs=-1), *(dict(eps=e) for e in bad_eps),
               dict(positions=None, first=-1), dict(positions=None, first=6)):
        assert call(name, **kw) == n.ERR_DIM, kw


def test_delta_arguments():
    for name in CALLS:
        if name.startswith("delta"):
            assert call(name, Hv=3) == n.ERR_DIM
            assert call(name, Dk=136) == n.ERR_UNSUPPORTED and call(name, Dv=136) == n.ERR_UNSUPPORTED


@pytest.mark.parametrize("name", CALLS)
def test_strides(name):
    tensors = HEADS[name].split()
    fine = [1 << 17, 1 << 10, 128] * len(tensors)     # up to 70 tokens a batch entry
    for i, x in enumerate(tensors):
        for at, bad, want in ((1, -1024, n.ERR_UNSUPPORTED), (1, (1 << 23) + 8, n.ERR_UNSUPPORTED), (0, 1 << 45, n.ERR_UNSUPPORTED),
                              (0, 4, n.ERR_ALIGN), (1, 1028, n.ERR_ALIGN), (2, 68, n.ERR_ALIGN)):
            s = list(fine)
            s[3 * i + at] = bad
            assert call(name, strides=(ctypes.c_int64 * len(s))(*s)) == want, (x, at, bad)
        if x in OUTPUTS[name].split():     # elements of an output on one another
            for at, bad in ((1, 0), (2, 0), (2, 8), (0, 0)):
                s = list(fine)
                s[3 * i + at] = bad
                assert call(name, strides=(ctypes.c_int64 * len(s))(*s)) == n.ERR_ALIAS, (x, at, bad)


def test_slices_that_meet():
    """dq, dk and dv as slices of one fused gradient: apart within a token, or refused."""
    H, D = 8, 64      # 4 + 2 + 2 heads a token
    s = []
    for t in (6, 9, 9, 6, 6, 6, 6, 6):
        s += [16 * H * D, H * D, D]
    strides = (ctypes.c_int64 * len(s))(*s)
    at = dict(dq=P(7), dk=P(7, 4 * D * 2), dv=P(7, 6 * D * 2))
    for bad in (dict(dk=P(7, 3 * D * 2)), dict(dv=P(7, 5 * D * 2)), dict(dv=P(7, 7 * D * 2)), dict(dq=P(7, 4 * D * 2))):
        assert call("window_attn_bwd", strides=strides, Tq=6, Tk=6, **{**at, **bad}) == n.ERR_ALIAS, bad
    # and the slices themselves get past that check
    assert call("window_attn_bwd", strides=strides, Tq=6, Tk=6, **at, ws=None) == n.ERR_WORKSPACE


def size(name, *args):
    out = ctypes.c_int64(-1)
    return getattr(g.load(), name)(*args, ctypes.byref(out)), out.value


def test_workspaces():
    for name, query, args in (
        ("qk_norm_rotate_bwd", "gspn_qk_norm_rotate_workspace_size", (2, 3, 4, 2, 64, 64, 0, g.BF16)),
        ("window_attn_bwd", "gspn_window_attn_workspace_size", (ATTN_BWD, 2, 6, 9, 4, 2, 64, 5, 0, 1, 3, g.BF16)),
        ("delta_rule_fwd", "gspn_delta_rule_workspace_size", (DELTA_FWD, 2, 70, 2, 4, 64, 32, g.BF16)),
        ("delta_rule_fwd_train", "gspn_delta_rule_workspace_size", (DELTA_FWD_TRAIN, 2, 70, 2, 4, 64, 32, g.BF16)),
        ("delta_rule_bwd_reserve", "gspn_delta_rule_workspace_size", (DELTA_BWD_RESERVE, 2, 70, 2, 4, 64, 32, g.BF16)),
    ):
        st, need = size(query, *args)
        assert st == n.OK and need >= 0
        if need:
            assert call(name, ws_bytes=need - 1) == n.ERR_WORKSPACE, name
            assert call(name, ws=None) == n.ERR_WORKSPACE, name
            assert call(name, ws=P(40, 8)) == n.ERR_ALIGN, name
            assert call(name, ws=CALLS[name][0]["q"]) == n.ERR_ALIAS, name
    st, need = size("gspn_delta_rule_reserve_size", 2, 70, 2, 4, 64, 32, g.BF16)
    assert st == n.OK and need > 0
    for name, out in (("delta_rule_fwd_train", "o"), ("delta_rule_bwd_reserve", "dq")):
        assert call(name, reserve_bytes=need - 1) == n.ERR_WORKSPACE
        assert call(name, reserve=None) == n.ERR_WORKSPACE
        assert call(name, reserve=P(30, 8)) == n.ERR_ALIGN
        assert call(name, reserve=CALLS[name][0][out]) == n.ERR_ALIAS


def test_size_queries():
    lib = g.load()
    assert lib.gspn_window_attn_workspace_size(0, 1, 1, 1, 1, 1, 64, -1, 0, 0, 0, 0, None) == n.ERR_NULL
    assert lib.gspn_qk_norm_rotate_workspace_size(1, 1, 1, 1, 64, 64, 0, 0, None) == n.ERR_NULL
    assert lib.gspn_delta_rule_workspace_size(0, 1, 1, 1, 1, 64, 64, 0, None) == n.ERR_NULL
    assert lib.gspn_delta_rule_reserve_size(1, 1, 1, 1, 64, 64, 0, None) == n.ERR_NULL
    assert size("gspn_window_attn_workspace_size", 3, 1, 1, 1, 1, 1, 64, -1, 0, 0, 0, 0)[0] == n.ERR_UNSUPPORTED
    assert size("gspn_delta_rule_workspace_size", -1, 1, 1, 1, 1, 64, 64, 0)[0] == n.ERR_UNSUPPORTED
    assert size("gspn_window_attn_workspace_size", 1, 0, 1, 1, 1, 1, 64, -1, 0, 0, 0, 0) == (n.ERR_DIM, 0)
    assert size("gspn_delta_rule_reserve_size", 1, 1, 1, 1, 64, 64, 5) == (n.ERR_DTYPE, 0)
    assert size("gspn_qk_norm_rotate_workspace_size", 1, 1, 1, 1, 63, 0, 0, 0) == (n.ERR_UNSUPPORTED, 0)
