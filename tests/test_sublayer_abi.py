"""Refusals of the state space sublayer's C entry points: every invalid argument is found on
the host, before any HIP call (the addresses here are never read, and there is no GPU)."""
import ctypes

import pytest

import paper_2606_00746_amd as g
from paper_2606_00746_amd import _native as n
from paper_2606_00746_amd._sublayer import (SELECTIVE_BWD_RESERVE, SELECTIVE_FWD,
                                             SELECTIVE_FWD_TRAIN)

BASE = 0x7F0000000000


def P(i, off=0):
    """Address i, 64 MiB from the next and aligned, plus an offset."""
    return BASE + i * (1 << 26) + off


CONV = dict(B=2, T=70, C=64, K=4, act=1, dtype=g.BF16)
SCAN = dict(B=2, T=300, C=64, G=2, N=16, softplus=1, dtype=g.BF16)
JOIN = dict(B=2, T=70, C=64, eps=1e-6, dtype=g.BF16, rdtype=g.F32)
WS = dict(ws=P(40), ws_bytes=1 << 25, stream=None)
RS = dict(reserve=P(30), reserve_bytes=1 << 25, **WS)


def pointers(names):
    return {name: P(i) for i, name in enumerate(names.split())}


# entry point: its pointers, and its other arguments in order behind `strides`
CALLS = {
    "short_conv_fwd": (pointers("x w bias state lens y state_out"), dict(CONV, stream=None)),
    "short_conv_bwd": (pointers("x w bias dy dstate_out state lens dx dw dbias dstate"), dict(CONV, **WS)),
    "selective_scan_fwd": (pointers("x dt A Bm Cm D z dt_bias state lens y state_out"), dict(SCAN, **WS)),
    "selective_scan_fwd_train": (pointers("x dt A Bm Cm D z dt_bias state lens y state_out"), dict(SCAN, **RS)),
    "selective_scan_bwd_reserve": (pointers("x dt A Bm Cm D z dt_bias dy dstate_out lens dx ddt dA dBm dCm dD dz ddt_bias dstate"),
                                   dict(SCAN, **RS)),
    "residual_norm_fwd": (pointers("r f w w_post scale gate y r_out"), dict(JOIN, stream=None)),
    "residual_norm_bwd": (pointers("r f w w_post scale gate dy dr_out dr df dw dw_post dscale dgate"), dict(JOIN, **WS)),
}
# NULL for these is a meaning of its own; without f its vectors may not be there
OPTIONAL = {"bias", "state", "lens", "state_out", "dstate_out", "dstate", "D", "z", "dt_bias", "w_post", "scale", "gate", "dr_out"}
# aligned to their elements only
SMALL = {"lens", "Bm", "Cm", "dBm", "dCm"}
STRIDED = {"short_conv_fwd": "x y", "short_conv_bwd": "x dy dx", "selective_scan_fwd": "x dt Bm Cm z y",
           "selective_scan_fwd_train": "x dt Bm Cm z y", "selective_scan_bwd_reserve": "x dt Bm Cm z dy dx ddt dBm dCm dz",
           "residual_norm_fwd": "r f y r_out", "residual_norm_bwd": "r f dy dr_out dr df"}
OUTPUTS = {"short_conv_fwd": "y state_out", "short_conv_bwd": "dx dw dbias dstate", "selective_scan_fwd": "y state_out",
           "selective_scan_fwd_train": "y state_out", "selective_scan_bwd_reserve": "dx ddt dA dBm dCm dD dz ddt_bias dstate",
           "residual_norm_fwd": "y r_out", "residual_norm_bwd": "dr df dw dw_post dscale dgate"}
# an output and the input that it may be
INPLACE = {("state_out", "state"), ("r_out", "r"), ("dr", "dr_out")}


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
        if x not in OPTIONAL and x not in ("w", "f") or x == "w" and "conv" in name:
            assert call(name, **{x: None}) == n.ERR_NULL, x
        off = 1 if x in SMALL else 8
        assert call(name, **{x: ptrs[x] + off}) == n.ERR_ALIGN, x
    for x in OUTPUTS[name].split():
        for y in ptrs:
            if y != x and (x, y) not in INPLACE and (y, x) not in INPLACE:
                assert call(name, **{x: ptrs[y]}) == n.ERR_ALIAS, (x, y)
    if name.startswith("residual"):
        assert call(name, f=None) == n.ERR_NULL      # with vectors that are f's


def test_a_gradient_for_what_was_given():
    """What a forward took has a place for its gradient."""
    for name, pairs in (("short_conv_bwd", [("bias", "dbias")]),
                        ("selective_scan_bwd_reserve", [("D", "dD"), ("z", "dz"), ("dt_bias", "ddt_bias")]),
                        ("residual_norm_bwd", [("w", "dw"), ("w_post", "dw_post"), ("scale", "dscale"), ("gate", "dgate"), ("f", "df")])):
        for given, grad in pairs:
            assert call(name, **{grad: None}) == n.ERR_NULL, (name, given)
            if given != "f":     # and is not looked for without
                assert call(name, **{given: None, grad: None}, ws=None) == n.ERR_WORKSPACE, (name, given)


@pytest.mark.parametrize("name", CALLS)
def test_sizes_and_types(name):
    _, rest = CALLS[name]
    for d in ("B", "T", "C", "K", "G", "N"):
        if d in rest:
            for bad in (0, -4):
                assert call(name, **{d: bad}) == n.ERR_DIM, d
    for d in ("B", "T"):
        assert call(name, **{d: (1 << 31) - 8}) == n.ERR_UNSUPPORTED, d
    for bad in (60, (1 << 20) + 8):
        assert call(name, **dict({"C": bad}, **({"G": 1} if "G" in rest else {}))) == n.ERR_UNSUPPORTED, bad
    for bad in (-1, 2, 9):
        assert call(name, dtype=bad) == n.ERR_DTYPE
    if "K" in rest:
        assert call(name, K=1) == n.ERR_UNSUPPORTED and call(name, K=9) == n.ERR_UNSUPPORTED
        assert call(name, act=2) == n.ERR_DIM and call(name, act=-1) == n.ERR_DIM
    if "G" in rest:
        assert call(name, G=3) == n.ERR_DIM                                  # does not divide C
        assert call(name, G=16) == n.ERR_UNSUPPORTED                         # groups of 4 channels
        assert call(name, N=65) == n.ERR_UNSUPPORTED
        assert call(name, softplus=2) == n.ERR_DIM
    if "eps" in rest:
        for bad in (-1.0, float("nan"), float("inf")):
            assert call(name, eps=bad) == n.ERR_DIM
        assert call(name, C=16392) == n.ERR_UNSUPPORTED
        assert call(name, dtype=g.F32, rdtype=g.BF16) == n.ERR_DTYPE
        assert call(name, rdtype=2) == n.ERR_DTYPE


@pytest.mark.parametrize("name", CALLS)
def test_strides(name):
    tensors = STRIDED[name].split()
    fine = [1 << 20, 1 << 10, 128] * len(tensors)
    for i, x in enumerate(tensors):
        small = x in SMALL
        for at, bad, want in ((1, -1024, n.ERR_UNSUPPORTED), (1, (1 << 23) + 8, n.ERR_UNSUPPORTED), (0, 1 << 45, n.ERR_UNSUPPORTED),
                              (0, (1 << 20) + 1, None if small else n.ERR_ALIGN), (1, 1025, None if small else n.ERR_ALIGN)):
            s = list(fine)
            s[3 * i + at] = bad
            if want is not None:
                assert call(name, strides=(ctypes.c_int64 * len(s))(*s)) == want, (x, at, bad)
        if x in OUTPUTS[name].split():     # elements of an output on one another
            for at, bad in ((1, 0), (1, 8), (0, 0)):
                s = list(fine)
                s[3 * i + at] = bad
                assert call(name, strides=(ctypes.c_int64 * len(s))(*s)) == n.ERR_ALIAS, (x, at, bad)


def test_in_place_by_the_same_strides_only():
    fine = [1 << 20, 1 << 10, 0] * 4
    other = list(fine)
    other[10] = 1 << 9
    assert call("residual_norm_fwd", r_out=P(0), strides=(ctypes.c_int64 * 12)(*other)) == n.ERR_ALIAS
    fine = [1 << 20, 1 << 10, 0] * 6
    other = list(fine)
    other[13] = 1 << 9
    at = CALLS["residual_norm_bwd"][0]["dr_out"]
    assert call("residual_norm_bwd", dr=at, strides=(ctypes.c_int64 * 18)(*other)) == n.ERR_ALIAS
    assert call("residual_norm_bwd", dr=at, strides=(ctypes.c_int64 * 18)(*fine), ws=None) == n.ERR_WORKSPACE


def size(name, *args):
    out = ctypes.c_int64(-1)
    return getattr(g.load(), name)(*args, ctypes.byref(out)), out.value


def test_workspaces():
    for name, query, args in (
        ("short_conv_bwd", "gspn_short_conv_workspace_size", (2, 70, 64, 4, g.BF16)),
        ("selective_scan_fwd", "gspn_selective_scan_workspace_size", (SELECTIVE_FWD, 2, 300, 64, 2, 16, g.BF16)),
        ("selective_scan_fwd_train", "gspn_selective_scan_workspace_size", (SELECTIVE_FWD_TRAIN, 2, 300, 64, 2, 16, g.BF16)),
        ("selective_scan_bwd_reserve", "gspn_selective_scan_workspace_size", (SELECTIVE_BWD_RESERVE, 2, 300, 64, 2, 16, g.BF16)),
        ("residual_norm_bwd", "gspn_residual_norm_workspace_size", (2, 70, 64, 1, g.BF16, g.F32)),
    ):
        st, need = size(query, *args)
        assert st == n.OK and need > 0, name
        first = next(iter(CALLS[name][0].values()))
        assert call(name, ws_bytes=need - 1) == n.ERR_WORKSPACE, name
        assert call(name, ws=None) == n.ERR_WORKSPACE, name
        assert call(name, ws=P(40, 8)) == n.ERR_ALIGN, name
        assert call(name, ws=first) == n.ERR_ALIAS, name
    assert size("gspn_selective_scan_workspace_size", SELECTIVE_FWD, 2, 8, 64, 2, 16, g.BF16) == (n.OK, 0)    # token by token
    st, need = size("gspn_selective_scan_reserve_size", 2, 300, 64, 2, 16, g.BF16)
    assert st == n.OK and need >= 2 * 38 * 16 * 64 * 4 + 2 * 300 * 2 * 2 * 16 * 4     # every eighth token's states, B and C
    for name, out in (("selective_scan_fwd_train", "y"), ("selective_scan_bwd_reserve", "dx")):
        assert call(name, reserve_bytes=need - 1) == n.ERR_WORKSPACE
        assert call(name, reserve=None) == n.ERR_WORKSPACE
        assert call(name, reserve=P(30, 8)) == n.ERR_ALIGN
        assert call(name, reserve=CALLS[name][0][out]) == n.ERR_ALIAS


def test_size_queries():
    lib = g.load()
    assert lib.gspn_short_conv_workspace_size(1, 1, 8, 2, 0, None) == n.ERR_NULL
    assert lib.gspn_selective_scan_workspace_size(0, 1, 1, 8, 1, 1, 0, None) == n.ERR_NULL
    assert lib.gspn_selective_scan_reserve_size(1, 1, 8, 1, 1, 0, None) == n.ERR_NULL
    assert lib.gspn_residual_norm_workspace_size(1, 1, 8, 0, 0, 0, None) == n.ERR_NULL
    assert size("gspn_selective_scan_workspace_size", 3, 1, 1, 8, 1, 1, 0)[0] == n.ERR_UNSUPPORTED
    assert size("gspn_short_conv_workspace_size", 1, 0, 8, 2, 0) == (n.ERR_DIM, 0)
    assert size("gspn_selective_scan_reserve_size", 1, 1, 8, 1, 1, 5) == (n.ERR_DTYPE, 0)
    assert size("gspn_residual_norm_workspace_size", 1, 1, 8, 2, 0, 0) == (n.ERR_DIM, 0)
