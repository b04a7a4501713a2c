"""Torch front end of the token mixers beside the scan (argument marshalling only).

The norm of query and key heads with the position rotation
(``qk_norm_rotate_*``), windowed attention (``window_attn_*``) and the gated
delta rule (``delta_rule_*``), see ``include/gspn.h`` for the formulas.  Tensors are [B, T, H, D] with D
contiguous and any other strides (slices of a fused projection or of a cache);
every call runs on the current stream of its tensors' device, or on a given one
(as if that were current: what it allocates belongs to it), and takes the
workspace it needs from torch unless it is handed one.
"""
from __future__ import annotations

import ctypes
import functools
import math

from ._native import (_check_raise, _current_device, _dtype_code, _stream_handle, load)

PAIRS = {"half": 0, "adjacent": 1}
ATTN_FWD, ATTN_BWD, ATTN_DECODE = 0, 1, 2
DELTA_FWD, DELTA_FWD_TRAIN, DELTA_BWD_RESERVE = 0, 1, 2


# A small call's time is this binding's: its checks are attribute reads in one
# expression a tensor, and only a failed one is gone into.

def _heads(first, *tensors):
    """(tensor, shape, name) each: on first's GPU, of its dtype, of that shape and
    contiguous in its last dimension."""
    dtype, dev = first.dtype, first.get_device()
    for t, shape, name in tensors:
        if t.shape != shape or t.dtype != dtype or t.get_device() != dev or t.stride(-1) != 1:
            _name_fault(first, t, shape, name)
    if dev < 0:
        raise ValueError("tensors must be on a GPU")


def _name_fault(first, t, shape, name):
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)}, not {list(t.shape)}")
    if t.dtype != first.dtype:
        raise ValueError(f"{name} must have dtype {first.dtype}, not {t.dtype}")
    if t.device != first.device:
        raise ValueError(f"{name} must be on {first.device}")
    if t.shape[-1] > 1:
        raise ValueError(f"{name} must be contiguous in its last dimension")


def _on(call, args):
    """call(**args) with args["stream"], a torch stream or a handle, as the current one."""
    import torch
    s = args.pop("stream")
    if not hasattr(s, "cuda_stream"):
        dev = args["q"].device
        s = torch.cuda.ExternalStream(int(s), device=dev) if s else torch.cuda.default_stream(dev)
    with torch.cuda.stream(s):
        return call(**args)


_MOST = 1 << 30


def _ints(**args):
    """Numbers that the library takes in 32 bits (ctypes would cut them off)."""
    for name, x in args.items():
        if not -_MOST <= x <= _MOST:
            raise ValueError(f"{name} must be between -2**30 and 2**30, not {x}")


_Strides = {n: ctypes.c_int64 * (3 * n) for n in (4, 6, 7, 8)}


def _strides(*tensors):
    """Batch, token and head strides of every tensor, in order; None where all are
    contiguous."""
    for t in tensors:
        if not t.is_contiguous():
            break
    else:
        return None
    out = []
    for t in tensors:
        out += t.stride()[:3]
    return _Strides[len(tensors)](*out)


def _plain(name, t, shape, dtype, like):
    """An optional contiguous tensor's pointer (None: none)."""
    if t is None:
        return None
    if (t.shape != shape or t.dtype != dtype or not t.is_contiguous()
            or t.get_device() != like.get_device()):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor {list(shape)} on {like.device}")
    return t.data_ptr()


def _take(nbytes, given, device):
    """The buffer a call works in: `given` where it is large enough, else a new one,
    as (pointer, bytes) and the tensor, which has to outlive the call."""
    if nbytes == 0:
        return (None, 0), None
    import torch
    if given is not None:
        if given.device != device or given.dtype != torch.uint8 or not given.is_contiguous():
            raise ValueError("workspace must be a contiguous uint8 tensor on the inputs' device")
        if given.numel() >= nbytes:
            return (given.data_ptr(), given.numel()), given
    buf = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return (buf.data_ptr(), nbytes), buf


@functools.lru_cache(maxsize=256)
def _sized(name, args, device):
    """A size query's answer, asked once per sizes and current device."""
    n = ctypes.c_int64(0)
    _check_raise(getattr(load(), name)(*args, ctypes.byref(n)))
    return n.value


# ---------------------------------------------------------------------------
# norm of query and key heads, with the position rotation
# ---------------------------------------------------------------------------

def _norm_sizes(q, k, wq, wk, cos, sin, positions, pairs, first):
    import torch
    if not 0 <= first <= _MOST:
        _ints(first=first)
    if pairs not in PAIRS:
        raise ValueError(f"pairs must be one of {list(PAIRS)}")
    B, T, Hq, D = q.shape
    rows = half = 0
    c = s = p = None
    if cos is not None and sin is not None:
        rows, half = cos.shape
        c = _plain("cos", cos, (rows, half), torch.float32, q)
        s = _plain("sin", sin, (rows, half), torch.float32, q)
        if positions is not None:
            p = _plain("positions", positions, (B, T), torch.int32, q)
    elif cos is not sin:
        raise ValueError("cos and sin go together")
    w = (D,)
    return (B, T, Hq, k.shape[2], D, 2 * half, rows,
            (_plain("wq", wq, w, q.dtype, q), _plain("wk", wk, w, q.dtype, q), c, s, p))


def qk_norm_rotate_fwd(q, k, wq=None, wk=None, cos=None, sin=None, eps: float = 1e-6,
                       positions=None, first: int = 0, pairs: str = "half", out=None,
                       stream=None):
    """(yq, yk): every head of q [B, T, Hq, D] and k [B, T, Hk, D] divided by
    its root mean square, times wq or wk [D] (None: ones), its first
    2 * cos.shape[1] entries turned by the angles of its token's row of cos and
    sin (fp32 [rows, R / 2]; None: no rotation): row positions[b, t] (int32), or
    first + t.  pairs: "half" turns entry i with R / 2 + i, "adjacent" 2i with
    2i + 1.  `out`: (yq, yk), which may be (q, k)."""
    if stream is not None:
        return _on(qk_norm_rotate_fwd, locals())
    import torch
    B, T, Hq, Hk, D, R, rows, ptrs = _norm_sizes(q, k, wq, wk, cos, sin, positions, pairs, first)
    if out is None:
        out = q.new_empty((B, T, Hq, D)), q.new_empty((B, T, Hk, D))
    yq, yk = out
    _heads(q, (q, (B, T, Hq, D), "q"), (k, (B, T, Hk, D), "k"), (yq, (B, T, Hq, D), "yq"),
           (yk, (B, T, Hk, D), "yk"))
    _check_raise(load().gspn_qk_norm_rotate_fwd(
        q.data_ptr(), k.data_ptr(), *ptrs, yq.data_ptr(), yk.data_ptr(),
        _strides(q, k, yq, yk), B, T, Hq, Hk, D, R, rows, first, PAIRS[pairs], eps,
        _dtype_code(q), _stream_handle(q, None)))
    return yq, yk


def qk_norm_rotate_bwd(q, k, wq, wk, dyq, dyk, cos=None, sin=None, eps: float = 1e-6,
                       positions=None, first: int = 0, pairs: str = "half", out=None,
                       stream=None, workspace=None):
    """(dq, dk, dwq, dwk) of qk_norm_rotate_fwd's q, k and weights, from the
    gradients dyq, dyk of its outputs (dwq, dwk None where the weight is)."""
    if stream is not None:
        return _on(qk_norm_rotate_bwd, locals())
    import torch
    B, T, Hq, Hk, D, R, rows, ptrs = _norm_sizes(q, k, wq, wk, cos, sin, positions, pairs, first)
    if out is None:
        kw = dict(dtype=q.dtype, device=q.device)
        out = (torch.empty((B, T, Hq, D), **kw), torch.empty((B, T, Hk, D), **kw),
               None if wq is None else torch.empty(D, **kw),
               None if wk is None else torch.empty(D, **kw))
    dq, dk, dwq, dwk = out
    _heads(q, (q, (B, T, Hq, D), "q"), (k, (B, T, Hk, D), "k"), (dyq, (B, T, Hq, D), "dyq"),
           (dyk, (B, T, Hk, D), "dyk"), (dq, (B, T, Hq, D), "dq"), (dk, (B, T, Hk, D), "dk"))
    dt = _dtype_code(q)
    n = _sized("gspn_qk_norm_rotate_workspace_size", (B, T, Hq, Hk, D, R, PAIRS[pairs], dt),
               _current_device())
    ws, held = _take(n, workspace, q.device)
    _check_raise(load().gspn_qk_norm_rotate_bwd(
        q.data_ptr(), k.data_ptr(), *ptrs, dyq.data_ptr(), dyk.data_ptr(), dq.data_ptr(),
        dk.data_ptr(), _plain("dwq", dwq, (D,), q.dtype, q), _plain("dwk", dwk, (D,), q.dtype, q),
        _strides(q, k, dyq, dyk, dq, dk), B, T, Hq, Hk, D, R, rows, first, PAIRS[pairs], eps, dt,
        *ws, _stream_handle(q, None)))
    return out


# ---------------------------------------------------------------------------
# attention with a sliding window and sinks
# ---------------------------------------------------------------------------

def _attn_sizes(q, k, v, lens, left, right, sinks, offset):
    import torch
    if not (-_MOST <= left <= _MOST and -_MOST <= right <= _MOST and -_MOST <= sinks <= _MOST and -_MOST <= offset <= _MOST):
        _ints(left=left, right=right, sinks=sinks, offset=offset)
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q, k and v must be [B, T, H, D]")
    B, Tq, Hq, D = q.shape
    Tk, Hkv = k.shape[1], k.shape[2]
    return B, Tq, Tk, Hq, Hkv, D, _plain("lens", lens, (B,), torch.int32, q)


def _attn_workspace(op, sizes, left, right, sinks, offset, dt, given, device):
    n = _sized("gspn_window_attn_workspace_size",
               (op, *sizes, left, right, sinks, offset, dt), _current_device())
    return _take(n, given, device)


def window_attn_fwd(q, k, v, left: int = -1, right: int = -1, sinks: int = 0, lens=None,
                    offset: int = 0, scale=None, o=None, lse=None, stream=None, workspace=None):
    """(o, lse): attention of q [B, Tq, Hq, D] over k, v [B, Tk, Hkv, D], where
    the query at position p = t + offset sees the keys p - left .. p + right
    (-1: no bound) and, up to p + right, the first `sinks` tokens; lens (int32
    [B]): the sequences' lengths, past which nothing is seen and sees nothing.
    scale: 1 / sqrt(D) unless given.  lse: fp32 [B, Hq, Tq], for the backward."""
    if stream is not None:
        return _on(window_attn_fwd, locals())
    import torch
    B, Tq, Tk, Hq, Hkv, D, lens_p = _attn_sizes(q, k, v, lens, left, right, sinks, offset)
    if o is None:
        o = q.new_empty((B, Tq, Hq, D))
    if lse is None:
        lse = torch.empty((B, Hq, Tq), dtype=torch.float32, device=q.device)
    _heads(q, (q, (B, Tq, Hq, D), "q"), (k, (B, Tk, Hkv, D), "k"), (v, (B, Tk, Hkv, D), "v"),
           (o, (B, Tq, Hq, D), "o"))
    dt = _dtype_code(q)
    ws, held = _attn_workspace(ATTN_FWD, (B, Tq, Tk, Hq, Hkv, D), left, right, sinks, offset, dt,
                               workspace, q.device)
    _check_raise(load().gspn_window_attn_fwd(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), lens_p, o.data_ptr(),
        _plain("lse", lse, (B, Hq, Tq), torch.float32, q), _strides(q, k, v, o), B, Tq, Tk, Hq,
        Hkv, D, left, right, sinks, offset, 1 / math.sqrt(D) if scale is None else scale, dt, *ws,
        _stream_handle(q, None)))
    return o, lse


def window_attn_bwd(q, k, v, o, lse, do, left: int = -1, right: int = -1, sinks: int = 0,
                    lens=None, offset: int = 0, scale=None, out=None, stream=None,
                    workspace=None):
    """(dq, dk, dv) from the gradient `do` of window_attn_fwd's o; o and lse are
    the forward's, the other arguments those it was called with."""
    if stream is not None:
        return _on(window_attn_bwd, locals())
    import torch
    B, Tq, Tk, Hq, Hkv, D, lens_p = _attn_sizes(q, k, v, lens, left, right, sinks, offset)
    if out is None:
        kw = dict(dtype=q.dtype, device=q.device)
        out = (torch.empty((B, Tq, Hq, D), **kw), torch.empty((B, Tk, Hkv, D), **kw),
               torch.empty((B, Tk, Hkv, D), **kw))
    dq, dk, dv = out
    qs, ks = (B, Tq, Hq, D), (B, Tk, Hkv, D)
    _heads(q, (q, qs, "q"), (k, ks, "k"), (v, ks, "v"), (o, qs, "o"), (do, qs, "do"),
           (dq, qs, "dq"), (dk, ks, "dk"), (dv, ks, "dv"))
    dt = _dtype_code(q)
    ws, held = _attn_workspace(ATTN_BWD, (B, Tq, Tk, Hq, Hkv, D), left, right, sinks, offset, dt,
                               workspace, q.device)
    _check_raise(load().gspn_window_attn_bwd(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
        _plain("lse", lse, (B, Hq, Tq), torch.float32, q), do.data_ptr(), lens_p, dq.data_ptr(),
        dk.data_ptr(), dv.data_ptr(), _strides(q, k, v, o, do, dq, dk, dv), B, Tq, Tk, Hq, Hkv, D,
        left, right, sinks, offset, 1 / math.sqrt(D) if scale is None else scale, dt, *ws,
        _stream_handle(q, None)))
    return dq, dk, dv


def window_attn_decode(q, k, v, lens=None, left: int = -1, sinks: int = 0, scale=None, o=None,
                       stream=None, workspace=None):
    """o for the last Tq tokens of each sequence, q [B, Tq, Hq, D], over a cache
    k, v [B, Tk, Hkv, D] of which lens[b] tokens (None: all) are there, the
    queries' own among them: query t stands at position lens[b] - Tq + t and
    sees the `left` keys before it (-1: all), itself and the first `sinks`.  For
    few tokens: every 16 rows (queries times heads that share a key head) read
    the keys again, and prompts of some hundred tokens are faster in
    window_attn_fwd with an offset, where sequences have one length."""
    if stream is not None:
        return _on(window_attn_decode, locals())
    import torch
    B, Tq, Tk, Hq, Hkv, D, lens_p = _attn_sizes(q, k, v, lens, left, 0, sinks, 0)
    if o is None:
        o = q.new_empty((B, Tq, Hq, D))
    _heads(q, (q, (B, Tq, Hq, D), "q"), (k, (B, Tk, Hkv, D), "k"), (v, (B, Tk, Hkv, D), "v"),
           (o, (B, Tq, Hq, D), "o"))
    dt = _dtype_code(q)
    ws, held = _attn_workspace(ATTN_DECODE, (B, Tq, Tk, Hq, Hkv, D), left, 0, sinks, 0, dt,
                               workspace, q.device)
    _check_raise(load().gspn_window_attn_decode(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), lens_p, o.data_ptr(), _strides(q, k, v, o), B,
        Tq, Tk, Hq, Hkv, D, left, sinks, 1 / math.sqrt(D) if scale is None else scale, dt, *ws,
        _stream_handle(q, None)))
    return o


# ---------------------------------------------------------------------------
# the gated delta rule
# ---------------------------------------------------------------------------

def _delta_sizes(q, k, v, g, beta, lens):
    import torch
    if q.dim() != 4 or v.dim() != 4:
        raise ValueError("q, k and v must be [B, T, H, D]")
    B, T, Hq, Dk = q.shape
    Hv, Dv = v.shape[2], v.shape[3]
    gates = (_plain("g", g, (B, T, Hv), q.dtype, q), _plain("beta", beta, (B, T, Hv), q.dtype, q))
    return (B, T, Hq, Hv, Dk, Dv), gates, _plain("lens", lens, (B,), torch.int32, q)


def _reserve(reserve, n, device):
    """The reserve's pointer and bytes."""
    import torch
    if (reserve.dtype != torch.uint8 or not reserve.is_contiguous() or not reserve.is_cuda
            or reserve.device != device):
        raise ValueError("reserve must be a contiguous uint8 tensor on the inputs' device")
    if reserve.numel() < n:
        raise ValueError(f"reserve of {reserve.numel()} bytes, smaller than the {n} bytes "
                         "these tensors take")
    return reserve.data_ptr(), reserve.numel()


def delta_reserve_size(q, v) -> int:
    """Bytes of the reserve of the delta rule's training pair for these tensors."""
    B, T, Hq, Dk = q.shape
    return _sized("gspn_delta_rule_reserve_size",
                  (B, T, Hq, v.shape[2], Dk, v.shape[3], _dtype_code(q)), _current_device())


def _delta_fwd(op, q, k, v, g, beta, state, lens, scale, o, state_out, reserve, workspace):
    import torch
    sizes, gates, lens_p = _delta_sizes(q, k, v, g, beta, lens)
    B, T, Hq, Hv, Dk, Dv = sizes
    if o is None:
        o = q.new_empty((B, T, Hv, Dv))
    if state_out is None:
        state_out = torch.empty((B, Hv, Dk, Dv), dtype=torch.float32, device=q.device)
    _heads(q, (q, (B, T, Hq, Dk), "q"), (k, (B, T, Hq, Dk), "k"), (v, (B, T, Hv, Dv), "v"),
           (o, (B, T, Hv, Dv), "o"))
    dt = _dtype_code(q)
    n = _sized("gspn_delta_rule_workspace_size", (op, *sizes, dt), _current_device())
    ws, held = _take(n, workspace, q.device)
    args = (q.data_ptr(), k.data_ptr(), v.data_ptr(), *gates,
            _plain("state", state, (B, Hv, Dk, Dv), torch.float32, q), lens_p, o.data_ptr(),
            _plain("state_out", state_out, (B, Hv, Dk, Dv), torch.float32, q),
            _strides(q, k, v, o), *sizes, 1 / math.sqrt(Dk) if scale is None else scale, dt)
    if op == DELTA_FWD:
        _check_raise(load().gspn_delta_rule_fwd(*args, *ws, _stream_handle(q, None)))
        return o, state_out
    n = delta_reserve_size(q, v)
    if reserve is None:
        reserve = torch.empty(n, dtype=torch.uint8, device=q.device)
    _check_raise(load().gspn_delta_rule_fwd_train(*args, *_reserve(reserve, n, q.device), *ws,
                                                  _stream_handle(q, None)))
    return o, state_out, reserve


def delta_rule_fwd(q, k, v, g, beta, state=None, lens=None, scale=None, o=None, state_out=None,
                   stream=None, workspace=None):
    """(o, state_out): S_t = exp(g_t) (I - beta_t k_t k_t^T) S_{t-1} + beta_t k_t v_t^T
    and o_t = scale S_t^T q_t for q, k [B, T, Hq, Dk], v [B, T, Hv, Dv] and g,
    beta [B, T, Hv], from `state` (fp32 [B, Hv, Dk, Dv]; None: zeros).  lens
    (int32 [B]): the sequences' lengths.  scale: 1 / sqrt(Dk) unless given.
    state_out may be state.  A token at a time is its serving form."""
    if stream is not None:
        return _on(delta_rule_fwd, locals())
    return _delta_fwd(DELTA_FWD, q, k, v, g, beta, state, lens, scale, o, state_out, None,
                      workspace)


def delta_rule_fwd_train(q, k, v, g, beta, state=None, lens=None, scale=None, o=None,
                         state_out=None, reserve=None, stream=None, workspace=None):
    """delta_rule_fwd that also fills the reserve that delta_rule_bwd_reserve
    reads (a uint8 device tensor of delta_reserve_size bytes, or None for a new
    one).  Returns (o, state_out, reserve)."""
    if stream is not None:
        return _on(delta_rule_fwd_train, locals())
    return _delta_fwd(DELTA_FWD_TRAIN, q, k, v, g, beta, state, lens, scale, o, state_out, reserve,
                      workspace)


def delta_rule_bwd_reserve(q, k, v, g, beta, do, reserve, dstate=None, state=None, lens=None,
                           scale=None, out=None, stream=None, workspace=None):
    """(dq, dk, dv, dg, dbeta, dstate_in) from the gradients `do` of o and
    `dstate` of state_out (None: zeros); the other arguments are those of
    delta_rule_fwd_train, which filled `reserve`.  dstate_in is the gradient of
    `state`, None where the forward began from zeros."""
    if stream is not None:
        return _on(delta_rule_bwd_reserve, locals())
    import torch
    sizes, gates, lens_p = _delta_sizes(q, k, v, g, beta, lens)
    B, T, Hq, Hv, Dk, Dv = sizes
    qs, vs, gs, ss = (B, T, Hq, Dk), (B, T, Hv, Dv), (B, T, Hv), (B, Hv, Dk, Dv)
    if out is None:
        kw = dict(dtype=q.dtype, device=q.device)
        out = (torch.empty(qs, **kw), torch.empty(qs, **kw), torch.empty(vs, **kw),
               torch.empty(gs, **kw), torch.empty(gs, **kw),
               None if state is None else torch.empty(ss, dtype=torch.float32, device=q.device))
    dq, dk, dv, dg, dbeta, din = out
    _heads(q, (q, qs, "q"), (k, qs, "k"), (v, vs, "v"), (do, vs, "do"), (dq, qs, "dq"),
           (dk, qs, "dk"), (dv, vs, "dv"))
    dt = _dtype_code(q)
    n = _sized("gspn_delta_rule_workspace_size", (DELTA_BWD_RESERVE, *sizes, dt),
               _current_device())
    ws, held = _take(n, workspace, q.device)
    _check_raise(load().gspn_delta_rule_bwd_reserve(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), *gates, do.data_ptr(),
        _plain("dstate", dstate, ss, torch.float32, q), lens_p, dq.data_ptr(), dk.data_ptr(),
        dv.data_ptr(), _plain("dg", dg, gs, q.dtype, q), _plain("dbeta", dbeta, gs, q.dtype, q),
        _plain("dstate_in", din, ss, torch.float32, q), _strides(q, k, v, do, dq, dk, dv), *sizes,
        1 / math.sqrt(Dk) if scale is None else scale, dt,
        *_reserve(reserve, delta_reserve_size(q, v), q.device), *ws, _stream_handle(q, None)))
    return out
