"""Torch front end of the state space sublayer (argument marshalling only).

The short causal convolution (``short_conv_*``), the selective state space scan
(``selective_scan_*``) and the joint between two sublayers (``residual_norm_*``),
see ``include/gspn.h`` for the formulas.  Tensors are [B, T, C] with C contiguous
and any other strides (slices of a projection); every call runs on the current
stream of its tensors' device, or on a given one (as if that were current: what
it allocates belongs to it), and takes the workspace it needs from torch unless
it is handed one.
"""
from __future__ import annotations

import ctypes

from ._mixers import _MOST, _plain, _reserve, _sized, _take
from ._native import (_check_raise, _current_device, _dtype_code, _stream_handle, load)

ACT_NONE, ACT_SILU = 0, 1
SELECTIVE_FWD, SELECTIVE_FWD_TRAIN, SELECTIVE_BWD_RESERVE = 0, 1, 2


def _elsewhere(t):
    """Whether t is on another GPU than the current one, which a call then has to be for."""
    dev = t.get_device()
    return dev >= 0 and dev != _current_device()


def _on(call, args, first):
    """call(**args) with args["stream"], a torch stream or a handle, as the current one, and its
    device (without one: that of the tensors, and its current stream)."""
    import torch
    s, dev = args.pop("stream"), args[first].device
    if s is None:
        s = torch.cuda.current_stream(dev)
    elif not hasattr(s, "cuda_stream"):
        s = torch.cuda.ExternalStream(int(s), device=dev) if s else torch.cuda.default_stream(dev)
    elif s.device != dev:   # the call would go to its own device's current stream instead
        raise ValueError(f"stream must be of {dev}, not of {s.device}")
    with torch.cuda.stream(s):
        return call(**args)


def _rows(first, *tensors):
    """(tensor, shape, name) each: on first's GPU, of its dtype, of that shape and
    contiguous in its last dimension."""
    dtype, dev = first.dtype, first.get_device()
    for t, shape, name in tensors:
        if (t.shape != shape or t.dtype != dtype or t.get_device() != dev
                or t.stride(-1) != 1 and shape[-1] != 1):
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
    raise ValueError(f"{name} must be contiguous in its last dimension")


def _sizes(name, t, n):
    if t.dim() != n:
        raise ValueError(f"{name} must have {n} dimensions, not {t.dim()}")
    return t.shape


_Strides = {n: ctypes.c_int64 * (3 * n) for n in (2, 3, 4, 6, 11)}


def _strides(*tensors):
    """Batch, token and head strides of every tensor, in order (0 for what it lacks);
    None where all are contiguous."""
    for t in tensors:
        if t is not None and not t.is_contiguous():
            break
    else:
        return None
    out = []
    for t in tensors:
        out += (0, 0, 0) if t is None else (*t.stride()[:-1], 0)[:3]
    return _Strides[len(tensors)](*out)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _gradients(*pairs):
    """(name, tensor, input's name, input) each: what a call was given to write a gradient to has
    an input that it is of (else it would be left as it is)."""
    for name, t, of, given in pairs:
        if t is not None and given is None:
            raise ValueError(f"{name} is the gradient of {of}, which is not given")


# What a call makes itself is not looked over (a small call's time is this binding's).


# ---------------------------------------------------------------------------
# short causal convolution
# ---------------------------------------------------------------------------

def _conv_sizes(x, w, bias, lens):
    import torch
    B, T, C = _sizes("x", x, 3)
    K = _sizes("w", w, 2)[1]
    return (B, T, C, K), (_plain("w", w, (C, K), x.dtype, x), _plain("bias", bias, (C,), x.dtype, x)), \
        _plain("lens", lens, (B,), torch.int32, x)


def short_conv_fwd(x, w, bias=None, state=None, lens=None, silu: bool = True, y=None,
                   state_out=None, stream=None):
    """(y, state_out): u_t = bias + sum_j w[:, j] x_{t-K+1+j} for every channel of x [B, T, C]
    with its own K taps w [C, K], and y = u sigmoid(u), or u with silu=False.  state
    [B, K - 1, C] (None: zeros) holds the inputs ahead of the first token, state_out the last
    ones behind the last; they may be the same tensor.  lens (int32 [B]): the sequences'
    lengths.  A token at a time is its serving form."""
    if stream is not None or _elsewhere(x):
        return _on(short_conv_fwd, locals(), "x")
    (B, T, C, K), weights, lens_p = _conv_sizes(x, w, bias, lens)
    rows, ends = (B, T, C), (B, K - 1, C)
    if y is None:
        _rows(x, (x, rows, "x"))
        y = x.new_empty(rows)
    else:
        _rows(x, (x, rows, "x"), (y, rows, "y"))
    if state_out is None:
        state_out = x.new_empty(ends)
        out_p = state_out.data_ptr()
    else:
        out_p = _plain("state_out", state_out, ends, x.dtype, x)
    _check_raise(load().gspn_short_conv_fwd(
        x.data_ptr(), *weights, _plain("state", state, ends, x.dtype, x), lens_p, y.data_ptr(),
        out_p, _strides(x, y), B, T, C, K, ACT_SILU if silu else ACT_NONE, _dtype_code(x),
        _stream_handle(x, None)))
    return y, state_out


def short_conv_bwd(x, w, bias, dy, dstate=None, state=None, lens=None, silu: bool = True, out=None,
                   stream=None, workspace=None):
    """(dx, dw, dbias, dstate_in) from the gradients `dy` of y and `dstate` of state_out (None:
    zeros); the other arguments are short_conv_fwd's.  dbias is None without a bias, dstate_in,
    the gradient of `state`, where the forward began from zeros."""
    if stream is not None or _elsewhere(x):
        return _on(short_conv_bwd, locals(), "x")
    import torch
    (B, T, C, K), weights, lens_p = _conv_sizes(x, w, bias, lens)
    ends = (B, K - 1, C)
    if out is None:
        kw = dict(dtype=x.dtype, device=x.device)
        out = (torch.empty((B, T, C), **kw), torch.empty((C, K), **kw),
               None if bias is None else torch.empty(C, **kw),
               None if state is None else torch.empty(ends, **kw))
    else:
        _gradients(("dbias", out[2], "bias", bias))
    dx, dw, dbias, din = out
    _rows(x, (x, (B, T, C), "x"), (dy, (B, T, C), "dy"), (dx, (B, T, C), "dx"))
    dt = _dtype_code(x)
    n = _sized("gspn_short_conv_workspace_size", (B, T, C, K, dt), _current_device())
    ws, held = _take(n, workspace, x.device)
    _check_raise(load().gspn_short_conv_bwd(
        x.data_ptr(), *weights, dy.data_ptr(), _plain("dstate", dstate, ends, x.dtype, x),
        _plain("state", state, ends, x.dtype, x), lens_p, dx.data_ptr(),
        _plain("dw", dw, (C, K), x.dtype, x), _plain("dbias", dbias, (C,), x.dtype, x),
        _plain("dstate_in", din, ends, x.dtype, x), _strides(x, dy, dx), B, T, C, K,
        ACT_SILU if silu else ACT_NONE, dt, *ws, _stream_handle(x, None)))
    return out


# ---------------------------------------------------------------------------
# the selective state space scan
# ---------------------------------------------------------------------------

def _selective_sizes(x, dt, A, B, C, D, z, dt_bias, lens):
    import torch
    b, T, ch = _sizes("x", x, 3)
    N, G = _sizes("A", A, 2)[1], _sizes("B", B, 4)[2]
    rows, shared, f32 = (b, T, ch), (b, T, G, N), torch.float32
    _rows(x, (x, rows, "x"), (dt, rows, "dt"), (B, shared, "B"), (C, shared, "C"),
          *(((z, rows, "z"),) if z is not None else ()))
    ptrs = (x.data_ptr(), dt.data_ptr(), _plain("A", A, (ch, N), f32, x), B.data_ptr(),
            C.data_ptr(), _plain("D", D, (ch,), f32, x), _ptr(z),
            _plain("dt_bias", dt_bias, (ch,), f32, x))
    return (b, T, ch, G, N), ptrs, _plain("lens", lens, (b,), torch.int32, x)


def selective_reserve_size(x, B) -> int:
    """Bytes of the reserve of the selective scan's training pair for these tensors (x
    [B, T, C], and B [B, T, G, N])."""
    return _sized("gspn_selective_scan_reserve_size", (*x.shape, *B.shape[2:], _dtype_code(x)),
                  _current_device())


def _selective_fwd(op, x, dt, A, B, C, D, z, dt_bias, state, lens, softplus, y, state_out, reserve,
                   workspace):
    import torch
    sizes, ptrs, lens_p = _selective_sizes(x, dt, A, B, C, D, z, dt_bias, lens)
    b, T, ch, G, N = sizes
    ss = (b, ch, N)
    if y is None:
        y = x.new_empty((b, T, ch))
    else:
        _rows(x, (y, (b, T, ch), "y"))
    if state_out is None:
        state_out = A.new_empty(ss)
        out_p = state_out.data_ptr()
    else:
        out_p = _plain("state_out", state_out, ss, torch.float32, x)
    code = _dtype_code(x)
    n = _sized("gspn_selective_scan_workspace_size", (op, *sizes, code), _current_device())
    ws, held = _take(n, workspace, x.device)
    args = (*ptrs, _plain("state", state, ss, torch.float32, x), lens_p, y.data_ptr(), out_p,
            _strides(x, dt, B, C, z, y), *sizes, int(bool(softplus)), code)
    if op == SELECTIVE_FWD:
        _check_raise(load().gspn_selective_scan_fwd(*args, *ws, _stream_handle(x, None)))
        return y, state_out
    n = selective_reserve_size(x, B)
    if reserve is None:
        reserve = torch.empty(n, dtype=torch.uint8, device=x.device)
    _check_raise(load().gspn_selective_scan_fwd_train(*args, *_reserve(reserve, n, x.device), *ws,
                                                      _stream_handle(x, None)))
    return y, state_out, reserve


def selective_scan_fwd(x, dt, A, B, C, D=None, z=None, dt_bias=None, state=None, lens=None,
                       softplus: bool = True, y=None, state_out=None, stream=None, workspace=None):
    """(y, state_out): with d = softplus(dt + dt_bias) (softplus=False: dt + dt_bias),
    h_t = exp(d A) h_{t-1} + d x_t B_t and y_t = (C_t . h_t + D x_t) z sigmoid(z) for every
    channel of x, dt, z [B, T, C] with its N states; A [C, N], D and dt_bias [C] fp32 (None:
    zeros; z None: no gate); B, C [B, T, G, N] shared by groups of C / G channels.  state
    (fp32 [B, C, N]; None: zeros) stands ahead of the first token, state_out behind the last;
    they may be the same tensor.  lens (int32 [B]): the sequences' lengths.  A token at a time
    is its serving form."""
    if stream is not None or _elsewhere(x):
        return _on(selective_scan_fwd, locals(), "x")
    return _selective_fwd(SELECTIVE_FWD, x, dt, A, B, C, D, z, dt_bias, state, lens, softplus, y,
                          state_out, None, workspace)


def selective_scan_fwd_train(x, dt, A, B, C, D=None, z=None, dt_bias=None, state=None, lens=None,
                             softplus: bool = True, y=None, state_out=None, reserve=None,
                             stream=None, workspace=None):
    """selective_scan_fwd that also fills the reserve that selective_scan_bwd_reserve reads (a
    uint8 device tensor of selective_reserve_size bytes, or None for a new one).  Returns
    (y, state_out, reserve)."""
    if stream is not None or _elsewhere(x):
        return _on(selective_scan_fwd_train, locals(), "x")
    return _selective_fwd(SELECTIVE_FWD_TRAIN, x, dt, A, B, C, D, z, dt_bias, state, lens, softplus,
                          y, state_out, reserve, workspace)


def selective_scan_bwd_reserve(x, dt, A, B, C, D, z, dt_bias, dy, reserve, dstate=None, state=None,
                               lens=None, softplus: bool = True, out=None, stream=None,
                               workspace=None):
    """(dx, ddt, dA, dB, dC, dD, dz, ddt_bias, dstate_in) from the gradients `dy` of y and
    `dstate` of state_out (None: zeros); the other arguments are those of
    selective_scan_fwd_train, which filled `reserve`.  dD, dz and ddt_bias are None where D, z
    and dt_bias are, dstate_in, the gradient of `state`, where the forward began from zeros."""
    if stream is not None or _elsewhere(x):
        return _on(selective_scan_bwd_reserve, locals(), "x")
    import torch
    if out is not None:
        _gradients(("dD", out[5], "D", D), ("dz", out[6], "z", z), ("ddt_bias", out[7], "dt_bias", dt_bias))
    sizes, ptrs, lens_p = _selective_sizes(x, dt, A, B, C, D, z, dt_bias, lens)
    b, T, ch, G, N = sizes
    rows, shared, ss, f32 = (b, T, ch), (b, T, G, N), (b, ch, N), torch.float32
    if out is None:
        kw, kf = dict(dtype=x.dtype, device=x.device), dict(dtype=f32, device=x.device)
        out = (torch.empty(rows, **kw), torch.empty(rows, **kw), torch.empty((ch, N), **kf),
               torch.empty(shared, **kw), torch.empty(shared, **kw),
               None if D is None else torch.empty(ch, **kf),
               None if z is None else torch.empty(rows, **kw),
               None if dt_bias is None else torch.empty(ch, **kf),
               None if state is None else torch.empty(ss, **kf))
    dx, ddt, dA, dB, dC, dD, dz, dbias, din = out
    _rows(x, (dy, rows, "dy"), (dx, rows, "dx"), (ddt, rows, "ddt"), (dB, shared, "dB"),
          (dC, shared, "dC"), *(((dz, rows, "dz"),) if dz is not None else ()))
    code = _dtype_code(x)
    n = _sized("gspn_selective_scan_workspace_size", (SELECTIVE_BWD_RESERVE, *sizes, code),
               _current_device())
    ws, held = _take(n, workspace, x.device)
    _check_raise(load().gspn_selective_scan_bwd_reserve(
        *ptrs, dy.data_ptr(), _plain("dstate", dstate, ss, f32, x), lens_p, dx.data_ptr(),
        ddt.data_ptr(), _plain("dA", dA, (ch, N), f32, x), dB.data_ptr(), dC.data_ptr(),
        _plain("dD", dD, (ch,), f32, x), _ptr(dz), _plain("ddt_bias", dbias, (ch,), f32, x),
        _plain("dstate_in", din, ss, f32, x), _strides(x, dt, B, C, z, dy, dx, ddt, dB, dC, dz),
        *sizes, int(bool(softplus)), code,
        *_reserve(reserve, selective_reserve_size(x, B), x.device), *ws, _stream_handle(x, None)))
    return out


# ---------------------------------------------------------------------------
# the joint between two sublayers
# ---------------------------------------------------------------------------

def _join_sizes(r, f, y, w, w_post, scale, gate):
    """Sizes, the tensor whose dtype the block has, and the vectors' pointers."""
    B, T, C = _sizes("r", r, 3)
    like = f if f is not None else y if y is not None else w if w is not None else r
    v, dt = (C,), like.dtype
    return (B, T, C), like, (_plain("w", w, v, dt, r), _plain("w_post", w_post, v, dt, r),
                             _plain("scale", scale, v, dt, r), _plain("gate", gate, (B, C), dt, r))


def _same_gpu(r, like):
    if like.get_device() != r.get_device():
        raise ValueError(f"tensors must be on {r.device}")


def residual_norm_fwd(r, f=None, w=None, w_post=None, scale=None, gate=None, eps: float = 1e-6,
                      out=None, stream=None):
    """(y, r_out): the output f [B, T, C] of a block, divided by its root mean square and times
    w_post [C] (None: f as it is), times gate [B, C] and scale [C] (None: ones), is added to the
    residual stream r: r_out; y is r_out divided by its root mean square, times w [C] (None:
    ones).  r and r_out have f's dtype or are fp32.  Without f, y is the norm of r, and r_out is
    r.  `out`: (y, r_out), where r_out may be r."""
    if stream is not None or _elsewhere(r):
        return _on(residual_norm_fwd, locals(), "r")
    if f is None and out is not None and out[1] is not None and out[1].data_ptr() != r.data_ptr():
        raise ValueError("r_out is r without f (nothing else is written)")
    sizes, like, ptrs = _join_sizes(r, f, None if out is None else out[0], w, w_post, scale, gate)
    _same_gpu(r, like)
    _rows(r, (r, sizes, "r"))
    if f is not None:
        _rows(like, (f, sizes, "f"))
    if out is None:
        y = like.new_empty(sizes)
        ro = r if f is None else r.new_empty(sizes)
        out = y, ro
    else:
        y, ro = out
        _rows(like, (y, sizes, "y"))
        if f is not None:
            _rows(r, (ro, sizes, "r_out"))
    _check_raise(load().gspn_residual_norm_fwd(
        r.data_ptr(), _ptr(f), *ptrs, y.data_ptr(), None if f is None else ro.data_ptr(),
        _strides(r, f, y, ro), *sizes, eps, _dtype_code(like), _dtype_code(r),
        _stream_handle(r, None)))
    return y, r if ro is None else ro


def residual_norm_bwd(r, f, w, w_post, scale, gate, dy, dr_out=None, eps: float = 1e-6,
                      out=None, stream=None, workspace=None):
    """(dr, df, dw, dw_post, dscale, dgate) from the gradients dy of y and dr_out of r_out, from
    what else reads it (None: nothing); the other arguments are those residual_norm_fwd was called
    with (r too: the sum is formed again).  A gradient is None where what it is of is.  `out`:
    the six, where dr may be dr_out."""
    if stream is not None or _elsewhere(r):
        return _on(residual_norm_bwd, locals(), "r")
    import torch
    sizes, like, ptrs = _join_sizes(r, dy, None, w, w_post, scale, gate)
    B, T, C = sizes
    if out is None:
        kw = dict(dtype=like.dtype, device=r.device)
        out = (torch.empty(sizes, dtype=r.dtype, device=r.device),
               None if f is None else torch.empty(sizes, **kw),
               *(None if t is None else torch.empty(C, **kw) for t in (w, w_post, scale)),
               None if gate is None else torch.empty((B, C), **kw))
    else:
        _gradients(("df", out[1], "f", f), ("dw", out[2], "w", w), ("dw_post", out[3], "w_post", w_post),
                   ("dscale", out[4], "scale", scale), ("dgate", out[5], "gate", gate))
    dr, df, *grads, dgate = out
    _same_gpu(r, like)
    _rows(r, (r, sizes, "r"), (dr, sizes, "dr"),
          *(((dr_out, sizes, "dr_out"),) if dr_out is not None else ()))
    _rows(like, (dy, sizes, "dy"), *(((f, sizes, "f"), (df, sizes, "df")) if f is not None else ()))
    codes = _dtype_code(like), _dtype_code(r)
    n = _sized("gspn_residual_norm_workspace_size", (*sizes, int(gate is not None), *codes),
               _current_device())
    ws, held = _take(n, workspace, r.device)
    _check_raise(load().gspn_residual_norm_bwd(
        r.data_ptr(), _ptr(f), *ptrs, dy.data_ptr(), _ptr(dr_out), dr.data_ptr(), _ptr(df),
        *(_plain(name, t, (C,), like.dtype, r) for name, t in zip(("dw", "dw_post", "dscale"), grads)),
        _plain("dgate", dgate, (B, C), like.dtype, r), _strides(r, f, dy, dr_out, dr, df),
        *sizes, eps, *codes, *ws, _stream_handle(r, None)))
    return out
