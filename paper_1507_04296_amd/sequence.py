"""Binding of the sequence operators: a recurrent core on the network's features.

Every function checks its tensors, allocates its outputs (torch) and makes one call
of the library on the current stream; include/gorila.h has the definitions, layouts
and errors.  Rows (x, y, their gradients, windows) are float32 or bfloat16,
parameters, parameter gradients, states and scales float32, resets uint8, slots
int32.  Inputs may be strided in their leading dimensions.  `ctx` needs a workspace
where a `*_workspace_bytes` function exists: ``Context(..., min_bytes=...)``.
"""
from __future__ import annotations

import ctypes

import torch

from . import GORILA_BF16, GORILA_F32, _check, lib

GORILA_CODES = 2
_DTYPES = {torch.float32: GORILA_F32, torch.bfloat16: GORILA_BF16}
_vp, _i32, _i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64


class _ConvArgs(ctypes.Structure):
    _fields_ = [(n, _i32) for n in ("dtype", "batch", "length", "channels", "taps", "silu")] + [
        ("x", _vp), ("x_batch_stride", _i64), ("x_step_stride", _i64), ("weight", _vp), ("bias", _vp),
        ("reset", _vp), ("window", _vp)]


class _ScanArgs(ctypes.Structure):
    _fields_ = [(n, _i32) for n in ("dtype", "batch", "length", "heads", "head_dim", "groups", "state_dim", "reserved")] + [
        (n + s, t) for n in ("x", "dt", "b", "c") for s, t in (("", _vp), ("_batch_stride", _i64), ("_step_stride", _i64))] + [
        (n, _vp) for n in ("a_log", "dt_bias", "skip", "reset", "state")]


_CA, _SA = ctypes.POINTER(_ConvArgs), ctypes.POINTER(_ScanArgs)
_f32 = ctypes.c_float
SIGNATURES = {
    "gorila_add_rmsnorm": (_i32, [_vp, _i64, _vp, _i64, _vp, _i64, _i32, _i32, _f32, _vp, _vp, _vp, _vp]),
    "gorila_add_rmsnorm_codes": (_i32, [_vp, _i64, _vp, _i64, _vp, _i64, _i32, _i32, _f32, _vp, _vp, _vp, _vp]),
    "gorila_add_rmsnorm_workspace_bytes": (ctypes.c_size_t, [_i32]),
    "gorila_add_rmsnorm_backward": (_i32, [_vp, _i64, _vp, _i64, _vp, _vp, _vp, _i64, _i32, _i32, _vp, _vp, _vp]),
    "gorila_causal_conv": (_i32, [_CA, _vp, _vp, _vp]),
    "gorila_causal_conv_workspace_bytes": (ctypes.c_size_t, [_i32, _i32]),
    "gorila_causal_conv_backward": (_i32, [_CA, _vp, _i64, _i64, _vp, _vp, _vp, _vp, _vp, _vp]),
    "gorila_causal_conv_step": (_i32, [_CA, _vp, _i64, _vp, _vp, _vp]),
    "gorila_scan_workspace_bytes": (ctypes.c_size_t, [_i32] * 7),
    "gorila_scan": (_i32, [_SA, _vp, _vp, _vp]),
    "gorila_scan_backward": (_i32, [_SA, _vp, _i64, _i64] + [_vp] * 10),
    "gorila_scan_step": (_i32, [_SA, _vp, _i64, _vp, _vp, _vp]),
    "gorila_quantize_weights": (_i32, [_vp, _i64, _i32, _i32, _i32, _i32, _vp, _vp, _vp]),
    "gorila_qmatvec": (_i32, [_vp, _i64, _vp, _i32, _i64, _vp, _vp, _i32, _i32, _i32, _vp, _vp]),
}


def _want(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _dtype(x) -> int:
    dt = _DTYPES.get(x.dtype)
    if dt is None:
        raise TypeError(f"rows must be float32 or bfloat16, got {x.dtype}")
    return dt


def _like(t):
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _at(index: int, t, name: str, shape, dtype, strided: int = 0):
    """Address of an optional tensor of `shape` and `dtype` on device `index`.  The
    dimensions from `strided` on are contiguous; the leading ones have strides of
    their own.  (Host time is what a single step costs, so the accepting path is short.)"""
    if t is None:
        return None
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.get_device() != index:
        raise ValueError(f"{name} must be on device {index}, got {t.device}")
    if not t.is_contiguous():
        run = 1
        for d in range(t.dim() - 1, strided - 1, -1):
            if t.shape[d] > 1:
                if t.stride(d) != run:
                    raise ValueError(f"{name} must be contiguous from dimension {strided} on")
                run *= t.shape[d]
    return t.data_ptr()


def _device(ctx) -> int:
    index = ctx.device.index
    return torch.cuda.current_device() if index is None else index


# ---- norm ----

def _norm_in(ctx, x, weight, residual):
    _want(x.dim() == 2, "x must be [rows, width]")
    dev = _device(ctx)
    rows, width = x.shape
    dt = _dtype(x)
    px = _at(dev, x, "x", x.shape, x.dtype, 1)
    pr = _at(dev, residual, "residual", x.shape, x.dtype, 1)
    return (px, x.stride(0), pr, 0 if residual is None else residual.stride(0),
            _at(dev, weight, "weight", (width,), torch.float32), rows, width, dt)


def add_rmsnorm(ctx, x, weight, residual=None, eps: float = 1e-6):
    """y, total, rstd of total = x + residual (x itself without one) and y = its norm times weight."""
    a = _norm_in(ctx, x, weight, residual)
    y = _like(x)
    total = _like(x) if residual is not None or not x.is_contiguous() else None
    rstd = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
    _check(lib().gorila_add_rmsnorm(*a, eps, y.data_ptr(), None if total is None else total.data_ptr(), rstd.data_ptr(),
                                    ctx.bind_stream()), "gorila_add_rmsnorm")
    return y, x if total is None else total, rstd


def add_rmsnorm_codes(ctx, x, weight, residual=None, eps: float = 1e-6):
    """codes (int8), scale, total: codes * scale[:, None] stands for add_rmsnorm's y."""
    a = _norm_in(ctx, x, weight, residual)
    codes = torch.empty(x.shape, dtype=torch.int8, device=x.device)
    total = _like(x) if residual is not None or not x.is_contiguous() else None
    scale = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
    _check(lib().gorila_add_rmsnorm_codes(*a, eps, codes.data_ptr(), scale.data_ptr(),
                                          None if total is None else total.data_ptr(), ctx.bind_stream()),
           "gorila_add_rmsnorm_codes")
    return codes, scale, x if total is None else total


def add_rmsnorm_workspace_bytes(width: int) -> int:
    return int(lib().gorila_add_rmsnorm_workspace_bytes(width))


def add_rmsnorm_backward(ctx, dy, total, rstd, weight, dtotal=None):
    """dx (of x and of residual), dweight for the gradients that reach y and total."""
    _want(total.dim() == 2, "total must be [rows, width]")
    dev = _device(ctx)
    rows, width = total.shape
    dt = _dtype(total)
    pdy = _at(dev, dy, "dy", total.shape, total.dtype, 1)
    pdt = _at(dev, dtotal, "dtotal", total.shape, total.dtype, 1)
    pt = _at(dev, total, "total", total.shape, total.dtype)
    dx = _like(total)
    dweight = torch.empty(width, dtype=torch.float32, device=total.device)
    _check(lib().gorila_add_rmsnorm_backward(
        pdy, dy.stride(0), pdt, 0 if dtotal is None else dtotal.stride(0), pt,
        _at(dev, rstd, "rstd", (rows,), torch.float32), _at(dev, weight, "weight", (width,), torch.float32), rows, width, dt,
        dx.data_ptr(), dweight.data_ptr(), ctx.bind_stream()), "gorila_add_rmsnorm_backward")
    return dx, dweight


# ---- short causal convolution ----

def _conv_args(ctx, x, weight, bias, reset, window, silu):
    _want(x.dim() == 3, "x must be [batch, length, channels]")
    batch, length, channels = x.shape
    dt, dev = _dtype(x), _device(ctx)
    _want(weight.dim() == 2 and weight.shape[0] == channels, "weight must be [channels, taps]")
    taps = weight.shape[1]
    return _ConvArgs(
        dt, batch, length, channels, taps, 1 if silu else 0, _at(dev, x, "x", x.shape, x.dtype, 2), x.stride(0), x.stride(1),
        _at(dev, weight, "weight", weight.shape, torch.float32), _at(dev, bias, "bias", (channels,), torch.float32),
        _at(dev, reset, "reset", (batch, length), torch.uint8), _at(dev, window, "window", (batch, taps - 1, channels), x.dtype))


def causal_conv(ctx, x, weight, bias=None, reset=None, window=None, silu: bool = True):
    """y [batch, length, channels] and the window [batch, taps - 1, channels] for the steps that follow."""
    a = _conv_args(ctx, x, weight, bias, reset, window, silu)
    y = _like(x)
    out = torch.empty((a.batch, max(0, a.taps - 1), a.channels), dtype=x.dtype, device=x.device)
    _check(lib().gorila_causal_conv(a, y.data_ptr(), out.data_ptr(), ctx.bind_stream()), "gorila_causal_conv")
    return y, out


def causal_conv_workspace_bytes(channels: int, taps: int) -> int:
    return int(lib().gorila_causal_conv_workspace_bytes(channels, taps))


def causal_conv_backward(ctx, dy, x, weight, bias=None, reset=None, window=None, silu: bool = True, dwindow_out=None):
    """dx, dweight, dbias, dwindow (the last two None without a bias or window)."""
    a, dev = _conv_args(ctx, x, weight, bias, reset, window, silu), _device(ctx)
    pdy = _at(dev, dy, "dy", x.shape, x.dtype, 2)
    pdw = _at(dev, dwindow_out, "dwindow_out", (a.batch, a.taps - 1, a.channels), x.dtype)
    dx = _like(x)
    dweight = torch.empty(weight.shape, dtype=torch.float32, device=x.device)
    dbias = None if bias is None else torch.empty_like(dweight[:, 0], memory_format=torch.contiguous_format)
    dwindow = None if window is None else _like(window)
    _check(lib().gorila_causal_conv_backward(
        a, pdy, dy.stride(0), dy.stride(1), pdw, dx.data_ptr(), dweight.data_ptr(), None if dbias is None else dbias.data_ptr(),
        None if dwindow is None else dwindow.data_ptr(), ctx.bind_stream()), "gorila_causal_conv_backward")
    return dx, dweight, dbias, dwindow


def causal_conv_step(ctx, x, window_pool, weight, bias=None, slot=None, reset=None, silu: bool = True):
    """One step of every row of x [rows, channels]; window_pool [slots, taps - 1, channels] is updated."""
    _want(x.dim() == 2, "x must be [rows, channels]")
    rows, channels = x.shape
    _want(weight.dim() == 2 and weight.shape[0] == channels, "weight must be [channels, taps]")
    taps, slots, dev = weight.shape[1], window_pool.shape[0], _device(ctx)
    a = _ConvArgs(
        _dtype(x), rows, 1, channels, taps, 1 if silu else 0, _at(dev, x, "x", x.shape, x.dtype, 1), x.stride(0), 0,
        _at(dev, weight, "weight", weight.shape, torch.float32), _at(dev, bias, "bias", (channels,), torch.float32),
        _at(dev, reset, "reset", (rows,), torch.uint8), None)
    pool = _at(dev, window_pool, "window_pool", (slots, taps - 1, channels), x.dtype)
    y = _like(x)
    _check(lib().gorila_causal_conv_step(a, pool, slots, _at(dev, slot, "slot", (rows,), torch.int32), y.data_ptr(),
                                         ctx.bind_stream()), "gorila_causal_conv_step")
    return y


# ---- selective scan ----

def _scan_args(ctx, x, dt, b, c, a_log, dt_bias, skip, reset, state):
    """x [..., heads, head_dim]; one leading dimension (single steps) or two."""
    dev = _device(ctx)
    lead = x.dim() - 2
    step = lead == 1
    shape, typ = x.shape, x.dtype
    heads, width = shape[lead], shape[lead + 1]
    _want(b.dim() == lead + 2, "b must be [..., groups, state_dim]")
    groups, n = b.shape[lead], b.shape[lead + 1]
    batch, length = shape[0], 1 if step else shape[1]
    par = (heads,)
    xs, ds, bs, cs = x.stride(), dt.stride(), b.stride(), c.stride()
    return _ScanArgs(
        _dtype(x), batch, length, heads, width, groups, n, 0,
        _at(dev, x, "x", shape, typ, lead), xs[0], 0 if step else xs[1],
        _at(dev, dt, "dt", shape[:lead] + par, typ, lead), ds[0], 0 if step else ds[1],
        _at(dev, b, "b", shape[:lead] + (groups, n), typ, lead), bs[0], 0 if step else bs[1],
        _at(dev, c, "c", shape[:lead] + (groups, n), typ, lead), cs[0], 0 if step else cs[1],
        _at(dev, a_log, "a_log", par, torch.float32), _at(dev, dt_bias, "dt_bias", par, torch.float32),
        _at(dev, skip, "skip", par, torch.float32), _at(dev, reset, "reset", shape[:lead], torch.uint8),
        _at(dev, state, "state", (batch, heads, width, n), torch.float32))


def scan_workspace_bytes(batch: int, length: int, heads: int, head_dim: int, groups: int, state_dim: int,
                         backward: bool = False) -> int:
    return int(lib().gorila_scan_workspace_bytes(batch, length, heads, head_dim, groups, state_dim, 1 if backward else 0))


def scan(ctx, x, dt, b, c, a_log, dt_bias, skip, reset=None, state=None):
    """y [batch, length, heads, head_dim] and the state after the last step (float32
    [batch, heads, head_dim, state_dim]); state: the one before the first (None: zeros)."""
    _want(x.dim() == 4, "x must be [batch, length, heads, head_dim]")
    a = _scan_args(ctx, x, dt, b, c, a_log, dt_bias, skip, reset, state)
    y = _like(x)
    out = torch.empty((a.batch, a.heads, a.head_dim, a.state_dim), dtype=torch.float32, device=x.device)
    _check(lib().gorila_scan(a, y.data_ptr(), out.data_ptr(), ctx.bind_stream()), "gorila_scan")
    return y, out


def scan_backward(ctx, dy, x, dt, b, c, a_log, dt_bias, skip, reset=None, state=None, dstate_out=None):
    """dx, ddt, db, dc, da_log, ddt_bias, dskip, dstate (None without a state)."""
    _want(x.dim() == 4, "x must be [batch, length, heads, head_dim]")
    a, dev = _scan_args(ctx, x, dt, b, c, a_log, dt_bias, skip, reset, state), _device(ctx)
    pdy = _at(dev, dy, "dy", x.shape, x.dtype, 2)
    pds = _at(dev, dstate_out, "dstate_out", (a.batch, a.heads, a.head_dim, a.state_dim), torch.float32)
    dx, ddt, db, dc = _like(x), _like(dt), _like(b), _like(c)
    par = torch.empty((3, a.heads), dtype=torch.float32, device=x.device)
    da_log, ddt_bias, dskip = par[0], par[1], par[2]
    dstate = None if state is None else _like(state)
    p0, row = par.data_ptr(), 4 * a.heads
    _check(lib().gorila_scan_backward(
        a, pdy, dy.stride(0), dy.stride(1), pds, dx.data_ptr(), ddt.data_ptr(), db.data_ptr(), dc.data_ptr(), p0, p0 + row,
        p0 + 2 * row, None if dstate is None else dstate.data_ptr(), ctx.bind_stream()), "gorila_scan_backward")
    return dx, ddt, db, dc, da_log, ddt_bias, dskip, dstate


def scan_step(ctx, x, dt, b, c, a_log, dt_bias, skip, state_pool, slot=None, reset=None):
    """One step of every row of x [rows, heads, head_dim]; state_pool [slots, heads, head_dim, state_dim] is updated."""
    _want(x.dim() == 3, "x must be [rows, heads, head_dim]")
    a, dev = _scan_args(ctx, x, dt, b, c, a_log, dt_bias, skip, reset, None), _device(ctx)
    slots = state_pool.shape[0]
    pool = _at(dev, state_pool, "state_pool", (slots, a.heads, a.head_dim, a.state_dim), torch.float32)
    y = _like(x)
    _check(lib().gorila_scan_step(a, pool, slots, _at(dev, slot, "slot", (a.batch,), torch.int32), y.data_ptr(),
                                  ctx.bind_stream()), "gorila_scan_step")
    return y


# ---- 4-bit weights ----

def quantize_weights(ctx, weights, group: int = 64):
    """codes (uint8 [outputs, 16 * ceil(inputs / 32)]), scales [outputs, ceil(inputs / group)] of [outputs, inputs]."""
    _want(weights.dim() == 2, "weights must be [outputs, inputs]")
    outputs, inputs = weights.shape
    dev = _device(ctx)
    _want(group in (32, 64, 128), "group must be 32, 64 or 128")
    codes = torch.empty((outputs, 16 * -(-inputs // 32)), dtype=torch.uint8, device=weights.device)
    scales = torch.empty((outputs, -(-inputs // group)), dtype=torch.float32, device=weights.device)
    _check(lib().gorila_quantize_weights(
        _at(dev, weights, "weights", weights.shape, weights.dtype, 1), weights.stride(0), outputs, inputs, _dtype(weights), group,
        codes.data_ptr(), scales.data_ptr(), ctx.bind_stream()), "gorila_quantize_weights")
    return codes, scales


def qmatvec(ctx, x, codes, scales, group: int = 64, x_scale=None):
    """y [rows, outputs] of x [rows, inputs] and 4-bit weights; int8 x with x_scale [rows] gives float32."""
    _want(x.dim() == 2 and codes.dim() == 2, "x must be [rows, inputs], codes [outputs, bytes]")
    rows, inputs = x.shape
    outputs, dev = codes.shape[0], _device(ctx)
    _want(group in (32, 64, 128), "group must be 32, 64 or 128")
    if x.dtype == torch.int8:
        _want(x_scale is not None, "int8 rows need x_scale")
        dt, typ = GORILA_CODES, torch.float32
    else:
        _want(x_scale is None, "x_scale goes with int8 rows")
        dt, typ = _dtype(x), x.dtype
    y = torch.empty((rows, outputs), dtype=typ, device=x.device)
    _check(lib().gorila_qmatvec(
        _at(dev, x, "x", x.shape, x.dtype, 1), x.stride(0), _at(dev, x_scale, "x_scale", (rows,), torch.float32), dt, rows,
        _at(dev, codes, "codes", (outputs, 16 * -(-inputs // 32)), torch.uint8),
        _at(dev, scales, "scales", (outputs, -(-inputs // group)), torch.float32), outputs, inputs, group, y.data_ptr(),
        ctx.bind_stream()), "gorila_qmatvec")
    return y
