"""Binding of the sequence operators: a recurrent core on feature rows.

Every function checks its tensors, allocates its outputs and makes one call of the
library on the current stream, in native code (csrc/binding.cpp): the host's time is
what a single step costs.  include/gorila.h has the definitions, layouts and errors.
Rows (x, y, their gradients, windows) are float32 or bfloat16, parameters, parameter
gradients, states and scales float32, resets uint8, slots int32.  Inputs may be strided
in their leading dimensions.  `ctx` needs a workspace where a `*_workspace_bytes`
function exists: ``Context(..., min_bytes=...)`` of the largest batch and length takes
the smaller ones too.
"""
from __future__ import annotations

import ctypes

import torch

from . import _check, lib

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


_raw_stream = torch._C._cuda_getCurrentRawStream
_native = None


def _load():
    """The native half (csrc/binding.cpp), on the library that the package loaded."""
    global _native
    from . import _binding
    names = [n for n, (res, _) in SIGNATURES.items() if res is _i32] + ["gorila_ctx_set_stream"]
    _binding.init({n: ctypes.cast(getattr(lib(), n), _vp).value for n in names}, _check)
    _native = _binding
    return _binding


# ---- norm ----

def add_rmsnorm(ctx, x, weight, residual=None, eps: float = 1e-6):
    """y, total, rstd of total = x + residual (x itself without one) and y = its norm times weight."""
    return (_native or _load()).add_rmsnorm(ctx.address, ctx.index, _raw_stream(ctx.index), x, weight, residual, eps)


def add_rmsnorm_codes(ctx, x, weight, residual=None, eps: float = 1e-6):
    """codes (int8), scale, total: codes * scale[:, None] stands for add_rmsnorm's y."""
    return (_native or _load()).add_rmsnorm_codes(ctx.address, ctx.index, _raw_stream(ctx.index), x, weight, residual, eps)


def add_rmsnorm_workspace_bytes(width: int) -> int:
    return int(lib().gorila_add_rmsnorm_workspace_bytes(width))


def add_rmsnorm_backward(ctx, dy, total, rstd, weight, dtotal=None):
    """dx (of x and of residual), dweight for the gradients that reach y and total."""
    return (_native or _load()).add_rmsnorm_backward(ctx.address, ctx.index, _raw_stream(ctx.index), dy, total, rstd, weight, dtotal)


# ---- short causal convolution ----

def causal_conv(ctx, x, weight, bias=None, reset=None, window=None, silu: bool = True):
    """y [batch, length, channels] and the window [batch, taps - 1, channels] for the steps that follow."""
    return (_native or _load()).causal_conv(ctx.address, ctx.index, _raw_stream(ctx.index), x, weight, bias, reset, window, silu)


def causal_conv_workspace_bytes(channels: int, taps: int) -> int:
    return int(lib().gorila_causal_conv_workspace_bytes(channels, taps))


def causal_conv_backward(ctx, dy, x, weight, bias=None, reset=None, window=None, silu: bool = True, dwindow_out=None):
    """dx, dweight, dbias, dwindow (the last two None without a bias or window)."""
    return (_native or _load()).causal_conv_backward(ctx.address, ctx.index, _raw_stream(ctx.index), dy, x, weight, bias, reset,
                                                     window, silu, dwindow_out)


def causal_conv_step(ctx, x, window_pool, weight, bias=None, slot=None, reset=None, silu: bool = True):
    """One step of every row of x [rows, channels]; window_pool [slots, taps - 1, channels] is updated."""
    return (_native or _load()).causal_conv_step(ctx.address, ctx.index, _raw_stream(ctx.index), x, weight, bias, reset,
                                                 window_pool, slot, silu)


# ---- selective scan ----

def scan_workspace_bytes(batch: int, length: int, heads: int, head_dim: int, groups: int, state_dim: int,
                         backward: bool = False) -> int:
    return int(lib().gorila_scan_workspace_bytes(batch, length, heads, head_dim, groups, state_dim, 1 if backward else 0))


def scan(ctx, x, dt, b, c, a_log, dt_bias, skip, reset=None, state=None):
    """y [batch, length, heads, head_dim] and the state after the last step (float32
    [batch, heads, head_dim, state_dim]); state: the one before the first (None: zeros)."""
    return (_native or _load()).scan(ctx.address, ctx.index, _raw_stream(ctx.index), x, dt, b, c, a_log, dt_bias, skip, reset, state)


def scan_backward(ctx, dy, x, dt, b, c, a_log, dt_bias, skip, reset=None, state=None, dstate_out=None):
    """dx, ddt, db, dc, da_log, ddt_bias, dskip, dstate (None without a state)."""
    return (_native or _load()).scan_backward(ctx.address, ctx.index, _raw_stream(ctx.index), dy, x, dt, b, c, a_log, dt_bias, skip,
                                              reset, state, dstate_out)


def scan_step(ctx, x, dt, b, c, a_log, dt_bias, skip, state_pool, slot=None, reset=None):
    """One step of every row of x [rows, heads, head_dim]; state_pool [slots, heads, head_dim, state_dim] is updated."""
    return (_native or _load()).scan_step(ctx.address, ctx.index, _raw_stream(ctx.index), x, dt, b, c, a_log, dt_bias, skip, reset,
                                          state_pool, slot)


# ---- 4-bit weights ----

def quantize_weights(ctx, weights, group: int = 64):
    """codes (uint8 [outputs, 16 * ceil(inputs / 32)]), scales [outputs, ceil(inputs / group)] of [outputs, inputs]."""
    return (_native or _load()).quantize_weights(ctx.address, ctx.index, _raw_stream(ctx.index), weights, group)


def qmatvec(ctx, x, codes, scales, group: int = 64, x_scale=None):
    """y [rows, outputs] of x [rows, inputs] and 4-bit weights; int8 x with x_scale [rows] gives float32."""
    return (_native or _load()).qmatvec(ctx.address, ctx.index, _raw_stream(ctx.index), x, codes, scales, group, x_scale)
