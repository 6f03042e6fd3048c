"""ctypes binding of the operators whose matrices are held in 8 bits, e4m3 codes with a scale for each block of 128 (include/fnn_net.h); as net.py: argument
marshalling only, the names and meanings of the C entry points, nothing enters torch's autograd graph.

All tensors of a call have to be on one device, which need not be the current one.
"""
from __future__ import annotations

import struct
from typing import NamedTuple, Optional

import torch

from .binding import _DTYPES, _empty, _ptr, load_library
from .net import _ACTS, _check, _like, _matrix, _pack_map, _scratch, _stream_ptr, _vector

SCALED_BLOCK = 128


class FnnScaled(NamedTuple):
    """A matrix in 8 bits: data [n][d] of float8_e4m3fn, scale float32 [n][blocks] or, one to a tile of 128 rows, [tiles][blocks], for blocks of 128 columns.
    Element (r, k) is data[r, k] * scale[r, k // 128], or scale[r // 128, k // 128]."""
    data: torch.Tensor
    scale: torch.Tensor


# a struct fnn_scaled
_pack_scaled = struct.Struct("=QQqiiqqq").pack


def _blocks(n: int) -> int:
    return -(-n // SCALED_BLOCK)


def _scaled(s: Optional[FnnScaled], what: str):
    """A struct fnn_scaled (None: NULL)."""
    if s is None:
        return None
    data, scale = s
    if data.dim() != 2 or scale.dim() != 2 or not data.is_cuda or not scale.is_cuda:
        raise ValueError(f"{what} must be 2-D device tensors of codes and scales")
    if data.dtype != torch.float8_e4m3fn or scale.dtype != torch.float32:
        raise ValueError(f"{what} must be of float8_e4m3fn, its scales of float32")
    n, d = data.shape
    high, blocks = scale.shape
    if blocks != _blocks(d) or (high != n and high != _blocks(n)):
        raise ValueError(f"{what} of {n} x {d} has scales of {n} or {_blocks(n)} x {_blocks(d)}, not {high} x {blocks}")
    row_stride, element_stride = data.stride()
    if d > 1 and element_stride != 1:
        raise ValueError(f"the rows of {what} must be contiguous")
    scale_row, scale_block = scale.stride()
    return _pack_scaled(data.data_ptr(), scale.data_ptr(), n, d, 1 if high == n else SCALED_BLOCK, row_stride if n > 1 else max(d, row_stride),
                        scale_row, scale_block)


def _empty_scaled(n: int, d: int, tiles: bool, device, stream):
    """Rows of codes on 16-byte boundaries, the scales of a column of blocks next to each other; and the struct fnn_scaled that they are."""
    high, blocks = _blocks(n) if tiles else n, _blocks(d)
    stride = d if d % 16 == 0 else (d + 15) // 16 * 16
    data = _empty((n, stride), torch.float8_e4m3fn, device, stream)
    scale = _empty((1, blocks) if high == 1 else (blocks, high), torch.float32, device, stream)
    packed = _pack_scaled(data.data_ptr(), scale.data_ptr(), n, d, 1 if high == n else SCALED_BLOCK, stride, 1, high)
    return FnnScaled(data if stride == d else data[:, :d], scale if high == 1 else scale.t()), packed


def _fresh(t: torch.Tensor, n: int, d: int):
    """The struct fnn_map of an output [n][d] of the call's own, without the checks of _matrix."""
    return _pack_map(t.data_ptr(), n, d, _DTYPES[t.dtype], d)


def _call(where: str, function, device, others, *args):
    """The call, on `device`; the tensors of `others` have to be there too."""
    index = -1 if device.index is None else device.index
    for t in others:
        if t is not None and t.get_device() != index:
            raise ValueError(f"{where}: tensors on {device} and {t.device}")
    if index < 0 or index == torch._C._cuda_getDevice():
        _check(function(*args), where)
    else:
        with torch.cuda.device(device):
            _check(function(*args), where)


def fnn_quantize(x: torch.Tensor, tiles: bool = False, transposed: bool = False, out: Optional[FnnScaled] = None, stream=None) -> FnnScaled:
    """x [n][d] in 8 bits, or with ``transposed`` its transpose [d][n]; a scale for each block of 128 of a row, or with ``tiles`` for each tile of 128 x 128."""
    lib = load_library()
    xm = _matrix(x, "x")
    n, d = x.shape
    if out is None:
        out, om = _empty_scaled(d, n, tiles, x.device, stream) if transposed else _empty_scaled(n, d, tiles, x.device, stream)
        others = ()
    else:
        om, others = _scaled(out, "out"), out
    _call("fnn_quantize", lib.fnn_quantize, x.device, others, xm, 1 if transposed else 0, om, _stream_ptr(stream, x.device))
    return out


def fnn_rms_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, eps: float = 1e-6, want_y: bool = True,
                 want_scaled: bool = False, want_rstd: bool = False, out: Optional[torch.Tensor] = None, out_scaled: Optional[FnnScaled] = None,
                 out_sum: Optional[torch.Tensor] = None, stream=None):
    """Root-mean-square norm over the rows of s = x + residual; weight [d] of x's dtype or fp32.  Returns (y, scaled, sum, rstd): y of x's dtype, or None without ``want_y``; the
    same in 8 bits as an FnnScaled with ``want_scaled``; s, or None without a residual; rstd float32 [n] for the gradient with ``want_rstd``.  ``out_sum`` may be
    x or residual itself."""
    lib = load_library()
    xm = _matrix(x, "x")
    n, d = x.shape
    wt = x.dtype if weight is None else weight.dtype
    others = (weight, residual, out, out_sum)
    ym, sm = _matrix(out, "out"), _matrix(out_sum, "out_sum")
    if out is None and want_y:
        out = _like(x, stream)
        ym = _fresh(out, n, d)
    if out_scaled is not None:
        cm = _scaled(out_scaled, "out_scaled")
        others += out_scaled
    elif want_scaled:
        out_scaled, cm = _empty_scaled(n, d, False, x.device, stream)
    else:
        cm = None
    if out_sum is None and residual is not None:
        out_sum = _like(x, stream)
        sm = _fresh(out_sum, n, d)
    rstd = _empty(n, torch.float32, x.device, stream) if want_rstd else None
    _call("fnn_rms_norm", lib.fnn_rms_norm, x.device, others, xm, _matrix(residual, "residual"),
          _vector(weight, d, wt, "weight"), _DTYPES.get(wt, -1), eps, sm, ym, cm, _ptr(rstd),
          _stream_ptr(stream, x.device))
    return out, out_scaled, out_sum, rstd


def fnn_rms_norm_backward_workspace_bytes(n: int, d: int) -> int:
    return int(load_library().fnn_rms_norm_backward_workspace_bytes(n, d))


def fnn_rms_norm_backward(dy: torch.Tensor, x: torch.Tensor, rstd: torch.Tensor, weight: Optional[torch.Tensor] = None, dsum: Optional[torch.Tensor] = None,
                          want_x: bool = True, want_weight: bool = True, out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """Gradient of fnn_rms_norm from dy, x (with a residual: the sum that it returned) and rstd; ``dsum`` [n][d], what else reaches the sum, is added to dx.  Returns
    (dx, dweight), the latter of weight's dtype (x's without a weight), None where not wanted."""
    lib = load_library()
    xm = _matrix(x, "x")
    n, d = x.shape
    wt = x.dtype if weight is None else weight.dtype
    dx = out
    if dx is None and want_x:
        dx = _like(x, stream)
    dweight = None
    if want_weight:
        dweight = _empty(d, wt, x.device, stream)
        if workspace is None:
            workspace = _scratch(lib.fnn_rms_norm_backward_workspace_bytes(n, d), x.device, stream)
    _call("fnn_rms_norm_backward", lib.fnn_rms_norm_backward, x.device, (dy, rstd, weight, dsum, dx, workspace), _matrix(dy, "dy"), xm,
          _vector(rstd, n, torch.float32, "rstd"), _vector(weight, d, wt, "weight"), _DTYPES.get(wt, -1), _matrix(dsum, "dsum"), _matrix(dx, "dx"), _ptr(dweight),
          _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_ptr(stream, x.device))
    return dx, dweight


def fnn_linear_e4m3_workspace_bytes(rows: int, inner: int, outer: int, dtype: torch.dtype) -> int:
    return int(load_library().fnn_linear_e4m3_workspace_bytes(rows, inner, outer, _DTYPES[dtype]))


def fnn_linear_e4m3(x: FnnScaled, w: FnnScaled, bias: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, act="none",
                    dtype: torch.dtype = torch.bfloat16, want_pre: bool = False, out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                    stream=None):
    """act(x w^T + bias) + residual for x [rows][inner] and w [outer][inner] in 8 bits; bias, residual and the results are of ``dtype`` (that of ``out``, if given).  Returns
    (y, pre), pre = x w^T + bias for the gradient, or None without ``want_pre``.  ``out`` may be ``residual``."""
    lib = load_library()
    xm, wm = _scaled(x, "x"), _scaled(w, "w")
    rows, inner = x.data.shape
    outer, device = w.data.shape[0], x.data.device
    if out is None:
        if dtype not in _DTYPES:
            raise ValueError(f"unsupported dtype {dtype} of the results")
        out = _empty((rows, outer), dtype, device, stream)
        om = _fresh(out, rows, outer)
    else:
        om = _matrix(out, "out")
    pre = _empty((rows, outer), out.dtype, device, stream) if want_pre else None
    if workspace is None:
        workspace = _scratch(lib.fnn_linear_e4m3_workspace_bytes(rows, inner, outer, _DTYPES[out.dtype]), device, stream)
    _call("fnn_linear_e4m3", lib.fnn_linear_e4m3, device, (x.scale, *w, bias, residual, out, workspace), xm, wm, _vector(bias, outer, out.dtype, "bias"), _ACTS[act],
          _matrix(residual, "residual"), om, None if pre is None else _fresh(pre, rows, outer), _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_ptr(stream, device))
    return out, pre


def fnn_linear_e4m3_backward_workspace_bytes(rows: int, inner: int, outer: int, dtype: torch.dtype) -> int:
    return int(load_library().fnn_linear_e4m3_backward_workspace_bytes(rows, inner, outer, _DTYPES[dtype]))


def fnn_linear_e4m3_backward(dy: torch.Tensor, x: torch.Tensor, w: FnnScaled, pre: Optional[torch.Tensor] = None, act="none", want_x: bool = True,
                             want_w: bool = True, want_bias: bool = True, out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """Gradient of fnn_linear_e4m3 from dy [rows][outer], x [rows][inner] as it was before its quantising, w in 8 bits with a scale to a tile (``fnn_quantize(..., tiles=True)``) and,
    with an activation, pre; dy times the activation's slope and x are quantised for the products.  Returns (dx, dw, dbias), None where not wanted."""
    lib = load_library()
    xm, wm = _matrix(x, "x"), _scaled(w, "w")
    rows, inner = x.shape
    outer = w.data.shape[0]
    dx = out
    if dx is None and want_x:
        dx = _empty((rows, inner), x.dtype, x.device, stream)
    dw = _empty((outer, inner), x.dtype, x.device, stream) if want_w else None
    dbias = _empty(outer, x.dtype, x.device, stream) if want_bias else None
    if workspace is None:
        workspace = _scratch(lib.fnn_linear_e4m3_backward_workspace_bytes(rows, inner, outer, _DTYPES[x.dtype]), x.device, stream)
    _call("fnn_linear_e4m3_backward", lib.fnn_linear_e4m3_backward, x.device, (dy, *w, pre, dx, workspace), _matrix(dy, "dy"), xm, wm, _matrix(pre, "pre"), _ACTS[act],
          _matrix(dx, "dx"), _matrix(dw, "dw"), _ptr(dbias), _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_ptr(stream, x.device))
    return dx, dw, dbias
