"""ctypes binding of the network's operators in libfnn.so (include/fnn_net.h): argument marshalling only.

Every function has the name and meaning of the C entry point it wraps; torch supplies device memory and the current stream.
Tensors are taken with the strides that they have, as long as the elements of a row are contiguous.  With ``stream`` a call runs on that stream: outputs and
workspaces that it is not given are of that stream's memory, and the inputs have to be ready there.

Nothing here enters torch's autograd graph, whether or not a tensor requires a gradient: gradients are calls of their own (fnn_..._backward).
"""
from __future__ import annotations

import struct
from typing import Optional

import torch

from .binding import _DTYPES, FnnError, _empty, _pack_map, _ptr, _workspace, load_library


def _matrix(t: Optional[torch.Tensor], what: str):
    """A struct fnn_map of a 2-D device tensor (None: NULL)."""
    if t is None:
        return None
    if t.dim() != 2 or not t.is_cuda:
        raise ValueError(f"{what} must be a 2-D device tensor")
    if t.dtype not in _DTYPES:
        raise ValueError(f"unsupported dtype {t.dtype} of {what}")
    n, d = t.shape
    row_stride, element_stride = t.stride()
    if d > 1 and element_stride != 1:
        raise ValueError(f"the rows of {what} must be contiguous")
    return _pack_map(t.data_ptr(), n, d, _DTYPES[t.dtype], row_stride if n > 1 else max(d, row_stride))


def _vector(t: Optional[torch.Tensor], count: int, dtype, what: str):
    """The address of a contiguous device tensor of `count` elements of `dtype` (None: NULL)."""
    if t is None:
        return None
    if not t.is_cuda or t.numel() != count or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous device tensor of {count} elements")
    if t.dtype != dtype:
        raise ValueError(f"{what} must be of {dtype}")
    return t.data_ptr()


def _stream_ptr(stream, device):
    # the current stream's handle as it stands: making the Stream object that names it takes 2 us, as long as these operators take on few tokens
    return stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(device.index)


def _like(t: torch.Tensor, stream):
    """_empty of t's shape and type; empty_like takes 2 us less on the host, a fifth of a call on one token."""
    return torch.empty_like(t) if stream is None else _empty(t.shape, t.dtype, t.device, stream)


def _scratch(need: int, device, stream):
    """A workspace of the call's own (None: none is needed)."""
    return _workspace(need, device, stream) if need else None


def _check(status: int, where: str):
    if status != 0:
        raise FnnError(status, where)


def _weight_dtype(x, weight, bias):
    of = weight if weight is not None else bias
    return x.dtype if of is None else of.dtype


def fnn_layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-6,
                   out: Optional[torch.Tensor] = None, want_stats: bool = False, stream=None):
    """Layer norm over the rows of x [n][d]; weight and bias [d] of x's dtype or fp32.  Returns (y, mean, rstd), the latter two
    float32 [n] for the gradient, or None without ``want_stats``."""
    lib = load_library()
    xm = _matrix(x, "x")
    n, d = x.shape
    wt = _weight_dtype(x, weight, bias)
    if out is None:
        out = _like(x, stream)
    mean = rstd = None
    if want_stats:
        mean = _empty(n, torch.float32, x.device, stream)
        rstd = _empty(n, torch.float32, x.device, stream)
    _check(lib.fnn_layer_norm(xm, _vector(weight, d, wt, "weight"), _vector(bias, d, wt, "bias"), _DTYPES.get(wt, -1), eps,
                              _matrix(out, "out"), _ptr(mean), _ptr(rstd), _stream_ptr(stream, x.device)), "fnn_layer_norm")
    return out, mean, rstd


def fnn_layer_norm_backward_workspace_bytes(n: int, d: int) -> int:
    return int(load_library().fnn_layer_norm_backward_workspace_bytes(n, d))


def fnn_layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                            weight: Optional[torch.Tensor] = None, want_x: bool = True, want_weight: bool = True,
                            out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """Gradient of fnn_layer_norm; returns (dx, dweight, dbias), the latter two of weight's dtype (x's without a weight), None
    where not wanted."""
    lib = load_library()
    n, d = x.shape
    wt = x.dtype if weight is None else weight.dtype
    dx = out
    if dx is None and want_x:
        dx = _like(x, stream)
    dweight = dbias = None
    if want_weight:
        dweight = _empty(d, wt, x.device, stream)
        dbias = _empty(d, wt, x.device, stream)
        if workspace is None:
            workspace = _scratch(lib.fnn_layer_norm_backward_workspace_bytes(n, d), x.device, stream)
    _check(lib.fnn_layer_norm_backward(_matrix(dy, "dy"), _matrix(x, "x"), _vector(mean, n, torch.float32, "mean"),
                                       _vector(rstd, n, torch.float32, "rstd"), _vector(weight, d, wt, "weight"),
                                       _DTYPES.get(wt, -1), _matrix(dx, "dx"), _ptr(dweight), _ptr(dbias), _ptr(workspace),
                                       0 if workspace is None else workspace.numel(), _stream_ptr(stream, x.device)),
           "fnn_layer_norm_backward")
    return dx, dweight, dbias


FNN_ACT_NONE, FNN_ACT_RELU, FNN_ACT_GELU, FNN_ACT_SILU = 0, 1, 2, 3
_ACTS = {"none": FNN_ACT_NONE, "relu": FNN_ACT_RELU, "gelu": FNN_ACT_GELU, "silu": FNN_ACT_SILU,
         FNN_ACT_NONE: FNN_ACT_NONE, FNN_ACT_RELU: FNN_ACT_RELU, FNN_ACT_GELU: FNN_ACT_GELU, FNN_ACT_SILU: FNN_ACT_SILU}


def fnn_linear_workspace_bytes(rows: int, inner: int, outer: int, dtype: torch.dtype) -> int:
    return int(load_library().fnn_linear_workspace_bytes(rows, inner, outer, _DTYPES[dtype]))


def fnn_linear(x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
               act="none", want_pre: bool = False, out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
               stream=None):
    """act(x w^T + bias) + residual for x [rows][inner], w [outer][inner]; act is "none", "relu", "gelu" or "silu".  Returns
    (y, pre), pre = x w^T + bias for the gradient, or None without ``want_pre``.  ``out`` may be ``residual``."""
    lib = load_library()
    xm, wm = _matrix(x, "x"), _matrix(w, "w")
    rows, inner = x.shape
    outer = w.shape[0]
    if out is None:
        out = _empty((rows, outer), x.dtype, x.device, stream)
    pre = _empty((rows, outer), x.dtype, x.device, stream) if want_pre else None
    if workspace is None:
        workspace = _scratch(lib.fnn_linear_workspace_bytes(rows, inner, outer, _DTYPES[x.dtype]), x.device, stream)
    _check(lib.fnn_linear(xm, wm, _vector(bias, outer, x.dtype, "bias"), _ACTS[act], _matrix(residual, "residual"),
                          _matrix(out, "out"), _matrix(pre, "pre"), _ptr(workspace), 0 if workspace is None else workspace.numel(),
                          _stream_ptr(stream, x.device)), "fnn_linear")
    return out, pre


def fnn_linear_backward_workspace_bytes(rows: int, inner: int, outer: int, dtype: torch.dtype, act="none") -> int:
    return int(load_library().fnn_linear_backward_workspace_bytes(rows, inner, outer, _DTYPES[dtype], _ACTS[act]))


def fnn_linear_backward(dy: torch.Tensor, x: torch.Tensor, w: torch.Tensor, pre: Optional[torch.Tensor] = None, act="none",
                        want_x: bool = True, want_w: bool = True, want_bias: bool = True, out: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None, stream=None):
    """Gradient of fnn_linear from dy [rows][outer] and, with an activation, pre; returns (dx, dw, dbias), None where not wanted
    (dx is written to ``out`` if given).  The residual's gradient is dy."""
    lib = load_library()
    rows, inner = x.shape
    outer = w.shape[0]
    dx = out
    if dx is None and want_x:
        dx = _empty((rows, inner), x.dtype, x.device, stream)
    dw = _empty((outer, inner), x.dtype, x.device, stream) if want_w else None
    dbias = _empty(outer, x.dtype, x.device, stream) if want_bias else None
    if workspace is None:
        workspace = _scratch(lib.fnn_linear_backward_workspace_bytes(rows, inner, outer, _DTYPES[x.dtype], _ACTS[act]), x.device, stream)
    _check(lib.fnn_linear_backward(_matrix(dy, "dy"), _matrix(x, "x"), _matrix(w, "w"), _matrix(pre, "pre"), _ACTS[act],
                                   _matrix(dx, "dx"), _matrix(dw, "dw"), _ptr(dbias), _ptr(workspace), 0 if workspace is None else workspace.numel(),
                                   _stream_ptr(stream, x.device)), "fnn_linear_backward")
    return dx, dw, dbias


# a struct fnn_heads
_pack_heads = struct.Struct("=QqiiiiQQ").pack


def _heads(t: torch.Tensor, what: str):
    if t.dim() != 3 or not t.is_cuda:
        raise ValueError(f"{what} must be a device tensor of [tokens][heads][dim]")
    if t.dtype not in _DTYPES:
        raise ValueError(f"unsupported dtype {t.dtype} of {what}")
    n, heads, d = t.shape
    row_stride, head_stride, element_stride = t.stride()
    if d > 1 and element_stride != 1:
        raise ValueError(f"the vectors of {what} must be contiguous")
    return _pack_heads(t.data_ptr(), n, heads, d, _DTYPES[t.dtype], 0, row_stride if n > 1 else max(d, row_stride), head_stride if heads > 1 else max(d, head_stride))


def _sequences(cu_q, cu_k):
    """batch and the two tables' addresses; None: one sequence of everything."""
    if cu_q is None and cu_k is None:
        return 1, None, None
    if cu_q is None or cu_k is None or cu_q.numel() != cu_k.numel():
        raise ValueError("cu_q and cu_k must be given together and have the same length")
    n = cu_q.numel()
    return n - 1, _vector(cu_q, n, torch.int32, "cu_q"), _vector(cu_k, n, torch.int32, "cu_k")


def fnn_attention_workspace_bytes(tokens_q: int, tokens_k: int, batch: int, heads: int, key_heads: int, d: int) -> int:
    return int(load_library().fnn_attention_workspace_bytes(tokens_q, tokens_k, batch, heads, key_heads, d))


def fnn_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: Optional[torch.Tensor] = None,
                  cu_k: Optional[torch.Tensor] = None, causal: bool = False, scale: Optional[float] = None,
                  out: Optional[torch.Tensor] = None, want_lse: bool = True, workspace: Optional[torch.Tensor] = None, stream=None):
    """Attention of q [tokens][heads][dim] over k, v [tokens][key heads][dim], sequences packed as cu_q, cu_k int32 [batch + 1] say;
    scale is 1 / sqrt(dim) unless given.  Returns (out, lse), lse float32 [tokens][heads] for the gradient."""
    lib = load_library()
    qm, km, vm = _heads(q, "q"), _heads(k, "k"), _heads(v, "v")
    tokens, heads, d = q.shape
    batch, cq, ck = _sequences(cu_q, cu_k)
    if out is None:
        out = _empty((tokens, heads, d), q.dtype, q.device, stream)
    lse = _empty((tokens, heads), torch.float32, q.device, stream) if want_lse else None
    if workspace is None:
        workspace = _scratch(lib.fnn_attention_workspace_bytes(tokens, k.shape[0], batch, heads, k.shape[1], d), q.device, stream)
    _check(lib.fnn_attention(qm, km, vm, batch, cq, ck, causal, d ** -0.5 if scale is None else scale, _heads(out, "out"),
                             _ptr(lse), _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_ptr(stream, q.device)),
           "fnn_attention")
    return out, lse


def fnn_attention_backward_workspace_bytes(tokens_q: int, tokens_k: int, batch: int, heads: int, key_heads: int, d: int) -> int:
    return int(load_library().fnn_attention_backward_workspace_bytes(tokens_q, tokens_k, batch, heads, key_heads, d))


def fnn_attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor,
                           cu_q: Optional[torch.Tensor] = None, cu_k: Optional[torch.Tensor] = None, causal: bool = False,
                           scale: Optional[float] = None, want_q: bool = True, want_kv: bool = True, out_grads=None,
                           workspace: Optional[torch.Tensor] = None, stream=None):
    """Gradient of fnn_attention from dout and the forward call's inputs and outputs; returns (dq, dk, dv), None where not wanted.
    ``out_grads``: three tensors to write them to (slices of one buffer, say)."""
    lib = load_library()
    tokens, heads, d = q.shape
    batch, cq, ck = _sequences(cu_q, cu_k)
    if out_grads is not None:
        dq, dk, dv = out_grads
    else:
        dq = _empty(q.shape, q.dtype, q.device, stream) if want_q else None
        dk = _empty(k.shape, k.dtype, k.device, stream) if want_kv else None
        dv = _empty(v.shape, v.dtype, v.device, stream) if want_kv else None
    if workspace is None:
        workspace = _scratch(lib.fnn_attention_backward_workspace_bytes(tokens, k.shape[0], batch, heads, k.shape[1], d), q.device, stream)
    grads = [None if g is None else _heads(g, "a gradient") for g in (dq, dk, dv)]
    _check(lib.fnn_attention_backward(_heads(dout, "dout"), _heads(q, "q"), _heads(k, "k"), _heads(v, "v"), _heads(out, "out"),
                                      _vector(lse, tokens * heads, torch.float32, "lse"), batch, cq, ck, causal, d ** -0.5 if scale is None else scale,
                                      *grads, _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_ptr(stream, q.device)),
           "fnn_attention_backward")
    return dq, dk, dv
