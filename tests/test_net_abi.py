"""Host-only checks of the network operators' C ABI: fnn_net.h's functions are exported and bad arguments are refused before
the device is touched (no GPU needed)."""
import math
import os
import subprocess

import pytest

import paper_2503_10017_amd as fnn
from paper_2503_10017_amd import binding
from test_abi import ROOT, declared_functions, lib  # noqa: F401

OK, NULL, SHAPE, DTYPE, RANGE, WORKSPACE, HIP, UNSUPPORTED = range(8)


def matrix(n=4, d=64, dtype=1, stride=None, data=0x10000):
    return binding._pack_map(data, n, d, dtype, d if stride is None else stride)


def test_every_declared_symbol_is_exported(lib):  # noqa: F811
    names = set(declared_functions("fnn_net.h"))
    assert {"fnn_layer_norm", "fnn_layer_norm_backward", "fnn_layer_norm_backward_workspace_bytes"} <= names
    for name in names:
        assert hasattr(lib, name) and hasattr(fnn, name), name


def test_header_is_plain_c(tmp_path):
    source = tmp_path / "use.c"
    source.write_text('#include "fnn_net.h"\nint main(void) { return 0; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), "-c", str(source), "-o", str(tmp_path / "use.o")], check=True)


def test_layer_norm_refusals(lib):  # noqa: F811
    def call(x=matrix(), y=matrix(data=0x20000), weight=0x3000, bias=0x4000, weight_dtype=1, eps=1e-6):
        return lib.fnn_layer_norm(x, weight, bias, weight_dtype, eps, y, None, None, None)

    assert call(x=None) == NULL and call(y=None) == NULL
    assert call(x=matrix(data=0)) == NULL and call(y=matrix(data=0)) == NULL
    for bad in (matrix(n=-1), matrix(n=2 ** 31), matrix(d=0), matrix(d=-4, stride=64), matrix(d=16385), matrix(stride=63), matrix(stride=2 ** 62), matrix(n=5), matrix(d=32)):
        assert call(x=bad) == SHAPE and call(y=bad) == SHAPE
    assert call(x=matrix(dtype=3)) == DTYPE and call(y=matrix(dtype=2)) == DTYPE
    assert call(weight_dtype=2) == DTYPE and call(weight_dtype=7) == DTYPE
    for eps in (-1e-9, math.nan, math.inf):
        assert call(eps=eps) == RANGE
    assert call(x=matrix(n=0, data=0), y=matrix(n=0, data=0)) == OK
    assert call(x=matrix(n=0, data=0, stride=0), y=matrix(n=0, data=0)) == OK


def test_layer_norm_backward_refusals(lib):  # noqa: F811
    need = fnn.fnn_layer_norm_backward_workspace_bytes(4, 64)
    assert need > 0
    for n, d in ((-1, 64), (4, 0), (4, 16385), (2 ** 31, 8)):
        assert fnn.fnn_layer_norm_backward_workspace_bytes(n, d) == 0

    def call(dy=matrix(), x=matrix(), mean=0x5000, rstd=0x6000, weight_dtype=1, dx=matrix(data=0x20000), dweight=0x7000, ws=0x100000, ws_bytes=need):
        return lib.fnn_layer_norm_backward(dy, x, mean, rstd, 0x3000, weight_dtype, dx, dweight, None, ws, ws_bytes, None)

    assert call(dy=None) == NULL and call(x=None) == NULL and call(mean=None) == NULL and call(rstd=None) == NULL
    for bad in (matrix(n=3), matrix(d=32), matrix(stride=1)):
        assert call(dy=bad) == SHAPE and call(x=bad) == SHAPE and call(dx=bad) == SHAPE
    assert call(dy=matrix(dtype=0)) == DTYPE and call(dx=matrix(dtype=2)) == DTYPE and call(weight_dtype=2) == DTYPE
    assert call(ws=None) == WORKSPACE and call(ws=0x100010) == WORKSPACE and call(ws_bytes=need - 1) == WORKSPACE
    assert call(dx=None, dweight=None) == OK     # nothing wanted


def test_linear_refusals(lib):  # noqa: F811
    x, w, y = matrix(n=100, d=64), matrix(n=32, d=64, data=0x20000), matrix(n=100, d=32, data=0x30000)
    assert fnn.net._DTYPES and lib.fnn_linear_workspace_bytes(100, 64, 32, 1) == 0
    need = lib.fnn_linear_workspace_bytes(100, 64000, 32, 1)
    assert need > 0
    for sizes in ((-1, 64, 32, 1), (100, -1, 32, 1), (100, 64, 2 ** 31, 1), (100, 64, 32, 5)):
        assert lib.fnn_linear_workspace_bytes(*sizes) == 0

    def call(x=x, w=w, y=y, act=0, residual=None, pre=None, ws=None, ws_bytes=0):
        return lib.fnn_linear(x, w, None, act, residual, y, pre, ws, ws_bytes, None)

    assert call(x=None) == NULL and call(w=None) == NULL and call(y=None) == NULL
    assert call(x=matrix(n=100, d=64, data=0)) == NULL
    for bad in (matrix(n=100, d=63), matrix(n=-1), matrix(n=100, d=64, stride=63)):
        assert call(x=bad) == SHAPE and call(y=bad) == SHAPE and call(residual=bad) == SHAPE and call(pre=bad) == SHAPE
    assert call(w=matrix(n=31, d=64)) == SHAPE and call(w=matrix(n=32, d=65)) == SHAPE
    for bad in (0, 2):
        assert call(w=matrix(n=32, d=64, dtype=bad)) == DTYPE and call(y=matrix(n=100, d=32, dtype=bad)) == DTYPE
        assert call(residual=matrix(n=100, d=32, dtype=bad)) == DTYPE and call(pre=matrix(n=100, d=32, dtype=bad)) == DTYPE
    assert call(x=matrix(n=100, d=64, dtype=9)) == DTYPE
    assert call(act=-1) == RANGE and call(act=4) == RANGE
    long = dict(x=matrix(n=100, d=64000), w=matrix(n=32, d=64000))
    assert call(**long) == WORKSPACE and call(**long, ws=0x100001, ws_bytes=need) == WORKSPACE and call(**long, ws=0x100000, ws_bytes=need - 1) == WORKSPACE
    nothing = dict(x=matrix(n=0, d=64, data=0), y=matrix(n=0, d=32, data=0))
    assert call(**nothing) == OK


def test_linear_backward_refusals(lib):  # noqa: F811
    need = lib.fnn_linear_backward_workspace_bytes(100, 64, 32, 1, 2)
    assert need >= 100 * 32 * 2
    for sizes in ((-1, 64, 32, 1, 0), (100, -1, 32, 1, 0), (100, 64, 2 ** 31, 1, 0), (100, 64, 32, 5, 0), (100, 64, 32, 1, 4)):
        assert lib.fnn_linear_backward_workspace_bytes(*sizes) == 0

    def call(dy=matrix(n=100, d=32), x=matrix(n=100, d=64), w=matrix(n=32, d=64), pre=matrix(n=100, d=32), act=2, dx=matrix(n=100, d=64, data=0x20000),
             dw=matrix(n=32, d=64, data=0x30000), dbias=None, ws=0x100000, ws_bytes=need):
        return lib.fnn_linear_backward(dy, x, w, pre, act, dx, dw, dbias, ws, ws_bytes, None)

    for name in ("dy", "x", "w", "pre"):
        assert call(**{name: None}) == NULL
    for name, good in (("dy", (100, 32)), ("x", (100, 64)), ("w", (32, 64)), ("pre", (100, 32)), ("dx", (100, 64)), ("dw", (32, 64))):
        n, d = good
        for bad in (matrix(n=n + 1, d=d), matrix(n=n, d=d - 1), matrix(n=n, d=d, stride=d - 1)):
            assert call(**{name: bad}) == SHAPE, name
        assert call(**{name: matrix(n=n, d=d, dtype=2)}) == DTYPE, name
    assert call(act=4) == RANGE
    assert call(ws=None) == WORKSPACE and call(ws=0x100008) == WORKSPACE and call(ws_bytes=need - 1) == WORKSPACE
    assert call(dx=None, dw=None) == OK      # nothing wanted


def heads(n=10, h=4, d=64, dtype=1, row=None, head=None, data=0x10000, reserved=0):
    return fnn.net._pack_heads(data, n, h, d, dtype, reserved, h * d if row is None else row, d if head is None else head)


def test_attention_refusals(lib):  # noqa: F811
    assert lib.fnn_attention_workspace_bytes(1000, 1000, 4, 4, 2, 64) == 0
    need = lib.fnn_attention_workspace_bytes(1, 100000, 1, 4, 2, 64)
    assert need > 0
    for sizes in ((-1, 9, 1, 4, 2, 64), (9, -1, 1, 4, 2, 64), (9, 9, 0, 4, 2, 64), (9, 9, 1, 4, 3, 64), (9, 9, 1, 0, 1, 64), (9, 9, 1, 4, 2, 129), (9, 9, 1, 4, 2, 0), (2 ** 30, 9, 1, 4, 2, 64)):
        assert lib.fnn_attention_workspace_bytes(*sizes) == 0 and lib.fnn_attention_backward_workspace_bytes(*sizes) == 0

    def call(q=heads(), k=heads(h=2), v=heads(h=2), batch=1, cu_q=0x500, cu_k=0x600, scale=0.125, out=heads(data=0x20000), ws=None, ws_bytes=0):
        return lib.fnn_attention(q, k, v, batch, cu_q, cu_k, 0, scale, out, None, ws, ws_bytes, None)

    for name, h in (("q", 4), ("k", 2), ("v", 2), ("out", 4)):
        assert call(**{name: None}) == NULL and call(**{name: heads(h=h, data=0)}) == NULL
        for bad in (heads(n=-1, h=h), heads(n=11, h=h), heads(h=3), heads(h=0), heads(h=h, d=63), heads(h=h, d=129), heads(h=h, d=0), heads(h=h, row=63), heads(h=h, head=63),
                    heads(h=h, row=2 ** 62), heads(h=h, reserved=1)):
            if name in ("k", "v") or bad != heads(n=11, h=h):
                assert call(**{name: bad}) == SHAPE, name
        assert call(**{name: heads(h=h, dtype=0)}) == DTYPE and call(**{name: heads(h=h, dtype=2)}) == DTYPE and call(**{name: heads(h=h, dtype=5)}) == DTYPE
    for scale in (0.0, -1.0, math.nan, math.inf):
        assert call(scale=scale) == RANGE
    assert call(batch=0) == RANGE
    assert call(cu_q=None) == NULL and call(cu_k=None) == NULL and call(cu_q=None, cu_k=None, batch=2) == NULL
    long = dict(q=heads(n=1), out=heads(n=1), k=heads(n=100000, h=2), v=heads(n=100000, h=2))
    assert call(**long) == WORKSPACE and call(**long, ws=0x100004, ws_bytes=need) == WORKSPACE and call(**long, ws=0x100000, ws_bytes=need - 1) == WORKSPACE
    assert call(q=heads(n=0, data=0), out=heads(n=0, data=0)) == OK


def test_attention_backward_refusals(lib):  # noqa: F811
    need = lib.fnn_attention_backward_workspace_bytes(10, 10, 1, 4, 2, 64)
    assert need >= 10 * 4 * 4

    def call(dout=heads(), q=heads(), k=heads(h=2), v=heads(h=2), out=heads(), lse=0x700, batch=1, scale=0.125, dq=heads(data=0x20000), dk=heads(h=2, data=0x30000),
             dv=heads(h=2, data=0x40000), ws=0x100000, ws_bytes=need):
        return lib.fnn_attention_backward(dout, q, k, v, out, lse, batch, 0x500, 0x600, 0, scale, dq, dk, dv, ws, ws_bytes, None)

    for name in ("dout", "q", "k", "v", "out", "lse"):
        assert call(**{name: None}) == NULL, name
    for name, h in (("dout", 4), ("out", 4), ("dq", 4), ("dk", 2), ("dv", 2)):
        for bad in (heads(n=11, h=h), heads(h=h + 1), heads(h=h, d=32), heads(h=h, row=1)):
            assert call(**{name: bad}) == SHAPE, name
        assert call(**{name: heads(h=h, dtype=2)}) == DTYPE and call(**{name: heads(h=h, dtype=0)}) == DTYPE
    assert call(scale=0.0) == RANGE and call(batch=-1) == RANGE
    assert call(ws=None) == WORKSPACE and call(ws=0x100080) == WORKSPACE and call(ws_bytes=need - 1) == WORKSPACE
    assert call(dq=None, dk=None, dv=None) == OK
