"""Matrices in 8 bits without rows or columns, as an empty batch has them: their strides say nothing and are not looked at.  The first test needs no GPU."""
import pytest
import torch

import paper_2503_10017_amd as fnn
from net_helpers import DEV, normal
from test_abi import lib  # noqa: F401
from test_net8_abi import scaled
from test_net_abi import OK, matrix

NOTHING = dict(n=0, data=0, scale=0, scale_block=0)


def test_strides_of_nothing_are_not_looked_at(lib):  # noqa: F811
    none = matrix(n=0, d=300, data=0)
    for high in (1, 128):
        assert lib.fnn_quantize(none, 0, scaled(high=high, d=300, **NOTHING), None) == OK
        assert lib.fnn_quantize(none, 1, scaled(n=300, d=0, high=high, data=0, scale=0, scale_row=0, scale_block=0), None) == OK
    assert lib.fnn_rms_norm(none, None, None, 1, 1e-6, None, None, scaled(d=300, **NOTHING), None, None) == OK
    w = scaled(n=32, d=300, high=128)
    assert lib.fnn_linear_e4m3(scaled(d=300, **NOTHING), w, None, 0, None, matrix(n=0, d=32, data=0), None, None, 0, None) == OK
    ws = lib.fnn_linear_e4m3_workspace_bytes(100, 300, 0, 1)
    assert lib.fnn_linear_e4m3(scaled(n=100, d=300), scaled(d=300, high=128, **NOTHING), None, 0, None, matrix(n=100, d=0, data=0), None, 0x100000, ws, None) == OK


@pytest.mark.gpu
@pytest.mark.parametrize("d", [1, 128, 129, 1000])
def test_an_empty_batch(d):
    """Norm, quantising, layer and gradients of no tokens."""
    bf = torch.bfloat16
    x, w = torch.zeros((0, d), device=DEV, dtype=bf), fnn.fnn_quantize(normal(1, 300, d), tiles=True)
    for tiles in (False, True):
        for transposed in (False, True):
            got = fnn.fnn_quantize(x, tiles=tiles, transposed=transposed)
            assert got.data.shape == ((d, 0) if transposed else (0, d))
            fnn.fnn_quantize(x, tiles=tiles, transposed=transposed, out=got)
    y, scaled_y, total, rstd = fnn.fnn_rms_norm(x, None, x, want_scaled=True, want_rstd=True)
    assert y.shape == total.shape == scaled_y.data.shape == (0, d) and rstd.shape == (0,)
    out, pre = fnn.fnn_linear_e4m3(scaled_y, w, act="gelu", want_pre=True)
    assert out.shape == pre.shape == (0, 300)
    dn, dw, db = fnn.fnn_linear_e4m3_backward(out, y, w, pre, act="gelu")
    assert dn.shape == (0, d) and not dw.any() and not db.any()
    dx, dnw = fnn.fnn_rms_norm_backward(dn, total, rstd)
    assert dx.shape == (0, d) and not dnw.any()
    empty = fnn.fnn_quantize(torch.zeros((0, d), device=DEV), tiles=True)
    assert fnn.fnn_linear_e4m3(fnn.fnn_quantize(normal(2, 40, d)), empty)[0].shape == (40, 0)
