"""Host-only checks of the C ABI of the operators in 8 bits: bad arguments are refused before the device is touched; and, with the library and the allocator stood in for,
what the binding refuses and whose memory it takes.  No GPU needed."""
import math

import pytest
import torch

import paper_2503_10017_amd as fnn
from paper_2503_10017_amd import net8
from test_abi import lib  # noqa: F401
from test_net_abi import DTYPE, NULL, OK, RANGE, SHAPE, WORKSPACE, matrix
from test_net_streams import OnDevice, Stream, allocator, given  # noqa: F401


def scaled(n=4, d=300, high=1, stride=None, scale_row=1, scale_block=None, data=0x10000, scale=0x20000):
    return net8._pack_scaled(data, scale, n, d, high, d if stride is None else stride, scale_row, n if scale_block is None else scale_block)


BAD = [dict(n=-1), dict(n=2 ** 31), dict(d=-1, stride=300), dict(d=2 ** 31 - 63, stride=2 ** 31), dict(high=0), dict(high=2), dict(high=64), dict(stride=299), dict(stride=2 ** 62), dict(scale_row=0), dict(scale_row=-5),
       dict(scale_row=2 ** 61), dict(scale_block=0), dict(scale_block=-1), dict(scale_block=2 ** 61)]


def test_quantize_refusals(lib):  # noqa: F811
    def call(x=matrix(d=300), transposed=0, q=scaled()):
        return lib.fnn_quantize(x, transposed, q, None)

    assert call(x=None) == NULL and call(q=None) == NULL and call(x=matrix(d=300, data=0)) == NULL
    assert call(q=scaled(data=0)) == NULL and call(q=scaled(scale=0)) == NULL
    for bad in BAD:
        assert call(q=scaled(**bad)) == SHAPE, bad
    assert call(x=matrix(d=301)) == SHAPE and call(x=matrix(n=5, d=300)) == SHAPE and call(transposed=1) == SHAPE and call(q=scaled(n=300, d=4, scale_block=300)) == SHAPE
    assert call(x=matrix(d=300, dtype=3)) == DTYPE
    nothing = dict(x=matrix(n=0, d=300, data=0), q=scaled(n=0, data=0, scale=0, scale_block=4))
    assert call(**nothing) == OK


def test_rms_norm_refusals(lib):  # noqa: F811
    def call(x=matrix(d=300), residual=matrix(d=300), weight_dtype=1, eps=1e-6, total=matrix(d=300, data=0x30000), y=matrix(d=300, data=0x40000), codes=scaled()):
        return lib.fnn_rms_norm(x, residual, 0x5000, weight_dtype, eps, total, y, codes, None, None)

    assert call(x=None) == NULL and call(x=matrix(d=300, data=0)) == NULL and call(residual=matrix(d=300, data=0)) == NULL and call(codes=scaled(scale=0)) == NULL
    for bad in (matrix(n=-1, d=300), matrix(n=5, d=300), matrix(d=299), matrix(d=0), matrix(d=300, stride=10), matrix(d=16385)):
        assert call(x=bad) == SHAPE and call(residual=bad) == SHAPE and call(total=bad) == SHAPE and call(y=bad) == SHAPE
    for bad in BAD + [dict(n=5), dict(d=128), dict(high=128)]:
        assert call(codes=scaled(**bad)) == SHAPE, bad
    for bad in (0, 2, 7):
        assert call(residual=matrix(d=300, dtype=bad)) == DTYPE and call(total=matrix(d=300, dtype=bad)) == DTYPE and call(y=matrix(d=300, dtype=bad)) == DTYPE
    assert call(weight_dtype=2) == DTYPE and call(x=matrix(d=300, dtype=4)) == DTYPE
    for eps in (-1e-9, math.nan, math.inf):
        assert call(eps=eps) == RANGE
    assert call(total=None, y=None, codes=None) == OK               # nothing wanted
    none = dict(n=0, d=300, data=0)
    assert call(x=matrix(**none), residual=matrix(**none), total=None, y=matrix(**none), codes=scaled(n=0, data=0, scale=0, scale_block=4)) == OK


def test_rms_norm_backward_refusals(lib):  # noqa: F811
    need = fnn.fnn_rms_norm_backward_workspace_bytes(4, 64)
    assert need > 0
    for n, d in ((-1, 64), (4, 0), (4, 16385), (2 ** 31, 8)):
        assert fnn.fnn_rms_norm_backward_workspace_bytes(n, d) == 0

    def call(dy=matrix(), x=matrix(), rstd=0x6000, weight_dtype=1, dsum=matrix(), dx=matrix(data=0x20000), dweight=0x7000, ws=0x100000, ws_bytes=need):
        return lib.fnn_rms_norm_backward(dy, x, rstd, 0x3000, weight_dtype, dsum, dx, dweight, ws, ws_bytes, None)

    assert call(dy=None) == NULL and call(x=None) == NULL and call(rstd=None) == NULL
    for bad in (matrix(n=3), matrix(d=32), matrix(stride=1)):
        assert call(dy=bad) == SHAPE and call(x=bad) == SHAPE and call(dx=bad) == SHAPE and call(dsum=bad) == SHAPE
    assert call(dy=matrix(dtype=0)) == DTYPE and call(dx=matrix(dtype=2)) == DTYPE and call(dsum=matrix(dtype=0)) == DTYPE and call(weight_dtype=2) == DTYPE
    assert call(ws=None) == WORKSPACE and call(ws=0x100010) == WORKSPACE and call(ws_bytes=need - 1) == WORKSPACE
    assert call(dx=None, dweight=None) == OK     # nothing wanted


def test_linear_e4m3_refusals(lib):  # noqa: F811
    x, w, y = scaled(n=100, d=300), scaled(n=32, d=300, high=128), matrix(n=100, d=32, data=0x30000)
    need = lib.fnn_linear_e4m3_workspace_bytes(100, 64000, 32, 1)
    # copies of rows that are no whole runs of 16 bytes, unless there are so few that any alignment does
    assert need > 0 and lib.fnn_linear_e4m3_workspace_bytes(100, 304, 32, 1) == 0 and lib.fnn_linear_e4m3_workspace_bytes(16, 301, 32, 1) == 0
    copies = lib.fnn_linear_e4m3_workspace_bytes(100, 300, 32, 1)
    assert 132 * 304 <= copies <= 132 * 304 + 512
    for sizes in ((-1, 64, 32, 1), (100, -1, 32, 1), (100, 64, 2 ** 31, 1), (100, 64000, 32, 3)):
        assert lib.fnn_linear_e4m3_workspace_bytes(*sizes) == 0

    def call(x=x, w=w, y=y, act=0, residual=None, pre=None, ws=0x200000, ws_bytes=copies):
        return lib.fnn_linear_e4m3(x, w, None, act, residual, y, pre, ws, ws_bytes, None)

    assert call(x=None) == NULL and call(w=None) == NULL and call(y=None) == NULL
    for bad in BAD:
        good = dict(n=100, d=300) | bad
        assert call(x=scaled(**good)) == SHAPE, bad
        if "scale_row" not in bad:
            assert call(w=scaled(**(dict(n=32, d=300, high=128) | bad))) == SHAPE, bad
    assert call(w=scaled(n=31, d=300, high=128)) == SHAPE and call(w=scaled(n=32, d=301, high=128)) == SHAPE and call(x=scaled(n=101, d=300)) == SHAPE
    for bad in (matrix(n=100, d=31), matrix(n=-1), matrix(n=100, d=32, stride=31)):
        assert call(y=bad) == SHAPE and call(residual=bad) == SHAPE and call(pre=bad) == SHAPE
    assert call(residual=matrix(n=100, d=32, dtype=0)) == DTYPE and call(pre=matrix(n=100, d=32, dtype=2)) == DTYPE and call(y=matrix(n=100, d=32, dtype=3)) == DTYPE
    assert call(act=-1) == RANGE and call(act=4) == RANGE
    long = dict(x=scaled(n=100, d=64000), w=scaled(n=32, d=64000, high=128))
    assert call(ws=None) == WORKSPACE and call(ws=0x200010) == WORKSPACE and call(ws_bytes=copies - 1) == WORKSPACE
    assert call(**long) == WORKSPACE and call(**long, ws=0x100001, ws_bytes=need) == WORKSPACE and call(**long, ws=0x100000, ws_bytes=need - 1) == WORKSPACE
    assert call(x=scaled(n=0, d=300, data=0, scale=0, scale_block=4), y=matrix(n=0, d=32, data=0)) == OK


def test_linear_e4m3_backward_refusals(lib):  # noqa: F811
    need = lib.fnn_linear_e4m3_backward_workspace_bytes(100, 300, 32, 1)
    assert need >= 100 * 32 * 2 + 300 * 32 + 300 * 100
    for sizes in ((-1, 64, 32, 1), (100, -1, 32, 1), (100, 64, 2 ** 31, 1), (100, 64, 32, 5)):
        assert lib.fnn_linear_e4m3_backward_workspace_bytes(*sizes) == 0

    def call(dy=matrix(n=100, d=32), x=matrix(n=100, d=300), w=scaled(n=32, d=300, high=128), pre=matrix(n=100, d=32), act=2, dx=matrix(n=100, d=300, data=0x20000),
             dw=matrix(n=32, d=300, data=0x30000), dbias=None, ws=0x100000, ws_bytes=need):
        return lib.fnn_linear_e4m3_backward(dy, x, w, pre, act, dx, dw, dbias, ws, ws_bytes, None)

    for name in ("dy", "x", "w", "pre"):
        assert call(**{name: None}) == NULL
    for name, (n, d) in (("dy", (100, 32)), ("x", (100, 300)), ("pre", (100, 32)), ("dx", (100, 300)), ("dw", (32, 300))):
        for bad in (matrix(n=n + 1, d=d), matrix(n=n, d=d - 1), matrix(n=n, d=d, stride=d - 1)):
            assert call(**{name: bad}) == SHAPE, name
        assert call(**{name: matrix(n=n, d=d, dtype=2)}) == DTYPE, name
    # the transpose of rows with scales of their own has none for its blocks
    assert call(w=scaled(n=32, d=300)) == SHAPE and call(w=scaled(n=31, d=300, high=128)) == SHAPE and call(w=scaled(n=32, d=299, high=128)) == SHAPE
    assert call(act=4) == RANGE
    assert call(ws=None) == WORKSPACE and call(ws=0x100008) == WORKSPACE and call(ws_bytes=need - 1) == WORKSPACE
    assert call(dx=None, dw=None) == OK      # nothing wanted


class Placed(OnDevice):
    """On a device that the test names."""
    device = property(lambda self: self.place)

    def get_device(self):
        return self.place.index


def codes(n, d, tiles=False):
    return fnn.FnnScaled(given(n, d, dtype=torch.float8_e4m3fn), given(net8._blocks(n) if tiles else n, net8._blocks(d), dtype=torch.float32))


X, Y, V, STATS = given(8, 64), given(8, 32), given(64), given(8, dtype=torch.float32)
CALLS = {
    "fnn_quantize": lambda **kw: net8.fnn_quantize(X, **kw),
    "fnn_quantize_across": lambda **kw: net8.fnn_quantize(X, tiles=True, transposed=True, **kw),
    "fnn_rms_norm": lambda **kw: (lambda y, s, t, r: (y, *s, t, r))(*net8.fnn_rms_norm(X, V, X, want_scaled=True, want_rstd=True, **kw)),
    "fnn_rms_norm_backward": lambda **kw: net8.fnn_rms_norm_backward(X, X, STATS, V, X, **kw),
    "fnn_linear_e4m3": lambda **kw: net8.fnn_linear_e4m3(codes(8, 64), codes(32, 64, True), want_pre=True, **kw),
    "fnn_linear_e4m3_backward": lambda **kw: net8.fnn_linear_e4m3_backward(Y, X, codes(32, 64, True), **kw),
}


@pytest.fixture
def with_net8(allocator, monkeypatch):  # noqa: F811
    from test_net_streams import Library

    monkeypatch.setattr(net8, "load_library", Library)
    return allocator


@pytest.mark.parametrize("name", list(CALLS))
def test_memory_is_of_the_stream_that_works_in_it(with_net8, name):
    side = Stream()
    results = [t for t in CALLS[name](stream=side) if t is not None]
    assert results and all(of is side for of, _ in with_net8.taken)
    # what is returned may be a view of what was asked for
    asked = [t for _, t in with_net8.taken]
    of = {t.untyped_storage().data_ptr(): t for t in asked}
    assert all("usual" in getattr(of[t.untyped_storage().data_ptr()], "recorded", []) for t in results)
    assert with_net8.current == "usual"


@pytest.mark.parametrize("name", list(CALLS))
def test_memory_is_of_the_current_stream(with_net8, name):
    results = [t for t in CALLS[name]() if t is not None]
    assert results and all(of == "usual" for of, _ in with_net8.taken)
    assert not any(hasattr(t, "recorded") for _, t in with_net8.taken)


def test_one_device_and_the_call_made_there(with_net8, monkeypatch):
    """Tensors on two devices are refused; a call on another device than the current one is made with that device current."""
    there = []

    class Current:
        def __init__(self, device):
            there.append(device)

        def __enter__(self):
            return self

        def __exit__(self, *args):
            there.append(None)

    monkeypatch.setattr(torch.cuda, "device", Current)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    first, second = torch.device("cuda", 0), torch.device("cuda", 1)
    net8._call("f", lambda *a: 0, first, ())
    assert not there
    net8._call("f", lambda *a: 0, second, ())
    assert there == [second, None]
    other = X.clone().as_subclass(Placed)
    other.place = second
    with pytest.raises(ValueError):
        net8._call("f", lambda *a: 0, first, (None, other))


def test_what_the_binding_refuses(with_net8):
    good = codes(32, 64, True)
    for bad in (fnn.FnnScaled(good.data, codes(8, 64).scale), fnn.FnnScaled(good.data, codes(32, 200, True).scale), fnn.FnnScaled(X, good.scale),
                fnn.FnnScaled(good.data, given(1, 1)), fnn.FnnScaled(torch.zeros(32, 64), good.scale), fnn.FnnScaled(good.data.t(), codes(64, 32, True).scale)):
        with pytest.raises(ValueError):
            net8.fnn_linear_e4m3(codes(8, 64), bad)
    with pytest.raises(ValueError):
        net8.fnn_rms_norm(X, given(63))
    with pytest.raises(ValueError):
        net8.fnn_linear_e4m3(codes(8, 64), good, bias=given(32, dtype=torch.float16))
    with pytest.raises(KeyError):
        net8.fnn_linear_e4m3(codes(8, 64), good, act="tanh")
