"""fnn_rms_norm and its gradient against the formulas in 64 bits."""
import math

import pytest
import torch

import paper_2503_10017_amd as fnn
from e4m3_helpers import block_scales, spread, values
from net_helpers import DEV, F32, TYPES, assert_within, normal, rounding, strided

pytestmark = pytest.mark.gpu


def formula(x, residual, weight, eps):
    s = x.double() + (0 if residual is None else residual.double())
    rstd = ((s * s).mean(1) + eps) ** -0.5
    return s, rstd, s * rstd[:, None] * (1 if weight is None else weight.double())


def check(x, residual, weight, eps=1e-6, **kw):
    dtype, d = x.dtype, x.shape[1]
    y, scaled, total, rstd = fnn.fnn_rms_norm(x, weight, residual, eps=eps, want_scaled=True, want_rstd=True, **kw)
    s, want_rstd, want = formula(x, residual, weight, eps)
    if residual is not None:
        assert_within(total, s, F32 * s.abs() + rounding(s, dtype), "sum")
    # the sum s: one rounding of each element; the sum of squares: one rounding per addition in the longest chain, at most d of them; then the division, eps, the root and
    # the reciprocal.  Half of what the square is off by ends in rstd.
    off = (2 + (d + 4) / 2 + 4) * F32
    # rows of 1e-42 with eps 0: 1 / 1e-42 is above 3.4e38, fp32's largest, so infinity in that type; y, of size 1, is not
    assert_within(rstd, want_rstd.masked_fill(want_rstd > torch.finfo(torch.float32).max, math.inf), off * want_rstd, "rstd")
    # two products more
    near = want.abs() * (off + 3 * F32) + 2.0 ** -149
    assert_within(y, want, near + rounding(want, dtype), "y")
    scale = block_scales(want)
    assert_within(scaled.scale, scale, scale.double() * (off + 6 * F32) + 2.0 ** -149, "scale")
    each = spread(scaled.scale, *want.shape)
    # a code is at most half a step from the quotient: 2^-4 of it, or half of 2^-9 where the codes are evenly spaced
    assert_within(values(scaled), want, torch.maximum(want.abs() * 2.0 ** -4, each * 2.0 ** -10) * (1 + 2.0 ** -10) + near + want.abs() * 4 * F32, "codes")
    return y, scaled, total, rstd


SIZES = [(1, 1), (1, 1024), (3, 24), (5, 127), (4, 130), (300, 512), (17, 777), (2500, 128), (9, 1021), (7, 2048), (5, 3001), (3, 8192), (2, 16384), (6, 16383)]


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,d", SIZES)
def test_forward(n, d, kind):
    dtype = TYPES[kind]
    x, r, w = normal(1, n, d, dtype=dtype), normal(2, n, d, std=3, dtype=dtype), 1 + normal(3, d, std=0.2)
    check(x, r, w.to(dtype))
    check(x, None, w)
    check(x, r, None)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,d", [(6, 130), (40, 1000), (9, 5000)])
def test_parts_strides_and_places(n, d, kind):
    dtype = TYPES[kind]
    x, r, w = normal(1, n, d, dtype=dtype), normal(2, n, d, dtype=dtype), normal(3, d, dtype=dtype)
    y, scaled, total, rstd = fnn.fnn_rms_norm(x, w, r, want_scaled=True, want_rstd=True)
    alone = fnn.fnn_rms_norm(x, w, r, want_y=False, want_scaled=True)
    assert alone[0] is None and alone[3] is None and torch.equal(alone[1].data.float(), scaled.data.float()) and torch.equal(alone[1].scale, scaled.scale)
    only = fnn.fnn_rms_norm(x, w, r)
    assert only[1] is None and torch.equal(only[0], y) and torch.equal(only[2], total)
    for extra, offset in ((8, 0), (1, 1), (3, 4)):
        out, out_sum = (strided(torch.zeros_like(x), extra, offset) for _ in range(2))
        room = torch.full((n, d + extra), 0x55, dtype=torch.uint8, device=DEV)
        codes = fnn.FnnScaled(room.view(torch.float8_e4m3fn)[:, :d], torch.empty((n, scaled.scale.shape[1] + 2), device=DEV)[:, :scaled.scale.shape[1]])
        got = fnn.fnn_rms_norm(strided(x, extra, offset), w, strided(r, 2, 1), out=out, out_sum=out_sum, out_scaled=codes)
        assert torch.equal(got[0], y) and torch.equal(got[2], total) and torch.equal(codes.data.float(), scaled.data.float()) and torch.equal(codes.scale, scaled.scale)
        assert (room[:, d:] == 0x55).all()
        for t in (out, out_sum):
            assert torch.isnan(torch.as_strided(t, (n, extra), (d + extra, 1), t.storage_offset() + d)).all()
    for name in ("x", "r"):                       # the residual stream updated where it is; y in the other one
        a, b = x.clone(), r.clone()
        got = fnn.fnn_rms_norm(a, w, b, out_sum=a if name == "x" else b, out=b if name == "x" else a)
        assert torch.equal(got[2], total) and torch.equal(got[0], y)
    here = x.clone()
    assert torch.equal(fnn.fnn_rms_norm(here, w, out=here)[0], fnn.fnn_rms_norm(x, w)[0])


@pytest.mark.parametrize("d", [100, 1024, 4096])
def test_rows_of_any_size(d):
    """Squares that fp32 does not have, and those that vanish beside it: y is of the size of the weights all the same, unless eps says otherwise."""
    x = normal(1, 12, d)
    for i, size in enumerate((1e30, 1e37, 1e19, 1e-18, 1e-25, 1e-38, 1e-42, 0.0)):
        x[i] *= size
    for dtype in (torch.float32, torch.bfloat16):
        for eps in (1e-6, 1e-12, 1e-30, 0.0):
            t = x.to(dtype)
            check(t[:7] if eps == 0 else t, None, None, eps=eps)
    y, scaled, _, rstd = fnn.fnn_rms_norm(x[7:8], eps=0.0, want_scaled=True, want_rstd=True)
    assert torch.isnan(y).all() and torch.isnan(scaled.data.float()).all() and rstd.item() == math.inf


@pytest.mark.parametrize("d", [130, 1024, 3001])
def test_infinities_and_nan_stay_in_their_rows(d):
    x, r = normal(1, 8, d, dtype=torch.bfloat16), normal(2, 8, d, dtype=torch.bfloat16)
    want = fnn.fnn_rms_norm(x, None, r, want_scaled=True, want_rstd=True)
    x[2, d - 1], x[4, 0] = math.nan, math.inf
    y, scaled, total, rstd = fnn.fnn_rms_norm(x, None, r, want_scaled=True, want_rstd=True)
    for i in (0, 1, 3, 5, 6, 7):
        assert torch.equal(y[i], want[0][i]) and torch.equal(scaled.data[i].float(), want[1].data[i].float()) and torch.equal(total[i], want[2][i])
    assert torch.isnan(y[2]).all() and torch.isnan(rstd[2]) and torch.isnan(scaled.data[2].float()).all()
    # 1 / infinity is 0: the row's finite elements are 0, and infinity times 0 is no number
    assert rstd[4] == 0 and torch.isnan(y[4, 0]) and not y[4, 1:].any() and torch.isnan(scaled.data[4, 0].float()) and not scaled.data[4, 1:].float().any()


def check_backward(dy, s, rstd, weight, dsum, **kw):
    dtype, (n, d) = s.dtype, s.shape
    dx, dweight = fnn.fnn_rms_norm_backward(dy, s, rstd, weight, dsum, **kw)
    w = 1 if weight is None else weight.double()
    r = rstd.double()[:, None]
    h, g = s.double() * r, dy.double() * w
    along = (g * h).mean(1, keepdim=True)
    want = r * (g - h * along) + (0 if dsum is None else dsum.double())
    # h and g are a rounding off each; the mean has d products summed in fp32; then three operations
    mean_off = (d + 8) * F32 * (g * h).abs().mean(1, keepdim=True)
    slack = r * (4 * F32 * g.abs() + 6 * F32 * (h * along).abs() + h.abs() * mean_off) + 2 * F32 * want.abs()
    assert_within(dx, want, slack + rounding(want, dtype), "dx")
    want = (dy.double() * h).sum(0)
    of = dtype if weight is None else weight.dtype
    assert_within(dweight, want, (n + 6) * F32 * (dy.double() * h).abs().sum(0) + rounding(want, of), "dweight")
    return dx, dweight


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,d", SIZES + [(6151, 65)])
def test_backward(n, d, kind):
    dtype = TYPES[kind]
    dy, s, dsum, w = normal(1, n, d, dtype=dtype), normal(2, n, d, std=2, dtype=dtype), normal(3, n, d, dtype=dtype), 1 + normal(4, d, std=0.2)
    rstd = fnn.fnn_rms_norm(s, want_rstd=True)[3]
    first = check_backward(dy, s, rstd, w.to(dtype), dsum)
    again = fnn.fnn_rms_norm_backward(dy, s, rstd, w.to(dtype), dsum)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    check_backward(dy, s, rstd, w, None)
    check_backward(dy, s, rstd, None, dsum)


@pytest.mark.parametrize("d", [130, 1000, 5000])
def test_backward_parts_strides_and_places(d):
    n, dtype = 37, torch.bfloat16
    dy, s, dsum, w = (normal(i, *shape, dtype=dtype) for i, shape in enumerate(((n, d), (n, d), (n, d), (d,))))
    rstd = fnn.fnn_rms_norm(s, want_rstd=True)[3]
    dx, dweight = fnn.fnn_rms_norm_backward(dy, s, rstd, w, dsum)
    assert torch.equal(fnn.fnn_rms_norm_backward(dy, s, rstd, w, dsum, want_weight=False)[0], dx)
    assert torch.equal(fnn.fnn_rms_norm_backward(dy, s, rstd, w, dsum, want_x=False)[1], dweight)
    far = fnn.fnn_rms_norm_backward(strided(dy, 3, 1), strided(s, 8, 0), rstd, w, strided(dsum, 1, 2), out=strided(torch.zeros_like(s), 5, 1))
    assert torch.equal(far[0], dx) and torch.equal(far[1], dweight)
    for which in range(3):
        a = [t.clone() for t in (dy, s, dsum)]
        got = fnn.fnn_rms_norm_backward(a[0], a[1], rstd, w, a[2], out=a[which])
        assert torch.equal(got[0], dx) and torch.equal(got[1], dweight)


def test_backward_against_differences():
    """d/dt of sum(c * norm(x + t u; w + t v)) + sum(e * (x + t u)) at 0 by central differences of the formula in 64 bits."""
    n, d = 20, 300
    x, w, c, e, u, v = normal(1, n, d), 1 + normal(2, d, std=0.3), normal(3, n, d), normal(4, n, d), normal(5, n, d).double(), normal(6, d).double()

    def value(t):
        s = x.double() + t * u
        return (c.double() * formula(s, None, w.double() + t * v, 1e-6)[2]).sum() + (e.double() * s).sum()

    want = ((value(1e-5) - value(-1e-5)) / 2e-5).item()
    rstd = fnn.fnn_rms_norm(x, w, want_rstd=True)[3]
    dx, dweight = fnn.fnn_rms_norm_backward(c, x, rstd, w, e)
    parts = [(dx.double() * u), (dweight.double() * v)]
    assert abs(sum(p.sum().item() for p in parts) - want) <= 1e-5 * sum(p.abs().sum().item() for p in parts)


def test_empty_rows():
    x = torch.zeros((0, 64), device=DEV)
    y, scaled, total, rstd = fnn.fnn_rms_norm(x, None, x, want_scaled=True, want_rstd=True)
    assert y.shape == (0, 64) and scaled.data.shape == (0, 64) and rstd.shape == (0,)
    dx, dweight = fnn.fnn_rms_norm_backward(x, x, rstd)
    assert dx.shape == (0, 64) and dweight.shape == (64,) and not dweight.any()
