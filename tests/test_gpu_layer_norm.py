"""fnn_layer_norm and its gradient against the formulas in 64 bits."""
import math

import pytest
import torch

import paper_2503_10017_amd as fnn
from net_helpers import DEV, F32, TYPES, assert_within, normal, rounding, strided

pytestmark = pytest.mark.gpu

EPS = 1e-6
# one token, ragged row counts, every width class of both element sizes and both sides of their borders, widths that no 16 bytes divide
SHAPES = [(1, 1), (1, 1024), (3, 7), (5, 64), (4, 255), (7, 256), (2, 257), (33, 511), (6, 512), (6, 513), (65, 1021), (130, 1024), (3, 1025),
          (9, 2047), (5, 2048), (5, 2049), (3, 4096), (3, 4097), (2, 8191), (2, 8193), (3, 16384), (2100, 72)]


def of_rows(x, eps=EPS):
    x = x.double()
    var, mean = torch.var_mean(x, 1, correction=0)
    return mean, 1 / torch.sqrt(var + eps)


def forward_slack(x, y, mean, rstd, weight, bias, dtype):
    """The fp32 arithmetic before the rounding.  A sum over d terms in chunks of at most 32 and a tree has at most 64 roundings, each of
    at most the sum of magnitudes: the mean is within 66 u of mean|x|; so is a centred value, plus its own rounding, of |x - mean|; the
    variance within 70 u plus twice the mean's error over the deviation (second order), rstd half of that plus division and root; three
    more roundings to y."""
    w = torch.ones(1, device=x.device, dtype=torch.float64) if weight is None else weight.double()
    b = torch.zeros(1, device=x.device, dtype=torch.float64) if bias is None else bias.double()
    off_mean = 66 * F32 * x.double().abs().mean(1, keepdim=True)
    h = ((x.double() - mean[:, None]) * rstd[:, None]).abs()
    drift = (off_mean * rstd[:, None]) ** 2
    return w.abs() * (off_mean * rstd[:, None] + h * (drift + 50 * F32)) + 4 * F32 * b.abs() + rounding(y, dtype)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,d", SHAPES)
def test_forward(n, d, kind):
    dtype = TYPES[kind]
    x = (normal(1, n, d) * 2 + 3).to(dtype)
    weight, bias = normal(2, d, dtype=dtype), normal(3, d, dtype=dtype)
    y, mean, rstd = fnn.fnn_layer_norm(x, weight, bias, eps=EPS, want_stats=True)
    m, r = of_rows(x)
    want = (x.double() - m[:, None]) * r[:, None] * weight.double() + bias.double()
    assert_within(mean, m, 66 * F32 * x.double().abs().mean(1), "mean")
    assert_within(y, want, forward_slack(x, want, m, r, weight, bias, dtype), "y")
    off = 66 * F32 * x.double().abs().mean(1) * r
    assert_within(rstd, r, r * (off ** 2 + 48 * F32), "rstd")


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("n,d", [(3, 100), (40, 768), (5, 3000)])
def test_weights_in_fp32_or_left_out(n, d, kind):
    dtype = TYPES[kind]
    x = normal(4, n, d, dtype=dtype)
    m, r = of_rows(x)
    h = (x.double() - m[:, None]) * r[:, None]
    for weight, bias in ((normal(5, d), normal(6, d)), (None, None), (normal(5, d), None), (None, normal(6, d))):
        y, mean, rstd = fnn.fnn_layer_norm(x, weight, bias, eps=EPS)
        assert mean is None and rstd is None
        want = h * (1 if weight is None else weight.double()) + (0 if bias is None else bias.double())
        assert_within(y, want, forward_slack(x, want, m, r, weight, bias, dtype))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("d,extra,offset", [(64, 8, 0), (64, 1, 1), (777, 3, 5), (2300, 1, 3)])
def test_strides_and_alignment(d, extra, offset, kind):
    dtype = TYPES[kind]
    plain = normal(7, 19, d, dtype=dtype)
    weight, bias = normal(8, d + 1, dtype=dtype)[1:], normal(9, d, dtype=dtype)
    want = fnn.fnn_layer_norm(plain, weight, bias)[0]
    out = strided(torch.zeros_like(plain), extra + 2, offset)
    got = fnn.fnn_layer_norm(strided(plain, extra, offset), weight, bias, out=out)[0]
    assert torch.equal(got, want)
    between = torch.as_strided(out, (19, extra + 2), (d + extra + 2, 1), out.storage_offset() + d)
    assert torch.isnan(between).all()
    in_place = strided(plain, extra, offset)
    fnn.fnn_layer_norm(in_place, weight, bias, out=in_place)
    assert torch.equal(in_place, want)


def test_constant_rows_and_rows_far_from_zero():
    x = torch.full((4, 1000), 5.0, device=DEV)
    y, mean, rstd = fnn.fnn_layer_norm(x, eps=EPS, want_stats=True)
    assert torch.equal(mean, torch.full((4,), 5.0, device=DEV)) and torch.equal(y, torch.zeros_like(x))
    assert_within(rstd, torch.full((4,), 1e3, dtype=torch.float64, device=DEV), 1e3 * 1e-6)
    far = normal(10, 8, 1000) + 1e4       # the variance is formed from centred values: a mean of 10^4 deviations costs what it costs x itself
    y, m, r = fnn.fnn_layer_norm(far, eps=EPS, want_stats=True)
    want_m, want_r = of_rows(far)
    want = (far.double() - want_m[:, None]) * want_r[:, None]
    assert_within(y, want, forward_slack(far, want, want_m, want_r, None, None, torch.float32))


@pytest.mark.parametrize("d", [100, 1024, 3000])
def test_infinities_and_nan_stay_in_their_rows(d):
    x = normal(11, 9, d, dtype=torch.float16)
    want = fnn.fnn_layer_norm(x)[0]
    x[2, d - 1], x[5, 0] = math.nan, math.inf
    y = fnn.fnn_layer_norm(x)[0]
    keep = [i for i in range(9) if i not in (2, 5)]
    assert torch.equal(y[keep], want[keep])
    assert torch.isnan(y[2]).all() and torch.isnan(y[5]).all()


def back_reference(dy, x, mean, rstd, weight):
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    h, g = (x - mean) * rstd, dy * (1 if weight is None else weight.double())
    dx = rstd * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    # fp32 arithmetic: h has 2 roundings, the two means up to 66 + 4 of their magnitudes, four more steps to dx
    slack = rstd * (8 * F32 * g.abs() + 70 * F32 * g.abs().mean(1, keepdim=True) + h.abs() * 80 * F32 * (g * h).abs().mean(1, keepdim=True))
    return dx, slack, (dy * h), dy


def column_check(got, terms, dtype, what):
    """A column's sum: a workgroup's rows one after the other, then a tree over workgroups; n roundings at most, of the sum of magnitudes, and
    three in each term."""
    n = terms.shape[0]
    want = terms.sum(0)
    assert_within(got, want, (min(n, 600) + 8) * F32 * terms.abs().sum(0) + rounding(want, dtype), what)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,d", SHAPES + [(5000, 96), (2049, 333)])
def test_backward(n, d, kind):
    dtype = TYPES[kind]
    x, dy, weight = normal(1, n, d, dtype=dtype), normal(2, n, d, dtype=dtype), normal(3, d, dtype=dtype)
    m, r = (t.float() for t in of_rows(x))
    dx, dweight, dbias = fnn.fnn_layer_norm_backward(dy, x, m, r, weight)
    want, slack, dw, db = back_reference(dy, x, m, r, weight)
    assert_within(dx, want, slack + rounding(want, dtype), "dx")
    column_check(dweight, dw, dtype, "dweight")
    column_check(dbias, db, dtype, "dbias")
    again = fnn.fnn_layer_norm_backward(dy, x, m, r, weight)
    assert all(torch.equal(a, b) for a, b in zip((dx, dweight, dbias), again))


@pytest.mark.parametrize("kind", ["f32", "f16"])
def test_backward_strides_types_and_parts(kind):
    dtype, n, d = TYPES[kind], 37, 777
    x, dy, weight = normal(1, n, d, dtype=dtype), normal(2, n, d, dtype=dtype), normal(3, d)
    m, r = (t.float() for t in of_rows(x))
    whole = fnn.fnn_layer_norm_backward(dy, x, m, r, weight)
    assert whole[1].dtype == torch.float32
    far = fnn.fnn_layer_norm_backward(strided(dy, 3, 1), strided(x, 5, 3), m, r, weight, out=strided(torch.zeros_like(x), 1, 1))
    assert all(torch.equal(a, b) for a, b in zip(whole, far))
    only_x = fnn.fnn_layer_norm_backward(dy, x, m, r, weight, want_weight=False)
    assert torch.equal(only_x[0], whole[0]) and only_x[1] is None and only_x[2] is None
    only_w = fnn.fnn_layer_norm_backward(dy, x, m, r, weight, want_x=False)
    assert only_w[0] is None and torch.equal(only_w[1], whole[1]) and torch.equal(only_w[2], whole[2])
    in_place = dy.clone()
    fnn.fnn_layer_norm_backward(in_place, x, m, r, weight, out=in_place)
    assert torch.equal(in_place, whole[0])
    none = fnn.fnn_layer_norm_backward(dy, x, m, r)
    ones = fnn.fnn_layer_norm_backward(dy, x, m, r, torch.ones(d, device=DEV, dtype=dtype))
    assert all(torch.equal(a, b) for a, b in zip(none, ones))


def test_gradient_against_differences():
    """d/dt of sum(c * layer_norm(x + t u)) at 0, by central differences of the formula in 64 bits, is sum(dx * u) with dy = c; the same for the
    weight and the bias.  The difference's own error at t = 1e-5 is below 1e-8; fp32 sums leave 1e-4 of the magnitudes with margin."""
    n, d = 6, 200
    x, c, weight, bias = normal(1, n, d), normal(2, n, d), normal(3, d), normal(4, d)
    ux, uw, ub = normal(5, n, d).double(), normal(6, d).double(), normal(7, d).double()

    def value(t):
        xs = x.double() + t * ux
        m, r = of_rows(xs)
        return (c.double() * ((xs - m[:, None]) * r[:, None] * (weight.double() + t * uw) + bias.double() + t * ub)).sum()

    slope = ((value(1e-5) - value(-1e-5)) / 2e-5).item()
    m, r = (t.float() for t in of_rows(x))
    dx, dweight, dbias = fnn.fnn_layer_norm_backward(c, x, m, r, weight)
    parts = [(dx.double() * ux), (dweight.double() * uw), (dbias.double() * ub)]
    assert abs(sum(p.sum().item() for p in parts) - slope) <= 1e-4 * sum(p.abs().sum().item() for p in parts) / math.sqrt(n * d)


def test_no_rows():
    x = torch.empty((0, 64), device=DEV)
    y, mean, rstd = fnn.fnn_layer_norm(x, want_stats=True)
    assert y.shape == (0, 64) and mean.shape == (0,)
    dx, dweight, dbias = fnn.fnn_layer_norm_backward(x, x, mean, rstd)
    assert dx.shape == (0, 64) and not dweight.any() and not dbias.any()


def test_on_another_stream_and_in_a_graph():
    x, weight, bias, dy = normal(1, 300, 768, dtype=torch.bfloat16), normal(2, 768), normal(3, 768), normal(4, 300, 768, dtype=torch.bfloat16)
    out, dx = torch.empty_like(x), torch.empty_like(x)
    ws = torch.empty(fnn.fnn_layer_norm_backward_workspace_bytes(300, 768), dtype=torch.uint8, device=DEV)

    def call(stream=None):
        y, mean, rstd = fnn.fnn_layer_norm(x, weight, bias, out=out, want_stats=True, stream=stream)
        return (y,) + fnn.fnn_layer_norm_backward(dy, x, mean, rstd, weight, out=dx, workspace=ws, stream=stream)

    want = [t.clone() for t in call()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out.zero_(), dx.zero_()
    torch.cuda.synchronize()
    got = call(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for seed in (1, 21, 22, 1):
        x.copy_(normal(seed, 300, 768, dtype=torch.bfloat16))
        for t in held:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        assert all(torch.equal(a, b) for a, b in zip(got, call()))
        torch.cuda.synchronize()
