"""fnn_linear_e4m3 and its gradient against the formulas in 64 bits."""
import math

import pytest
import torch

import paper_2503_10017_amd as fnn
from e4m3_helpers import nearest_e4m3, placed, quantized, scaled_of, spread, values
from net_helpers import DEV, F32, TYPES, assert_within, normal, rounding, strided
from test_gpu_linear import ACTS, act_slack, slope

pytestmark = pytest.mark.gpu


def product_slack(xv, wv, dtype):
    """How far the products of two matrices (values in 64 bits) may be off.  fp32 results: a rounding per addition of exact products, the scales' product and one by it.  16-bit results: of
    eight neighbouring products each is cut at 2^-13 of the largest's power of two; the largest itself has 8 digits and loses none."""
    k = xv.shape[1]
    xa, wa = xv.abs(), wv.abs()
    slack = (k + 8) * F32 * (xa @ wa.t())
    if dtype != torch.float32:
        for first in range(0, k, 8):
            top = torch.zeros_like(slack)
            for i in range(first, min(k, first + 8)):
                top = torch.maximum(top, torch.outer(xa[:, i], wa[:, i]))
            slack += 7 * 2.0 ** -13 * top
    return slack


def check_forward(x, w, bias, residual, act, dtype, **kw):
    y, pre = fnn.fnn_linear_e4m3(x, w, bias, residual, act=act, dtype=dtype, **kw)
    xv, wv = values(x), values(w)
    p = xv @ wv.t() + (0 if bias is None else bias.double())
    off = product_slack(xv, wv, dtype) + (0 if bias is None else 2 * F32 * (bias.double().abs() + p.abs()))
    want = ACTS[act](p) + (0 if residual is None else residual.double())
    # every activation's slope is below 1.13
    assert_within(y, want, 1.13 * off + act_slack(p, act, dtype) + 2 * F32 * want.abs() + rounding(want, dtype), "y")
    if pre is not None:
        assert_within(pre, p, off + rounding(p, dtype), "pre")
    return y


SIZES = [(1, 1, 1), (1, 1024, 512), (2, 777, 33), (16, 256, 100), (17, 96, 16), (33, 520, 200), (64, 1024, 129), (64, 2049, 7), (65, 64, 64), (65, 8, 8),
         (100, 4000, 96), (129, 100, 200), (300, 320, 257), (200, 1, 300), (500, 72, 401), (260, 1040, 640), (531, 777, 401)]


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_forward(m, k, n, kind):
    dtype = TYPES[kind]
    x, w = scaled_of(normal(1, m, k), extra=-k % 16), scaled_of(normal(2, n, k, std=1 / math.sqrt(k)), tiles=True, extra=-k % 16)
    check_forward(x, w, normal(3, n, dtype=dtype), normal(4, m, n, dtype=dtype), "gelu", dtype, want_pre=True)
    check_forward(x, w, None, None, "none", dtype)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("m,k,n", [(5, 200, 300), (2304, 130, 2200), (700, 1050, 300)])
@pytest.mark.parametrize("act", list(ACTS))
def test_activations_and_scales_of_rows(m, k, n, act, kind):
    """Scales for each row of w, and for tiles of x, which another program may have."""
    dtype = TYPES[kind]
    x, w = scaled_of(normal(1, m, k, std=3), tiles=True, extra=-k % 16), scaled_of(normal(2, n, k, std=1 / math.sqrt(k)), extra=-k % 16)
    check_forward(x, w, normal(3, n, dtype=dtype), normal(4, m, n, dtype=dtype), act, dtype, want_pre=True)


@pytest.mark.parametrize("kind", ["f32", "f16"])
@pytest.mark.parametrize("tiles", [False, True])
@pytest.mark.parametrize("m,k,n", [(9, 130, 60), (200, 136, 150), (2300, 264, 2100), (130, 3000, 70)])
def test_strides_and_alignment(m, k, n, tiles, kind):
    dtype = TYPES[kind]
    (x, sx), (w, sw) = quantized(normal(1, m, k)), quantized(normal(2, n, k), tiles)
    r, bias = normal(4, m, n, dtype=dtype), normal(3, n + 1, dtype=dtype)
    want = fnn.fnn_linear_e4m3(placed(x, sx), placed(w, sw), bias[1:].clone(), r, act="silu", dtype=dtype)[0]
    for extra, offset, gap, by_rows in ((-k % 16, 0, 0, True), (-k % 16 + 16, 16, 3, False), (1, 1, 5, True), (3, 7, 0, False)):
        out = strided(torch.zeros_like(r), 3, 1)
        got = fnn.fnn_linear_e4m3(placed(x, sx, extra, offset, gap, by_rows), placed(w, sw, extra, offset, gap, by_rows), bias[1:], strided(r, 2, 1), act="silu", out=out)[0]
        assert torch.equal(got, want)
        assert torch.isnan(torch.as_strided(out, (m, 3), (n + 3, 1), out.storage_offset() + n)).all()
    in_place = r.clone()
    fnn.fnn_linear_e4m3(placed(x, sx), placed(w, sw), bias[1:], in_place, act="silu", out=in_place)
    assert torch.equal(in_place, want)


def test_values_of_few_digits_come_out_exact():
    """Products of small whole numbers, and their sums and scales that are powers of two: every class of sizes has to give them to the bit."""
    for m, k, n in ((1, 512, 64), (40, 1000, 70), (130, 777, 130), (400, 4096, 300), (2304, 192, 2304), (2300, 200, 2311)):
        gen = torch.Generator().manual_seed(m)
        for tiles in (False, True):
            (x, sx), (w, sw) = ((torch.randint(-2, 3, (r, k), generator=gen).double().to(DEV),
                                 2.0 ** torch.randint(-2, 3, (-(-r // 128) if t else r, -(-k // 128)), generator=gen).float().to(DEV)) for r, t in ((m, False), (n, tiles)))
            want = (x * spread(sx, m, k)) @ (w * spread(sw, n, k)).t()
            for kind in ("f32", "f16", "bf16"):
                y = fnn.fnn_linear_e4m3(placed(x, sx, extra=-k % 16), placed(w, sw, extra=-k % 16), dtype=TYPES[kind])[0]
                assert torch.equal(y, want.to(TYPES[kind])), (m, k, n, kind)


@pytest.mark.parametrize("m,k,n", [(3, 100, 40), (200, 72, 136), (2304, 136, 2304), (150, 1300, 130)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_nan_stays_in_its_row_and_column(m, k, n, kind):
    x, w = normal(1, m, k), normal(2, n, k)
    (xd, sx), (wd, sw) = quantized(x), quantized(w, True)
    want = fnn.fnn_linear_e4m3(placed(xd, sx), placed(wd, sw), dtype=TYPES[kind])[0]
    xd[m - 2, k - 1], wd[n - 1, 0] = math.nan, math.nan
    sx = sx.clone()
    sx[0, -1] = math.inf
    y = fnn.fnn_linear_e4m3(placed(xd, sx), placed(wd, sw), dtype=TYPES[kind])[0]
    assert torch.equal(y[1:m - 2, :n - 1], want[1:m - 2, :n - 1])
    assert torch.isnan(y[m - 2]).all() and torch.isnan(y[:, n - 1]).all() and not torch.isfinite(y[0]).any()


def check_backward(dy, x, w, pre, act, **kw):
    dtype = x.dtype
    dx, dw, dbias = fnn.fnn_linear_e4m3_backward(dy, x, w, pre, act=act, **kw)
    q = dy.double() * (1 if pre is None else slope(pre.double(), act))
    q_off = torch.zeros_like(q)
    if act in ("gelu", "silu"):
        q_off = dy.double().abs() * (4e-6 if dtype != torch.float32 else 16 * F32) + 2 * F32 * q.abs()

    def in_8_bits(v, off):
        """Values by the definition, and how far the call's may be from them: where q is a little off, a code next to a border may be the next one."""
        data, scale = quantized(v)
        each = spread(scale, *v.shape)
        if not off.any():
            return data * each, torch.zeros_like(data)
        quotient, near = v / each, off / each + v.abs() / each * 4 * F32 + 4 * F32
        near = near + quotient.abs() * (off.abs().amax() / v.abs().amax())        # the scale is of a value that is off, too
        low, high = nearest_e4m3((quotient - near).clamp(-448, 448)), nearest_e4m3((quotient + near).clamp(-448, 448))
        return data * each, torch.maximum((data - low).abs(), (high - data).abs()) * each + data.abs() * each * (off.abs().amax() / v.abs().amax())

    (q1, off1), (q2, off2), (x2, _) = in_8_bits(q, q_off), in_8_bits(q.t().contiguous(), q_off.t().contiguous()), in_8_bits(x.double().t().contiguous(), torch.zeros(1, device=DEV))
    wv = values(w)
    want = q1 @ wv
    assert_within(dx, want, off1 @ wv.abs() + product_slack(q1, wv.t().contiguous(), dtype) + rounding(want, dtype), "dx")
    want = q2 @ x2.t()
    assert_within(dw, want, off2 @ x2.abs().t() + product_slack(q2, x2, dtype) + rounding(want, dtype), "dw")
    want = q.sum(0)
    assert_within(dbias, want, q_off.sum(0) + (len(q) + 4) * F32 * q.abs().sum(0) + rounding(want, dtype), "dbias")
    return dx, dw, dbias


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_backward(m, k, n, kind):
    dtype = TYPES[kind]
    x, dy, pre = normal(1, m, k, dtype=dtype), normal(3, m, n, dtype=dtype), normal(4, m, n, dtype=dtype)
    w = scaled_of(normal(2, n, k, std=1 / math.sqrt(k)), tiles=True)
    first = check_backward(dy, x, w, None, "none")
    again = fnn.fnn_linear_e4m3_backward(dy, x, w)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    check_backward(dy, x, w, pre, "relu")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("m,k,n", [(70, 200, 136), (1100, 264, 700)])
def test_backward_activations(m, k, n, act, kind):
    dtype = TYPES[kind]
    x, dy, pre = (normal(i, *s, dtype=dtype) for i, s in enumerate(((m, k), (m, n), (m, n))))
    check_backward(dy, x, scaled_of(normal(5, n, k), tiles=True), pre, act)


@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("m,k,n", [(70, 130, 66), (2304, 260, 2100)])
def test_backward_strides_and_parts(m, k, n, act):
    x, dy, pre = (normal(i, *s, dtype=torch.float16) for i, s in enumerate(((m, k), (m, n), (m, n))))
    wd, sw = quantized(normal(5, n, k), True)
    w = placed(wd, sw)
    whole = fnn.fnn_linear_e4m3_backward(dy, x, w, pre, act=act)
    far = fnn.fnn_linear_e4m3_backward(strided(dy, 3, 1), strided(x, 5, 2), placed(wd, sw, 3, 1, 2, True), strided(pre, 1, 1), act=act, out=strided(torch.zeros_like(x), 1, 1))
    assert all(torch.equal(a, b) for a, b in zip(whole, far))
    for i in range(3):
        part = fnn.fnn_linear_e4m3_backward(dy, x, w, pre, act=act, want_x=i == 0, want_w=i == 1, want_bias=i == 2)
        assert torch.equal(part[i], whole[i]) and all(part[j] is None for j in range(3) if j != i)


def test_empty_sizes():
    def zeros(*s):
        return torch.zeros(s, device=DEV, dtype=torch.float16)

    def codes(*s, tiles=False):
        return fnn.fnn_quantize(zeros(*s), tiles=tiles)

    bias = normal(1, 5, dtype=torch.float16)
    for rows in (3, 100):
        y, _ = fnn.fnn_linear_e4m3(codes(rows, 0), codes(5, 0, tiles=True), bias, act="relu", dtype=torch.float16)
        assert torch.equal(y, bias.clamp(min=0).expand(rows, 5))
    assert fnn.fnn_linear_e4m3(codes(0, 4), codes(5, 4, tiles=True), bias, dtype=torch.float16)[0].shape == (0, 5)
    assert fnn.fnn_linear_e4m3(codes(3, 4), codes(0, 4, tiles=True))[0].shape == (3, 0)
    dx, dw, db = fnn.fnn_linear_e4m3_backward(zeros(0, 5), zeros(0, 4), codes(5, 4, tiles=True), zeros(0, 5), act="gelu")
    assert dx.shape == (0, 4) and dw.shape == (5, 4) and not dw.any() and not db.any()
    dx, dw, db = fnn.fnn_linear_e4m3_backward(zeros(3, 0), zeros(3, 4), codes(0, 4, tiles=True))
    assert dx.shape == (3, 4) and not dx.any() and dw.shape == (0, 4)


def test_offsets_past_32_bits():
    """Rows of codes that lie 2^31 bytes and more apart from the first."""
    rows, d, stride = 140, 64, 33 << 20
    buf = torch.empty(rows * stride, dtype=torch.uint8, device=DEV)
    plain = fnn.fnn_quantize(normal(1, rows, d))
    codes = buf.view(torch.float8_e4m3fn).view(rows, stride)[:, :d]
    buf.view(rows, stride)[:, :d] = plain.data.view(torch.uint8)
    w = fnn.fnn_quantize(normal(2, 96, d), tiles=True)
    assert torch.equal(fnn.fnn_linear_e4m3(fnn.FnnScaled(codes, plain.scale), w)[0], fnn.fnn_linear_e4m3(plain, w)[0])
    assert torch.equal(fnn.fnn_linear_e4m3(w, fnn.FnnScaled(codes, plain.scale))[0], fnn.fnn_linear_e4m3(w, plain)[0])


@pytest.mark.parametrize("m", [9, 100, 140])
def test_scales_far_apart(m):
    """Scales that lie 2^31 bytes and more apart: their offsets do not fit 32 bits."""
    k, n, apart = 300, 130, 9 << 20
    x, w = fnn.fnn_quantize(normal(1, m, k)), fnn.fnn_quantize(normal(2, n, k))
    want = fnn.fnn_linear_e4m3(x, w)[0]
    buf = torch.zeros(max(m, n) * apart, device=DEV)             # 5 GB

    def far(s):
        scale = buf.view(-1, apart)[:s.scale.shape[0], :s.scale.shape[1]]
        scale.copy_(s.scale)
        return fnn.FnnScaled(s.data, scale)

    assert torch.equal(fnn.fnn_linear_e4m3(far(x), w)[0], want)
    assert torch.equal(fnn.fnn_linear_e4m3(x, far(w))[0], want)
    by_blocks = torch.zeros(3 * (200 << 20), device=DEV).view(3, -1)[:, :m].t()     # or the blocks' do
    by_blocks.copy_(x.scale)
    assert torch.equal(fnn.fnn_linear_e4m3(fnn.FnnScaled(x.data, by_blocks), w)[0], want)


@pytest.mark.parametrize("m,k,n", [(8, 512, 768), (300, 2048, 200), (2304, 256, 2304)])
def test_on_another_stream_and_in_a_graph(m, k, n):
    """The norm, the layer on its codes and both gradients, as a training step takes them, captured and replayed."""
    bf = torch.bfloat16
    x, r, nw, b, dy = normal(1, m, k, dtype=bf), normal(2, m, k, dtype=bf), normal(3, k, dtype=bf), normal(4, n, dtype=bf), normal(5, m, n, dtype=bf)
    w = fnn.fnn_quantize(normal(6, n, k, std=1 / math.sqrt(k)), tiles=True)

    def call(stream=None):
        y, scaled, total, rstd = fnn.fnn_rms_norm(x, nw, r, want_scaled=True, want_rstd=True, stream=stream)
        out, pre = fnn.fnn_linear_e4m3(scaled, w, b, act="gelu", want_pre=True, stream=stream)
        dn, dw, db = fnn.fnn_linear_e4m3_backward(dy, y, w, pre, act="gelu", stream=stream)
        dx, dnw = fnn.fnn_rms_norm_backward(dn, total, rstd, nw, r, stream=stream)
        return out, pre, total, dn, dw, db, dx, dnw

    want = [t.clone() for t in call()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = call(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for seed in (1, 21, 22, 1):
        x.copy_(normal(seed, m, k, dtype=bf))
        for t in held:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        assert all(torch.equal(a, b) for a, b in zip(got, call()))
        torch.cuda.synchronize()
