"""fnn_linear and its gradient against the formulas in 64 bits."""
import math

import pytest
import torch

import paper_2503_10017_amd as fnn
from net_helpers import DEV, F32, TYPES, assert_within, normal, rounding, strided

pytestmark = pytest.mark.gpu

ACTS = {
    "none": lambda p: p,
    "relu": lambda p: p.clamp(min=0),
    "gelu": lambda p: p * torch.special.ndtr(p),
    "silu": lambda p: p * torch.sigmoid(p),
}


def slope(p, act):
    if act == "none":
        return torch.ones_like(p)
    if act == "relu":
        return (p > 0).to(p.dtype)
    if act == "gelu":
        return torch.special.ndtr(p) + p * torch.exp(-p * p / 2) / math.sqrt(2 * math.pi)
    s = torch.sigmoid(p)
    return s * (1 + p * (1 - s))


def sum_slack(magnitudes, terms):
    """fp32 sums of `terms` products (exact in 16-bit types, rounded in fp32) in any order: a rounding per addition, each of at most the sum of
    magnitudes; the instructions may add several products before they round, which is no worse."""
    return (terms + 4) * F32 * magnitudes


def act_slack(p, act, dtype):
    """What the activation adds: in fp32 a few roundings of the function and its result; in 16-bit types 1.5e-7 in erf, which
    the formula's p carries, and the hardware's exp and reciprocal (1e-6 relative)."""
    if act in ("none", "relu"):
        return 0
    return p.abs() * (4e-7 + 2e-6) if dtype != torch.float32 else p.abs() * 8 * F32


def check_forward(x, w, bias, residual, act, **kw):
    dtype = x.dtype
    y, pre = fnn.fnn_linear(x, w, bias, residual, act=act, **kw)
    p = x.double() @ w.double().t() + (0 if bias is None else bias.double())
    mag = x.double().abs() @ w.double().abs().t() + (0 if bias is None else bias.double().abs())
    off = sum_slack(mag, x.shape[1])
    want = ACTS[act](p) + (0 if residual is None else residual.double())
    # every activation's slope is below 1.13
    assert_within(y, want, 1.13 * off + act_slack(p, act, dtype) + 2 * F32 * want.abs() + rounding(want, dtype), "y")
    if pre is not None:
        assert_within(pre, p, off + rounding(p, dtype), "pre")
    return y


# one token and few, both sides of every class of sizes, odd everything, a long and an empty sum
SIZES = [(1, 1, 1), (1, 1024, 4096), (2, 777, 33), (15, 64, 48), (16, 256, 100), (17, 96, 16), (33, 520, 1000), (64, 1024, 129), (64, 4097, 7),
         (65, 64, 64), (65, 8, 8), (100, 8000, 96), (129, 100, 200), (300, 320, 257), (500, 1, 500), (1000, 72, 1001), (511, 2048, 640), (1531, 777, 1001)]


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_forward(m, k, n, kind):
    dtype = TYPES[kind]
    x, w = normal(1, m, k, dtype=dtype), normal(2, n, k, std=1 / math.sqrt(k), dtype=dtype)
    check_forward(x, w, normal(3, n, dtype=dtype), normal(4, m, n, dtype=dtype), "gelu", want_pre=True)
    check_forward(x, w, None, None, "none")


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,k,n", [(5, 200, 300), (2304, 320, 2200), (700, 2050, 300)])
@pytest.mark.parametrize("act", list(ACTS))
def test_activations(m, k, n, act, kind):
    dtype = TYPES[kind]
    x, w = normal(1, m, k, std=3, dtype=dtype), normal(2, n, k, std=1 / math.sqrt(k), dtype=dtype)
    check_forward(x, w, normal(3, n, dtype=dtype), None, act, want_pre=True)
    check_forward(x, w, None, normal(4, m, n, dtype=dtype), act)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("m,k,n", [(9, 130, 60), (200, 136, 150), (2300, 264, 2100), (130, 3000, 70)])
def test_strides_and_alignment(m, k, n, kind):
    dtype = TYPES[kind]
    x, w, r = normal(1, m, k, dtype=dtype), normal(2, n, k, dtype=dtype), normal(4, m, n, dtype=dtype)
    bias = normal(3, n + 1, dtype=dtype)
    want = fnn.fnn_linear(x, w, bias[1:].clone(), r, act="silu")[0]
    for extra, offset in ((8, 0), (1, 1), (3, 4)):
        out = strided(torch.zeros_like(r), extra, offset)
        got = fnn.fnn_linear(strided(x, extra, offset), strided(w, extra, offset + 1), bias[1:], strided(r, 2, 1), act="silu", out=out)[0]
        assert torch.equal(got, want)
        between = torch.as_strided(out, (m, extra), (n + extra, 1), out.storage_offset() + n)
        assert torch.isnan(between).all()
    in_place = r.clone()
    fnn.fnn_linear(x, w, bias[1:], in_place, act="silu", out=in_place)
    assert torch.equal(in_place, want)


def test_values_of_few_digits_come_out_exact():
    """Sums of small whole numbers are exact in fp32 whatever the order: every class of sizes has to give them to the bit."""
    for m, k, n in ((1, 512, 64), (40, 1000, 70), (130, 777, 130), (400, 4096, 300), (2304, 192, 2304), (2300, 200, 2311)):
        for kind in ("f32", "f16", "bf16"):
            gen = torch.Generator().manual_seed(m)
            x, w = (torch.randint(-2, 3, (r, k), generator=gen).to(TYPES[kind]).to(DEV) for r in (m, n))
            y = fnn.fnn_linear(x, w)[0]
            assert torch.equal(y, (x.double() @ w.double().t()).to(TYPES[kind])), (m, k, n, kind)


@pytest.mark.parametrize("m,k,n", [(3, 100, 40), (200, 72, 136), (2304, 136, 2304), (150, 1300, 130)])
def test_infinities_and_nan_stay_in_their_rows_and_columns(m, k, n):
    x, w = normal(1, m, k, dtype=torch.bfloat16), normal(2, n, k, dtype=torch.bfloat16)
    want = fnn.fnn_linear(x, w, act="gelu")[0]
    x[m - 2, k - 1], x[m - 1, 0], w[n - 1, k - 1] = math.nan, math.inf, math.nan
    y = fnn.fnn_linear(x, w, act="gelu")[0]
    assert torch.equal(y[:m - 2, :n - 1], want[:m - 2, :n - 1])
    assert torch.isnan(y[m - 2]).all() and torch.isnan(y[:, n - 1]).all() and not torch.isfinite(y[m - 1, :n - 1][w[:n - 1, 0] > 0]).any()


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("kind", ["f32", "f16"])
def test_activations_at_their_ends(act, kind):
    dtype = TYPES[kind]
    p = torch.tensor([0.0, -0.0, 1e-7, -1e-7, 3.0, -3.0, 6.0, -6.0, 12.0, -12.0, 60.0, -60.0, 6e4, -6e4, math.inf, math.nan], dtype=dtype, device=DEV)
    one = torch.ones((1, 1), dtype=dtype, device=DEV)
    y = fnn.fnn_linear(p[:, None].contiguous(), one, act=act)[0][:, 0]
    want = ACTS[act](p.double())
    assert torch.isnan(y[-1]) and y[-2] == math.inf
    assert_within(y[:-2], want[:-2], act_slack(p[:-2].double().clamp(-60, 60), act, dtype) + rounding(want[:-2], dtype), act)
    q = fnn.fnn_linear_backward(torch.ones((14, 1), dtype=dtype, device=DEV), p[:14, None].contiguous(), one, p[:14, None].contiguous(), act=act)[0][:, 0]
    want = slope(p[:14].double(), act)
    assert_within(q, want, (0 if act == "relu" else 4e-6) + rounding(want, dtype), act)


def check_backward(dy, x, w, pre, act, **kw):
    dtype = x.dtype
    dx, dw, dbias = fnn.fnn_linear_backward(dy, x, w, pre, act=act, **kw)
    q = dy.double() * (1 if pre is None else slope(pre.double(), act))
    # q itself: the slope's error (below 4e-6), then one rounding to the type that is multiplied (an activation's only)
    q_off = torch.zeros_like(q)
    if act in ("gelu", "silu"):
        q_off = dy.double().abs() * (4e-6 if dtype != torch.float32 else 16 * F32) + 2 * F32 * q.abs()
    q_round = q_off + (0 if act in ("none", "relu") or dtype == torch.float32 else rounding(q, dtype))
    xa, wa, qa = x.double().abs(), w.double().abs(), q.abs()
    want = q @ w.double()
    assert_within(dx, want, q_round @ wa + sum_slack(qa @ wa, w.shape[0]) + rounding(want, dtype), "dx")
    want = q.t() @ x.double()
    assert_within(dw, want, q_round.t() @ xa + sum_slack(qa.t() @ xa, x.shape[0]) + rounding(want, dtype), "dw")
    want = q.sum(0)
    assert_within(dbias, want, q_off.sum(0) + sum_slack(qa.sum(0), x.shape[0]) + rounding(want, dtype), "dbias")
    return dx, dw, dbias


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,k,n", SIZES + [(2304, 320, 2200), (5000, 40, 56)])
def test_backward(m, k, n, kind):
    dtype = TYPES[kind]
    x, w, dy, pre = normal(1, m, k, dtype=dtype), normal(2, n, k, std=1 / math.sqrt(k), dtype=dtype), normal(3, m, n, dtype=dtype), normal(4, m, n, dtype=dtype)
    check_backward(dy, x, w, pre, "gelu")
    first = check_backward(dy, x, w, None, "none")
    again = fnn.fnn_linear_backward(dy, x, w)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("act", ["relu", "silu"])
@pytest.mark.parametrize("m,k,n", [(70, 200, 136), (2304, 264, 2200)])
def test_backward_activations(m, k, n, act):
    x, w, dy, pre = (normal(i, *s, dtype=torch.bfloat16) for i, s in enumerate(((m, k), (n, k), (m, n), (m, n))))
    check_backward(dy, x, w, pre, act)


@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("m,k,n", [(70, 130, 66), (2304, 260, 2100)])
def test_backward_strides_and_parts(m, k, n, act):
    x, w, dy, pre = (normal(i, *s, dtype=torch.float16) for i, s in enumerate(((m, k), (n, k), (m, n), (m, n))))
    whole = fnn.fnn_linear_backward(dy, x, w, pre, act=act)
    far = fnn.fnn_linear_backward(strided(dy, 3, 1), strided(x, 5, 2), strided(w, 6, 0), strided(pre, 1, 1), act=act, out=strided(torch.zeros_like(x), 1, 1))
    assert all(torch.equal(a, b) for a, b in zip(whole, far))
    for i in range(3):
        part = fnn.fnn_linear_backward(dy, x, w, pre, act=act, want_x=i == 0, want_w=i == 1, want_bias=i == 2)
        assert torch.equal(part[i], whole[i]) and all(part[j] is None for j in range(3) if j != i)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,k,n", [(2310, 2049, 2601), (2600, 2302, 2304), (900, 901, 903), (901, 904, 907), (800, 905, 904)])
def test_large_products_of_odd_rows(m, k, n, kind):
    """Operands whose rows do not end on 16-byte boundaries are copied where the product is large; zeros behind a copy's rows must not be
    what NaN behind the caller's rows would be."""
    dtype = TYPES[kind]
    x, w, dy = (strided(normal(i, *s, std=t, dtype=dtype), 3, 1) for i, s, t in ((1, (m, k), 1), (2, (n, k), 1 / math.sqrt(k)), (3, (m, n), 1)))
    check_forward(x, w, normal(4, n, dtype=dtype), None, "relu")
    check_backward(dy, x, w, None, "none")
    check_backward(dy, x, w, normal(5, m, n, dtype=dtype), "silu")


def test_gradient_against_differences():
    """d/dt of sum(c * linear(x + t u, w + t v, b + t z)) at 0 by central differences of the formula in 64 bits.  pre is the exact one
    rounded to fp32."""
    m, k, n = 90, 70, 80
    x, w, b, c = normal(1, m, k), normal(2, n, k), normal(3, n), normal(4, m, n)
    u, v, z = normal(5, m, k).double(), normal(6, n, k).double(), normal(7, n).double()
    for act in ("gelu", "silu", "none"):
        def value(t):
            return (c.double() * ACTS[act]((x.double() + t * u) @ (w.double() + t * v).t() + b.double() + t * z)).sum()

        want = ((value(1e-5) - value(-1e-5)) / 2e-5).item()
        pre = (x.double() @ w.double().t() + b.double()).float()
        parts = [(g.double() * d) for g, d in zip(fnn.fnn_linear_backward(c, x, w, pre, act=act), (u, v, z))]
        assert abs(sum(p.sum().item() for p in parts) - want) <= 1e-5 * sum(p.abs().sum().item() for p in parts)


def test_empty_sizes():
    def zeros(*s):
        return torch.zeros(s, device=DEV, dtype=torch.float16)

    bias = normal(1, 5, dtype=torch.float16)
    y, _ = fnn.fnn_linear(zeros(3, 0), zeros(5, 0), bias, act="relu")
    assert torch.equal(y, bias.clamp(min=0).expand(3, 5))
    y, _ = fnn.fnn_linear(zeros(100, 0), zeros(5, 0), bias)
    assert torch.equal(y, bias.expand(100, 5))
    assert fnn.fnn_linear(zeros(0, 4), zeros(5, 4), bias)[0].shape == (0, 5)
    assert fnn.fnn_linear(zeros(3, 4), zeros(0, 4))[0].shape == (3, 0)
    dx, dw, db = fnn.fnn_linear_backward(zeros(0, 5), zeros(0, 4), zeros(5, 4), zeros(0, 5), act="gelu")
    assert dx.shape == (0, 4) and dw.shape == (5, 4) and not dw.any() and not db.any()
    dx, dw, db = fnn.fnn_linear_backward(zeros(3, 0), zeros(3, 4), zeros(0, 4))
    assert dx.shape == (3, 4) and not dx.any() and dw.shape == (0, 4)


def test_offsets_past_32_bits():
    """A view whose rows lie 2^31 bytes and more apart from the first: the last rows' products are those of a compact copy."""
    rows, d, stride = 70, 64, 33 << 20          # 70 rows of 66 MB: 4.6 GB
    buf = torch.empty(rows * stride, dtype=torch.bfloat16, device=DEV)
    x = buf.view(rows, stride)[:, :d]
    x.copy_(normal(1, rows, d, dtype=torch.bfloat16))
    w = normal(2, 96, d, dtype=torch.bfloat16)
    plain = x.contiguous()
    assert torch.equal(fnn.fnn_linear(x, w)[0], fnn.fnn_linear(plain, w)[0])
    dy = normal(3, rows, 96, dtype=torch.bfloat16)
    got, want = fnn.fnn_linear_backward(dy, x, w), fnn.fnn_linear_backward(dy, plain, w)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(fnn.fnn_layer_norm(x)[0], fnn.fnn_layer_norm(plain)[0])


@pytest.mark.parametrize("m,k,n", [(8, 512, 768), (300, 2048, 200), (2304, 256, 2304)])
def test_on_another_stream_and_in_a_graph(m, k, n):
    bf = torch.bfloat16
    x, w, b, dy = normal(1, m, k, dtype=bf), normal(2, n, k, dtype=bf), normal(3, n, dtype=bf), normal(4, m, n, dtype=bf)
    forward = torch.empty(max(256, fnn.fnn_linear_workspace_bytes(m, k, n, bf)), dtype=torch.uint8, device=DEV)
    back = torch.empty(fnn.fnn_linear_backward_workspace_bytes(m, k, n, bf, "gelu"), dtype=torch.uint8, device=DEV)

    def call(stream=None):
        y, pre = fnn.fnn_linear(x, w, b, act="gelu", want_pre=True, workspace=forward, stream=stream)
        return (y, pre) + fnn.fnn_linear_backward(dy, x, w, pre, act="gelu", workspace=back, stream=stream)

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
