"""The gradient of a layer in 8 bits where its products take the tiles of large sizes, asserted through the trace; GELU and SiLU in fp16; and what is not finite."""
import math

import pytest
import torch

import paper_2503_10017_amd as fnn
from e4m3_helpers import placed, scaled_of, spread
from net_helpers import DEV, TYPES, normal
from test_gpu_linear_e4m3 import check_backward
from test_gpu_linear_e4m3_variants import launches

pytestmark = pytest.mark.gpu

FEW, SMALL, BOTH, MIDDLE, LARGE = 16, 64, 65, 128, 256

# rows, inner, outer; the tiles of dx and of dw, and whether dw is cut into shares: in 16-bit types, and in fp32, which has no large tile
CASES = [((3000, 2100, 2300), (MIDDLE, MIDDLE, False), (MIDDLE, MIDDLE, False)), ((5000, 3100, 3000), (MIDDLE, LARGE, False), (MIDDLE, MIDDLE, False)),
         ((9000, 1300, 1200), (LARGE, MIDDLE, True), (MIDDLE, MIDDLE, True)), ((6000, 1700, 2900), (LARGE, LARGE, True), (MIDDLE, MIDDLE, True))]


def ways(kind, halves, floats):
    """The launches of a gradient: its operands, the columns' sums where they are not in the join of dw's shares, dx, dw and that join."""
    x, w, shares = floats if kind == "f32" else halves
    return [0, x, w, 0] if shares else [0, x, 0, w]


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size,halves,floats", CASES)
def test_large_tiles_are_exact_on_few_digits(size, halves, floats, kind):
    """Values whose codes and scales are exact (a block's largest is 448 times a power of two), so that every product, sum and share is."""
    m, k, n = size
    dtype = TYPES[kind]
    gen = torch.Generator(device=DEV).manual_seed(m)

    def of(rows, columns, top):
        return torch.randint(-2, 3, (rows, columns), generator=gen, device=DEV).float() * (top / 2)

    dy, x = of(m, n, 7.0), of(m, k, 3.5)
    w = torch.randint(-2, 3, (n, k), generator=gen, device=DEV).float()
    sw = 2.0 ** torch.randint(-1, 2, (-(-n // 128), -(-k // 128)), generator=gen, device=DEV).float()
    # multiples of 3.5 / 2 and 3.5 * 1.75, at most 2^24 of them however they are added: exact in fp32
    got = []
    ran = launches(lambda: got.extend(fnn.fnn_linear_e4m3_backward(dy.to(dtype), x.to(dtype), placed(w, sw))), "linear_e4m3_backward_kernels")
    assert ran == ways(kind, halves, floats)
    wide = [t.double() for t in (dy, x, w * spread(sw, n, k))]
    assert torch.equal(got[0], (wide[0] @ wide[2]).to(dtype))
    assert torch.equal(got[1], (wide[0].t().contiguous() @ wide[1]).to(dtype))
    assert torch.equal(got[2], wide[0].sum(0).to(dtype))


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("size,halves,floats", CASES)
def test_large_tiles(size, halves, floats, act, kind):
    m, k, n = size
    dtype = TYPES[kind]
    x, dy, pre = normal(1, m, k, dtype=dtype), normal(3, m, n, dtype=dtype), normal(4, m, n, dtype=dtype)
    w = scaled_of(normal(2, n, k, std=1 / math.sqrt(k)), tiles=True)
    ran = launches(lambda: check_backward(dy, x, w, None if act == "none" else pre, act), "linear_e4m3_backward_kernels")
    assert ran == ways(kind, halves, floats)


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("m,k,n", [(1, 300, 500), (70, 200, 136), (1100, 264, 700)])
def test_activations_in_fp16(m, k, n, act):
    x, dy, pre = (normal(i, *s, dtype=torch.float16) for i, s in enumerate(((m, k), (m, n), (m, n))))
    check_backward(dy, x, scaled_of(normal(5, n, k), tiles=True), pre, act)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("m,k,n", [(6, 264, 300), (200, 264, 300), (100, 70, 9000), (3000, 2100, 2300), (6000, 1700, 2900)])
def test_what_is_not_finite_stays_in_its_rows_and_columns(m, k, n, act, kind):
    """Infinities and NaN in dy, pre and x reach the rows of dx and the rows or columns of dw that are made of them; everything else has the bits that zeros in their places give, since
    neither enters a scale."""
    dtype = TYPES[kind]
    x, dy, pre = normal(1, m, k, dtype=dtype), normal(3, m, n, dtype=dtype), normal(4, m, n, dtype=dtype)
    w = scaled_of(normal(2, n, k, std=1 / math.sqrt(k)), tiles=True)
    given = None if act == "none" else pre
    bad = [(0, 5, math.inf), (m // 2, n - 1, math.nan), (m - 1, n // 2, -math.inf)]       # of dy
    of_pre, of_x = (m // 3, n // 3), [(m - 1, 3, math.inf), (1, k - 1, math.nan)]
    for i, j, _ in bad:
        dy[i, j] = 0
        pre[i, j] = 1                       # where no activation's slope is 0
    for i, j, _ in of_x:
        x[i, j] = 0
    if act != "none":
        dy[of_pre] = 0
    clean = fnn.fnn_linear_e4m3_backward(dy, x, w, given, act=act)
    assert all(torch.isfinite(t).all() for t in clean)
    for i, j, v in bad:
        dy[i, j] = v
    for i, j, v in of_x:
        x[i, j] = v
    rows, columns = [i for i, _, _ in bad], [j for _, j, _ in bad]
    if act != "none":
        dy[of_pre] = 1
        pre[of_pre] = math.nan
        rows.append(of_pre[0])
        columns.append(of_pre[1])
    dx, dw, dbias = fnn.fnn_linear_e4m3_backward(dy, x, w, given, act=act)

    def others(count, but):
        kept = torch.ones(count, dtype=torch.bool, device=DEV)
        kept[but] = False
        return kept

    r, c, kept = others(m, rows), others(n, columns), others(k, [j for _, j, _ in of_x])
    assert torch.isnan(dx[~r]).all() and torch.equal(dx[r], clean[0][r])
    assert torch.isnan(dw[~c]).all() and torch.isnan(dw[:, ~kept]).all() and torch.equal(dw[c][:, kept], clean[1][c][:, kept])
    assert not torch.isfinite(dbias[~c]).any() and torch.equal(dbias[c], clean[2][c])


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_infinities_in_pre(act, kind):
    """Far to the right ReLU's slope is 1 and far to the left 0; the formulas of the others have infinity times 0 there."""
    m, k, n = 200, 264, 300
    dtype = TYPES[kind]
    x, dy, pre = normal(1, m, k, dtype=dtype), normal(3, m, n, dtype=dtype), normal(4, m, n, dtype=dtype)
    w = scaled_of(normal(2, n, k, std=1 / math.sqrt(k)), tiles=True)
    pre[7, 11], pre[9, 13] = (1, -1) if act == "relu" else (0, 0)
    if act != "relu":
        dy[7, 11] = dy[9, 13] = 0
    clean = fnn.fnn_linear_e4m3_backward(dy, x, w, pre, act=act)
    pre[7, 11], pre[9, 13] = math.inf, -math.inf
    if act != "relu":
        dy[7, 11] = dy[9, 13] = 1
    got = fnn.fnn_linear_e4m3_backward(dy, x, w, pre, act=act)
    if act == "relu":
        assert all(torch.equal(a, b) for a, b in zip(got, clean))
        return
    r, c = torch.ones(m, dtype=torch.bool, device=DEV), torch.ones(n, dtype=torch.bool, device=DEV)
    r[[7, 9]] = c[[11, 13]] = False
    assert torch.isnan(got[0][~r]).all() and torch.equal(got[0][r], clean[0][r])
    assert torch.isnan(got[1][~c]).all() and torch.equal(got[1][c], clean[1][c])
    assert torch.isnan(got[2][~c]).all() and torch.equal(got[2][c], clean[2][c])


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu"])
@pytest.mark.parametrize("m,k,n", [(6, 264, 300), (200, 264, 300), (531, 777, 401), (100, 70, 9000), (3000, 2100, 2300), (6000, 1700, 2900)])
def test_gradient_is_made_of_the_other_operators(m, k, n, act, kind):
    """Without an activation, or with one whose slope is 0 or 1, q is not rounded on the way: its codes are those of fnn_quantize, and the products those of fnn_linear_e4m3, to the bit."""
    dtype = TYPES[kind]
    x, dy, pre = normal(1, m, k, dtype=dtype), normal(3, m, n, dtype=dtype), normal(4, m, n, dtype=dtype)
    w = scaled_of(normal(2, n, k, std=1 / math.sqrt(k)), tiles=True)
    dx, dw, _ = fnn.fnn_linear_e4m3_backward(dy, x, w, None if act == "none" else pre, act=act)
    q = dy if act == "none" else torch.where(pre > 0, dy, torch.zeros_like(dy))
    across = fnn.FnnScaled(w.data.view(torch.uint8).t().contiguous().view(torch.float8_e4m3fn), w.scale.t())
    assert torch.equal(dx, fnn.fnn_linear_e4m3(fnn.fnn_quantize(q), across, dtype=dtype)[0])
    assert torch.equal(dw, fnn.fnn_linear_e4m3(fnn.fnn_quantize(q, transposed=True), fnn.fnn_quantize(x, transposed=True), dtype=dtype)[0])


@pytest.mark.parametrize("kind", ["f32", "f16"])
def test_sums_of_nothing_in_tiles(kind):
    """No rows, no outputs or no inputs, with the other sizes beyond few rows: zeros where something is asked for, whatever the memory held."""
    def zeros(*s):
        return torch.zeros(s, device=DEV, dtype=TYPES[kind])

    def weights(n, k):
        return fnn.fnn_quantize(zeros(n, k), tiles=True)

    for act in ("none", "gelu"):
        dx, dw, dbias = fnn.fnn_linear_e4m3_backward(zeros(0, 300), zeros(0, 264), weights(300, 264), zeros(0, 300), act=act)
        assert dx.shape == (0, 264) and dw.shape == (300, 264) and not dw.any() and dbias.shape == (300,) and not dbias.any()
        out = torch.full((300, 264), 7.0, device=DEV, dtype=TYPES[kind])
        dx, dw, dbias = fnn.fnn_linear_e4m3_backward(zeros(300, 0), zeros(300, 264), weights(0, 264), zeros(300, 0), act=act, out=out)
        assert dx is out and not out.any() and dw.shape == (0, 264) and dbias.shape == (0,)
        dx, dw, dbias = fnn.fnn_linear_e4m3_backward(zeros(300, 264) + 1, zeros(300, 0), weights(264, 0), zeros(300, 264), act=act)
        assert dx.shape == (300, 0) and dw.shape == (264, 0) and (dbias == (300 if act == "none" else 150)).all()
