"""Every way that a product in 8 bits can take, asserted through the trace: few rows, the three tiles, shares of a long sum, operands off 16-byte boundaries; each exact on values of few digits, within the
derived bounds on others, and with all that the epilogue has."""
import math

import pytest
import torch

import paper_2503_10017_amd as fnn
from e4m3_helpers import placed, quantized, scaled_of, spread
from net_helpers import DEV, TYPES, normal
from test_gpu_linear_e4m3 import check_backward, check_forward

pytestmark = pytest.mark.gpu

FEW, FEW_32, SMALL, MIDDLE, LARGE, THROUGH_REGISTERS = 16, 32, 64, 128, 256, 129


GRADIENT = 65     # both products and the columns' sums in one launch


def launches(call, kernels="linear_e4m3_kernels"):
    fnn.fnn_trace_begin(64)
    try:
        call()
        torch.cuda.synchronize()
    finally:
        trace = fnn.fnn_trace_end(64, details=True)
    return [detail for name, _, detail in trace if name == kernels]


# size, what its product runs as, and whether its sum is cut into shares; fp32 has no large tile
CASES = [((1, 300, 50), FEW, False), ((16, 5000, 33), FEW, False), ((17, 300, 520), FEW_32, False), ((32, 1000, 40), FEW_32, False), ((33, 200, 520), SMALL, False), ((100, 6000, 130), SMALL, True),
         ((200, 272, 300), SMALL, False), ((2100, 8320, 1100), MIDDLE, True),
         ((700, 777, 600), SMALL, False), ((3000, 260, 2100), MIDDLE, False), ((2100, 8300, 1100), MIDDLE, True), ((4000, 1100, 4000), LARGE, False), ((2048, 20100, 2300), LARGE, True)]


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("tiles", [True, False])
@pytest.mark.parametrize("size,way,shares", CASES)
def test_each_way_is_exact_on_few_digits(size, way, shares, tiles, kind):
    m, k, n = size
    gen = torch.Generator(device=DEV).manual_seed(m)
    (x, sx), (w, sw) = ((torch.randint(-2, 3, (r, k), generator=gen, device=DEV).float(),
                         2.0 ** torch.randint(-1, 2, (-(-r // 128) if t else r, -(-k // 128)), generator=gen, device=DEV).float()) for r, t in ((m, False), (n, tiles)))
    # sums of whole numbers times quarters to fours, far below 2^24 quarters: exact in fp32 whatever the order
    want = ((x * spread(sx, m, k).float()) @ (w * spread(sw, n, k).float()).t()).to(TYPES[kind])
    got = []
    ran = launches(lambda: got.append(fnn.fnn_linear_e4m3(placed(x, sx, extra=-k % 16), placed(w, sw, extra=-k % 16), dtype=TYPES[kind])[0]))
    assert torch.equal(got[0], want)
    if kind != "f32" or way != LARGE:
        assert ran[0] == way and len(ran) == 1 + shares, ran
    for where in ((1, 1, 3), (3, 2, 0, True)):
        ran = launches(lambda: got.append(fnn.fnn_linear_e4m3(placed(x, sx, *where), placed(w, sw, *where), dtype=TYPES[kind])[0]))
        assert torch.equal(got.pop(), want)
        if way > FEW_32:     # copied to aligned rows where k is no multiple of 16, and otherwise through registers
            assert ran[0] == (0 if k % 16 else THROUGH_REGISTERS) and len(ran) == 1 + (k % 16 > 0) + shares, ran


@pytest.mark.parametrize("size,way,shares", [c for c in CASES if c[1] in (SMALL, MIDDLE)] + [((4000, 330, 4000), LARGE, False)])
def test_each_way_with_the_epilogue(size, way, shares):
    m, k, n = size
    x, w = scaled_of(normal(1, m, k), extra=-k % 16), scaled_of(normal(2, n, k, std=1 / math.sqrt(k)), tiles=True, extra=-k % 16)
    r, b = normal(4, m, n, dtype=torch.float16), normal(3, n, dtype=torch.float16)
    if k < 2000:                                   # the bound is formed product by product
        check_forward(x, w, b, r, "silu", torch.float16, want_pre=True)
    y, pre = fnn.fnn_linear_e4m3(x, w, b, r, act="relu", dtype=torch.float16, want_pre=True)
    plain = fnn.fnn_linear_e4m3(x, w, b, dtype=torch.float16)[0]
    assert torch.equal(pre, plain)
    in_place = r.clone()
    assert torch.equal(fnn.fnn_linear_e4m3(x, w, b, in_place, act="relu", out=in_place)[0], y)


def test_neighbouring_calls_share_nothing():
    """Calls one after the other with workspaces of their own, of one with shares and of one without, give what each gives alone."""
    calls = []
    for i, (m, k, n) in enumerate(((100, 6000, 130), (2100, 8300, 1100), (4000, 330, 4000), (300, 300, 300))):
        x, w = scaled_of(normal(i, m, k), extra=-k % 16), scaled_of(normal(i + 9, n, k), tiles=True, extra=-k % 16)
        calls.append(lambda x=x, w=w: fnn.fnn_linear_e4m3(x, w)[0])
    alone = []
    for call in calls:
        alone.append(call())
        torch.cuda.synchronize()
    together = [call() for call in calls + calls[::-1]]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(together, alone + alone[::-1]))


def test_two_streams_at_once():
    """Two calls at once on two streams, and two graphs that share one workspace in turn."""
    m, k, n = 2100, 8300, 1100
    x, w = scaled_of(normal(1, m, k), extra=-k % 16), scaled_of(normal(2, n, k), tiles=True, extra=-k % 16)
    x2 = scaled_of(normal(3, m, k), extra=-k % 16)
    want, want2 = fnn.fnn_linear_e4m3(x, w)[0].clone(), fnn.fnn_linear_e4m3(x2, w)[0].clone()
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        a, b = fnn.fnn_linear_e4m3(x, w, stream=one)[0], fnn.fnn_linear_e4m3(x2, w, stream=two)[0]
        torch.cuda.synchronize()
        assert torch.equal(a, want) and torch.equal(b, want2)
    ws = torch.empty(fnn.fnn_linear_e4m3_workspace_bytes(m, k, n, torch.bfloat16), dtype=torch.uint8, device=DEV)
    graphs, outs = [], []
    for given in (x, x2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(fnn.fnn_linear_e4m3(given, w, workspace=ws)[0])
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want2)
        ws.fill_(0x7F)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size,one", [((200, 264, 300), True), ((33, 129, 40), True), ((700, 65, 1001), True), ((6, 264, 300), False), ((100, 70, 9000), False), ((9000, 70, 100), False)])
def test_a_gradient_in_one_launch_or_product_by_product(size, one, kind):
    m, k, n = size
    dtype = TYPES[kind]
    dy, x, w = normal(1, m, n, dtype=dtype), normal(2, m, k, dtype=dtype), scaled_of(normal(3, n, k, std=1 / math.sqrt(k)), tiles=True)
    got = []
    ran = launches(lambda: got.extend(check_backward(dy, x, w, None, "none")), "linear_e4m3_backward_kernels")
    assert (ran == [0, GRADIENT]) == one, ran
    if size == (9000, 70, 100):     # operands, two products, and the shares of dw joined with the columns' sums
        assert len(ran) == 4, ran
    parts = (fnn.fnn_linear_e4m3_backward(dy, x, w, want_x=i == 0, want_w=i == 1, want_bias=i == 2)[i] for i in range(3))
    for part, whole in zip(parts, got):
        assert torch.equal(part, whole)
    if one:     # without sums, and twice the same bits
        again = fnn.fnn_linear_e4m3_backward(dy, x, w, want_bias=False)
        assert again[2] is None and torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
