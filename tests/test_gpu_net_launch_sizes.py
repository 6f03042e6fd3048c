"""Sizes at which one launch has no room for all workgroups (a launch has fewer than 2^32 threads)."""
import gc

import pytest
import torch

import paper_2503_10017_amd as fnn
from net_helpers import DEV

pytestmark = pytest.mark.gpu

OUTER = 2 ** 27 + 40      # 16 results to a workgroup of 512 threads, 32 columns to one of 1024: 2^32 threads at 2^27


def whole(shape, most, dtype):
    """Whole numbers up to `most` in size; made on the device, the same every time."""
    gen = torch.Generator(device=DEV).manual_seed(1)
    return torch.randint(-most, most + 1, shape, generator=gen, device=DEV, dtype=torch.int8).to(dtype)


def codes(v, tiles):
    n = -(-v.shape[0] // 128) if tiles else v.shape[0]
    return fnn.FnnScaled(v.to(torch.float8_e4m3fn), torch.ones((-(-v.shape[1] // 128), n), device=DEV).t())


@pytest.mark.parametrize("rows", [1, 17])
def test_few_rows_over_many_columns(rows):
    w, x = whole((OUTER, 16), 2, torch.bfloat16), whole((rows, 16), 2, torch.bfloat16)
    y = fnn.fnn_linear_e4m3(codes(x, False), codes(w, True))[0]
    for i in range(rows):
        assert torch.equal(y[i], (w * x[i]).sum(1))      # sums below 65: exact


@pytest.mark.parametrize("rows", [1, 17])
def test_few_rows_over_many_columns_in_16_bits(rows):
    w, x = whole((OUTER, 16), 2, torch.float16), whole((rows, 16), 2, torch.float16)
    y = fnn.fnn_linear(x, w)[0]
    for i in range(rows):
        assert torch.equal(y[i], (w * x[i]).sum(1))


def test_a_launch_of_too_many_workgroups_is_refused():
    """A workgroup of 256 threads for each of 2^24 sequences and more: an error instead of rows that nothing has written."""
    batch = 2 ** 24 + 100
    q = torch.zeros((batch, 1, 8), dtype=torch.float16, device=DEV)
    starts = torch.arange(batch + 1, dtype=torch.int32, device=DEV)
    with pytest.raises(fnn.FnnError):
        fnn.fnn_attention(q, q, q, starts, starts)
    with pytest.raises(fnn.FnnError):
        fnn.fnn_attention_backward(q, q, q, q, q, torch.zeros((batch, 1), device=DEV), starts, starts)


def test_as_many_rows_as_a_matrix_may_have():
    rows = 2 ** 31 - 65
    data, scale = torch.zeros((rows, 16), dtype=torch.uint8, device=DEV), torch.ones((1, rows), device=DEV).t()
    data[-5:, 3] = 0x38                                   # 1
    y = fnn.fnn_linear_e4m3(fnn.FnnScaled(data.view(torch.float8_e4m3fn), scale), codes(torch.ones((1, 16), device=DEV), True))[0]
    assert (y[-5:] == 1).all() and not y[:-5].any()


def test_the_bias_gradient_of_many_columns():
    dy = whole((1, OUTER), 2, torch.bfloat16) * 3.5       # codes and scales of these are exact: a block's largest is 448 times a power of two
    x, w = whole((1, 16), 2, torch.bfloat16) * 1.75, whole((OUTER, 16), 2, torch.bfloat16)
    dx, dw, dbias = fnn.fnn_linear_e4m3_backward(dy, x, codes(w, True))
    assert torch.equal(dbias, dy[0])
    assert torch.equal(dw, dy.t() * x)                    # 49 / 8 times 0, 1, 2 or 4
    want = sum((dy[0, i:i + 2 ** 24, None].double() * w[i:i + 2 ** 24]).sum(0) for i in range(0, OUTER, 2 ** 24))
    assert torch.equal(dx[0], want.bfloat16())            # multiples of 3.5, far fewer than 2^24 of them
    del dw
    assert torch.equal(fnn.fnn_linear_backward(dy, x, w, want_x=False, want_w=False)[2], dy[0])


def test_copies_of_many_rows():
    """Rows of 33 codes copied to 16-byte boundaries: three runs of 16 bytes each, of which 2^32 are 64 GB."""
    rows, inner = 1440 * 10 ** 6, 33
    gc.collect()
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 150 << 30:
        pytest.skip("needs 130 GB")
    data = torch.zeros((rows, inner), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
    scale = torch.ones((1, rows), device=DEV).t()
    every = 2 ** 20 - 3                                   # these rows hold something, the first and the last among them
    some = torch.cat([torch.arange(0, rows, every), torch.tensor([rows - 1])]).to(DEV)
    v, w = whole((len(some), inner), 2, torch.bfloat16), whole((1, inner), 2, torch.bfloat16)
    data.view(torch.uint8)[some] = v.to(torch.float8_e4m3fn).view(torch.uint8)
    y = fnn.fnn_linear_e4m3(fnn.FnnScaled(data, scale), codes(w, True))[0]
    assert torch.equal(y[some], (v * w).sum(1, keepdim=True))
    y[some] = 0
    assert not y.any()
    del data, scale, y
    gc.collect()
    torch.cuda.empty_cache()
