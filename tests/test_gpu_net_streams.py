"""Calls of the network's operators on another stream do not take memory that the current stream has given up but may still work in."""
import math

import pytest
import torch

import paper_2503_10017_amd as fnn
from net_helpers import DEV, normal

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def calls():
    x, w, dy = normal(1, 600, 512, dtype=BF), normal(2, 520, 512, std=1 / math.sqrt(512), dtype=BF), normal(3, 600, 520, dtype=BF)
    dx = normal(4, 600, 512, dtype=BF)
    q, k, v = normal(5, 2, 16, 64, dtype=BF), normal(6, 5000, 4, 64, dtype=BF), normal(7, 5000, 4, 64, dtype=BF)
    weight = normal(8, 512, dtype=BF)
    _, mean, rstd = fnn.fnn_layer_norm(x, weight, want_stats=True)
    out, lse = fnn.fnn_attention(q, k, v)
    return [
        lambda **kw: fnn.fnn_layer_norm(x, weight, want_stats=True, **kw),
        lambda **kw: fnn.fnn_layer_norm_backward(dx, x, mean, rstd, weight, **kw),
        lambda **kw: fnn.fnn_linear(x, w, act="gelu", want_pre=True, **kw),
        lambda **kw: fnn.fnn_linear_backward(dy, x, w, dy, act="silu", **kw),
        lambda **kw: fnn.fnn_attention(q, k, v, causal=True, **kw),
        lambda **kw: fnn.fnn_attention_backward(q, q, k, v, out, lse, **kw),
    ]


@pytest.mark.parametrize("which", range(6))
def test_no_block_of_the_current_stream(which):
    call = calls()[which]
    want = [t.clone() for t in call()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    freed = call()
    addresses = {t.data_ptr() for t in freed}
    del freed                                        # the current stream's pool has these blocks, and its work is not waited for
    got = call(stream=side)
    assert not addresses & {t.data_ptr() for t in got}
    torch.cuda.current_stream().wait_stream(side)
    again = call()                                   # and the other way round
    assert not {t.data_ptr() for t in got} & {t.data_ptr() for t in again}
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(a, b) for a, b in zip(again, want))
    torch.cuda.synchronize()
