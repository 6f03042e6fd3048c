"""fnn_attention in fp16 where one key outweighs each of very many others, which together weigh as much: their weights, far below fp16's normal range beside the
largest, are not to lose their digits."""
import math

import pytest
import torch

import paper_2503_10017_amd as fnn
from net_helpers import DEV, F32

pytestmark = pytest.mark.gpu


# a part of the keys has a largest of its own: with many rows there is one part
@pytest.mark.parametrize("queries,heads", [(1, 2), (70, 1), (4000, 16)])
@pytest.mark.parametrize("keys,bits", [(60000, 14.37), (60000, 16.53), (500000, 18.53), (1000000, 20.53)])
def test_many_small_weights(keys, bits, queries, heads):
    """Scores of ln 2 * bits for one key and 0 for all others: weights of 2^-bits beside it, below the type's normal range or close to it.  As they are formed 2^7
    times larger, a weight is rounded to half of 2^-31 of the largest, which at 2^-20.53 is a 2^-11.5th of it: with the values 1 and 0, of all of the sum.  Then
    the result's own rounding, half of 2^-10, and the fp32 sums, in parts of at most 2^14 keys one after the other."""
    d = 32
    k = torch.zeros((keys, 1, d), dtype=torch.float16, device=DEV)
    v = torch.ones((keys, 1, d), dtype=torch.float16, device=DEV)
    q = torch.ones((queries, heads, d), dtype=torch.float16, device=DEV)
    k[0], v[0] = 1, 0
    scale = math.log(2) * bits / d                                  # <q, k> is 32, exactly
    out, lse = fnn.fnn_attention(q, k, v, scale=scale)
    mass = (keys - 1) * 2.0 ** -bits
    want, want_lse = mass / (1 + mass), math.log(2) * bits + math.log1p(mass)
    relative = 2.0 ** -32 * 2.0 ** bits + 2.0 ** -11 + 2.0 ** 14 * F32 + 32 * bits * F32
    assert (out.double() - want).abs().max().item() <= relative * want
    assert (lse.double() - want_lse).abs().max().item() <= (2.0 ** 14 + 64) * F32 + 4 * F32 * want_lse
