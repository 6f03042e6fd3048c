"""NaN and infinities in calls of fnn_attention whose keys are split: a share that holds nothing but NaN, or a weight of 0, is not a share
without keys."""
import math

import pytest
import torch

import paper_2503_10017_amd as fnn
from test_gpu_attention import Problem

pytestmark = pytest.mark.gpu

# few rows a sequence and many of them, joined by a workgroup a row (below 2048 rows) and by a group of lanes a row
SPLIT = [
    ([2], [6000], 4, 2, 64, True),
    ([1, 2], [3000, 2500], 16, 4, 128, True),
    ([1] * 64, [4000] * 64, 32, 1, 32, False),
    ([40], [6000], 16, 2, 64, False),
    ([40], [6000], 64, 2, 32, True),
]


def split_problem(case, kind):
    prob = Problem(*case, kind)
    assert fnn.fnn_attention_workspace_bytes(prob.q.shape[0], prob.k.shape[0], len(prob.lq), prob.heads, prob.groups, prob.d) > 0
    return prob


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("case", SPLIT)
def test_a_query_of_nan_answers_nan(case, kind):
    prob = split_problem(case, kind)
    want, want_lse = prob.call()
    rows = [(0, 0), (prob.q.shape[0] - 1, prob.heads - 1)]
    for i, h in rows:
        prob.q[i, h, 3] = math.nan
    out, lse = prob.call()
    for i, h in rows:
        assert torch.isnan(out[i, h]).all() and torch.isnan(lse[i, h])
        out[i, h], lse[i, h] = want[i, h], want_lse[i, h]
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("case", SPLIT)
def test_keys_of_nan_throughout_answer_nan(case):
    """1024 keys of the first sequence in a row: whole parts of them."""
    prob = split_problem(case, "bf16")
    want, want_lse = prob.call()
    prob.k[512:1536, 0] = math.nan
    out, lse = prob.call()
    first, share = prob.lq[0], prob.heads // prob.groups
    assert torch.isnan(out[:first, :share]).all() and torch.isnan(lse[:first, :share]).all()
    out[:first, :share], lse[:first, :share] = want[:first, :share], want_lse[:first, :share]
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("case", SPLIT)
def test_a_value_under_a_vanishing_weight_is_not_lost(case, bad):
    """The first 256 keys score 200 and more above all others, whose shares weigh 0 in fp32: what is no number there stays none, as it
    does within a share."""
    prob = split_problem(case, "bf16")
    prob.q[:, :, 0] = 8
    prob.k[:, :, 0] = -100 * 8 / prob.d ** 0.5
    first = 0
    for n in prob.lk:
        prob.k[first:first + 256, :, 0] *= -1
        first += n
    want, want_lse = prob.call()
    assert torch.isfinite(want).all()
    prob.v[2400, 0, 5] = bad
    out, lse = prob.call()
    rows, share = prob.lq[0], prob.heads // prob.groups
    assert not torch.isfinite(out[:rows, :share, 5]).any()
    out[:rows, :share, 5] = want[:rows, :share, 5]
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
