"""fnn_attention where scores are minus infinity: such keys weigh 0, a query that sees no others has no softmax (NaN), and neither is a
query that sees no key (0)."""
import math

import pytest
import torch

import paper_2503_10017_amd as fnn
from test_gpu_attention import Problem, backward, check_forward

pytestmark = pytest.mark.gpu

# not split and split, few rows and many, rows without keys
CASES = [
    ([130], [300], 2, 1, 64, True),
    ([5], [200], 4, 2, 96, True),
    ([90, 7], [20, 7], 2, 2, 64, True),
    ([2], [6000], 4, 2, 64, True),
    ([1] * 64, [4000] * 64, 32, 1, 32, False),
    ([40], [6000], 16, 2, 64, False),
    ([40], [6000], 64, 2, 32, True),
]


@pytest.mark.parametrize("case", CASES)
def test_no_other_scores(case):
    prob = Problem(*case, "bf16")
    prob.k[:, :, 0] = -1
    want, want_lse = prob.call()
    last = (prob.q.shape[0] - 1, prob.heads - 1)
    rows = [(0, 0), last]
    for i, h in rows:
        prob.q[i, h, 0] = math.inf
    out, lse = prob.call()
    for i, h in rows:
        sees = not prob.causal or i + prob.lk[0] - prob.lq[0] >= 0 or (i, h) == last
        if sees:
            assert torch.isnan(out[i, h]).all()
        else:
            assert not out[i, h].any()
        assert lse[i, h] == -math.inf
        out[i, h], lse[i, h] = want[i, h], want_lse[i, h]
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("case", CASES[:3])
def test_gradient_without_other_scores(case):
    prob = Problem(*case, "bf16")
    prob.k[:, :, 0] = -1
    out, lse = prob.call()
    want = backward(prob, out, lse)
    i, h = prob.q.shape[0] - 1, prob.heads - 1
    prob.q[i, h, 0] = math.inf
    out, lse = prob.call()
    dq, dk, dv = backward(prob, out, lse)
    group = h // (prob.heads // prob.groups)
    keys = slice(prob.k.shape[0] - prob.lk[-1], None)       # the last query sees all of its sequence's
    assert torch.isnan(dq[i, h]).all() and torch.isnan(dk[keys, group]).all() and torch.isnan(dv[keys, group]).all()
    for got, w in ((dq, want[0]),):
        got[i, h] = w[i, h]
        assert torch.equal(got, w)
    for got, w in ((dk, want[1]), (dv, want[2])):
        got[keys, group] = w[keys, group]
        assert torch.equal(got, w)


@pytest.mark.parametrize("case", [([5], [200], 4, 2, 64, False), ([2], [6000], 4, 2, 64, False), ([40], [6000], 16, 2, 64, False), ([130], [1500], 2, 2, 64, False)])
def test_such_keys_weigh_nothing(case):
    """1024 (or 100) keys in a row score minus infinity: the answer is that of the call without them."""
    prob = Problem(*case, "bf16")
    prob.q[:, :, 7] = 1
    drop = slice(512, 1536) if prob.lk[0] > 2000 else slice(50, 150)
    kept = [torch.cat((t[:drop.start], t[drop.stop:])) for t in (prob.k, prob.v)]
    prob.k[drop, :, 7] = -math.inf
    out, lse = prob.call()
    prob.k, prob.v = kept
    prob.lk = [prob.k.shape[0]]
    check_forward(prob, out, lse)


def test_no_key_at_all_is_still_zero():
    prob = Problem([70], [40], 2, 1, 64, True, "f16")
    prob.q[:10] = math.inf
    out, lse = prob.call()
    assert not out[:10].any() and (lse[:10] == -math.inf).all()
    dq = fnn.fnn_attention_backward(prob.dout, prob.q, prob.k, prob.v, out, lse, prob.cu_q, prob.cu_k, causal=True)[0]
    assert not dq[:10].any()
