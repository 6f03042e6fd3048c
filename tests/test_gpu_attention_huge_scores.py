"""fnn_attention on finite inputs whose scores are far larger than fp32's 24 bits resolve: one key has all the weight, and nothing
overflows."""
import math

import pytest
import torch

from net_helpers import F32
from test_gpu_attention import Problem, backward, check_forward

pytestmark = pytest.mark.gpu

CASES = [([130], [300], 2, 1, 64, False), ([90, 7], [90, 700], 2, 2, 128, True), ([5], [200], 4, 2, 96, True), ([2], [6000], 4, 2, 64, True), ([40], [6000], 64, 2, 32, False)]


def huge(case, kind):
    prob = Problem(*case, kind, scale=0.5)
    size, most = (2e4, 6e4) if kind == "f16" else (1e12, 1e13)
    prob.q, prob.k = ((t.float() * size).clamp(-most, most).to(t.dtype) for t in (prob.q, prob.k))
    return prob


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("case", CASES)
def test_the_largest_score_takes_it_all(case, kind):
    prob = huge(case, kind)
    out, lse = prob.call()
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    told = total = 0
    for rows, keys, h, g, p, want_lse, mag in prob.sequences():
        off = (prob.d + 8) * F32 * mag.amax(1)              # of a score, as it is a sum of d exact products in fp32
        z = prob.scale * (prob.q[rows, h].double() @ prob.k[keys, g].double().t())
        if prob.causal:
            z = z + torch.full_like(z, -math.inf).triu(1 + z.shape[1] - z.shape[0])
        (first, second), best = z.topk(2, 1).values.unbind(1), z.argmax(1)
        clear = first - second > 2 * off + 200              # nothing comes near the largest, whichever way the scores are rounded
        told, total = told + int(clear.sum()), total + clear.numel()
        assert torch.equal(out[rows, h][clear], prob.v[keys, g][best][clear])
        assert ((lse[rows, h].double() - want_lse).abs() <= off + 4 * F32 * want_lse.abs() + math.log(p.shape[1])).all()
    assert told > 0.8 * total


@pytest.mark.parametrize("case", CASES)
def test_scores_of_thousands(case):
    prob = Problem(*case, "f16", spread=500.0, scale=1.0)
    check_forward(prob, *prob.call())


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("case", CASES)
def test_gradients_stay_finite(case, kind):
    """lse has 24 bits, so the weights of such rows are not told; they are weights all the same, of at most about 1."""
    prob = huge(case, kind)
    prob.dout.mul_(2.0 ** -10)                              # dq and dk stay below fp16's largest
    out, lse = prob.call()
    dq, dk, dv = backward(prob, out, lse)
    assert torch.isfinite(dq).all() and torch.isfinite(dk).all() and torch.isfinite(dv).all()
    share = prob.heads // prob.groups
    rows = prob.q.shape[0]
    assert (dv.abs() <= 2 * rows * share * prob.dout.abs().max().item()).all()
