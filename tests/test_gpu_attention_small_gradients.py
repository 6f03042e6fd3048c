"""fnn_attention_backward in fp16 where dout is small (an unscaled mean loss) or large: what p (dout v^T - delta) is rounded to has the type's digits
relative to the largest of its row (dq) and of its key (dk), whatever its size."""
import math

import pytest
import torch

from net_helpers import DEV, F32, ROUND, assert_within, rounding
from test_gpu_attention import Problem, backward, weight_slack

pytestmark = pytest.mark.gpu

U = ROUND[torch.float16]
CASES = [([40], [20000], 1, 1, 32, False), ([300, 65], [300, 65], 4, 2, 64, True), ([130], [700], 2, 2, 128, False), ([200, 1, 33], [64, 500, 33], 6, 2, 96, True), ([5], [40], 3, 1, 40, True)]


def check(prob, out, lse, grads):
    """ds is formed in fp32, times a power of two, and rounded once: half a unit of its own (U), or half of fp16's last step, 2^-25, while the largest of the row (key) so
    far is 1 and more by that power of two.  The sums are fp32."""
    want = [torch.zeros(t.shape, dtype=torch.float64, device=DEV) for t in (prob.q, prob.k)]
    slack = [torch.zeros_like(t) for t in want]
    most = torch.zeros(prob.k.shape[:2], dtype=torch.float64, device=DEV)       # the largest ds of a key
    parts = []
    for rows, keys, h, g, p, _, mag in prob.sequences():
        q, k, v, dout, o = (t.double() for t in (prob.q[rows, h], prob.k[keys, g], prob.v[keys, g], prob.dout[rows, h], out[rows, h]))
        rel = weight_slack(p, mag, prob.d) + 2.2 * 16 * F32
        dp, exact_out = dout @ v.t(), p @ v
        delta = (dout * exact_out).sum(1, keepdim=True)
        delta_off = (dout.abs() * ((exact_out - o).abs() + (prob.d + 8) * F32 * o.abs())).sum(1, keepdim=True)
        ds = p * (dp - delta)
        off = p * ((prob.d + 8) * F32 * (dout.abs() @ v.abs().t()) + delta_off + 4 * F32 * (dp.abs() + delta.abs())) + (rel + U + prob.heads * (max(p.shape) + 8) * F32) * ds.abs()
        want[0][rows, h] = prob.scale * (ds @ k)
        slack[0][rows, h] = prob.scale * ((off + 1.01 * 2.0 ** -25 * ds.abs().amax(1, keepdim=True)) @ k.abs()) if p.shape[1] else 0
        want[1][keys, g] += prob.scale * (ds.t() @ q)
        if p.shape[1]:
            most[keys, g] = torch.maximum(most[keys, g], ds.abs().amax(0))
        parts.append((keys, g, off, q))
    for keys, g, off, q in parts:
        slack[1][keys, g] += prob.scale * ((off + 1.01 * 2.0 ** -25 * most[keys, g]).t() @ q.abs())
    for name, got, w, s in zip(("dq", "dk"), grads, want, slack):
        assert_within(got, w, s + rounding(w, torch.float16), name)
    return want


@pytest.mark.parametrize("size", [1e-5, 1e-4, 1.0])
@pytest.mark.parametrize("large", ["q", "k"])
@pytest.mark.parametrize("case", CASES)
def test_small_gradients(case, large, size):
    """Flat rows; keys (queries) of 64 bring dq (dk) into fp16's normal range, so that what is lost of ds shows."""
    prob = Problem(*case, "f16")
    for name in "qk":
        getattr(prob, name).mul_(64 if name == large else 2.0 ** -10)
    prob.dout = (prob.dout.float() * size).half()
    out, lse = prob.call()
    grads = backward(prob, out, lse)
    want = check(prob, out, lse, grads)
    got, w = (grads[1], want[1]) if large == "q" else (grads[0], want[0])
    # roundings of ds of random signs, and the result's own: below 2^-10 of the norm each, and out's, through delta, as large again
    last = 2.0 ** -24 * math.sqrt(w.numel())
    assert (got.double() - w).norm() <= 2.0 ** -8 * w.norm() + last


@pytest.mark.parametrize("case", [([64], [4], 2, 1, 64, False), ([300], [3], 1, 1, 128, False), ([130, 5], [5, 5], 4, 2, 32, True)])
def test_large_gradients(case):
    """dout and v whose products pass fp16's largest number, with keys and queries small enough that dq and dk do not."""
    prob = Problem(*case, "f16")
    prob.q.mul_(2.0 ** -6)
    prob.k.mul_(2.0 ** -6)
    prob.v.mul_(100)
    prob.dout.mul_(500)
    out, lse = prob.call()
    grads = backward(prob, out, lse)
    check(prob, out, lse, grads)


def test_rows_of_one_call_keep_their_own_scale():
    """Rows of very different dout, large and small next to each other: dq of the small ones is as exact as alone."""
    prob = Problem([96], [500], 2, 2, 64, False, "f16")
    prob.q.mul_(2.0 ** -10)
    prob.k.mul_(64)
    prob.dout[1::2] = (prob.dout[1::2].float() * 1e-5).half()
    prob.dout[::2] *= 100
    out, lse = prob.call()
    dq = backward(prob, out, lse)[0]
    want = check(prob, out, lse, (dq, backward(prob, out, lse)[1]))[0]
    small = (dq[1::2].double() - want[1::2]).norm()
    assert small <= 2.0 ** -8 * want[1::2].norm() + 2.0 ** -24 * math.sqrt(want[1::2].numel())


def test_nothing_to_learn_is_zero():
    prob = Problem([70], [300], 2, 1, 64, True, "f16")
    prob.dout.zero_()
    out, lse = prob.call()
    assert not any(g.any() for g in backward(prob, out, lse))
