"""What a causal query does not see, in fp16: the gradient scales what it rounds row by row and key by key, and the scale of one must not be another's."""
import math

import pytest

import test_gpu_attention as bf16

pytestmark = pytest.mark.gpu


@pytest.fixture
def f16(monkeypatch):
    of = bf16.Problem
    monkeypatch.setattr(bf16, "Problem", lambda *args: of(*args[:-1], "f16"))
    return bf16


BAD = pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
SIZES = pytest.mark.parametrize("nq,nk,heads,groups,d,j", bf16.NOT_YET_SEEN)


@BAD
@SIZES
def test_forward(f16, nq, nk, heads, groups, d, j, bad):
    f16.test_causal_queries_know_nothing_of_later_keys(nq, nk, heads, groups, d, j, bad)


@BAD
@pytest.mark.parametrize("which", ["q", "k", "v", "dout"])
@SIZES
def test_gradients(f16, nq, nk, heads, groups, d, j, which, bad):
    f16.test_causal_gradients_know_nothing_of_what_is_not_seen(nq, nk, heads, groups, d, j, which, bad)
