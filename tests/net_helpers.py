"""Shared pieces of the tests of the network's operators (include/fnn_net.h): plain forms in 64 bits and derived tolerances."""
import math

import torch

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# unit roundoff of a type: the largest relative error of one rounding to nearest
ROUND = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
# values below this are stored with an absolute error of up to half the smallest subnormal
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}
F32 = ROUND[torch.float32]


def normal(seed, *shape, std=1.0, dtype=torch.float32):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=gen, dtype=torch.float64) * std).to(dtype).to(DEV)


def strided(t, extra, offset=0):
    """The same matrix with rows `extra` elements further apart, the first `offset` elements into its buffer; NaN between the rows."""
    n, d = t.shape
    buf = torch.full((offset + n * (d + extra) + 8,), math.nan, dtype=t.dtype, device=t.device)
    view = buf[offset:offset + n * (d + extra)].view(n, d + extra)[:, :d]
    view.copy_(t)
    return view


def assert_within(got, want, slack, what=""):
    """|got - want| <= slack (a tensor or a number) wherever want is finite, and got is finite exactly there."""
    want = want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    got = got.double()
    finite = torch.isfinite(want)
    assert torch.equal(finite, torch.isfinite(got)), what
    off = torch.where(finite, (got - want).abs() - slack, torch.zeros_like(want))
    worst = off.max().item() if off.numel() else 0.0
    assert worst <= 0, (what, worst, int((off > 0).sum()), off.numel())



def rounding(want, dtype):
    """The error of rounding `want`, or a value near it, once to dtype (1 % more than the bound: the rounded value is the computed one)."""
    return want.double().abs() * ROUND[dtype] * 1.01 + TINY[dtype]
