"""Shared pieces of the tests of the operators in 8 bits: the definitions of include/fnn_net.h in 64 bits."""
import torch

import paper_2503_10017_amd as fnn

BLOCK = 128


def nearest_e4m3(v):
    """The e4m3 value nearest to each number of v (float64, at most 448 in size), halves to the even one."""
    _, exponent = torch.frexp(v)
    step = (((exponent - 1).clamp(min=-6).long() + (1023 - 3)) << 52).view(torch.float64)     # the power of two by its bits
    return torch.round(v / step) * step


def blocks(n):
    return -(-n // BLOCK)


def spread(scale, n, d):
    """A scale for every element."""
    scale = scale.double()
    if scale.shape[0] != n:
        scale = scale.repeat_interleave(BLOCK, 0)[:n]
    return scale.repeat_interleave(BLOCK, 1)[:, :d]


def block_scales(v, tiles=False):
    """The scales of v (float64): the largest finite magnitude over 448, in fp32."""
    n, d = v.shape
    high = BLOCK if tiles else 1
    v = torch.where(torch.isfinite(v), v.abs(), 0.0)
    v = torch.nn.functional.pad(v, (0, -d % BLOCK, 0, -n % high))
    top = v.view(v.shape[0] // high, high, -1, BLOCK).amax((1, 3))
    return torch.maximum(top / 448, torch.full_like(top, 2.0 ** -126)).float()


def quantized(v, tiles=False):
    """Values of the codes (float64) and scales (float32) of v."""
    v = v.double()
    scale = block_scales(v, tiles)
    quotient = (v / spread(scale, *v.shape)).float().double()
    return torch.where(torch.isfinite(v), nearest_e4m3(quotient.clamp(-448, 448)), torch.nan), scale


def values(s):
    """What an FnnScaled stands for, in 64 bits."""
    return s.data.double() * spread(s.scale, *s.data.shape)


def scaled_of(v, tiles=False, extra=0, offset=0, scale_gap=0, scale_by_rows=False):
    """v in 8 bits by the definition, with rows `extra` bytes apart, the first `offset` bytes into its buffer, NaN codes between them; scales `scale_gap` floats apart, by columns of blocks
    (or by rows), NaN between them."""
    data, scale = quantized(v, tiles)
    return placed(data, scale, extra, offset, scale_gap, scale_by_rows)


def placed(data, scale, extra=0, offset=0, scale_gap=0, scale_by_rows=False):
    n, d = data.shape
    room = torch.full((offset + n * (d + extra) + 16,), 0x7F, dtype=torch.uint8, device=data.device)
    codes = room[offset:offset + n * (d + extra)].view(n, d + extra)[:, :d]
    codes.copy_(data.float().to(torch.float8_e4m3fn).view(torch.uint8))
    lines = scale if scale_by_rows else scale.t()
    kept = torch.full((lines.shape[0], lines.shape[1] + scale_gap), torch.nan, device=data.device)[:, :lines.shape[1]]
    kept.copy_(lines)
    return fnn.FnnScaled(room.view(torch.float8_e4m3fn)[offset:offset + n * (d + extra)].view(n, d + extra)[:, :d], kept if scale_by_rows else kept.t())


def same(got, want):
    """Equal, NaN where NaN is wanted."""
    return torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))
