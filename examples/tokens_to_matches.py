"""From the tokens of image pairs to matches: a pre-norm transformer block and a matching head made of the library's operators, whose rows
fnn_reciprocal matches; and the gradients of the same, as a training step takes them.

    python examples/tokens_to_matches.py             # one pair of 512x384 images, random weights
    python examples/tokens_to_matches.py --pairs 8 --train

Weights are random (there are no pretrained ones here), so the matches mean nothing; the shapes are those of a 512x384 pair in patches of 16x16
pixels: 768 tokens an image, 24 channels a pixel.
"""
from __future__ import annotations

import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2503_10017_amd as fnn  # noqa: E402

PATCH, CHANNELS = 16, 24


def random_weights(width, dtype, device, seed=0):
    """The weights of one block and of the head, hidden layers four times as wide; matrices [outer][inner]."""
    gen = torch.Generator().manual_seed(seed)

    def matrix(outer, inner):
        return (torch.randn(outer, inner, generator=gen) / math.sqrt(inner)).to(dtype).to(device)

    def vector(n, around=0.0):
        return (around + 0.1 * torch.randn(n, generator=gen)).to(dtype).to(device)

    p = {}
    for name, outer, inner in (("qkv", 3 * width, width), ("proj", width, width), ("up", 4 * width, width), ("down", width, 4 * width),
                               ("head_up", 4 * width, width), ("head_down", PATCH * PATCH * CHANNELS, 4 * width)):
        p[name], p[name + "_b"] = matrix(outer, inner), vector(outer)
    for name in ("norm1", "norm2", "norm3"):
        p[name], p[name + "_b"] = vector(width, 1.0), vector(width)
    return p


def forward(p, x, cu, heads, train=False):
    """x [tokens][width] -> one row of PATCH * PATCH * CHANNELS numbers per token, and with ``train`` what the gradient takes."""
    tokens, width = x.shape
    keep = {"x": x}

    def norm(name, t):
        y, keep[name + ".mean"], keep[name + ".rstd"] = fnn.fnn_layer_norm(t, p[name], p[name + "_b"], want_stats=train)
        keep[name] = y
        return y

    def linear(name, t, **kw):
        y, keep[name + ".pre"] = fnn.fnn_linear(t, p[name], p[name + "_b"], **kw)
        keep[name] = y
        return y

    # queries, keys and values are slices of one product; attention takes them where they are
    qkv = linear("qkv", norm("norm1", x)).view(tokens, 3, heads, width // heads)
    keep["att"], keep["lse"] = fnn.fnn_attention(qkv[:, 0], qkv[:, 1], qkv[:, 2], cu, cu, want_lse=train)
    h = linear("proj", keep["att"].view(tokens, width), residual=x)
    h = linear("down", linear("up", norm("norm2", h), act="gelu", want_pre=train), residual=h)
    return linear("head_down", linear("head_up", norm("norm3", h), act="gelu", want_pre=train)), keep


def backward(p, keep, drows, cu, heads):
    """Gradients of sum(rows * drows) for every weight, and for x."""
    g, x = {}, keep["x"]
    tokens, width = x.shape

    def linear(name, dy, inputs, act="none"):
        dx, g[name], g[name + "_b"] = fnn.fnn_linear_backward(dy, inputs, p[name], keep[name + ".pre"], act=act)
        return dx

    def norm(name, dy, inputs):
        dx, g[name], g[name + "_b"] = fnn.fnn_layer_norm_backward(dy, inputs, keep[name + ".mean"], keep[name + ".rstd"], p[name])
        return dx

    d = linear("head_up", linear("head_down", drows, keep["head_up"]), keep["norm3"], "gelu")
    dh = norm("norm3", d, keep["down"])
    d = linear("up", linear("down", dh, keep["up"]), keep["norm2"], "gelu")
    dh = dh + norm("norm2", d, keep["proj"])
    datt = linear("proj", dh, keep["att"].view(tokens, width)).view(tokens, heads, width // heads)
    qkv, dqkv = (t.view(tokens, 3, heads, width // heads) for t in (keep["qkv"], torch.empty_like(keep["qkv"])))
    fnn.fnn_attention_backward(datt, qkv[:, 0], qkv[:, 1], qkv[:, 2], keep["att"], keep["lse"], cu, cu, out_grads=(dqkv[:, 0], dqkv[:, 1], dqkv[:, 2]))
    d = linear("qkv", dqkv.view(tokens, 3 * width), keep["norm1"])
    return g, dh + norm("norm1", d, x)


def to_maps(rows, images, width, height):
    """Rows of tokens -> descriptor maps [images][pixels][CHANNELS], pixel id y * width + x."""
    across, down = width // PATCH, height // PATCH
    return rows.view(images, down, across, PATCH, PATCH, CHANNELS).permute(0, 1, 3, 2, 4, 5).reshape(images, width * height, CHANNELS)


def match(maps, width, height, stride=8, max_iter=10):
    """Images 2 b and 2 b + 1 are pair b; every stride-th pixel is a seed; the head's raw rows are normalised by the call."""
    device = maps.device
    ys, xs = torch.meshgrid(torch.arange(0, height, stride), torch.arange(0, width, stride), indexing="ij")
    seeds = (ys * width + xs).reshape(1, -1).to(torch.int32).repeat(maps.shape[0] // 2, 1).to(device)
    compute = "bf16" if maps.dtype == torch.bfloat16 else "f16"
    return fnn.fnn_reciprocal(maps[0::2], maps[1::2], seeds, max_iter=max_iter, compute=compute, normalize=True)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--pairs", type=int, default=1)
    ap.add_argument("--width", type=int, default=512, help="of the images, in pixels")
    ap.add_argument("--height", type=int, default=384)
    ap.add_argument("--channels", type=int, default=512, help="of a token")
    ap.add_argument("--dtype", default="bf16", choices=["bf16", "f16"])
    ap.add_argument("--train", action="store_true", help="also the gradients of all weights")
    args = ap.parse_args()
    dtype, heads, images = {"bf16": torch.bfloat16, "f16": torch.float16}[args.dtype], args.channels // 64, 2 * args.pairs
    per_image = (args.width // PATCH) * (args.height // PATCH)
    p = random_weights(args.channels, dtype, "cuda:0")
    x = torch.randn(images * per_image, args.channels, generator=torch.Generator().manual_seed(1)).to(dtype).to("cuda:0")
    cu = torch.arange(0, images + 1, dtype=torch.int32, device="cuda:0") * per_image

    def run():
        rows, keep = forward(p, x, cu, heads, train=args.train)
        found = match(to_maps(rows, images, args.width, args.height), args.width, args.height)
        return found, backward(p, keep, rows, cu, heads) if args.train else None

    run()
    torch.cuda.synchronize()
    began = time.perf_counter()
    found, grads = run()
    torch.cuda.synchronize()
    print(f"{args.pairs} pair(s): {found['n_pairs'].tolist()} matches, {1e3 * (time.perf_counter() - began):.2f} ms"
          + (f", {len(grads[0])} gradients" if grads else ""))


if __name__ == "__main__":
    main()
