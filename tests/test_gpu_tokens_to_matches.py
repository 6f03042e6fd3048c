"""The block and the head of examples/tokens_to_matches.py against the same in fp32 torch with its own gradients, and the maps that they end
in through the matching."""
import importlib.util
import os

import pytest
import torch

import paper_2503_10017_amd as fnn
from net_helpers import DEV

pytestmark = pytest.mark.gpu

spec = importlib.util.spec_from_file_location("tokens_to_matches", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "tokens_to_matches.py"))
example = importlib.util.module_from_spec(spec)
spec.loader.exec_module(example)

WIDTH, HEIGHT, CHANNELS, HEADS, IMAGES = 96, 64, 128, 2, 4


def plain(p, x, lengths, heads):
    def norm(name, t):
        return torch.nn.functional.layer_norm(t, t.shape[1:], p[name], p[name + "_b"], 1e-6)

    def linear(name, t):
        return t @ p[name].t() + p[name + "_b"]

    gelu = torch.nn.functional.gelu
    q, k, v = linear("qkv", norm("norm1", x)).view(len(x), 3, heads, -1).unbind(1)
    parts = []
    for a, b, c in zip(*(t.split(lengths) for t in (q, k, v))):
        w = torch.softmax(torch.matmul(a.transpose(0, 1), b.permute(1, 2, 0)) / a.shape[-1] ** 0.5, -1)
        parts.append(torch.matmul(w, c.transpose(0, 1)).transpose(0, 1).reshape(len(a), -1))
    h = x + linear("proj", torch.cat(parts))
    h = h + linear("down", gelu(linear("up", norm("norm2", h))))
    return linear("head_down", gelu(linear("head_up", norm("norm3", h))))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_rows_gradients_and_matches(dtype):
    per_image = (WIDTH // 16) * (HEIGHT // 16)
    p = example.random_weights(CHANNELS, dtype, DEV)
    x = torch.randn(IMAGES * per_image, CHANNELS, generator=torch.Generator().manual_seed(3)).to(dtype).to(DEV)
    cu = torch.arange(0, IMAGES + 1, dtype=torch.int32, device=DEV) * per_image
    rows, keep = example.forward(p, x, cu, HEADS, train=True)
    assert torch.equal(rows, example.forward(p, x, cu, HEADS)[0])

    wide = {k: v.float().cpu().double().requires_grad_() for k, v in p.items()}
    wide_x = x.float().cpu().double().requires_grad_()
    want = plain(wide, wide_x, [per_image] * IMAGES, HEADS)
    u = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype]

    def off(got, ref):
        return ((got.double().cpu() - ref).norm() / ref.norm()).item()

    # a dozen roundings of independent sign lie between the input and the rows, each of up to u of its own tensor's size: 12 u is far outside
    # what they add up to, and far inside what a wrong term would make
    assert off(rows, want.detach()) < 12 * u
    drows = torch.randn(rows.shape, generator=torch.Generator().manual_seed(4)).to(dtype).to(DEV)
    grads, dx = example.backward(p, keep, drows, cu, HEADS)
    want.backward(drows.double().cpu())
    assert set(grads) == set(p)
    for name, g in [*grads.items(), ("x", dx)]:
        ref = (wide_x if name == "x" else wide[name]).grad
        assert g.shape == ref.shape and g.dtype == dtype
        assert off(g, ref) < 30 * u, name        # twice the way, and what was rounded on the first

    maps = example.to_maps(rows, IMAGES, WIDTH, HEIGHT)
    for y, xx in ((0, 0), (17, 33), (63, 95)):
        token = per_image + (y // 16) * (WIDTH // 16) + xx // 16
        assert torch.equal(maps[1, y * WIDTH + xx], rows[token].view(16, 16, 24)[y % 16, xx % 16])
    found = example.match(maps, WIDTH, HEIGHT)
    again = example.match(maps.clone(), WIDTH, HEIGHT)
    assert all(torch.equal(found[k], again[k]) for k in found)
    # every match is mutual on the same maps
    compute = "bf16" if dtype == torch.bfloat16 else "f16"
    dense = fnn.fnn_mutual_dense(maps[0::2], maps[1::2], compute=compute, normalize=True)
    for b in range(IMAGES // 2):
        n = int(found["n_pairs"][b])
        assert n > 0
        mutual = {tuple(r) for r in dense["pairs"][b, :int(dense["n_pairs"][b])].tolist()}
        inside = sum(tuple(r) in mutual for r in found["pairs"][b, :n].tolist())
        assert inside >= 0.98 * n

