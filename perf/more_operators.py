"""What the 8-bit operators of the network before the matcher are timed on: the root-mean-square norm with the residual's addition, whose
result leaves in 8 bits with a scale for each block of 128, its gradient, the quantising of whole matrices (by rows, by tiles and across), the linear layer over
such operands, and that layer's gradient.

A 512x384 image in patches of 16x16 pixels is 768 tokens; a call of 16 pairs has 32 such images.  Widths are generic; the head's layer is
4096 -> 16 * 16 pixels of 24 channels.  8 bits are e4m3: 4 bits of exponent, 3 of mantissa, values up to 448.
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6
BLOCK = 128


def listed():
    return [
        # one token of a step that answers token by token: the residual stream is updated, the norm leaves in 8 bits; launches and latency only
        {"name": "norm_token", "op": "norm", "rows": 1, "width": 1024, "type": "bf16", "residual": True, "train": False},
        # the tokens of 16 image pairs
        {"name": "norm_images", "op": "norm", "rows": 24576, "width": 1024, "type": "bf16", "residual": True, "train": False},
        # its gradient in training on the same tokens, joined with what comes down the residual stream
        {"name": "norm_train", "op": "norm_back", "rows": 24576, "width": 1024, "type": "bf16", "residual": True},
        # fine-tuning in fp32 with a width that no vector load divides, ragged rows, no residual
        {"name": "norm_train_odd", "op": "norm_back", "rows": 6151, "width": 1021, "type": "f32", "residual": False},
        # the hidden activations of 16 image pairs before a layer in 8 bits
        {"name": "quantize_rows", "op": "quantize", "rows": 24576, "width": 4096, "type": "bf16", "tiles": False, "across": False},
        # the same kind of matrix as the weights' gradient takes it, with blocks that run over the tokens; odd everything
        {"name": "quantize_across", "op": "quantize", "rows": 12289, "width": 1021, "type": "f16", "tiles": False, "across": True},
        # one token through the first layer of a feed-forward block: the weights are read once
        {"name": "linear_token", "op": "linear", "rows": 1, "inner": 1024, "outer": 4096, "type": "bf16", "act": "gelu", "residual": False, "pre": False, "tight": False},
        # a layer that closes a block (residual in the epilogue), two images of 517x389 pixels, odd widths, fp32 results
        {"name": "linear_odd", "op": "linear", "rows": 1531, "inner": 777, "outer": 1001, "type": "f32", "act": "none", "residual": True, "pre": False, "tight": False},
        # the first layer of a feed-forward block over the tokens of 16 image pairs
        {"name": "linear_images", "op": "linear", "rows": 24576, "inner": 1024, "outer": 4096, "type": "bf16", "act": "gelu", "residual": False, "pre": False, "tight": False},
        # the last layer of the matching head over the same tokens
        {"name": "linear_head", "op": "linear", "rows": 24576, "inner": 4096, "outer": 6144, "type": "bf16", "act": "none", "residual": False, "pre": False, "tight": False},
        # the gradients of the first layer of a feed-forward block over the tokens of 8 image pairs
        {"name": "linear_train", "op": "linear_back", "rows": 12288, "inner": 1024, "outer": 4096, "type": "bf16", "act": "gelu"},
        # those of odd widths and ragged rows
        {"name": "linear_train_odd", "op": "linear_back", "rows": 1531, "inner": 777, "outer": 1001, "type": "f16", "act": "silu"},
    ]


def _spread(rng, low, high):
    """A whole number between the two, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["norm", "norm_back", "quantize", "quantize", "linear", "linear", "linear", "linear_back", "linear_back"])
    case = {"op": op, "type": rng.choice(["f16", "bf16"])}
    if op in ("norm", "norm_back", "quantize"):
        rows, width = _spread(rng, 1, 24576), _spread(rng, 64, 4096)
        width = width if rng.random() < 0.3 else max(64, width // 64 * 64)
        if rng.random() < 0.25:
            case["type"] = "f32"
        case |= {"rows": max(1, min(rows, 24576 * 1024 // width)), "width": width}
        if op == "quantize":
            return {**case, "tiles": rng.random() < 0.4, "across": rng.random() < 0.4}
        case["residual"] = rng.random() < 0.6
        return case if op == "norm_back" else {**case, "train": rng.random() < 0.4}
    rows, inner, outer = _spread(rng, 1, 24576), _spread(rng, 64, 8192), _spread(rng, 64, 8192)
    if rng.random() < 0.7:
        inner, outer = max(64, inner // 64 * 64), max(64, outer // 64 * 64)
    most = 24576 * 4096 * 6144 if op == "linear" else 12288 * 1024 * 4096
    case |= {"rows": max(1, min(rows, most // (inner * outer))), "inner": inner, "outer": outer, "act": rng.choice(["none", "relu", "gelu", "silu"])}
    if op == "linear_back":
        return case
    if rng.random() < 0.2:
        case["type"] = "f32"
    # tight: rows of codes end to end, as another program may hand them over
    return {**case, "residual": rng.random() < 0.5, "pre": rng.random() < 0.3, "tight": rng.random() < 0.2}


def _blocks(n):
    return -(-n // BLOCK)


def work(case):
    op, es = case["op"], SIZE[case["type"]]
    if op in ("norm", "norm_back"):
        n, w = case["rows"], case["width"]
        if op == "norm":
            more = (es * n * w + 4 * n) * case["train"] + 2 * es * n * w * case["residual"]
            return {"bytes": es * (n * w + w) + n * w + 4 * n * _blocks(w) + more, "flops": 8 * n * w}
        return {"bytes": es * ((3 + case["residual"]) * n * w + 2 * w) + 4 * n, "flops": 10 * n * w}
    if op == "quantize":
        n, w = case["rows"], case["width"]
        if case["across"]:
            n, w = w, n
        return {"bytes": (es + 1) * n * w + 4 * _blocks(w) * (_blocks(n) if case["tiles"] else n), "flops": 4 * n * w}
    m, k, n = case["rows"], case["inner"], case["outer"]
    if op == "linear":
        scales = 4 * _blocks(k) * (m + _blocks(n))
        return {"bytes": m * k + n * k + scales + es * (n + m * n * (1 + case["residual"] + case["pre"])), "flops": 2 * m * n * k}
    return {"bytes": es * (m * n * (1 if case["act"] == "none" else 2) + 2 * m * k + n * k + n) + n * k + 4 * _blocks(k) * _blocks(n), "flops": 4 * m * n * k}


# ---- 8 bits with scales, in the plain form ----

def _block_scale(v, tiles):
    """v fp32 [n][d] -> the scales of its blocks [n or tiles of 128][blocks of 128]: the largest magnitude becomes 448."""
    n, d = v.shape
    high = BLOCK if tiles else 1
    v = torch.nn.functional.pad(v.abs(), (0, -d % BLOCK, 0, -n % high))
    top = v.view(v.shape[0] // high, high, -1, BLOCK).amax((1, 3))
    return (top / torch.full_like(top, 448)).clamp(min=2.0 ** -126)  # by a number alone torch multiplies with a rounded reciprocal


def _spread_scale(scale, n, d):
    """One scale for every element."""
    if scale.shape[0] != n:
        scale = scale.repeat_interleave(BLOCK, 0)[:n]
    return scale.repeat_interleave(BLOCK, 1)[:, :d]


def _quantized(v, tiles=False):
    """v fp32 [n][d] -> codes [n][d] and scales."""
    scale = _block_scale(v, tiles)
    return (v / _spread_scale(scale, *v.shape)).to(torch.float8_e4m3fn), scale


def _values(data, scale):
    return data.float() * _spread_scale(scale, *data.shape)


def _kept(data, scale, tight):
    """As the framework's quantising leaves them: rows of codes on 16-byte boundaries unless `tight`, scales of one block of columns next to each other."""
    n, d = data.shape
    if not tight:
        room = torch.zeros((n, -(-d // 16) * 16), dtype=torch.uint8, device=data.device)
        room[:, :d] = data.view(torch.uint8)
        data = room.view(torch.float8_e4m3fn)[:, :d]
    return data, scale.t().contiguous().t()


def prepare(case, seed):
    device = "cuda" if torch.cuda.is_available() else "cpu"
    gen = torch.Generator(device=device).manual_seed(seed)
    kind, op = TYPES[case["type"]], case["op"]

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device=device) * std

    def activations(n, w):
        # of a trained block: channels of different spread, a few far larger than the rest, off zero
        spread = torch.exp(normal(w, std=0.5))
        spread[torch.randint(0, w, (max(1, w // 200),), generator=gen, device=device)] *= 20
        return normal(n, w) * spread + normal(w, std=0.3)

    state = {"case": dict(case)}
    if op in ("norm", "norm_back"):
        n, w = case["rows"], case["width"]
        state["x"], state["weight"] = activations(n, w).to(kind), (1 + normal(w, std=0.1)).to(kind)
        if op == "norm":
            state["residual"] = activations(n, w).to(kind) if case["residual"] else None
        else:
            state["dy"] = normal(n, w).to(kind)
            state["dsum"] = normal(n, w).to(kind) if case["residual"] else None
            state["rstd"] = torch.rsqrt(state["x"].float().square().mean(1) + EPS)
        return state
    if op == "quantize":
        state["x"] = activations(case["rows"], case["width"]).to(kind)
        return state
    m, k, n = case["rows"], case["inner"], case["outer"]
    x, w, bias = activations(m, k), normal(n, k, std=1 / math.sqrt(k)), normal(n, std=0.1).to(kind)
    tight = case.get("tight", False)
    state["w"] = _kept(*_quantized(w, tiles=True), tight)
    if op == "linear":
        state["x"], state["bias"] = _kept(*_quantized(x), tight), bias
        state["residual"] = normal(m, n).to(kind) if case["residual"] else None
    else:
        state["x"], state["dy"] = x.to(kind), normal(m, n, std=1e-3).to(kind)
        state["pre"] = None if case["act"] == "none" else (torch.matmul(x, w.t()) + bias.float()).to(kind)
    return state


# ---- the plain forms ----

def _act(pre, act):
    if act == "relu":
        return pre.clamp(min=0)
    if act == "gelu":
        return 0.5 * pre * (1 + torch.erf(pre * math.sqrt(0.5)))
    if act == "silu":
        return pre * torch.sigmoid(pre)
    return pre


def _act_slope(pre, act):
    if act == "relu":
        return (pre > 0).to(pre.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(pre * math.sqrt(0.5))) + pre * torch.exp(-0.5 * pre * pre) * (1 / math.sqrt(2 * math.pi))
    s = torch.sigmoid(pre)
    return s * (1 + pre * (1 - s))


def _plain(s):
    c, op = s["case"], s["case"]["op"]
    if op == "norm":
        kind, v = s["x"].dtype, s["x"].float()
        got = {}
        if c["residual"]:
            v = v + s["residual"].float()
            got["sum"] = v.to(kind)
        rstd = torch.rsqrt(v.square().mean(1, keepdim=True) + EPS)
        y = v * rstd * s["weight"].float()
        got["data"], got["scale"] = _quantized(y)
        return got | {"y": y.to(kind), "rstd": rstd[:, 0]} if c["train"] else got
    if op == "norm_back":
        kind, dy, rstd = s["x"].dtype, s["dy"].float(), s["rstd"][:, None]
        h, g = s["x"].float() * rstd, dy * s["weight"].float()
        dx = (g - h * (g * h).mean(1, keepdim=True)) * rstd
        if c["residual"]:
            dx = dx + s["dsum"].float()
        return {"dx": dx.to(kind), "dweight": (dy * h).sum(0).to(kind)}
    if op == "quantize":
        v = s["x"].float()
        data, scale = _quantized(v.t().contiguous() if c["across"] else v, c["tiles"])
        return {"data": data, "scale": scale}
    if op == "linear":
        kind = TYPES[c["type"]]
        pre = torch.matmul(_values(*s["x"]), _values(*s["w"]).t()) + s["bias"].float()
        y = _act(pre, c["act"])
        if c["residual"]:
            y = y + s["residual"].float()
        return {"y": y.to(kind), "pre": pre.to(kind)} if c["pre"] else {"y": y.to(kind)}
    kind, q = s["x"].dtype, s["dy"].float()
    if c["act"] != "none":
        q = q * _act_slope(s["pre"].float(), c["act"])
    dx = torch.matmul(_values(*_quantized(q)), _values(*s["w"]))
    q_t, x_t = (_values(*_quantized(t.t().contiguous())) for t in (q, s["x"].float()))
    return {"dx": dx.to(kind), "dweight": torch.matmul(q_t, x_t.t()).to(kind), "dbias": q.sum(0).to(kind)}


# ---- the framework's ----

def _framework(s):
    import paper_2503_10017_amd as fnn

    c, op = s["case"], s["case"]["op"]
    if op == "norm":
        y, scaled, total, rstd = fnn.fnn_rms_norm(s["x"], s["weight"], s["residual"], eps=EPS, want_y=c["train"], want_scaled=True, want_rstd=c["train"])
        got = {"data": scaled.data, "scale": scaled.scale}
        if c["residual"]:
            got["sum"] = total
        return got | {"y": y, "rstd": rstd} if c["train"] else got
    if op == "norm_back":
        dx, dweight = fnn.fnn_rms_norm_backward(s["dy"], s["x"], s["rstd"], s["weight"], s["dsum"])
        return {"dx": dx, "dweight": dweight}
    if op == "quantize":
        scaled = fnn.fnn_quantize(s["x"], tiles=c["tiles"], transposed=c["across"])
        return {"data": scaled.data, "scale": scaled.scale}
    w = fnn.FnnScaled(*s["w"])
    if op == "linear":
        y, pre = fnn.fnn_linear_e4m3(fnn.FnnScaled(*s["x"]), w, s["bias"], s["residual"], act=c["act"], dtype=TYPES[c["type"]], want_pre=c["pre"])
        return {"y": y, "pre": pre} if c["pre"] else {"y": y}
    dx, dweight, dbias = fnn.fnn_linear_e4m3_backward(s["dy"], s["x"], w, s["pre"], act=c["act"])
    return {"dx": dx, "dweight": dweight, "dbias": dbias}


def run(state):
    return _framework(state) if own else _plain(state)


# ---- the definitions in 64 bits ----

def _nearest_e4m3(v):
    """The nearest e4m3 value of numbers up to 448 in 64 bits, halves to the even one: steps of an eighth of the power of two below, of 2^-9 under 2^-6."""
    _, exponent = torch.frexp(v)
    step = (((exponent - 1).clamp(min=-6).long() + (1023 - 3)) << 52).view(torch.float64)  # ldexp and pow are a little off on a GPU
    return torch.round(v / step) * step


def _exact_blocks(v, tiles=False):
    """Values of the codes and the scales of v [n][d], block by block of columns.  That a scale is a number of fp32, and that a quotient by it is rounded to fp32 before it
    is to e4m3, belongs to the definition: inputs of few digits lie on the border of two codes often."""
    n, d = v.shape
    data, scales = [], []
    for first in range(0, d, BLOCK):
        part = v[:, first:first + BLOCK]
        top = part.abs().amax(1)
        if tiles:
            top = torch.stack([t.amax() for t in top.split(BLOCK)])
        scale = torch.maximum(top / 448, torch.full_like(top, 2.0 ** -126)).float().double()
        scales.append(scale)
        each = scale.repeat_interleave(BLOCK)[:n] if tiles else scale
        data.append(_nearest_e4m3((part / each[:, None]).float().double().clamp(-448, 448)))
    return torch.cat(data, 1), torch.stack(scales, 1)


def _exact_values(data, scale):
    n, d = data.shape
    at = torch.arange(n, device=data.device) // (1 if scale.shape[0] == n else BLOCK)
    return data.double() * scale.double()[at][:, torch.arange(d, device=data.device) // BLOCK]


def _phi(x):
    return torch.special.erfc(-x / math.sqrt(2)) / 2


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    if op == "norm":
        got, v = {}, wide["x"]
        if case["residual"]:
            v = got["sum"] = v + wide["residual"]
        rstd = ((v * v).sum(1) / case["width"] + EPS) ** -0.5
        y = torch.einsum("rw,r,w->rw", v, rstd, wide["weight"])
        got["data"], got["scale"] = _exact_blocks(y)
        return got | {"y": y, "rstd": rstd} if case["train"] else got
    if op == "norm_back":
        x, dy, w, n = wide["x"], wide["dy"], wide["weight"], case["width"]
        rstd = ((x * x).sum(1) / n + EPS) ** -0.5
        along = torch.einsum("rw,rw,w->r", dy, x, w)
        dx = rstd[:, None] * dy * w - (rstd ** 3 * along / n)[:, None] * x
        return {"dx": dx + wide["dsum"] if case["residual"] else dx, "dweight": torch.einsum("rw,rw,r->w", dy, x, rstd)}
    if op == "quantize":
        data, scale = _exact_blocks(wide["x"].t() if case["across"] else wide["x"], case["tiles"])
        return {"data": data, "scale": scale}
    act, w = case["act"], _exact_values(*s["w"])
    if op == "linear":
        pre = torch.addmm(wide["bias"], _exact_values(*s["x"]), w.t())
        y = {"none": lambda: pre, "relu": lambda: pre * (pre > 0), "gelu": lambda: pre * _phi(pre), "silu": lambda: pre / (1 + torch.exp(-pre))}[act]()
        y = y + wide["residual"] if case["residual"] else y
        return {"y": y, "pre": pre} if case["pre"] else {"y": y}
    q, pre = wide["dy"], wide.get("pre")
    if act == "relu":
        q = torch.where(pre > 0, q, 0.0)
    elif act == "gelu":
        q = q * (_phi(pre) + pre * torch.exp(-pre ** 2 / 2) / math.sqrt(2 * math.pi))
    elif act == "silu":
        e = 1 + torch.exp(-pre)
        q = q * (1 / e + pre * torch.exp(-pre) / e ** 2)
    dx = _exact_values(*_exact_blocks(q)) @ w
    dweight = _exact_values(*_exact_blocks(q.t())) @ _exact_values(*_exact_blocks(wide["x"].t())).t()
    return {"dx": dx, "dweight": dweight, "dbias": q.sum(0)}
