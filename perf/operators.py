"""What the operators of the network before the matcher are timed on: the pre-norm transformer block over image tokens and
the matching head whose rows `fnn_reciprocal` takes -- layer norm, linear layers with their epilogue, attention over packed
sequences, and their gradients.

A 512x384 image in patches of 16x16 pixels is 768 tokens; a call of 16 pairs has 32 such images.  Widths are generic.
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6


def listed():
    return [
        # layer norm: one token, as a step that answers token by token calls it; launches and latency only
        {"name": "norm_token", "op": "norm", "rows": 1, "width": 1024, "type": "f16"},
        # the tokens of 16 image pairs
        {"name": "norm_images", "op": "norm", "rows": 24576, "width": 1024, "type": "bf16"},
        # its gradient in training on the same tokens
        {"name": "norm_train", "op": "norm_back", "rows": 24576, "width": 1024, "type": "bf16"},
        # fine-tuning in fp32 with a width that no vector load divides, ragged rows
        {"name": "norm_train_odd", "op": "norm_back", "rows": 6151, "width": 1021, "type": "f32"},
        # linear: one token through the first layer of a feed-forward block: the weights are read once
        {"name": "linear_token", "op": "linear", "rows": 1, "inner": 1024, "outer": 4096, "type": "bf16", "act": "gelu", "residual": False, "pre": False},
        # the same layer over the tokens of 8 image pairs
        {"name": "linear_images", "op": "linear", "rows": 12288, "inner": 1024, "outer": 4096, "type": "f16", "act": "gelu", "residual": False, "pre": False},
        # a layer that closes a block (residual in the epilogue), two images of 517x389 pixels, odd widths, fp32
        {"name": "linear_odd", "op": "linear", "rows": 1531, "inner": 777, "outer": 1001, "type": "f32", "act": "none", "residual": True, "pre": False},
        # the gradients of the layer above over 8 pairs
        {"name": "linear_train", "op": "linear_back", "rows": 12288, "inner": 1024, "outer": 4096, "type": "bf16", "act": "gelu"},
        # attention: one new token for each of 32 streams over caches of different lengths, four query heads to a key head
        {"name": "attention_step", "op": "attention", "batch": 32, "queries": 1, "keys": 4096, "ragged": True, "heads": 16, "groups": 4, "dim": 128, "type": "bf16", "causal": True},
        # the tokens of 32 images, each over its own image
        {"name": "attention_images", "op": "attention", "batch": 32, "queries": 768, "keys": 768, "ragged": False, "heads": 16, "groups": 16, "dim": 64, "type": "bf16", "causal": False},
        # packed prompts of different lengths, empty and single ones among them
        {"name": "attention_prompts", "op": "attention", "batch": 17, "queries": 4001, "keys": 4001, "ragged": True, "heads": 16, "groups": 8, "dim": 128, "type": "f16", "causal": True},
        # gradients of images packed at different sizes
        {"name": "attention_train", "op": "attention_back", "batch": 12, "queries": 2048, "keys": 2048, "ragged": True, "heads": 12, "groups": 12, "dim": 64, "type": "bf16", "causal": False},
    ]


def _spread(rng, low, high):
    """A whole number between the two, spread over its logarithm."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    return n if n != 3072 else n + 1


def draw(rng):
    op = rng.choice(["norm", "norm_back", "linear", "linear", "linear_back", "attention", "attention", "attention_back"])
    case = {"op": op, "type": rng.choice(["f16", "bf16"])}
    if op in ("norm", "norm_back"):
        rows, width = _spread(rng, 1, 24576), _spread(rng, 64, 4096)
        width = width if rng.random() < 0.3 else max(64, width // 64 * 64)
        if rng.random() < 0.25:
            case["type"] = "f32"
        return {**case, "rows": max(1, min(rows, 24576 * 1024 // width)), "width": width}
    if op in ("linear", "linear_back"):
        rows, inner, outer = _spread(rng, 1, 12288), _spread(rng, 64, 4096), _spread(rng, 64, 4096)
        if rng.random() < 0.7:
            inner, outer = max(64, inner // 64 * 64), max(64, outer // 64 * 64)
        case |= {"rows": max(1, min(rows, 12288 * 4096 * 1024 // (inner * outer))), "inner": inner, "outer": outer, "act": rng.choice(["none", "relu", "gelu", "silu"])}
        if rng.random() < 0.15:
            case |= {"type": "f32", "rows": max(1, case["rows"] // 8)}
        return case if op == "linear_back" else {**case, "residual": rng.random() < 0.5, "pre": rng.random() < 0.3}
    dim = rng.choice([64, 64, 128, 128, 32, 80, 96])
    groups = rng.choice([1, 2, 4, 8, 12, 16])
    heads = groups * rng.choice([1, 1, 2, 4] if groups <= 4 else [1, 2])
    batch, keys = _spread(rng, 1, 32), _spread(rng, 16, 4096)
    keys = max(16, min(keys, int(math.sqrt((4e8 if op == "attention" else 1e8) / (batch * heads)))))
    queries = rng.choice([1, rng.randint(2, 16)]) if op == "attention" and rng.random() < 0.35 else keys
    return {**case, "batch": batch, "queries": queries, "keys": keys, "ragged": rng.random() < 0.7, "heads": heads, "groups": groups, "dim": dim, "causal": rng.random() < 0.5}


def _lengths(case):
    """Queries and keys of each sequence: the case's, or lengths up to them with an empty one, one of one token and one of the full length
    among three and more.  Where the queries are as many as the keys, each sequence has as many of both."""
    batch, queries, keys = case["batch"], case["queries"], case["keys"]
    if not case["ragged"]:
        return [queries] * batch, [keys] * batch
    rng = random.Random(batch * 1000003 + keys * 101 + queries)
    of_keys = [max(1, int(keys * rng.uniform(0.05, 1.0))) for _ in range(batch)]
    of_keys[0] = keys
    if batch > 2:
        of_keys[1], of_keys[2] = 1, 0
        rng.shuffle(of_keys)
    return (of_keys, of_keys) if queries == keys else ([queries] * batch, of_keys)


def _visible(lengths, causal):
    pairs = 0
    for lq, lk in zip(*lengths):
        if not causal:
            pairs += lq * lk
        else:
            first = max(1, lk - lq + 1)  # what the first row that sees anything sees
            pairs += (first + lk) * (lk - first + 1) // 2
    return pairs


def work(case):
    op, es = case["op"], SIZE[case["type"]]
    if op in ("norm", "norm_back"):
        n, w = case["rows"], case["width"]
        if op == "norm":
            return {"bytes": es * (2 * n * w + 2 * w) + 8 * n, "flops": 8 * n * w}
        return {"bytes": es * (3 * n * w + 3 * w) + 8 * n, "flops": 14 * n * w}
    if op in ("linear", "linear_back"):
        m, k, n = case["rows"], case["inner"], case["outer"]
        if op == "linear":
            return {"bytes": es * (m * k + n * k + n + m * n * (1 + case["residual"] + case["pre"])), "flops": 2 * m * n * k}
        return {"bytes": es * (m * n * (1 if case["act"] == "none" else 2) + 2 * m * k + 2 * n * k + n), "flops": 4 * m * n * k}
    lengths = _lengths(case)
    tq, tk = sum(lengths[0]), sum(lengths[1])
    rows, keys = tq * case["heads"] * case["dim"], tk * case["groups"] * case["dim"]
    pairs = _visible(lengths, case["causal"]) * case["heads"]
    if op == "attention":
        return {"bytes": es * (2 * rows + 2 * keys) + 4 * tq * case["heads"], "flops": 4 * pairs * case["dim"]}
    return {"bytes": es * (4 * rows + 4 * keys) + 4 * tq * case["heads"], "flops": 10 * pairs * case["dim"]}


def prepare(case, seed):
    device = "cuda" if torch.cuda.is_available() else "cpu"
    gen = torch.Generator(device=device).manual_seed(seed)
    kind, op = TYPES[case["type"]], case["op"]

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device=device) * std

    state = {"case": dict(case)}
    if op in ("norm", "norm_back"):
        n, w = case["rows"], case["width"]
        # activations of a trained block: channels of different spread, a few far larger than the rest, off zero
        spread = torch.exp(normal(w, std=0.5))
        spread[torch.randint(0, w, (max(1, w // 200),), generator=gen, device=device)] *= 20
        x = normal(n, w) * spread + normal(w, std=0.3)
        state["x"], state["weight"] = x.to(kind), (1 + normal(w, std=0.1)).to(kind)
        if op == "norm":
            state["bias"] = normal(w, std=0.1).to(kind)
        else:
            state["dy"] = normal(n, w).to(kind)
            x = state["x"].float()
            state["mean"] = x.mean(1)
            state["rstd"] = torch.rsqrt((x - state["mean"][:, None]).square().mean(1) + EPS)
        return state
    if op in ("linear", "linear_back"):
        m, k, n = case["rows"], case["inner"], case["outer"]
        state["x"], state["weight"] = normal(m, k).to(kind), normal(n, k, std=1 / math.sqrt(k)).to(kind)
        bias = normal(n, std=0.1).to(kind)
        if op == "linear":
            state["bias"], state["residual"] = bias, normal(m, n).to(kind) if case["residual"] else None
        else:
            state["dy"] = normal(m, n).to(kind)
            state["pre"] = None if case["act"] == "none" else (state["x"].float() @ state["weight"].float().t() + bias.float()).to(kind)
        return state
    lq, lk = _lengths(case)
    heads, groups, dim = case["heads"], case["groups"], case["dim"]
    state["q"] = normal(sum(lq), heads, dim).to(kind)
    state["k"], state["v"] = normal(sum(lk), groups, dim).to(kind), normal(sum(lk), groups, dim).to(kind)
    state["cu_q"] = torch.tensor([0, *torch.tensor(lq).cumsum(0).tolist()], dtype=torch.int32, device=device)
    state["cu_k"] = torch.tensor([0, *torch.tensor(lk).cumsum(0).tolist()], dtype=torch.int32, device=device)
    state["scale"], state["longest"] = 1 / math.sqrt(dim), (max(lq), max(lk))
    if op == "attention_back":
        state["out"], state["lse"] = _attention(state)
        state["dout"] = normal(sum(lq), heads, dim).to(kind)
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


def _padded(t, cu, longest):
    """[tokens][heads][dim] packed -> fp32 [batch][heads][longest][dim], and which of its tokens there are."""
    at = cu[:-1, None].long() + torch.arange(longest, device=t.device)
    there = at < cu[1:, None]
    rows = t.float()[at.clamp(max=max(0, t.shape[0] - 1))] * there[:, :, None, None]
    return rows.permute(0, 2, 1, 3).contiguous(), there


def _packed(t, there, kind):
    return t.permute(0, 2, 1, 3)[there].to(kind).contiguous()


def _scores(s):
    """Padded q, k, v (key heads repeated), the masked scores, and which rows and keys there are."""
    c = s["case"]
    q, there_q = _padded(s["q"], s["cu_q"], s["longest"][0])
    k, there_k = _padded(s["k"], s["cu_k"], s["longest"][1])
    v, _ = _padded(s["v"], s["cu_k"], s["longest"][1])
    share = c["heads"] // c["groups"]
    k, v = k.repeat_interleave(share, 1), v.repeat_interleave(share, 1)
    score = torch.matmul(q, k.transpose(2, 3).contiguous()) * s["scale"]
    seen = (there_q[:, :, None] & there_k[:, None, :])[:, None]
    if c["causal"]:
        more = (s["cu_k"][1:] - s["cu_k"][:-1]) - (s["cu_q"][1:] - s["cu_q"][:-1])
        i, j = (torch.arange(n, device=q.device) for n in s["longest"])
        seen = seen & (j[None, None, :] <= i[None, :, None] + more[:, None, None])[:, None]
    return q, k, v, score.masked_fill_(~seen, -math.inf), there_q, there_k


def _attention(s):
    q, k, v, score, there, _ = _scores(s)
    top = score.amax(-1, keepdim=True).clamp(min=-3e38)
    e = score.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    out = torch.matmul(e, v) / total.clamp(min=1e-38)
    lse = (top + total.log())[..., 0]
    return _packed(out, there, s["q"].dtype), lse.permute(0, 2, 1)[there].contiguous()


def _attention_back(s):
    c = s["case"]
    q, k, v, score, there_q, there_k = _scores(s)
    dout, _ = _padded(s["dout"], s["cu_q"], s["longest"][0])
    out, _ = _padded(s["out"], s["cu_q"], s["longest"][0])
    lse, _ = _padded(s["lse"][..., None], s["cu_q"], s["longest"][0])
    p = score.sub_(lse.clamp(min=-3e38)).exp_()
    dv = torch.matmul(p.transpose(2, 3), dout)
    ds = (torch.matmul(dout, v.transpose(2, 3).contiguous()) - (dout * out).sum(-1, keepdim=True)) * p * s["scale"]
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3), q)
    b, _, longest, dim = dk.shape
    dk, dv = (t.view(b, c["groups"], -1, longest, dim).sum(2) for t in (dk, dv))
    kind = s["q"].dtype
    return _packed(dq, there_q, kind), _packed(dk, there_k, kind), _packed(dv, there_k, kind)


def _plain(s):
    c, op = s["case"], s["case"]["op"]
    if op == "norm":
        x = s["x"].float()
        mean = x.mean(1, keepdim=True)
        rstd = torch.rsqrt((x - mean).square().mean(1, keepdim=True) + EPS)
        y = (x - mean) * rstd * s["weight"].float() + s["bias"].float()
        return {"y": y.to(s["x"].dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if op == "norm_back":
        kind, x, dy = s["x"].dtype, s["x"].float(), s["dy"].float()
        h = (x - s["mean"][:, None]) * s["rstd"][:, None]
        g = dy * s["weight"].float()
        dx = (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True)) * s["rstd"][:, None]
        return {"dx": dx.to(kind), "dweight": (dy * h).sum(0).to(kind), "dbias": dy.sum(0).to(kind)}
    if op == "linear":
        kind = s["x"].dtype
        pre = torch.matmul(s["x"].float(), s["weight"].float().t()) + s["bias"].float()
        y = _act(pre, c["act"])
        if c["residual"]:
            y = y + s["residual"].float()
        return {"y": y.to(kind), "pre": pre.to(kind)} if c["pre"] else {"y": y.to(kind)}
    if op == "linear_back":
        kind, p = s["x"].dtype, s["dy"].float()
        if c["act"] != "none":
            p = p * _act_slope(s["pre"].float(), c["act"])
        return {"dx": torch.matmul(p, s["weight"].float()).to(kind), "dweight": torch.matmul(p.t(), s["x"].float()).to(kind), "dbias": p.sum(0).to(kind)}
    if op == "attention":
        out, lse = _attention(s)
        return {"out": out, "lse": lse}
    dq, dk, dv = _attention_back(s)
    return {"dq": dq, "dk": dk, "dv": dv}


# ---- the framework's ----

def _framework(s):
    import paper_2503_10017_amd as fnn

    c, op = s["case"], s["case"]["op"]
    if op == "norm":
        y, mean, rstd = fnn.fnn_layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, want_stats=True)
        return {"y": y, "mean": mean, "rstd": rstd}
    if op == "norm_back":
        dx, dweight, dbias = fnn.fnn_layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["weight"])
        return {"dx": dx, "dweight": dweight, "dbias": dbias}
    if op == "linear":
        y, pre = fnn.fnn_linear(s["x"], s["weight"], s["bias"], s["residual"], act=c["act"], want_pre=c["pre"])
        return {"y": y, "pre": pre} if c["pre"] else {"y": y}
    if op == "linear_back":
        dx, dweight, dbias = fnn.fnn_linear_backward(s["dy"], s["x"], s["weight"], s["pre"], act=c["act"])
        return {"dx": dx, "dweight": dweight, "dbias": dbias}
    if op == "attention":
        out, lse = fnn.fnn_attention(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], causal=c["causal"], scale=s["scale"])
        return {"out": out, "lse": lse}
    dq, dk, dv = fnn.fnn_attention_backward(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["cu_q"], s["cu_k"],
                                            causal=c["causal"], scale=s["scale"])
    return {"dq": dq, "dk": dk, "dv": dv}


def run(state):
    return _framework(state) if own else _plain(state)


# ---- the definitions in 64 bits ----

def _phi(x):
    return torch.special.erfc(-x / math.sqrt(2)) / 2


def _exact_sequence(q, k, v, scale, causal, dout=None):
    """One sequence: q [heads][rows][dim], k and v [groups][keys][dim]; out and lse, or the three gradients."""
    heads, rows, _ = q.shape
    groups, keys, _ = k.shape
    out, lse = torch.zeros_like(q), torch.full((heads, rows), -math.inf, dtype=q.dtype, device=q.device)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for h in range(heads if keys and rows else 0):
        g = h // (heads // groups)
        z = scale * (q[h] @ k[g].t())
        if causal:
            z = z + torch.full_like(z, -math.inf).triu(1 + keys - rows)
        lse[h] = torch.logsumexp(z, 1)
        p = torch.where(lse[h][:, None] > -math.inf, torch.exp(z - lse[h][:, None]), torch.zeros_like(z)).nan_to_num(0.0)
        out[h] = p @ v[g]
        if dout is not None:
            dp = dout[h] @ v[g].t()
            ds = scale * p * (dp - (p * dp).sum(1, keepdim=True))
            dq[h] = ds @ k[g]
            dk[g] += ds.t() @ q[h]
            dv[g] += p.t() @ dout[h]
    return (out, lse) if dout is None else (dq, dk, dv)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if op == "norm":
        x = wide["x"]
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + EPS) ** -0.5
        return {"y": torch.addcmul(wide["bias"], (x - mean[:, None]) * rstd[:, None], wide["weight"]), "mean": mean, "rstd": rstd}
    if op == "norm_back":
        x, dy, n = wide["x"], wide["dy"], case["width"]
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + EPS)[:, None] ** -0.5
        h, g = (x - mean[:, None]) * rstd, dy * wide["weight"]
        dx = rstd / n * (n * g - g.sum(1, keepdim=True) - h * (g * h).sum(1, keepdim=True))
        return {"dx": dx, "dweight": torch.einsum("rw,rw->w", dy, h), "dbias": torch.ones(len(dy), dtype=dy.dtype, device=dy.device) @ dy}
    if op in ("linear", "linear_back"):
        act = case["act"]
        pre = torch.addmm(wide["bias"], wide["x"], wide["weight"].t()) if op == "linear" else wide.get("pre")
        if op == "linear":
            y = {"none": lambda: pre, "relu": lambda: pre * (pre > 0), "gelu": lambda: pre * _phi(pre), "silu": lambda: pre / (1 + torch.exp(-pre))}[act]()
            y = y + wide["residual"] if case["residual"] else y
            return {"y": y, "pre": pre} if case["pre"] else {"y": y}
        p = wide["dy"]
        if act == "relu":
            p = torch.where(pre > 0, p, 0.0)
        elif act == "gelu":
            p = p * (_phi(pre) + pre * torch.exp(-pre ** 2 / 2) / math.sqrt(2 * math.pi))
        elif act == "silu":
            e = 1 + torch.exp(-pre)
            p = p * (1 / e + pre * torch.exp(-pre) / e ** 2)
        return {"dx": p @ wide["weight"], "dweight": p.t() @ wide["x"], "dbias": p.sum(0)}
    parts = []
    cu_q, cu_k = s["cu_q"].tolist(), s["cu_k"].tolist()
    for b in range(case["batch"]):
        rows, keys = slice(cu_q[b], cu_q[b + 1]), slice(cu_k[b], cu_k[b + 1])
        q, k, v = (wide[x][y].transpose(0, 1).contiguous() for x, y in (("q", rows), ("k", keys), ("v", keys)))
        dout = wide["dout"][rows].transpose(0, 1).contiguous() if op == "attention_back" else None
        parts.append([t.transpose(0, 1) for t in _exact_sequence(q, k, v, s["scale"], case["causal"], dout)])
    names = ("out", "lse") if op == "attention" else ("dq", "dk", "dv")
    return {name: torch.cat([p[i] for p in parts]).contiguous() for i, name in enumerate(names)}
