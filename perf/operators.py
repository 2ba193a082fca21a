"""The operators of the 8-bit path: what they compute, in plain torch and through the framework's calls.

An 8-bit tensor here is a float8_e4m3fn tensor with fp32 scales: activations have one scale for each row and
128 consecutive columns, weights one for each block of 128 x 128.  The value of an element is q * scale.  Quantising takes
scale = a / 448 and q = v * 448 / a, rounded to the nearest, with a the group's largest magnitude; the product
comes first, so that quotients of short numbers that lie half way between two 8-bit values do so in any precision.
A pass is one call of a public entry point on tensors that are already on the GPU; buffers for the
results, the weights and the layer object are made beforehand, as a serving program keeps them.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128
TOP = 448.0   # the largest e4m3 value

QWEN3 = dict(hidden=2048, inter=768, n_experts=128, top_k=8, n_local=128, n_shared=0, max_tokens=8192)
DSV3 = dict(hidden=7168, inter=2048, n_experts=256, top_k=8, n_local=32, n_shared=1, max_tokens=8192)
DSV2 = dict(hidden=2048, inter=1408, n_experts=64, top_k=6, n_local=64, n_shared=2, max_tokens=8192)


def listed():
    return [
        # the norm in front of a DeepSeek-V3-shaped layer: one decoded token, everything the layer behind it reads
        dict(name="norm_token", op="norm", rows=1, cols=7168, dtype="bf16", residual=True, plain_out=True, quantized=True),
        # the same at prefill size
        dict(name="norm_prefill", op="norm", rows=8192, cols=7168, dtype="bf16", residual=True, plain_out=True, quantized=True),
        # activations of a mixed decode batch, quantised by themselves, in the width of a Qwen3-30B-A3B-shaped layer
        dict(name="quantize_rows", op="quantize", rows=333, cols=2048, dtype="bf16", block_rows=1),
        # an expert's first matrix on its way into an 8-bit pool
        dict(name="quantize_weights", op="quantize", rows=4096, cols=7168, dtype="bf16", block_rows=128),
        # down projection of a dense expert for one token, added to the residual stream
        dict(name="matmul_token", op="matmul", m=1, n=7168, k=2048, out="bf16", add=True),
        # a projection of sizes that are whole blocks nowhere, fp32 result
        dict(name="matmul_ragged", op="matmul", m=333, n=1544, k=1424, out="f32", add=False),
        # down projection at prefill size
        dict(name="matmul_prefill", op="matmul", m=8192, n=7168, k=2048, out="bf16", add=True),
        # first half of a dense expert for a small decode batch, DeepSeek-V2-Lite-shaped
        dict(name="swiglu_decode", op="swiglu", m=17, inter=1408, k=2048),
        # the same of a DeepSeek-V3-shaped shared expert for a prefill chunk
        dict(name="swiglu_prefill", op="swiglu", m=4096, inter=2048, k=7168),
        # decode batch of routed tokens on a DeepSeek-V3-shaped rank of EP=8
        dict(DSV3, name="layer_decode", op="layer", tokens=64, given="bf16"),
        # a Qwen3-30B-A3B-shaped layer with a prompt chunk mixed into the batch, tokens quantised by the norm
        dict(QWEN3, name="layer_chunk", op="layer", tokens=333, given="e4m3"),
        # the DeepSeek-V3-shaped rank at prefill size
        dict(DSV3, name="layer_prefill", op="layer", tokens=8192, given="e4m3"),
    ]


def _log_int(rng, lo, hi):
    """A whole number spread evenly over the logarithm of [lo, hi], often an odd one."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, step, most):
    """A width of one of the layers, or any whole number of `step`s."""
    if rng.random() < 0.5:
        return rng.choice([w for w in (768, 1408, 2048, 4096, 7168) if w <= most])
    return step * _log_int(rng, 1, most // step)


def draw(rng):
    """Another case: any operator over the token counts, widths and types that the listed ones stand for."""
    op = rng.choice(("norm", "quantize", "matmul", "matmul", "swiglu", "swiglu", "layer", "layer", "layer"))
    if op == "norm":
        c = dict(op=op, rows=_log_int(rng, 1, 8192), cols=_width(rng, 8, 7168), dtype=rng.choice(("bf16", "bf16", "f32")),
                 residual=rng.random() < 0.7, plain_out=rng.random() < 0.7, quantized=True)
        if c["dtype"] == "f32":
            c["rows"] = min(c["rows"], 4096)
        return c
    if op == "quantize":
        return dict(op=op, rows=_log_int(rng, 1, 8192), cols=_width(rng, 8, 7168), dtype=rng.choice(("bf16", "bf16", "f32")),
                    block_rows=rng.choice((1, 1, 128)))
    if op == "matmul":
        return dict(op=op, m=_log_int(rng, 1, 8192), n=_width(rng, 8, 7168), k=_width(rng, 16, 2048),
                    out=rng.choice(("bf16", "bf16", "f32")), add=rng.random() < 0.5)
    if op == "swiglu":
        return dict(op=op, m=_log_int(rng, 1, 4096), inter=_width(rng, 16, 2048), k=_width(rng, 16, 7168))
    shape = rng.choice((QWEN3, DSV3, DSV2))
    local = rng.choice({128: (16, 32, 128), 256: (16, 32), 64: (16, 64)}[shape["n_experts"]])
    return dict(shape, op=op, tokens=_log_int(rng, 1, 6000), n_local=local, given=rng.choice(("bf16", "e4m3")))


# ---- inputs ----

def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _activations(g, rows, cols, dtype=torch.float32):
    """Hidden states: every column with a spread of its own, a few of them large."""
    spread = torch.exp(0.6 * torch.randn(cols, device="cuda", generator=g))
    return (torch.randn(rows, cols, device="cuda", generator=g) * spread).to(dtype)


def _quantized_rows(x):
    """(q, scale) of rows of values, one scale for each 128 columns: inputs of the products."""
    rows, cols = x.shape
    nb = _blocks(cols)
    parts = torch.nn.functional.pad(x, (0, nb * BLOCK - cols)).view(rows, nb, BLOCK)
    top = parts.abs().amax(-1, keepdim=True)
    q = torch.where(top > 0, parts * TOP / top, 0.0).view(rows, nb * BLOCK)[:, :cols]
    return q.contiguous().to(torch.float8_e4m3fn), (top / TOP).view(rows, nb)


def _weights(g, n, k, parts=1):
    """An 8-bit weight matrix [n, k] of normal values around 0.02 and its scales; `parts` matrices one below the other have blocks of their own."""
    q = (torch.randn(n, k, device="cuda", generator=g) * 100.0).clamp_(-TOP, TOP).to(torch.float8_e4m3fn)
    scale = 2e-4 * (0.7 + 0.6 * torch.rand(parts * _blocks(n // parts), _blocks(k), device="cuda", generator=g))
    return q, scale


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    c, op = case, case["op"]
    empty = lambda *shape, dtype=torch.float32: torch.empty(shape, device="cuda", dtype=dtype)  # noqa: E731
    s = {"case": c}
    if op == "norm":
        dt, rows, cols = _dtype(c["dtype"]), c["rows"], c["cols"]
        s["x"] = _activations(g, rows, cols, dt)
        s["residual"] = _activations(g, rows, cols, dt) if c["residual"] else None
        s["weight"] = (1.0 + 0.2 * torch.randn(cols, device="cuda", generator=g)).to(dt)
        s["sum"] = empty(rows, cols, dtype=dt) if c["residual"] else None
        s["out"] = empty(rows, cols, dtype=dt) if c["plain_out"] else None
        if c["quantized"]:
            s["q"], s["scale"] = empty(rows, cols, dtype=torch.float8_e4m3fn), empty(rows, _blocks(cols))
    elif op == "quantize":
        rows, cols = c["rows"], c["cols"]
        s["x"] = _activations(g, rows, cols, _dtype(c["dtype"]))
        s["q"], s["scale"] = empty(rows, cols, dtype=torch.float8_e4m3fn), empty(-(-rows // c["block_rows"]), _blocks(cols))
    elif op == "matmul":
        s["a"], s["a_scale"] = _quantized_rows(_activations(g, c["m"], c["k"]))
        s["w"], s["w_scale"] = _weights(g, c["n"], c["k"])
        s["add"] = torch.randn(c["m"], c["n"], device="cuda", generator=g).to(_dtype(c["out"])) if c["add"] else None
        s["out"] = empty(c["m"], c["n"], dtype=_dtype(c["out"]))
    elif op == "swiglu":
        s["a"], s["a_scale"] = _quantized_rows(_activations(g, c["m"], c["k"]))
        s["w"], s["w_scale"] = _weights(g, 2 * c["inter"], c["k"], parts=2)
        s["q"], s["scale"] = empty(c["m"], c["inter"], dtype=torch.float8_e4m3fn), empty(c["m"], _blocks(c["inter"]))
        if own:
            from paper_2510_02613_amd import scaled
            s["workspace"] = scaled.swiglu_workspace(c["m"], c["inter"], c["k"])
    else:
        _prepare_layer(s, c, g)
    return s


def _prepare_layer(s, c, g):
    T, H, I, E, k, n_local = c["tokens"], c["hidden"], c["inter"], c["n_experts"], c["top_k"], c["n_local"]
    slots = n_local + c["n_shared"]
    x = _activations(g, T, H)
    s["x"] = x.to(torch.bfloat16)
    s["xq"], s["x_scale"] = _quantized_rows(x if c["given"] == "e4m3" else s["x"].float())
    # the tokens that reach this rank after the dispatch: every one of them has an expert here
    order = torch.rand(T, E, device="cuda", generator=g).topk(k, dim=1).indices
    here = torch.randint(n_local, (T,), device="cuda", generator=g)
    order[:, 0] = torch.where((order < n_local).any(1), order[:, 0], here)
    s["ids"] = order.to(torch.int32).contiguous()
    s["weights"] = torch.softmax(torch.randn(T, k, device="cuda", generator=g), dim=1)
    s["shared_range"] = (0, -(-T // 8)) if c["n_shared"] else (0, 0)
    s["w13"] = torch.empty((slots, 2 * I, H), device="cuda", dtype=torch.float8_e4m3fn)
    s["w2"] = torch.empty((slots, H, I), device="cuda", dtype=torch.float8_e4m3fn)
    s["w13_scale"] = torch.empty((slots, 2 * _blocks(I), _blocks(H)), device="cuda")
    s["w2_scale"] = torch.empty((slots, _blocks(H), _blocks(I)), device="cuda")
    for e in range(slots):
        s["w13"][e], s["w13_scale"][e] = _weights(g, 2 * I, H, parts=2)
        s["w2"][e], s["w2_scale"][e] = _weights(g, H, I)
    s["out"] = torch.empty((T, H), device="cuda", dtype=torch.bfloat16)
    if own:
        import numpy as np
        from paper_2510_02613_amd.layer import MoELayer, ScaledExperts
        layer = MoELayer(hidden=H, inter=I, n_experts=E, top_k=k, n_slots=slots, max_tokens=c["max_tokens"], n_shared=c["n_shared"],
                         router_w=np.zeros((E, H), np.float32),
                         scaled=ScaledExperts(s["w13"], s["w13_scale"], s["w2"], s["w2_scale"]))
        layer.set_expert_map([e if e < n_local else -1 for e in range(E)], list(range(n_local, slots)))
        s["layer"] = layer


# ---- one pass ----

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2510_02613_amd import scaled
    c, op = s["case"], s["case"]["op"]
    if op == "norm":
        scaled.rms_norm(s["x"], s["weight"], residual=s["residual"], eps=1e-6, sum_out=s["sum"], out=s["out"],
                        q=s.get("q"), q_scale=s.get("scale"))
        return {k: s[k] for k in ("sum", "out", "q", "scale") if s.get(k) is not None}
    if op == "quantize":
        scaled.quantize(s["x"], block_rows=c["block_rows"], q=s["q"], scale=s["scale"])
        return {"q": s["q"], "scale": s["scale"]}
    if op == "matmul":
        return {"out": scaled.matmul(s["a"], s["a_scale"], s["w"], s["w_scale"], add=s["add"], out=s["out"])}
    if op == "swiglu":
        scaled.swiglu(s["a"], s["a_scale"], s["w"], s["w_scale"], q=s["q"], scale=s["scale"], workspace=s["workspace"])
        return {"q": s["q"], "scale": s["scale"]}
    if c["given"] == "e4m3":
        s["layer"].forward_scaled(s["xq"], s["x_scale"], topk_ids=s["ids"], topk_w=s["weights"], out=s["out"], shared_range=s["shared_range"])
    else:
        s["layer"].forward_routed(s["x"], s["ids"], s["weights"], out=s["out"], shared_range=s["shared_range"])
    return {"out": s["out"]}


def _spread_rows(scale, cols):
    """Row scales [rows, blocks] as one factor per element."""
    return scale.repeat_interleave(BLOCK, dim=1)[:, :cols]


def _spread_blocks(scale, n, k):
    """Block scales as one factor per weight."""
    return scale.repeat_interleave(BLOCK, dim=0)[:n].repeat_interleave(BLOCK, dim=1)[:, :k]


def _gate_and_up(a, w, w_scale, inter):
    """silu(a Wg^T) * (a Wu^T) in fp32; gate rows first, then the up rows, with blocks of their own."""
    k, nb = w.shape[1], _blocks(inter)
    gate = a @ (w[:inter].float() * _spread_blocks(w_scale[:nb], inter, k)).t()
    up = a @ (w[inter:].float() * _spread_blocks(w_scale[nb:], inter, k)).t()
    return gate / (1.0 + torch.exp(-gate)) * up


def _run_plain(s):
    c, op = s["case"], s["case"]["op"]
    if op == "norm":
        r = s["x"].float() + s["residual"].float() if c["residual"] else s["x"].float()
        y = r * torch.rsqrt((r * r).mean(dim=1, keepdim=True) + 1e-6) * s["weight"].float()
        got = {}
        if c["residual"]:
            got["sum"] = r.to(s["x"].dtype)
        if c["plain_out"]:
            got["out"] = y.to(s["x"].dtype)
        if c["quantized"]:
            got["q"], got["scale"] = _quantized_rows(y)
        return got
    if op == "quantize":
        x = s["x"].float()
        if c["block_rows"] == 1:
            q, scale = _quantized_rows(x)
            return {"q": q, "scale": scale}
        rows, cols = x.shape
        rb, cb = _blocks(rows), _blocks(cols)
        parts = torch.nn.functional.pad(x, (0, cb * BLOCK - cols, 0, rb * BLOCK - rows)).view(rb, BLOCK, cb, BLOCK)
        top = parts.abs().amax(dim=(1, 3))
        per = _spread_blocks(top, rows, cols)
        return {"q": torch.where(per > 0, x * TOP / per, 0.0).to(torch.float8_e4m3fn), "scale": top / TOP}
    if op == "matmul":
        a = s["a"].float() * _spread_rows(s["a_scale"], c["k"])
        w = s["w"].float() * _spread_blocks(s["w_scale"], c["n"], c["k"])
        y = a @ w.t()
        if c["add"]:
            y = y + s["add"].float()
        return {"out": y.to(_dtype(c["out"]))}
    if op == "swiglu":
        a = s["a"].float() * _spread_rows(s["a_scale"], c["k"])
        q, scale = _quantized_rows(_gate_and_up(a, s["w"], s["w_scale"], c["inter"]))
        return {"q": q, "scale": scale}
    if c["given"] == "e4m3":
        x = s["xq"].float() * _spread_rows(s["x_scale"], c["hidden"])
    else:
        q, scale = _quantized_rows(s["x"].float())
        x = q.float() * _spread_rows(scale, c["hidden"])
    y = torch.zeros(x.shape, device=x.device)
    for e in range(c["n_local"] + c["n_shared"]):   # expert by expert: their weights together, in 32 bits, would be six gigabytes
        if e < c["n_local"]:
            token, col = (s["ids"] == e).nonzero(as_tuple=True)
            weight = s["weights"][token, col]
        else:
            token = torch.arange(*s["shared_range"], device=x.device)
            weight = torch.ones(len(token), device=x.device)
        q, scale = _quantized_rows(_gate_and_up(x[token], s["w13"][e], s["w13_scale"][e], c["inter"]))
        h = q.float() * _spread_rows(scale, c["inter"])
        out = h @ (s["w2"][e].float() * _spread_blocks(s["w2_scale"][e], c["hidden"], c["inter"])).t()
        y.index_add_(0, token, weight[:, None] * out)
    return {"out": y.to(torch.bfloat16)}


# ---- the definitions in 64 bits ----

def _wide(q, scale, block_rows):
    """The values of an 8-bit tensor, element (i, j) = q[i, j] * scale[i // block_rows, j // 128], in 64 bits."""
    i = torch.arange(q.shape[0], device=q.device) // block_rows
    j = torch.arange(q.shape[1], device=q.device) // BLOCK
    return q.double() * scale.double()[i][:, j]


def _row_quotients(v):
    """(v * 448 / a, a / 448) with a = the largest magnitude of 128 columns: the quotients before their rounding to 8 bits, and the scales."""
    quotients, scales = torch.zeros_like(v), []
    for at in range(0, v.shape[1], BLOCK):
        part = v[:, at:at + BLOCK]
        a = part.abs().max(dim=1).values
        quotients[:, at:at + BLOCK] = part * TOP / torch.where(a > 0, a, torch.ones_like(a))[:, None]
        scales.append(a / TOP)
    return quotients, torch.stack(scales, dim=1)


def _ffn_first(x, w, w_scale):
    half = w.shape[0] // 2
    nb = w_scale.shape[0] // 2
    g = x.matmul(_wide(w[:half], w_scale[:nb], BLOCK).t())
    u = x.matmul(_wide(w[half:], w_scale[nb:], BLOCK).t())
    return g * torch.sigmoid(g) * u


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        r = s["x"].double()
        if s["residual"] is not None:
            r = r + s["residual"].double()
        y = r / torch.sqrt(r.pow(2).sum(1, keepdim=True) / r.shape[1] + 1e-6) * s["weight"].double()
        got = {"sum": r} if s["residual"] is not None else {}
        if case["plain_out"]:
            got["out"] = y
        if case["quantized"]:
            got["q"], got["scale"] = _row_quotients(y)
        return got
    if op == "quantize":
        x = s["x"].double()
        if case["block_rows"] == 1:
            q, scale = _row_quotients(x)
            return {"q": q, "scale": scale}
        q, scale = torch.zeros_like(x), torch.zeros(s["scale"].shape, device=x.device, dtype=torch.float64)
        for i in range(0, x.shape[0], BLOCK):
            for j in range(0, x.shape[1], BLOCK):
                part = x[i:i + BLOCK, j:j + BLOCK]
                a = part.abs().max()
                scale[i // BLOCK, j // BLOCK] = a / TOP
                q[i:i + BLOCK, j:j + BLOCK] = part * TOP / torch.where(a > 0, a, torch.ones_like(a))
        return {"q": q, "scale": scale}
    if op == "matmul":
        y = _wide(s["a"], s["a_scale"], 1).matmul(_wide(s["w"], s["w_scale"], BLOCK).t())
        return {"out": y if s["add"] is None else y + s["add"].double()}
    if op == "swiglu":
        q, scale = _row_quotients(_ffn_first(_wide(s["a"], s["a_scale"], 1), s["w"], s["w_scale"]))
        return {"q": q, "scale": scale}
    if case["given"] == "e4m3":
        x = _wide(s["xq"], s["x_scale"], 1)
    else:
        q, scale = _row_quotients(s["x"].double())
        x = _wide(q.float().to(torch.float8_e4m3fn), scale, 1)
    y = torch.zeros_like(x)
    first, last = s["shared_range"]
    for e in range(s["w13"].shape[0]):
        if e < case["n_local"]:
            weight = torch.where(s["ids"] == e, s["weights"].double(), torch.zeros((), device=x.device, dtype=torch.float64)).sum(1)
            token = (s["ids"] == e).any(1).nonzero().flatten()
        else:
            weight = torch.ones(x.shape[0], device=x.device, dtype=torch.float64)
            token = torch.arange(first, last, device=x.device)
        if len(token) == 0:
            continue
        q, scale = _row_quotients(_ffn_first(x[token], s["w13"][e], s["w13_scale"][e]))
        h = _wide(q.float().to(torch.float8_e4m3fn), scale, 1)
        y[token] += weight[token, None] * h.matmul(_wide(s["w2"][e], s["w2_scale"][e], BLOCK).t())
    return {"out": y}


# ---- what a pass cannot do without ----

def work(case):
    c, op = case, case["op"]
    if op == "norm":
        n, es = c["rows"] * c["cols"], 2 if c["dtype"] == "bf16" else 4
        tensors = 1 + 2 * c["residual"] + c["plain_out"]   # x, the residual and the sum, the result
        return {"bytes": n * es * tensors + es * c["cols"] + c["quantized"] * (n + 4 * c["rows"] * _blocks(c["cols"])), "flops": 8.0 * n}
    if op == "quantize":
        n, es = c["rows"] * c["cols"], 2 if c["dtype"] == "bf16" else 4
        return {"bytes": n * (es + 1) + 4 * -(-c["rows"] // c["block_rows"]) * _blocks(c["cols"]), "flops": 3.0 * n}
    if op == "matmul":
        m, n, k = c["m"], c["n"], c["k"]
        es = 2 if c["out"] == "bf16" else 4
        return {"bytes": m * k + 4 * m * _blocks(k) + n * k + 4 * _blocks(n) * _blocks(k) + m * n * es * (1 + c["add"]), "flops": 2.0 * m * n * k}
    if op == "swiglu":
        m, n, k = c["m"], c["inter"], c["k"]
        return {"bytes": m * k + 4 * m * _blocks(k) + 2 * n * k + 8 * _blocks(n) * _blocks(k) + m * n + 4 * m * _blocks(n), "flops": 4.0 * m * n * k}
    T, H, I, E, k, n_local = c["tokens"], c["hidden"], c["inter"], c["n_experts"], c["top_k"], c["n_local"]
    none = math.prod(max(0, E - n_local - i) / (E - i) for i in range(k))    # share of the tokens that had no expert here
    rows = T * (k * n_local / E + none)                                      # assignments to this rank, on average
    shared = -(-T // 8) * c["n_shared"]
    used = n_local * (1.0 - (1.0 - 1.0 / n_local) ** rows) + c["n_shared"]   # experts with a row at least
    expert = 3 * I * H + 4 * (3 * _blocks(I) * _blocks(H))
    x = T * (2 * H if c["given"] == "bf16" else H + 4 * _blocks(H))
    return {"bytes": used * expert + x + 2 * T * H + 8 * T * k, "flops": 6.0 * (rows + shared) * H * I}
