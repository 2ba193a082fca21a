"""Tokens sorted by expert and back, and the products of experts held in 4 bits: what they compute, in plain torch and through
the framework's calls.

Sorting: assignment a = t * top_k + j sends token t to group map[ids[t, j]] (without a map to group ids[t, j]); ids and groups that do not exist
are assignments that are not this rank's.  Rows are ordered by group, inside a group by assignment; row r is a copy of token source[r] // top_k,
row[t, j] is the place of the assignment or -1, group g has rows offsets[g] .. offsets[g + 1] - 1.  Back: out[t] = sum over j of weights[t, j] * y[row[t, j]].

A 4-bit matrix is two e2m1 values a byte (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, the even column in the low half) and one
power of two, an e8m0 byte b for 2^(b - 127), for each row and 32 columns.  Quantising takes the smallest power of two that leaves no magnitude of
the 32 above 6, and rounds to the nearest, ties to the even code.
A pass is one use of a public entry point on tensors that are already on the GPU; result buffers and weights are made beforehand, as a serving
program keeps them, and results that a training step differentiates are made by the step.
"""
from __future__ import annotations

import math

import torch

own = False

GROUP = 32                                       # columns that share a power of two
STEPS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)

QWEN3 = dict(hidden=2048, inter=768, n_experts=128, top_k=8)
DSV3 = dict(hidden=7168, inter=2048, n_experts=256, top_k=8)
DSV2 = dict(hidden=2048, inter=1408, n_experts=64, top_k=6)
LOCAL = {128: (16, 32, 128), 256: (16, 32), 64: (16, 64)}


def _routed(shape, **kw):
    return dict(n_experts=shape["n_experts"], top_k=shape["top_k"], **kw)


def listed():
    return [
        # one decoded token on a DeepSeek-V3-shaped rank of EP=8: its rows for the experts that are here
        _routed(DSV3, name="sort_token", op="sort", tokens=1, cols=7168, n_local=32, dtype="bf16", grad=False),
        # a prompt chunk of a DeepSeek-V2-Lite-shaped layer, fp32 rows
        _routed(DSV2, name="sort_chunk", op="sort", tokens=333, cols=2048, n_local=64, dtype="f32", grad=False),
        # a training step's batch of a Qwen3-30B-A3B-shaped layer, and the gradient of its tokens
        _routed(QWEN3, name="sort_step", op="sort", tokens=8192, cols=2048, n_local=128, dtype="bf16", grad=True),
        # a decode batch of the DeepSeek-V3-shaped rank, back to token order
        _routed(DSV3, name="combine_decode", op="combine", tokens=64, cols=7168, n_local=32, dtype="bf16", grad=False),
        # the way back in a training step, with the gradients of the expert outputs and of the weights
        _routed(QWEN3, name="combine_step", op="combine", tokens=5001, cols=2048, n_local=128, dtype="bf16", grad=True),
        # an expert's first matrix on its way into a 4-bit pool, Qwen3-30B-A3B-shaped
        dict(name="quantize_expert", op="quantize", rows=1536, cols=2048, dtype="bf16", values=False),
        # a DeepSeek-V3-shaped one from fp32, with the values that are left of it (what a calibration compares)
        dict(name="quantize_values", op="quantize", rows=4096, cols=7168, dtype="f32", values=True),
        # down projection of a dense expert for one token, added to the residual stream
        dict(name="matmul_token", op="matmul", m=1, n=7168, k=2048, out="bf16", add=True),
        # a projection of sizes that are whole tiles nowhere, fp32 result
        dict(name="matmul_ragged", op="matmul", m=173, n=1543, k=1440, out="f32", add=False),
        # second products of all experts of a Qwen3-30B-A3B-shaped layer for a prompt chunk, some 20 rows each
        _routed(QWEN3, name="matmul_experts", op="matmul_experts", tokens=333, n_local=128, n=2048, k=768, out="bf16"),
        # first half of a dense expert for a few decoded tokens, DeepSeek-V2-Lite-shaped
        dict(name="swiglu_few", op="swiglu", m=3, inter=1408, k=2048, out="bf16"),
        # first half of the DeepSeek-V3-shaped rank's experts for a decode batch, a row or two each
        _routed(DSV3, name="swiglu_experts", op="swiglu_experts", tokens=64, n_local=32, inter=2048, k=7168, out="bf16"),
    ]


def _log_int(rng, lo, hi):
    """A whole number spread evenly over the logarithm of [lo, hi], often an odd one."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, step, most):
    """A width of one of the layers, or any whole number of `step`s."""
    if rng.random() < 0.5:
        return rng.choice([w for w in (768, 1408, 2048, 7168) if w <= most])
    return step * _log_int(rng, 1, most // step)


def draw(rng):
    """Another case: any operator over the token counts, widths and types that the listed ones stand for."""
    op = rng.choice(("sort", "sort", "combine", "combine", "quantize", "matmul", "matmul", "matmul_experts", "swiglu", "swiglu_experts"))
    out = rng.choice(("bf16", "bf16", "f32"))
    shape = rng.choice((QWEN3, DSV3, DSV2))
    local = rng.choice(LOCAL[shape["n_experts"]])
    if op in ("sort", "combine"):
        cols = shape["hidden"] if rng.random() < 0.6 else _width(rng, 8, 7168)
        dtype = rng.choice(("bf16", "bf16", "f32"))
        # a training step writes all rows: as many bytes at most as the largest listed ones
        most = min(8192 if op == "sort" else 5001, 8192 * 2048 * 2 // (cols * (2 if dtype == "bf16" else 4)))
        return _routed(shape, op=op, tokens=_log_int(rng, 1, most), cols=cols, n_local=local, dtype=dtype, grad=rng.random() < 0.5)
    if op == "quantize":
        return dict(op=op, rows=_log_int(rng, 1, 4096), cols=_width(rng, GROUP, 7168), dtype=rng.choice(("bf16", "bf16", "f32")), values=rng.random() < 0.5)
    if op == "matmul":
        return dict(op=op, m=_log_int(rng, 1, 512), n=_log_int(rng, 16, 7168) if rng.random() < 0.5 else _width(rng, 8, 7168), k=_width(rng, GROUP, 2048),
                    out=out, add=rng.random() < 0.5)
    if op == "swiglu":
        return dict(op=op, m=_log_int(rng, 1, 256), inter=_width(rng, 8, 2048), k=_width(rng, GROUP, 7168), out=out)
    tokens = _log_int(rng, 1, 333)
    if op == "matmul_experts":
        return _routed(shape, op=op, tokens=tokens, n_local=local, n=shape["hidden"], k=shape["inter"], out=out)
    return _routed(shape, op=op, tokens=tokens, n_local=local, inter=shape["inter"], k=shape["hidden"], out=out)


# ---- inputs ----

def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _activations(g, rows, cols, dtype):
    """Hidden states: every column with a spread of its own, a few of them large."""
    spread = torch.exp(0.6 * torch.randn(cols, device="cuda", generator=g))
    return (torch.randn(rows, cols, device="cuda", generator=g) * spread).to(dtype)


def _routing(g, c):
    """(ids [T, k], the rank's expert map [E]): every token has an expert here, as after a dispatch; the experts sit in shuffled slots."""
    T, E, k, n_local = c["tokens"], c["n_experts"], c["top_k"], c["n_local"]
    ids = torch.rand(T, E, device="cuda", generator=g).topk(k, dim=1).indices
    here = torch.randint(n_local, (T,), device="cuda", generator=g)
    ids[:, 0] = torch.where((ids < n_local).any(1), ids[:, 0], here)
    slots = torch.full((E,), -1, device="cuda", dtype=torch.int32)
    slots[:n_local] = torch.randperm(n_local, device="cuda", generator=g).to(torch.int32)
    return ids.to(torch.int32).contiguous(), slots


def _order(ids, slots, n_groups):
    """(offsets, source, row) of the sorted assignments, as 32-bit numbers."""
    A = ids.numel()
    group = slots[ids.flatten().long()].long()
    group = torch.where((group >= 0) & (group < n_groups), group, n_groups)
    place = torch.argsort(group, stable=True)                     # row -> assignment, those of other ranks last
    counts = torch.zeros(n_groups + 1, device=ids.device, dtype=torch.long).index_add_(0, group, torch.ones_like(group))
    offsets = torch.zeros(n_groups + 1, device=ids.device, dtype=torch.long)
    offsets[1:] = counts[:n_groups].cumsum(0)
    at = torch.arange(A, device=ids.device)
    source = torch.where(at < offsets[-1], place, -1)
    row = torch.empty_like(at)
    row[place] = torch.where(at < offsets[-1], at, -1)
    return offsets.int(), source.int(), row.int().view(ids.shape)


def _quantized(x):
    """(bytes, powers) of rows of fp32 values."""
    rows, cols = x.shape
    parts = x.view(rows, cols // GROUP, GROUP)
    top = parts.abs().amax(-1)
    mantissa, exponent = torch.frexp(top)
    power = (exponent - 2 - (mantissa <= 0.75).to(exponent.dtype)).clamp(-127, 127)
    power = torch.where(top > 0, power, -127)
    t = torch.ldexp(parts, -power[..., None]).abs()
    code = (t > 0.25).to(torch.uint8)
    for border, tie_up in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (t >= border) if tie_up else (t > border)
    code += 8 * torch.signbit(parts).to(torch.uint8)
    code = code.view(rows, cols // 2, 2)
    return code[..., 0] + 16 * code[..., 1], (power + 127).to(torch.uint8)


def _values(q, scale):
    """What a 4-bit matrix stands for, in fp32."""
    steps = torch.tensor(STEPS + tuple(-v for v in STEPS), device=q.device)
    codes = torch.stack((q & 15, q >> 4), dim=-1).flatten(-2).int()
    power = torch.ldexp(torch.ones((), device=q.device), scale.int() - 127)
    return steps[codes] * power.repeat_interleave(GROUP, dim=-1)


def _weights(g, n, k):
    """A 4-bit weight matrix [n, k] of normal values around 0.02."""
    return _quantized(0.02 * torch.randn(n, k, device="cuda", generator=g))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    c, op = case, case["op"]
    empty = lambda *shape, dtype=torch.float32: torch.empty(shape, device="cuda", dtype=dtype)  # noqa: E731
    s = {"case": c}
    if op == "quantize":
        dt, rows, cols = _dtype(c["dtype"]), c["rows"], c["cols"]
        spread = torch.exp(0.3 * torch.randn(rows, 1, device="cuda", generator=g))
        s["x"] = (0.02 * spread * torch.randn(rows, cols, device="cuda", generator=g)).to(dt)
        s["q"], s["scale"] = empty(rows, cols // 2, dtype=torch.uint8), empty(rows, cols // GROUP, dtype=torch.uint8)
        s["values"] = empty(rows, cols, dtype=dt) if c["values"] else None
    elif op in ("matmul", "swiglu"):
        n = c["n"] if op == "matmul" else c["inter"]
        s["a"] = _activations(g, c["m"], c["k"], torch.bfloat16)
        s["w"], s["w_scale"] = _weights(g, n if op == "matmul" else 2 * n, c["k"])
        # rows of the result start on 16 bytes whatever n is
        s["out"] = empty(c["m"], (n + 7) // 8 * 8, dtype=_dtype(c["out"]))[:, :n]
        if op == "matmul":
            s["add"] = None
            if c["add"]:
                s["add"] = torch.randn(s["out"].shape[0], s["out"].stride(0), device="cuda", generator=g).to(_dtype(c["out"]))[:, :n]
    else:
        s["ids"], s["map"] = _routing(g, c)
        A = s["ids"].numel()
        s["offsets"], s["source"], s["row"] = _order(s["ids"], s["map"], c["n_local"])
        if op == "sort":
            dt = _dtype(c["dtype"])
            s["x"] = _activations(g, c["tokens"], c["cols"], dt).requires_grad_(c["grad"])
            if c["grad"]:
                s["grad"] = torch.randn(A, c["cols"], device="cuda", generator=g).to(dt)
            else:
                s["rows"] = torch.zeros(A, c["cols"], device="cuda", dtype=dt)       # what is behind the last row stays as it is here
        elif op == "combine":
            dt = _dtype(c["dtype"])
            s["y"] = _activations(g, A, c["cols"], dt).requires_grad_(c["grad"])
            s["weights"] = torch.softmax(torch.randn(c["tokens"], c["top_k"], device="cuda", generator=g), dim=1).requires_grad_(c["grad"])
            if c["grad"]:
                s["grad"] = torch.randn(c["tokens"], c["cols"], device="cuda", generator=g).to(dt)
            else:
                s["out"] = empty(c["tokens"], c["cols"], dtype=dt)
        else:
            first = op == "swiglu_experts"
            n, k, G = (2 * c["inter"] if first else c["n"]), c["k"], c["n_local"]
            s["a"] = _activations(g, A, k, torch.bfloat16)
            s["w"], s["w_scale"] = empty(G, n, k // 2, dtype=torch.uint8), empty(G, n, k // GROUP, dtype=torch.uint8)
            for e in range(G):
                s["w"][e], s["w_scale"][e] = _weights(g, n, k)
            s["out"] = torch.zeros(A, c["inter"] if first else n, device="cuda", dtype=_dtype(c["out"]))
    return s


# ---- one pass ----

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2510_02613_amd import dispatch, four_bit
    c, op = s["case"], s["case"]["op"]
    if op == "sort":
        if c["grad"]:
            rows, order = dispatch.sort_tokens(s["x"], s["ids"], c["n_local"], expert_map=s["map"])
            dx, = torch.autograd.grad(rows, s["x"], s["grad"])
            return {"rows": rows, "offsets": order.offsets, "source": order.source, "row": order.row, "dx": dx}
        order = dispatch.Order(s["offsets"], s["source"], s["row"])
        dispatch.sort_tokens(s["x"], s["ids"], c["n_local"], expert_map=s["map"], rows=s["rows"], order=order)
        return {"rows": s["rows"], "offsets": s["offsets"], "source": s["source"], "row": s["row"]}
    if op == "combine":
        order = dispatch.Order(s["offsets"], s["source"], s["row"])
        if c["grad"]:
            out = dispatch.combine_tokens(s["y"], order, s["weights"])
            dy, dw = torch.autograd.grad(out, (s["y"], s["weights"]), s["grad"])
            return {"out": out, "dy": dy, "dweights": dw}
        return {"out": dispatch.combine_tokens(s["y"], order, s["weights"], out=s["out"])}
    if op == "quantize":
        four_bit.quantize(s["x"], q=s["q"], scale=s["scale"], values=s["values"])
        return {k: s[k] for k in ("q", "scale", "values") if s[k] is not None}
    if op == "matmul":
        return {"out": four_bit.matmul(s["a"], s["w"], s["w_scale"], add=s["add"], out=s["out"])}
    if op == "matmul_experts":
        return {"out": four_bit.matmul(s["a"], s["w"], s["w_scale"], offsets=s["offsets"], out=s["out"])}
    if op == "swiglu":
        return {"out": four_bit.swiglu(s["a"], s["w"], s["w_scale"], out=s["out"])}
    return {"out": four_bit.swiglu(s["a"], s["w"], s["w_scale"], offsets=s["offsets"], out=s["out"])}


def _sum_back(y, row, weights):
    """[T, H] in fp32: the rows of every token, times their weights, added up."""
    T, k = row.shape
    there = (row >= 0)[..., None]
    parts = torch.where(there, y.float()[row.clamp(min=0).flatten().long()].view(T, k, -1), 0.0)
    return parts.sum(1) if weights is None else (parts * weights[..., None]).sum(1)


def _silu_product(gate, up):
    return gate / (1.0 + torch.exp(-gate)) * up


def _run_plain(s):
    c, op = s["case"], s["case"]["op"]
    with torch.no_grad():
        if op == "sort":
            offsets, source, row = _order(s["ids"], s["map"], c["n_local"])
            there = (source >= 0)[:, None]
            rows = torch.where(there, s["x"][(source.clamp(min=0) // c["top_k"]).long()], 0.0)
            got = {"rows": rows, "offsets": offsets, "source": source, "row": row}
            if c["grad"]:
                got["dx"] = _sum_back(s["grad"], row, None).to(rows.dtype)
            return got
        if op == "combine":
            out = _sum_back(s["y"], s["row"], s["weights"]).to(s["y"].dtype)
            if not c["grad"]:
                return {"out": out}
            there = (s["source"] >= 0)[:, None]
            at = s["source"].clamp(min=0).long()
            of_row = s["grad"].float()[at // c["top_k"]]
            dots = torch.where(there[:, 0], (of_row * s["y"].float()).sum(1), 0.0)
            dy = torch.where(there, of_row * s["weights"].flatten()[at][:, None], 0.0).to(s["y"].dtype)
            dw = torch.where(s["row"] >= 0, dots[s["row"].clamp(min=0).long()], 0.0)
            return {"out": out, "dy": dy, "dweights": dw}
        if op == "quantize":
            q, scale = _quantized(s["x"].float())
            got = {"q": q, "scale": scale}
            if c["values"]:
                got["values"] = _values(q, scale).to(s["x"].dtype)
            return got
        if op == "matmul":
            y = s["a"].float() @ _values(s["w"], s["w_scale"]).t()
            if c["add"]:
                y = y + s["add"].float()
            return {"out": y.to(_dtype(c["out"]))}
        if op == "swiglu":
            y = s["a"].float() @ _values(s["w"], s["w_scale"]).t()
            return {"out": _silu_product(y[:, :c["inter"]], y[:, c["inter"]:]).to(_dtype(c["out"]))}
        out = torch.zeros(s["out"].shape, device="cuda", dtype=_dtype(c["out"]))
        ends = s["offsets"].tolist()
        for e in range(c["n_local"]):   # expert by expert: their weights together, in 32 bits, would be gigabytes
            lo, hi = ends[e], ends[e + 1]
            if lo == hi:
                continue
            y = s["a"][lo:hi].float() @ _values(s["w"][e], s["w_scale"][e]).t()
            out[lo:hi] = (_silu_product(y[:, :c["inter"]], y[:, c["inter"]:]) if op == "swiglu_experts" else y).to(out.dtype)
        return {"out": out}


# ---- the definitions in 64 bits ----

def _wide(q, scale):
    """The values of a 4-bit matrix in 64 bits, from the fields of its codes: sign, two exponent bits, one mantissa bit."""
    n, half = q.shape
    code = torch.empty(n, 2 * half, device=q.device, dtype=torch.int64)
    code[:, 0::2], code[:, 1::2] = (q % 16).long(), (q // 16).long()
    exponent, mantissa = (code // 2) % 4, code % 2
    size = torch.where(exponent == 0, 0.5 * mantissa.double(), (1.0 + 0.5 * mantissa.double()) * 2.0 ** (exponent - 1).double())
    column = torch.arange(2 * half, device=q.device) // GROUP
    return torch.where(code >= 8, -size, size) * (2.0 ** (scale.double() - 127.0))[:, column]


def _place(case, s):
    """For every assignment in order its group (n_local: none), by comparing with each group: [A], and the rows of each group."""
    group = torch.full((s["ids"].numel(),), case["n_local"], device="cuda", dtype=torch.int64)
    flat = s["ids"].reshape(-1)
    slots = s["map"].tolist()
    for e, slot in enumerate(slots):
        if 0 <= slot < case["n_local"]:
            group[flat == e] = slot
    return group


def _exact_order(case, s):
    group = _place(case, s)
    source, row = torch.full_like(group, -1), torch.full_like(group, -1)
    offsets = [0]
    for slot in range(case["n_local"]):
        mine = (group == slot).nonzero().flatten()
        at = offsets[-1] + torch.arange(len(mine), device="cuda")
        source[at] = mine
        row[mine] = at
        offsets.append(offsets[-1] + len(mine))
    return torch.tensor(offsets, device="cuda", dtype=torch.int32), source.int(), row.int().view(s["ids"].shape)


def _exact_product(case, a, q, scale, first):
    y = a.double().matmul(_wide(q, scale).t())
    if not first:
        return y
    gate, up = y[:, :case["inter"]], y[:, case["inter"]:]
    return gate * torch.sigmoid(gate) * up


@torch.no_grad()
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "sort":
        offsets, source, row = _exact_order(case, s)
        total, k = int(offsets[-1]), case["top_k"]
        rows = torch.zeros(source.shape[0], case["cols"], device="cuda", dtype=torch.float64)
        rows[:total] = s["x"].double()[source[:total].long() // k]
        got = {"rows": rows, "offsets": offsets, "source": source, "row": row}
        if case["grad"]:
            dx = torch.zeros(s["x"].shape, device="cuda", dtype=torch.float64)
            got["dx"] = dx.index_add_(0, source[:total].long() // k, s["grad"][:total].double())
        return got
    if op == "combine":
        k = case["top_k"]
        out = torch.zeros(case["tokens"], case["cols"], device="cuda", dtype=torch.float64)
        dy = torch.zeros(s["y"].shape, device="cuda", dtype=torch.float64)
        dw = torch.zeros(case["tokens"], k, device="cuda", dtype=torch.float64)
        for j in range(k):
            t = (s["row"][:, j] >= 0).nonzero().flatten()
            r = s["row"][t, j].long()
            w = s["weights"][t, j].double()[:, None]
            out[t] += w * s["y"][r].double()
            if case["grad"]:
                dy[r] = w * s["grad"][t].double()
                dw[t, j] = s["grad"][t].double().mul(s["y"][r].double()).sum(1)
        return {"out": out, "dy": dy, "dweights": dw} if case["grad"] else {"out": out}
    if op == "quantize":
        x = s["x"].double()
        top = torch.stack([p.abs().amax(1) for p in x.split(GROUP, dim=1)], dim=1)
        power = torch.ceil(torch.log2(top / 6.0))                 # of a magnitude of 6 * 2^p exactly the logarithm is exact too
        power = torch.where(top > 0, power, -127.0).clamp(-127.0, 127.0)
        t = x / (2.0 ** power)[:, torch.arange(x.shape[1], device="cuda") // GROUP]
        size = t.abs()
        step = torch.where(size < 2.0, 0.5, torch.where(size < 4.0, 1.0, 2.0))
        size = torch.round(size / step) * step                    # ties to even: the even multiple is the even code
        values = torch.where(t < 0, -size, size) * (2.0 ** power)[:, torch.arange(x.shape[1], device="cuda") // GROUP]
        got = {"q": None, "scale": (power + 127.0).to(torch.uint8)}
        if case["values"]:
            got["values"] = values
        return got
    if op in ("matmul", "swiglu"):
        y = _exact_product(case, s["a"], s["w"], s["w_scale"], op == "swiglu")
        return {"out": y + s["add"].double() if s.get("add") is not None else y}
    y = torch.zeros(s["out"].shape, device="cuda", dtype=torch.float64)
    for e in range(case["n_local"]):
        lo, hi = int(s["offsets"][e]), int(s["offsets"][e + 1])
        if hi > lo:
            y[lo:hi] = _exact_product(case, s["a"][lo:hi], s["w"][e], s["w_scale"][e], op == "swiglu_experts")
    return {"out": y}


# ---- what a pass cannot do without ----

def _rows_here(c):
    """Assignments to this rank, on average."""
    T, E, k, n_local = c["tokens"], c["n_experts"], c["top_k"], c["n_local"]
    none = math.prod(max(0, E - n_local - i) / (E - i) for i in range(k))    # share of the tokens that had no expert here
    return T * (k * n_local / E + none)


def work(case):
    c, op = case, case["op"]
    if op in ("sort", "combine"):
        T, A, H, es = c["tokens"], c["tokens"] * c["top_k"], c["cols"], 2 if c["dtype"] == "bf16" else 4
        rows = _rows_here(c)
        if op == "sort":
            moved = T * H + (A if c["grad"] else rows) * H            # the tokens, their rows (a step's own are written to the end)
            if c["grad"]:
                moved += rows * H + T * H                             # the rows' gradient, the tokens'
            return {"bytes": es * moved + 12 * A + 4 * c["n_experts"] + 4 * (c["n_local"] + 1), "flops": rows * H if c["grad"] else 0}
        moved = rows * H + T * H
        if c["grad"]:
            moved += T * H + A * H                                    # the result's gradient, the rows'
        return {"bytes": es * moved + 8 * A + (8 * A if c["grad"] else 0), "flops": (6.0 if c["grad"] else 2.0) * rows * H}
    if op == "quantize":
        n, es = c["rows"] * c["cols"], 2 if c["dtype"] == "bf16" else 4
        return {"bytes": n * (es * (1 + c["values"]) + 0.5) + n / GROUP, "flops": 3.0 * n}
    es = 2 if c["out"] == "bf16" else 4
    k, n = c["k"], (c["n"] if "n" in c else 2 * c["inter"])
    cols = c["n"] if "n" in c else c["inter"]
    matrix = n * k / 2 + n * k / GROUP
    if op in ("matmul", "swiglu"):
        return {"bytes": 2 * c["m"] * k + matrix + es * c["m"] * cols * (1 + c.get("add", False)), "flops": 2.0 * c["m"] * n * k}
    rows = _rows_here(c)
    used = c["n_local"] * (1.0 - (1.0 - 1.0 / c["n_local"]) ** rows)         # experts with a row at least
    return {"bytes": 2 * rows * k + used * matrix + es * rows * cols + 4 * (c["n_local"] + 1), "flops": 2.0 * rows * n * k}
