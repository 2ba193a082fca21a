"""How far the operators of the 8-bit path are expected to be from 64 bits, as a sum of squares over many elements.

The element-wise bounds of scaled_ref.py are worst cases, many times what happens: an output that is one per cent off everywhere passes them.  Here every
rounding is taken as independent of the others, so that squares add up:
  * a sum of n products in fp32 makes n roundings of partial sums, none of which is expected above the root of the sum of the products' squares:
    sqrt(n) half steps of that, whatever the order;
  * a byte falls to the other side of an e4m3 border that lies within d of a value with probability d / step, and is a step off then: d * step
    expected for its square;
  * the final rounding of y + e is as large as that of y, and independent of e.
A sum of squares over ten thousand elements and more is within some per cent of what is expected; SLACK is 1.2 on the squares, 1.1 on the norm.
"""
import torch

import scaled_ref as R

SLACK = 1.2


def product_noise(a, w):
    """Expected error of a w^T in fp32 from exact products; a, w in 64 bits."""
    n = R.BLOCK + R.blocks(a.shape[1])
    return n ** 0.5 * R.F32 * ((a * a) @ (w * w).t()).sqrt() + 4 * R.F32 * (a @ w.t()).abs()


def swiglu_noise(a, w):
    half = w.shape[0] // 2
    g, u = a @ w[:half].t(), a @ w[half:].t()
    s = g * torch.sigmoid(g)
    return s * u, 1.1 * product_noise(a, w[:half]) * u.abs() + s.abs() * product_noise(a, w[half:]) + 8 * R.F32 * (s * u).abs()


def quantized_noise(v, dv):
    """(v in 8 bits, expected square of its error) for values expected within dv."""
    _, per = R.group_max(v)
    safe = torch.where(per > 0, per, 1.0)
    t = v * R.TOP / safe
    q = R.e4m3_round(t) * per / R.TOP
    step = R.e4m3_step(t) * per / R.TOP
    _, dper = R.group_max(dv)
    d = dv + v.abs() * (dper / safe + 2 * R.F32)          # of the quotient: the value and the group's largest
    return q, d * step + (q * (dper / safe + 2 * R.F32)) ** 2


def layer_noise(experts, n_local, x, ids, w, shared_range=(0, 0)):
    """(outputs, expected squares of their errors before the last rounding) of a layer for 8-bit tokens of values x; experts as Layer.experts."""
    T, H = x.shape[0], experts[0][5].shape[0]
    y, e2 = torch.zeros(T, H, dtype=torch.float64), torch.zeros(T, H, dtype=torch.float64)
    for i, e in enumerate(experts):
        if i < n_local:
            token, col = (ids == i).nonzero(as_tuple=True)
            wt = w[token, col].double()[:, None]
        else:
            token = torch.arange(*shared_range)
            wt = torch.ones(len(token), 1, dtype=torch.float64)
        if len(token) == 0:
            continue
        h, dh = swiglu_noise(x[token], e[2])
        v, ev2 = quantized_noise(h, dh)
        o = v @ e[5].t()
        y.index_add_(0, token, wt * o)
        e2.index_add_(0, token, wt ** 2 * (ev2 @ (e[5] ** 2).t() + product_noise(v, e[5]) ** 2 + (4 * R.F32 * o) ** 2))
    return y, e2


def bf16(y):
    return y.float().bfloat16().double()


def excess(out, y, e2=0.0):
    """|out - y|^2 over what is expected of it (bf16 results): above SLACK something else than roundings is in it."""
    expected = ((bf16(y) - y) ** 2 + e2).sum()
    return (((out.double() - y) ** 2).sum() / expected).item()
