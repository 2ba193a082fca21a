"""The operators of the 8-bit path in 64 bits on the CPU, with how far a computation in fp32 may be from them.

Roundings are off by half a step at most: bf16 2^-8 of the value, fp32 2^-24, e4m3 2^-4 (2^-10 below 2^-6).
"""
import torch

BLOCK, TOP = 128, 448.0
F32, BF16 = 2.0 ** -24, 2.0 ** -8
HALF_STEP = {torch.float32: F32, torch.bfloat16: BF16}


def blocks(n):
    return (n + BLOCK - 1) // BLOCK


def spread_rows(scale, cols):
    return scale.double().repeat_interleave(BLOCK, 1)[:, :cols]


def spread_blocks(scale, n, k):
    return scale.double().repeat_interleave(BLOCK, 0)[:n].repeat_interleave(BLOCK, 1)[:, :k]


def e4m3_step(t):
    """Distance of neighbouring e4m3 values around |t|."""
    e = torch.frexp(t.abs().clamp(min=2.0 ** -6))[1] - 1      # 2^e <= |t|
    return torch.ldexp(torch.ones_like(t), e - 3)


def e4m3_round(t):
    """|t| <= 448 to the nearest e4m3 value, ties to even, in the type of t."""
    step = e4m3_step(t)
    return torch.round(t / step) * step     # torch.round: half to even; the quotient is 8 .. 16, so that even is the even mantissa


def group_max(v, block_rows=1):
    """Largest magnitude of each group, as one value per element."""
    rows, cols = v.shape
    rb = -(-rows // block_rows)
    p = torch.zeros(rb * block_rows, blocks(cols) * BLOCK, dtype=v.dtype)
    p[:rows, :cols] = v.abs()
    top = p.view(rb, block_rows, blocks(cols), BLOCK).amax((1, 3))
    return top, top.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :cols]


def check_quantized(q, scale, v, dv, block_rows=1):
    """q, scale (of the GPU) against values v known to within dv: every scale is max / 448 to within the largest dv of the group, and
    every q * scale is within half an e4m3 step of a value that v may be."""
    top, per = group_max(v, block_rows)
    dtop, dper = group_max(dv, block_rows)
    assert (scale.double() - top / TOP).abs().le((dtop + 4 * F32 * top) / TOP).all()
    s = scale.double().repeat_interleave(block_rows, 0)[:v.shape[0]].repeat_interleave(BLOCK, 1)[:, :v.shape[1]]
    got = q.double() * s
    worst = (v.abs() + dv) * (1 + 8 * F32)
    half = torch.where(s > 0, 0.5 * s * e4m3_step(worst / torch.where(s > 0, s, 1.0)), 0.0)
    off = (got - v).abs() - (half * (1 + 2.0 ** -20) + dv + 8 * F32 * v.abs())
    assert (off <= 0).all(), f"an 8-bit value is {off.max().item():.3e} further off than its rounding"


def quantize(v, dv):
    """(value, how far off) of v in 8 bits, v known to within dv: where no e4m3 border lies within dv of the quotient the byte is certain."""
    _, per = group_max(v)
    _, dper = group_max(dv)
    safe = torch.where(per > 0, per, 1.0)
    t = v * TOP / safe
    dt = (dv + v.abs() * dper / safe + 8 * F32 * v.abs()) * TOP / safe
    lo, hi = e4m3_round((t - dt).clamp(-TOP, TOP)), e4m3_round((t + dt).clamp(-TOP, TOP))
    s = per / TOP
    value = e4m3_round(t) * s
    off = torch.maximum((hi * s - value).abs(), (value - lo * s).abs()) + (value.abs() + s * 2.0 ** -6) * (dper / safe + 8 * F32)
    return value, off


# The 8-bit matrix instructions add their products in groups of eight, each product cut to a multiple of 2^-14 of the power of two of
# the largest (measured: beside 448^2, whose power is 2^17, seven products of 4 vanish and seven of 8 count in full): eight times
# that of the largest product, per group.
FAST = 8 * 2.0 ** -14


def product(a, da, w, fast=False):
    """(a w^T, how far off): a known to within da, w exact.  Sums of 128 products, then of the blocks, then two scales, in fp32; whatever the
    order, a sum of n terms is off by n half steps of the sum of their magnitudes.  fast: where the 8-bit instructions may be used.  In one
    block all products have the same scales, so that a block's largest product per eight bounds what is dropped."""
    y = a @ w.t()
    mag = a.abs() @ w.abs().t()
    off = (BLOCK + blocks(a.shape[1]) + 8) * F32 * mag + da @ w.abs().t()
    if fast:
        # the largest product of any eight is at most their largest a times their largest w; which eight belong together is not known: the largest
        # of a's block times w's block, for each of the block's 16 groups of eight, and never more than all of the block's magnitudes
        for k0 in range(0, a.shape[1], BLOCK):
            pa, pw = a[:, k0:k0 + BLOCK].abs(), w[:, k0:k0 + BLOCK].abs()
            most = torch.minimum(pa @ pw.t(), 16 * pa.amax(1, keepdim=True) * pw.amax(1, keepdim=True).t())
            off = off + FAST * most
    return y, off


def swiglu(a, da, w, fast=False):
    """(silu(g) u, how far off) of gate rows and up rows of w; silu's slope is below 1.1, its exponential and reciprocal are off by a few steps each."""
    half = w.shape[0] // 2
    g, dg = product(a, da, w[:half], fast)
    u, du = product(a, da, w[half:], fast)
    s = g * torch.sigmoid(g)
    h = s * u
    return h, 1.1 * dg * (u.abs() + du) + s.abs() * du + h.abs() * 16 * F32 * (1 + g.abs() / 8)
