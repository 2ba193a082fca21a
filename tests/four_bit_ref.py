"""The 4-bit operators in 64 bits on the CPU, with how far a computation in fp32 may be from them.

Roundings are off by half a step at most: bf16 2^-8 of the value, fp32 2^-24.
"""
import torch

GROUP = 32
F32, BF16 = 2.0 ** -24, 2.0 ** -8
HALF_STEP = {torch.float32: F32, torch.bfloat16: BF16}
STEPS = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)


def values(q, scale):
    """What codes [..., n, k / 2] and powers [..., n, k / 32] stand for."""
    q, scale = q.cpu().view(torch.uint8), scale.cpu().view(torch.uint8)
    codes = torch.stack((q & 15, q >> 4), -1).flatten(-2).long()
    power = torch.where(scale == 255, float("nan"), torch.ldexp(torch.ones((), dtype=torch.float64), scale.int() - 127))
    return STEPS[codes] * power.repeat_interleave(GROUP, -1)


def quantize(x):
    """(codes one by one [rows, cols], powers), by trying every code: the nearest, of two as near the even one."""
    x = x.double()
    rows, cols = x.shape
    codes, powers = torch.zeros(rows, cols, dtype=torch.uint8), torch.zeros(rows, cols // GROUP, dtype=torch.uint8)
    order = [0, 2, 4, 6, 1, 3, 5, 7]                             # even codes first: argmin takes the first of equals
    for b in range(cols // GROUP):
        v = x[:, b * GROUP:(b + 1) * GROUP]
        top = v.abs().amax(1)
        p = torch.full((rows,), -127.0, dtype=torch.float64)
        while (top.nan_to_num(0, 0) > 6 * 2.0 ** p).any():
            p = torch.where(top.nan_to_num(0, 0) > 6 * 2.0 ** p, p + 1, p)
        t = v.abs() / (2.0 ** p)[:, None]
        off = (t[..., None] - STEPS[order]).abs()
        code = torch.tensor(order, dtype=torch.uint8)[off.argmin(-1)] + 8 * torch.signbit(v).to(torch.uint8)
        fine = torch.isfinite(v).all(1)
        codes[:, b * GROUP:(b + 1) * GROUP] = torch.where(fine[:, None], code, 0)
        powers[:, b] = torch.where(fine, (p + 127).to(torch.uint8), 255)
    return codes, powers


def packed(codes):
    return codes[:, 0::2] + 16 * codes[:, 1::2]


def product(a, da, w):
    """(a w^T, how far off): a known to within da, w exact; a sum of k products is off by k half steps of the sum of their magnitudes, whatever the
    order, and a dozen of them are partial sums of other wavefronts."""
    y = a @ w.t()
    mag = a.abs() @ w.abs().t()
    return y, (a.shape[1] + 12) * F32 * mag + da @ w.abs().t()


def swiglu(a, da, w):
    """(silu(g) u, how far off); silu's slope is below 1.1, its exponential and reciprocal are off by a few steps each."""
    half = w.shape[0] // 2
    g, dg = product(a, da, w[:half])
    u, du = product(a, da, w[half:])
    s = g * torch.sigmoid(g)
    h = s * u
    return h, 1.1 * dg * (u.abs() + du) + s.abs() * du + h.abs() * 16 * F32 * (1 + g.abs() / 8)


def check(got, want, off, what=""):
    """got (rounded once to its type) against values known to within off; what is NaN or infinite has to be so."""
    g = got.double().cpu()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(g), fine), what
    worst = ((g - want).abs() - off - HALF_STEP[got.dtype] * (want.abs() + off))[fine]
    assert not worst.numel() or worst.max().item() <= 1e-40, f"{what}: {worst.max().item():.3e} further off than its roundings"


def check_norm(got, want, rounded):
    """The error's norm over the result's: independent roundings of fp32 sums (the longest here have some 7000 terms) stay below 2^-20, one of bf16 is
    at most 2^-8 / sqrt(3) of every value, and typically 2^-9.2."""
    rel = ((got.double().cpu() - want).norm() / want.norm()).item()
    assert rel <= (2.0 ** -8.7 if rounded is torch.bfloat16 else 2.0 ** -20), rel
