"""The operators that sort tokens by expert and add them up again, on the CPU: the order by its definition, sums in 64 bits with how far fp32 may be off.

Roundings are off by half a step at most: bf16 2^-8 of the value, fp32 2^-24.
"""
import torch

F32 = 2.0 ** -24
HALF_STEP = {torch.float32: F32, torch.bfloat16: 2.0 ** -8}


def groups(ids, n_groups, expert_map=None):
    """The group of every assignment, n_groups where it has none."""
    g = ids.flatten().long()
    if expert_map is not None:
        there = (g >= 0) & (g < len(expert_map))
        g = torch.where(there, expert_map.long()[g.clamp(0, len(expert_map) - 1)], -1)
    return torch.where((g >= 0) & (g < n_groups), g, n_groups)


def order(ids, n_groups, expert_map=None):
    """(offsets, source, row), one assignment after the other."""
    g = groups(ids, n_groups, expert_map).tolist()
    of = [[] for _ in range(n_groups + 1)]
    for a, s in enumerate(g):
        of[s].append(a)
    offsets, source, row = [0], [-1] * len(g), [-1] * len(g)
    for s in range(n_groups):
        for i, a in enumerate(of[s]):
            source[offsets[-1] + i] = a
            row[a] = offsets[-1] + i
        offsets.append(offsets[-1] + len(of[s]))
    return (torch.tensor(offsets, dtype=torch.int32), torch.tensor(source, dtype=torch.int32), torch.tensor(row, dtype=torch.int32).view(ids.shape))


def combine(y, row, weights=None):
    """(out, how far fp32 sums may be off): a sum of n products is off by n half steps of the sum of their magnitudes, whatever the order."""
    T, k = row.shape
    there = (row >= 0)[..., None]
    parts = torch.where(there, y.double()[row.clamp(min=0).flatten().long()].view(T, k, -1), 0.0)
    if weights is not None:
        parts = parts * torch.where(row >= 0, weights.double(), 0.0)[..., None]
    return parts.sum(1), (k + 1) * F32 * parts.abs().sum(1)


def backward(grad, y, row, weights=None):
    """(dy, off, dw, off): a product and its roundings; a dot product, 64 columns side by side in fp32 and then their sums."""
    T, k = row.shape
    cols = grad.shape[1]
    dy, dw, mag = torch.zeros(T * k, cols, dtype=torch.float64), torch.zeros(T, k, dtype=torch.float64), torch.zeros(T, k, dtype=torch.float64)
    for t in range(T):
        for j in range(k):
            r = int(row[t, j])
            if r >= 0:
                g = grad[t].double()
                dy[r] = g * (1.0 if weights is None else float(weights[t, j]))
                dw[t, j], mag[t, j] = (g * y[r].double()).sum(), (g * y[r].double()).abs().sum()
    return dy, F32 * dy.abs(), dw, (cols / 64 + 16) * F32 * mag


def check(got, want, off, what):
    """got (rounded once to its type) against values known to within off."""
    g = got.double().cpu()
    assert torch.isfinite(g).all(), what
    worst = ((g - want).abs() - off - HALF_STEP[got.dtype] * (want.abs() + off)).max().item() if g.numel() else 0.0
    assert worst <= 1e-40, f"{what}: {worst:.3e} further off than its roundings"
