"""The norm bounds of the 8-bit path's GPU tests tell roundings from mistakes: mistakes are planted in the oracle, on the CPU."""
import pytest
import torch

import scaled_norms as N
import scaled_ref as R
from test_gpu_scaled import eight_bit_rows, eight_bit_weights
from test_gpu_scaled_layer import SHAPES, weights


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


class Oracle:
    """Experts, tokens and a routing as the GPU tests make them, and a pass in fp32 with a mistake."""

    def __init__(self, shape, T, seed):
        s = self.s = SHAPES[shape]
        self.experts = [weights(1000 * seed + 10 * e, 2 * s["I"], s["H"], parts=2) + weights(1000 * seed + 10 * e + 5, s["H"], s["I"]) for e in range(s["n_local"])]
        g = torch.Generator().manual_seed(T)
        self.ids = torch.rand(T, s["E"], generator=g).topk(s["k"], 1).indices.to(torch.int32)
        self.w = torch.rand(T, s["k"], generator=g) + 0.1
        x = randn(9, T, s["H"]).bfloat16().double()
        _, per = R.group_max(x)
        self.x = R.e4m3_round(x * 448 / per) * per / 448
        self.y, self.e2 = N.layer_noise(self.experts, s["n_local"], self.x, self.ids, self.w)

    def in_fp32(self, weight=lambda w: w, rows=lambda o: o):
        products = lambda a, w: a.float() @ w.float().t()  # noqa: E731
        y = torch.zeros(self.y.shape)
        for i, e in enumerate(self.experts):
            token, col = (self.ids == i).nonzero(as_tuple=True)
            half = e[2].shape[0] // 2
            g, u = products(self.x[token], e[2][:half]), products(self.x[token], e[2][half:])
            h = g * torch.sigmoid(g) * u
            _, per = R.group_max(h)
            v = R.e4m3_round((h * 448 / per).clamp(-448, 448)) * (per / 448)
            y.index_add_(0, token, weight(self.w[token, col])[:, None] * rows(products(v, e[5])))
        return y


@pytest.mark.parametrize("shape,T", [(2, 130), (3, 300), (4, 200)])
def test_layers(shape, T):
    o = Oracle(shape, T, shape)
    assert N.excess(N.bf16(o.in_fp32()), o.y, o.e2) < N.SLACK                                     # fp32 with one rounding: inside
    # expert outputs rounded to bf16, weights off by one per cent, weights rounded to bf16.  (Products with the precision of the 8-bit matrix instructions are
    # below the roundings here; sums whose large products cancel tell them apart.)
    for mistake in (dict(rows=lambda r: r.bfloat16().float()), dict(weight=lambda w: w * 1.01), dict(weight=lambda w: w.bfloat16().float())):
        assert N.excess(N.bf16(o.in_fp32(**mistake)), o.y, o.e2) > N.SLACK, mistake
    for factor in (1.01, 1.005, 0.995):
        assert N.excess(N.bf16(o.y * factor), o.y, o.e2) > N.SLACK


@pytest.mark.parametrize("m,n,k", [(300, 1000, 48), (513, 256, 512), (257, 520, 640), (2000, 64, 1168)])
def test_products(m, n, k):
    _, _, a = eight_bit_rows(m, m, k)
    _, _, w = eight_bit_weights(k, n, k)
    y, e2 = a @ w.t(), N.product_noise(a, w) ** 2
    assert N.excess(N.bf16(a.float() @ w.float().t()), y, e2) < N.SLACK
    for factor in (1.005, 0.995):
        assert N.excess(N.bf16(y * factor), y, e2) > N.SLACK
