"""Where 4 bits stand for more than fp32 and bf16 hold: 2^128 and above are infinities, in the values that are left and in the weights of a product."""
import pytest
import torch

from test_gpu_four_bit import BF16, F32, Q

pytestmark = pytest.mark.gpu

STEPS = [0, 0.5, 1, 1.5, 2, 3, 4, 6]


@pytest.mark.parametrize("dt", [BF16, F32])
def test_quantize_next_to_the_largest_numbers(dt):
    """From 3.5 * 2^126 on the nearest of 3 and 4 times 2^126 is the upper one, 2^128.  3 * 2^126 itself is 6 * 2^125, and takes that power."""
    tops = [3.0, 3.25, 3.484375, 3.5, 3.75, 3.984375]              # times 2^126; all of them numbers of bf16
    x = torch.zeros(len(tops), 32, dtype=F32)
    x[:, 0] = torch.tensor(tops) * 2.0 ** 126
    x[:, 1], x[:, 2] = -x[:, 0], 2.0 ** 126
    x = x.to(dt)
    assert torch.isfinite(x).all()
    values = torch.zeros_like(x).cuda()
    q, scale = Q().quantize(x.cuda(), values=values)
    assert scale[:, 0].tolist() == [252] + [253] * 5
    up = torch.tensor([t >= 3.5 for t in tops])
    code, one = torch.where(up, 6, 5).to(torch.uint8), torch.full((len(tops),), 2, dtype=torch.uint8)
    code[0], one[0] = 7, 4
    assert torch.equal(q[:, 0].cpu(), code + 16 * (code + 8)) and torch.equal(q[:, 1].cpu(), one) and not q[:, 2:].any()
    values = values.cpu()
    assert torch.equal(values[:, 0], torch.where(up, float("inf"), 3 * 2.0 ** 126).to(dt)) and torch.equal(values[:, 1], -values[:, 0])
    assert values[:, 2].eq(2.0 ** 126).all() and not values[:, 3:].any()


@pytest.mark.parametrize("power", [252, 253, 254])
def test_weights_next_to_the_largest_numbers(power):
    """One code in each weight row, times 2^-20: exact where the weight is below 2^128, infinite from there."""
    q = torch.zeros(16, 16, dtype=torch.uint8)
    q[:, 0] = torch.arange(16, dtype=torch.uint8)
    scale = torch.full((16, 1), power, dtype=torch.uint8)
    a = torch.zeros(2, 32, dtype=BF16)
    a[0, 0] = 2.0 ** -20
    got = Q().matmul(a.cuda(), q.cuda(), scale.cuda(), out_dtype=F32).cpu()
    weights = torch.tensor(STEPS + [-s for s in STEPS], dtype=torch.float64) * 2.0 ** (power - 127)
    fine = weights.abs() < 2.0 ** 128
    assert fine.sum().item() == {252: 16, 253: 12, 254: 8}[power]
    assert torch.equal(got[0][fine].double(), weights[fine] * 2.0 ** -20)
    assert torch.equal(got[0][~fine].double(), torch.sign(weights[~fine]) * float("inf"))
    assert not got[1][fine].any() and got[1][~fine].isnan().all()       # nothing times an infinity
