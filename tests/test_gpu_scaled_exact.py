"""Products of the 8-bit path are exact and their sums fp32's unless the caller asks for the 8-bit matrix instructions."""
import pytest
import torch

import scaled_ref as R
from test_gpu_scaled import MATMUL, eight_bit_rows, eight_bit_weights, randn, strided

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn


def cancelling(m, n, k):
    """Rows and weights whose large products, 448 * 448, cancel pair by pair, with products of 4 between them: a sum of k is k / 2 * 4, a whole
    number as every partial sum (below 2^24 in any order: exact in fp32), of which the 8-bit instructions keep nothing."""
    a, w = torch.full((m, k), 2.0), torch.full((n, k), 2.0)
    a[:, ::2] = 448.0
    w[:, 0::4], w[:, 2::4] = 448.0, -448.0
    return a.to(E4M3).cuda(), w.to(E4M3).cuda()


# streamed, and tiles of every number of 32-row parts
@pytest.mark.parametrize("m,n,k", [(1, 256, 128), (17, 136, 512), (300, 1000, 256), (2000, 1032, 512), (2001, 520, 128), (3000, 1000, 400), (5000, 1104, 272), (9000, 2100, 112)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_small_products_beside_large_ones_that_cancel(m, n, k, dtype):
    from paper_2510_02613_amd import scaled as S
    a, w = cancelling(m, n, k)
    ones = lambda *s: torch.ones(s, device="cuda")  # noqa: E731
    add = randn(m, m, n).to(dtype)
    out = S.matmul(a, ones(m, R.blocks(k)), w, ones(R.blocks(n), R.blocks(k)), out_dtype=dtype)
    want = torch.full((m, n), 2.0 * k, dtype=dtype)
    assert torch.equal(out.cpu(), want)
    out = S.matmul(a, ones(m, R.blocks(k)), w, ones(R.blocks(n), R.blocks(k)), add=strided(add, (n + 7) // 8 * 8))
    assert torch.equal(out.cpu(), (2.0 * k + add.float()).to(dtype))


@pytest.mark.parametrize("m,n,k", MATMUL)
def test_matmul_fast(m, n, k):
    """The caller's choice of the 8-bit instructions: what they may drop, and one rounding."""
    from paper_2510_02613_amd import scaled as S
    q, scale, a = eight_bit_rows(m + k, m, k, zero_rows=True)
    wq, ws, w = eight_bit_weights(n + k, n, k)
    y, dy = R.product(a, torch.zeros_like(a), w, fast=True)
    ld = (n + 7) // 8 * 8 + 8
    add = randn(m * n, m, n).bfloat16()
    for with_add in (False, True):
        out = strided(torch.zeros(m, n, dtype=torch.bfloat16), ld)
        if with_add:
            out.copy_(add.cuda())
        S.matmul(q.cuda(), scale.cuda(), wq.cuda(), ws.cuda(), add=out if with_add else None, out=out, fast=True)
        want = y + add.double() if with_add else y
        off = (out.cpu().double() - want).abs() - (dy + R.F32 * want.abs()) * (1 + R.BF16) - R.BF16 * want.abs()
        assert (off <= 0).all(), (with_add, off.max().item())
        assert torch.isnan(out.as_strided((m, ld - n), (ld, 1), n)).all()


def test_only_those_who_ask_get_the_8bit_instructions():
    from gpu_util import kernels_of
    from paper_2510_02613_amd import scaled as S
    m, n, k = 3000, 1000, 400
    q, scale, _ = eight_bit_rows(1, m, k)
    w, ws, _ = eight_bit_weights(2, n, k)
    q, scale, w, ws, out = q.cuda(), scale.cuda(), w.cuda(), ws.cuda(), torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    names = [kernels_of(lambda stream: S.matmul(q, scale, w, ws, out=out, fast=f, stream=stream)) for f in (False, True)]
    assert [len(n_) for n_ in names] == [1, 1]
    assert "k_scaled_tiles<false, true, 4" in names[0][0] and "k_scaled_tiles<false, false, 8" in names[1][0], names


@pytest.mark.parametrize("m,n,k", [(1000, 1032, 1152), (4500, 2100, 1152), (9000, 4100, 384)])
def test_a_row_is_the_same_wherever_it_stands_fast(m, n, k):
    from paper_2510_02613_amd import scaled as S
    q, scale, _ = eight_bit_rows(m + k, m // 2, k)
    q, scale = torch.cat([q.view(torch.uint8)] * 2).view(q.dtype).cuda(), torch.cat([scale] * 2).cuda()
    wq, ws, _ = eight_bit_weights(n + k, n, k)
    out = S.matmul(q, scale, wq.cuda(), ws.cuda(), fast=True)
    assert torch.equal(out[:m // 2], out[m // 2:])
