"""The workspace of the SwiGLU product for every number of rows up to a limit."""
import pytest
import torch

from paper_2510_02613_amd import binding as B

SHAPES = [(1408, 2048), (2048, 7168), (768, 2048), (16, 16), (32768, 128), (144, 272)]


@pytest.mark.parametrize("inter,k", SHAPES)
def test_the_largest_need_of_fewer_rows(inter, k):
    need = [B.moe_scaled_swiglu_workspace_bytes(m, inter, k) for m in range(1, 4001)]
    most = 0
    for m, n in enumerate(need, 1):
        most = max(most, n)
        assert B.moe_scaled_swiglu_max_workspace_bytes(m, inter, k) == most


def test_a_buffer_for_the_largest_batch_serves_the_smaller_ones():
    """Sized at 4096 rows, which need no workspace themselves."""
    inter, k, most = 1408, 2048, 4096
    assert B.moe_scaled_swiglu_workspace_bytes(most, inter, k) == 0
    size = B.moe_scaled_swiglu_max_workspace_bytes(most, inter, k)
    for m in (1, 17, 300):
        assert 0 < B.moe_scaled_swiglu_workspace_bytes(m, inter, k) <= size


def test_sizes_that_are_refused():
    for sizes in ((0, 256, 2048), (4, 0, 2048), (4, 256, 0), (-1, 256, 256), (1 << 22, 256, 256), (4, 1 << 22, 256)):
        assert B.moe_scaled_swiglu_max_workspace_bytes(*sizes) == 0
    assert B.moe_scaled_swiglu_max_workspace_bytes(1 << 21, 16, 16) >= B.moe_scaled_swiglu_workspace_bytes(1 << 20, 16, 16)


@pytest.mark.gpu
def test_one_workspace_for_every_batch():
    from paper_2510_02613_amd import scaled as S
    inter, k = 1408, 2048
    g = torch.Generator(device="cuda").manual_seed(1)
    w, ws = S.quantize(torch.randn(2 * inter, k, device="cuda", generator=g) * 0.02, block_rows=128)
    space = S.swiglu_workspace(4096, inter, k, up_to=True)
    for m in (1, 17, 300, 4096):
        a, s = S.quantize(torch.randn(m, k, device="cuda", generator=g))
        want = S.swiglu(a, s, w, ws)
        got = S.swiglu(a, s, w, ws, workspace=space)
        assert torch.equal(got.q.view(torch.uint8), want.q.view(torch.uint8)) and torch.equal(got.scale, want.scale)
