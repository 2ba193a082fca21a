"""A layer in pieces (sorted tokens, 4-bit products, their weighted sums), without a GPU: registers and scratch memory of the kernels, from the metadata of the
built library, and memory that a call allocates itself, which belongs to the stream it works on."""
import re

import pytest
import torch

from test_kernel_resources import _waves, kernels  # noqa: F401
from test_stream_allocations import Recorder, SIDE


@pytest.mark.parametrize("pattern,waves", [
    (r"k_sort_count", 8), (r"k_sort_scan", 8), (r"k_sort_place<.*>", 8), (r"k_combine_rows<.*>", 8), (r"k_combine_rows_backward<.*>", 7), (r"k_four_quantize<.*>", 8),
    (r"k_four_rows<(true|false), 8, 1, 1, .*>", 4),        # up to 16 rows a group: two workgroups of eight wavefronts a compute unit
    (r"k_four_rows<(true|false), 4, 1, 1, .*>", 3), (r"k_four_rows<false, 4, 1, 2, .*>", 3), (r"k_four_rows<true, 4, 1, 2, 1, .*>", 3),
    (r"k_four_rows<.*>", 2)])
def test_wavefronts_per_simd(kernels, pattern, waves):  # noqa: F811
    mine = {n: k for n, k in kernels.items() if re.fullmatch(pattern, n)}
    assert mine
    for name, k in mine.items():
        assert _waves(k) >= waves, (name, k[".vgpr_count"])
        assert k[".private_segment_fixed_size"] <= 16 and k[".vgpr_spill_count"] <= 2, name     # an address or two at most, outside the loops


@pytest.fixture
def rec(monkeypatch):
    return Recorder(monkeypatch)


def on_the_cpu(monkeypatch, rec, module, *names):
    monkeypatch.setattr(module, "_device_of", lambda t: -1)
    monkeypatch.setattr(module, "_current_device", lambda: -1)
    monkeypatch.setattr(module, "_current_stream", lambda dev: 7)
    rec.library(monkeypatch, module.B, *names)
    return module



def z(*shape, dt=torch.uint8):
    return torch.zeros(*shape).to(dt)


BF16, I32 = torch.bfloat16, torch.int32
FOUR = {
    "quantize": (2, lambda Q, **kw: Q.quantize(z(4, 256, dt=BF16), **kw)),
    "matmul": (1, lambda Q, **kw: Q.matmul(z(4, 256, dt=BF16), z(64, 128), z(64, 8), **kw)),
    "swiglu": (1, lambda Q, **kw: Q.swiglu(z(4, 256, dt=BF16), z(64, 128), z(64, 8), **kw)),
}
PIECES = {
    "sort": (4, lambda D, **kw: D.sort_tokens(z(4, 64, dt=BF16), z(4, 2, dt=I32), 3, **kw)),
    "sort, counted first": (5, lambda D, **kw: D.sort_tokens(z(600, 64, dt=BF16), z(600, 8, dt=I32), 3, **kw)),
    "combine": (1, lambda D, **kw: D.combine_tokens(z(8, 64, dt=BF16), D.Order(None, None, z(4, 2, dt=I32)), **kw)),
}


@pytest.mark.parametrize("call", sorted(FOUR))
@pytest.mark.parametrize("side", [None, SIDE])
def test_products_allocate_on_their_stream(monkeypatch, rec, call, side):
    from paper_2510_02613_amd import four_bit
    Q = on_the_cpu(monkeypatch, rec, four_bit, "moe_four_bit_quantize", "moe_four_bit_matmul", "moe_four_bit_swiglu")
    n, run = FOUR[call]
    run(Q, stream=side)
    assert len(rec.calls) == 1 and rec.calls[0][0][1] == (7 if side is None else side.cuda_stream)
    assert [at for at, _ in rec.allocations] == [side] * n


@pytest.mark.parametrize("call", sorted(PIECES))
@pytest.mark.parametrize("side", [None, SIDE])
def test_sorted_tokens_allocate_on_their_stream(monkeypatch, rec, call, side):
    from paper_2510_02613_amd import dispatch
    D = on_the_cpu(monkeypatch, rec, dispatch, "moe_sort_tokens", "moe_combine_tokens")
    real = D.sort_workspace
    monkeypatch.setattr(D, "sort_workspace", lambda t, k, n, device: real(t, k, n, "cpu"))
    n, run = PIECES[call]
    run(D, stream=side)
    assert len(rec.calls) == 1 and rec.calls[0][0][1] == (7 if side is None else side.cuda_stream)
    assert [at for at, _ in rec.allocations] == [side] * n


def test_given_results_of_products_count_as_changed(monkeypatch, rec):
    from paper_2510_02613_amd import four_bit
    Q = on_the_cpu(monkeypatch, rec, four_bit, "moe_four_bit_quantize", "moe_four_bit_matmul", "moe_four_bit_swiglu")
    x, q, scale, out, half = z(4, 256, dt=BF16), z(4, 128), z(4, 8), z(4, 64, dt=BF16), z(4, 32, dt=BF16)
    before = [t._version for t in (x, q, scale, out, half)]
    Q.quantize(x, q=q, scale=scale, values=x)
    Q.matmul(x, z(64, 128), z(64, 8), out=out)
    Q.swiglu(x, z(64, 128), z(64, 8), out=half)
    assert [t._version for t in (x, q, scale, out, half)] == [v + 1 for v in before]
    with torch.inference_mode():
        own = z(4, 64, dt=BF16)
        assert Q.matmul(x, z(64, 128), z(64, 8), out=own) is own


def test_given_results_count_as_changed(monkeypatch, rec):
    from paper_2510_02613_amd import dispatch
    D = on_the_cpu(monkeypatch, rec, dispatch, "moe_sort_tokens", "moe_combine_tokens")
    rows, order, out = z(8, 64, dt=BF16), D.Order(z(4, dt=I32), z(8, dt=I32), z(4, 2, dt=I32)), z(4, 64, dt=BF16)
    before = [t._version for t in (rows, *order, out)]
    D.sort_tokens(out.clone(), order.row, 3, rows=rows, order=order)
    D.combine_tokens(rows, order, out=out)
    assert [t._version for t in (rows, *order, out)] == [v + 1 for v in before]
