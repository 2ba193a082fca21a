"""Passes of a layer with 8-bit experts: exact products and fp32 sums unless the caller asks for the 8-bit matrix instructions."""
import numpy as np
import pytest
import torch

import scaled_ref as R
from test_gpu_scaled_layer import Layer

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn


def cancelling_layer(H, I, E, max_tokens):
    """Experts in whose products large numbers cancel and small ones are left.
    GEMM-1: tokens (448, 2, 448, 2, ..), gate rows and the up rows of even columns (448, 2, -448, 2, ..): of products 448 * 448 and 4 a sum of H / 2 * 4
    is left; the up rows of odd columns hold 2^-7 in the places of 2 and nothing else: a 256th of it.  So h is (448, 1.75, 448, 1.75, ..) times its scale.
    GEMM-2: rows (448, 2, -448, 2, ..): of 448 * 448 and 3.5 a sum of I / 2 * 3.5 is left.  All sums are exact in fp32, in any order."""
    from paper_2510_02613_amd.layer import MoELayer, ScaledExperts

    def pattern(n):
        v = torch.full((n,), 2.0)
        v[0::4], v[2::4] = 448.0, -448.0
        return v
    w13 = pattern(H).repeat(2 * I, 1)
    odd = torch.zeros(H)
    odd[1::2] = 2.0 ** -7
    w13[I + 1::2] = odd
    w2 = pattern(I).repeat(H, 1)
    s13 = torch.full((2 * R.blocks(I), R.blocks(H)), 2.0 / H)                # gate = up = 4 for tokens of scale 1
    pools = ScaledExperts(w13.to(E4M3).repeat(E, 1, 1).cuda(), s13.repeat(E, 1, 1).contiguous().cuda(), w2.to(E4M3).repeat(E, 1, 1).cuda(),
                          (torch.arange(1, E + 1)[:, None, None] * torch.ones(1, R.blocks(H), R.blocks(I))).contiguous().cuda())
    layer = MoELayer(hidden=H, inter=I, n_experts=E, top_k=2, n_slots=E, max_tokens=max_tokens, router_w=np.zeros((E, H), np.float32), scaled=pools)
    layer.set_expert_map(list(range(E)))
    x = torch.full((max_tokens, H), 2.0)
    x[:, ::2] = 448.0
    return layer, x.to(E4M3).cuda(), torch.ones(max_tokens, R.blocks(H)).cuda()


@pytest.mark.parametrize("T,tiles", [(3, False), (400, True), (4000, True)])
def test_small_products_beside_large_ones_that_cancel(T, tiles):
    from gpu_util import kernels_of
    H, I, E = 256, 256, 96
    layer, x, s = cancelling_layer(H, I, E, T)
    ids = torch.randint(E, (T, 2), generator=torch.Generator().manual_seed(1)).to(torch.int32)
    w = torch.rand(T, 2, generator=torch.Generator().manual_seed(2)) + 0.5
    out, d_ids, d_w = torch.empty(T, H, dtype=torch.bfloat16, device="cuda"), ids.cuda(), w.cuda()
    run = lambda stream=None: layer.forward_scaled(x, s, topk_ids=d_ids, topk_w=d_w, out=out, stream=stream)  # noqa: E731
    names = kernels_of(run)
    assert sum("k_scaled_tiles" in n for n in names) == (2 if tiles else 0) and sum("k_scaled_stream" in n for n in names) == (0 if tiles else 2)
    run()
    h = 4.0 / (1.0 + np.exp(-4.0)) * 4.0
    # 1.75 I times h's scale times the expert's number times the weight; fp32: silu some steps, a handful of products and one addition
    want = ((ids.double() + 1) * w.double()).sum(1, keepdim=True) * (1.75 * I * h / 448.0)
    assert ((out.cpu().double() - want).abs() <= (R.BF16 + 64 * R.F32) * want).all()
    layer.close()


SHAPE = dict(H=256, I=272, E=64, k=3, n_local=60, n_shared=1, seed=31)


def test_only_passes_that_ask_get_the_8bit_instructions():
    from gpu_util import kernels_of
    from paper_2510_02613_amd import binding as B
    T = 300
    L = Layer(**SHAPE)
    ids, w = L.routing(7, T)
    x, q, scale, _ = L.tokens(9, T)
    x, q, scale, ids, w, out = x.cuda(), q.cuda(), scale.cuda(), ids.cuda(), w.cuda(), torch.empty(T, L.H, dtype=torch.bfloat16, device="cuda")
    want = {0: ("k_scaled_tiles<true, true, 4", "k_scaled_tiles<false, true, 4, float", "k_scaled_combine<true"),
            B.MOE_FLAG_FAST_PRODUCTS: ("k_scaled_tiles<true, false, 8", "k_scaled_tiles<false, false, 8", "k_scaled_combine<false")}
    for flags, kernels in want.items():
        for call in (lambda stream: L.layer.forward_scaled(q, scale, topk_ids=ids, topk_w=w, out=out, flags=flags, stream=stream),
                     lambda stream: L.layer.forward_routed(x, ids, w, out=out, flags=flags, stream=stream),
                     lambda stream: L.layer.forward(x, out=out, flags=flags, stream=stream)):
            names = [n for n in kernels_of(call) if "k_scaled" in n]
            assert len(names) == 3 and all(k in n for k, n in zip(kernels, names)), names
    L.close()


def test_fast_passes():
    """The caller's choice, over groups from no row to over a thousand: what the 8-bit instructions may drop and the 16-bit outputs' rounding."""
    from paper_2510_02613_amd import binding as B
    for H, I in ((256, 272), (400, 256), (512, 384)):
        L = Layer(H=H, I=I, E=12, k=1, n_local=10, n_shared=1, seed=21, max_tokens=2500)
        counts = [5, 0, 20, 50, 100, 170, 230, 600, 1, 1040]
        ids = torch.cat([torch.full((n,), e) for e, n in enumerate(counts)] + [torch.full((30,), 11)]).to(torch.int32)
        ids = ids[torch.randperm(len(ids), generator=torch.Generator().manual_seed(1))][:, None].contiguous()
        T = len(ids)
        w = torch.rand(T, 1, generator=torch.Generator().manual_seed(2)) + 0.1
        x, q, scale, value = L.tokens(3, T)
        run = lambda: L.layer.forward_scaled(q.cuda(), scale.cuda(), topk_ids=ids.cuda(), topk_w=w.cuda(), shared_range=(100, 400),  # noqa: E731
                                             flags=B.MOE_FLAG_FAST_PRODUCTS)
        out = run()
        L.check(out, value, ids, w, (100, 400))
        assert torch.equal(out, L.layer.forward_routed(x.cuda(), ids.cuda(), w.cuda(), shared_range=(100, 400), flags=B.MOE_FLAG_FAST_PRODUCTS))
        L.close()
