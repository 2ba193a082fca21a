"""The 8-bit path against 64 bits by the norm of the error (scaled_norms.py says what is expected of it): products, the SwiGLU form, whole passes of a
layer, streamed and in tiles, and tiles of one slot that are worked on side by side."""
import pytest
import torch

import scaled_norms as N
import scaled_ref as R
from test_gpu_scaled import MATMUL, SWIGLU, eight_bit_rows, eight_bit_weights
from test_gpu_scaled_layer import SHAPES, Layer

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn
# The 8-bit matrix instructions' share of a result's norm: measured 1.5e-5 on normal values, 6e-5 on spread ones; of a layer's outputs through the bytes of h
# that it moves: one of 3000 by a step, 1/16 to 1/8 of the value, 1/11 on average: (1/3000)^(1/2) / 11 = 0.0017.
FAST_PRODUCT, FAST_LAYER = 6e-5, 0.0017


@pytest.mark.parametrize("m,n,k", [s for s in MATMUL if s[0] * s[1] >= 10000])
@pytest.mark.parametrize("fast", [False, True])
def test_matmul(m, n, k, fast):
    from paper_2510_02613_amd import scaled as S
    q, scale, a = eight_bit_rows(m + k, m, k)
    wq, ws, w = eight_bit_weights(n + k, n, k)
    y = a @ w.t()
    e2 = N.product_noise(a, w) ** 2 + ((FAST_PRODUCT * y) ** 2 if fast else 0.0)
    assert N.excess(S.matmul(q.cuda(), scale.cuda(), wq.cuda(), ws.cuda(), fast=fast).cpu(), y, e2) < N.SLACK
    if not fast:
        out = S.matmul(q.cuda(), scale.cuda(), wq.cuda(), ws.cuda(), out_dtype=torch.float32).cpu().double()
        assert ((out - y) ** 2).sum() < N.SLACK * (e2 + (R.F32 * y) ** 2).sum()


@pytest.mark.parametrize("m,inter,k", [s for s in SWIGLU if s[0] * s[1] >= 10000])
def test_swiglu(m, inter, k):
    """Bytes that differ from those of 64 bits: as many as values lie within the expected error of a border, give or take."""
    from paper_2510_02613_amd import scaled as S
    q, scale, a = eight_bit_rows(m + k, m, k)
    wq, ws, w = eight_bit_weights(inter + k, 2 * inter, k, parts=2)
    got = S.swiglu(q.cuda(), scale.cuda(), wq.cuda(), ws.cuda())
    h, dh = N.swiglu_noise(a, w)
    v, ev2 = N.quantized_noise(h, dh)
    value = got.q.cpu().double() * R.spread_rows(got.scale.cpu(), inter)
    _, per = R.group_max(h)
    step = R.e4m3_step(h * R.TOP / per) * per / R.TOP
    moved = ((value - v).abs() > 0.25 * step).sum().item()
    expected = (ev2 / step ** 2).sum().item()
    assert moved <= N.SLACK * expected + 6 * expected ** 0.5 + 6, (moved, expected)


@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("T", [130, 512])
@pytest.mark.parametrize("fast", [False, True])
def test_routed_pass(shape, T, fast):
    from paper_2510_02613_amd import binding as B
    L = Layer(**SHAPES[shape], seed=shape)
    ids, w = L.routing(7 + T, T)
    _, q, scale, value = L.tokens(9 + T, T)
    sr = (0, 0) if not L.n_shared else (T // 3, T)
    out = L.layer.forward_scaled(q.cuda(), scale.cuda(), topk_ids=ids.cuda(), topk_w=w.cuda(), shared_range=sr, flags=B.MOE_FLAG_FAST_PRODUCTS if fast else 0)
    y, e2 = N.layer_noise(L.experts, L.n_local, value, ids, w, sr)
    assert N.excess(out.cpu(), y, e2 + (FAST_LAYER * y) ** 2 * fast) < N.SLACK
    L.close()


@pytest.mark.parametrize("fast", [False, True])
def test_many_rows_of_a_slot(fast):
    """Slots with several tiles each, unevenly loaded, that share a slice of the weights while it is in a cache: 34 tiles taken four at a time, with the 8-bit
    instructions 19 taken two at a time.  And every expert gets its own tokens' rows."""
    from gpu_util import kernels_of
    from paper_2510_02613_amd import binding as B
    counts = [1300, 37, 0, 900, 611, 256, 896]
    T = sum(counts)
    L = Layer(H=256, I=272, E=7, k=1, n_local=7, seed=41, max_tokens=T)
    ids = torch.cat([torch.full((n,), e) for e, n in enumerate(counts)]).to(torch.int32)
    ids = ids[torch.randperm(T, generator=torch.Generator().manual_seed(1))][:, None].contiguous()
    w = torch.rand(T, 1, generator=torch.Generator().manual_seed(2)) + 0.1
    _, q, scale, value = L.tokens(3, T)
    q, scale, d_ids, d_w, out = q.cuda(), scale.cuda(), ids.cuda(), w.cuda(), torch.empty(T, L.H, dtype=torch.bfloat16, device="cuda")
    flags = B.MOE_FLAG_FAST_PRODUCTS if fast else 0
    run = lambda stream=None: L.layer.forward_scaled(q, scale, topk_ids=d_ids, topk_w=d_w, out=out, flags=flags, stream=stream)  # noqa: E731
    assert sum("k_scaled_tiles" in n for n in kernels_of(run)) == 2
    run()
    L.check(out, value, ids, w)
    y, e2 = N.layer_noise(L.experts, L.n_local, value, ids, w)
    assert N.excess(out.cpu(), y, e2 + (FAST_LAYER * y) ** 2 * fast) < N.SLACK
    for e, n in enumerate(counts):
        mine = (ids[:, 0] == e)
        if n:
            assert N.excess(out.cpu()[mine], y[mine], e2[mine] + (FAST_LAYER * y[mine]) ** 2 * fast) < N.SLACK
    first = out.clone()
    out.fill_(7.0)
    run()
    assert torch.equal(out, first)
    L.close()


def exact_h_layer(H, I, E, max_tokens):
    """Experts whose rows of h are the same in any arithmetic: gate rows read one column of a token, up rows too, times an e4m3 value of their own, the
    largest of 128 of them 448, so that h's bytes are those values.  What is left is GEMM-2, the outputs between it and the sum, and the sum."""
    from paper_2510_02613_amd.layer import MoELayer, ScaledExperts
    import numpy as np
    g = torch.Generator().manual_seed(5)
    up = (torch.randn(E, I, generator=g) * 100).clamp(-448, 448).to(E4M3).float()
    up[:, ::128] = 448.0
    w13 = torch.zeros(E, 2 * I, H)
    w13[:, :I, 0] = 1.0
    w13[:, I:, 0] = up
    w2 = (torch.randn(E, H, I, generator=g) * 100).clamp(-448, 448).to(E4M3)
    s2 = torch.exp(0.5 * torch.randn(E, R.blocks(H), R.blocks(I), generator=g)) * 3e-4
    pools = ScaledExperts(w13.to(E4M3).cuda(), torch.ones(E, 2 * R.blocks(I), R.blocks(H)).cuda(), w2.cuda(), s2.cuda())
    layer = MoELayer(hidden=H, inter=I, n_experts=E, top_k=2, n_slots=E, max_tokens=max_tokens, router_w=np.zeros((E, H), np.float32), scaled=pools)
    layer.set_expert_map(list(range(E)))
    h = 1.0 / (1.0 + np.exp(-1.0)) * up.double()                       # silu(1) u for tokens of 1
    y = torch.stack([R.spread_blocks(s2[e], H, I) * w2[e].double() @ h[e] for e in range(E)])
    noise = torch.stack([N.product_noise(h[e:e + 1], R.spread_blocks(s2[e], H, I) * w2[e].double())[0] for e in range(E)])
    return layer, y, noise


@pytest.mark.parametrize("T,tiles", [(40, False), (3000, True)])
@pytest.mark.parametrize("fast", [False, True])
def test_outputs_are_rounded_once(T, tiles, fast):
    """bf16 rows between GEMM-2 and the weighted sum would double the square of the error."""
    from paper_2510_02613_amd import binding as B
    H, I, E = 512, 256, 96
    layer, y_of, noise = exact_h_layer(H, I, E, T)
    g = torch.Generator().manual_seed(T)
    ids, w = torch.rand(T, E, generator=g).topk(2, 1).indices.to(torch.int32), torch.rand(T, 2, generator=g) + 0.1
    x, s = torch.ones(T, H).to(E4M3).cuda(), torch.ones(T, R.blocks(H)).cuda()
    from gpu_util import kernels_of
    out, d_ids, d_w = torch.empty(T, H, dtype=torch.bfloat16, device="cuda"), ids.cuda(), w.cuda()
    run = lambda stream=None: layer.forward_scaled(x, s, topk_ids=d_ids, topk_w=d_w, out=out, flags=B.MOE_FLAG_FAST_PRODUCTS if fast else 0, stream=stream)  # noqa: E731
    assert any("k_scaled_tiles" in n for n in kernels_of(run)) == (tiles or fast)      # 108 workgroups of tiles for 40 tokens
    run()
    terms = w.double()[:, :, None] * y_of[ids.long()]
    y = terms.sum(1)
    # fp32 throughout; fast: products 6e-5 of an output's norm, 16-bit outputs half of a 32767th of the largest of 64, which is below six times the norm's share
    e2 = ((w.double()[:, :, None] * noise[ids.long()]) ** 2).sum(1) + (8 * R.F32 * terms).pow(2).sum(1)
    e2 = e2 + fast * (FAST_PRODUCT ** 2 + (6 / 65534) ** 2) * terms.pow(2).sum(1)
    assert N.excess(out.cpu(), y, e2) < N.SLACK
    rows = (w.double()[:, :, None] * N.bf16(y_of)[ids.long()]).sum(1)
    assert N.excess(N.bf16(rows), y, e2) > N.SLACK                     # the mistake, planted in the reference
    layer.close()
