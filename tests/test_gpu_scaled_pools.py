"""Layers with 8-bit experts on page pools and on pools of another process: the passes of a layer on plain memory, bit for bit."""
import os
import subprocess
import sys

import pytest
import torch

from test_gpu_scaled_layer import Layer

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn


def over_pools(L, p13, p2, s13, s2):
    """A layer like L's over other pools."""
    from paper_2510_02613_amd.layer import MoELayer, ScaledExperts
    layer = MoELayer(hidden=L.H, inter=L.I, n_experts=L.E, top_k=L.k, n_slots=L.pools.w13.shape[0], max_tokens=L.layer.cfg.max_tokens, n_shared=L.n_shared,
                     router_w=L.layer.router_w.cpu().numpy(), scaled=ScaledExperts(p13, s13, p2, s2))
    layer.set_expert_map(L.map, L.slot[L.n_local:])
    return layer


def same_as_plain(L, layer, sizes=(3, 400)):
    for T in sizes:
        ids, w = L.routing(7 + T, T)
        x, q, scale, value = L.tokens(9 + T, T)
        x, q, scale, d_ids, d_w = (t.cuda() for t in (x, q, scale, ids, w))
        sr = (0, T if L.n_shared else 0)
        out = layer.forward_scaled(q, scale, topk_ids=d_ids, topk_w=d_w, shared_range=sr)
        assert torch.equal(out, L.layer.forward_scaled(q, scale, topk_ids=d_ids, topk_w=d_w, shared_range=sr))
        L.check(out, value, ids, w, sr)
        assert torch.equal(layer.forward(x, shared_range=sr), L.layer.forward(x, shared_range=sr))


def test_grow_exchange_and_shrink_on_pages():
    from paper_2510_02613_amd import binding as B
    from paper_2510_02613_amd.layer import VirtualPool
    H, I, n = 512, 384, 40                                            # 400 tokens: 159 workgroups of tiles
    L = Layer(H=H, I=I, E=48, k=2, n_local=n, n_shared=1, seed=51, spare=3)
    S = L.pools.w13.shape[0]
    s13, s2 = (torch.full_like(t, float("nan")) for t in (L.pools.w13_scale, L.pools.w2_scale))
    p13, p2 = VirtualPool(S, (2 * I, H), E4M3), VirtualPool(S, (H, I), E4M3)
    layer = None
    try:
        assert p13.tensor.dtype == E4M3 and p13.tensor.shape == (S, 2 * I, H) and p13.slot_bytes == 2 * I * H
        late = L.slot[3]                                              # this slot's page comes later
        for s in L.slot:
            if s != late:
                for pool, mine in ((p13, L.pools.w13), (p2, L.pools.w2)):
                    pool.map(s, pool.page_alloc())
                    pool.tensor[s].copy_(mine[s])
                s13[s].copy_(L.pools.w13_scale[s])
                s2[s].copy_(L.pools.w2_scale[s])
        from paper_2510_02613_amd.layer import MoELayer, ScaledExperts
        layer = MoELayer(hidden=H, inter=I, n_experts=L.E, top_k=L.k, n_slots=S, max_tokens=512, n_shared=1, router_w=L.layer.router_w.cpu().numpy(),
                         scaled=ScaledExperts(p13, s13, p2, s2))
        assert layer.w13.data_ptr() == p13.tensor.data_ptr() and layer.w2.data_ptr() == p2.tensor.data_ptr()
        w13, t13, _, w2, t2, _ = [t.cuda() if t.dtype != torch.float64 else t for t in L.experts[3]]
        copy = torch.cuda.Stream()
        for call in (lambda: layer.set_expert_map(L.map, L.slot[n:]),                                       # names the slot without a page
                     lambda: layer.load_expert_async(late, w13, w2, copy, w13_scale=t13, w2_scale=t2)):
            with pytest.raises(B.MoEError) as e:
                call()
            assert e.value.status == B.MOE_ERR_MAP
        # grow: a page under the slot, filled in the background with its scales, then the switch
        for pool in (p13, p2):
            pool.map(late, pool.page_alloc())
        layer.load_expert_async(late, w13, w2, copy, w13_scale=t13, w2_scale=t2)
        layer.set_expert_map(L.map, L.slot[n:])
        same_as_plain(L, layer)
        # the pages of two slots change places, and with them the scales and the map's entries
        torch.cuda.synchronize()
        a, b = L.slot[5], L.slot[11]
        for pool in (p13, p2):
            pages = pool.page_of(a), pool.page_of(b)
            pool.unmap(a)
            pool.unmap(b)
            pool.map(a, pages[1])
            pool.map(b, pages[0])
        for s in (s13, s2):
            s[[a, b]] = s[[b, a]]
        moved = list(L.map)
        moved[5], moved[11] = b, a
        layer.set_expert_map(moved, L.slot[n:])
        same_as_plain(L, layer)
        # a page that the placement in force names is taken away: refused on the host
        torch.cuda.synchronize()
        page = p2.page_of(a)
        p2.unmap(a)
        x = torch.zeros(2, H, dtype=torch.bfloat16, device="cuda")
        with pytest.raises(B.MoEError) as e:
            layer.forward(x)
        assert e.value.status == B.MOE_ERR_MAP
        p2.map(a, page)
        same_as_plain(L, layer, (3,))
    finally:
        torch.cuda.synchronize()
        if layer is not None:
            layer.close()
        L.close()
        p13.close()
        p2.close()


def test_pools_that_do_not_fit_are_refused():
    from paper_2510_02613_amd.layer import MoELayer, ScaledExperts, VirtualPool
    L = Layer(H=512, I=256, E=4, k=1, n_local=2, seed=52)
    S = L.pools.w13.shape[0]
    kw = dict(hidden=512, inter=256, n_experts=4, top_k=1, n_slots=S, max_tokens=8, router_w=L.layer.router_w.cpu().numpy())
    for elt, shape in ((torch.int16, (512, 512)), (E4M3, (512, 256))):
        pool = VirtualPool(S, shape, elt)
        try:
            with pytest.raises(AssertionError):
                MoELayer(scaled=ScaledExperts(pool, *L.pools[1:]), **kw)
        finally:
            pool.close()
    L.close()


def test_serving_process_runs_on_8bit_pools_of_another_process():
    script = os.path.join(os.path.dirname(os.path.abspath(__file__)), "ipc_scaled_roles.py")
    r = subprocess.run([sys.executable, "-u", script, "launcher"], capture_output=True, text=True, timeout=110)
    print(r.stdout)
    print(r.stderr[-3000:])
    assert r.returncode == 0, f"launcher exit {r.returncode}"
    assert "attached 8-bit pools OK" in r.stdout
