"""The layer with 8-bit experts against the same passes in 64 bits: every placement, entry point and batch size goes through
quantised tokens, the two block-scaled products per expert and the weighted sum."""
import numpy as np
import pytest
import torch

import scaled_ref as R

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn


def randn(seed, *shape):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g)


def weights(seed, n, k, parts=1):
    q = (randn(seed, n, k) * 100).clamp(-448, 448).to(E4M3)
    nb = R.blocks(n // parts)
    scale = torch.exp(0.5 * randn(seed + 1, parts * nb, R.blocks(k))) * 3e-4
    values = torch.cat([q[i * (n // parts):(i + 1) * (n // parts)].double() * R.spread_blocks(scale[i * nb:(i + 1) * nb], n // parts, k)
                        for i in range(parts)])
    return q, scale, values


class Layer:
    """A layer of experts 0 .. n_local - 1 of E in shuffled slots (the unused ones hold NaN), and what it computes."""

    def __init__(self, H, I, E, k, n_local, n_shared=0, spare=2, max_tokens=512, gate="softmax", seed=0, copies=0, slots=None, **kw):
        from paper_2510_02613_amd.layer import MoELayer, ScaledExperts
        self.H, self.I, self.E, self.k, self.n_shared, self.n_local = H, I, E, k, n_shared, n_local
        S = n_local + n_shared + spare + copies
        self.pools = ScaledExperts(torch.full((S, 2 * I, H), float("nan")).to(E4M3).cuda(), torch.full((S, 2 * R.blocks(I), R.blocks(H)), float("nan")).cuda(),
                                   torch.full((S, H, I), float("nan")).to(E4M3).cuda(), torch.full((S, R.blocks(H), R.blocks(I)), float("nan")).cuda())
        order = np.random.RandomState(seed).permutation(S) if slots is None else np.asarray(slots)
        self.experts = [weights(1000 * seed + 10 * e, 2 * I, H, parts=2) + weights(1000 * seed + 10 * e + 5, H, I) for e in range(n_local + n_shared)]
        self.slot = [int(order[e]) for e in range(n_local + n_shared)]
        self.copy_slots = [int(s) for s in order[n_local + n_shared:n_local + n_shared + copies]]
        for e, s in enumerate(self.slot):
            self.fill(s, e)
        for s in self.copy_slots:
            self.fill(s, 0)
        self.layer = MoELayer(hidden=H, inter=I, n_experts=E, top_k=k, n_slots=S, max_tokens=max_tokens, gate=gate, n_shared=n_shared,
                              router_w=(np.random.RandomState(seed + 1).randn(E, H) * 0.05).astype(np.float32), scaled=self.pools, **kw)
        self.map = [self.slot[e] if e < n_local else -1 for e in range(E)]
        shared = self.slot[n_local:]
        if copies:
            self.layer.set_expert_replicas([([self.slot[0]] + self.copy_slots if e == 0 else [self.slot[e]] if e < n_local else []) for e in range(E)], shared)
        else:
            self.layer.set_expert_map(self.map, shared)

    def fill(self, slot, e):
        w13, s13, _, w2, s2, _ = self.experts[e]
        for pool, t in zip(self.pools, (w13, s13, w2, s2)):
            pool[slot].copy_(t)

    def routing(self, seed, T):
        """Ids of k different experts of all of them, some of them -1 (no assignment), and weights."""
        g = torch.Generator()
        g.manual_seed(seed)
        ids = torch.rand(T, self.E, generator=g).topk(self.k, 1).indices.to(torch.int32)
        ids[torch.rand(T, self.k, generator=g) < 0.05] = -1
        return ids, torch.rand(T, self.k, generator=g) + 0.1

    def tokens(self, seed, T):
        """(bf16 tokens, their 8-bit form, its scales, its values)"""
        x = randn(seed, T, self.H).bfloat16()
        _, per = R.group_max(x.double())
        q = R.e4m3_round(torch.where(per > 0, x.double() * 448 / per, 0.0))
        scale = (R.group_max(x.double())[0].float() / 448.0)
        return x, q.to(E4M3), scale, q * R.spread_rows(scale, self.H)

    def check(self, out, x, ids, w, shared_range=(0, 0), dx=None):
        """out against the layer's sum for 8-bit tokens of values x."""
        T = x.shape[0]
        y, dy = torch.zeros(T, self.H, dtype=torch.float64), torch.zeros(T, self.H, dtype=torch.float64)
        dx = torch.zeros_like(x) if dx is None else dx
        for e in range(self.n_local + self.n_shared):
            if e < self.n_local:
                token, col = (ids == e).nonzero(as_tuple=True)
                wt = w[token, col].double()[:, None]
            else:
                token = torch.arange(*shared_range)
                wt = torch.ones(len(token), 1, dtype=torch.float64)
            if len(token) == 0:
                continue
            # the large tiles' 8-bit products of GEMM-1 and GEMM-2: see FAST
            h, dh = R.swiglu(x[token], dx[token], self.experts[e][2], fast=True)
            v, dv = R.quantize(h, dh)
            o, do = R.product(v, dv, self.experts[e][5], fast=True)
            y.index_add_(0, token, wt * o)
            # between the GEMM and the sum: fp32, or 16-bit numbers of a 32767th of the largest of 64 columns, off by half of one
            top = torch.nn.functional.pad(o.abs() + do, (0, -self.H % 64)).view(len(token), -1, 64).amax(2).repeat_interleave(64, 1)[:, :self.H]
            dy.index_add_(0, token, wt * (do + top / 65534 * (1 + 2.0 ** -10) + 64 * R.F32 * o.abs()))
        off = (out.cpu().view(torch.bfloat16).double() - y).abs() - dy - (R.BF16 + 64 * R.F32) * (y.abs() + dy)
        assert (off <= 0).all(), f"{off.max().item():.3e} beyond the roundings, of {y.abs().max().item():.3e}"
        return y

    def close(self):
        self.layer.close()


SHAPES = [dict(H=128, I=128, E=8, k=2, n_local=8), dict(H=256, I=144, E=16, k=4, n_local=5, n_shared=1), dict(H=272, I=400, E=12, k=3, n_local=12),
          dict(H=512, I=256, E=32, k=4, n_local=9, n_shared=2), dict(H=1040, I=272, E=4, k=1, n_local=2)]


@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("T", [1, 2, 5, 33, 130, 512])
def test_routed_pass(shape, T):
    L = Layer(**SHAPES[shape], seed=shape)
    ids, w = L.routing(7 + T, T)
    x, q, scale, value = L.tokens(9 + T, T)
    sr = (0, 0) if not L.n_shared else (T // 3, T)
    out = L.layer.forward_scaled(q.cuda(), scale.cuda(), topk_ids=ids.cuda(), topk_w=w.cuda(), shared_range=sr)
    want = L.check(out, value, ids, w, sr)
    # bf16 tokens, quantised by the pass, are the same tokens
    again = L.layer.forward_routed(x.cuda(), ids.cuda(), w.cuda(), shared_range=sr)
    assert torch.equal(again, out)
    assert ((want.abs().sum(1) == 0) == (out.cpu().double().abs().sum(1) == 0)).all()     # tokens without a local expert: zero rows
    L.close()


@pytest.mark.parametrize("H,I", [(256, 272), (400, 256), (512, 384)])
def test_groups_of_every_size(H, I):
    """Groups from no row to over a thousand in one pass: tiles of every number of rows, several tiles of a group, and a shared expert."""
    from gpu_util import kernels_of
    L = Layer(H=H, I=I, E=12, k=1, n_local=10, n_shared=1, seed=21, max_tokens=2500)
    counts = [5, 0, 20, 50, 100, 170, 230, 600, 1, 1040]
    ids = torch.cat([torch.full((n,), e) for e, n in enumerate(counts)] + [torch.full((30,), 11)]).to(torch.int32)
    ids = ids[torch.randperm(len(ids), generator=torch.Generator().manual_seed(1))][:, None].contiguous()
    T = len(ids)
    w = torch.rand(T, 1, generator=torch.Generator().manual_seed(2)) + 0.1
    x, q, scale, value = L.tokens(3, T)
    q, scale, d_ids, d_w = q.cuda(), scale.cuda(), ids.cuda(), w.cuda()
    out = torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
    run = lambda stream=None: L.layer.forward_scaled(q, scale, topk_ids=d_ids, topk_w=d_w, out=out, shared_range=(100, 400), stream=stream)  # noqa: E731
    assert sum("k_scaled_tiles" in n for n in kernels_of(run)) == 2
    run()
    L.check(out, value, ids, w, (100, 400))
    first = out.clone()
    run()
    assert torch.equal(out, first)
    L.close()


def test_few_tokens_are_streamed():
    from gpu_util import kernels_of
    L = Layer(**SHAPES[0], seed=0)
    ids, w = L.routing(7, 3)
    x, q, scale, _ = L.tokens(9, 3)
    q, scale, ids, w, out = q.cuda(), scale.cuda(), ids.cuda(), w.cuda(), torch.empty(3, L.H, dtype=torch.bfloat16, device="cuda")
    names = kernels_of(lambda stream: L.layer.forward_scaled(q, scale, topk_ids=ids, topk_w=w, out=out, stream=stream))
    assert sum("k_scaled_stream" in n for n in names) == 2
    L.close()


def test_tokens_without_experts_here():
    L = Layer(**SHAPES[1], seed=11)
    T = 20
    ids = torch.full((T, L.k), -1, dtype=torch.int32)
    ids[:, 0] = L.n_local                                  # an expert of another rank
    x, q, scale, _ = L.tokens(1, T)
    out = torch.full((T, L.H), 7.0, dtype=torch.bfloat16, device="cuda")
    L.layer.forward_scaled(q.cuda(), scale.cuda(), topk_ids=ids.cuda(), topk_w=torch.ones(T, L.k).cuda(), out=out)
    assert (out == 0).all()
    out.fill_(7.0)
    L.layer.forward_scaled(q[:0].cuda(), scale[:0].cuda(), topk_ids=ids[:0].cuda(), topk_w=torch.ones(0, L.k).cuda(), out=out[:0])
    assert (out == 7).all()
    L.close()


@pytest.mark.parametrize("T", [3, 70, 400])
def test_one_expert_gets_every_token_and_ids_repeat(T):
    """All rows in one group, several tiles of it; the same expert twice in a token counts twice."""
    L = Layer(H=256, I=256, E=8, k=2, n_local=4, seed=3)
    ids = torch.full((T, 2), 2, dtype=torch.int32)
    w = torch.rand(T, 2, generator=torch.Generator().manual_seed(4))
    x, q, scale, value = L.tokens(5, T)
    out = L.layer.forward_scaled(q.cuda(), scale.cuda(), topk_ids=ids.cuda(), topk_w=w.cuda())
    L.check(out, value, ids, w)
    L.close()


@pytest.mark.parametrize("gate,kw", [("softmax", {}), ("sigmoid_group", dict(n_group=4, topk_group=2, routed_scale=2.5))])
@pytest.mark.parametrize("T", [1, 40, 300])
def test_gated_pass(gate, kw, T):
    """The gate of the bf16 layer in front: its selection, then the sum for those experts."""
    L = Layer(H=512, I=128, E=16, k=4, n_local=10, n_shared=1, gate=gate, seed=6, **kw)
    x, q, scale, value = L.tokens(T, T)
    out = L.layer.forward(x.cuda(), shared_range=(0, T))
    v = L.layer.view(T)
    ids, w = torch.from_numpy(v["topk_ids"]), torch.from_numpy(v["topk_w"])
    logits = x.double() @ torch.from_numpy(L.layer.router_w.cpu().numpy()).double().t()
    if gate == "softmax":
        assert torch.equal(ids.long().sort(1).values, logits.topk(4, 1).indices.sort(1).values)
    L.check(out, value, ids, w, (0, T))
    assert torch.equal(L.layer.forward_scaled(q.cuda(), scale.cuda(), x.cuda(), shared_range=(0, T)), out)
    assert torch.equal(L.layer.forward(x.view(torch.int16).cuda(), shared_range=(0, T)).view(torch.bfloat16), out)   # bit patterns, as other layers take
    unfused = L.layer.forward(x.cuda(), shared_range=(0, T), flags=8)
    assert torch.equal(unfused, out)
    L.close()


def test_the_slots_do_not_matter():
    T = 200
    outs = []
    for slots in (np.arange(14), np.random.RandomState(1).permutation(14)):
        L = Layer(**SHAPES[2], seed=2, slots=slots)
        ids, w = L.routing(3, T)
        x, q, scale, _ = L.tokens(4, T)
        outs.append(L.layer.forward_scaled(q.cuda(), scale.cuda(), topk_ids=ids.cuda(), topk_w=w.cuda()).cpu())
        L.close()
    assert torch.equal(outs[0], outs[1])


def test_copies_of_an_expert():
    T = 90
    L = Layer(H=256, I=128, E=8, k=2, n_local=4, seed=8, copies=2)
    ids, w = L.routing(1, T)
    ids[:, 0] = 0
    ids[ids[:, 1] == 0, 1] = 1
    x, q, scale, value = L.tokens(2, T)
    out = L.layer.forward_scaled(q.cuda(), scale.cuda(), topk_ids=ids.cuda(), topk_w=w.cuda())
    L.check(out, value, ids, w)
    L.close()


def test_identity_experts_and_profile():
    from paper_2510_02613_amd import binding as B
    T = 50
    L = Layer(**SHAPES[3], seed=9)
    ids, w = L.routing(1, T)
    x, q, scale, value = L.tokens(2, T)
    B.moe_profile_enable(L.layer.handle, 1)
    out = L.layer.forward_scaled(q.cuda(), scale.cuda(), x.cuda(), topk_ids=ids.cuda(), topk_w=w.cuda(), flags=B.MOE_FLAG_IDENTITY_EXPERTS)
    here = (w.double() * ((ids >= 0) & (ids < L.n_local))).sum(1, keepdim=True) * x.double()
    assert ((out.cpu().double() - here).abs() <= (R.BF16 + 8 * R.F32) * here.abs() + 8 * R.F32 * x.double().abs() * w.double().sum(1, keepdim=True)).all()
    L.layer.forward_scaled(q.cuda(), scale.cuda(), topk_ids=ids.cuda(), topk_w=w.cuda())
    ms = B.moe_profile_read(L.layer.handle)
    assert len(ms) == 5 and all(0 <= v < 1000 for v in ms) and ms[2] > 0
    with pytest.raises(B.MoEError) as e:
        L.layer.forward(x.cuda(), flags=B.MOE_FLAG_FORCE_GENERIC)
    assert e.value.status == B.MOE_ERR_UNSUPPORTED
    with pytest.raises(B.MoEError) as e:       # the identity experts read x
        L.layer.forward_scaled(q.cuda(), scale.cuda(), topk_ids=ids.cuda(), topk_w=w.cuda(), flags=B.MOE_FLAG_IDENTITY_EXPERTS)
    assert e.value.status == B.MOE_ERR_ARG
    with pytest.raises(ValueError):
        L.layer.forward_static(x.cuda())
    L.close()


def test_fill_and_switch_between_replays_of_a_graph():
    """A captured pass is replayed on changed tokens, and across a slot fill and a switch of the placement; every replay is the eager pass's."""
    T = 60
    L = Layer(H=384, I=256, E=8, k=2, n_local=8, seed=12, spare=3)
    from paper_2510_02613_amd import scaled
    x = torch.empty(T, L.H, dtype=torch.bfloat16, device="cuda")
    q, s = torch.empty(T, L.H, dtype=E4M3, device="cuda"), torch.empty(T, R.blocks(L.H), device="cuda")
    out = torch.empty_like(x)
    copy = torch.cuda.Stream()

    def step():
        scaled.rms_norm(x, q=q, q_scale=s)
        L.layer.forward_scaled(q, s, x, out=out)

    def check(seed):
        x.copy_(randn(seed, T, L.H))
        step()
        want = out.clone()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        v = L.layer.view(T)
        L.check(out, q.cpu().double() * R.spread_rows(s.cpu(), L.H), torch.from_numpy(v["topk_ids"]), torch.from_numpy(v["topk_w"]))

    x.copy_(randn(1, T, L.H))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    check(2)
    check(3)
    # expert 5 moves to a spare slot
    free = next(s_ for s_ in range(11) if s_ not in L.slot)
    w13, s13, _, w2, s2, _ = [t.cuda() if t.dtype != torch.float64 else t for t in L.experts[5]]
    L.layer.load_expert_async(free, w13, w2, copy, w13_scale=s13, w2_scale=s2)
    check(4)
    L.layer.set_expert_map([free if e == 5 else L.slot[e] for e in range(8)])
    check(5)
    torch.cuda.synchronize()
    for pool, t in zip(L.pools, (w13, s13, w2, s2)):
        assert torch.equal(pool[free].view(torch.uint8) if pool.dtype == E4M3 else pool[free], t.view(torch.uint8) if t.dtype == E4M3 else t)
    L.close()


def test_page_pools_of_8bit_slots():
    """Page pools under an 8-bit layer have slots of 2 I H and H I bytes; a placement that names a slot without a page is refused."""
    from paper_2510_02613_amd import binding as B
    H, I = 2048, 1024
    cfg = B.MoEConfig(H, I, 4, 1, 4, 16, B.MOE_BF16, B.MOE_F32, 0, 1, 1, 1, 1.0, 0)
    p13, p2 = B.moe_vpool_create(2 * I * H, 4), B.moe_vpool_create(H * I, 4)
    small = B.moe_vpool_create(2 << 20, 4)
    ws = torch.empty(B.moe_scaled_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    scales = torch.zeros(4 * 2 * 8 * 16, device="cuda")
    router = torch.zeros(4, H, device="cuda")
    h = B.moe_layer_create_scaled(cfg, B.MoEBuffers(router.data_ptr(), 0, 0, B.moe_vpool_base(p13), B.moe_vpool_base(p2), ws.data_ptr(), ws.numel()),
                                  scales.data_ptr(), scales.data_ptr())
    try:
        with pytest.raises(B.MoEError) as e:
            B.moe_layer_bind_vpools(h, small, p2)
        assert e.value.status == B.MOE_ERR_ARG
        B.moe_layer_bind_vpools(h, p13, p2)
        with pytest.raises(B.MoEError) as e:
            B.moe_set_expert_map(h, [0, -1, -1, -1])
        assert e.value.status == B.MOE_ERR_MAP
    finally:
        B.moe_layer_destroy(h)
        for p in (p13, p2, small):
            B.moe_vpool_destroy(p)
