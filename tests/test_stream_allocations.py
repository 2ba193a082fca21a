"""Memory that a call allocates itself belongs to the stream it works on, whichever stream is current: the allocator hands a block that was
dropped on to later work of the stream it was allocated on, and to nobody who is not ordered behind the kernels that still use it.
Nothing runs here (no GPU needed): the allocations and the calls into the library are recorded."""
import contextlib
import types

import pytest
import torch

E4M3 = torch.float8_e4m3fn


class Recorder:
    def __init__(self, monkeypatch):
        self.at, self.allocations, self.calls = None, [], []
        monkeypatch.setattr(torch.cuda, "stream", self.stream)
        for name in ("empty", "empty_like"):
            monkeypatch.setattr(torch, name, self.recording(getattr(torch, name)))

    @contextlib.contextmanager
    def stream(self, s):
        before, self.at = self.at, s
        yield
        self.at = before

    def recording(self, real):
        def allocate(*args, **kw):
            t = real(*args, **kw)
            if t.numel():
                self.allocations.append((self.at, t.data_ptr()))
            return t
        return allocate

    def library(self, monkeypatch, module, *names):
        for name in names:
            monkeypatch.setattr(module, name, lambda *a, **kw: self.calls.append((a, kw)))


SIDE = types.SimpleNamespace(cuda_stream=0x1234)


@pytest.fixture
def rec(monkeypatch):
    return Recorder(monkeypatch)


def scaled_module(monkeypatch, rec):
    from paper_2510_02613_amd import scaled
    monkeypatch.setattr(scaled, "_device_of", lambda t: -1)              # the CPU's
    monkeypatch.setattr(scaled, "_current_device", lambda: -1)
    monkeypatch.setattr(scaled, "_current_stream", lambda dev: 7)
    rec.library(monkeypatch, scaled.B, "moe_rms_norm", "moe_quantize", "moe_scaled_matmul", "moe_scaled_swiglu")
    return scaled


CALLS = {
    "rms_norm": (2, lambda S, z, **kw: S.rms_norm(z(4, 256, torch.bfloat16), residual=z(4, 256, torch.bfloat16), **kw)),
    "quantize": (2, lambda S, z, **kw: S.quantize(z(4, 256, torch.bfloat16), **kw)),
    "matmul": (1, lambda S, z, **kw: S.matmul(z(4, 256, E4M3), z(4, 2, torch.float32), z(128, 256, E4M3), z(1, 2, torch.float32), **kw)),
    # q, scale and, as it is streamed, the workspace
    "swiglu": (3, lambda S, z, **kw: S.swiglu(z(4, 2048, E4M3), z(4, 16, torch.float32), z(256, 2048, E4M3), z(2, 16, torch.float32), **kw)),
}


@pytest.mark.parametrize("call", sorted(CALLS))
@pytest.mark.parametrize("side", [None, SIDE])
def test_operators_allocate_on_their_stream(monkeypatch, rec, call, side):
    S = scaled_module(monkeypatch, rec)
    n, run = CALLS[call]
    z = lambda rows, cols, dt: torch.zeros(rows, cols).to(dt)  # noqa: E731
    run(S, z, stream=side)
    assert len(rec.calls) == 1 and rec.calls[0][0][1] == (7 if side is None else side.cuda_stream)
    assert [at for at, _ in rec.allocations] == [side] * n


@pytest.mark.parametrize("method", ["forward", "forward_routed", "forward_static", "forward_scaled"])
@pytest.mark.parametrize("side", [None, SIDE])
def test_layers_allocate_on_their_stream(monkeypatch, rec, method, side):
    from paper_2510_02613_amd import layer as Lm
    rec.library(monkeypatch, Lm.B, "moe_forward", "moe_forward_routed", "moe_forward_static", "moe_forward_scaled")
    monkeypatch.setattr(Lm, "_stream_ptr", lambda s, device: 7 if s is None else s.cuda_stream)
    L = object.__new__(Lm.MoELayer)
    T, H, k = 4, 256, 2
    L.cfg, L.handle, L.device = types.SimpleNamespace(hidden=H, top_k=k), None, torch.device("cpu")
    L.elt, L.scaled = torch.int16, (None if method == "forward_static" else ())
    L.buf, L.plain_map = types.SimpleNamespace(router_w=0, logit_bias=0, select_bias=0, w13=0, w2=0), (None, None)
    x = torch.zeros(T, H, dtype=torch.int16)
    ids, w = torch.zeros(T, k, dtype=torch.int32), torch.zeros(T, k)
    args = {"forward": (x,), "forward_static": (x,), "forward_routed": (x, ids, w),
            "forward_scaled": (torch.zeros(T, H).to(E4M3), torch.zeros(T, 2))}[method]
    kw = dict(topk_ids=ids, topk_w=w) if method == "forward_scaled" else {}
    getattr(L, method)(*args, stream=side, **kw)
    assert len(rec.calls) == 1 and (7 if side is None else side.cuda_stream) in list(rec.calls[0][0]) + list(rec.calls[0][1].values())
    assert [at for at, _ in rec.allocations] == [side]


@pytest.mark.gpu
def test_a_dropped_workspace_stays_with_its_stream(monkeypatch):
    """The workspace that swiglu allocated for a call on another stream is not what the current stream's next allocation gets; the result is that of a
    call on the current stream."""
    from paper_2510_02613_amd import scaled as S
    g = torch.Generator(device="cuda").manual_seed(1)
    m, inter, k = 9, 768, 2048
    q, scale = S.quantize(torch.randn(m, k, device="cuda", generator=g))
    w, ws = S.quantize(torch.randn(2 * inter, k, device="cuda", generator=g) * 0.02, block_rows=128)
    want = S.swiglu(q, scale, w, ws)
    spaces, real = [], S.swiglu_workspace
    monkeypatch.setattr(S, "swiglu_workspace", lambda *a: spaces.append(real(*a)) or spaces[-1])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = S.swiglu(q, scale, w, ws, stream=side)
    at, size = spaces[0].data_ptr(), spaces[0].numel()
    spaces.clear()
    next_blocks = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(4)]
    assert at not in [b.data_ptr() for b in next_blocks]
    with torch.cuda.stream(side):
        assert torch.empty(size, dtype=torch.uint8, device="cuda").data_ptr() == at
    side.synchronize()
    assert torch.equal(got.q.view(torch.uint8), want.q.view(torch.uint8)) and torch.equal(got.scale, want.scale)
