"""Tensors that a layer's passes and fills would read or write out of range by their address are refused before the library is called (no GPU needed: nothing
runs, the calls into the library are recorded)."""
import types

import pytest
import torch

E4M3 = torch.float8_e4m3fn
T, H, K = 4, 256, 2
CPU, META = torch.device("cpu"), torch.device("meta")


@pytest.fixture
def calls(monkeypatch):
    from paper_2510_02613_amd import layer as Lm
    seen = []
    for name in ("moe_forward", "moe_forward_routed", "moe_forward_static", "moe_forward_scaled", "moe_load_expert", "moe_load_expert_scaled"):
        monkeypatch.setattr(Lm.B, name, lambda *a, name=name, **kw: seen.append(name))
    monkeypatch.setattr(Lm, "_stream_ptr", lambda s, device: 7)
    return seen


def layer(scaled, device=CPU):
    from paper_2510_02613_amd.layer import MoELayer, ScaledExperts
    L = object.__new__(MoELayer)
    L.cfg, L.handle, L.device, L.elt = types.SimpleNamespace(hidden=H, top_k=K), None, device, torch.int16
    L.buf, L.plain_map = types.SimpleNamespace(router_w=0, logit_bias=0, select_bias=0, w13=0, w2=0), (None, None)
    L.w13, L.w2 = torch.zeros(3, 128, H).to(E4M3 if scaled else torch.int16), torch.zeros(3, H, 64).to(E4M3 if scaled else torch.int16)
    L.slot13, L.slot2 = L.w13.shape[1:], L.w2.shape[1:]
    L.scaled = ScaledExperts(L.w13, torch.zeros(3, 2, 2), L.w2, torch.zeros(3, 2, 1)) if scaled else None
    return L


def run(L, method, x=None, out=None, xq=None):
    rows = lambda dt=torch.int16: torch.zeros(T, H).to(dt)  # noqa: E731
    ids, w = torch.zeros(T, K, dtype=torch.int32), torch.zeros(T, K)
    x = rows() if x is None else x
    args = {"forward": (x,), "forward_static": (x,), "forward_routed": (x, ids, w), "forward_scaled": (rows(E4M3), torch.zeros(T, 2), x)}[method]
    return getattr(L, method)(*args, out=out)


METHODS = [("forward", False), ("forward_routed", False), ("forward_static", False), ("forward", True), ("forward_routed", True), ("forward_scaled", True)]


@pytest.mark.parametrize("method,scaled", METHODS)
def test_passes(calls, method, scaled):
    good = torch.zeros(T, H, dtype=torch.int16)
    run(layer(scaled), method, out=good)
    run(layer(scaled), method, x=good, out=good)                                   # in place
    assert len(calls) == 2
    for bad in (torch.zeros(T - 1, H, dtype=torch.int16), torch.zeros(T, H - 8, dtype=torch.int16), torch.zeros(T, H, dtype=torch.int8), torch.zeros(T * H, dtype=torch.int16),
                torch.zeros(T, 2 * H, dtype=torch.int16)[:, :H], torch.zeros(T, H, dtype=torch.int16, device=META)):
        with pytest.raises(AssertionError):
            run(layer(scaled), method, out=bad)
    for bad in (torch.zeros(T, H - 8, dtype=torch.int16), torch.zeros(T, H, dtype=torch.int8), torch.zeros(T, 2 * H, dtype=torch.int16)[:, :H],
                torch.zeros(T, H, dtype=torch.int16, device=META)):
        with pytest.raises(AssertionError):
            run(layer(scaled), method, x=bad)
    assert len(calls) == 2


@pytest.mark.parametrize("scaled", [False, True])
def test_fills(calls, scaled):
    L = layer(scaled)
    good = dict(w13=L.w13[0], w2=L.w2[0], **(dict(w13_scale=L.scaled.w13_scale[0], w2_scale=L.scaled.w2_scale[0]) if scaled else {}))
    copy = types.SimpleNamespace(cuda_stream=1)
    fill = lambda **kw: L.load_expert_async(1, copy_stream=copy, **{**good, **kw})  # noqa: E731
    fill()
    assert len(calls) == 1
    for name, t in good.items():
        for bad in (t.to(META), t[:-1], t.to(torch.float64), t[None]):
            with pytest.raises(AssertionError):
                fill(**{name: bad})
    assert len(calls) == 1
