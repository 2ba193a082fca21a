"""What the operators of the 8-bit path refuse, before anything is launched (no GPU needed), and the reference that their GPU tests use."""
import ctypes
import os
import re

import pytest
import torch

import scaled_ref as R
from paper_2510_02613_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("struct,name", [(B.MoERmsNorm, "moe_rms_norm_t"), (B.MoEQuantize, "moe_quantize_t"), (B.MoEScaledMatmul, "moe_scaled_matmul_t"),
                                         (B.MoEScaledSwiglu, "moe_scaled_swiglu_t")])
def test_structs_match_the_header(struct, name):
    hdr = open(os.path.join(ROOT, "include", "elasticmoe_scaled.h")).read()
    end = hdr.index("} %s;" % name)
    body = re.sub(r"/\*.*?\*/", "", hdr[hdr.rindex("typedef struct {", 0, end):end], flags=re.S)
    ctype = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float, "size_t": ctypes.c_size_t}
    fields = []
    for kind, names in re.findall(r"(int32_t|int64_t|size_t|const void|const float|float|void)\s+([^;]+);", body):
        for n in names.split(","):
            fields.append((n.strip(" *"), ctypes.c_void_p if "*" in n else ctype[kind]))
    assert fields == struct._fields_


def test_library_exports_every_declared_symbol():
    hdr = open(os.path.join(ROOT, "include", "elasticmoe_scaled.h")).read()
    declared = set(re.findall(r"^(?:moe_status_t|size_t) (moe_[a-z_0-9]+)\(", hdr, re.M))
    assert declared == set(B.EXPORTS_SCALED)
    for name in declared:
        assert hasattr(B.lib(), name), name


def norm(**kw):
    d = dict(rows=4, cols=256, dtype=B.MOE_BF16, eps=1e-6, x=0x10000, ld_x=256, residual=0x20000, ld_residual=256, weight=0x30000,
             sum=0x40000, ld_sum=256, out=0x50000, ld_out=256, q=0x60000, ld_q=256, q_scale=0x70000, ld_scale=2)
    d.update(kw)
    return lambda: B.moe_rms_norm(B.MoERmsNorm(**d))


def quantize(**kw):
    d = dict(rows=4, cols=256, dtype=B.MOE_BF16, block_rows=1, x=0x10000, ld_x=256, q=0x60000, ld_q=256, scale=0x70000, ld_scale=2)
    d.update(kw)
    return lambda: B.moe_quantize(B.MoEQuantize(**d))


def matmul(**kw):
    d = dict(m=4, n=256, k=256, out_dtype=B.MOE_BF16, a=0x10000, ld_a=256, a_scale=0x20000, ld_a_scale=2, w=0x30000, w_scale=0x40000,
             add=0x50000, ld_add=256, out=0x60000, ld_out=256)
    d.update(kw)
    return lambda: B.moe_scaled_matmul(B.MoEScaledMatmul(**d))


def swiglu(**kw):
    d = dict(m=4, inter=256, k=2048, a=0x10000, ld_a=2048, a_scale=0x20000, ld_a_scale=16, w=0x30000, w_scale=0x40000,
             q=0x50000, ld_q=256, q_scale=0x60000, ld_scale=2, workspace=0x70000, workspace_bytes=1 << 30)
    d.update(kw)
    return lambda: B.moe_scaled_swiglu(B.MoEScaledSwiglu(**d))


ARG, SHAPE, UNSUPPORTED, CAPACITY = B.MOE_ERR_ARG, B.MOE_ERR_SHAPE, B.MOE_ERR_UNSUPPORTED, B.MOE_ERR_CAPACITY
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), SHAPE), (dict(cols=0), SHAPE), (dict(cols=252), UNSUPPORTED), (dict(cols=32776, ld_x=40000), UNSUPPORTED),
    (dict(rows=(1 << 21) + 1), UNSUPPORTED), (dict(dtype=2), ARG), (dict(eps=-1.0), ARG), (dict(eps=NAN), ARG), (dict(eps=INF), ARG), (dict(x=0), ARG),
    (dict(x=0x10008), ARG), (dict(ld_x=248), ARG), (dict(ld_x=260), ARG), (dict(residual=0x20004), ARG), (dict(ld_residual=1), ARG),
    (dict(residual=0), ARG), (dict(weight=0x30008), ARG), (dict(sum=0x40004), ARG), (dict(ld_sum=0), ARG), (dict(out=0x50001), ARG),
    (dict(ld_out=255), ARG), (dict(q=0x60004), ARG), (dict(ld_q=252), ARG), (dict(q=0), ARG), (dict(q_scale=0), ARG), (dict(q_scale=0x70002), ARG),
    (dict(ld_scale=1), ARG), (dict(sum=0, out=0, q=0, q_scale=0), ARG)])
def test_norm_refuses(kw, status):
    with pytest.raises(B.MoEError) as e:
        norm(**kw)()
    assert e.value.status == status and e.value.message


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), SHAPE), (dict(cols=0), SHAPE), (dict(cols=4), UNSUPPORTED), (dict(block_rows=64), ARG), (dict(block_rows=0), ARG), (dict(dtype=-1), ARG),
    (dict(x=0), ARG), (dict(q=0), ARG), (dict(scale=0), ARG), (dict(ld_x=264 - 4), ARG), (dict(ld_scale=1), ARG), (dict(cols=40000, ld_x=40000, ld_q=40000, ld_scale=400), UNSUPPORTED),
    (dict(cols=(1 << 21) + 8, block_rows=128, ld_x=1 << 22, ld_q=1 << 22, ld_scale=1 << 20), UNSUPPORTED)])
def test_quantize_refuses(kw, status):
    with pytest.raises(B.MoEError) as e:
        quantize(**kw)()
    assert e.value.status == status and e.value.message


PRODUCT = [(dict(m=-1), SHAPE), (dict(k=0), SHAPE), (dict(k=264, ld_a=272), UNSUPPORTED), (dict(m=(1 << 21) + 1), UNSUPPORTED), (dict(ld_a=1 << 23), UNSUPPORTED),
           (dict(a=0), ARG), (dict(a=0x10008), ARG), (dict(ld_a=240), ARG), (dict(ld_a=264), ARG), (dict(a_scale=0), ARG), (dict(a_scale=0x20002), ARG),
           (dict(ld_a_scale=1), ARG), (dict(ld_a_scale=1 << 21), UNSUPPORTED), (dict(w=0), ARG), (dict(w=0x30004), ARG), (dict(w_scale=0), ARG), (dict(w_scale=0x40001), ARG)]


@pytest.mark.parametrize("kw,status", PRODUCT + [
    (dict(n=0), SHAPE), (dict(n=(1 << 21) + 1, ld_out=1 << 22), UNSUPPORTED), (dict(out_dtype=3), ARG), (dict(out=0), ARG), (dict(out=0x60004), ARG), (dict(ld_out=252), ARG),
    (dict(ld_out=260), ARG), (dict(add=0x50002), ARG), (dict(ld_add=4), ARG), (dict(m=1 << 21, n=1 << 21, ld_out=1 << 21, ld_add=1 << 21), UNSUPPORTED)])
def test_matmul_refuses(kw, status):
    with pytest.raises(B.MoEError) as e:
        matmul(**kw)()
    assert e.value.status == status and e.value.message


@pytest.mark.parametrize("kw,status", PRODUCT + [
    (dict(inter=0), SHAPE), (dict(inter=264, ld_q=264), UNSUPPORTED), (dict(inter=32784, ld_q=40000, ld_scale=400), UNSUPPORTED), (dict(q=0), ARG), (dict(q_scale=0), ARG),
    (dict(q=0x50004), ARG), (dict(ld_q=250), ARG), (dict(ld_scale=1), ARG), (dict(workspace=0, workspace_bytes=0), ARG), (dict(workspace=0x70010), ARG),
    (dict(workspace_bytes=4 * 256 * 4 - 1), CAPACITY)])
def test_swiglu_refuses(kw, status):
    with pytest.raises(B.MoEError) as e:
        swiglu(**kw)()
    assert e.value.status == status and e.value.message


@pytest.mark.parametrize("call", ["moe_rms_norm", "moe_quantize", "moe_scaled_matmul", "moe_scaled_swiglu"])
def test_null_arguments(call):
    assert getattr(B.lib(), call)(None, 0) == ARG


def test_workspace_of_the_swiglu_product():
    """fp32 rows for the products that are streamed, none for the others; nothing for sizes that are refused."""
    assert B.moe_scaled_swiglu_workspace_bytes(4, 256, 2048) == 4 * 256 * 4
    assert B.moe_scaled_swiglu_workspace_bytes(4096, 2048, 7168) == 0
    for sizes in ((0, 256, 2048), (4, 0, 2048), (4, 256, 0), (-1, 256, 256), (1 << 22, 256, 256)):
        assert B.moe_scaled_swiglu_workspace_bytes(*sizes) == 0


def test_no_rows_are_no_work():
    norm(rows=0, x=0)()
    quantize(rows=0, x=0)()
    matmul(m=0, a=0, out=0)()
    swiglu(m=0, a=0, q=0)()


def test_wrong_tensors_are_refused():
    from paper_2510_02613_amd import scaled
    with pytest.raises(ValueError):
        scaled.quantize(torch.zeros(4, 128))                    # not on the GPU
    with pytest.raises(ValueError):
        scaled._matrix(torch.zeros(4, 128), (4, 128), torch.bfloat16, -1, "x")
    with pytest.raises(ValueError):
        scaled._matrix(torch.zeros(128, 4).t(), (4, 128), torch.float32, -1, "x")
    with pytest.raises(ValueError):
        scaled._matrix(torch.zeros(4, 128), (4, 128), torch.float32, 0, "x")        # on another device
    assert scaled._matrix(torch.zeros(4, 256)[:, :128], (4, 128), torch.float32, -1, "x")[1] == 256


def test_reference_rounding_is_e4m3():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    every = every[every.isfinite()].unique()
    assert torch.equal(R.e4m3_round(every), every)
    mid = (every[1:] + every[:-1]) / 2
    near = torch.cat([mid, mid * (1 + 2.0 ** -20), mid * (1 - 2.0 ** -20)])
    assert torch.equal(R.e4m3_round(near), near.float().to(torch.float8_e4m3fn).double())


# ---- the layer with 8-bit experts ----

def layer_cfg(**kw):
    d = dict(hidden=128, inter=64, n_experts=8, top_k=2, n_slots=8, max_tokens=64, act_dtype=B.MOE_BF16,
             router_dtype=0, gate=0, n_group=1, topk_group=1, renormalize=1, routed_scale=1.0, n_shared=0)
    d.update(kw)
    return B.MoEConfig(*[d[f] for f, _ in B.MoEConfig._fields_])


def buffers(cfg):
    return B.MoEBuffers(0x10000, 0, 0, 0x20000, 0x30000, 0x40000, B.moe_scaled_workspace_bytes(cfg))


@pytest.fixture
def layer():
    cfg = layer_cfg()
    h = B.moe_layer_create_scaled(cfg, buffers(cfg), 0x80000, 0x90000)
    yield h
    B.moe_layer_destroy(h)


@pytest.mark.parametrize("kw", [dict(act_dtype=B.MOE_F32), dict(hidden=136), dict(inter=72), dict(hidden=32784), dict(inter=40000), dict(max_tokens=(1 << 20) + 1), dict(hidden=32768, max_tokens=1 << 17)])
def test_layers_that_cannot_have_8bit_experts(kw):
    cfg = layer_cfg(**kw)
    assert B.lib().moe_scaled_workspace_bytes(ctypes.byref(cfg)) == 0
    h = ctypes.c_void_p()
    buf = B.MoEBuffers(0x10000, 0, 0, 0x20000, 0x30000, 0x40000, 1 << 40)
    assert B.lib().moe_layer_create_scaled(ctypes.byref(cfg), ctypes.byref(buf), 0x80000, 0x90000, ctypes.byref(h)) == UNSUPPORTED and h.value is None


@pytest.mark.parametrize("s13,s2,ws,status", [(0, 0x90000, 0, ARG), (0x80000, 0, 0, ARG), (0x80002, 0x90000, 0, ARG), (0x80000, 0x90001, 0, ARG), (0x80000, 0x90000, -1, CAPACITY)])
def test_layer_creation_refuses(s13, s2, ws, status):
    cfg = layer_cfg()
    buf = buffers(cfg)
    buf.workspace_bytes += ws
    with pytest.raises(B.MoEError) as e:
        B.moe_layer_create_scaled(cfg, buf, s13, s2)
    assert e.value.status == status


def refused(status, call, *args):
    with pytest.raises(B.MoEError) as e:
        call(*args)
    assert e.value.status == status, e.value


def test_passes_and_fills_that_are_refused(layer):
    fwd = lambda x=0x100000, xq=0x200000, xs=0x300000, T=4, ids=0x400000, w=0x500000, out=0x600000, b=0, e=0, flags=0: (  # noqa: E731
        B.moe_forward_scaled(layer, x, xq, xs, T, ids, w, out, b, e, 0, flags))
    refused(B.MOE_ERR_MAP, fwd)                                                  # no placement yet
    # the placement's upload needs a GPU: what follows is refused in front of it, or before the map is looked at
    refused(ARG, lambda: fwd(xq=0))
    refused(ARG, lambda: fwd(xs=0))
    refused(ARG, lambda: fwd(xq=0x200008))
    refused(ARG, lambda: fwd(xs=0x300002))
    refused(ARG, lambda: fwd(ids=0))
    refused(ARG, lambda: fwd(w=0))
    refused(ARG, lambda: fwd(ids=0x400001))
    refused(ARG, lambda: fwd(T=-1))
    refused(CAPACITY, lambda: fwd(T=65))
    refused(ARG, lambda: fwd(b=2, e=1))
    refused(ARG, lambda: fwd(flags=1 << 20))
    refused(ARG, lambda: B.moe_forward_scaled(None, 0x100000, 0x200000, 0x300000, 4, 0x400000, 0x500000, 0x600000))
    refused(UNSUPPORTED, lambda: B.moe_load_expert(layer, 3, 0x100000, 0x200000, 1, 2))
    load = lambda slot=3, a=0x100000, b=0x200000, c=0x300000, d=0x400000, cs=1, ss=2, n=0: B.moe_load_expert_scaled(layer, slot, a, b, c, d, cs, ss, n)  # noqa: E731
    for kw in (dict(slot=8), dict(slot=-1), dict(a=0), dict(b=0), dict(c=0), dict(d=0), dict(a=0x100008), dict(b=0x200001), dict(cs=2), dict(n=-1)):
        refused(ARG, lambda: load(**kw))


def test_layers_of_the_other_kind():
    cfg = layer_cfg()
    h = B.moe_layer_create(cfg, B.MoEBuffers(0x10000, 0, 0, 0x20000, 0x30000, 0x40000, B.moe_workspace_bytes(cfg)))
    refused(UNSUPPORTED, lambda: B.moe_forward_scaled(h, 0x100000, 0x200000, 0x300000, 4, 0x400000, 0x500000, 0x600000))
    refused(UNSUPPORTED, lambda: B.moe_load_expert_scaled(h, 3, 0x100000, 0x200000, 0x300000, 0x400000, 1, 2))
    B.moe_layer_destroy(h)
