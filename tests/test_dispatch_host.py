"""What the operators that sort tokens by expert refuse, before anything is launched (no GPU needed), and the reference of their GPU tests."""
import ctypes
import os
import re

import pytest
import torch

import dispatch_ref as R
from paper_2510_02613_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "elasticmoe_dispatch.h")
ARG, SHAPE, UNSUPPORTED, CAPACITY = B.MOE_ERR_ARG, B.MOE_ERR_SHAPE, B.MOE_ERR_UNSUPPORTED, B.MOE_ERR_CAPACITY


@pytest.mark.parametrize("struct,name", [(B.MoESortTokens, "moe_sort_tokens_t"), (B.MoECombineTokens, "moe_combine_tokens_t"),
                                         (B.MoECombineTokensBackward, "moe_combine_tokens_backward_t")])
def test_structs_match_the_header(struct, name):
    hdr = open(HEADER).read()
    end = hdr.index("} %s;" % name)
    body = re.sub(r"/\*.*?\*/", "", hdr[hdr.rindex("typedef struct {", 0, end):end], flags=re.S)
    ctype = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float, "size_t": ctypes.c_size_t}
    fields = []
    for kind, names in re.findall(r"(const int32_t|int32_t|int64_t|size_t|const void|const float|float|void)\s+([^;]+);", body):
        for n in names.split(","):
            fields.append((n.strip(" *"), ctypes.c_void_p if "*" in n else ctype[kind]))
    assert fields == struct._fields_


def test_library_exports_every_declared_symbol():
    declared = set(re.findall(r"^(?:moe_status_t|size_t) (moe_[a-z_0-9]+)\(", open(HEADER).read(), re.M))
    assert declared == set(B.EXPORTS_DISPATCH)
    for name in declared:
        assert hasattr(B.lib(), name), name


def sort(**kw):
    d = dict(tokens=600, top_k=8, n_groups=16, n_experts=32, cols=256, dtype=B.MOE_BF16, zero_rest=0, ids=0x10000, expert_map=0x20000, x=0x30000, ld_x=256,
             rows=0x40000, ld_rows=256, offsets=0x50000, source=0x60000, row=0x70000, workspace=0x80000, workspace_bytes=5 * 17 * 4)
    d.update(kw)
    return lambda: B.moe_sort_tokens(B.MoESortTokens(**d))


def combine(**kw):
    d = dict(tokens=4, top_k=8, cols=256, dtype=B.MOE_BF16, y=0x10000, ld_y=256, row=0x20000, weights=0x30000, out=0x40000, ld_out=256)
    d.update(kw)
    return lambda: B.moe_combine_tokens(B.MoECombineTokens(**d))


def backward(**kw):
    d = dict(tokens=4, top_k=8, cols=256, dtype=B.MOE_BF16, grad_out=0x10000, ld_grad_out=256, y=0x20000, ld_y=256, row=0x30000, weights=0x40000, source=0x50000,
             grad_y=0x60000, ld_grad_y=256, grad_weights=0x70000)
    d.update(kw)
    return lambda: B.moe_combine_tokens_backward(B.MoECombineTokensBackward(**d))


COMMON = [(dict(tokens=-1), SHAPE), (dict(top_k=0), SHAPE), (dict(cols=0), SHAPE), (dict(cols=252), UNSUPPORTED), (dict(cols=(1 << 21) + 8), UNSUPPORTED),
          (dict(tokens=(1 << 21) + 1), UNSUPPORTED), (dict(top_k=33), UNSUPPORTED), (dict(dtype=2), ARG), (dict(row=0), ARG), (dict(row=0x20002), ARG)]


def refused(call, status):
    with pytest.raises(B.MoEError) as e:
        call()
    assert e.value.status == status and e.value.message


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(n_groups=0), SHAPE), (dict(n_groups=2048), UNSUPPORTED), (dict(n_experts=0), SHAPE), (dict(expert_map=0x20001), ARG), (dict(ids=0), ARG), (dict(ids=0x10001), ARG),
    (dict(x=0), ARG), (dict(rows=0), ARG), (dict(x=0x30008), ARG), (dict(rows=0x40002), ARG), (dict(ld_x=248), ARG), (dict(ld_x=260), ARG), (dict(ld_rows=0), ARG),
    (dict(ld_rows=(1 << 40) + 8), UNSUPPORTED), (dict(offsets=0), ARG), (dict(offsets=0x50002), ARG), (dict(source=0), ARG), (dict(source=0x60003), ARG),
    (dict(workspace=0), ARG), (dict(workspace=0x80008), ARG), (dict(workspace_bytes=5 * 17 * 4 - 1), CAPACITY), (dict(tokens=0, offsets=0), ARG)])
def test_sort_refuses(kw, status):
    refused(sort(**kw), status)


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(y=0), ARG), (dict(y=0x10004), ARG), (dict(ld_y=8), ARG), (dict(weights=0x30001), ARG), (dict(out=0), ARG), (dict(out=0x40008), ARG), (dict(ld_out=252), ARG)])
def test_combine_refuses(kw, status):
    refused(combine(**kw), status)


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(grad_out=0), ARG), (dict(grad_out=0x10004), ARG), (dict(ld_grad_out=8), ARG), (dict(y=0), ARG), (dict(y=0x20008), ARG), (dict(ld_y=255), ARG), (dict(weights=0x40002), ARG),
    (dict(source=0x50001), ARG), (dict(grad_y=0x60008), ARG), (dict(ld_grad_y=8), ARG), (dict(grad_weights=0x70002), ARG), (dict(grad_y=0, grad_weights=0), ARG)])
def test_backward_refuses(kw, status):
    refused(backward(**kw), status)


@pytest.mark.parametrize("call", ["moe_sort_tokens", "moe_combine_tokens", "moe_combine_tokens_backward"])
def test_null_arguments(call):
    assert getattr(B.lib(), call)(None, 0) == ARG


def test_no_tokens_is_nothing_to_add_up():
    combine(tokens=0, y=0, row=0, out=0)()
    backward(tokens=0, grad_out=0, row=0)()


def test_workspace_of_the_sort():
    size = B.moe_sort_tokens_workspace_bytes
    assert size(512, 8, 128) == 0 and size(513, 8, 128) == 5 * 129 * 4 and size(1 << 21, 32, 2047) == (1 << 16) * 2048 * 4
    assert size(-1, 8, 8) == size(1000, 33, 8) == size(1000, 8, 2048) == size(1000, 8, 0) == 0
    sizes = [size(t, 8, 100) for t in range(0, 3000, 50)]
    assert sizes == sorted(sizes)


def test_the_python_calls_refuse(monkeypatch):
    from paper_2510_02613_amd import dispatch as D
    monkeypatch.setattr(D, "_device_of", lambda t: -1)              # the CPU's
    monkeypatch.setattr(D, "_current_device", lambda: -1)
    monkeypatch.setattr(D, "_current_stream", lambda dev: 0)
    for name in ("moe_sort_tokens", "moe_combine_tokens", "moe_combine_tokens_backward"):
        monkeypatch.setattr(D.B, name, lambda *a: None)
    x, ids = torch.zeros(4, 64), torch.zeros(4, 2, dtype=torch.int32)
    order = D.Order(torch.zeros(4, dtype=torch.int32), torch.zeros(8, dtype=torch.int32), ids)
    D.sort_tokens(x, ids, 3, order=order)
    D.combine_tokens(torch.zeros(8, 64), order, torch.zeros(4, 2))
    bad = [lambda: D.sort_tokens(x.half(), ids, 3), lambda: D.sort_tokens(x[0], ids, 3), lambda: D.sort_tokens(x, ids.long(), 3), lambda: D.sort_tokens(x, ids[:3], 3),
           lambda: D.sort_tokens(x, ids[:, 0], 3), lambda: D.sort_tokens(x, ids, 0), lambda: D.sort_tokens(x, ids, 3, expert_map=ids), lambda: D.sort_tokens(x, ids, 4, order=order),
           lambda: D.sort_tokens(x, ids, 3, expert_map=torch.zeros(4)), lambda: D.sort_tokens(x, ids, 3, rows=torch.zeros(7, 64)), lambda: D.sort_tokens(x.t(), ids, 3),
           lambda: D.sort_tokens(x, ids, 3, rows=torch.zeros(8, 64, dtype=torch.bfloat16)), lambda: D.sort_tokens(x, torch.zeros(2, 4, dtype=torch.int32).t(), 3),
           lambda: D.sort_tokens(x, ids, 3, workspace=torch.zeros(8, 2).t()),
           lambda: D.combine_tokens(torch.zeros(7, 64), order), lambda: D.combine_tokens(torch.zeros(8, 64), order, torch.zeros(4, 2).bfloat16()),
           lambda: D.combine_tokens(torch.zeros(8, 64), order, torch.zeros(2, 4)), lambda: D.combine_tokens(torch.zeros(8, 64), order, out=torch.zeros(4, 32)),
           lambda: D.combine_tokens(torch.zeros(8, 64), order._replace(row=ids.flatten())), lambda: D.combine_tokens(torch.zeros(8, 64), order._replace(row=ids.long()))]
    leaf = torch.zeros(4, 64, requires_grad=True)
    bad += [lambda: D.sort_tokens(leaf, ids, 3, rows=torch.zeros(8, 64)), lambda: D.sort_tokens(leaf, ids, 3, order=order), lambda: D.sort_tokens(leaf, ids, 3, stream=object()),
            lambda: D.combine_tokens(torch.zeros(8, 64, requires_grad=True), order, out=torch.zeros(4, 64)),
            lambda: D.combine_tokens(torch.zeros(8, 64, requires_grad=True), order._replace(source=order.source.long())),
            lambda: D.combine_tokens(torch.zeros(8, 64, requires_grad=True), order._replace(source=order.source[:7])),
            lambda: D.combine_tokens(torch.zeros(8, 64, requires_grad=True), order._replace(source=None)),
            lambda: D.sort_tokens(x, ids, 3, rows=torch.zeros(8, 64, requires_grad=True)),
            lambda: D.combine_tokens(torch.zeros(8, 64), order, out=torch.zeros(4, 64, requires_grad=True))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    with torch.no_grad():
        D.sort_tokens(leaf, ids, 3, rows=torch.zeros(8, 64), order=order)


def test_tensors_on_the_cpu_are_refused():
    from paper_2510_02613_amd import dispatch as D
    with pytest.raises(ValueError):
        D.sort_tokens(torch.zeros(4, 64), torch.zeros(4, 2, dtype=torch.int32), 3)


def test_the_reference_tells_orders_apart():
    ids = torch.tensor([[2, 0], [0, 2], [5, 1]], dtype=torch.int32)
    offsets, source, row = R.order(ids, 3)
    assert offsets.tolist() == [0, 2, 3, 5] and source.tolist() == [1, 2, 5, 0, 3, -1] and row.tolist() == [[3, 0], [1, 4], [-1, 2]]
    offsets, source, row = R.order(ids, 2, torch.tensor([1, -1, 0], dtype=torch.int32))
    assert offsets.tolist() == [0, 2, 4] and source.tolist() == [0, 3, 1, 2, -1, -1]
    y = torch.randn(6, 8)
    out, off = R.combine(y, row, torch.ones(3, 2))
    R.check(out.float(), out, off, "same")
    for planted in (1.001, -1.0):
        with pytest.raises(AssertionError):
            R.check((out * planted).float(), out, off, "other")
