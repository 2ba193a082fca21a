"""What the 4-bit operators refuse, before anything is launched (no GPU needed), and the reference of their GPU tests."""
import ctypes
import os
import re

import pytest
import torch

import four_bit_ref as R
from paper_2510_02613_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "elasticmoe_four_bit.h")
ARG, SHAPE, UNSUPPORTED = B.MOE_ERR_ARG, B.MOE_ERR_SHAPE, B.MOE_ERR_UNSUPPORTED


@pytest.mark.parametrize("struct,name", [(B.MoEFourBitQuantize, "moe_four_bit_quantize_t"), (B.MoEFourBitMatmul, "moe_four_bit_matmul_t"),
                                         (B.MoEFourBitSwiglu, "moe_four_bit_swiglu_t")])
def test_structs_match_the_header(struct, name):
    hdr = open(HEADER).read()
    end = hdr.index("} %s;" % name)
    body = re.sub(r"/\*.*?\*/", "", hdr[hdr.rindex("typedef struct {", 0, end):end], flags=re.S)
    ctype = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64}
    fields = []
    for kind, names in re.findall(r"(const int32_t|int32_t|int64_t|const void|void)\s+([^;]+);", body):
        for n in names.split(","):
            fields.append((n.strip(" *"), ctypes.c_void_p if "*" in n else ctype[kind]))
    assert fields == struct._fields_


def test_library_exports_every_declared_symbol():
    declared = set(re.findall(r"^(?:moe_status_t|size_t) (moe_[a-z_0-9]+)\(", open(HEADER).read(), re.M))
    assert declared == set(B.EXPORTS_FOUR_BIT)
    for name in declared:
        assert hasattr(B.lib(), name), name


def quantize(**kw):
    d = dict(rows=4, cols=256, dtype=B.MOE_BF16, x=0x10000, ld_x=256, q=0x20000, ld_q=128, scale=0x30001, ld_scale=8, values=0x40000, ld_values=256)
    d.update(kw)
    return lambda: B.moe_four_bit_quantize(B.MoEFourBitQuantize(**d))


def matmul(**kw):
    d = dict(m=4, n=100, k=256, groups=3, out_dtype=B.MOE_BF16, a=0x10000, ld_a=256, offsets=0x20000, w=0x30000, w_scale=0x40001, add=0x50000, ld_add=104,
             out=0x60000, ld_out=104)
    d.update(kw)
    return lambda: B.moe_four_bit_matmul(B.MoEFourBitMatmul(**d))


def swiglu(**kw):
    d = dict(m=4, inter=100, k=256, groups=3, out_dtype=B.MOE_BF16, a=0x10000, ld_a=256, offsets=0x20000, w=0x30000, w_scale=0x40001, out=0x60000, ld_out=104)
    d.update(kw)
    return lambda: B.moe_four_bit_swiglu(B.MoEFourBitSwiglu(**d))


def refused(call, status):
    with pytest.raises(B.MoEError) as e:
        call()
    assert e.value.status == status and e.value.message


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), SHAPE), (dict(cols=0), SHAPE), (dict(cols=240), UNSUPPORTED), (dict(rows=(1 << 21) + 1), UNSUPPORTED), (dict(cols=(1 << 21) + 32), UNSUPPORTED), (dict(dtype=2), ARG),
    (dict(x=0), ARG), (dict(x=0x10008), ARG), (dict(ld_x=248), ARG), (dict(ld_x=260), ARG), (dict(q=0), ARG), (dict(q=0x20002), ARG), (dict(ld_q=124), ARG), (dict(ld_q=130), ARG),
    (dict(scale=0), ARG), (dict(ld_scale=7), ARG), (dict(values=0x40004), ARG), (dict(ld_values=8), ARG), (dict(ld_q=(1 << 40) + 4), UNSUPPORTED), (dict(ld_x=(1 << 40) + 8), UNSUPPORTED)])
def test_quantize_refuses(kw, status):
    refused(quantize(**kw), status)


PRODUCT = [(dict(m=-1), SHAPE), (dict(k=0), SHAPE), (dict(k=272, ld_a=272), UNSUPPORTED), (dict(k=(1 << 21) + 32), UNSUPPORTED), (dict(m=(1 << 21) + 1), UNSUPPORTED), (dict(groups=0), SHAPE),
           (dict(groups=2048), UNSUPPORTED), (dict(offsets=0), ARG), (dict(offsets=0x20002), ARG), (dict(out_dtype=2), ARG), (dict(a=0), ARG), (dict(a=0x10008), ARG), (dict(ld_a=248), ARG),
           (dict(ld_a=260), ARG), (dict(ld_a=1 << 24), UNSUPPORTED), (dict(w=0), ARG), (dict(w=0x30008), ARG), (dict(w_scale=0), ARG), (dict(out=0), ARG), (dict(out=0x60004), ARG), (dict(ld_out=96), ARG), (dict(ld_out=100), ARG)]


@pytest.mark.parametrize("kw,status", PRODUCT + [
    (dict(n=0), SHAPE), (dict(n=(1 << 21) + 1, ld_out=1 << 22, ld_add=1 << 22), UNSUPPORTED), (dict(add=0x50008), ARG), (dict(ld_add=96), ARG),
    (dict(n=1 << 21, groups=2047, ld_out=1 << 21, ld_add=1 << 21), UNSUPPORTED)])
def test_matmul_refuses(kw, status):
    refused(matmul(**kw), status)


@pytest.mark.parametrize("kw,status", PRODUCT + [(dict(inter=0), SHAPE), (dict(inter=(1 << 20) + 1, ld_out=1 << 22), UNSUPPORTED)])
def test_swiglu_refuses(kw, status):
    refused(swiglu(**kw), status)


@pytest.mark.parametrize("call", ["moe_four_bit_quantize", "moe_four_bit_matmul", "moe_four_bit_swiglu"])
def test_null_arguments(call):
    assert getattr(B.lib(), call)(None, 0) == ARG


def test_no_rows_are_no_work():
    quantize(rows=0, x=0, q=0, scale=0)()
    matmul(m=0, a=0, out=0)()
    swiglu(m=0, a=0, out=0)()


def test_the_python_calls_refuse(monkeypatch):
    from paper_2510_02613_amd import four_bit as Q
    monkeypatch.setattr(Q, "_device_of", lambda t: -1)              # the CPU's
    monkeypatch.setattr(Q, "_current_device", lambda: -1)
    monkeypatch.setattr(Q, "_current_stream", lambda dev: 0)
    for name in ("moe_four_bit_quantize", "moe_four_bit_matmul", "moe_four_bit_swiglu"):
        monkeypatch.setattr(Q.B, name, lambda *a: None)
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)  # noqa: E731
    a, w, s = torch.zeros(5, 64, dtype=torch.bfloat16), u8(24, 32), u8(24, 2)
    off = torch.zeros(4, dtype=torch.int32)
    assert Q.matmul(a, w, s).shape == (5, 24) and Q.swiglu(a, w, s, out_dtype=torch.float32).shape == (5, 12)
    assert Q.matmul(a, w.view(torch.float4_e2m1fn_x2), s.view(torch.float8_e8m0fnu)).dtype == torch.bfloat16
    assert not Q.swiglu(a, u8(3, 24, 32), u8(3, 24, 2), offsets=off).any()
    bad = [lambda: Q.matmul(a.float(), w, s), lambda: Q.matmul(a, w.int(), s), lambda: Q.matmul(a, w, s.float()), lambda: Q.matmul(a, w, u8(24, 3)), lambda: Q.matmul(a, u8(24, 31), s),
           lambda: Q.matmul(a, w, s, offsets=off), lambda: Q.matmul(a, u8(3, 24, 32), u8(3, 24, 2)), lambda: Q.matmul(a, u8(4, 24, 32), u8(4, 24, 2), offsets=off),
           lambda: Q.matmul(a, w, s, out=torch.zeros(5, 23)), lambda: Q.matmul(a, w, s, out=torch.zeros(5, 24).half()), lambda: Q.matmul(a, w, s, add=torch.zeros(5, 24), out=torch.zeros(5, 24).bfloat16()),
           lambda: Q.matmul(a, w.t().contiguous().t(), s), lambda: Q.matmul(a, u8(3, 24, 32), u8(3, 24, 2), offsets=off.long()), lambda: Q.swiglu(a, u8(23, 32), u8(23, 2)),
           lambda: Q.matmul(a.clone().requires_grad_(), w, s), lambda: Q.swiglu(a.clone().requires_grad_(), w, s), lambda: Q.matmul(a, w, s, add=torch.zeros(5, 24, requires_grad=True)),
           lambda: Q.quantize(torch.zeros(4, 64).half()), lambda: Q.quantize(torch.zeros(4)), lambda: Q.quantize(torch.zeros(4, 64), q=u8(4, 31)), lambda: Q.quantize(torch.zeros(4, 64), scale=torch.zeros(4, 2)),
           lambda: Q.quantize(torch.zeros(4, 64), values=torch.zeros(4, 64).bfloat16()), lambda: Q.quantize(torch.zeros(4, 64, requires_grad=True))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    with torch.no_grad():
        Q.matmul(a.clone().requires_grad_(), w, s)


def test_the_reference_rounds_as_the_format_says():
    x = torch.zeros(1, 32)
    x[0, :14] = torch.tensor([6.0, 0.25, 0.2500001, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.0000005, -0.0, -0.1, -6.0, 0.7499999])
    codes, powers = R.quantize(x)
    assert powers.item() == 127 and codes[0, :14].tolist() == [7, 0, 1, 2, 2, 4, 4, 6, 6, 7, 8, 8, 15, 1]
    for top, power in ((6.0000005, 128), (12.0, 128), (3.0, 126), (3.0000002, 127), (0.0, 0), (2.0 ** -149, 0), (3.4e38, 253)):
        x[0, 0] = top
        x[0, 1:] = 0
        assert R.quantize(x)[1].item() == power, top
    x[0, 5] = float("inf")
    codes, powers = R.quantize(x)
    assert powers.item() == 255 and not codes.any()
    assert torch.equal(R.values(R.packed(torch.arange(16, dtype=torch.uint8).repeat(2)[None]), torch.tensor([[129]], dtype=torch.uint8))[0, :8], 4 * R.STEPS[:8])


def test_the_reference_tells_mistakes_apart():
    g = torch.Generator().manual_seed(1)
    codes, powers = R.quantize(0.02 * torch.randn(8, 256, generator=g))
    w, a = R.values(R.packed(codes), powers), torch.randn(4, 256, generator=g).bfloat16().double()
    y, off = R.product(a, torch.zeros_like(a), w)
    R.check(y.float(), y, off)
    R.check(y.bfloat16(), y, off)
    for planted in (y * 1.01, y + 0.01 * w[:, 3], torch.full_like(y, float("nan"))):
        with pytest.raises(AssertionError):
            R.check(planted.bfloat16(), y, off)
    with pytest.raises(AssertionError):
        R.check_norm((y * (1 + 2.0 ** -8)).float(), y, torch.float32)
