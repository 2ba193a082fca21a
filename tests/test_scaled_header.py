"""The header of the 8-bit path names every limit that a layer's configuration is refused for (no GPU needed)."""
import ctypes
import os

import pytest

from paper_2510_02613_amd import binding as B
from test_scaled_host import ROOT, UNSUPPORTED, layer_cfg

HEADER = open(os.path.join(ROOT, "include", "elasticmoe_scaled.h")).read()
LAYER = HEADER[HEADER.index("A layer whose experts are held in 8 bits"):]


@pytest.mark.parametrize("kw,text", [
    (dict(act_dtype=B.MOE_F32), "act_dtype not MOE_BF16"), (dict(hidden=136), "H or I no multiple of 16"), (dict(inter=72), "H or I no multiple of 16"),
    (dict(hidden=32784), "or > 32768"), (dict(inter=32784), "or > 32768"), (dict(hidden=32768, max_tokens=1 << 17), "max_tokens * hidden >= 2^32"),
    (dict(max_tokens=(1 << 20) + 1), "max_tokens * (top_k + n_shared) > 2^21")])
def test_limits_of_layers(kw, text):
    cfg, h = layer_cfg(**kw), ctypes.c_void_p()
    buf = B.MoEBuffers(0x10000, 0, 0, 0x20000, 0x30000, 0x40000, 1 << 40)
    assert B.lib().moe_layer_create_scaled(ctypes.byref(cfg), ctypes.byref(buf), 0x80000, 0x90000, ctypes.byref(h)) == UNSUPPORTED
    assert text in LAYER
