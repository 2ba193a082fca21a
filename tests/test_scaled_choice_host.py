"""What the calls of the 8-bit path refuse of the choice of the 8-bit matrix instructions (no GPU needed)."""
import pytest

from paper_2510_02613_amd import binding as B
from test_scaled_host import buffers, layer_cfg, matmul, refused


@pytest.mark.parametrize("out_dtype,status", [(B.MOE_F32 | B.MOE_FAST_PRODUCTS, B.MOE_ERR_UNSUPPORTED), (2 | B.MOE_FAST_PRODUCTS, B.MOE_ERR_ARG),
                                              (B.MOE_BF16 | 0x200, B.MOE_ERR_ARG), (B.MOE_BF16 | 0x1100, B.MOE_ERR_ARG)])
def test_matmul_refuses(out_dtype, status):
    with pytest.raises(B.MoEError) as e:
        matmul(out_dtype=out_dtype)()
    assert e.value.status == status and e.value.message


def test_matmul_takes_the_choice():
    """Refused for its rows, not for its type."""
    with pytest.raises(B.MoEError) as e:
        matmul(out_dtype=B.MOE_BF16 | B.MOE_FAST_PRODUCTS, out=0)()
    assert e.value.message == "out is NULL"
    matmul(out_dtype=B.MOE_BF16 | B.MOE_FAST_PRODUCTS, m=0)()


def test_only_layers_with_8bit_experts_take_the_flag():
    cfg = layer_cfg()
    h = B.moe_layer_create_scaled(cfg, buffers(cfg), 0x80000, 0x90000)
    refused(B.MOE_ERR_MAP, lambda: B.moe_forward(h, 0x100000, 4, 0x600000, 0, 0, 0, B.MOE_FLAG_FAST_PRODUCTS))      # no placement yet: the flag is fine
    refused(B.MOE_ERR_MAP, lambda: B.moe_forward_scaled(h, 0x100000, 0x200000, 0x300000, 4, 0x400000, 0x500000, 0x600000, 0, 0, 0, B.MOE_FLAG_FAST_PRODUCTS))
    B.moe_layer_destroy(h)
    h = B.moe_layer_create(cfg, B.MoEBuffers(0x10000, 0, 0, 0x20000, 0x30000, 0x40000, B.moe_workspace_bytes(cfg)))
    refused(B.MOE_ERR_ARG, lambda: B.moe_forward(h, 0x100000, 4, 0x600000, 0, 0, 0, B.MOE_FLAG_FAST_PRODUCTS))
    B.moe_layer_destroy(h)
