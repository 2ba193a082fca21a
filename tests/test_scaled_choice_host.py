"""What the calls of the 8-bit path refuse of the choice of the 8-bit matrix instructions (no GPU needed)."""
import pytest

from paper_2510_02613_amd import binding as B
from test_scaled_host import matmul


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
