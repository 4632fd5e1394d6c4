"""How many blocks moe_quantize_e4m3 takes: they are counted in 32 bits, so more than 2^31 are refused."""
import pytest

import paper_2506_23635_amd as moe

E_ARG, E_SHAPE = -1, -2


@pytest.mark.parametrize("T,n,status", [(1 << 24, 128 * 128, E_ARG), (1 << 24, 128 * 128 + 16, E_SHAPE), (1 << 24, 1 << 24, E_SHAPE),
                                        ((1 << 14) + 1, 1 << 24, E_SHAPE), (1 << 14, 1 << 24, E_ARG), (1 << 14, (1 << 24) - 128, E_ARG),
                                        ((1 << 14) + 1, (1 << 24) - 128, E_SHAPE)])
def test_most_blocks(T, n, status):
    """codes and scales at one address: what fits is refused next, for the overlap."""
    assert (T * -(-n // 128) > 1 << 31) == (status == E_SHAPE)
    assert moe.lib().moe_quantize_e4m3(1 << 55, n, moe.T_BF16, T, n, 1 << 50, 1 << 50, None) == status
