"""How much the calls on e4m3 take: blocks are counted in 32 bits, so more than 2^31 are refused, and
numbers past int32 are refused as what they are, not taken modulo 2^32."""
import pytest

import paper_2506_23635_amd as moe

E_ARG, E_SHAPE, E_CAPACITY = -1, -2, -4


@pytest.mark.parametrize("T,n,status", [(1 << 24, 128 * 128, E_ARG), (1 << 24, 128 * 128 + 16, E_SHAPE), (1 << 24, 1 << 24, E_SHAPE),
                                        ((1 << 14) + 1, 1 << 24, E_SHAPE), (1 << 14, 1 << 24, E_ARG), (1 << 14, (1 << 24) - 128, E_ARG),
                                        ((1 << 14) + 1, (1 << 24) - 128, E_SHAPE)])
def test_most_blocks(T, n, status):
    """codes and scales at one address: what fits is refused next, for the overlap."""
    assert (T * -(-n // 128) > 1 << 31) == (status == E_SHAPE)
    assert moe.lib().moe_quantize_e4m3(1 << 55, n, moe.T_BF16, T, n, 1 << 50, 1 << 50, None) == status


@pytest.mark.parametrize("T,n", [(1 << 32, 16), ((1 << 32) + 1, 16), (1 << 40, 16), (1, (1 << 32) + 16), (1 << 31, 16)])
def test_rows_past_32_bits(T, n):
    with pytest.raises(moe.MoeError) as err:
        moe.moe_quantize_e4m3(1 << 50, n, moe.T_BF16, T, n, 1 << 55, 1 << 58)
    assert err.value.status == E_SHAPE


@pytest.mark.parametrize("T,status", [(1 << 32, E_CAPACITY), ((1 << 32) + 1, E_CAPACITY), (-(1 << 32), E_ARG), (-(1 << 32) + 1, E_ARG)])
def test_product_of_rows_past_32_bits(T, status):
    ctx = moe.moe_linear_init(moe.make_linear_config(128, 256, max_tokens=4), 1 << 20, 1 << 30)
    try:
        with pytest.raises(moe.MoeError) as err:
            moe.moe_linear_forward(ctx, 1 << 32, 128, 1 << 33, moe.T_F32, T)
        assert err.value.status == status
    finally:
        moe.lib().moe_linear_destroy(ctx)


@pytest.mark.parametrize("layer", [1 << 32, -(1 << 32), (1 << 32) + 1, 1 << 31])
def test_policy_of_a_layer_past_32_bits(layer):
    ctx = moe.moe_init(moe.make_config(256, 128, 4, 2, n_layers=2), 1 << 20, 1 << 30)
    try:
        with pytest.raises(moe.MoeError) as err:
            moe.moe_set_policy(ctx, layer, moe.make_policy())
        assert err.value.status == E_ARG
    finally:
        moe.moe_destroy(ctx)
