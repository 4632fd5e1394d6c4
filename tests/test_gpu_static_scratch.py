"""moe_forward_static's scratch: the tokens that fit, and routings whose partial sums share the space
of O there, bit for bit as moe_forward."""
import pytest

import paper_2506_23635_amd as moe

pytestmark = pytest.mark.gpu

SCRATCH = 8 << 20    # MOE_STATIC_SCRATCH_BYTES


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def make(torch, d, f, E, k, T, flags=0, first=0, local=0):
    layer = moe.MoeLayer(moe.make_config(d, f, E, k, expert_begin=first, n_local_experts=local, max_tokens=T, flags=flags))
    g = torch.Generator(device="cuda").manual_seed(d + f + E)

    def normal(*shape, sigma=1.0):
        return torch.randn(shape, generator=g, device="cuda") * sigma
    layer.load_router(0, normal(d, E, sigma=d ** -0.5), normal(E, sigma=0.5))
    for e in range(first, first + (local or E)):
        layer.load_expert(0, e, *(normal(*s, sigma=s[0] ** -0.5).to(torch.bfloat16) for s in ((d, f), (d, f), (f, d))))
    return layer, normal(T, d).to(torch.bfloat16)


def check_equal(torch, layer, x):
    y, s = torch.full_like(x, 3.0), torch.full_like(x, 5.0)
    layer.forward(0, x, y)
    layer.forward_static(0, x, s)
    assert torch.equal(y, s)


# the most tokens for which the arrays, with 2 KiB of partial sums for each 512 of d, are 8 MiB
@pytest.mark.parametrize("d,f,E,k,T", [(256, 512, 8, 2, 2015), (1024, 2048, 8, 2, 509), (4096, 2048, 32, 2, 203),
                                       (6144, 1024, 64, 8, 39)])
def test_the_scratch_holds_as_many_tokens(torch, d, f, E, k, T):
    more = SCRATCH // (k * (2 * f + 4 * d)) + 1          # H and O alone are more than the scratch
    layer, x = make(torch, d, f, E, k, more)
    for n in (T, 17, 16, 1):
        check_equal(torch, layer, x[:n])
    s = torch.full_like(x, 7.0)
    with pytest.raises(moe.MoeError) as err:
        layer.forward_static(0, x, s)
    assert err.value.status == -4 and bool((s == 7).all())
    layer.close()


@pytest.mark.parametrize("flags", [0, moe.MOE_E4M3])
@pytest.mark.parametrize("d,E,k,first,local", [(1024, 16, 2, 0, 0), (1536, 40, 1, 0, 0), (2048, 64, 8, 60, 1), (512, 8, 2, 3, 2)])
def test_partial_sums_beside_the_rounded_rows(torch, d, E, k, first, local, flags):
    """Few tokens and few slots, where the partial sums are as large as O or larger, up to many."""
    layer, x = make(torch, d, 256, E, k, 400, flags, first, local)
    layer.set_policy(0, moe.make_policy(moe.SCORE_SIGMOID))
    for T in (1, 2, 5, 16, 17, 18, 33, 100, 400):
        check_equal(torch, layer, x[:T])
    layer.close()


@pytest.mark.parametrize("d,f,E,k,T", [(256, 512, 8, 2, 2015), (1024, 2048, 8, 2, 509), (4096, 2048, 32, 2, 203),
                                       (256, 10752, 16, 4, 92)])
def test_as_many_tokens_with_experts_in_e4m3(torch, d, f, E, k, T):
    """The fp32 values of H of few tokens take no space from a call of more; calls of few tokens beside
    them stay right in a context for many."""
    layer, x = make(torch, d, f, E, k, T, moe.MOE_E4M3)
    for n in (T, 16, 3, T, 1):
        check_equal(torch, layer, x[:n])
    layer.close()
