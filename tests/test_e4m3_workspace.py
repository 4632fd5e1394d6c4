"""The workspace of layers with experts in e4m3, on the host."""
import pytest

import paper_2506_23635_amd as moe


@pytest.mark.parametrize("d,f,E,k,local", [(256, 512, 8, 2, 8), (6144, 10752, 16, 4, 16), (6144, 10752, 16, 4, 4), (512, 384, 8, 6, 2)])
def test_few_tokens_values_take_no_more_than_many_tokens_rows(d, f, E, k, local):
    """A call of up to 16 tokens needs 6 bytes per element of H (bf16 and fp32), a larger one 2: from 48
    tokens on the workspace is that of a bf16 layer, below it lies between the two needs."""
    def size(T, flags):
        return moe.moe_workspace_bytes(moe.make_config(d, f, E, k, n_local_experts=local, max_tokens=T, flags=flags))
    row = min(k, local) * f
    for T in (1, 3, 16, 17, 40, 48, 49, 100, 2048):
        more = size(T, moe.MOE_E4M3) - size(T, 0)
        need = max(6 * min(T, 16), 2 * T) * row - 2 * T * row
        assert need <= more <= need + 512, T          # (256-byte alignment)
    assert size(48, moe.MOE_E4M3) == size(48, 0)
