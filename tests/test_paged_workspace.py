"""The paged cache's workspace on the host."""
import paper_2506_23635_amd as moe


def config(**kw):
    base = dict(n_heads=48, n_kv_heads=8, head_dim=128, page_size=64, n_pages=100, max_seqs=4, max_tokens=64, max_blocks=16)
    base.update(kw)
    return moe.make_paged_config(**base)


def test_partial_sums_are_for_positions_that_there_are():
    """Row blocks are divided into steps of 64 positions: sequences of one step are not divided at
    all, and a few blocks of a few steps need no more partial sums than that.  (A block's sums of one
    range: 128 rows of 132 fp32.)"""
    part = 128 * 132 * 4
    small = moe.attn_paged_workspace_bytes(config(max_blocks=1))
    assert small < 4 << 20
    # 64 tokens of 6 heads a key/value head: at most 384 / 64 + 4 blocks of each of 8 heads
    for blocks in (2, 3, 5):
        more = moe.attn_paged_workspace_bytes(config(max_blocks=blocks)) - small
        assert 0 < more <= 8 * 10 * blocks * part + (4 << 20)
    assert moe.attn_paged_workspace_bytes(config(max_tokens=32768, max_blocks=4096)) < 200 << 20
