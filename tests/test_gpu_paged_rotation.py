"""The rotation of the paged cache's append against angles of more than fp64."""
import numpy as np
import pytest

import paged_ref as ref
import paper_2506_23635_amd as moe

pytestmark = pytest.mark.gpu

THETA = 5e5


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def angles(pos, hd):
    """pos theta^(-2i/hd) with 64 bits of mantissa (their error is below 2^-36 at any position)."""
    wide = np.longdouble
    assert np.finfo(wide).nmant >= 63
    i = np.arange(hd // 2).astype(wide)
    return np.asarray(pos).astype(wide)[:, None] * wide(THETA) ** (-2 * i / hd)


def positions_near_zeros(hd, lo, hi, n):
    """Positions of lo .. hi - 1 at which some cosine or sine comes nearest to zero."""
    pos = np.arange(lo, hi)
    a = angles(pos, hd)
    near = np.minimum(np.abs(np.cos(a)), np.abs(np.sin(a)))
    near[pos == 0] = 1
    return pos[np.argsort(near.min(1))[:n]]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lo,hi", [(1, 4096), (87000, 91000), ((1 << 20) - 4096, 1 << 20), ((1 << 24) - 8192, 1 << 24)], ids=str)
def test_cosines_and_sines(torch, hd, lo, hi):
    """Of pairs (1, 0) and (0, 1) the rotation returns cos and sin themselves, rounded to bf16: off
    by 2^-23 beside that rounding, and by the angle's error (its factor and the product rounded to
    fp64: 2^-52 + 2^-53 of it)."""
    P, blocks, n = 256, 65536, 16
    pos = np.concatenate([positions_near_zeros(hd, lo, hi, n - 2), [lo, hi - 1]])
    cache = moe.PagedCache(moe.make_paged_config(2, 1, hd, page_size=P, n_pages=n, max_seqs=n, max_tokens=n, max_blocks=blocks,
                                                 rope_theta=THETA))
    table = np.full((n, blocks), -1, np.int32)
    table[np.arange(n), pos // P] = np.arange(n)
    cache.set_batch([1] * n, pos, table)
    x = torch.zeros((n, 4, hd), device="cuda")
    x[:, 0, :hd // 2] = 1                                  # query head 0 and the key head: (1, 0)
    x[:, 1, hd // 2:] = 1                                  # query head 1: (0, 1)
    x[:, 2] = x[:, 0]
    q = torch.empty((n, 2 * hd), dtype=torch.bfloat16, device="cuda")
    cache.append(0, x.view(n, -1), q)
    torch.cuda.synchronize()
    K = cache.views(0)[0].float().cpu().numpy()
    got = q.float().cpu().numpy().reshape(n, 2, 2, hd // 2).astype(np.float64)
    keys = np.stack([K[s, 0, p % P] for s, p in enumerate(pos)]).reshape(n, 2, hd // 2)
    a = angles(pos, hd)
    c, s = np.cos(a).astype(np.float64), np.sin(a).astype(np.float64)
    off = 2.0 ** -23 + np.abs(a).astype(np.float64) * (2.0 ** -52 + 2.0 ** -53)
    for have, want in ((got[:, 0, 0], c), (got[:, 0, 1], s), (got[:, 1, 0], -s), (got[:, 1, 1], c), (keys[:, 0], c), (keys[:, 1], s)):
        bound = ref.BF16 * np.abs(want) + (1 + ref.BF16) * off
        assert (np.abs(have - want) <= bound).all(), (np.abs(have - want) / bound).max()
