"""Single tokens whose positions many workgroups share: rows with more partial sums than one pass of
the merge takes."""
import numpy as np
import pytest

import paged_ref as ref
from test_gpu_paged import Case, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("shape", [(2, 1, 64), (6, 1, 128)], ids=lambda s: "%d-%d-%d" % s)
@pytest.mark.parametrize("context", [12000, 33000, 65535])
def test_many_partial_sums(torch, shape, context, e4m3):
    """One key/value head: some 94, 258 and 512 partial sums a row, all of them with weight; the
    queries are small, so that every position counts alike, or their largest score is at one of
    the last positions (past 256 partial sums)."""
    H, G, hd = shape
    c = Case(torch, H, G, hd, 256, e4m3, [(context, 1)], seed=context)
    c.fill_context(new_too=True)
    c.set_batch()
    K = c.cache.views(0)[0]
    for peak in (None, 0, context * 3 // 4, context - 5):
        q = c.queries(sigma=0.05)
        if peak is not None:                               # along that position's key
            key = f64(K[int(c.table[0, peak // 256]), 0, peak % 256])
            if e4m3:
                key = key * 2.0 ** float(c.pool.ks[int(c.table[0, peak // 256]), 0])
            q = torch.from_numpy(np.tile(key, H)[None]).to(torch.bfloat16).cuda()
        out = torch.full_like(q, 7.0)
        c.cache.attend(0, q, out)
        first = out.clone()
        c.cache.attend(0, q, out)
        torch.cuda.synchronize()
        assert torch.equal(first.view(torch.int16), out.view(torch.int16))
        c.check_attend(q, out)
        # a share left out or counted twice moves a mean of equal weights by its part of the
        # positions: more than the bound where the mean is small beside the values
        o, wv, ew = ref.attend(f64(q).reshape(1, H, hd), c.pool, context, c.table[0])
        assert (ref.attend_bound(o, wv, ew, context + 1, one_term=False) < 0.05 * wv).all()
