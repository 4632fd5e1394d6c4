"""The weights of the paged attention keep 16 bits on their way into the matrix products, whatever
the kind of share that a row is in."""
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
@pytest.mark.parametrize("lens", [[(300, 1), (20, 2)], [(7, 5), (61, 9), (130, 17)], [(300, 130)], [(0, 300)], [(3000, 9)],
                                  [(700, 1), (33, 70)], [(0, 130)] * 24], ids=str)
@pytest.mark.parametrize("shape", [(4, 2, 64), (6, 1, 128), (16, 1, 64), (48, 8, 128)], ids=lambda s: "%d-%d-%d" % s)
def test_weights_keep_sixteen_bits(torch, shape, lens, e4m3):
    """Where values cancel the output's own rounding is small, and weights of fewer bits show."""
    if shape[0] == 48 and len(lens) > 3:
        lens = lens[:3]
    c = Case(torch, *shape, 16, e4m3, lens, seed=61)
    c.fill_context(new_too=True)
    c.set_batch()
    q = c.queries()
    out = torch.empty_like(q)
    c.cache.attend(0, q, out)
    torch.cuda.synchronize()
    qh, oh = (f64(t).reshape(-1, c.H, c.hd) for t in (q, out))
    at = 0
    for s, (p0, n) in enumerate(c.lens):
        o, wv, ew = ref.attend(qh[at:at + n], c.pool, p0, c.table[s])
        err = np.abs(oh[at:at + n] - o)
        assert (err <= ref.attend_bound(o, wv, ew, p0 + n, one_term=False)).all(), (s, p0, n)
        at += n
