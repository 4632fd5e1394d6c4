"""Infinities in the keys of bf16 pages: they act through the scores, and a value that is not finite
spoils its dimension for every row that sees it, whatever its position's weight."""
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


def plain(q, K, V, pos0):
    """fp64 (q [n, hd] of one head, K and V [L, hd]) -> o [n, hd], NaN where it is not finite."""
    n, hd = q.shape
    o = np.zeros((n, hd))
    with np.errstate(invalid="ignore"):
        s = np.array([[np.sum(qr * kr) for kr in K] for qr in q]) / np.sqrt(hd)
    for i in range(n):
        si, Vi = s[i, :pos0 + i + 1], V[:pos0 + i + 1]
        bad = ~np.isfinite(Vi).all(0)
        if np.isnan(si).any() or (si == np.inf).any():
            o[i] = np.nan
            continue
        if (si > -np.inf).any():
            w = np.exp(si - si.max())
            o[i] = (w / w.sum()) @ np.where(np.isfinite(Vi), Vi, 0.0)
        o[i, bad] = np.nan
    return o


@pytest.mark.parametrize("lens,positions", [([(0, 1)], [0]), ([(0, 3)], [0, 2]), ([(20, 2)], [5]), ([(20, 2)], [20, 21]),
                                            ([(300, 1)], [10, 290]), ([(300, 1)], [300]), ([(1200, 1)], [3, 700, 1199]),
                                            ([(70, 40)], [6, 80, 100]), ([(0, 130)], [0, 64, 129]), ([(900, 9)], [4, 905])], ids=str)
@pytest.mark.parametrize("value_too", [False, True], ids=["key", "key-and-value"])
@pytest.mark.parametrize("shape", [(4, 2, 64), (6, 1, 128)], ids=lambda s: "%d-%d-%d" % s)
def test_infinite_keys(torch, shape, value_too, lens, positions):
    """Key/value head 0 holds an infinity at the positions, so that the scores there are +inf for
    queries of one sign and -inf for the other; dim 7 of the values there is infinite too."""
    H, G, hd = shape
    c = Case(torch, H, G, hd, 16, False, lens, seed=71)
    c.fill_context(new_too=True)
    c.set_batch()
    (p0, n), = lens
    K, V, _, _ = c.cache.views(0)
    for p in positions:
        pg, slot = int(c.table[0, p // 16]), p % 16
        K[pg, 0, slot, 3] = float("inf")
        if value_too:
            V[pg, 0, slot, 7] = float("-inf")
    q = c.queries()
    qh = q.view(-1, H, hd)
    # head 0 sees no score of +inf; head 1 none in its first tokens
    qh[:, 0, 3] = -qh[:, 0, 3].abs()
    if H // G > 1:
        qh[:n // 2 + 1, 1, 3] = -qh[:n // 2 + 1, 1, 3].abs()
    out = torch.full_like(q, 7.0)
    c.cache.attend(0, q, out)
    torch.cuda.synchronize()
    blocks = [int(t) for t in c.table[0] if t >= 0]
    got, qs = f64(out).reshape(n, H, hd), f64(q).reshape(n, H, hd)
    kept = 0
    for j in range(H):
        Kj, Vj = (np.concatenate([f64(t[b, j // (H // G)]) for b in blocks])[:p0 + n] for t in (K, V))
        want = plain(qs[:, j], Kj, Vj, p0)
        ok = np.isfinite(want)
        assert np.array_equal(np.isfinite(got[:, j]), ok), j
        # the scores' and weights' errors stay far below this at scores of some ten
        scale = np.abs(np.where(np.isfinite(Vj), Vj, 0.0)).max()
        assert (np.abs(got[:, j] - want)[ok] <= ref.BF16 * np.abs(want[ok]) + 1e-3 * scale).all(), j
        kept += ok[:, 0].all() if j == 0 else 0
    assert kept == 1                                       # (head 0 has no +inf: rows that stay finite)
