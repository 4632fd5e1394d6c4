"""Attention over the paged cache where scores are large: the weights are those of the scores'
differences, however large the scores themselves."""
import numpy as np
import pytest

import paged_ref as ref
from test_gpu_paged import Case, f64

pytestmark = pytest.mark.gpu

SHAPES = [(4, 2, 64), (6, 1, 128), (16, 1, 64)]
# single tokens, whole and divided; rows in blocks of 64 and of 128, whole and divided; mixed
LENS = {"single": [(0, 1), (40, 1)], "few": [(700, 1), (5, 1)], "divided": [(5000, 1)], "rows": [(70, 40)], "prompt": [(0, 130)],
        "piece": [(3000, 9)], "mixed": [(900, 1), (33, 70)]}


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def write_context(c, keys, values):
    """A key row for every position of a sequence, the same for all heads, and values."""
    for s, (p0, n) in enumerate(c.lens):
        k = np.broadcast_to(keys(s, p0 + n)[:, None], (p0 + n, c.G, c.hd))
        c.pool.append(k, values(s, p0 + n), 0, c.table[s])
    torch = c.torch
    K, V, ks, vs = c.cache.views(0)
    for t, scale, val, code, exp in ((K, ks, c.pool.k, c.pool.kc, c.pool.ks), (V, vs, c.pool.v, c.pool.vc, c.pool.vs)):
        if c.e4m3:
            t.view(torch.uint8).copy_(torch.from_numpy(code))
            scale.copy_(torch.from_numpy(2.0 ** exp.astype(np.float64)).float())
        else:
            t.copy_(torch.from_numpy(val).to(torch.bfloat16))


def attend_twice(c, q):
    out = c.torch.full_like(q, 7.0)
    c.cache.attend(0, q, out)
    first = out.clone()
    c.cache.attend(0, q, out)
    c.torch.cuda.synchronize()
    assert c.torch.equal(first.view(c.torch.int16), out.view(c.torch.int16))
    return f64(out).reshape(-1, c.H, c.hd)


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "%d-%d-%d" % s)
def test_differences_of_large_scores(torch, shape, lens, e4m3):
    """Scores s 2^B + j 2^(B - 23), j = 0 .. 7, s 1 or 0 by position, B and the sign of 2^B by row:
    exact in fp32, so that the weights are those of fp64 but for the exponential's own rounding.  Of
    rows in one wave some have maxima that fp32's product with 1/sqrt(head_dim) holds closely, and
    some (B up to 100) maxima whose product is off by more than all of fp32's range."""
    H, G, hd = shape
    powers = [0, 20, 24, 26, 27, 28, 29, 31, 33, 36, 40, 60, 100]
    a = 8 if e4m3 else 4                                   # the keys' large dim is 2^a
    for thirds in ((1, 0, 1), (0, 1, 0), (1, 1, 1)):       # s by third of the positions
        c = Case(torch, H, G, hd, 16, e4m3, LENS[lens], seed=23)
        rng = np.random.default_rng(sum(thirds))

        def keys(s, L):
            k = np.zeros((L, hd))
            k[:, 0] = np.repeat(thirds, -(-L // 3))[:L] * 2.0 ** a
            k[:, 1] = rng.integers(0, 8, L) * 2.0 ** (a - 4)
            return k

        write_context(c, keys, lambda s, L: ref.bf16_round(rng.standard_normal((L, G, hd))))
        B = rng.choice(powers, (c.T, H)).astype(np.float64)
        q = np.zeros((c.T, H, hd))
        q[..., 0] = rng.choice([-1.0, 1.0], (c.T, H)) * 2.0 ** (B - a)
        q[..., 1] = 2.0 ** (B - 23 - a + 4)
        assert np.array_equal(ref.bf16_round(q), q)
        c.set_batch()
        got = attend_twice(c, torch.from_numpy(q.reshape(c.T, -1)).to(torch.bfloat16).cuda())
        at = 0
        for s, (p0, n) in enumerate(c.lens):
            o, wv, _ = ref.attend(q[at:at + n], c.pool, p0, c.table[s])
            # an exponent of up to 2^-110 (less weighs nothing): the difference of the scores, the
            # factor 1/sqrt(head_dim) log2 e and the product with it are rounded once each, and the
            # exponential 2 ulp; the weight and the sum that divides it carry it
            ew = 2 * (3 * 110 + 2) * ref.U32
            bound = ref.attend_bound(o, wv, ew, p0 + n, one_term=False)
            err = np.abs(got[at:at + n] - o)
            assert np.isfinite(got[at:at + n]).all() and (err <= bound).all(), (thirds, s, np.nanmax(err / bound))
            at += n


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("shape", SHAPES[:2], ids=lambda s: "%d-%d-%d" % s)
@pytest.mark.parametrize("sigma", [13, 15, 16, 20, 50])
def test_the_largest_of_large_scores_alone_counts(torch, sigma, shape, lens, e4m3):
    """Queries and keys of standard deviation 2^sigma: the largest score of a row is alone, and the
    output that position's value, exactly (rows whose two largest are nearer to each other than 150
    in the exponent beside the scores' own fp32 error are left out: few)."""
    H, G, hd = shape
    c = Case(torch, H, G, hd, 16, e4m3, LENS[lens], seed=sigma)
    c.fill_context(sigma=2.0 ** sigma, new_too=True)
    c.set_batch()
    q = c.queries(sigma=2.0 ** sigma)
    got, qh = attend_twice(c, q), f64(q).reshape(-1, H, hd)
    at = left_out = 0
    for s, (p0, n) in enumerate(c.lens):
        blocks = [int(t) for t in c.table[s] if t >= 0]
        for g in range(G):
            K, V = (np.concatenate([c.pool.value(w, t, g) for t in blocks])[:p0 + n] for w in (0, 1))
            for j in range(g * (H // G), (g + 1) * (H // G)):
                score, mag = qh[at:at + n, j] @ K.T, np.abs(qh[at:at + n, j]) @ np.abs(K).T
                for i in range(n):
                    sc = score[i, :p0 + i + 1]
                    top = int(sc.argmax())
                    rest = np.delete(sc, top).max(initial=-np.inf)
                    if sc[top] - rest <= 150 * np.sqrt(hd) + 2 * hd * ref.U32 * mag[i, :p0 + i + 1].max():
                        left_out += 1
                        continue
                    assert np.array_equal(got[at + i, j], V[top]), (s, i, j)
        at += n
    assert left_out <= 0.02 * c.T * H + 1


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("shape", SHAPES[:2], ids=lambda s: "%d-%d-%d" % s)
def test_equal_large_scores_weigh_the_same(torch, shape, lens, e4m3):
    """All keys of a sequence alike: the mean of the values that a row sees."""
    H, G, hd = shape
    c = Case(torch, H, G, hd, 16, e4m3, LENS[lens], seed=29)
    row = ref.bf16_round(c.rng.standard_normal(hd) * 2.0 ** 17)
    write_context(c, lambda s, L: np.broadcast_to(row, (L, hd)), lambda s, L: c.rng.standard_normal((L, G, hd)))
    c.set_batch()
    q = c.queries(sigma=2.0 ** 17)
    got = attend_twice(c, q)
    at = 0
    for s, (p0, n) in enumerate(c.lens):
        o, wv, _ = ref.attend(np.zeros((n, H, hd)), c.pool, p0, c.table[s])
        bound = ref.attend_bound(o, wv, 8 * ref.U32, p0 + n, one_term=False)
        assert (np.abs(got[at:at + n] - o) <= bound).all()
        at += n
