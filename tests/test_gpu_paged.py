"""GPU parity of the paged cache (include/attn.h) against plain fp64 (paged_ref.py): appending with
the rotation, attention over pages of bf16 and of e4m3 with scales, both together, and the
attention block on top of them."""
import numpy as np
import pytest

import moe_inputs as mi
import oracle
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


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Case:
    """A PagedCache on shuffled pages and the same pool in fp64."""

    def __init__(self, torch, H, G, hd, P, e4m3, lens, seed=0, n_layers=1, spare=2, max_tokens=None, extra=0):
        self.torch, self.rng = torch, np.random.default_rng(seed)
        self.H, self.G, self.hd, self.P, self.e4m3, self.lens = H, G, hd, P, e4m3, list(lens)
        need = [(p + n + extra + P - 1) // P for p, n in lens]
        n_pages = sum(need) + spare
        ids = self.rng.permutation(n_pages)
        self.blocks = max(need + [1])
        self.table = np.full((len(lens), self.blocks), -1, np.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = ids[at:at + n]
            at += n
        self.spare_pages = ids[at:]
        self.T = sum(n for _, n in lens)
        cfg = moe.make_paged_config(H, G, hd, page_size=P, n_pages=n_pages, n_layers=n_layers, max_seqs=max(len(lens), 1),
                                    max_tokens=max_tokens or max(self.T, 1), max_blocks=self.blocks, rope_theta=THETA,
                                    flags=moe.ATTN_PAGED_E4M3 if e4m3 else 0)
        self.cfg = cfg
        self.cache = moe.PagedCache(cfg)
        self.cache.cache.fill_(0xFF)     # NaN, as bf16, as a code and as a scale, wherever nothing is written
        self.pool = ref.Pool(n_pages, G, P, hd, e4m3)

    def set_batch(self):
        self.cache.set_batch([n for _, n in self.lens], [p for p, _ in self.lens], self.table)

    def fill_context(self, sigma=1.5, layer=0, new_too=False):
        """Positions before the new tokens (new_too: theirs too), written from the host."""
        torch = self.torch
        for s, (p0, n) in enumerate(self.lens):
            L = p0 + (n if new_too else 0)
            if not L:
                continue
            k, v = (self.rng.standard_normal((L, self.G, self.hd)) * sigma for _ in range(2))
            self.pool.append(k.astype(np.float32).astype(np.float64), v.astype(np.float32).astype(np.float64), 0, self.table[s])
        K, V, ks, vs = self.cache.views(layer)
        for dst, scale, val, code, exp in ((K, ks, self.pool.k, self.pool.kc, self.pool.ks),
                                           (V, vs, self.pool.v, self.pool.vc, self.pool.vs)):
            for s, (p0, n) in enumerate(self.lens):
                L = p0 + (n if new_too else 0)
                for b in range((L + self.P - 1) // self.P):
                    m, pg = min(self.P, L - b * self.P), int(self.table[s, b])
                    if self.e4m3:
                        dst.view(torch.uint8)[pg, :, :m] = torch.from_numpy(code[pg, :, :m]).to(dst.device)
                        scale[pg] = torch.from_numpy(2.0 ** exp[pg].astype(np.float64)).float().to(dst.device)
                    else:
                        dst[pg, :, :m] = torch.from_numpy(val[pg, :, :m]).to(torch.bfloat16).to(dst.device)
        torch.cuda.synchronize()

    def queries(self, sigma=1.5):
        q = self.torch.from_numpy(self.rng.standard_normal((self.T, self.H * self.hd)) * sigma).to(self.torch.bfloat16)
        return q.cuda()

    def check_attend(self, q, out):
        at, group = 0, self.H // self.G
        qh, oh = f64(q).reshape(-1, self.H, self.hd), f64(out).reshape(-1, self.H, self.hd)
        for s, (p0, n) in enumerate(self.lens):
            if n:
                o, wv, ew = ref.attend(qh[at:at + n], self.pool, p0, self.table[s])
                bound = ref.attend_bound(o, wv, ew, p0 + n, one_term=n * group > 16)
                err = np.abs(oh[at:at + n] - o)
                assert np.isfinite(oh[at:at + n]).all(), (s, p0, n)
                assert (err <= bound).all(), (s, p0, n, (err / bound).max(), np.unravel_index((err / bound).argmax(), err.shape))
            at += n


SHAPES = [(4, 2, 64), (6, 1, 128), (8, 8, 128), (16, 1, 64), (48, 8, 128)]
LENS = {
    "single": [(0, 1)],
    "edges": [(15, 1), (16, 1), (17, 1), (31, 1), (32, 1), (63, 1), (64, 1), (127, 1), (128, 1), (129, 1), (255, 1), (256, 1)],
    "none": [(5, 0), (40, 1), (0, 0), (300, 1), (0, 1)],
    "few": [(3, 2), (0, 2), (62, 2), (130, 1)],
    "long": [(5000, 1), (1, 1), (2300, 1)],
    "rows": [(0, 3), (7, 5), (61, 9), (130, 17), (0, 33)],
    "prompt": [(0, 100), (77, 64), (300, 130)],
    "mixed": [(700, 1), (33, 70), (0, 0), (129, 2), (64, 16)],
}


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("shape,P", [(s, P) for s in SHAPES for P in (16, 64, 256) if s != SHAPES[-1] or P == 64],
                         ids=lambda v: "%d-%d-%d" % v if isinstance(v, tuple) else "page%d" % v)
def test_attend(torch, shape, P, lens, e4m3):
    c = Case(torch, *shape, P, e4m3, LENS[lens], seed=P + len(lens))
    c.fill_context(new_too=True)
    c.set_batch()
    q = c.queries()
    out = torch.full((c.T + 3, shape[0] * shape[2]), 7.0, dtype=torch.bfloat16, device="cuda")
    c.cache.attend(0, q, out)
    first = out.clone()
    c.cache.attend(0, q, out)
    torch.cuda.synchronize()
    assert torch.equal(first.view(torch.int16), out.view(torch.int16))       # the same bits again
    assert (out[c.T:] == 7.0).all()                                          # rows behind the last stay
    c.check_attend(q, out[:c.T])


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lens", [[(2000, 300)], [(0, 130)] * 24, [(0, 1200)], [(3000, 8)]],
                         ids=["piece", "prompts", "prompt", "few-tokens"])
@pytest.mark.parametrize("shape", [(4, 2, 64), (6, 1, 128), (16, 1, 64)], ids=lambda s: "%d-%d-%d" % s)
def test_attend_many_rows(torch, shape, lens, e4m3):
    """Enough rows, or positions, that both kinds of row blocks appear, whole and divided."""
    c = Case(torch, *shape, 64, e4m3, lens, seed=17)
    c.fill_context(new_too=True)
    c.set_batch()
    q = c.queries()
    out = torch.full_like(q, 7.0)
    c.cache.attend(0, q, out)
    first = out.clone()
    c.cache.attend(0, q, out)
    torch.cuda.synchronize()
    assert torch.equal(first.view(torch.int16), out.view(torch.int16))
    c.check_attend(q, out)


def check_append(c, qkv, q, before, layer=0):
    """Queries, pages and scales after an append; `before`: the pages' bytes before it."""
    torch = c.torch
    H, G, hd, P = c.H, c.G, c.hd, c.P
    x = f64(qkv).reshape(-1, H + 2 * G, hd)
    pos = np.concatenate([np.arange(p, p + n) for p, n in c.lens] + [np.zeros(0, int)])
    turned, err = ref.rotate(x[:, :H + G], pos, THETA), ref.rotation_error(x[:, :H + G])
    qh = f64(q).reshape(-1, H, hd)
    assert (np.abs(qh - turned[:, :H]) <= ref.BF16 * np.abs(turned[:, :H]) + (1 + ref.BF16) * err[:, :H] + 1e-37).all()
    K, V, ks, vs = c.cache.views(layer)
    at = 0
    for s, (p0, n) in enumerate(c.lens):
        c.pool.append(turned[at:at + n, H:], x[at:at + n, H + G:], p0, c.table[s])
        at += n
    touched = np.zeros((c.cfg.n_pages, P), bool)
    earlier = np.zeros_like(touched)
    for s, (p0, n) in enumerate(c.lens):
        for p in range(p0, p0 + n):
            touched[c.table[s, p // P], p % P] = True
        for p in range(p0):
            if n and c.table[s, p // P] == c.table[s, p0 // P]:
                earlier[c.table[s, p // P], p % P] = True
    new = np.broadcast_to(touched[:, None, :, None], c.pool.k.shape)
    old = np.broadcast_to(earlier[:, None, :, None], c.pool.k.shape)
    errk = np.zeros(c.pool.k.shape)
    at = 0
    for s, (p0, n) in enumerate(c.lens):
        for i in range(n):
            errk[c.table[s, (p0 + i) // P], :, (p0 + i) % P] = err[at + i, H:]
        at += n
    if not c.e4m3:
        k, v = f64(K), f64(V)
        assert (np.abs(k - c.pool.k)[new] <= (ref.BF16 * np.abs(c.pool.k) * 2 + (1 + ref.BF16) * errk)[new] + 1e-37).all()
        assert np.array_equal(v[new], c.pool.v[new])                         # one rounding of fp32: exact
    else:
        live = touched.any(1)
        assert np.array_equal(np.log2(ks.cpu().numpy()[live]), c.pool.ks[live])
        assert np.array_equal(np.log2(vs.cpu().numpy()[live]), c.pool.vs[live])
        kc, vc = K.view(torch.uint8).cpu().numpy(), V.view(torch.uint8).cpu().numpy()
        assert np.array_equal(vc[new], c.pool.vc[new])
        both = new | (old & live[:, None, None, None])
        assert np.array_equal(kc[old & live[:, None, None, None]], c.pool.kc[old & live[:, None, None, None]])
        assert np.array_equal(vc[both], c.pool.vc[both])
        # keys: the nearest code of a value that is off by the fp32 rotation at most
        scale = 2.0 ** c.pool.ks[:, :, None, None].astype(np.float64)
        got, want = ref.E4M3[kc] * scale, ref.E4M3[c.pool.kc] * scale
        step = np.maximum(np.abs(want), 2.0 ** -6 * scale) * 2.0 ** -3
        near = np.abs(got - want) <= step * (1 + 1e-12)
        assert near[new].all() and (got[new] != want[new]).mean() <= 1e-3
    # nothing else changed
    now = c.cache.views(layer)[:2]
    keep = ~(new | (old if c.e4m3 else np.zeros_like(old)))
    for a, b in zip(now, before):
        w = torch.uint8 if c.e4m3 else torch.int16
        assert np.array_equal(a.view(w).cpu().numpy()[keep], b.view(w).cpu().numpy()[keep])


def rows_of(c, dtype, sigma=1.0, pad=0):
    n = (c.H + 2 * c.G) * c.hd
    spread = np.repeat(2.0 ** c.rng.uniform(-6, 6, c.H + 2 * c.G), c.hd)
    x = c.torch.from_numpy(c.rng.standard_normal((c.T, n)) * spread * sigma).to(dtype)
    full = c.torch.full((c.T, n + pad), float("nan"), dtype=dtype)
    full[:, :n] = x
    return full.cuda()[:, :n]


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("P", [16, 64, 256])
@pytest.mark.parametrize("shape", SHAPES[:4], ids=lambda s: "%d-%d-%d" % s)
def test_append(torch, shape, P, lens, e4m3, src):
    c = Case(torch, *shape, P, e4m3, LENS[lens], seed=3 * P + len(lens))
    c.fill_context(sigma=0.3)
    c.set_batch()
    qkv = rows_of(c, torch.float32 if src == "f32" else torch.bfloat16, pad=8 * (P // 16))
    before = [t.clone() for t in c.cache.views(0)[:2]]
    q = torch.full((c.T + 2, shape[0] * shape[2]), 7.0, dtype=torch.bfloat16, device="cuda")
    c.cache.append(0, qkv, q)
    torch.cuda.synchronize()
    assert (q[c.T:] == 7.0).all()
    check_append(c, qkv, q[:c.T], before)
    # once more: the same pages, and the same result
    again = [t.clone() for t in c.cache.views(0) if t is not None]
    c.cache.append(0, qkv, q)
    torch.cuda.synchronize()
    for a, b in zip(again, [t for t in c.cache.views(0) if t is not None]):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_append_the_shape_of_the_model(torch):
    for e4m3 in (False, True):
        c = Case(torch, 48, 8, 128, 64, e4m3, [(130, 1), (0, 90), (63, 3)], seed=9)
        c.fill_context(sigma=0.3)
        c.set_batch()
        qkv = rows_of(c, torch.float32)
        before = [t.clone() for t in c.cache.views(0)[:2]]
        q = torch.empty((c.T, 48 * 128), dtype=torch.bfloat16, device="cuda")
        c.cache.append(0, qkv, q)
        torch.cuda.synchronize()
        check_append(c, qkv, q, before)


# ------------------------------------------------------------- e4m3 values --

def test_every_code_is_read_exactly(torch):
    """One position a sequence: its weight is 1 and the output its value, code * scale, exactly
    (under 2^120, which append never sets, the codes whose values no bf16 holds are not finite)."""
    hd, P, exps = 128, 16, [-100, -60, -9, -1, 0, 3, 50, 119, 120]
    codes = np.array([c for c in range(256) if c & 0x7F != 0x7F])
    per = 2 * len(exps)                       # 254 codes in two rows of 127
    c = Case(torch, 2, 1, hd, P, True, [(0, 1)] * per, seed=1)
    K, V, ks, vs = c.cache.views(0)
    want = np.zeros((per, hd))
    for s in range(per):
        row = np.zeros(hd, np.uint8)
        row[:127] = codes[s % 2 * 127:s % 2 * 127 + 127]
        pg, e = int(c.table[s, 0]), exps[s // 2]
        V.view(torch.uint8)[pg, 0, 0] = torch.from_numpy(row).cuda()
        K.view(torch.uint8)[pg, 0, 0] = 0
        vs[pg, 0], ks[pg, 0] = 2.0 ** e, 1.0
        want[s] = ref.E4M3[row] * 2.0 ** e
    c.set_batch()
    q = c.queries()
    out = torch.empty_like(q)
    c.cache.attend(0, q, out)
    torch.cuda.synchronize()
    got = f64(out).reshape(per, 2, hd)
    is_bf16 = np.abs(want) < 2.0 ** 128                   # 2^128 - 2^120 is the largest
    for j in (0, 1):
        assert np.array_equal(got[:, j][is_bf16], want[is_bf16]) and not np.isfinite(got[:, j][~is_bf16]).any()
    assert (~is_bf16).any()


def test_every_rounding_to_a_code(torch):
    """Values at, half way between and next to half way between all codes, under several scales
    (a row's 448 * 2^e sets its page's)."""
    hd, P, exps = 128, 16, [-100, -30, 0, 7, 111]
    pos = ref.E4M3[:127]
    mid = (pos[:-1] + pos[1:]) / 2
    grid = np.concatenate([pos, mid, np.nextafter(mid.astype(np.float32), np.float32(0)).astype(np.float64),
                           np.nextafter(mid.astype(np.float32), np.float32(1e9)).astype(np.float64)])
    grid = np.concatenate([grid, -grid])
    rows = np.zeros((-(-grid.size // (hd - 1)), hd))
    rows[:, 0] = 448.0
    rows[:, 1:].flat[:grid.size] = grid
    n = rows.shape[0]
    c = Case(torch, 1, 1, hd, P, True, [(0, n)] * len(exps), seed=2)
    c.set_batch()
    qkv = np.zeros((c.T, 3, hd))
    for i, e in enumerate(exps):
        qkv[i * n:(i + 1) * n, 2] = rows * 2.0 ** e
    x = torch.from_numpy(qkv.reshape(c.T, 3 * hd)).float().cuda()
    assert np.array_equal(f64(x).reshape(qkv.shape), qkv)                    # all of them fp32 values
    c.cache.append(0, x, torch.empty((c.T, hd), dtype=torch.bfloat16, device="cuda"))
    torch.cuda.synchronize()
    _, V, _, vs = c.cache.views(0)
    V, vs = V.view(torch.uint8).cpu().numpy(), vs.cpu().numpy()
    for i, e in enumerate(exps):
        want = ref.e4m3_codes(rows)
        for t in range(n):
            pg = c.table[i, t // P]
            assert vs[pg, 0] == 2.0 ** e
            assert np.array_equal(ref.E4M3[V[pg, 0, t % P]], ref.E4M3[want[t]]), (e, t)


def test_values_that_are_not_finite_are_stored_as_nan_and_set_no_scale(torch):
    c = Case(torch, 2, 1, 64, 16, True, [(3, 4)], seed=3)
    c.fill_context(sigma=0.01)
    c.set_batch()
    x = torch.randn((4, 4 * 64), device="cuda")
    x[1, 3 * 64 + 5], x[2, 3 * 64 + 6], x[3, 3 * 64 + 7], x[0, 2 * 64 + 9] = float("inf"), float("-inf"), float("nan"), float("nan")
    c.cache.append(0, x, torch.empty((4, 128), dtype=torch.bfloat16, device="cuda"))
    torch.cuda.synchronize()
    K, V, ks, vs = (t.cpu() for t in c.cache.views(0))
    pg = int(c.table[0, 0])
    v = f64(V)[pg, 0, 3:7]
    bad = np.zeros_like(v, bool)
    bad[1, 5] = bad[2, 6] = bad[3, 7] = True
    assert np.array_equal(np.isnan(v), bad)
    xs = f64(x)[:, 3 * 64:]
    assert float(vs[pg, 0]) == 2.0 ** ref.scale_exponent(np.abs(xs[~bad]).max())
    k = f64(K)[pg, 0, 3:7]
    assert np.isnan(k[0, [9, 41]]).all() and np.isnan(k).sum() == 2          # the pair of the rotation
    assert np.isfinite(float(ks[pg, 0]))


def test_the_largest_values(torch):
    """Past 448 * 2^119 values are stored as that, which a bf16 still holds."""
    c = Case(torch, 1, 1, 64, 16, True, [(0, 3)], seed=8)
    c.set_batch()
    x = torch.zeros((3, 3 * 64), device="cuda")
    x[:, 2 * 64:2 * 64 + 4] = torch.tensor([3.4e38, -3.4e38, 448 * 2.0 ** 119, 2.0 ** 119], device="cuda")
    c.cache.append(0, x, torch.empty((3, 64), dtype=torch.bfloat16, device="cuda"))
    _, V, _, vs = c.cache.views(0)
    pg = int(c.table[0, 0])
    assert float(vs[pg, 0]) == 2.0 ** 119
    assert np.array_equal(f64(V)[pg, 0, :3, :4], np.tile([448.0, -448.0, 448.0, 1.0], (3, 1)))


def test_zeros_and_tiny_values(torch):
    c = Case(torch, 1, 1, 64, 16, True, [(0, 2), (0, 2)], seed=4)
    c.set_batch()
    x = torch.zeros((4, 3 * 64), device="cuda")
    x[2:, 64:] = 1e-40
    c.cache.append(0, x, torch.empty((4, 64), dtype=torch.bfloat16, device="cuda"))
    K, V, ks, vs = c.cache.views(0)
    for s in range(2):
        pg = int(c.table[s, 0])
        assert float(ks[pg, 0]) == float(vs[pg, 0]) == 2.0 ** -100
        assert (f64(K)[pg, 0, :2] == 0).all() and (f64(V)[pg, 0, :2] == 0).all()


# ---------------------------------------------------------------- masks --

HOLED = [(100, 1), (64, 70), (30, 3), (200, 17), (0, 1)]


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("P", [16, 32, 64])
@pytest.mark.parametrize("shape", [(4, 2, 64), (6, 1, 128)], ids=lambda s: "%d-%d-%d" % s)
def test_pages_that_are_missing(torch, shape, P, e4m3):
    """Positions without a page are left out (one sequence has none but its last page)."""
    c = Case(torch, *shape, P, e4m3, HOLED, seed=P)
    c.fill_context(new_too=True)
    rng = np.random.default_rng(P)
    table = c.table.copy()
    for s, (p0, n) in enumerate(HOLED):
        for b in range(p0 // P):
            if s == 0 or rng.random() < 0.5:
                table[s, b] = -1
    c.table = table
    c.set_batch()
    q = c.queries()
    out = torch.full_like(q, 7.0)
    c.cache.attend(0, q, out)
    torch.cuda.synchronize()
    c.check_attend(q, out)


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lens", [[(32, 1)], [(0, 2), (40, 1)], [(16, 40)], [(0, 130), (600, 1), (9, 9)]], ids=str)
@pytest.mark.parametrize("shape", [(4, 2, 64), (6, 1, 128)], ids=lambda s: "%d-%d-%d" % s)
def test_rows_that_see_nothing_are_zero(torch, shape, lens, e4m3):
    """Without any page, or without the first ones: rows before the first page are zeros, the others
    right.  Such a batch is for reading: append refuses it."""
    c = Case(torch, *shape, 16, e4m3, lens, seed=len(lens))
    c.fill_context(new_too=True)
    for keep in (0, 1):                                   # the last page of each sequence, or none
        table = np.full_like(c.table, -1)
        for s, (p0, n) in enumerate(lens):
            last = (p0 + n - 1) // 16
            if keep:
                table[s, last] = c.table[s, last]
        whole, c.table = c.table, table
        c.set_batch()
        q = c.queries()
        out = torch.full_like(q, 7.0)
        c.cache.attend(0, q, out)
        torch.cuda.synchronize()
        c.check_attend(q, out)
        if not keep:
            assert (out == 0).all()
        if not keep or any((p0 + n - 1) // 16 != p0 // 16 for p0, n in lens):
            before = c.cache.cache.clone()
            with pytest.raises(moe.MoeError) as e:
                c.cache.append(0, rows_of(c, torch.float32), q)
            assert e.value.status == -5
            assert torch.equal(before, c.cache.cache)
        c.table = whole


def test_a_replayed_append_leaves_out_tokens_without_a_page(torch):
    for e4m3 in (False, True):
        c = Case(torch, 4, 2, 64, 16, e4m3, [(20, 2), (5, 1)], seed=9)
        c.fill_context()
        c.set_batch()
        qkv = rows_of(c, torch.float32)
        q = torch.empty((c.T, 256), dtype=torch.bfloat16, device="cuda")
        c.cache.append(0, qkv, q)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.cache.append(0, qkv, q)
        table = c.table.copy()
        table[0] = -1
        c.cache.set_batch([2, 1], [20, 5], table)
        before = c.cache.cache.clone()
        pg = int(c.table[1, 0])
        for t in c.cache.views(0)[:2]:
            t.view(torch.uint8 if e4m3 else torch.int16)[pg, :, 5] = 0
        for _ in range(3):
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(before, c.cache.cache)     # sequence 1 is written as before, 0 is not


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lens", [[(20, 3)], [(20, 8)], [(70, 40)], [(0, 130)], [(90, 2), (10, 50)]], ids=str)
@pytest.mark.parametrize("shape", [(4, 2, 64), (6, 1, 128)], ids=lambda s: "%d-%d-%d" % s)
def test_a_value_that_is_not_finite_stays_with_the_rows_that_see_it(torch, shape, lens, e4m3):
    """NaN and infinities in some new tokens' values (one dim) and one key: rows before them are
    right, rows that see a value are not finite in its dim and right in the others, rows that see
    the key are not finite at all."""
    H, G, hd = shape
    c = Case(torch, H, G, hd, 16, e4m3, lens, seed=7)
    c.fill_context(new_too=True)
    c.set_batch()
    q = c.queries()
    K, V, _, _ = c.cache.views(0)
    clean = torch.empty_like(q)
    c.cache.attend(0, q, clean)
    bits = 0x7F if e4m3 else None
    where = {}                                            # sequence -> (position of the value, of the key)
    for s, (p0, n) in enumerate(lens):
        pv, pk = p0 + n // 2, p0 + n - 1
        where[s] = (pv, pk)
        for t, p, d in ((V, pv, 5), (K, pk, 3)):
            row = t[int(c.table[s, p // 16]), 0, p % 16]
            if e4m3:
                row.view(torch.uint8)[d] = bits
            else:
                row[d] = float("inf") if d == 5 else float("nan")
    out = torch.full_like(q, 7.0)
    c.cache.attend(0, q, out)
    torch.cuda.synchronize()
    a, b = f64(clean).reshape(-1, H, hd), f64(out).reshape(-1, H, hd)
    at = 0
    for s, (p0, n) in enumerate(lens):
        for i in range(n):
            for j in range(H):
                x, y = a[at + i, j], b[at + i, j]
                if j >= H // G:                           # another key/value head
                    assert np.array_equal(x, y)
                elif p0 + i >= where[s][1]:
                    assert not np.isfinite(y).any()
                elif p0 + i >= where[s][0]:
                    assert not np.isfinite(y[5]) and np.array_equal(np.delete(x, 5), np.delete(y, 5))
                else:
                    assert np.array_equal(x, y), (s, i, j)
        at += n


@pytest.mark.parametrize("bad", [float("nan"), float("inf")], ids=str)
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lens", [[(700, 1), (9, 1)], [(20, 6)], [(70, 40)], [(300, 1), (40, 40), (10, 8)]], ids=str)
def test_a_query_that_is_not_finite_spoils_its_own_row(torch, lens, e4m3, bad):
    c = Case(torch, 6, 1, 128, 16, e4m3, lens, seed=15)
    c.fill_context(new_too=True)
    c.set_batch()
    q = c.queries()
    clean, out = torch.empty_like(q), torch.empty_like(q)
    c.cache.attend(0, q, clean)
    at = 0
    for _, n in lens:                                     # head 2 of each sequence's last token
        at += n
        q[at - 1, 2 * 128 + 17] = bad
    c.cache.attend(0, q, out)
    torch.cuda.synchronize()
    a, b = f64(clean).reshape(-1, 6, 128), f64(out).reshape(-1, 6, 128)
    spoiled = np.zeros(a.shape[:2], bool)
    spoiled[np.cumsum([n for _, n in lens]) - 1, 2] = True
    assert np.isnan(b[spoiled]).all() and np.array_equal(a[~spoiled], b[~spoiled])


# ------------------------------------------------------------- together --

@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("shape,P", [((4, 2, 64), 16), ((6, 1, 128), 32), ((48, 8, 128), 64)], ids=str)
def test_prompts_then_generation(torch, shape, P, e4m3):
    """As a server runs them: prompts of several sequences, then single tokens of all of them,
    pieces and tokens mixed, a sequence that ends and another that takes its pages; append and
    attend on two layers, each step checked against the fp64 pages."""
    H, G, hd = shape
    steps = [[(0, 37), (0, 5), (0, 0)], [(37, 1), (5, 1), (0, 20)], [(38, 1), (6, 1), (20, 33)],
             [(39, 3), (7, 1), (53, 1)], [(42, 1), (0, 18), (54, 1)]]          # the last: sequence 1 anew
    c = Case(torch, H, G, hd, P, e4m3, [(42, 1), (0, 18), (54, 1)], seed=11, n_layers=2, max_tokens=64)
    pools = [ref.Pool(c.cfg.n_pages, G, P, hd, e4m3) for _ in range(2)]
    for lens in steps:
        c.lens, c.T = lens, sum(n for _, n in lens)
        c.set_batch()
        for layer in range(2):
            c.pool = pools[layer]
            qkv = rows_of(c, torch.float32)
            before = [t.clone() for t in c.cache.views(layer)[:2]]
            q = torch.empty((c.T, H * hd), dtype=torch.bfloat16, device="cuda")
            out = torch.empty_like(q)
            c.cache.append(layer, qkv, q)
            c.cache.attend(layer, q, out)
            torch.cuda.synchronize()
            check_append(c, qkv, q, before, layer)
            # the attention is held to the pages as they are (a key's code may be the other neighbour)
            K, V, ks, vs = c.cache.views(layer)
            if e4m3:
                c.pool.kc[:] = K.view(torch.uint8).cpu().numpy()
            else:
                c.pool.k[:] = np.where(np.isnan(f64(K)), c.pool.k, f64(K))
            c.check_attend(q, out)


def attn_block(torch, wl, max_tokens, heads=None):
    cfg = moe.make_attn_config(wl.d, wl.n_heads, wl.n_kv, wl.hd, n_layers=1, max_seq=wl.max_seq, max_tokens=max_tokens,
                               rope_theta=wl.theta, norm_eps=wl.eps)
    att = moe.AttnLayer(cfg)
    gamma, wqkv, wo = wl.gamma(), wl.wqkv(), wl.wo()
    att.load_layer(0, torch.from_numpy(gamma), torch.from_numpy(wqkv.view(np.int16)), torch.from_numpy(wo.view(np.int16)))
    return att, gamma, wqkv, wo


def block_on_codes(c, s, x, gamma, wqkv, wo, wl):
    """The fp64 block of sequence s (roundings as the block defines them) with its attention over
    the device's e4m3 pages, whose new entries are checked against the block's keys and values."""
    p0, n = c.lens[s]
    H, G, hd = wl.n_heads, wl.n_kv, wl.hd
    w64 = [mi.bf16_bits_to_f32(w).astype(np.float64) for w in (wqkv, wo)]
    h = ref.bf16_round((x - x.mean(1, keepdims=True)) / np.sqrt(x.var(1, keepdims=True) + wl.eps) * gamma)
    qkv = (h @ w64[0].reshape(wl.d, -1)).reshape(n, H + 2 * G, hd)
    pos = np.arange(p0, p0 + n)
    q = ref.bf16_round(ref.rotate(qkv[:, :H], pos, wl.theta))
    K, V, ks, vs = c.cache.views(0)
    pool = ref.Pool(c.cfg.n_pages, G, c.P, hd, True)
    pool.kc[:], pool.vc[:] = (t.view(c.torch.uint8).cpu().numpy() for t in (K, V))
    for dst, src in ((pool.ks, ks), (pool.vs, vs)):
        v = src.cpu().numpy()
        ok = np.isfinite(v) & (v > 0)
        dst[ok] = np.log2(v[ok])
    new = (ref.rotate(qkv[:, H:H + G], pos, wl.theta), qkv[:, H + G:])
    for i in range(n):
        pg, slot = c.table[s, (p0 + i) // c.P], (p0 + i) % c.P
        for which in (0, 1):
            for g in range(G):
                v, e = new[which][i, g], (pool.ks, pool.vs)[which][pg, g]
                step = np.maximum(np.abs(v), 2.0 ** (e - 6.0)) * 2.0 ** -3
                # (h may be its other neighbour in places: a relative 2^-8 of some terms)
                assert (np.abs(pool.value(which, pg, g)[slot] - v) <= step + 2e-2 * np.abs(v).max()).all()
    a = ref.bf16_round(ref.attend(q, pool, p0, c.table[s])[0]).reshape(n, H * hd)
    return x + a @ w64[1].reshape(H * hd, wl.d)


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lens", [[(29, 1)], [(29, 4)], [(0, 3), (17, 1), (40, 12)], [(0, 20), (31, 1)], [(5, 200), (64, 30)]], ids=str)
def test_the_block_on_pages(torch, lens, e4m3):
    """attn_forward_paged against the fp64 block of each sequence by itself, within the block's
    end-to-end bars; rows of other sequences never matter.  On e4m3 pages the block is put together
    from its parts, its attention over the pages as they are, and the pages hold the parts' keys
    and values within a code's step."""
    wl = mi.ATTN_WORKLOADS["attn_tiny"]
    T = sum(n for _, n in lens)
    c = Case(torch, wl.n_heads, wl.n_kv, wl.hd, 16, e4m3, lens, seed=5)
    cfg = moe.make_paged_config(wl.n_heads, wl.n_kv, wl.hd, page_size=16, n_pages=c.cfg.n_pages, max_seqs=len(lens),
                                max_tokens=T, max_blocks=c.blocks, rope_theta=wl.theta,
                                flags=moe.ATTN_PAGED_E4M3 if e4m3 else 0)
    c.cache = moe.PagedCache(cfg)
    c.fill_context(sigma=1.0)
    c.set_batch()
    att, gamma, wqkv, wo = attn_block(torch, wl, max(T, 16))
    x = torch.from_numpy(c.rng.standard_normal((T, wl.d))).to(torch.bfloat16).cuda()
    y, z = torch.empty_like(x), torch.empty_like(x)
    g2 = 1 + 0.1 * c.rng.standard_normal(wl.d).astype(np.float32)
    with pytest.raises(moe.MoeError):                     # no post norm loaded
        att.forward_paged(0, c.cache, x, y, z)
    att.forward_paged(0, c.cache, x, y)
    first = y.clone()
    att.load_post_norm(0, torch.from_numpy(g2))
    att.forward_paged(0, c.cache, x, y, z)
    torch.cuda.synchronize()
    assert torch.equal(first.view(torch.int16), y.view(torch.int16))
    at = 0
    for s, (p0, n) in enumerate(lens):
        kc, vc = np.zeros((wl.max_seq + 300, wl.n_kv, wl.hd), np.uint16), np.zeros((wl.max_seq + 300, wl.n_kv, wl.hd), np.uint16)
        for p in range(p0):
            for which, dst in ((0, kc), (1, vc)):
                v = np.stack([c.pool.value(which, c.table[s, p // 16], g)[p % 16] for g in range(wl.n_kv)])
                dst[p] = (v.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
        xs = x[at:at + n].cpu().view(torch.int16).numpy().view(np.uint16)
        if e4m3:
            want = block_on_codes(c, s, f64(x[at:at + n]), gamma, wqkv, wo, wl)
        else:
            want = oracle.attention_block(xs, gamma, wqkv, wo, kc, vc, p0, wl.n_heads, wl.n_kv, wl.eps, wl.theta)["y64"]
        got = f64(y[at:at + n])
        rel = np.linalg.norm(got - want) / np.linalg.norm(want)
        assert rel <= 2e-3 and np.abs(got - want).max() <= 1e-2 * max(1.0, np.abs(want).max()), (s, p0, n)
        at += n
    zr = f64(y)
    zr = (zr - zr.mean(1, keepdims=True)) / np.sqrt(zr.var(1, keepdims=True) + wl.eps) * g2
    assert (np.abs(f64(z) - zr) <= ref.BF16 * np.abs(zr) * 2 + 1e-5).all()


def test_a_sequence_alone_and_in_a_batch_give_the_same_block(torch):
    """One token each: the projections and the attention of a sequence do not see the others (the
    position ranges, and with them the last bits, may differ: the bf16 outputs by a step)."""
    wl = mi.ATTN_WORKLOADS["attn_tiny"]
    lens = [(20, 1), (3, 1), (47, 1)]
    c = Case(torch, wl.n_heads, wl.n_kv, wl.hd, 16, False, lens, seed=6)
    cfg = moe.make_paged_config(wl.n_heads, wl.n_kv, wl.hd, page_size=16, n_pages=c.cfg.n_pages, max_seqs=3, max_tokens=3,
                                max_blocks=c.blocks, rope_theta=wl.theta)
    c.cache = moe.PagedCache(cfg)
    c.fill_context()
    att, *_ = attn_block(torch, wl, 16)
    x = torch.randn((3, wl.d), device="cuda").to(torch.bfloat16)
    c.set_batch()
    y = torch.empty_like(x)
    att.forward_paged(0, c.cache, x, y)
    for s in range(3):
        c.cache.set_batch([1], [lens[s][0]], c.table[s:s + 1])
        ys = torch.empty_like(x[:1])
        att.forward_paged(0, c.cache, x[s:s + 1].contiguous(), ys)
        d = np.abs(f64(ys) - f64(y[s:s + 1]))
        assert (d <= 2 * ref.BF16 * np.abs(f64(ys)) + 1e-6).all()


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lens", [[(29, 1), (8, 2)], [(0, 20), (31, 1)]], ids=str)
def test_the_block_in_place_and_captured(torch, lens, e4m3):
    """y may be x; and the block replays on the batches of later steps."""
    wl = mi.ATTN_WORKLOADS["attn_tiny"]
    T, ends = sum(n for _, n in lens), [(p + 40, n) for p, n in lens]
    c = Case(torch, wl.n_heads, wl.n_kv, wl.hd, 16, e4m3, ends, seed=8)
    c.cache = moe.PagedCache(moe.make_paged_config(wl.n_heads, wl.n_kv, wl.hd, page_size=16, n_pages=c.cfg.n_pages,
                                                   max_seqs=2, max_tokens=T, max_blocks=c.blocks, rope_theta=wl.theta,
                                                   flags=moe.ATTN_PAGED_E4M3 if e4m3 else 0))
    c.fill_context(sigma=1.0)
    att, *_ = attn_block(torch, wl, 16 if T <= 16 else 32)
    new = [n for _, n in lens]
    start = c.cache.cache.clone()
    x = torch.from_numpy(c.rng.standard_normal((T, wl.d))).to(torch.bfloat16).cuda()
    buf, y = x.clone(), torch.empty_like(x)
    c.cache.set_batch(new, [p for p, _ in lens], c.table)
    att.forward_paged(0, c.cache, x, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        att.forward_paged(0, c.cache, buf, buf)
    for more in (0, 1, 17, 40, 3):
        c.cache.set_batch(new, [p + more for p, _ in lens], c.table)
        c.cache.cache.copy_(start)
        att.forward_paged(0, c.cache, x, y)
        want = c.cache.cache.clone()
        c.cache.cache.copy_(start)
        buf.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(buf.view(torch.int16), y.view(torch.int16)) and torch.equal(want, c.cache.cache), more


def test_the_block_refuses_a_batch_it_has_no_room_for(torch):
    wl = mi.ATTN_WORKLOADS["attn_tiny"]
    c = Case(torch, wl.n_heads, wl.n_kv, wl.hd, 16, False, [(0, 17)], seed=10)
    cache = moe.PagedCache(moe.make_paged_config(wl.n_heads, wl.n_kv, wl.hd, page_size=16, n_pages=c.cfg.n_pages,
                                                 max_tokens=32, max_blocks=c.blocks, rope_theta=wl.theta))
    att, *_ = attn_block(torch, wl, 16)
    x = torch.zeros((17, wl.d), dtype=torch.bfloat16, device="cuda")
    for new, table, status in ((17, c.table, -4), (16, np.full_like(c.table, -1), -5)):
        cache.set_batch([new], [0], table)
        with pytest.raises(moe.MoeError) as e:
            att.forward_paged(0, cache, x, torch.empty_like(x))
        assert e.value.status == status


def test_calls_with_the_wrong_tensors_are_refused(torch):
    c = Case(torch, 4, 2, 64, 16, False, [(3, 2)], seed=12)
    c.set_batch()
    q, out = (torch.zeros((2, 256), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    qkv = torch.zeros((2, 512), device="cuda")
    before = c.cache.cache.clone()
    for bad in (qkv.half(), qkv.cpu(), qkv[:1], qkv[:, :504], torch.zeros((2, 1024), device="cuda")[:, ::2],
                torch.zeros((2, 514), device="cuda")[:, :512], torch.zeros(1025, device="cuda")[1:].view(2, 512)):
        with pytest.raises(moe.MoeError):
            c.cache.append(0, bad, q)
    for bad in (q.float(), q.cpu(), q[:1], torch.zeros((256, 2), dtype=torch.bfloat16, device="cuda").t()):
        with pytest.raises(moe.MoeError):
            c.cache.append(0, qkv, bad)
        with pytest.raises(moe.MoeError):
            c.cache.attend(0, bad, out)
        with pytest.raises(moe.MoeError):
            c.cache.attend(0, q, bad)
    with pytest.raises(moe.MoeError):
        c.cache.attend(0, q, q)
    with pytest.raises(moe.MoeError):
        c.cache.set_batch([1], [0], torch.zeros((1, 1), dtype=torch.int32, device="cuda"))
    for n_new, pos0, table in (([1, 1], [0], [[0], [0]]), ([1], [0], [0]), ([[1]], [[0]], [[0]]), ([1], [0], [[0], [1]])):
        with pytest.raises(moe.MoeError):
            c.cache.set_batch(n_new, pos0, table)
    torch.cuda.synchronize()
    assert torch.equal(before, c.cache.cache)


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("n", [2, 40])
def test_the_last_positions(torch, n, e4m3):
    """The largest positions that a config allows, 2^24 - 256 on, in a sequence whose other pages
    are missing: the rotation by them, and attention over the last page alone."""
    H, G, hd, P, blocks = 4, 2, 64, 256, 65536
    p0 = blocks * P - P
    cache = moe.PagedCache(moe.make_paged_config(H, G, hd, page_size=P, n_pages=3, max_tokens=n, max_blocks=blocks,
                                                 rope_theta=THETA, flags=moe.ATTN_PAGED_E4M3 if e4m3 else 0))
    cache.cache.fill_(0xFF)
    table = np.full((1, blocks), -1, np.int32)
    table[0, -1] = 2
    cache.set_batch([n], [p0], table)
    c = Case(torch, H, G, hd, P, e4m3, [(0, n)], seed=14)
    c.cache, c.table, c.pool = cache, np.array([[2]], np.int32), ref.Pool(3, G, P, hd, e4m3)
    qkv = rows_of(c, torch.float32)
    q = torch.empty((n, H * hd), dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    cache.append(0, qkv, q)
    cache.attend(0, q, out)
    torch.cuda.synchronize()
    x = f64(qkv).reshape(n, H + 2 * G, hd)
    turned, err = ref.rotate(x[:, :H + G], p0 + np.arange(n), THETA), ref.rotation_error(x[:, :H + G])
    assert (np.abs(f64(q).reshape(n, H, hd) - turned[:, :H]) <= ref.BF16 * np.abs(turned[:, :H]) + (1 + ref.BF16) * err[:, :H] + 1e-37).all()
    c.pool.append(turned[:, H:], x[:, H + G:], 0, [2])
    K, V, ks, vs = cache.views(0)
    if e4m3:
        assert (K.view(torch.uint8)[2, :, :n].cpu().numpy() != c.pool.kc[2, :, :n]).mean() <= 1e-3
        c.pool.kc[2] = K.view(torch.uint8)[2].cpu().numpy()
    else:
        assert (np.abs(f64(K)[2, :, :n] - c.pool.k[2, :, :n]) <= (ref.BF16 * 2 * np.abs(c.pool.k[2, :, :n]) + (1 + ref.BF16) * err[:, H:].transpose(1, 0, 2) + 1e-37)).all()
        c.pool.k[2, :, :n] = f64(K)[2, :, :n]
    c.check_attend(q, out)


# ------------------------------------------------ graphs, streams, memory --

@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("new", [[1, 1, 1], [1, 40, 2]], ids=str)
def test_graph_replays_follow_the_batch(torch, new, e4m3):
    """append and attend captured once, replayed on the batches of five steps (longer contexts,
    more ranges, other pages), eager work in between: the eager results, bit for bit."""
    H, G, hd, P = 6, 1, 128, 16
    ctx = [[10, 3, 50], [300, 31, 900], [301, 0, 16], [2000, 700, 5], [5000, 64, 3000]]
    last = [(max(s[i] for s in ctx), new[i]) for i in range(3)]
    c = Case(torch, H, G, hd, P, e4m3, last, seed=13)
    c.fill_context()
    g = torch.Generator(device="cuda").manual_seed(3)
    T = sum(new)
    nqkv = (H + 2 * G) * hd
    qkv = torch.empty((T, nqkv), device="cuda")
    q, out = (torch.full((T, H * hd), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    start = c.cache.cache.clone()

    def batch(i):
        c.cache.set_batch(new, ctx[i], c.table)
        qkv.copy_(torch.randn((T, nqkv), generator=g, device="cuda"))

    batch(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.cache.append(0, qkv, q)
        c.cache.attend(0, q, out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.append(0, qkv, q)
        c.cache.attend(0, q, out)
        with pytest.raises(moe.MoeError) as e:
            c.cache.set_batch(new, ctx[0], c.table)
        assert e.value.status == -5
    for i in [0, 1, 2, 3, 4, 4, 1]:
        batch(i)
        c.cache.cache.copy_(start)
        c.cache.append(0, qkv, q)
        c.cache.attend(0, q, out)
        torch.cuda.synchronize()
        want = [q.clone(), out.clone(), c.cache.cache.clone()]
        c.cache.cache.copy_(start)
        q.fill_(7.0)
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, [q, out, c.cache.cache]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), i
        torch.randn(1000, device="cuda").sum().item()


@pytest.mark.parametrize("order", [[0, 2000, 500, 4000, 0], [2000, 0, 4000, 100]], ids=str)
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_graph_replays_take_the_blocks_of_a_later_batch(torch, e4m3, order):
    """A prompt's pieces, captured at one length and replayed at others, for which the rows are
    divided into blocks of the other kind, and positions into ranges."""
    H, G, hd, P, n = 16, 1, 64, 64, 300
    c = Case(torch, H, G, hd, P, e4m3, [(max(order), n)], seed=19)
    c.fill_context(new_too=True)
    q = c.queries()
    want, out = torch.empty_like(q), torch.empty_like(q)
    c.cache.set_batch([n], order[:1], c.table)
    c.cache.attend(0, q, want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.attend(0, q, out)
    for p0 in order:
        c.cache.set_batch([n], [p0], c.table)
        c.cache.attend(0, q, want)
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(want.view(torch.int16), out.view(torch.int16)), p0
        c.lens = [(p0, n)]
        c.check_attend(q, out)


def test_two_contexts_on_two_streams(torch):
    """Two caches, each on a stream of its own at the same time, many steps: as one after the other."""
    cases = [Case(torch, 4, 2, 64, 16, e, [(500, 1), (37, 20)], seed=s) for s, e in ((21, False), (22, True))]
    streams = [torch.cuda.Stream() for _ in cases]
    data = []
    for c in cases:
        c.fill_context()
        data.append((rows_of(c, torch.float32), *(torch.empty((c.T, 256), dtype=torch.bfloat16, device="cuda") for _ in range(2))))

    def step(c, x, q, out):
        c.set_batch()
        c.cache.append(0, x, q)
        c.cache.attend(0, q, out)
    want = []
    for c, d in zip(cases, data):
        step(c, *d)
        torch.cuda.synchronize()
        want.append(d[2].clone())
        d[2].zero_()
    torch.cuda.synchronize()
    for _ in range(10):
        for c, d, st in zip(cases, data, streams):
            with torch.cuda.stream(st):
                step(c, *d)
    torch.cuda.synchronize()
    for d, w in zip(data, want):
        assert torch.equal(d[2].view(torch.int16), w.view(torch.int16))


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_nothing_is_written_outside(torch, e4m3):
    """Cache, workspace, q and out inside patterned margins."""
    H, G, hd, P, lens = 48, 8, 128, 16, [(900, 1), (30, 100), (0, 2), (333, 9)]
    c = Case(torch, H, G, hd, P, e4m3, lens, seed=31)
    cb, wb = moe.attn_paged_cache_bytes(c.cfg), moe.attn_paged_workspace_bytes(c.cfg)
    pad = 1 << 16

    def guarded(n):
        t = torch.full((n + 2 * pad,), 0xA5, dtype=torch.uint8, device="cuda")
        return t, t[pad:pad + n]
    (call, cin), (wall, win) = guarded(cb), guarded(wb)
    qall, qin = guarded(c.T * H * hd * 2)
    oall, oin = guarded(c.T * H * hd * 2)
    c.cache = moe.PagedCache(c.cfg, cache=cin, workspace=win)
    c.fill_context()
    c.set_batch()
    q, out = (t.view(torch.bfloat16).view(c.T, H * hd) for t in (qin, oin))
    c.cache.append(0, rows_of(c, torch.float32), q)
    c.cache.attend(0, q, out)
    torch.cuda.synchronize()
    for t in (call, wall, qall, oall):
        assert (t[:pad] == 0xA5).all() and (t[-pad:] == 0xA5).all()
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_pages_behind_four_gigabytes(torch, e4m3):
    """A pool whose keys alone pass 2^32 bytes and 2^31 elements; a sequence on its last pages."""
    H, G, hd, P = 48, 8, 128, 256
    n_pages = (1 << 32) // (G * P * hd * (1 if e4m3 else 2)) + 64
    cfg = moe.make_paged_config(H, G, hd, page_size=P, n_pages=n_pages, max_seqs=2, max_tokens=64, max_blocks=4,
                                rope_theta=THETA, flags=moe.ATTN_PAGED_E4M3 if e4m3 else 0)
    lens = [(300, 1), (10, 30)]
    c = Case(torch, H, G, hd, P, e4m3, lens, seed=41)
    big = {int(p): n_pages - 1 - i for i, p in enumerate(c.table[c.table >= 0])}
    pool = c.pool
    c.cache = moe.PagedCache(cfg)
    small = c.table.copy()
    c.fill_context_at = None
    K, V, ks, vs = c.cache.views(0)
    for s, (p0, n) in enumerate(lens):
        k, v = (c.rng.standard_normal((p0, G, hd)) for _ in range(2))
        pool.append(k, v, 0, small[s])
    for p, b in big.items():
        if e4m3:
            K.view(torch.uint8)[b] = torch.from_numpy(pool.kc[p]).cuda()
            V.view(torch.uint8)[b] = torch.from_numpy(pool.vc[p]).cuda()
            ks[b] = torch.from_numpy(2.0 ** pool.ks[p].astype(np.float64)).float().cuda()
            vs[b] = torch.from_numpy(2.0 ** pool.vs[p].astype(np.float64)).float().cuda()
        else:
            K[b] = torch.from_numpy(pool.k[p]).to(torch.bfloat16).cuda()
            V[b] = torch.from_numpy(pool.v[p]).to(torch.bfloat16).cuda()
    table = np.array([[big.get(int(p), -1) for p in row] for row in small], np.int32)
    c.cache.set_batch([n for _, n in lens], [p for p, _ in lens], table)
    qkv = rows_of(c, torch.float32)
    q = torch.empty((c.T, H * hd), dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    c.cache.append(0, qkv, q)
    c.cache.attend(0, q, out)
    torch.cuda.synchronize()
    x = f64(qkv).reshape(-1, H + 2 * G, hd)
    pos = np.concatenate([np.arange(p, p + n) for p, n in lens])
    turned = ref.rotate(x[:, :H + G], pos, THETA)
    at = 0
    for s, (p0, n) in enumerate(lens):
        pool.append(turned[at:at + n, H:], x[at:at + n, H + G:], p0, small[s])
        at += n
    for p, b in big.items():                              # the keys as they are stored
        if e4m3:
            assert (K.view(torch.uint8)[b].cpu().numpy() != pool.kc[p]).mean() <= 1e-3
            pool.kc[p] = K.view(torch.uint8)[b].cpu().numpy()
        else:
            pool.k[p] = f64(K[b])
    c.table = small
    c.check_attend(q, out)


def test_a_batch_of_nothing(torch):
    c = Case(torch, 4, 2, 64, 16, False, [(3, 1), (0, 0)], seed=51)
    q = torch.full((1, 256), 7.0, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(moe.MoeError) as e:
        c.cache.attend(0, q, torch.empty_like(q))
    assert e.value.status == -5                           # no batch yet
    for lens in ([], [(5, 0), (0, 0)]):
        c.cache.set_batch([n for _, n in lens], [p for p, _ in lens], c.table[:0] if not lens else np.zeros((2, 1), np.int32))
        out = torch.full_like(q, 7.0)
        c.cache.append(0, torch.empty((0, 512), device="cuda"), q)
        c.cache.attend(0, q, out)
        torch.cuda.synchronize()
        assert (out == 7.0).all() and (q == 7.0).all()
