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
        self.cache.cache.fill_(0x7F)     # NaN codes, and large bf16 values, wherever nothing is written
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
