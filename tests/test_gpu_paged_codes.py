"""Where the page numbers and positions are large, every stored value and code for itself: no share
of wrong ones is let through."""
import numpy as np
import pytest

import paged_ref as ref
import paper_2506_23635_amd as moe
from test_gpu_paged import THETA, Case, f64, rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def check_new(c, where, qkv, pos, pages):
    """The new tokens' keys and values as stored: token t at slot where[t][1] of the device's page
    where[t][0], which is page where[t][2] of the fp64 pool (appended to before)."""
    torch = c.torch
    K, V, ks, vs = pages
    x = f64(qkv).reshape(-1, c.H + 2 * c.G, c.hd)[:, c.H:c.H + c.G]
    turned, err = ref.rotate(x, pos, THETA), ref.rotation_error(x)
    # (the angle's own rounding to fp64, in the kernel and in ref.rotate)
    a, b = np.split(np.abs(x), 2, axis=-1)
    err = err + np.concatenate([a + b, a + b], axis=-1) * np.asarray(pos)[:, None, None] * 2.0 ** -51
    for t, (dev, slot, pool) in enumerate(where):
        if not c.e4m3:
            k, v = f64(K[dev, :, slot]), f64(V[dev, :, slot])
            assert (np.abs(k - turned[t]) <= ref.BF16 * np.abs(turned[t]) + (1 + ref.BF16) * err[t] + 1e-37).all(), t
            assert np.array_equal(v, c.pool.v[pool, :, slot]), t
            continue
        assert np.array_equal(np.log2(f64(ks[dev])), c.pool.ks[pool]) and np.array_equal(np.log2(f64(vs[dev])), c.pool.vs[pool]), t
        kc, vc = (p[dev, :, slot].view(torch.uint8).cpu().numpy() for p in (K, V))
        assert np.array_equal(vc, c.pool.vc[pool, :, slot]), t
        # a key: a code no further from the exact value than half a step, beside the rotation's error
        scale = 2.0 ** c.pool.ks[pool][:, None].astype(np.float64)
        half = np.maximum(np.abs(turned[t]), 2.0 ** -6 * scale) * 2.0 ** -4
        assert (np.abs(ref.E4M3[kc] * scale - turned[t]) <= half * (1 + 1e-12) + (1 + 2.0 ** -4) * err[t]).all(), t


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("n", [2, 40])
def test_the_last_positions(torch, n, e4m3):
    H, G, hd, P, blocks = 4, 2, 64, 256, 65536
    p0 = blocks * P - P
    cache = moe.PagedCache(moe.make_paged_config(H, G, hd, page_size=P, n_pages=3, max_tokens=n, max_blocks=blocks,
                                                 rope_theta=THETA, flags=moe.ATTN_PAGED_E4M3 if e4m3 else 0))
    table = np.full((1, blocks), -1, np.int32)
    table[0, -1] = 2
    cache.set_batch([n], [p0], table)
    c = Case(torch, H, G, hd, P, e4m3, [(0, n)], seed=91)
    c.pool = ref.Pool(3, G, P, hd, e4m3)
    qkv = rows_of(c, torch.float32)
    q = torch.empty((n, H * hd), dtype=torch.bfloat16, device="cuda")
    cache.append(0, qkv, q)
    torch.cuda.synchronize()
    x, pos = f64(qkv).reshape(n, H + 2 * G, hd), p0 + np.arange(n)
    c.pool.append(ref.rotate(x[:, H:H + G], pos, THETA), x[:, H + G:], 0, [2])
    check_new(c, [(2, i, 2) for i in range(n)], qkv, pos, cache.views(0))


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_pages_behind_four_gigabytes(torch, e4m3):
    H, G, hd, P = 48, 8, 128, 256
    n_pages = (1 << 32) // (G * P * hd * (1 if e4m3 else 2)) + 64
    cfg = moe.make_paged_config(H, G, hd, page_size=P, n_pages=n_pages, max_seqs=2, max_tokens=64, max_blocks=4,
                                rope_theta=THETA, flags=moe.ATTN_PAGED_E4M3 if e4m3 else 0)
    lens = [(0, 5), (256, 30)]                             # (from a page's first slot on: its scale is the new tokens')
    c = Case(torch, H, G, hd, P, e4m3, lens, seed=93)
    table = np.where(c.table >= 0, n_pages - 1 - c.table, -1)
    cache = moe.PagedCache(cfg)
    cache.set_batch([n for _, n in lens], [p for p, _ in lens], table)
    qkv = rows_of(c, torch.float32)
    q = torch.empty((c.T, H * hd), dtype=torch.bfloat16, device="cuda")
    cache.append(0, qkv, q)
    torch.cuda.synchronize()
    x = f64(qkv).reshape(-1, H + 2 * G, hd)
    pos = np.concatenate([np.arange(p, p + n) for p, n in lens])
    turned, where, at = ref.rotate(x[:, :H + G], pos, THETA), [], 0
    for s, (p0, n) in enumerate(lens):
        c.pool.append(turned[at:at + n, H:], x[at:at + n, H + G:], p0, c.table[s])
        where += [(int(table[s, p // P]), p % P, int(c.table[s, p // P])) for p in range(p0, p0 + n)]
        at += n
    check_new(c, where, qkv, pos, cache.views(0))
