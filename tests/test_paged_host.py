"""The paged cache's C-ABI and binding on the host: sizes, refusals before anything is launched, the
fp64 reference's own pins, and that its bounds fail planted errors."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import paged_ref as ref
import paper_2506_23635_amd as moe

E_ARG, E_SHAPE, E_ALIGN, E_CAPACITY, E_STATE = -1, -2, -3, -4, -5


def cfg(**kw):
    base = dict(n_heads=48, n_kv_heads=8, head_dim=128, page_size=64, n_pages=100, n_layers=2, max_seqs=4, max_tokens=64,
                max_blocks=16)
    base.update(kw)
    return moe.make_paged_config(**base)


def test_cache_bytes():
    data = 100 * 8 * 64 * 128
    assert moe.attn_paged_cache_bytes(cfg()) == 2 * 2 * data * 2
    scales = (100 * 8 * 4 + 255) // 256 * 256
    assert moe.attn_paged_cache_bytes(cfg(flags=moe.ATTN_PAGED_E4M3)) == 2 * 2 * (data + scales)
    assert moe.attn_paged_workspace_bytes(cfg()) > 0


@pytest.mark.parametrize("bad", [dict(head_dim=96), dict(n_kv_heads=5), dict(n_kv_heads=0), dict(n_heads=0),
                                 dict(n_heads=136, n_kv_heads=8), dict(page_size=8), dict(page_size=48),
                                 dict(page_size=512), dict(n_pages=0), dict(n_pages=(1 << 24) + 1), dict(n_layers=0),
                                 dict(max_seqs=0), dict(max_seqs=5000), dict(max_tokens=0), dict(max_tokens=32769),
                                 dict(max_blocks=0), dict(max_blocks=65537), dict(max_blocks=65536, page_size=512),
                                 dict(max_seqs=4096, max_blocks=65536), dict(rope_theta=1.0),
                                 dict(rope_theta=float("nan")), dict(flags=2), dict(n_heads=1024, n_kv_heads=64)],
                         ids=str)
def test_bad_configs_are_refused(bad):
    c = cfg(**bad)
    assert moe.attn_paged_cache_bytes(c) == 0 and moe.attn_paged_workspace_bytes(c) == 0
    out = ctypes.c_void_p()
    assert moe.lib().attn_paged_init(ctypes.byref(c), 4096, 8192, ctypes.byref(out)) == E_SHAPE
    assert out.value is None and moe.lib().attn_paged_last_error(None)


def test_init_pointers():
    L, c, out = moe.lib(), cfg(), ctypes.c_void_p()
    assert L.attn_paged_init(ctypes.byref(c), 4096, 8192, None) == E_ARG
    assert L.attn_paged_init(ctypes.byref(c), None, 8192, ctypes.byref(out)) == E_ARG
    assert L.attn_paged_init(ctypes.byref(c), 4096 + 16, 8192, ctypes.byref(out)) == E_ALIGN
    assert L.attn_paged_init(None, 4096, 8192, ctypes.byref(out)) == E_SHAPE


@pytest.fixture
def ctx():
    # fake device addresses: every call below fails its checks, or has nothing to do
    c = moe.attn_paged_init(cfg(), 1 << 20, 1 << 30)
    yield c
    moe.lib().attn_paged_destroy(c)


def set_batch(ctx, n_new, pos0, table):
    n, p, t = (np.ascontiguousarray(a, np.int32) for a in (n_new, pos0, table))
    return moe.lib().attn_paged_set_batch(ctx, n.size, n.ctypes.data, p.ctypes.data, t.ctypes.data, t.shape[1], None)


PAGES = np.arange(64).reshape(4, 16)


@pytest.mark.parametrize("n_new,pos0,table,status", [
    ([1] * 5, [0] * 5, np.arange(80).reshape(5, 16), E_CAPACITY),          # more than max_seqs
    ([65], [0], PAGES[:1], E_CAPACITY),                                    # more than max_tokens
    ([40, 40], [0, 0], PAGES[:2], E_CAPACITY),
    ([1], [16 * 64], PAGES[:1], E_CAPACITY),                               # longer than max_blocks pages
    ([1], [2 ** 31 - 1], PAGES[:1], E_CAPACITY),
    ([-1], [0], PAGES[:1], E_ARG),
    ([1], [-1], PAGES[:1], E_ARG),
    ([1], [64], PAGES[:1, :1], E_ARG),                                     # a row too short for its pages
    ([1], [0], [[100]], E_ARG),                                            # no such page
    ([1], [0], [[-2]], E_ARG),
    ([1], [70], [[2 ** 31 - 1, 1]], E_ARG),
    ([1, 1], [0, 5], [[3], [3]], E_ARG),                                   # two sequences write one page
    ([64], [32], [[4, 4]], E_ARG),                                         # two blocks of one do
], ids=str)
def test_bad_batches_are_refused(ctx, n_new, pos0, table, status):
    assert set_batch(ctx, [0], [0], PAGES[:1]) == 0                        # nothing new: no launch
    assert set_batch(ctx, n_new, pos0, table) == status
    assert moe.lib().attn_paged_last_error(ctx)
    # the batch before is still set
    assert moe.lib().attn_paged_attend(ctx, 0, None, None, None) == 0


def test_null_arrays_are_refused(ctx):
    L, a = moe.lib(), np.zeros(4, np.int32).ctypes.data
    assert L.attn_paged_set_batch(ctx, -1, a, a, a, 1, None) == E_ARG
    assert L.attn_paged_set_batch(ctx, 1, None, a, a, 1, None) == E_ARG
    assert L.attn_paged_set_batch(ctx, 1, a, None, a, 1, None) == E_ARG
    assert L.attn_paged_set_batch(ctx, 1, a, a, None, 1, None) == E_ARG
    assert L.attn_paged_set_batch(ctx, 1, a, a, a, 0, None) == E_ARG
    assert L.attn_paged_set_batch(None, 0, None, None, None, 0, None) == E_ARG
    assert L.attn_paged_set_batch(ctx, 0, None, None, None, 0, None) == 0


def test_calls_are_refused_before_a_launch(ctx):
    L = moe.lib()
    nqkv = (48 + 16) * 128
    assert L.attn_paged_append(ctx, 0, 4096, nqkv, 0, 4096, None) == E_STATE       # no batch
    assert L.attn_paged_attend(ctx, 0, 4096, 8192, None) == E_STATE
    assert set_batch(ctx, [0], [0], PAGES[:1]) == 0
    for layer in (-1, 2):
        assert L.attn_paged_append(ctx, layer, 4096, nqkv, 0, 4096, None) == E_ARG
        assert L.attn_paged_attend(ctx, layer, 4096, 8192, None) == E_ARG
    assert L.attn_paged_append(ctx, 0, 4096, nqkv, 2, 8192, None) == E_ARG         # unknown type
    assert L.attn_paged_append(ctx, 0, 4096, nqkv - 4, 0, 8192, None) == E_ARG     # rows too close
    assert L.attn_paged_append(ctx, 0, 4096, nqkv + 2, 0, 8192, None) == E_ALIGN
    assert L.attn_paged_append(ctx, 0, 4096, nqkv + 4, 1, 8192, None) == E_ALIGN
    assert L.attn_paged_append(ctx, 0, 4096, 2 ** 62, 0, 8192, None) == E_ARG
    assert L.attn_paged_append(ctx, 0, None, nqkv, 0, None, None) == 0             # no tokens: nothing to do
    assert L.attn_paged_append(None, 0, 4096, nqkv, 0, 8192, None) == E_ARG
    assert L.attn_paged_attend(None, 0, 4096, 8192, None) == E_ARG
    L.attn_paged_destroy(None)


def test_the_block_refuses(ctx):
    L = moe.lib()

    def block(**kw):
        base = dict(d_model=256, n_heads=48, n_kv_heads=8, head_dim=128, n_layers=1, max_seq=1, max_tokens=4)
        base.update(kw)
        return moe.attn_init(moe.make_attn_config(**base), 1 << 20, 1 << 24, 1 << 26)
    a = block()
    assert L.attn_forward_paged(None, 0, ctx, 4096, 4096, None, None) == E_ARG
    assert L.attn_forward_paged(a, 0, None, 4096, 4096, None, None) == E_ARG
    assert L.attn_forward_paged(a, 0, ctx, 4096, 4096, None, None) == E_STATE      # no batch
    assert set_batch(ctx, [0], [0], PAGES[:1]) == 0
    assert L.attn_forward_paged(a, 1, ctx, 4096, 4096, None, None) == E_ARG        # layer of the block
    assert L.attn_forward_paged(a, 0, ctx, 4096, 4096, None, None) == E_STATE      # not loaded
    L.attn_destroy(a)
    for kw in (dict(n_heads=32), dict(n_kv_heads=16), dict(rope_theta=1e4), dict(n_heads=24, n_kv_heads=4, head_dim=64)):
        a = block(**kw)
        assert L.attn_forward_paged(a, 0, ctx, 4096, 4096, None, None) == E_SHAPE
        L.attn_destroy(a)


def test_the_binding_checks_arrays():
    assert moe._int32([1, 2], "n").dtype == np.int32
    for bad in ([1.5], ["1"], [2 ** 31], [-2 ** 31 - 1]):
        with pytest.raises(moe.MoeError):
            moe._int32(bad, "n")
    assert moe._int32([], "n").size == 0


# ------------------------------------------------------- the reference's pins --

def test_e4m3_values():
    torch = pytest.importorskip("torch")
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(t[np.isfinite(t)], ref.E4M3[np.isfinite(ref.E4M3)])
    assert np.array_equal(np.isnan(t), np.isnan(ref.E4M3)) and np.nanmax(ref.E4M3) == 448


def test_e4m3_rounding():
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(1)
    v = np.concatenate([rng.uniform(-448, 448, 20000), rng.standard_normal(20000) * 2.0 ** rng.integers(-12, 6, 20000),
                        (ref.E4M3[:126] + ref.E4M3[1:127]) / 2, ref.E4M3[:127]]).astype(np.float32)
    v = v[np.abs(v) <= 448]
    want = torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ref.e4m3_codes(v), want)


def test_scale_exponents():
    for e in (-99, -1, 0, 5, 118):
        for a, want in ((448.0, e), (np.nextafter(448.0, 500.0), e + 1), (449.0, e + 1), (224.5, e)):
            assert ref.scale_exponent(a * 2.0 ** e) == want
    assert ref.scale_exponent(0.0) == -100 and ref.scale_exponent(3.4e38) == 119


def test_append_in_pieces_is_the_bf16_append_at_once():
    rng = np.random.default_rng(2)
    k, v = rng.standard_normal((2, 50, 2, 64))
    a, b = ref.Pool(5, 2, 16, 64, False), ref.Pool(5, 2, 16, 64, False)
    a.append(k, v, 0, [3, 1, 0, 4])
    for i in range(0, 50, 7):
        b.append(k[i:i + 7], v[i:i + 7], i, [3, 1, 0, 4])
    assert np.array_equal(a.k, b.k) and np.array_equal(a.v, b.v)


def test_a_scale_that_grows_rounds_earlier_codes_again():
    p = ref.Pool(1, 1, 16, 64, True)
    x = np.full((1, 1, 64), 2.0 ** -6)
    p.append(x, x, 0, [0])
    before = p.value(0, 0, 0)[0].copy()
    p.append(np.full((1, 1, 64), 448.0 * 4), x, 1, [0])
    assert p.ks[0, 0] == 2 and p.vs[0, 0] == ref.scale_exponent(2.0 ** -6)
    assert (np.abs(p.value(0, 0, 0)[0] - before) <= 2.0 ** (2 - 9) / 2).all() and (p.value(0, 0, 0)[1] == 448 * 4).all()


@pytest.mark.parametrize("one_term,L", [(False, 90), (True, 12)])
def test_the_bound_fails_planted_errors(one_term, L):
    """A right result rounded to bf16 passes; a key left out, a position too many, a neighbour's
    value and a wrong scale do not.  (One position among 90 can weigh less than 2^-8, the rounding
    of a weight to one bf16 term, and is then no error to be seen: 12 positions there.)"""
    rng = np.random.default_rng(3)
    P, hd, n = 16, 64, 3
    pool = ref.Pool(8, 1, P, hd, False)
    table = [5, 2, 7, 0, 1, 3]
    pool.append(*(rng.standard_normal((2, L, 1, hd)) * 1.5), 0, table)
    q = ref.bf16_round(rng.standard_normal((n, 2, hd)) * 1.5)
    o, wv, ew = ref.attend(q, pool, L - n, table)
    bound = ref.attend_bound(o, wv, ew, L, one_term)
    assert (np.abs(ref.bf16_round(o) - o) <= bound).all()
    for plant in ("late", "early", "scale", "value"):
        if plant in ("late", "early"):
            bad, _, _ = ref.attend(q, pool, L - n + (1 if plant == "late" else -1), table)
        elif plant == "scale":
            bad, _, _ = ref.attend(q * 1.05, pool, L - n, table)
        else:
            other = ref.Pool(8, 1, P, hd, False)
            other.k, other.v = pool.k, np.roll(pool.v, 1, axis=3)
            bad, _, _ = ref.attend(q, other, L - n, table)
        assert (np.abs(bad - o) > bound).any(), plant


def test_batches_are_divided_into_shares_once_each(tmp_path):
    """paged_divide.cpp, under the address and undefined-behaviour sanitizers."""
    here = os.path.dirname(os.path.abspath(__file__))
    exe = str(tmp_path / "paged_divide")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-D__HIP_PLATFORM_AMD__", "-I", rocm + "/include", os.path.join(here, "paged_divide.cpp"), "-o", exe,
                    "-L", rocm + "/lib", "-lamdhip64", "-Wl,-rpath," + rocm + "/lib"], check=True)
    for seed in (1, 2):
        r = subprocess.run([exe, str(seed), "700"], capture_output=True, text=True,
                           env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
        assert r.returncode == 0, r.stdout + r.stderr
        few, tile = map(int, r.stdout.split())
        assert few > 100 and tile > 50                    # divided batches of both kinds were among them
