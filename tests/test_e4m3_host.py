"""Routing policies and products in e4m3 on the host: sizes, refusals before anything is launched, the
coding of weights in host memory, and the references' own pins."""
import ctypes

import numpy as np
import pytest

import e4m3_ref as ref
import paper_2506_23635_amd as moe

E_ARG, E_SHAPE, E_ALIGN, E_CAPACITY, E_STATE = -1, -2, -3, -4, -5


# -------------------------------------------------------------- references --

def test_grid_agrees_with_torch():
    """The reference's rounding against torch's conversion, over values around every code and tie."""
    torch = pytest.importorskip("torch")
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    codes = np.unique(codes[np.isfinite(codes)])
    mids = (codes[1:] + codes[:-1]) / 2
    v = np.concatenate([codes, mids, np.nextafter(mids, np.inf), np.nextafter(mids, -np.inf)]).astype(np.float32)
    v = np.concatenate([v, np.nextafter(v, np.float32(500)), np.nextafter(v, np.float32(-500))])
    v = v[np.abs(v) <= 448]
    want = torch.from_numpy(v).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.grid(v), want)


def test_exponent_is_the_least():
    amax = np.array([0.0, 2.0 ** -140, 448.0, np.nextafter(448.0, 500), 1.75, 1.0, 3.0e38, 448 * 2.0 ** -100])
    assert ref.exponent(amax).tolist() == [-100, -100, 0, 1, -8, -8, 119, -100]


def test_choice_by_hand():
    l = np.log(np.array([[1.0, 2.0, 3.0, 4.0]]))
    ids, w = ref.choose(l, 2, 1, renormalize=False)
    assert ids.tolist() == [[3, 2]] and np.allclose(w, [[0.4, 0.3]], rtol=1e-6)
    ids, w = ref.choose(l, 2, 1, balance=np.array([0.5, 0.0, 0.0, 0.0]), renormalize=False, scale=2.0)
    assert ids.tolist() == [[0, 3]] and np.allclose(w, [[0.2, 0.8]], rtol=1e-6)     # the balance is not in the weights
    # groups {0, 1} and {2, 3}: the largest single value is in the second, the largest pair in the first
    l = np.array([[2.0, 1.9, 2.1, -9.0]])
    assert ref.choose(l, 2, 0, n_groups=2, top_groups=1, best=1)[0].tolist() == [[2, 3]]
    assert ref.choose(l, 2, 0, n_groups=2, top_groups=1, best=2)[0].tolist() == [[0, 1]]


# ---------------------------------------------------------------- policies --

@pytest.fixture
def ctx():
    # fake device addresses: every call below fails its checks, or is host work
    c = moe.moe_init(moe.make_config(256, 128, 12, 4, n_layers=2, max_tokens=8), 1 << 20, 1 << 30)
    yield c
    moe.moe_destroy(c)


def set_policy(ctx, layer=0, balance=None, **kw):
    p = moe.make_policy(**kw)
    p.balance = balance
    return moe.lib().moe_set_policy(ctx, layer, ctypes.byref(p))


def test_policies_accepted(ctx):
    assert moe.lib().moe_set_policy(ctx, 1, None) == 0
    for score in (moe.SCORE_SELECTED, moe.SCORE_SOFTMAX, moe.SCORE_SIGMOID):
        assert set_policy(ctx, score=score, renormalize=False, scale=-1.0) == 0
    assert set_policy(ctx, n_groups=3, top_groups=1, group_best=2) == 0
    assert set_policy(ctx, n_groups=12, top_groups=4, balance=1 << 21) == 0


@pytest.mark.parametrize("kw,status", [(dict(layer=2), E_ARG), (dict(layer=-1), E_ARG), (dict(score=3), E_ARG),
                                       (dict(score=-1), E_ARG), (dict(n_groups=0), E_SHAPE), (dict(n_groups=5), E_SHAPE),
                                       (dict(n_groups=24), E_SHAPE), (dict(n_groups=3, top_groups=0), E_ARG),
                                       (dict(n_groups=3, top_groups=4), E_ARG),
                                       (dict(n_groups=6, top_groups=1), E_SHAPE),       # two experts for four slots
                                       (dict(group_best=0), E_ARG), (dict(group_best=3), E_ARG),
                                       (dict(n_groups=12, top_groups=4, group_best=2), E_ARG),
                                       (dict(renormalize=2), E_ARG), (dict(scale=float("nan")), E_ARG),
                                       (dict(scale=float("inf")), E_ARG), (dict(balance=(1 << 20) + 4), E_ALIGN)], ids=str)
def test_policies_refused(ctx, kw, status):
    kw = dict(kw)
    renormalize = kw.pop("renormalize", None)
    p = moe.make_policy(**{k: v for k, v in kw.items() if k not in ("layer", "balance")})
    if renormalize is not None:
        p.renormalize = renormalize
    p.balance = kw.get("balance")
    assert moe.lib().moe_set_policy(ctx, kw.get("layer", 0), ctypes.byref(p)) == status
    assert moe.moe_last_error(ctx)


def test_policy_without_a_context():
    assert moe.lib().moe_set_policy(None, 0, None) == E_ARG


# ----------------------------------------------------------- e4m3's layers --

def test_layer_bytes():
    d, f = 512, 384
    cfg = moe.make_config(d, f, 4, 2, n_layers=3, flags=moe.MOE_E4M3 | moe.MOE_PARTIAL_F32)
    scales = 2 * (f // 128) * 4 * 1 + (d // 128) * 4 * 1          # dwords of four blocks: 512 and 384 take one
    expert = (3 * d * f + scales + 255) // 256 * 256
    assert moe.moe_weight_bytes(cfg) == 3 * (d * 4 * 4 + 256 + 4 * expert)
    m = moe.moe_workspace_map(cfg)
    assert list(m) == moe.WS_REGIONS and moe.moe_workspace_bytes(cfg) >= sum(m["o"])
    assert moe.moe_weight_bytes(cfg) < moe.moe_weight_bytes(moe.make_config(d, f, 4, 2, n_layers=3))


@pytest.mark.parametrize("flags", [2, 3, 6, 8, 12])
def test_other_flags_stay_refused(flags):
    assert moe.moe_weight_bytes(moe.make_config(256, 128, 4, 2, flags=flags)) == 0


# -------------------------------------------------------------- quantising --

@pytest.mark.parametrize("args,status", [
    ((4096, 64, 2, 4, 64, 8192, 16384), E_ARG), ((4096, 64, -1, 4, 64, 8192, 16384), E_ARG),     # type
    ((4096, 64, 0, -1, 64, 8192, 16384), E_ARG), ((None, 64, 0, 4, 64, 8192, 16384), E_ARG),
    ((4096, 64, 0, 4, 64, None, 16384), E_ARG), ((4096, 64, 0, 4, 64, 8192, None), E_ARG),
    ((4096, 63, 0, 4, 64, 8192, 16384), E_ARG),                                                  # ld below n
    ((4096, 2 ** 32 + 8, 0, 4, 64, 8192, 16384), E_ARG), ((4096, 2 ** 63 - 8, 0, 4, 64, 8192, 16384), E_ARG),
    ((4096, 64, 0, 4, 0, 8192, 16384), E_SHAPE), ((4096, 64, 0, 4, 24, 8192, 16384), E_SHAPE),
    ((4096, 64, 0, 4, (1 << 24) + 16, 8192, 16384), E_SHAPE), ((4096, 64, 0, (1 << 24) + 1, 64, 8192, 16384), E_SHAPE),
    ((4100, 64, 0, 4, 64, 8192, 16384), E_ALIGN), ((4096, 64, 0, 4, 64, 8196, 16384), E_ALIGN),
    ((4096, 66, 0, 4, 64, 8192, 16384), E_ALIGN), ((4096, 68, 1, 4, 64, 8192, 16384), E_ALIGN),  # rows
    ((4096, 64, 0, 4, 64, 4096 + 1008, 16384), E_ARG), ((8192, 64, 0, 4, 64, 8192 - 16, 16384), E_ARG),   # overlaps
    ((4096, 64, 0, 4, 64, 8192, 4100), E_ARG), ((4096, 64, 0, 4, 64, 8192, 8192 + 255), E_ARG),
    ((4096, 96, 0, 4, 64, 4096 + 256, 16384), E_ARG),                                            # between x's rows
    ((None, 0, 1, 0, 64, None, None), 0),                                                        # nothing to do
], ids=str)
def test_quantize_arguments(args, status):
    assert moe.lib().moe_quantize_e4m3(*args, None) == status


# ----------------------------------------------------------------- product --

def test_linear_bytes():
    cfg = moe.make_linear_config(144, 272, max_tokens=5)
    K, N = 256, 512
    assert moe.moe_linear_weight_bytes(cfg) == (K * N + N // 128 * 4 + 255) // 256 * 256
    assert moe.moe_linear_workspace_bytes(cfg) >= 5 * K * 2


@pytest.mark.parametrize("bad", [dict(in_dim=0), dict(in_dim=8), dict(in_dim=24), dict(in_dim=(1 << 20) + 16),
                                 dict(out_dim=0), dict(out_dim=-16), dict(out_dim=40), dict(out_dim=(1 << 20) + 16),
                                 dict(max_tokens=0), dict(max_tokens=(1 << 20) + 1), dict(flags=1),
                                 dict(in_dim=1 << 16, out_dim=1 << 15), dict(in_dim=1 << 14, max_tokens=1 << 16)], ids=str)
def test_linear_configs_refused(bad):
    c = moe.make_linear_config(**{**dict(in_dim=128, out_dim=256, max_tokens=4), **bad})
    assert moe.moe_linear_weight_bytes(c) == 0 and moe.moe_linear_workspace_bytes(c) == 0
    out = ctypes.c_void_p()
    assert moe.lib().moe_linear_init(ctypes.byref(c), 4096, 8192, ctypes.byref(out)) == E_SHAPE
    assert out.value is None and moe.lib().moe_linear_last_error(None)


def test_linear_calls_refused():
    L, out = moe.lib(), ctypes.c_void_p()
    c = moe.make_linear_config(128, 256, max_tokens=4)
    assert L.moe_linear_init(ctypes.byref(c), 4096, 8192, None) == E_ARG
    assert L.moe_linear_init(ctypes.byref(c), None, 8192, ctypes.byref(out)) == E_ARG
    assert L.moe_linear_init(ctypes.byref(c), 4096 + 16, 8192, ctypes.byref(out)) == E_ALIGN
    ctx = moe.moe_linear_init(c, 1 << 20, 1 << 30)
    x, y = 1 << 32, 1 << 33
    try:
        assert L.moe_linear_load(None, x, None) == E_ARG
        assert L.moe_linear_load(ctx, None, None) == E_ARG
        assert L.moe_linear_load(ctx, x + 2, None) == E_ALIGN
        assert L.moe_linear_forward(None, x, 128, y, 0, 1, None) == E_ARG
        assert L.moe_linear_forward(ctx, x, 128, y, 0, -1, None) == E_ARG
        assert L.moe_linear_forward(ctx, x, 128, y, 0, 5, None) == E_CAPACITY
        assert L.moe_linear_forward(ctx, x, 128, y, 2, 1, None) == E_ARG
        assert L.moe_linear_forward(ctx, x, 128, y, 0, 1, None) == E_STATE       # nothing loaded
    finally:
        L.moe_linear_destroy(ctx)
    L.moe_linear_destroy(None)


@pytest.mark.parametrize("n_in,n_out", [(16, 16), (6144, 8192), (1040, 1488), (6144, 256), (128, 1 << 20), (1 << 20, 256),
                                        (2048, 33024)])
def test_linear_workspace_holds_the_ranges_sums(n_in, n_out):
    """A context for more rows has space for what one for fewer rows has: the sums of the ranges of K
    are those of the largest such call, not of max_tokens."""
    K = -(-n_in // 128) * 128
    need = 0
    for T in sorted({1, 16, 17, 40, 63, 64, 65, 127, 128, 129, 200, 256, 257, 500, 1000, 1025, 4000, 16384, 16385}):
        ws = moe.moe_linear_workspace_bytes(moe.make_linear_config(n_in, n_out, max_tokens=T))
        if ws == 0:                                    # beyond the limit on rows
            assert T * K * 2 > 2 ** 31 - 1
            continue
        rows = (T * K * 2 + 255) // 256 * 256
        assert ws >= rows
        need = max(need, ws - rows)
        assert ws - rows >= need


def test_bindings_match_the_header():
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "moe.h")).read()
    assert int(re.search(r"#define MOE_E4M3 0x(\w+)", text).group(1), 16) == moe.MOE_E4M3
    for name, value in (("MOE_SCORE_SELECTED", moe.SCORE_SELECTED), ("MOE_SCORE_SOFTMAX", moe.SCORE_SOFTMAX),
                        ("MOE_SCORE_SIGMOID", moe.SCORE_SIGMOID), ("MOE_T_F32", moe.T_F32), ("MOE_T_BF16", moe.T_BF16)):
        assert re.search(rf"\b{name} = {value}\b", text), name
    fields = re.search(r"typedef struct \{\s*int32_t score,(.*?)\} moe_policy;", text, re.S).group(0)
    assert [n for n, _ in moe.MoePolicy._fields_] == re.findall(r"\b(score|n_groups|top_groups|group_best|renormalize|scale|balance)\b",
                                                                fields)
    assert ctypes.sizeof(moe.MoePolicy) == 32 and ctypes.sizeof(moe.LinearConfig) == 16
