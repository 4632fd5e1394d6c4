"""Routing policies on the GPU against the fp64 reference (e4m3_ref.choose), from the GPU's own fp32
logits: every way a layer is routed (one workgroup, partial logits, many tokens, given logits)."""
import numpy as np
import pytest

import e4m3_ref as ref
import moe_inputs as mi
import paper_2506_23635_amd as moe

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def make(torch, d, E, k, T, first=0, local=0, bias=True, seed=0, f=128, flags=0):
    layer = moe.MoeLayer(moe.make_config(d, f, E, k, expert_begin=first, n_local_experts=local, max_tokens=T, flags=flags))
    rng = np.random.default_rng(seed)
    wr = rng.standard_normal((d, E)).astype(np.float32) * 0.1
    b = rng.standard_normal(E).astype(np.float32) if bias else None
    layer.load_router(0, torch.from_numpy(wr), torch.from_numpy(b) if bias else None)
    x = torch.from_numpy(ref.bf16_bits(rng.standard_normal((T, d))).view(np.int16)).cuda()
    return layer, x


def check(rt, k, E, first, local, **policy):
    """ids and permutation equal, weights rounded once to fp32 (half a step, 2^-24, and the fp64
    terms' own errors, below 2^-40 of the value)."""
    ids, w = ref.choose(rt["logits"], k, **policy)
    assert np.array_equal(rt["idx"], ids)
    assert np.array_equal(np.isnan(rt["w"]), np.isnan(w))
    ok = ~np.isnan(w)
    assert np.all(np.abs(rt["w"][ok] - w[ok]) <= np.abs(w[ok]) * (2.0 ** -24 + 2.0 ** -40) + 2.0 ** -149)
    offsets, pair_row, tokens = ref.permute(ids, first, local, E)
    assert np.array_equal(rt["offsets"], offsets) and np.array_equal(rt["pair_row"], pair_row)
    assert np.array_equal(rt["row_token"], tokens)


POLICIES = [dict(score=1), dict(score=1, renormalize=False, scale=2.5), dict(score=2), dict(score=0, scale=0.5),
            dict(score=2, n_groups=4, top_groups=2, best=2, scale=2.5), dict(score=1, n_groups=4, top_groups=2),
            dict(score=0, n_groups=2, top_groups=1, renormalize=False), dict(score=2, n_groups=8, top_groups=4, renormalize=False)]


def set_policy(layer, balance=None, best=1, **kw):
    layer.set_policy(0, moe.make_policy(group_best=best, **kw), balance)


# (d, T): one workgroup, partial logits, many tokens
@pytest.mark.parametrize("d,T", [(256, 1), (256, 3), (512, 16), (768, 1), (1024, 7), (1024, 16), (256, 17), (768, 130), (6144, 33),
                                 (3840, 300)])
@pytest.mark.parametrize("E,k", [(8, 2), (16, 4), (16, 8), (12, 4), (24, 6), (64, 8)])
@pytest.mark.parametrize("balanced", [False, True])
def test_from_x(torch, d, T, E, k, balanced):
    layer, x = make(torch, d, E, k, T, seed=T + E)
    balance = torch.randn(E, generator=torch.Generator().manual_seed(E)).cuda() * 0.2 if balanced else None
    for p in POLICIES:
        if E % p.get("n_groups", 1) or p.get("top_groups", 1) * E // p.get("n_groups", 1) < k:
            continue
        set_policy(layer, balance, **p)
        rt = layer.routing_tensors(layer.route(0, x))
        check(rt, k, E, 0, E, balance=balance.cpu().numpy() if balanced else None, **p)
    layer.close()


@pytest.mark.parametrize("T", [1, 5, 64, 333])
@pytest.mark.parametrize("E,k,groups,top,best", [(1, 1, 1, 1, 1), (3, 2, 3, 2, 1), (48, 6, 6, 3, 2), (64, 8, 8, 4, 2),
                                                 (64, 64, 1, 1, 1), (60, 9, 15, 5, 1), (16, 4, 16, 4, 1),
                                                 (60, 8, 4, 2, 2), (12, 4, 4, 2, 2), (63, 5, 7, 3, 2)])
@pytest.mark.parametrize("score", [0, 1, 2])
def test_given_logits(torch, T, E, k, groups, top, best, score):
    layer, _ = make(torch, 256, E, k, T)
    g = torch.Generator().manual_seed(T * 100 + E)
    logits = (torch.randn((T, E), generator=g) * 3).cuda()
    logits[0] = 1.25                                                   # all equal: by id
    balance = (torch.randn(E, generator=g) * 0.3).cuda()
    for bal in (None, balance):
        set_policy(layer, bal, best, score=score, n_groups=groups, top_groups=top)
        rt = layer.routing_tensors(layer.route(0, None, logits_in=logits))
        check(rt, k, E, 0, E, score=score, n_groups=groups, top_groups=top, best=best,
              balance=None if bal is None else bal.cpu().numpy())
    layer.close()


@pytest.mark.parametrize("first,local", [(0, 4), (4, 4), (12, 4), (5, 1)])
@pytest.mark.parametrize("T", [2, 16, 40])
def test_a_share_of_the_experts(torch, first, local, T):
    layer, x = make(torch, 768, 16, 4, T, first, local)
    set_policy(layer, score=2, n_groups=4, top_groups=2, best=2)
    check(layer.routing_tensors(layer.route(0, x)), 4, 16, first, local, score=2, n_groups=4, top_groups=2, best=2)
    layer.close()


INF, NAN = float("inf"), float("nan")
ROWS = [[-INF] * 8, [NAN] * 8, [INF] * 8, [0.0] * 8, [-INF] * 7 + [1.0], [1, NAN, 2, 3, 4, 5, 6, 7],
        [1, INF, 2, 3, 4, 5, 6, 7], [-INF, 3, -INF, 3, 5, -INF, 5, -INF], [800, -800, 0, 1, 2, -900, 3, -850],
        [-900, -800, -1000, -950, -801, -802, -803, -804], [3.0e38, -3.0e38, 1, 2, 3, 4, 5, 6],
        [60, 50, 70, 80, 45, 65, 55, 75], [NAN, -INF, INF, 0, NAN, -INF, 0, 0]]


@pytest.mark.parametrize("score", [0, 1, 2])
@pytest.mark.parametrize("groups,top,best", [(1, 1, 1), (4, 2, 1), (4, 3, 2), (2, 1, 2)])
@pytest.mark.parametrize("renormalize", [False, True])
def test_rows_at_the_edges(torch, score, groups, top, best, renormalize):
    """Rows without a finite logit, NaN, equal and far logits, balances that ban experts."""
    T, E, k = len(ROWS), 8, 3
    layer, _ = make(torch, 256, E, k, T)
    logits = torch.tensor(ROWS, dtype=torch.float32).cuda()
    bans = torch.tensor([0, -INF, 0, -INF, -INF, 0, -INF, -INF]).cuda()
    for balance in (None, bans, torch.full((E,), -INF).cuda(), torch.full((E,), NAN).cuda()):
        p = dict(score=score, n_groups=groups, top_groups=top, best=best, renormalize=renormalize)
        set_policy(layer, balance, **p)
        rt = layer.routing_tensors(layer.route(0, None, logits_in=logits))
        check(rt, k, E, 0, E, balance=None if balance is None else balance.cpu().numpy(), **p)
        assert all(len(set(r)) == k for r in rt["idx"].tolist())
    layer.close()


def test_edges_from_x(torch):
    """The decode paths on rows whose logits are NaN or infinite."""
    for d in (256, 1024):
        layer, x = make(torch, d, 16, 4, 4, bias=False)
        x = x.view(torch.bfloat16).clone()
        x[1, 5], x[2, 7], x[3, 9] = NAN, INF, -INF
        for p in (dict(score=1), dict(score=2, n_groups=4, top_groups=2, best=2), dict(score=0)):
            set_policy(layer, **p)
            check(layer.routing_tensors(layer.route(0, x)), 4, 16, 0, 16, **p)
        layer.close()


@pytest.mark.parametrize("T,E,k", [(1100, 64, 8), (3000, 16, 4), (9000, 20, 2)])
def test_many_tokens(torch, T, E, k):
    """Several workgroups of the permutation and of every range of the reduction axis, or one range."""
    layer, x = make(torch, 1536, E, k, T, first=E // 4, local=E // 2)
    p = dict(score=2, n_groups=4, top_groups=2, best=2, scale=2.5)
    set_policy(layer, **p)
    rt = layer.routing_tensors(layer.route(0, x))
    ids, w = ref.choose(rt["logits"], k, **p)
    assert np.array_equal(rt["idx"], ids)
    assert np.all(np.abs(rt["w"] - w) <= np.abs(w) * (2.0 ** -24 + 2.0 ** -40))
    offsets, pair_row, tokens = ref.permute(ids, E // 4, E // 2, E)
    assert np.array_equal(rt["offsets"], offsets) and np.array_equal(rt["pair_row"], pair_row)
    assert np.array_equal(rt["row_token"], tokens) and np.array_equal(rt["counts"], np.diff(offsets))
    layer.close()


@pytest.mark.parametrize("d,T,E", [(256, 1, 64), (6144, 5, 16), (6144, 40, 16), (6144, 40, 64), (4096, 700, 17)])
def test_logits_are_the_exact_sums_rounded(torch, d, T, E):
    """fp32 of the exact sum: the fp64 sums' own error, d 2^-53 of the sum of magnitudes, may move one
    that lies at a border by a step."""
    layer, x = make(torch, d, E, 1, T, bias=False, seed=7)
    wr = np.random.default_rng(7).standard_normal((d, E)).astype(np.float32) * 0.1
    rt = layer.routing_tensors(layer.route(0, x))
    v = ref.f64(x.cpu().numpy().view(np.uint16))
    exact = v @ wr.astype(np.float64)
    slack = 2 * d * 2.0 ** -53 * (np.abs(v) @ np.abs(wr.astype(np.float64)))
    assert np.all(np.abs(rt["logits"] - exact) <= np.abs(exact) * 2.0 ** -24 + slack)
    assert np.mean(rt["logits"] == exact.astype(np.float32)) > 0.999
    layer.close()


@pytest.mark.parametrize("T", [4, 40])
def test_no_policy_is_what_it_was(torch, T):
    layer, x = make(torch, 256, 16, 4, T)
    before = layer.routing_tensors(layer.route(0, x))
    set_policy(layer, score=2)
    other = layer.routing_tensors(layer.route(0, x))
    assert not np.array_equal(other["w"], before["w"])
    layer.set_policy(0, None)
    after = layer.routing_tensors(layer.route(0, x))
    for name in before:
        assert np.array_equal(before[name], after[name]), name
    # "selected" without more is the same choice, its weights formed in fp64: 8 fp32 roundings (the
    # largest exponential of an fp32 softmax has 3, their sum k - 1, the quotient and product 2)
    set_policy(layer, score=0)
    same = layer.routing_tensors(layer.route(0, x))
    assert np.array_equal(same["idx"], before["idx"])
    assert np.allclose(same["w"], before["w"], rtol=8 * 2.0 ** -24, atol=0)
    layer.close()


def test_layers_have_their_own_policies(torch):
    layer = moe.MoeLayer(moe.make_config(256, 128, 8, 2, n_layers=2, max_tokens=9))
    rng = np.random.default_rng(5)
    for l in range(2):
        layer.load_router(l, torch.from_numpy(rng.standard_normal((256, 8)).astype(np.float32)))
    x = torch.from_numpy(ref.bf16_bits(rng.standard_normal((9, 256))).view(np.int16)).cuda()
    layer.set_policy(1, moe.make_policy(moe.SCORE_SIGMOID, renormalize=False))
    check(layer.routing_tensors(layer.route(1, x)), 2, 8, 0, 8, score=2, renormalize=False)
    check_w = layer.routing_tensors(layer.route(0, x))["w"]
    assert np.allclose(check_w.sum(axis=1), 1.0, rtol=1e-6)            # layer 0: the softmax over the selected
    layer.close()


def load(torch, layer, wl):
    from harness import load_workload_host
    load_workload_host(layer, wl)


def test_forwards_follow_the_policy(torch):
    """moe_forward with its own routing equals moe_route and moe_forward of it, and so do the static,
    residual and stacked forms; a routing from before a new policy is refused."""
    wl = mi.WORKLOADS["tiny"].with_(T=40)
    layer = moe.MoeLayer(moe.make_config(wl.d, wl.f, wl.E, wl.k, max_tokens=40))
    load(torch, layer, wl)
    x = torch.from_numpy(wl.x().view(np.int16)).cuda()
    balance = torch.linspace(-0.3, 0.3, wl.E).cuda()
    plain = torch.empty_like(x)
    layer.forward(0, x, plain)
    set_policy(layer, balance, score=2, n_groups=4, top_groups=2, best=2, scale=2.0)
    for T in (1, 16, 40):
        a, b, c, r = (torch.empty_like(x[:T]) for _ in range(4))
        layer.forward(0, x[:T], a)
        layer.forward(0, x[:T], b, routing=layer.route(0, x[:T]))
        layer.forward_static(0, x[:T], c)
        r.copy_(x[:T])
        layer.forward_residual(0, x[:T], r)
        s = x[:T].clone()
        layer.forward_stack(s)
        assert torch.equal(a, b) and torch.equal(a, c) and not torch.equal(a, plain[:T])
        assert torch.equal(r, s)
        want = (x[:T].view(torch.bfloat16).double() + a.view(torch.bfloat16).double()).to(torch.bfloat16)
        assert torch.equal(r.view(torch.bfloat16), want)
    routing = layer.route(0, x)
    set_policy(layer, score=1)
    with pytest.raises(moe.MoeError) as err:
        layer.forward(0, x, a, routing=routing)
    assert err.value.status == -5
    layer.close()


@pytest.mark.parametrize("T", [3, 30])
def test_a_captured_routing_reads_the_balance(torch, T):
    """Replays see what the balance holds then, with eager work of the same layer between them."""
    layer, x = make(torch, 768, 16, 4, T)
    balance = torch.zeros(16, device="cuda")
    p = dict(score=2, n_groups=4, top_groups=2, best=2)
    set_policy(layer, balance, **p)
    routing = layer.route(0, x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.route(0, x)
    for i in range(4):
        balance.copy_(torch.randn(16, generator=torch.Generator().manual_seed(i)) * 0.4)
        graph.replay()
        torch.cuda.synchronize()
        rt = layer.routing_tensors(routing)
        check(rt, 4, 16, 0, 16, balance=balance.cpu().numpy(), **p)
        eager = layer.routing_tensors(layer.route(0, x))
        assert np.array_equal(rt["w"], eager["w"])
    layer.close()


def test_set_policy_arguments(torch):
    layer, _ = make(torch, 256, 8, 2, 1)
    p = moe.make_policy(moe.SCORE_SOFTMAX)
    for bad in (torch.zeros(8), torch.zeros(8, dtype=torch.float64, device="cuda"), torch.zeros(7, device="cuda"),
                torch.zeros(16, device="cuda")[::2]):
        with pytest.raises(moe.MoeError):
            layer.set_policy(0, p, bad)
    with pytest.raises(moe.MoeError):
        layer.set_policy(0, None, torch.zeros(8, device="cuda"))
    with pytest.raises(moe.MoeError):
        layer.set_policy(1, p)
    layer.close()
