"""A policy's balance and the streams that read it (MoeLayer.set_policy): recorded on each stream that a
routing goes to, kept where the routing is captured."""
import numpy as np
import pytest

import e4m3_ref as ref
import paper_2506_23635_amd as moe


class FakeStream:
    def __init__(self, handle):
        self.cuda_stream = handle


class FakeCuda:
    current, capturing = FakeStream(1), False

    def current_stream(self, device):
        return self.current

    def is_current_stream_capturing(self):
        return self.capturing


class FakeTorch:
    def __init__(self):
        self.cuda = FakeCuda()


class FakeBalance:
    def __init__(self):
        self.recorded = []

    def record_stream(self, stream):
        self.recorded.append(stream.cuda_stream)


@pytest.fixture
def layer(monkeypatch):
    """A layer whose calls end before the library."""
    L = object.__new__(moe.MoeLayer)
    L.torch, L.device, L.ctx = FakeTorch(), "cuda:0", None
    L.cfg = moe.make_config(256, 128, 4, 2, n_layers=6)
    L._balance, L._captured = {}, []
    monkeypatch.setattr(moe, "_raw_stream", lambda torch, device: torch.cuda.current.cuda_stream)
    monkeypatch.setattr(moe, "_on_device", lambda torch, device: moe._HERE)
    monkeypatch.setattr(moe, "_tensor_ptr", lambda *a: 0)
    monkeypatch.setattr(moe, "_bf16_types", lambda torch: ())
    for name in ("moe_set_policy", "moe_route", "moe_forward", "moe_forward_static", "moe_forward_stack", "moe_forward_residual",
                 "moe_forward_layers"):
        monkeypatch.setattr(moe, name, lambda *a: None)
    L.torch.float32 = None
    return L


CALLS = [lambda L, x: L.route(2, x, T=1), lambda L, x: L.forward(2, x, x, T=1), lambda L, x: L.forward_static(2, x, x, T=1),
         lambda L, x: L.forward_residual(2, x, x, T=1), lambda L, x: L.forward_layers(1, 2, x, T=1), lambda L, x: L.forward_stack(x, T=1)]


@pytest.mark.parametrize("call", range(len(CALLS)))
def test_each_call_records_its_stream_once(layer, call):
    a, other = FakeBalance(), FakeBalance()
    policy = moe.make_policy()
    layer.set_policy(2, policy, a)
    layer.set_policy(5, policy, other)
    x = object()
    for handle in (1, 2, 1, 2):
        layer.torch.cuda.current = FakeStream(handle)
        CALLS[call](layer, x)
    assert a.recorded == [1, 2]
    assert other.recorded == ([1, 2] if call == 5 else [])           # only the stack routes layer 5
    b = FakeBalance()
    layer.set_policy(2, policy, b)
    CALLS[call](layer, x)
    assert a.recorded == [1, 2] and b.recorded == [2]
    layer.set_policy(2, policy)
    layer.set_policy(5, None)
    CALLS[call](layer, x)
    assert b.recorded == [2] and not layer._captured


def test_captured_calls_keep_the_balance(layer):
    a, b = FakeBalance(), FakeBalance()
    layer.set_policy(0, moe.make_policy(), a)
    layer.torch.cuda.capturing = True
    layer.route(0, object(), T=1)
    layer.route(0, object(), T=1)
    assert layer._captured == [a] and not a.recorded
    layer.set_policy(0, moe.make_policy(), b)
    assert layer._captured == [a]
    layer.torch.cuda.capturing = False
    layer.route(0, object(), T=1)
    assert layer._captured == [a] and b.recorded == [1]


# ------------------------------------------------------------------- GPU --

@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def gpu_layer(torch, T):
    L = moe.MoeLayer(moe.make_config(256, 128, 16, 4, max_tokens=T))
    L.load_router(0, torch.zeros((256, 16)))
    return L, torch.randn((T, 16), generator=torch.Generator().manual_seed(1)).cuda()


def balance(torch, seed):
    return torch.randn(16, generator=torch.Generator().manual_seed(seed)).cuda()


@pytest.mark.gpu
def test_a_routing_on_another_stream_reads_what_was_set(torch):
    """Routings wait on a side stream while their policy is replaced, its balance dropped and memory of
    that size taken and written."""
    L, logits = gpu_layer(torch, 40)
    policy = moe.make_policy(moe.SCORE_SIGMOID)
    b = balance(torch, 2)
    want, _ = ref.choose(logits.cpu().numpy(), 4, 2, balance=b.cpu().numpy())
    L.set_policy(0, policy, b)
    L.route(0, None, logits_in=logits)                                 # (loads the kernels)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)                                  # some 10 ms
        r = L.route(0, None, logits_in=logits)
    L.set_policy(0, None)
    del b
    taken = [torch.full((16,), float(i % 5), device="cuda") for i in range(400)]
    side.synchronize()
    got = L.routing_tensors(r)
    assert np.array_equal(got["idx"], want)
    del taken
    L.close()


@pytest.mark.gpu
def test_a_graph_reads_the_balance_that_it_was_captured_with(torch):
    L, logits = gpu_layer(torch, 40)
    policy = moe.make_policy(moe.SCORE_SIGMOID)
    b = balance(torch, 3)
    want, _ = ref.choose(logits.cpu().numpy(), 4, 2, balance=b.cpu().numpy())
    other = balance(torch, 4)
    want_other, _ = ref.choose(logits.cpu().numpy(), 4, 2, balance=other.cpu().numpy())
    L.set_policy(0, policy, b)
    r = L.route(0, None, logits_in=logits)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.route(0, None, logits_in=logits)
    L.set_policy(0, policy, other)
    del b
    taken = [torch.full((16,), float(i % 5), device="cuda") for i in range(400)]
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(L.routing_tensors(r)["idx"], want)
        assert np.array_equal(L.routing_tensors(L.route(0, None, logits_in=logits))["idx"], want_other)
    del taken
    L.close()
