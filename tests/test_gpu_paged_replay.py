"""Graphs over the paged cache's calls, replayed on batches that they were not captured for."""
import pytest

from test_gpu_paged import Case, rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("new,others", [([2, 1, 1], [[2, 1, 0], [0, 0, 0], [3, 1, 1], [1, 60, 1]]),
                                        ([1, 40, 2], [[1, 39, 2], [2, 2, 0], [0, 0, 0], [1, 1, 60], [40, 40, 40]])], ids=str)
def test_a_batch_of_other_tokens_is_left_alone(torch, new, others, e4m3):
    """Fewer tokens, none, more: pages, queries and results stay as they are; on a batch of the
    captured kind the graph gives the eager results again."""
    H, G, hd, P = 6, 1, 128, 16
    ctx = [300, 31, 900]
    c = Case(torch, H, G, hd, P, e4m3, [(p + 20, 64) for p in ctx], seed=83)
    c.fill_context()
    c.lens = [(p, n) for p, n in zip(ctx, new)]
    c.T = sum(new)
    qkv = rows_of(c, torch.float32)
    q, out = (torch.full((c.T, H * hd), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c.cache.set_batch(new, ctx, c.table)
    c.cache.append(0, qkv, q)
    c.cache.attend(0, q, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.append(0, qkv, q)
        c.cache.attend(0, q, out)
    for n in others:
        c.cache.set_batch(n, ctx, c.table)
        before = c.cache.cache.clone()
        q.fill_(7.0)
        out.fill_(7.0)
        for _ in range(2):
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(before, c.cache.cache) and (q == 7.0).all() and (out == 7.0).all(), n
        c.cache.set_batch(new, [p + 13 for p in ctx], c.table)
        start = c.cache.cache.clone()
        c.cache.append(0, qkv, q)
        c.cache.attend(0, q, out)
        torch.cuda.synchronize()
        want = [t.clone() for t in (c.cache.cache, q, out)]
        c.cache.cache.copy_(start)
        q.fill_(7.0)
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (c.cache.cache, q, out)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), n
