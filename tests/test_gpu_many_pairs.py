"""More pairs than the permutation's workgroups place in one round each: 1024 workgroups take 1024
pairs a round, so from 1 048 577 pairs on a workgroup places several rounds and carries each expert's
next row from one to the next.  (Up to there a workgroup has one round, however many tokens.)  Routing
alone, from given logits, against a stable sort on the host."""
import numpy as np
import pytest

import e4m3_ref as ref
import paper_2506_23635_amd as moe

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


# (T, k): the last pair of one round each; two rounds, the last workgroup's second one missing; one pair
# into a second round; three rounds with an uneven end
@pytest.mark.parametrize("T,E,k", [(16384, 64, 64), (16400, 64, 64), (349526, 16, 3), (140001, 64, 16)])
@pytest.mark.parametrize("first,local", [(0, 0), (3, 5)])
@pytest.mark.parametrize("policy", [False, True])
def test_rounds_of_a_workgroup(torch, T, E, k, first, local, policy):
    layer = moe.MoeLayer(moe.make_config(256, 128, E, k, expert_begin=first, n_local_experts=local, max_tokens=T))
    layer.load_router(0, torch.zeros((256, E)))
    if policy:
        layer.set_policy(0, moe.make_policy(moe.SCORE_SIGMOID, scale=0.5))
    g = torch.Generator(device="cuda").manual_seed(T + k)
    logits = torch.randn((T, E), generator=g, device="cuda")
    logits[:, 1] += torch.linspace(-2.0, 2.0, T, device="cuda")      # loads that change from round to round
    logits[T // 3:T // 2, 3] -= 50.0                                 # chunks without a pair of an expert, ...
    logits[T // 2:2 * T // 3, 4] += 50.0                             # ... and full of one
    got = layer.routing_tensors(layer.route(0, None, logits_in=logits))
    layer.close()
    ids = np.argsort(-logits.cpu().numpy(), axis=1, kind="stable")[:, :k]
    assert np.array_equal(got["idx"], ids)
    offsets, pair_row, tokens = ref.permute(ids, first, local or E, E)
    assert np.array_equal(got["offsets"], offsets) and np.array_equal(got["counts"], np.diff(offsets))
    assert np.array_equal(got["pair_row"], pair_row)
    assert np.array_equal(got["row_token"], tokens)
