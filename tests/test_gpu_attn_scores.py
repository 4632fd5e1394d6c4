"""The attention block on its own cache where scores are large: the weights are those of the scores'
differences, however large the scores themselves."""
import numpy as np
import pytest

import paged_ref as ref
import paper_2506_23635_amd as moe

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def f64(bits):
    """bf16 bits (numpy uint16) -> fp64."""
    return (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


# (tokens, first position): prompts whole and in pieces, divided ranges, few tokens on either path
CALLS = [(130, 0), (40, 130), (17, 1400), (1, 170), (5, 171), (1, 1700), (9, 1600)]


@pytest.mark.parametrize("sigma", [13, 16, 20, 40])
@pytest.mark.parametrize("H,G,hd", [(4, 2, 64), (6, 1, 128), (8, 8, 64)], ids=str)
def test_the_largest_of_large_scores_alone_counts(torch, H, G, hd, sigma):
    """Queries and keys of about 2^sigma (by the projections' weights): the largest score of a row is
    alone, and the attention's result that position's value, exactly (rows whose two largest are
    nearer to each other than 150 in the exponent beside the scores' own fp32 error are left out:
    few)."""
    d = 256
    rng = np.random.default_rng(sigma)
    cfg = moe.make_attn_config(d, H, G, hd, n_layers=1, max_seq=2048, max_tokens=160)
    att = moe.AttnLayer(cfg)
    n_rot, nqkv = (H + G) * hd, (H + 2 * G) * hd
    w = rng.standard_normal((d, nqkv)) / np.sqrt(d)
    w[:, :n_rot] *= 2.0 ** sigma
    wqkv = torch.from_numpy(w).to(torch.bfloat16)
    wo = torch.from_numpy(rng.standard_normal((H * hd, d)) * 2.0 ** -7).to(torch.bfloat16)
    att.load_layer(0, torch.ones(d), wqkv, wo)
    K, V = att.cache_views(0)
    for t, s in ((K, 2.0 ** sigma), (V, 1.0)):             # positions that no call writes
        t.copy_(torch.from_numpy(rng.standard_normal(tuple(t.shape)) * s).to(torch.bfloat16).view(torch.int16))
    left_out = rows = 0
    for T, pos0 in CALLS:
        x = torch.from_numpy(rng.standard_normal((T, d))).to(torch.bfloat16).cuda()
        y = torch.empty_like(x)
        att.forward(0, x, y, pos0, T)
        torch.cuda.synchronize()
        got = att.intermediates(T)
        q, a = (f64(got[k]).reshape(T, H, hd) for k in ("q", "a"))
        kc, vc = (f64(t.cpu().numpy().view(np.uint16)) for t in (K, V))
        for j in range(H):
            Kj, Vj = kc[j // (H // G), :pos0 + T], vc[j // (H // G), :pos0 + T]
            score, mag = q[:, j] @ Kj.T, np.abs(q[:, j]) @ np.abs(Kj).T
            for i in range(T):
                sc, rows = score[i, :pos0 + i + 1], rows + 1
                top = int(sc.argmax())
                rest = np.delete(sc, top).max(initial=-np.inf)
                if sc[top] - rest <= 150 * np.sqrt(hd) + 2 * hd * ref.U32 * mag[i, :pos0 + i + 1].max():
                    left_out += 1
                    continue
                assert np.array_equal(a[i, j], Vj[top]), (T, pos0, i, j)
    assert left_out <= 0.02 * rows + 1
