"""The codes and scales that moe_load_expert leaves in the arena, from weights on the GPU and in host
memory: byte for byte the same, and the reference's values where the packed layout has them."""
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


def quads(K):
    return -(-K // 512)


def places(K, N, mul, add):
    """Byte of element (k, n): 16-row x 64-K tiles of 1 KiB, four row tiles side by side; in a tile 256 g +
    16 r for granule (g, r), which holds K 8 g .. 8 g + 7 and 32 + 8 g .. 32 + 8 g + 7 of row r."""
    k, n = np.meshgrid(np.arange(K), np.arange(N), indexing="ij")
    rt, q = n // 16 * mul + add, k % 64
    tile = (rt // 4 * (K // 64) + k // 64) * 4 + rt % 4
    return tile * 1024 + q % 32 // 8 * 256 + n % 16 * 16 + q // 32 * 8 + q % 8


def code_values():
    c = np.arange(256)
    e, m = c >> 3 & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * 2.0 ** (e - 7.0))
    v[(c & 0x7F) == 0x7F] = np.nan
    return np.where(c & 0x80, -v, v)


def weights(d, f, spread, seed):
    """Magnitudes that differ from block to block, and within one, by up to 2^spread."""
    rng = np.random.default_rng(seed)
    out = []
    for K, N in ((d, f), (d, f), (f, d)):
        w = rng.standard_normal((K, N)) * np.exp2(rng.integers(-spread, spread + 1, (K, N)))
        w *= np.kron(np.exp2(rng.integers(-20, 21, (K // 128, N // 128))), np.ones((128, 128)))
        out.append(ref.bf16_bits(w))
    return out


@pytest.mark.parametrize("d,f", [(256, 128), (256, 384), (768, 640), (2304, 256)])
@pytest.mark.parametrize("spread", [0, 12])
def test_arena(torch, d, f, spread):
    bits = weights(d, f, spread, d + f)
    E, arenas = 3, []
    for host in (False, True):
        layer = moe.MoeLayer(moe.make_config(d, f, E, 2, flags=moe.MOE_E4M3))
        layer.arena.fill_(0xA5)
        t = [torch.from_numpy(b.view(np.int16)) for b in bits]
        layer.load_expert(0, 1, *(t if host else [v.cuda() for v in t]))
        torch.cuda.synchronize()
        arenas.append(layer.arena.cpu().numpy())
        layer.close()
    codes, up = 3 * d * f, f // 128 * quads(d) * 4
    written = codes + 2 * up + d // 128 * quads(f) * 4
    first, expert = (d * E * 4 + 255) // 256 * 256 + 256, -(-written // 256) * 256
    at = first + expert
    a, b = (v[at:at + written] for v in arenas)
    assert np.array_equal(a, b)
    for v in arenas:                                                   # the experts beside it
        assert np.all(v[first:at] == 0xA5) and np.all(v[at + expert:at + 2 * expert] == 0xA5)
    table = code_values()
    parts = [(bits[0], d, f, 0, 2, 0, codes), (bits[1], d, f, 0, 2, 1, codes + up), (bits[2], f, d, 2 * d * f, 1, 0, codes + 2 * up)]
    for w, K, N, base, mul, add, s0 in parts:
        s = a[s0:s0 + N // 128 * quads(K) * 4].reshape(N // 128, -1)[:, :K // 128].astype(int) - 127
        got = table[a[base + places(K, N, mul, add)]] * np.kron(np.exp2(s.T.astype(float)), np.ones((128, 128)))
        assert np.array_equal(got, ref.weights(ref.f64(w)))
