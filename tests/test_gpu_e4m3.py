"""Coding to e4m3, the product with e4m3 weights and MoE layers of MOE_E4M3, on the GPU against the
fp64 references of e4m3_ref (codes and scales bit for bit, products within the bounds of fp32 sums of
exact terms)."""
import numpy as np
import pytest

import e4m3_ref as ref
import moe_inputs as mi
import paper_2506_23635_amd as moe
from harness import gamma, read_intermediates

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def activations(T, n, seed=0):
    """Columns of different spread, some far out."""
    rng = np.random.default_rng(seed)
    spread = np.exp2(rng.uniform(-2, 2, n))
    spread[rng.random(n) < 0.01] *= 16
    return rng.standard_normal((T, n)) * spread


def dev16(torch, bits):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda()


# -------------------------------------------------------------- quantising --

def quantize(torch, x):
    T, n = x.shape
    codes = torch.full((T, n), 0x55, dtype=torch.uint8, device="cuda")
    scales = torch.full((T, -(-n // 128)), 0x55, dtype=torch.uint8, device="cuda")
    moe.quantize_e4m3(x, codes, scales)
    return codes.view(torch.float8_e4m3fn).double().cpu().numpy(), scales.cpu().numpy().astype(int)


def check_codes(got, v):
    _, e, codes = ref.rows(v)
    assert np.array_equal(got[1] - 127, e)
    assert np.array_equal(got[0], codes, equal_nan=True)


@pytest.mark.parametrize("T,n", [(1, 16), (1, 128), (3, 144), (5, 240), (17, 6144), (300, 400), (2, 10752), (1000, 128)])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("gap", [0, 24])
def test_quantize(torch, T, n, f32, gap):
    wide = activations(T, n + gap, seed=T + n).astype(np.float32)
    x = torch.from_numpy(wide).cuda() if f32 else dev16(torch, ref.bf16_bits(wide)).view(torch.bfloat16)
    v = wide.astype(np.float64) if f32 else ref.f64(ref.bf16_bits(wide))
    check_codes(quantize(torch, x[:, :n]), v[:, :n])


def test_quantize_edges(torch):
    """Zeros, values at a scale's border, the range's ends, values that are not finite."""
    v = np.zeros((12, 256), np.float32)
    v[1, 3], v[1, 200] = 448.0, np.nextafter(np.float32(448), np.float32(500))
    v[2, :4] = 3.4e38, -3.4e38, 2.0 ** 119 * 448, 1.0
    v[3, :4] = 2.0 ** -140, 2.0 ** -149, -2.0 ** -109, 2.0 ** -110
    v[4, :3] = NAN, 2.0, INF
    v[5] = NAN
    v[6, :128], v[6, 128:] = -INF, 1.0
    v[7] = np.arange(256) - 128.0
    v[8] = np.ldexp(1.0 + np.arange(256) / 256.0, 3)                  # every step of a binade and its ties
    v[9] = np.ldexp(np.arange(256) / 16.0, -9)
    v[9, 0] = 448.0                                                   # codes below the least normal one
    v[9, 128] = 448.0
    v[10] = -0.0
    v[11] = 1.75 * 2.0 ** 8 * np.where(np.arange(256) % 2, -1, 1)
    check_codes(quantize(torch, torch.from_numpy(v).cuda()), v.astype(np.float64))
    b = torch.from_numpy(v).cuda().to(torch.bfloat16)
    check_codes(quantize(torch, b), b.double().cpu().numpy())


def test_quantize_all_codes(torch):
    """Every bf16 whose block has a scale of 1."""
    bits = np.arange(1 << 16, dtype=np.uint16)
    v = ref.f64(bits)
    bits = bits[np.isfinite(v) & (np.abs(v) <= 448)]
    bits = np.resize(bits, -(-bits.size // 127) * 127).reshape(-1, 127)
    bits = np.concatenate([bits, np.full((len(bits), 1), 0x43E0, np.uint16)], axis=1)      # 448
    check_codes(quantize(torch, dev16(torch, bits).view(torch.bfloat16)), ref.f64(bits))


def test_quantize_leaves_the_rest(torch):
    x = torch.randn((4, 144), device="cuda")
    codes = torch.full((6 * 144,), 0x11, dtype=torch.uint8, device="cuda")
    scales = torch.full((6 * 2,), 0x22, dtype=torch.uint8, device="cuda")
    moe.quantize_e4m3(x, codes[144:5 * 144].view(4, 144), scales[2:10].view(4, 2))
    assert bool((codes[:144] == 0x11).all()) and bool((codes[5 * 144:] == 0x11).all())
    assert bool((scales[:2] == 0x22).all()) and bool((scales[10:] == 0x22).all())
    moe.quantize_e4m3(x[:0], codes[:0], scales[:0])


def test_quantize_arguments(torch):
    x = torch.zeros((4, 64), device="cuda")
    c, s = torch.empty((4, 64), dtype=torch.uint8, device="cuda"), torch.empty((4, 1), dtype=torch.uint8, device="cuda")
    for bad in ((x.double(), c, s), (x.cpu(), c, s), (x.t(), c, s), (x, c[:3], s), (x, c, s[:3]), (x, c.cpu(), s),
                (x, c.int(), s), (x[0], c, s), (x[:, :40], c, s), (x[:, 1:33], c, s), (None, c, s), (x, None, s)):
        with pytest.raises((moe.MoeError, AttributeError)):
            moe.quantize_e4m3(*bad)


# ----------------------------------------------------------------- product --

def linear(torch, T, n_in, n_out, seed=0, max_tokens=None, w=None):
    rng = np.random.default_rng(seed)
    w = ref.bf16_bits(rng.standard_normal((n_in, n_out)) / np.sqrt(n_in)) if w is None else w
    lin = moe.E4m3Linear(moe.make_linear_config(n_in, n_out, max_tokens=max_tokens or T))
    lin.load(dev16(torch, w))
    return lin, ref.weights(ref.f64(w))


def check_product(y, x, w, terms, bf16):
    """fp32 sums of exact products; bf16: half a step more, 2^-8 of the value."""
    y64, bound = x @ w, ref.product_bound(x, w, terms) + 1e-37
    if bf16:
        bound = bound + 2.0 ** -8 * (np.abs(y64) + bound)
    err = np.abs(y - y64)
    assert np.all(err <= bound), float((err / bound).max())


SHAPES = [(1, 16, 16), (1, 128, 256), (1, 1040, 1488), (2, 6144, 8192), (3, 144, 272), (15, 512, 48), (16, 2048, 512), (17, 128, 128),
          (31, 784, 1024), (33, 208, 272), (64, 3200, 512), (65, 1040, 1488), (128, 256, 16), (129, 640, 2064), (200, 6144, 1024),
          # 256 x 256 tiles: two stages of K, whole and partial tiles, an odd number of stages
          (2100, 16, 4096), (2304, 200 - 8, 4112), (1537, 320, 6000), (2050, 704, 4096), (40, 128, 32784), (300, 256, 32784),
          (255, 272, 784), (256, 512, 256), (257, 128, 1040), (300, 1152, 2304), (513, 144, 528), (700, 2048, 4096), (1025, 6144, 256)]


@pytest.mark.parametrize("T,n_in,n_out", SHAPES)
def test_linear(torch, T, n_in, n_out):
    lin, w = linear(torch, T, n_in, n_out, seed=T)
    bits = ref.bf16_bits(activations(T, n_in, seed=T))
    x, _, _ = ref.rows(ref.f64(bits))
    xt = dev16(torch, bits)
    for dt in (torch.float32, torch.bfloat16):
        y = torch.full((T + 2, n_out), 77.0, dtype=dt, device="cuda")
        lin.forward(xt, y[1:T + 1])
        assert bool((y[0] == 77).all()) and bool((y[T + 1] == 77).all())
        check_product(y[1:T + 1].double().cpu().numpy(), x, w, lin.cfg.in_dim, dt == torch.bfloat16)
        again = torch.empty_like(y[1:T + 1])
        lin.forward(xt, again)
        assert torch.equal(again, y[1:T + 1])                          # one order of sums
    lin.close()


def test_linear_fewer_rows_and_strides(torch):
    """One context for calls of all sizes; rows that are columns of a wider array."""
    lin, w = linear(torch, 1, 272, 400, max_tokens=300)
    bits = ref.bf16_bits(activations(300, 272 + 40, seed=3))
    wide = dev16(torch, bits).view(torch.bfloat16)
    x, _, _ = ref.rows(ref.f64(bits)[:, 8:280])
    for T in (300, 1, 16, 17, 140, 300):
        y = torch.empty((T, 400), device="cuda")
        lin.forward(wide[:T, 8:280], y)
        check_product(y.double().cpu().numpy(), x[:T], w, 272, False)
    lin.forward(wide[:0, 8:280], y)
    lin.close()


@pytest.mark.parametrize("T", [4, 40, 300])
def test_linear_values_that_are_not_finite(torch, T):
    """A row or a weight column with NaN or an infinity is NaN, all others are untouched by it."""
    w = ref.bf16_bits(np.random.default_rng(1).standard_normal((256, 272)))
    w[7, 30], w[9, 200] = 0x7FC0, 0x7F80
    lin, w64 = linear(torch, T, 256, 272, w=w)
    bits = ref.bf16_bits(activations(T, 256))
    bits[1, 3], bits[2, 200] = 0x7FC0, 0xFF80
    y = torch.empty((T, 272), device="cuda")
    lin.forward(dev16(torch, bits), y)
    y = y.cpu().numpy()
    bad = np.zeros(y.shape, bool)
    bad[[1, 2]] = True
    bad[:, [30, 200]] = True
    assert np.array_equal(np.isnan(y), bad)
    rows = [t for t in range(T) if t not in (1, 2)]
    cols = [n for n in range(272) if n not in (30, 200)]
    x, _, _ = ref.rows(ref.f64(bits[rows]))
    check_product(y[np.ix_(rows, cols)].astype(np.float64), x, w64[:, cols], 256, False)
    lin.close()


def test_linear_wide_range(torch):
    """Blocks whose scales are far apart, zero rows and zero blocks."""
    rng = np.random.default_rng(2)
    w = rng.standard_normal((512, 384))
    w[:128, :128] *= 2.0 ** 60
    w[128:256, 128:256] = 0.0
    w[256:384] *= 2.0 ** -60
    v = rng.standard_normal((40, 512))
    v[:, 128:256] *= 2.0 ** 40
    v[:, 256:384] *= 2.0 ** 50
    v[5] = 0.0
    wb, xb = ref.bf16_bits(w), ref.bf16_bits(v)
    for T in (3, 40):
        lin, w64 = linear(torch, T, 512, 384, w=wb)
        y = torch.empty((T, 384), device="cuda")
        lin.forward(dev16(torch, xb[:T]), y)
        check_product(y.double().cpu().numpy(), ref.rows(ref.f64(xb[:T]))[0], w64, 512, False)
        lin.close()


def test_weights_on_the_grid_stay(torch):
    """Weights that are codes times powers of two already keep their values through load."""
    rng = np.random.default_rng(4)
    codes = rng.choice(ref.grid(rng.uniform(-448, 448, 4096)), (256, 256))
    codes[::2] = ref.grid(rng.uniform(-2.0 ** -5, 2.0 ** -5, (128, 256)))
    w = codes * np.kron(np.exp2(rng.integers(-9, 9, (2, 2)).astype(float)), np.ones((128, 128)))
    bits = ref.bf16_bits(w)
    assert np.array_equal(ref.f64(bits), w)
    lin, w64 = linear(torch, 256, 256, 256, w=bits)
    assert np.array_equal(w64, w)
    eye = dev16(torch, ref.bf16_bits(np.eye(256)))
    y = torch.empty((256, 256), device="cuda")
    lin.forward(eye, y)
    assert np.array_equal(y.double().cpu().numpy(), w)
    lin.close()


@pytest.mark.parametrize("T", [1, 16, 60, 300])
def test_linear_captured(torch, T):
    """Replays on new rows, eager calls of the same context between them."""
    lin, w = linear(torch, T, 640, 528)
    x = torch.empty((T, 640), dtype=torch.bfloat16, device="cuda").normal_()
    y, eager = torch.empty((T, 528), device="cuda"), torch.empty((T, 528), device="cuda")
    lin.forward(x, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lin.forward(x, y)
    for i in range(4):
        x.normal_(generator=torch.Generator(device="cuda").manual_seed(i))
        y.zero_()
        graph.replay()
        lin.forward(x, eager)
        torch.cuda.synchronize()
        assert torch.equal(y, eager)
        check_product(y.double().cpu().numpy(), ref.rows(x.double().cpu().numpy())[0], w, 640, False)
    lin.close()


@pytest.mark.parametrize("n_in,n_out,T", [(6144, 256, 100), (2048, 512, 300), (4096, 1040, 64), (8192, 48, 17)])
def test_linear_in_ranges_stays_in_its_workspace(torch, n_in, n_out, T):
    """Products whose reduction is cut in ranges: the sums' space ends the workspace, rows past T and
    bytes past the workspace stay as they were, for the largest call and for smaller ones."""
    cfg = moe.make_linear_config(n_in, n_out, max_tokens=T)
    n = moe.moe_linear_workspace_bytes(cfg)
    ws = torch.full((n + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    lin = moe.E4m3Linear(cfg, workspace=ws)
    w = ref.bf16_bits(np.random.default_rng(3).standard_normal((n_in, n_out)) / np.sqrt(n_in))
    lin.load(dev16(torch, w))
    bits = ref.bf16_bits(activations(T, n_in))
    x, _, _ = ref.rows(ref.f64(bits))
    for rows in (T, T - 3, 17):
        y = torch.full((rows + 1, n_out), 7.0, dtype=torch.bfloat16, device="cuda")
        lin.forward(dev16(torch, bits[:rows]), y[:-1])
        check_product(y[:-1].double().cpu().numpy(), x[:rows], ref.weights(ref.f64(w)), n_in + 4, True)
        assert bool((y[-1] == 7).all())
    assert bool((ws[n:] == 0x5A).all())
    lin.close()


def test_layer_stays_in_its_workspace(torch):
    for T, share in ((16, (0, 4)), (40, (1, 2)), (300, (0, 4))):
        cfg = moe.make_config(512, 384, 4, 2, expert_begin=share[0], n_local_experts=share[1], max_tokens=T, flags=moe.MOE_E4M3)
        n, m = moe.moe_workspace_bytes(cfg), moe.moe_weight_bytes(cfg)
        ws = torch.full((n + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
        arena = torch.full((m + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
        layer = moe.MoeLayer(cfg, arena=arena, workspace=ws)
        layer.load_router(0, torch.randn((512, 4)))
        for e in range(share[0], share[0] + share[1]):
            layer.load_expert(0, e, *(torch.randn(s, device="cuda").to(torch.bfloat16) for s in ((512, 384), (512, 384), (384, 512))))
        for rows in (T, min(T, 17), 3, 1):
            x = torch.randn((rows, 512), device="cuda").to(torch.bfloat16)
            layer.forward(0, x, torch.empty_like(x))
        torch.cuda.synchronize()
        assert bool((ws[n:] == 0x5A).all()) and bool((arena[m:] == 0x5A).all())
        layer.close()


def test_linear_on_another_stream(torch):
    lin, w = linear(torch, 50, 256, 272)
    x = torch.randn((50, 256), device="cuda").to(torch.bfloat16)
    y = torch.empty((50, 272), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lin.forward(x, y)
    side.synchronize()
    check_product(y.double().cpu().numpy(), ref.rows(x.double().cpu().numpy())[0], w, 256, False)
    lin.close()


def test_linear_arguments(torch):
    lin, _ = linear(torch, 4, 128, 256)
    x = torch.zeros((4, 128), dtype=torch.bfloat16, device="cuda")
    y = torch.zeros((4, 256), device="cuda")
    for bad in ((x.float(), y), (x.cpu(), y), (x, y.cpu()), (x, y.double()), (x, y[:3]), (x[:, :64], y), (x.t(), y), (x[0], y),
                (None, y), (x, None), (torch.cat([x, x]), torch.cat([y, y])), (x, y.t())):
        with pytest.raises(moe.MoeError):
            lin.forward(*bad)
    buf = torch.zeros(4 * 256, device="cuda")
    with pytest.raises(moe.MoeError):                                  # y over x
        lin.forward(buf.view(torch.bfloat16)[:512].view(4, 128), buf.view(4, 256))
    odd = torch.zeros(4 * 136 + 8, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(moe.MoeError):                                  # rows that are not 16-byte aligned
        lin.forward(odd[:4 * 132].view(4, 132)[:, :128], y)
    with pytest.raises(moe.MoeError):
        lin.forward(odd[1:513].view(4, 128), y)
    for bad in (torch.zeros((128, 255), dtype=torch.bfloat16, device="cuda"), torch.zeros((256, 128), dtype=torch.bfloat16, device="cuda"),
                torch.zeros((128, 256), device="cuda"), torch.zeros((128, 256), dtype=torch.bfloat16)):
        with pytest.raises(moe.MoeError):
            lin.load(bad)
    lin.close()


# ------------------------------------------------------------------ layers --

def expert_weights(d, f, E, seed):
    rng = np.random.default_rng(seed)
    gate, up = (ref.bf16_bits(rng.standard_normal((E, d, f)) * 1.5 / np.sqrt(d)) for _ in range(2))
    return gate, up, ref.bf16_bits(rng.standard_normal((E, f, d)) / np.sqrt(f))


class Layer:
    """A loaded MOE_E4M3 layer and its weights on the grid, fp64."""

    def __init__(self, torch, d, f, E, k, T, first=0, local=0, flags=0, seed=0, host=False, policy=None):
        local = local or E
        self.torch, self.first, self.local, self.E, self.k, self.d, self.f = torch, first, local, E, k, d, f
        self.layer = moe.MoeLayer(moe.make_config(d, f, E, k, expert_begin=first, n_local_experts=local, max_tokens=T,
                                                  flags=moe.MOE_E4M3 | flags))
        rng = np.random.default_rng(seed + 1)
        self.layer.load_router(0, torch.from_numpy(rng.standard_normal((d, E)).astype(np.float32) * 0.05),
                               torch.from_numpy(rng.standard_normal(E).astype(np.float32) * 0.5))
        bits = expert_weights(d, f, E, seed)
        for e in range(first, first + local):
            t = [torch.from_numpy(b[e].view(np.int16)) for b in bits]
            self.layer.load_expert(0, e, *(t if host else [a.cuda() for a in t]))
        self.w = [[ref.weights(ref.f64(b[e])) if first <= e < first + local else None for e in range(E)] for b in bits]
        if policy:
            self.layer.set_policy(0, moe.make_policy(**policy))

    def check(self, bits, y, f32=False, routing=None):
        """Every stage of the last forward, y fp64 [T, d], against fp64 from the stage before:
        H   a value of the grid within half a step and the fp32 bound of silu(G) U (the products'
            gamma_d, 8 roundings of the logistic) of the exact value;
        O   gamma_f sum |h| |w2|;
        y   gamma_k sum |w o|, and half a bf16 step."""
        torch, layer = self.torch, self.layer
        T, d, f, k = len(bits), self.d, self.f, self.k
        rt = routing
        n = int(rt["offsets"][-1])
        H, O = read_intermediates(torch, layer, n)
        H = ref.f64(H)
        x, _, _ = ref.rows(ref.f64(bits))
        same, near = 0, 0
        for e in range(self.first, self.first + self.local):
            r0, r1 = int(rt["offsets"][e]), int(rt["offsets"][e + 1])
            if r0 == r1:
                continue
            a = x[rt["row_token"][r0:r1]]
            gw, uw, dw = (w[e] for w in self.w)
            g, u = a @ gw, a @ uw
            bg, bu = ref.product_bound(a, gw, d), ref.product_bound(a, uw, d)
            sig = 1.0 / (1.0 + np.exp(-g))
            silu, slope = g * sig, np.abs(sig * (1.0 + g * (1.0 - sig)))
            h = silu * u
            # first order, and the products of the errors (|silu'| <= 1.1, |silu''| <= 1/2)
            bh = (slope + bg) * bg * np.abs(u) + np.abs(silu) * bu + 1.2 * bg * bu + 8 * ref.U32 * np.abs(h)
            hq, eh, _ = ref.rows(h)
            # a block whose largest value is near a border may take the next scale: its smallest
            # steps are twice as wide then
            step = ref.half_step(np.abs(h) + bh, np.repeat(eh, 128, axis=1)[:, :f] + 1)
            assert np.all(np.abs(H[r0:r1] - h) <= step + bh), e
            same += int((H[r0:r1] == hq).sum())
            near += H[r0:r1].size
            again, _, _ = ref.rows(H[r0:r1])
            assert np.array_equal(again, H[r0:r1])                     # on the grid
            ob = gamma(f) * (np.abs(H[r0:r1]) @ np.abs(dw)) + 1e-37
            assert np.all(np.abs(O[r0:r1] - H[r0:r1] @ dw) <= ob), e
        # roundings differ only where an exact value is within its fp32 error of a border: a share of
        # the elements far below one in a hundred
        assert near == 0 or same / near > 0.99
        want, mag = np.zeros((T, d)), np.zeros((T, d))
        for j in range(k):
            r = rt["pair_row"][:, j]
            o = np.where((r >= 0)[:, None], O[np.maximum(r, 0)] if n else 0.0, 0.0) * rt["w"][:, j:j + 1].astype(np.float64)
            want += o
            mag += np.abs(o)
        bound = gamma(k + 1) * mag + 1e-37
        if not f32:
            bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
        assert np.all(np.abs(y - want) <= bound)
        return want

    def run(self, bits, f32=False):
        torch, layer = self.torch, self.layer
        x = dev16(torch, bits)
        y = torch.full((len(bits) + 1, self.d), 55.0, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
        routing = layer.route(0, x)
        layer.forward(0, x, y[:-1], routing=routing)
        assert bool((y[-1] == 55).all())
        self.check(bits, y[:-1].double().cpu().numpy(), f32, layer.routing_tensors(routing))
        return y[:-1]


@pytest.mark.parametrize("T", [1, 2, 16, 17, 40, 150, 300, 700])
@pytest.mark.parametrize("d,f,E,k", [(256, 128, 4, 2), (512, 384, 8, 2), (768, 640, 8, 4)])
def test_layer(torch, T, d, f, E, k):
    L = Layer(torch, d, f, E, k, T, seed=T)
    L.run(ref.bf16_bits(activations(T, d, seed=T)))
    L.layer.close()


@pytest.mark.parametrize("T", [17, 70, 130, 260, 400, 900])
@pytest.mark.parametrize("d,f,E,k", [(256, 128, 4, 2), (512, 384, 8, 2), (768, 640, 3, 1), (256, 896, 2, 2)])
def test_layer_on_the_large_tiles(torch, T, d, f, E, k):
    """The 256 x 256 tiles, which smaller calls take while a timeline is recorded: tiles of few, half
    of and all rows, one to many rounds of their rings, and the same bits as the small tiles."""
    L = Layer(torch, d, f, E, k, T, seed=T)
    bits = ref.bf16_bits(activations(T, d, seed=T))
    small = L.run(bits).clone()
    stamps = torch.zeros((4, 8), dtype=torch.int64, device="cuda")
    moe.moe_profile_gemm_timeline(L.layer.ctx, stamps.data_ptr(), None, 4)
    large = L.run(bits).clone()
    torch.cuda.synchronize()
    assert int(stamps.abs().sum()) > 0
    moe.moe_profile_gemm_timeline(L.layer.ctx, None, None, 0)
    assert torch.equal(small, large)
    L.layer.close()


def test_layer_that_takes_the_large_tiles(torch):
    """Enough rows and tiles that the layer chooses them itself."""
    L = Layer(torch, 256, 2048, 8, 2, 3300, seed=5)
    L.run(ref.bf16_bits(activations(3300, 256, seed=5)))
    L.layer.close()


def test_layer_of_more_rows_than_the_small_tiles_take(torch):
    """640 tiles of 256 x 256 for gate/up, 1050 rows to an expert."""
    L = Layer(torch, 256, 2048, 8, 2, 4200, seed=6)
    L.run(ref.bf16_bits(activations(4200, 256, seed=6)))
    L.layer.close()


@pytest.mark.parametrize("T,d,f,E,k", [(1600, 2048, 128, 8, 2), (601, 1536, 384, 32, 4), (3000, 512, 256, 16, 4),
                                       (2501, 1024, 128, 16, 2)])
def test_down_on_tiles_of_two_feature_blocks(torch, T, d, f, E, k):
    """384 and more tiles of 256 features and 64 rows, full and partial ones, two and more stages of
    K: against the oracle, and the same bits as the 256 x 256 tiles."""
    L = Layer(torch, d, f, E, k, T, seed=T)
    bits = ref.bf16_bits(activations(T, d, seed=T))
    small = L.run(bits).clone()
    stamps = torch.zeros((4, 8), dtype=torch.int64, device="cuda")
    moe.moe_profile_gemm_timeline(L.layer.ctx, None, stamps.data_ptr(), 4)
    large = L.run(bits).clone()
    torch.cuda.synchronize()
    assert int(stamps.abs().sum()) > 0
    moe.moe_profile_gemm_timeline(L.layer.ctx, None, None, 0)
    assert torch.equal(small, large)
    L.layer.close()


@pytest.mark.parametrize("T", [3, 16, 50, 600])
@pytest.mark.parametrize("first,local", [(0, 2), (5, 3), (7, 1)])
def test_a_share(torch, T, first, local):
    L = Layer(torch, 512, 256, 8, 2, T, first, local, flags=moe.MOE_PARTIAL_F32,
              policy=dict(score=moe.SCORE_SIGMOID, n_groups=4, top_groups=2, group_best=2, scale=2.5))
    L.run(ref.bf16_bits(activations(T, 512, seed=T)), f32=True)
    L.layer.close()


def test_one_expert_takes_all(torch):
    """Every token to the same experts: long and empty groups."""
    for T in (9, 100, 400):
        L = Layer(torch, 256, 384, 8, 2, T)
        bias = torch.full((8,), -1e4)
        bias[2], bias[7] = 1e4, 1.1e4
        L.layer.load_router(0, torch.zeros((256, 8)), bias)
        L.run(ref.bf16_bits(activations(T, 256, seed=T)))
        L.layer.close()


def test_host_and_device_weights_are_the_same(torch):
    a, b = (Layer(torch, 256, 384, 3, 2, 8, host=h) for h in (False, True))
    torch.cuda.synchronize()
    assert torch.equal(a.layer.arena, b.layer.arena) or all(
        torch.equal(p, q) for p, q in ((a.run(bits), b.run(bits)) for bits in (ref.bf16_bits(activations(8, 256)),)))
    wild = [ref.bf16_bits(np.random.default_rng(9).standard_normal(s) * 2.0 ** np.random.default_rng(8).integers(-130, 120, s))
            for s in ((256, 384), (256, 384), (384, 256))]
    for w in wild:
        w.reshape(-1)[::997] = 0x7FC0
        w.reshape(-1)[5::1201] = 0xFF80
    t = [torch.from_numpy(w.view(np.int16)) for w in wild]
    off = (256 * 3 * 4 + 255) // 256 * 256 + 256                       # the router, then the first expert
    codes, scales = 3 * 256 * 384, 2 * 3 * 4 + 2 * 4
    a.layer.load_expert(0, 0, *[v.cuda() for v in t])
    b.layer.load_expert(0, 0, *t)
    torch.cuda.synchronize()
    # NaN has two codes, either may stand for what is not finite
    x, y = (l.layer.arena[off:off + codes].cpu().numpy() for l in (a, b))
    nan = x & 0x7F == 0x7F
    assert nan.any() and np.array_equal(nan, y & 0x7F == 0x7F) and np.array_equal(x[~nan], y[~nan])
    x, y = (l.layer.arena[off + codes:off + codes + scales] for l in (a, b))
    assert torch.equal(x, y)
    a.layer.close()
    b.layer.close()


@pytest.mark.parametrize("T", [1, 16, 40, 300])
def test_all_forwards_agree(torch, T):
    """forward, static, residual and stack of one layer, and replays of a captured forward."""
    L = Layer(torch, 256, 384, 8, 2, 300, policy=dict(score=moe.SCORE_SOFTMAX, scale=1.5))
    layer = L.layer
    x = dev16(torch, ref.bf16_bits(activations(T, 256)))
    y, s, r = torch.empty_like(x), torch.empty_like(x), x.clone()
    layer.forward(0, x, y)
    layer.forward_static(0, x, s)
    assert torch.equal(y, s)
    layer.forward_residual(0, x, r)
    want = (x.view(torch.bfloat16).double() + y.view(torch.bfloat16).double()).to(torch.bfloat16)
    assert torch.equal(r.view(torch.bfloat16), want)
    stack = x.clone()
    layer.forward_stack(stack)
    assert torch.equal(stack, r)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward(0, x, y)
    for i in range(3):
        x.copy_(dev16(torch, ref.bf16_bits(activations(T, 256, seed=i + 10))))
        y.zero_()
        graph.replay()
        layer.forward_static(0, x, s)
        torch.cuda.synchronize()
        assert torch.equal(y, s)
    layer.close()


def test_rows_that_are_not_finite_stay_alone(torch):
    for T in (6, 60, 400):
        L = Layer(torch, 256, 256, 4, 2, T)
        bits = ref.bf16_bits(activations(T, 256, seed=T))
        clean = L.run(bits).clone()
        bits[2, 5] = 0x7F80
        x = dev16(torch, bits)
        logits = torch.from_numpy(np.random.default_rng(T).standard_normal((T, 4)).astype(np.float32)).cuda()
        routing = L.layer.route(0, None, logits_in=logits)
        y = torch.empty_like(clean)
        L.layer.forward(0, x, y, routing=routing)
        assert bool(torch.isnan(y[2]).all()) and not bool(torch.isnan(torch.cat([y[:2], y[3:]])).any())
        L.layer.close()


def test_layer_then_product(torch):
    """A decoder layer's end as it is used: policy, experts in e4m3 into the residual, then a product
    of the result in e4m3, against the same steps from the fp64 references."""
    for T in (1, 5, 70):
        L = Layer(torch, 512, 384, 8, 2, T, policy=dict(score=moe.SCORE_SIGMOID, n_groups=2, top_groups=1, group_best=2, scale=2.0))
        lin, w = linear(torch, T, 512, 1040)
        bits = ref.bf16_bits(activations(T, 512, seed=T))
        x = dev16(torch, bits)
        routing = L.layer.route(0, x)
        y = torch.empty_like(x).view(torch.bfloat16)
        L.layer.forward(0, x, y, routing=routing)
        L.check(bits, y.double().cpu().numpy(), routing=L.layer.routing_tensors(routing))
        r = x.clone()
        L.layer.forward_residual(0, x, r)
        out = torch.empty((T, 1040), device="cuda")
        lin.forward(r, out)
        res = (x.view(torch.bfloat16).double() + y.double()).to(torch.bfloat16)
        assert torch.equal(r.view(torch.bfloat16), res)
        check_product(out.double().cpu().numpy(), ref.rows(res.double().cpu().numpy())[0], w, 512, False)
        lin.close()
        L.layer.close()
