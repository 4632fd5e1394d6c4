"""The paged cache in plain fp64 (numpy), for the tests: e4m3 values, page scales, the rotation,
append and attention as include/attn.h defines them, and the bounds that the kernels are held to."""
import numpy as np

U32 = 2.0 ** -24       # half a step of fp32, relative
BF16 = 2.0 ** -8       # half a step of bf16, relative

# the value of every e4m3 code: 1 sign, 4 exponent (bias 7), 3 mantissa bits, 0x7f / 0xff NaN
_c = np.arange(256)
_e, _m = (_c >> 3) & 15, _c & 7
E4M3 = np.where(_e > 0, (1 + _m / 8.0) * 2.0 ** (_e - 7.0), _m / 8.0 * 2.0 ** -6.0) * np.where(_c < 128, 1.0, -1.0)
E4M3[[127, 255]] = np.nan


def e4m3_codes(v):
    """The code of the nearest e4m3 value (ties to the even code; past 448: 448) of v, NaN to 0x7f."""
    v = np.asarray(v, np.float64)
    pos = E4M3[:127]
    a = np.minimum(np.abs(np.where(np.isnan(v), 0.0, v)), 448.0)
    hi = np.clip(np.searchsorted(pos, a), 1, 126)
    lo = hi - 1
    mid = (pos[lo] + pos[hi]) / 2
    code = np.where(a < mid, lo, np.where(a > mid, hi, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(a == 0, 0, code)
    code = np.where(np.signbit(v), code | 128, code)
    return np.where(np.isnan(v), 127, code).astype(np.uint8)


def scale_exponent(amax):
    """The least e of -100 .. 119 with amax <= 448 * 2^e (119, if none is)."""
    e = -100
    while amax > 448.0 * 2.0 ** e and e < 119:
        e += 1
    return e


def rotate(x, pos, theta):
    """x [n, heads, hd] fp64 rotated by pos [n]."""
    hd = x.shape[-1]
    ang = np.asarray(pos, np.float64)[:, None] * theta ** (-2.0 * np.arange(hd // 2) / hd)
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = x[..., :hd // 2], x[..., hd // 2:]
    return np.concatenate([a * c - b * s, b * c + a * s], axis=-1)


def rotation_error(x):
    """Bound of the fp32 rotation's error: cos and sin within 2 2^-24 beside their angle (which,
    reduced in fp64, enters rounded to fp32: pi 2^-24), two products and a sum."""
    a, b = np.split(np.abs(x), 2, axis=-1)
    e = (np.pi + 2 * 2 + 3) * U32 * (a + b)
    return np.concatenate([e, e], axis=-1)


def bf16_round(v):
    """fp64 -> the nearest bf16, ties to even (normal range)."""
    v = np.asarray(v, np.float64)
    m, e = np.frexp(v)
    return np.ldexp(np.rint(m * 256.0), e - 8)


class Pool:
    """One layer's pages: bf16 values, or codes and scale exponents."""

    def __init__(self, n_pages, G, P, hd, e4m3):
        self.e4m3, self.P, self.G, self.hd = e4m3, P, G, hd
        shape = (n_pages, G, P, hd)
        self.k, self.v = np.zeros(shape), np.zeros(shape)            # values (bf16) ...
        self.kc, self.vc = np.zeros(shape, np.uint8), np.zeros(shape, np.uint8)   # ... or codes
        self.ks, self.vs = np.full(shape[:2], -100), np.full(shape[:2], -100)     # exponents

    def value(self, which, page, g):
        if not self.e4m3:
            return (self.k, self.v)[which][page, g]
        return E4M3[(self.kc, self.vc)[which][page, g]] * 2.0 ** (self.ks, self.vs)[which][page, g]

    def put(self, which, page, slot0, x):
        """x [n, G, hd] at slots slot0 .. of a page."""
        n = x.shape[0]
        if not self.e4m3:
            (self.k, self.v)[which][page, :, slot0:slot0 + n] = bf16_round(x).transpose(1, 0, 2)
            return
        codes, exps = (self.kc, self.vc)[which], (self.ks, self.vs)[which]
        for g in range(self.G):
            xg = x[:, g]
            ok = np.isfinite(xg)
            e = scale_exponent(np.abs(xg[ok]).max(initial=0.0))
            if slot0 > 0:
                old = exps[page, g]
                e = max(e, old)
                codes[page, g, :slot0] = e4m3_codes(E4M3[codes[page, g, :slot0]] * 2.0 ** float(old - e))
            codes[page, g, slot0:slot0 + n] = e4m3_codes(np.where(ok, xg * 2.0 ** float(-e), np.nan))
            exps[page, g] = e

    def append(self, k, v, pos0, table):
        """A sequence's new keys (rotated) and values [n, G, hd] at positions pos0 .."""
        n, at = k.shape[0], 0
        while at < n:
            p = pos0 + at
            m = min(n - at, self.P - p % self.P)
            for which, x in ((0, k), (1, v)):
                self.put(which, table[p // self.P], p % self.P, x[at:at + m])
            at += m


def attend(q, pool, pos0, table, scale=None):
    """q [n, H, hd] of a sequence's new tokens -> (o, bound pieces): o fp64, and per element
    sum w |v| and the weights' relative error from the scores' fp32 sums."""
    n, H, hd = q.shape
    G, P = pool.G, pool.P
    L = pos0 + n
    blocks = (L + P - 1) // P
    o, wv, ew = np.zeros((n, H, hd)), np.zeros((n, H, hd)), np.zeros((n, H, 1))
    mapped = np.repeat([t >= 0 for t in table[:blocks]], P)[:L]
    for g in range(G):
        K = np.concatenate([pool.value(0, t, g) if t >= 0 else np.zeros((P, hd)) for t in table[:blocks]])[:L]
        V = np.concatenate([pool.value(1, t, g) if t >= 0 else np.zeros((P, hd)) for t in table[:blocks]])[:L]
        for j in range(g * (H // G), (g + 1) * (H // G)):
            s = q[:, j] @ K.T / np.sqrt(hd)
            mag = np.abs(q[:, j]) @ np.abs(K).T / np.sqrt(hd)
            for t in range(n):
                see = mapped & (np.arange(L) <= pos0 + t)
                if not see.any():
                    continue
                st = s[t, see]
                w = np.exp(st - st.max())
                w /= w.sum()
                o[t, j] = w @ V[see]
                wv[t, j] = w @ np.abs(V[see])
                # scores: hd products summed in fp32, the scaled difference to the maximum in
                # fp32 (two roundings of numbers up to 2 |s|), the exponential's 2 ulp; both the
                # weight and the sum that divides it carry it
                es = hd * U32 * mag[t, see].max() + 4 * U32 * np.abs(st).max() + 4 * U32
                ew[t, j] = 2 * es
    return o, wv, ew


def attend_bound(o, wv, ew, n_pos, one_term):
    """The kernels' bound: the result's bf16 rounding; the weights' error; sums over n_pos
    positions in fp32 (of p v, of p, and over ranges); weights entering as one bf16 term (2^-8)
    or two (2^-16)."""
    weights = (2.0 ** -8 if one_term else 2.0 ** -16) * (1 + BF16)
    return (1 + BF16) * (ew + weights + 3 * (n_pos + 64) * U32) * wv + BF16 * np.abs(o) + 1e-30
