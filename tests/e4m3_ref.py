"""fp64 references of routing policies and of products in e4m3 (include/moe.h), in numpy.

A value in e4m3 is a code times 2^e, e the least integer from -100 to 119 with amax <= 448 * 2^e over
its block; codes are rounded to nearest, ties to even.
"""
import numpy as np

import moe_inputs as mi

U32 = 2.0 ** -24


def gamma(n):
    """The relative error of an n-term fp32 sum of exact products, in any order."""
    return n * U32 / (1 - n * U32)


def bf16_bits(v):
    """fp32 / fp64 values as bf16 bits, rounded to nearest even (finite, in range)."""
    u = np.asarray(v, np.float32).view(np.uint32)
    return ((u.astype(np.uint64) + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def f64(bits):
    with np.errstate(invalid="ignore"):          # (NaN of all kinds among the bits)
        return mi.bf16_bits_to_f32(np.asarray(bits, np.uint16)).astype(np.float64)


def exponent(amax):
    """Brute force over all exponents."""
    amax = np.asarray(amax, np.float64)
    es = np.arange(-100, 120)
    fits = amax[..., None] <= 448.0 * np.exp2(es.astype(np.float64))
    return np.where(fits.any(-1), es[np.argmax(fits, axis=-1)], 119)


def grid(v):
    """fp64 values to the nearest e4m3 value (ties to even), at most 448; not finite: NaN."""
    v = np.asarray(v, np.float64)
    ok = np.isfinite(v)
    c = np.clip(np.where(ok, v, 0.0), -448.0, 448.0)
    _, x = np.frexp(c)
    step = np.exp2(np.maximum(x, -5).astype(np.float64) - 4)
    return np.where(ok, np.round(c / step) * step, np.nan)      # np.round: ties to even


def _amax(v, axis):
    return np.max(np.where(np.isfinite(v), np.abs(v), 0.0), axis=axis)


def rows(v):
    """(values on the grid, exponents [T, blocks], codes' values) of rows v [T, n]."""
    v = np.asarray(v, np.float64)
    T, n = v.shape
    nb = -(-n // 128)
    wide = np.zeros((T, nb * 128))
    wide[:, :n] = v
    wide = wide.reshape(T, nb, 128)
    e = exponent(_amax(wide, 2))
    codes = grid(wide * np.exp2(-e[..., None].astype(np.float64)))
    out = codes * np.exp2(e[..., None].astype(np.float64))
    return out.reshape(T, -1)[:, :n], e, codes.reshape(T, -1)[:, :n]


def weights(w):
    """Values on the grid of weights w [K, N] (fp64), 128 x 128 blocks."""
    K, N = w.shape
    out = np.empty((K, N))
    for k in range(0, K, 128):
        for n in range(0, N, 128):
            b = w[k:k + 128, n:n + 128]
            s = np.exp2(float(exponent(_amax(b, (0, 1)))))
            out[k:k + 128, n:n + 128] = grid(b / s) * s
    return out


def half_step(v, e):
    """Half a step of the grid at |v| with scale 2^e: 2^-4 of the value, and 2^-10 below the least
    normal code."""
    return np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10 * np.exp2(np.asarray(e, np.float64)))


def product_bound(x, w, terms):
    """|fp32 sum - exact| of x [T, K] by w [K, N], both exact."""
    return gamma(terms) * (np.abs(x) @ np.abs(w))


def choose(logits, k, score, balance=None, n_groups=1, top_groups=1, best=1, renormalize=True, scale=1.0):
    """ids [T, k] and weights [T, k] (fp64) of fp32 logits [T, E], expert by expert."""
    l = np.asarray(logits, np.float32).astype(np.float64)
    T, E = l.shape
    ids, ws = np.empty((T, k), np.int32), np.empty((T, k))
    with np.errstate(all="ignore"):
        for t in range(T):
            x = l[t]
            if score == 1:
                m = np.max(np.where(np.isnan(x), -np.inf, x))
                p = np.where(~np.isnan(x) & (m == -np.inf), 0.0, np.exp(x - m))
                z = p.sum()
                s = np.zeros(E) if z == 0 else p / z
            elif score == 2:
                s = 1.0 / (1.0 + np.exp(-x))
            else:
                s = x.copy()
            c = s + (np.asarray(balance, np.float64) if balance is not None else 0.0)
            c = np.where(np.isnan(c), -np.inf, c)
            lo = np.where(np.isnan(x), -np.inf, x)
            n = E // n_groups
            value = []
            for g in range(n_groups):
                top = np.sort(c[g * n:(g + 1) * n])[::-1][:best].sum()
                value.append(-np.inf if np.isnan(top) else top)
            kept = sorted(range(n_groups), key=lambda g: (-value[g], g))[:top_groups]
            experts = [e for e in range(E) if e // n in kept]
            S = sorted(experts, key=lambda e: (-c[e], -lo[e], e))[:k]
            w = s[S]
            if score == 0:
                m = np.max(np.where(np.isnan(w), -np.inf, w))
                w = np.where(~np.isnan(w) & (m == -np.inf), 0.0, np.exp(w - m))
            if renormalize or score == 0:
                z = w.sum()
                w = np.zeros(k) if z == 0 else w / z
            ids[t], ws[t] = S, w * scale
    return ids, ws


def permute(ids, first, n_local, E):
    """offsets [E + 1], pair_row [T, k], row_token: rows grouped by local expert, then token."""
    T, k = ids.shape
    flat = ids.reshape(-1)
    local = (flat >= first) & (flat < first + n_local)
    pairs = np.flatnonzero(local)
    order = pairs[np.argsort(flat[pairs], kind="stable")]
    pair_row = np.full(T * k, -1)
    pair_row[order] = np.arange(order.size)
    counts = np.bincount(flat[pairs], minlength=E)
    return np.concatenate([[0], np.cumsum(counts)]), pair_row.reshape(T, k), order // k
