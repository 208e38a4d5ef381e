"""Float64 oracle of the operators beside the projected update: gradient norm, AdamW with 32- or
8-bit moments, routing to experts. NumPy, written from the definitions; shares no code with the library."""
from __future__ import annotations

import math
from typing import Optional, Sequence

import numpy as np

BLOCK = 32


# ---------------------------------------------------------------- gradient norm

def grad_norm(grads: Sequence[np.ndarray], max_norm: float):
    norm = math.sqrt(sum(float(np.sum(np.square(g.astype(np.float64)))) for g in grads))
    return norm, (min(1.0, max_norm / (norm + 1e-6)) if math.isfinite(norm) else math.nan)


# ---------------------------------------------------------------- AdamW

def moments(g, m, v, beta1, beta2):
    return beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g


def adamw_param(p, m, v, t, lr, beta1, beta2, eps, decay):
    return p - lr * decay * p - lr * (m / (1 - beta1 ** t)) / (np.sqrt(v / (1 - beta2 ** t)) + eps)


def _mix(x):
    x = ((x ^ (x >> 16)) * 0x9E3779B1) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x6A09E667) & 0xFFFFFFFF
    return x ^ (x >> 16)


def random16(start: int, n: int, seed: int, tensor: int) -> np.ndarray:
    """The 16 random bits of elements start .. start + n - 1 of a tensor."""
    k0 = _mix((seed & 0xFFFFFFFF) ^ _mix((seed >> 32) ^ _mix(tensor)))
    k1 = _mix(k0 ^ 0xB7E15163)
    i = np.arange(start, start + n, dtype=np.uint64)
    c = i >> np.uint64(1)
    low = np.uint64(0xFFFFFFFF)
    x = (c + (c >> np.uint64(32)) * np.uint64(0xB7E15163) + np.uint64(k0)) & low
    x = (((x ^ (x >> np.uint64(16))) * np.uint64(0x9E3779B1)) & low) ^ np.uint64(k1)
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0x6A09E667)) & low
    x = x ^ (x >> np.uint64(16))
    return np.where(i & np.uint64(1), x >> np.uint64(16), x & np.uint64(0xFFFF)).astype(np.int64)


def _pad(x, fill=0):
    return np.concatenate([x, np.full(-x.size % BLOCK, fill, x.dtype)]).reshape(-1, BLOCK)


def block_exponents(x, least):
    """Biased exponent of each block's largest finite magnitude, one more over a significand of 1.75."""
    b = np.abs(_pad(x))
    top = np.where(np.isfinite(b), b, 0).max(axis=1)
    frac, e = np.frexp(top)             # top = frac 2^e, frac in [1/2, 1)
    e = np.where(top > 0, e + 126 + (frac > 0.875), 0)
    return np.clip(e, least, 254).astype(np.int64)


def e4m3_values() -> np.ndarray:
    """The 128 magnitudes of E4M3, by code; the last is no number."""
    c = np.arange(128)
    E, f = c >> 3, c & 7
    v = np.where(E > 0, (8 + f) * 2.0 ** (E - 10), f * 2.0 ** -9)
    v[127] = math.nan
    return v


def e5m3_values() -> np.ndarray:
    """The 256 values of the unsigned E5M3 codes in units of code 1; the last is no number."""
    c = np.arange(256)
    E, f = c >> 3, c & 7
    v = np.where(E > 0, (8 + f) * 2.0 ** (E - 1.0), f)
    v[255] = math.nan
    return v


def decode_m(codes, em):
    c = _pad(codes)
    v = e4m3_values()[c & 127] * np.where(c & 128, -1.0, 1.0)
    return (v * 2.0 ** (em[:, None] - 135.0)).reshape(-1)[:codes.size]


def decode_v(codes, ev):
    return (e5m3_values()[_pad(codes)] * 2.0 ** (ev[:, None] - 160.0)).reshape(-1)[:codes.size]


def encode_m(m, em):
    """Codes of the values nearest to m, the even code on ties."""
    x = _pad(m) * 2.0 ** (135.0 - em[:, None])
    grid = e4m3_values()[:127]
    a = np.minimum(np.abs(np.where(np.isfinite(x), x, 0)), 448.0)
    hi = np.clip(np.searchsorted(grid, a), 1, 126)
    lo = hi - 1
    dl, dh = a - grid[lo], grid[hi] - a
    c = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    c = np.where(np.isfinite(x), c | np.where(np.signbit(x), 128, 0), 127)
    return c.reshape(-1)[:m.size].astype(np.uint8)


def encode_v(v, ev, r16):
    """Codes of v, up with the probability (from r16 / 65536) that keeps the mean."""
    x = _pad(v) * 2.0 ** (160.0 - ev[:, None])
    r = _pad(r16)
    grid = e5m3_values()[:255]
    a = np.where(np.isfinite(x), x, 0)
    lo = np.clip(np.searchsorted(grid, a, side="right") - 1, 0, 254)
    unit = np.where(lo < 8, 1.0, 2.0 ** ((lo >> 3) - 1.0))
    c = lo + ((a - grid[lo]) / unit + r / 65536.0 >= 1)
    c = np.clip(np.maximum(c, a > 0), 0, 254)
    return np.where(np.isfinite(x), c, 255).reshape(-1)[:v.size].astype(np.uint8)


# ---------------------------------------------------------------- routing

def scores(logits, sigmoid: bool):
    with np.errstate(all="ignore"):
        if sigmoid:
            return 1 / (1 + np.exp(-logits))
        e = np.exp(logits - logits.max(axis=1, keepdims=True))
        return e / e.sum(axis=1, keepdims=True)


def selection(logits, sigmoid, bias=None, mask=None, groups=1, top_groups=1, group_best=1):
    """What experts are chosen by, -inf where one cannot be chosen."""
    c = scores(logits, sigmoid) + (0 if bias is None else bias)
    c = np.where(np.isnan(c), -np.inf, c)
    if mask is not None:
        c[~mask] = -np.inf
    if groups > 1:
        T, E = c.shape
        g = c.reshape(T, groups, E // groups)
        for t in range(T):
            value = []
            for q in range(groups):
                there = np.sort(g[t, q][g[t, q] > -np.inf])[::-1][:group_best]
                value.append(there.sum() if there.size else -np.inf)
            kept = sorted(range(groups), key=lambda q: (-value[q], q))[:top_groups]
            for q in range(groups):
                if q not in kept:
                    g[t, q] = -np.inf
        c = g.reshape(T, E)
    return c


def route(logits, k, sigmoid, bias=None, mask=None, groups=1, top_groups=1, group_best=1, renorm=False, scale=1.0):
    c = selection(logits, sigmoid, bias, mask, groups, top_groups, group_best)
    order = np.argsort(-c, axis=1, kind="stable")[:, :k]
    there = np.take_along_axis(c, order, 1) > -np.inf
    index = np.where(there, order, -1)
    return index, weights(logits, index, sigmoid, renorm, scale), c


def weights(logits, index, sigmoid, renorm, scale):
    there = index >= 0
    at = np.maximum(index, 0)
    if not renorm:
        return scale * np.where(there, np.take_along_axis(scores(logits, sigmoid), at, 1), 0)
    # the quotient of the scores, from their logarithms: it exists where all of them underflow
    x = np.take_along_axis(logits, at, 1)
    with np.errstate(all="ignore"):
        log = np.minimum(x, 0) - np.log1p(np.exp(-np.abs(x))) if sigmoid else x
        log = np.where(there, log, -np.inf)
        s = np.exp(log - np.maximum(log.max(axis=1, keepdims=True), np.finfo(np.float64).min))
    total = s.sum(axis=1, keepdims=True)
    return scale * np.divide(s, total, out=np.zeros_like(s), where=total > 0)


def balance(counts, bias, rate):
    return bias + rate * np.sign(counts.mean() - counts)
