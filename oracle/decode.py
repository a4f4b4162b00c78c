"""Decoding from a prepared prompt: scaled rotary tables, norms and rotation, the
8-bit cache, attention over it and eviction by accumulated attention weight.

Plain float64 restatements of the formulas (position interpolation and its
frequency-aware variants; RMS norm per head, Eq. 3 for the rotation; symmetric
8-bit codes with one scale for each block of tokens and head; softmax attention,
Eq. 2).  Test infrastructure only: the library's kernels never call this module.
"""
import numpy as np

from . import numerics

NONE, LINEAR, NTK, PARTS, INDEX = range(5)
HALF, INTERLEAVED = 0, 1
I8, E4M3 = 0, 1


def frequencies(theta, rot, kind=NONE, factor=1.0, original_len=1.0, low=1.0, high=32.0):
    i = np.arange(rot // 2, dtype=np.float64)
    if kind == NTK:
        theta = theta * factor ** (rot / (rot - 2.0))
    w = theta ** (-2.0 * i / rot)
    if kind == LINEAR:
        return w / factor
    turns = original_len * w / (2 * np.pi)
    if kind == PARTS:
        g = np.clip((turns - low) / (high - low), 0, 1)
        return g * w + (1 - g) * w / factor
    if kind == INDEX:
        at = lambda r: rot / 2 * np.log(original_len / (2 * np.pi * r)) / np.log(theta)  # noqa: E731
        i0, i1 = max(np.floor(at(high)), 0.0), min(np.ceil(at(low)), rot - 1.0)
        h = np.clip((i - i0) / max(i1 - i0, 0.001), 0, 1)
        return (1 - h) * w + h * w / factor
    return w


def table(w, pos, attn_factor=1.0):
    a = np.asarray(pos, np.float64)[:, None] * w
    return (np.cos(a) * attn_factor).astype(np.float32), (np.sin(a) * attn_factor).astype(np.float32)


def norm_rope(x, weight, eps, cos, sin, rot, pairing):
    """``x`` [T][H][d]; ``cos``/``sin`` [T][rot/2] (the tokens' rows).  Returns the result and,
    for tolerances, |y_a c| + |y_b s| of every output."""
    x = np.asarray(x, np.float64)
    y = x
    if weight is not None:
        y = x * np.asarray(weight, np.float64) / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps)
    out, size = y.copy(), np.abs(y)
    i = np.arange(rot // 2)
    a, b = (i, i + rot // 2) if pairing == HALF else (2 * i, 2 * i + 1)
    c, s = (np.asarray(t, np.float64)[:, None, :] for t in (cos, sin))
    out[..., a] = y[..., a] * c - y[..., b] * s
    out[..., b] = y[..., b] * c + y[..., a] * s
    size[..., a] = np.abs(y[..., a] * c) + np.abs(y[..., b] * s)
    size[..., b] = np.abs(y[..., b] * c) + np.abs(y[..., a] * s)
    return out, size


def e4m3_values():
    """The 256 e4m3 codes (sign, 4 exponent bits, 3 fraction bits, bias 7; 0x7F and 0xFF are NaN)."""
    c = np.arange(256)
    e, f = c >> 3 & 15, c & 7
    v = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


def quantise(x, code):
    """One block (any shape) -> (scale float32, codes uint8 of the same shape); e4m3 keeps the sign of a zero."""
    x = np.asarray(x, np.float64)
    if not np.isfinite(x).all():
        return np.float32(np.nan), np.zeros(x.shape, np.uint8)
    top = np.abs(x).max()
    if top == 0:
        return np.float32(0), np.zeros(x.shape, np.uint8)
    if code == I8:
        scale = np.float32(np.float32(top) / np.float32(127))
        c = np.clip(np.rint(x / np.float64(scale)), -127, 127)
        return scale, c.astype(np.int8).view(np.uint8)
    m, e = np.frexp(top)
    scale = np.ldexp(1.0, int(e) - (9 if m <= 0.875 else 8))
    v = e4m3_values()[:127]  # the numbers from 0 to 448
    t = np.abs(x) / scale
    hi = np.clip(np.searchsorted(v, t), 0, 126)
    lo = np.maximum(hi - 1, 0)
    d = (v[hi] - t) - (t - v[lo])  # ties: the even code
    c = np.where(d < 0, hi, np.where(d > 0, lo, np.where(hi % 2 == 0, hi, lo)))
    return np.float32(scale), (c + 128 * np.signbit(x)).astype(np.uint8)


def values(codes, scale, code):
    v = codes.view(np.int8).astype(np.float64) if code == I8 else e4m3_values()[codes]
    with np.errstate(invalid="ignore"):
        return v * np.float64(scale)


def attention(q, k, v, scale):
    """``q`` [n][d], the last n of the tokens; ``k``, ``v`` [T][d].  Returns out, lse, probabilities."""
    n, T = len(q), len(k)
    s = scale * (q.astype(np.float64) @ k.T)
    s[np.arange(T)[None, :] > (T - n + np.arange(n))[:, None]] = -np.inf
    top = s.max(1, initial=-np.inf)
    p = np.exp(s - np.where(np.isfinite(top), top, 0)[:, None])
    total = p.sum(1)
    with np.errstate(divide="ignore"):
        lse = np.where(total > 0, top + np.log(total), -np.inf)
    p = p / np.where(total > 0, total, 1)[:, None]
    return p @ v, lse, p


def evict(table, weights, nb, budget, first, recent):
    """One table row: (table, weights) after the eviction."""
    M = len(table)
    if nb <= budget:
        return table.copy(), weights.copy()
    middle = np.arange(first, nb - recent)
    w = weights[middle].astype(np.float64)
    w = np.where(np.isnan(w), -np.inf, w + 0.0)
    nan_last = np.isnan(weights[middle])  # below -infinity too
    order = np.lexsort((middle, nan_last, -w))
    keep = np.zeros(nb, bool)
    keep[:first] = keep[nb - recent:] = True
    keep[middle[order[:budget - first - recent]]] = True
    at = np.concatenate([np.nonzero(keep)[0], np.arange(nb, M), np.nonzero(~keep)[0]])
    w = weights[at].copy()
    w[M - (nb - budget):] = 0
    return table[at].copy(), w


def bf16(x):
    return numerics.bf16_round(np.asarray(x, np.float32))
