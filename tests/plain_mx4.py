"""Microscaled 4-bit floats and scores of given tokens, in 64 bits on the host, from their formulas."""
import numpy as np
import torch

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BORDERS = (VALUES[1:] + VALUES[:-1]) / 2
NAN = 255


def quantize(x):
    """x [rows, cols] -> (codes [rows, 32 * blocks] 0 to 15, scale bytes [rows, blocks])."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    n = (cols + 31) // 32
    v = np.zeros((rows, n * 32))
    v[:, :cols] = x
    v = v.reshape(rows, n, 32)
    bad = ~np.isfinite(v).all(axis=2)
    v = np.where(bad[:, :, None], 0.0, v)
    peak = np.abs(v).max(axis=2)
    e = np.maximum(np.frexp(peak)[1] - 1 - 2 + 127, 0)
    e = np.where(peak == 0, 127, e)
    u = np.abs(np.ldexp(v, (127 - e)[:, :, None]))
    below = np.searchsorted(BORDERS, u, side="left")    # a value on a border counts as below it
    on = (below < 7) & (u == BORDERS[np.minimum(below, 6)])
    code = np.where(on & (below % 2 == 1), below + 1, below)
    code = code + 8 * (np.signbit(v) & ~bad[:, :, None])
    return code.reshape(rows, n * 32).astype(np.uint8), np.where(bad, NAN, e).astype(np.uint8)


def values(code, scale):
    """Codes [rows, 32 * blocks] and scale bytes [rows, blocks] -> float64 [rows, 32 * blocks]."""
    v = np.where(code & 8, -1.0, 1.0) * VALUES[code & 7]
    s = np.where(scale == NAN, np.nan, np.ldexp(1.0, scale.astype(np.int64) - 127))
    return (v.reshape(code.shape[0], -1, 32) * s[:, :, None]).reshape(code.shape[0], -1)


def split(packed):
    """Bytes -> codes, the low bits first."""
    return np.stack([packed & 15, packed >> 4], axis=2).reshape(packed.shape[0], -1)


def join(code):
    return (code[:, 0::2] | (code[:, 1::2] << 4)).astype(np.uint8)


def sum_tolerance(K, magnitude):
    """What a sum of K products may be off by.  An instruction cuts its 128 products and the sum so far at 2^-27 of the largest magnitude
    among them, each by less than that, and rounds once (2^-24): 129 * 2^-27 + 2^-24 < 2^-19 of a magnitude that the sum of all of them
    bounds.  There are 2 ceil(K / 256) instructions; up to 8 partial sums of these are joined by fp32 additions (2^-24 each)."""
    return (2 * ((K + 255) // 256) * 2.0 ** -19 + 8 * 2.0 ** -24) * magnitude


def scores(logits, token, n_top):
    """logits [rows, V] (any float array), token [rows] or None -> (logp, entropy, tokens, values)."""
    x = np.asarray(logits, np.float64)
    rows, V = x.shape
    with np.errstate(all="ignore"):
        bad = (np.isnan(x) | (x == np.inf)).any(axis=1)
        none = (x == -np.inf).all(axis=1)
        top = np.where(none, 0.0, x.max(axis=1))[:, None]
        # (the two apart: next to the largest numbers of fp32 the logarithm would vanish)
        lp = (x - top) - np.log(np.exp(x - top).sum(axis=1))[:, None]
        p = np.exp(lp)
        entropy = -np.where(p > 0, p * lp, 0.0).sum(axis=1)
    entropy = np.where(bad, np.nan, np.where(none, 0.0, entropy))
    lp = np.where(bad[:, None], np.nan, np.where(none[:, None], -np.inf, lp))
    logp = None
    if token is not None:
        t = np.asarray(token)
        inside = np.clip(t, 0, V - 1)
        logp = np.where(t < 0, 0.0, np.where(t >= V, np.nan, lp[np.arange(rows), inside]))
    at = np.argsort(-np.where(bad[:, None], -np.inf, x), axis=1, kind="stable")[:, :n_top]
    found = np.take_along_axis(np.where(bad[:, None], -np.inf, lp), at, axis=1)
    tokens = np.where(found == -np.inf, -1, at)
    pad = ((0, 0), (0, n_top - at.shape[1]))
    return logp, entropy, np.pad(tokens, pad, constant_values=-1), np.pad(found, pad, constant_values=-np.inf)


def scores_tolerance(V, dtype=torch.float32):
    """What lse and the entropy may be off by, in steps of 2^-24.  x log2(e) - r, with r at most 12 binary digits (8.4 natural units)
    below the largest, is rounded once, and so is the constant: 1.25 of |x - r|, on average over the probabilities at most ln V + 8.4
    (the mean of lse - x is the entropy).  An exponential has a step of its own (2), 32 of them are added in fp32 (31; 7 for V <= 512),
    then the lanes of a wave (1 + 6), and three joins cost an exponential each (6): less than 50 + 4 ln V in all.  The entropy has the
    mean of x - m, at most ln V + 8 in magnitude, with twice that, and lse."""
    lse = (25 + 2 * np.log(V)) * 2.0 ** -23
    return lse, 2 * (9 + np.log(V)) * lse
