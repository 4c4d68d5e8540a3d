"""The operators of 8-bit layers with a scale for each token, of the selection over large vocabularies and of the reordering
of states, in 64 bits on the host, from their formulas."""
import numpy as np
import torch

HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def token_codes(u, root=None):
    """u [rows, cols] float64 (exact products) -> codes int8 and scale float64; root: what divides a row's range."""
    u = np.asarray(u, np.float64)
    with np.errstate(all="ignore"):
        peak = np.abs(u).max(axis=1)
        bad = ~np.isfinite(u).all(axis=1)
        safe = np.where((peak > 0) & ~bad, peak, 1.0)
        codes = np.where(bad[:, None], 0.0, np.rint((127.0 * np.where(bad[:, None], 0.0, u)) / safe[:, None]))
        scale = peak / 127.0 if root is None else peak / root / 127.0
    scale = np.where(bad, np.nan, np.where(peak == 0, 1.0, scale))
    return codes.astype(np.int8), scale


def rms_norm_quant(x, weight, eps, residual=None):
    """Tensors on the host -> (codes, scale, sum)."""
    h = x
    if residual is not None:
        h = (x.float() + residual.float()).to(x.dtype)   # the sum of two values of a type is rounded once to fp32, once to it
    h64 = h.double().numpy()
    w64 = np.ones(x.shape[1]) if weight is None else weight.double().numpy()
    with np.errstate(all="ignore"):
        u = h64 * w64
        u = np.where(np.isfinite(h64), u, np.nan)        # (a weight of 0 does not make a value finite)
        root = np.sqrt((h64 * h64).mean(axis=1) + float(np.float32(eps)))
    codes, scale = token_codes(u, root)
    return codes, scale, h


def linear(codes, scale, w_codes, w_scale, bias):
    """(y float64, magnitude of the product) for codes [M, K], w_codes [N, K]."""
    acc = codes.astype(np.float64) @ w_codes.astype(np.float64).T   # exact: below 2^53
    p = acc * scale.astype(np.float64)[:, None] * w_scale.astype(np.float64)[None, :]
    return p + (0.0 if bias is None else bias.astype(np.float64)), np.abs(p)


def candidates(score, logits, log_softmax, finished=None, end_token=None):
    """Values [B, W, V] float64 of all candidates; -inf: never taken."""
    B, W = score.shape
    x = logits.astype(np.float64).reshape(B, W, -1)
    with np.errstate(all="ignore"):
        if log_softmax:
            top = x.max(axis=2, keepdims=True)
            x = (x - top) - np.log(np.exp(x - top).sum(axis=2, keepdims=True))
        v = score.astype(np.float64)[:, :, None] + x
    if finished is not None:
        through = finished.astype(bool)
        v[through] = -np.inf
        v[through, end_token] = score.astype(np.float64)[through]
    return np.where(np.isnan(v), -np.inf, v)


def select(v, n):
    """The n best of v [B, W, V] by (value, lowest hypothesis, lowest token): parent, token, value."""
    B, W, V = v.shape
    flat = v.reshape(B, W * V)
    at = np.argsort(-flat, axis=1, kind="stable")[:, :n]
    best = np.take_along_axis(flat, at, axis=1)
    none = best == -np.inf
    parent, token = np.where(none, -1, at // V), np.where(none, -1, at % V)
    if at.shape[1] < n:   # fewer candidates than ranks
        pad = ((0, 0), (0, n - at.shape[1]))
        parent, token = np.pad(parent, pad, constant_values=-1), np.pad(token, pad, constant_values=-1)
        best = np.pad(best, pad, constant_values=-np.inf)
    return parent, token, best
