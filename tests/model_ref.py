"""Plain 64-bit references of the model-side calls, one row and head at a time, with the
bounds that the kernels' fp32 arithmetic and roundings keep to.

u = 2^-24 is half an fp32 step, 2^-8 half a bf16 step, 2^-4 half an e4m3 step (relative).
"""
import math

import numpy as np
import torch

U = 2.0 ** -24


def f64(t):
    return t.detach().float().cpu().double().numpy()


def rows_of(lens, draft_len, n, b):
    T, L = int(lens[b]), n - 1 if draft_len is None else int(draft_len[b])
    return (L + 1 if T >= 1 and 0 <= L < n else 0), T - 1


def cache_rows(cache, scale, table, b, head, count):
    """Positions 0..count-1 of sequence b: fp64 [count][D], NaN where the page is bad."""
    P, page, _, D = cache.shape
    out = np.full((count, D), np.nan)
    for j0 in range(0, count, page):
        at = table[b, j0 // page] if j0 // page < table.shape[1] else -1
        if 0 <= at < P:
            m = min(page, count - j0)
            rows = f64(cache[int(at), :m, head])
            if scale is not None:
                rows = rows * f64(scale[int(at), head, :m])[:, None]
            out[j0:j0 + m] = rows
    return out


def attn_row(q, k, v, pos, scale, softcap, window):
    """One query row: (weights over 0..pos, out, lse, bound of a score's error, sum p|v|);
    keys that are not seen are left out, whatever they hold."""
    lo = max(0, pos + 1 - window) if window else 0
    seen = slice(lo, pos + 1)
    x = k[seen] @ q * scale
    size = np.abs(k[seen]) @ np.abs(q) * scale
    # D products and sums, the scale's and the e4m3 scale's products
    tol = (len(q) + 8) * U * (np.max(size) if len(size) else 0.0)
    if softcap:
        x = softcap * np.tanh(x / softcap)
        tol += 16 * U * softcap
    if not len(x) or np.isnan(x).any():
        return None, np.full(v.shape[1], np.nan), np.nan, 0.0, np.zeros(v.shape[1])
    m = x.max()
    lse = m + math.log(np.exp(x - m).sum())
    w = np.zeros(pos + 1)
    w[seen] = np.exp(x - lse)
    return w, w[seen] @ v[seen], lse, tol, w[seen] @ np.abs(v[seen])


def lse_bound(tol, lse, count):
    """Of a log sum of `count` exponentials of scores that are off by tol."""
    return tol + 8 * U * (abs(lse) + 1) + (math.log2(count + 1) + 64) * 2 * U


def out_bound(ref, spread, tol):
    """Of an attention output: its own rounding, the weights' rounding to bf16 before the
    product (half a step of each term) and the scores' error in the weights."""
    return 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 * 1.02 + 4 * tol + 2.0 ** -16) * spread + 1e-30


def turned(x, rope, pos, halves):
    if rope is None:
        return x
    r = rope.shape[1]
    c, s = rope[pos, :r // 2], rope[pos, r // 2:]
    y = x.copy()
    if halves:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y[..., :r // 2], y[..., r // 2:r] = a * c - b * s, b * c + a * s
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y[..., 0:r:2], y[..., 1:r:2] = a * c - b * s, b * c + a * s
    return y


def normed(x, w, eps):
    return x if w is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w


def logprob_row(z, tau):
    """(log probabilities, entropy, ids in order) of one row of logits."""
    order = np.argsort(-z, kind="stable")
    m = z.max()
    if not m > -np.inf:
        return np.full(len(z), -np.inf), 0.0, order
    with np.errstate(over="ignore"):   # the type's lowest value over a small temperature
        x = (z - m) / tau
    lp = x - math.log(np.exp(x).sum())
    p = np.exp(lp)
    return lp, float(-(p[p > 0] * lp[p > 0]).sum()), order
