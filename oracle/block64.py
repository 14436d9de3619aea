"""Dropout, layer norm and the biased attention softmax in numpy, 64 bits, from their definitions: what the CUDA kernels are
compared with.  Shares no code with them."""
from __future__ import annotations

import math

import numpy as np

MASK = np.uint64(0xFFFFFFFF)


def philox(counter, key):
    """Philox4x32-10 (Salmon et al., SC 2011): counter is four uint32 arrays (or numbers), key two numbers."""
    c = [np.asarray(v, dtype=np.uint64) for v in counter]
    c = list(np.broadcast_arrays(*c))
    k = [int(key[0]), int(key[1])]
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & MASK, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & MASK]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def threshold(p: float) -> int:
    return int(np.rint(np.float32(p) * np.float32(65536)))


def dropout_factors(rows: int, cols: int, p: float, seed: int, step: int, site: int) -> np.ndarray:
    """[rows, cols] of 0 (dropped) or the factor of a kept element."""
    t = threshold(p)
    if t == 65536:
        return np.zeros((rows, cols))
    groups = -(-cols // 8)
    w = philox([np.arange(groups)[None, :], np.arange(rows)[:, None], step % 2 ** 32, site], (seed % 2 ** 32, seed >> 32))
    bits = np.empty((rows, groups, 8), dtype=np.int64)
    for lane in range(8):
        bits[:, :, lane] = (w[lane // 2] >> np.uint64(16 * (lane % 2))) & np.uint64(0xFFFF)
    return np.where(bits.reshape(rows, groups * 8)[:, :cols] >= t, 65536.0 / (65536 - t), 0.0)


def dropped(x: np.ndarray, factors) -> np.ndarray:
    return np.where(factors == 0, 0.0, x * factors) if factors is not None else x


def layer_norm(x, residual, weight, bias, eps, factors=None):
    """(y, h, mean, rstd)"""
    h = dropped(x, factors)
    if residual is not None:
        h = h + residual
    mean = h.mean(1)
    rstd = 1.0 / np.sqrt(((h - mean[:, None]) ** 2).mean(1) + eps)
    y = (h - mean[:, None]) * rstd[:, None]
    if weight is not None:
        y = y * weight
    if bias is not None:
        y = y + bias
    return y, h, mean, rstd


def layer_norm_backward(dy, dh_in, h, weight, mean, rstd, factors=None):
    """(dx, dresidual, dweight, dbias)"""
    xhat = (h - mean[:, None]) * rstd[:, None]
    g = dy if weight is None else dy * weight
    dh = rstd[:, None] * (g - g.mean(1, keepdims=True) - xhat * (g * xhat).mean(1, keepdims=True))
    if dh_in is not None:
        dh = dh + dh_in
    return dropped(dh, factors), dh, (dy * xhat).sum(0), dy.sum(0)


def bucket(distance: int, num_buckets: int, max_distance: int, bidirectional: bool) -> int:
    """Bucket of distance = key - query, by the formula: half of a side's buckets one distance each, then equal ratios."""
    n = num_buckets // 2 if bidirectional else num_buckets
    away = abs(distance) if bidirectional else max(-distance, 0)
    exact = n // 2
    if away < exact:
        b = away
    else:
        at = math.log(away / exact) / math.log(max_distance / exact) * (n - exact)
        b = min(n - 1, exact + int(math.floor(at + 1e-7)))
    return b + (n if bidirectional and distance > 0 else 0)


def buckets(q: int, k: int, q_offset: int, num_buckets: int, max_distance: int, bidirectional: bool) -> np.ndarray:
    lo, hi = -(q - 1 + q_offset), k - 1 - q_offset
    line = np.array([bucket(d, num_buckets, max_distance, bidirectional) for d in range(lo, hi + 1)], dtype=np.int64)
    d = np.arange(k)[None, :] - (np.arange(q)[:, None] + q_offset)
    return line[d - lo] if q and k else np.zeros((q, k), np.int64)


def kept(batch, q, k, causal, q_offset, key_len) -> np.ndarray:
    m = np.ones((batch, 1, q, k), dtype=bool)
    if causal:
        m &= np.arange(k)[None, :] <= np.arange(q)[:, None] + q_offset
    if key_len is not None:
        m &= (np.arange(k)[None, :] < np.asarray(key_len)[:, None])[:, None, None, :]
    return m


def softmax(scores, bias, scale, keep):
    """(undropped probabilities, lse); bias [heads, q, k] or None.  Rows with nothing kept, or nothing above -inf: zeros."""
    with np.errstate(all="ignore"):
        t = scores * scale if bias is None else scores * scale + bias
        t = np.where(keep, t, -np.inf)
        top = t.max(-1, keepdims=True, initial=-np.inf)
        e = np.where(np.broadcast_to(keep, t.shape), np.exp(t - np.where(top == -np.inf, 0.0, top)), 0.0)
        s = e.sum(-1, keepdims=True)
        probs = np.where(s == 0, 0.0, e / np.where(s == 0, 1.0, s))
        lse = np.where(s == 0, -np.inf, np.where(top == -np.inf, 0.0, top) + np.log(s))[..., 0]
    return probs, lse


def softmax_backward(dprobs, probs, factors, scale, bucket_ids, num_buckets):
    """(dscores, dtable) from the undropped probabilities; factors [batch, heads, q, k] or None."""
    dp = np.where(probs == 0, 0.0, dropped(dprobs, factors))
    ds = probs * (dp - (probs * dp).sum(-1, keepdims=True))
    dtable = None
    if bucket_ids is not None:
        over = ds.sum(0)
        dtable = np.stack([np.where(bucket_ids == b, over, 0.0).sum((1, 2)) for b in range(num_buckets)])
    return ds * scale, dtable
