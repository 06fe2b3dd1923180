"""fp64 reference of the windowed and the tree attention over the paged cache, and
of the calls that rearrange its pages -- TEST INFRASTRUCTURE ONLY.

Plain numpy, one row at a time: the positions a row sees are listed, their keys and
values taken from those that some row of the request sees, and nothing else is read.  Next to each
output stands what an error bound needs: the sum of the absolute weighted values
and the largest sum of absolute products in a score.
"""
from __future__ import annotations

import numpy as np

import oracle

PAGE = 16


def window_sees(p, window, sinks):
    """Positions a row at position p sees."""
    j = np.arange(p + 1)
    return j[(j > p - window) | (j < sinks)]


def tree_sees(prefix, n, words):
    """Positions a draft sees: the prefix and the drafts (of n) its mask words name."""
    bits = np.unpackbits(np.asarray(words, np.uint32).astype("<u4").view(np.uint8), bitorder="little")[:n]
    return np.concatenate([np.arange(prefix), prefix + np.nonzero(bits)[0]])


def widen(x, scale=None):
    """Cache elements as float64: bf16 bits, fp32, or E4M3 codes times their head's scale (last axis but one)."""
    if x.dtype == np.uint8:
        return oracle.e4m3_value(np.arange(256))[x] * np.asarray(scale, np.float64)
    if x.dtype == np.uint16:
        return (x.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    return x.astype(np.float64)


def attention(q, k_pool, v_pool, page_table, cu, prefix, scale, sees, k_scale=None, v_scale=None):
    """sees(r, i): the positions row i of request r sees.

    Returns (out [T][Hq][d], lse [T][Hq], weighted [T][Hq][d], products [T][Hq]): weighted = sum p |v| / sum p,
    products = max over the row's keys of scale * sum |q k|."""
    qw = widen(np.asarray(q))
    t, hq, d = qw.shape
    hkv = k_pool.shape[1]
    g = hq // hkv
    out, weighted = np.zeros((t, hq, d)), np.zeros((t, hq, d))
    lse, products = np.full((t, hq), -np.inf), np.zeros((t, hq))
    with np.errstate(invalid="ignore", over="ignore"):
        for r in range(len(prefix)):
            rows = [np.asarray(sees(r, i), np.int64) for i in range(int(cu[r + 1] - cu[r]))]
            union = np.unique(np.concatenate(rows)) if rows else np.zeros(0, np.int64)
            page, slot = page_table[r, union // PAGE], union % PAGE
            assert (page >= 0).all()
            for c in range(hkv if len(union) else 0):
                keys = widen(k_pool[page, c, slot, :], None if k_scale is None else k_scale[c])
                values = widen(v_pool[page, c, :, slot], None if v_scale is None else v_scale[c])
                h = slice(c * g, (c + 1) * g)
                for i, pos in enumerate(rows):
                    if len(pos) == 0:
                        continue
                    at = np.searchsorted(union, pos)
                    k, v, row = keys[at], values[at], int(cu[r]) + i
                    s = scale * qw[row, h] @ k.T
                    m = s.max(1, keepdims=True)
                    e = np.exp(s - m)
                    z = e.sum(1, keepdims=True)
                    out[row, h] = e @ v / z
                    weighted[row, h] = e @ np.abs(v) / z
                    lse[row, h] = (m + np.log(z))[:, 0]
                    products[row, h] = (abs(scale) * np.abs(qw[row, h]) @ np.abs(k).T).max(1)
    return out, lse, weighted, products


def compact(k_pool, v_pool, page_table, prefix, accepted, count):
    """Pools [layers][pages]... after the accepted drafts moved behind their prefix."""
    k, v = k_pool.copy(), v_pool.copy()
    for r in range(len(prefix)):
        for i in range(min(max(int(count[r]), 0), accepted.shape[1])):
            fr, to = int(prefix[r]) + int(accepted[r, i]), int(prefix[r]) + i
            pf, pd = page_table[r, fr // PAGE], page_table[r, to // PAGE]
            k[:, pd, :, to % PAGE, :] = k_pool[:, pf, :, fr % PAGE, :]
            v[:, pd, :, :, to % PAGE] = v_pool[:, pf, :, :, fr % PAGE]
    return k, v


def copy_pages(k_pool, v_pool, src, dst):
    k, v = k_pool.copy(), v_pool.copy()
    for s, t in zip(src, dst):
        if 0 <= s < k.shape[1] and 0 <= t < k.shape[1]:
            k[:, t], v[:, t] = k_pool[:, s], v_pool[:, s]
    return k, v
