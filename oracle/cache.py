"""The paged key-value cache's operators from their definitions, numpy fp64.

Caches are plain arrays: k, v [B][Hkv, n_b, d] per sequence (what the pages
hold, in order), so the paging itself is the caller's to undo.
"""
import numpy as np


def pages_to_rows(pages, table_row, n):
    """[num_pages, page, Hkv, d], a row of page numbers -> [Hkv, n, d]."""
    page = pages.shape[1]
    cols = -(-n // page)
    rows = pages[np.asarray(table_row[:cols], np.int64)] if cols else pages[:0]
    return rows.reshape(-1, *pages.shape[2:])[:n].transpose(1, 0, 2)


def cache_attention(q, k, v, scale):
    """One sequence: q [H,d], k / v [Hkv,n,d] -> o [H,d], lse [H], w [Hkv,n]
    (the mean over a KV head's query heads of the softmax weights)."""
    H, d = q.shape
    Hkv, n, _ = k.shape
    q = np.asarray(q, np.float64).reshape(Hkv, H // Hkv, d)
    k, v = np.asarray(k, np.float64), np.asarray(v, np.float64)
    if n == 0:
        return np.zeros((H, d)), np.full(H, -np.inf), np.zeros((Hkv, 0))
    x = scale * np.einsum("hgd,hnd->hgn", q, k)
    top = x.max(-1, keepdims=True)
    e = np.exp(x - top)
    z = e.sum(-1, keepdims=True)
    p = e / z
    o = np.einsum("hgn,hnd->hgd", p, v)
    return o.reshape(H, d), (top + np.log(z)).reshape(H), p.mean(1)


def cache_keep(acc, keep, sinks, recent):
    """One row of accumulated weights [n] -> the kept places, ascending."""
    n = len(acc)
    if n <= keep:
        return np.arange(n)
    inside = range(sinks, n - recent)
    worth = [(-np.inf if np.isnan(acc[j]) else float(acc[j]), np.isnan(acc[j])) for j in inside]
    # largest first; a NaN below -inf; equal ones by their place
    order = sorted(range(len(worth)), key=lambda i: (worth[i][1], -worth[i][0], i))
    best = [sinks + i for i in order[:keep - sinks - recent]]
    return np.array(sorted(list(range(sinks)) + best + list(range(n - recent, n))), np.int64)
