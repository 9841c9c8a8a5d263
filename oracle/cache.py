"""Operators of long and shared contexts in plain numpy and 64 bits.

Written from the definitions in include/cp_cache.h, one row, token and head at a
time, without the library's kernels.  Tensors of the pools are [NB][Hkv][B][D]
(K) and [NB][Hkv][D][B] (V) as float64; rows are (req, start, len, ctx).
"""

from __future__ import annotations

import numpy as np

LARGEST = float(np.float32(np.array([0x7f7f0000], np.uint32).view(np.float32)[0]))  # finite bf16


def tokens(rows):
    """(token, row, position) of every new token."""
    t = 0
    for r, (_, start, n, _) in enumerate(rows):
        for j in range(n):
            yield t, r, start + j
            t += 1


def append(k_cache, v_cache, k, v, table, rows):
    """The pools (copies) with the tokens' k and v [T][Hkv][D] in their slots."""
    kc, vc = k_cache.copy(), v_cache.copy()
    block = kc.shape[2]
    for t, r, p in tokens(rows):
        b = table[rows[r][0], p // block]
        if 0 <= b < kc.shape[0]:
            kc[b, :, p % block], vc[b, :, :, p % block] = k[t], v[t]
    return kc, vc


def bounds(k_cache, table, rows, old):
    """``old`` [NB][Hkv][2][D] with the bounds of the pages that the rows wrote to."""
    out, block = old.copy(), k_cache.shape[2]
    for req, start, n, ctx in rows:
        if n == 0:
            continue
        for p in range(start // block, (ctx - 1) // block + 1):
            b = table[req, p]
            if not 0 <= b < k_cache.shape[0]:
                continue
            k = k_cache[b, :, :min(block, ctx - p * block)]
            bad = ~np.isfinite(k)
            out[b, :, 0] = np.where(bad, -LARGEST, k).min(1)
            out[b, :, 1] = np.where(bad, LARGEST, k).max(1)
    return out


def select(q, page_bounds, table, rows, block, n_pages, n_first, n_last):
    """pages [T][Hkv][n_pages]."""
    t_all, hq, _ = q.shape
    hkv = page_bounds.shape[1]
    out = np.full((t_all, hkv, n_pages), -1, np.int32)
    for t, r, p in tokens(rows):
        n = p // block + 1
        for h in range(hkv):
            score = np.full(n, -np.inf)
            for i in range(n):
                b = table[rows[r][0], i]
                if not 0 <= b < page_bounds.shape[0]:
                    continue
                lo, hi = page_bounds[b, h]
                for e in range(h * hq // hkv, (h + 1) * hq // hkv):
                    score[i] = max(score[i], np.maximum(q[t, e] * lo, q[t, e] * hi).sum())
            score[:n_first] = np.inf
            score[max(0, n - n_last):] = np.inf
            best = np.lexsort((np.arange(n), -score))[:n_pages]
            out[t, h, :len(best)] = np.sort(best)
    return out


def usable(entries, top):
    """The entries of a page list that count: rising, in 0 .. top."""
    out = []
    for e in entries:
        if not 0 <= e <= top or (out and e <= out[-1]):
            break
        out.append(int(e))
    return out


def _attend(q, k, v, scale, out, spread, size):
    with np.errstate(invalid="ignore", over="ignore"):
        s = (k @ q) * scale
        w = np.exp(s - s.max())
        w /= w.sum()
        o = w @ v
        out[:], spread[:], size[:] = o, w @ np.abs(v - o), w @ np.abs(v)


def attn(q, k_cache, v_cache, table, rows, scale, pages=None):
    """Causal attention, over the listed pages only where ``pages`` [T][Hkv][P] is
    given.  Returns (out, spread, size): with the softmax weights w, out = sum w v,
    spread = sum w |v - out| and size = sum w |v|, the factors of the rounding
    errors of a kernel."""
    t_all, hq, d = q.shape
    hkv, block = k_cache.shape[1], k_cache.shape[2]
    out, spread, size = (np.zeros((t_all, hq, d)) for _ in range(3))
    for t, r, p in tokens(rows):
        for h in range(hkv):
            listed = range(p // block + 1) if pages is None else usable(pages[t, h], p // block)
            key = np.array([i * block + s for i in listed for s in range(block)], int)
            key = key[key <= p]
            if len(key) == 0:
                continue
            b = table[rows[r][0], key // block]
            k, v = k_cache[b, h, key % block], v_cache[b, h, :, key % block]
            for e in range(h * hq // hkv, (h + 1) * hq // hkv):
                _attend(q[t, e], k, v, scale, out[t, e], spread[t, e], size[t, e])
    return out, spread, size
