"""Drafted trees and forks in plain numpy, attention in 64 bits.

Written from the definitions in include/cp_tree.h, one row, node and head at a
time, without the library's kernels.  Tensors of the pools are [NB][Hkv][B][D]
(K) and [NB][Hkv][D][B] (V); rows are (req, start, nodes, ctx).
"""

from __future__ import annotations

import numpy as np


def ancestors(parents, j):
    """Node j and its ancestors; a parent that is no earlier node ends the chain."""
    chain = [j]
    while 0 <= parents[chain[-1]] < chain[-1]:
        chain.append(int(parents[chain[-1]]))
    return chain


def layout(parents, rows, words):
    """(mask uint64 [T][words], positions int32 [T])."""
    total = int(sum(r[2] for r in rows))
    mask, pos, at = np.zeros((total, words), np.uint64), np.zeros(total, np.int32), 0
    for _, start, n, _ in rows:
        for j in range(n):
            chain = ancestors(parents[at:at + n], j)
            for k in chain:
                mask[at + j, k // 64] |= np.uint64(1 << (k % 64))
            pos[at + j] = start + len(chain) - 1
        at += n
    return mask, pos


def seen(mask_row, n):
    """Which of a row's n nodes a mask names."""
    return np.array([(int(mask_row[j // 64]) >> (j % 64)) & 1 for j in range(n)], bool)


def attn(q, k_cache, v_cache, table, mask, rows, scale):
    """q [T][Hq][D] and the pools as float64.  Returns (out, spread, size): with
    the softmax weights w, out = sum w v, spread = sum w |v - out| and
    size = sum w |v|, the factors of the rounding errors of a kernel."""
    q = np.asarray(q, np.float64)
    t, hq, d = q.shape
    hkv, block = k_cache.shape[1], k_cache.shape[2]
    out, spread, size = (np.zeros((t, hq, d)) for _ in range(3))
    at = 0
    for req, start, n, ctx in rows:
        blocks = table[req, :-(-ctx // block)] if ctx else table[req, :0]
        for h in range(hkv):
            k = k_cache[blocks, h].reshape(-1, d)[:ctx]
            v = v_cache[blocks, h].transpose(0, 2, 1).reshape(-1, d)[:ctx]
            for j in range(n):
                vis = np.concatenate([np.ones(start, bool), seen(mask[at + j], n)])
                if not vis.any():
                    continue
                for g in range(h * hq // hkv, (h + 1) * hq // hkv):
                    with np.errstate(invalid="ignore", over="ignore"):
                        s = (k[vis] @ q[at + j, g]) * scale
                        w = np.exp(s - s.max())
                        w /= w.sum()
                        o = w @ v[vis]
                        out[at + j, g] = o
                        spread[at + j, g] = w @ np.abs(v[vis] - o)
                        size[at + j, g] = w @ np.abs(v[vis])
        at += n
    return out, spread, size


def argmax(row):
    """The first largest value; NaN is larger than any number."""
    nan = np.flatnonzero(np.isnan(row))
    return int(nan[0]) if len(nan) else int(np.flatnonzero(row == row.max())[0])


def verify(logits, tokens, parents, rows, max_path):
    """(target, path, n_accepted, next_token)."""
    target = np.array([argmax(r) for r in logits], np.int32)
    path = np.full((len(rows), max_path), -1, np.int32)
    count, after, at = np.zeros(len(rows), np.int32), np.full(len(rows), -1, np.int32), 0
    for r, (_, _, n, _) in enumerate(rows):
        cur = 0 if n else -1
        while cur >= 0 and count[r] < max_path:
            path[r, count[r]] = cur
            count[r] += 1
            after[r] = target[at + cur]
            cur = next((j for j in range(cur + 1, n) if parents[at + j] == cur
                        and tokens[at + j] == after[r]), -1)
        at += n
    return target, path, count, after


def usable(path, count, n, max_path):
    """The entries of a row's path that count."""
    out = []
    for p in path[:max(0, min(int(count), max_path))]:
        if not 0 <= p < n or (out and p <= out[-1]):
            break
        out.append(int(p))
    return out


def compact(k_cache, v_cache, table, rows, path, n_accepted):
    """The pools after the moves (copies)."""
    k, v = k_cache.copy(), v_cache.copy()
    nb, _, block, _ = k.shape
    for r, (req, start, n, _) in enumerate(rows):
        for i, p in enumerate(usable(path[r], n_accepted[r], n, path.shape[1])):
            a, b = start + p, start + i
            x, y = int(table[req, a // block]), int(table[req, b // block])
            if 0 <= x < nb and 0 <= y < nb:
                k[y, :, b % block] = k_cache[x, :, a % block]
                v[y, :, :, b % block] = v_cache[x, :, :, a % block]
    return k, v


def fork(k_cache, v_cache, table, forks):
    """(K, V, table) after the forks (copies)."""
    k, v, t = k_cache.copy(), v_cache.copy(), table.copy()
    nb, block = k.shape[0], k.shape[2]
    for src, dst, ctx, page in forks:
        full = ctx // block
        t[dst, :full] = table[src, :full]
        if ctx % block:
            t[dst, full] = page
            if 0 <= table[src, full] < nb:
                k[page], v[page] = k_cache[table[src, full]], v_cache[table[src, full]]
    return k, v, t
