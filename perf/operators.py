"""Operators of speculative decoding and forked requests over the paged cache.

Five kinds, each one call of the framework:

* ``layout``   parents of drafted trees to visibility masks and rotary positions.
* ``attn``     attention of every drafted node over its request's committed
               keys and its own ancestors, K/V in the paged pools.
* ``verify``   greedy verification: the argmax of every node's logits, and the
               longest path of drafted tokens that agrees with them.
* ``compact``  the K/V of each accepted path moved to consecutive slots, in
               every layer's pools.
* ``fork``     requests that continue others: shared full pages, a copy of the
               partly filled one in every layer's pools.

``own`` chooses between the framework's calls and their plain forms in
elementary torch operations.  A case is a dict of plain values; row lengths
follow from it (``rows_seed``), trees and tensor contents from the seed.
"""

import math
from functools import reduce

import numpy as np
import torch

own = False

DEV = "cuda:0"
LAYERS, VOCAB = 36, 151936


# ---------------------------------------------------------------- the cases

def _attn(hq, hkv, d, block, reqs, nodes, median, spread, longest, rows_seed):
    """``reqs`` requests of up to ``nodes`` drafted nodes over committed contexts
    of log-normal length (median, sigma ``spread``, at most ``longest``)."""
    return {"kind": "attn", "hq": hq, "hkv": hkv, "d": d, "block": block, "reqs": reqs,
            "nodes": nodes, "median": median, "spread": spread, "longest": longest,
            "rows_seed": rows_seed}


def _layout(reqs, nodes, rows_seed):
    return {"kind": "layout", "reqs": reqs, "nodes": nodes, "rows_seed": rows_seed}


def _verify(reqs, nodes, vocab, rows_seed):
    return {"kind": "verify", "reqs": reqs, "nodes": nodes, "vocab": vocab, "rows_seed": rows_seed}


def _pages(kind, hkv, d, block, layers, reqs, median, rows_seed):
    return {"kind": kind, "hkv": hkv, "d": d, "block": block, "layers": layers, "reqs": reqs,
            "median": median, "rows_seed": rows_seed}


def listed():
    return [
        # one short request with a small tree on few heads: latency
        {"name": "attn-1x8", **_attn(4, 2, 64, 16, 1, 8, 300, 0.1, 512, 1)},
        # an ordinary round: 32 requests with short drafts, contexts of about a thousand
        {"name": "attn-32x8", **_attn(32, 8, 128, 16, 32, 8, 1024, 1.0, 8192, 2)},
        # wide trees on the 64/8-head layer: a product-bound round
        {"name": "attn-24x64", **_attn(64, 8, 128, 32, 24, 64, 2048, 0.7, 8192, 3)},
        # few requests, very long contexts: split over the keys
        {"name": "attn-4x16-far", **_attn(32, 8, 128, 16, 4, 16, 32768, 0.1, 40000, 4)},
        # one request's tree
        {"name": "layout-1x8", **_layout(1, 8, 5)},
        # a large batch of wide trees
        {"name": "layout-256x64", **_layout(256, 64, 6)},
        # one request's tree against the whole vocabulary
        {"name": "verify-1x8", **_verify(1, 8, VOCAB, 7)},
        # a busy round: the logits are the traffic
        {"name": "verify-32x32", **_verify(32, 32, VOCAB, 8)},
        # one request's accepted path, every layer of the 36-layer model
        {"name": "compact-1", **_pages("compact", 8, 128, 16, LAYERS, 1, 400, 9)},
        # a busy round's accepted paths
        {"name": "compact-64", **_pages("compact", 8, 128, 16, LAYERS, 64, 100, 10)},
        # one request continued by a second
        {"name": "fork-1", **_pages("fork", 8, 128, 16, LAYERS, 1, 1000, 11)},
        # parallel samples of many requests
        {"name": "fork-64", **_pages("fork", 8, 128, 32, LAYERS, 64, 200, 12)},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "layout", "verify", "verify", "compact", "fork"])
    seed = rng.randrange(1 << 30)
    if kind == "attn":
        largest = work(listed()[2])
        while True:
            hq, hkv, d, block = rng.choice([(4, 2, 64, 16), (16, 16, 64, 32), (32, 8, 128, 16),
                                            (32, 8, 128, 16), (64, 8, 128, 32), (8, 1, 128, 32),
                                            (16, 8, 128, 32)])
            case = _attn(hq, hkv, d, block, _log_int(rng, 1, 64), _log_int(rng, 1, 256),
                         _log_int(rng, 16, 16384), rng.choice([0.1, 0.5, 1.0]), 32768, seed)
            w = work(case)
            starts, lens = _rows(case)
            padded = len(starts) * hq * int(lens.max()) * int((starts + lens).max())
            if w["bytes"] <= largest["bytes"] and w["flops"] <= largest["flops"] and padded <= 1e9:
                return case
    if kind == "layout":
        return _layout(_log_int(rng, 1, 250), _log_int(rng, 1, 256), seed)
    if kind == "verify":
        nodes = _log_int(rng, 1, 200)
        return _verify(_log_int(rng, 1, max(1, 1000 // nodes)), nodes, _log_int(rng, 1000, VOCAB - 1),
                       seed)
    hkv, d, block = rng.choice([(8, 128, 16), (8, 128, 32), (2, 64, 16), (1, 128, 32)])
    return _pages(kind, hkv, d, block, rng.choice([2, 4, 12, 24, 36]), _log_int(rng, 1, 60),
                  _log_int(rng, 20, 400), seed)


# ---------------------------------------------------------------- rows and work

def _rows(case):
    """(committed lengths, drafted nodes) of every row."""
    rng = np.random.default_rng(case["rows_seed"])
    n = case["reqs"]
    median, spread = case.get("median", 500), case.get("spread", 0.5)
    starts = np.round(rng.lognormal(math.log(median), spread, n)).astype(np.int64)
    starts = np.clip(starts, 1, case.get("longest", 4096))
    nodes = case.get("nodes", 32)
    lens = rng.integers(max(1, nodes // 2), nodes + 1, n)
    lens[0] = nodes
    return starts, lens


def _accepted(case, lens):
    """Accepted nodes of every row: 1 to 8."""
    rng = np.random.default_rng(case["rows_seed"] + 1)
    return np.minimum(1 + rng.binomial(7, 0.4, len(lens)), lens)


def work(case):
    starts, lens = _rows(case)
    t, kind = int(lens.sum()), case["kind"]
    if kind == "attn":
        hq, hkv, d, block = (case[k] for k in ("hq", "hkv", "d", "block"))
        words = -(-int(lens.max()) // 64)
        depth = np.log(np.maximum(lens, 1)) + 1.0          # ancestors of a node, about
        keys = float((starts + lens).sum())
        return {"bytes": 4.0 * hkv * d * keys + t * (4.0 * hq * d + 8.0 * words)
                + 4.0 * float((-(-(starts + lens) // block)).sum()),
                "flops": 4.0 * hq * d * float((lens * (starts + depth)).sum())}
    if kind == "layout":
        return {"bytes": t * (8.0 + 8.0 * -(-int(lens.max()) // 64)), "flops": 0.0}
    if kind == "verify":
        return {"bytes": t * (2.0 * case["vocab"] + 12.0), "flops": 0.0}
    hkv, d, block, layers = (case[k] for k in ("hkv", "d", "block", "layers"))
    if kind == "compact":
        moved = float((_accepted(case, lens) - 1).sum()) + 1.0
        return {"bytes": moved * layers * hkv * d * 8.0 + 40.0 * len(lens), "flops": 0.0}
    partial = float((starts % block != 0).sum())
    return {"bytes": partial * layers * hkv * d * block * 8.0 + 8.0 * float((starts // block + 1).sum()),
            "flops": 0.0}


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.bfloat16)


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).to(DEV)


def _parents(lens, rng):
    """A random tree for every row, packed: node 0 is the root, a later node
    hangs from an earlier one."""
    out = []
    for n in lens:
        j = np.arange(n)
        out.append(np.where(j == 0, -1, np.floor(rng.random(n) * np.maximum(j, 1)).astype(np.int64)))
    return np.concatenate(out).astype(np.int32)


def _ancestors(parents, n):
    a = np.zeros((n, n), bool)
    for j in range(n):
        if j:
            a[j] = a[parents[j]]
        a[j, j] = True
    return a


def _meta(starts, lens, slots):
    return np.stack([slots, starts, lens, starts + lens], 1).astype(np.int32)


def _table(rng, need, slots, spare=0):
    """A block table over a pool of sum(need) + spare + 1 pages in random order:
    row slots[i] names need[i] of them, the other entries the last page."""
    pool = int(sum(need)) + spare + 1
    perm = rng.permutation(pool).astype(np.int32)
    table = np.full((int(max(slots)) + 1, int(max(need)) + 1), perm[-1], np.int32)
    at = 0
    for slot, n in zip(slots, need):
        table[slot, :n] = perm[at:at + n]
        at += n
    return table, pool, perm[at:at + spare]


def _prepare_attn(case, seed, rng, starts, lens):
    hq, hkv, d, block = (case[k] for k in ("hq", "hkv", "d", "block"))
    slots = rng.permutation(len(lens))
    table, pool, _ = _table(rng, -(-(starts + lens) // block), slots)
    meta, t = _meta(starts, lens, slots), int(lens.sum())
    words = -(-int(lens.max()) // 64)
    parents, at, mask = _parents(lens, rng), 0, np.zeros((t, words), np.uint64)
    for n in lens:
        a = np.zeros((n, words * 64), np.uint64)
        a[:, :n] = _ancestors(parents[at:at + n], n)
        mask[at:at + n] = (a.reshape(n, words, 64) << np.arange(64, dtype=np.uint64)).sum(
            -1, dtype=np.uint64)
        at += n
    g = _gen(seed)
    s = {"rows": meta, "table": _i32(table), "scale": 1.0 / math.sqrt(d),
         "mask": torch.from_numpy(mask.view(np.int64)).to(DEV), "q": _randn(g, t, hq, d),
         "kc": _randn(g, pool, hkv, block, d), "vc": _randn(g, pool, hkv, d, block),
         "out": torch.empty(t, hq, d, dtype=torch.bfloat16, device=DEV)}
    if own:
        from paper_2606_09061_amd import tree
        s["desc"] = _desc(hq, hkv, d, block, pool, table)
        s["ws"] = _bytes(tree.attn_workspace_bytes(s["desc"], meta))
    return s


def _bytes(n):
    return torch.empty(max(n, 256), dtype=torch.uint8, device=DEV)


def _desc(hq, hkv, d, block, pool, table):
    from paper_2606_09061_amd import binding
    return binding.make_desc(hq, hkv, d, block, pool, table.shape[1], table.shape[0],
                             1.0 / math.sqrt(d))


def _prepare_layout(case, seed, rng, starts, lens):
    t = int(lens.sum())
    return {"rows": _meta(starts, lens, np.arange(len(lens))), "parents": _i32(_parents(lens, rng)),
            "mask": torch.empty(t, -(-int(lens.max()) // 64), dtype=torch.int64, device=DEV),
            "positions": torch.empty(t, dtype=torch.int32, device=DEV)}


def _prepare_verify(case, seed, rng, starts, lens):
    """Logits N(0, 1) in bf16, where the maximum is often shared; two thirds of
    the nodes with children favour one child's token."""
    t, vocab, n = int(lens.sum()), case["vocab"], len(lens)
    parents, tokens = _parents(lens, rng), rng.integers(0, vocab, t)
    logits = _randn(_gen(seed), t, vocab)
    first = np.repeat(np.cumsum(lens) - lens, lens)
    liked = (parents >= 0) & (rng.random(t) < 0.67)
    up = first + np.maximum(parents, 0)
    logits[torch.from_numpy(up[liked]).to(DEV), torch.from_numpy(tokens[liked]).to(DEV)] = 9.0

    def ints(*shape):
        return torch.empty(*shape, dtype=torch.int32, device=DEV)

    depth = 16
    s = {"rows": _meta(starts, lens, np.arange(n)), "logits": logits, "tokens": _i32(tokens),
         "parents": _i32(parents), "target": ints(t), "path": ints(n, depth),
         "n_accepted": ints(n), "next_token": ints(n)}
    if own:
        from paper_2606_09061_amd import tree
        s["ws"] = _bytes(tree.verify_workspace_bytes(t, vocab))
    return s


def _pools(case, g, pool, table):
    """Every layer's pools, and the handle of them that a server keeps."""
    hkv, d, block, layers = (case[k] for k in ("hkv", "d", "block", "layers"))
    k, v = _randn(g, layers, pool, hkv, block, d), _randn(g, layers, pool, hkv, d, block)
    s = {"k_pools": k, "v_pools": v}
    if own:
        from paper_2606_09061_amd import tree
        s["layers"] = tree.kv_layers(_desc(4 * hkv, hkv, d, block, pool, table), list(k.unbind(0)),
                                     list(v.unbind(0)))
    return s


def _prepare_compact(case, seed, rng, starts, lens):
    """Trees laid out level by level: an accepted path is the root, often its
    first child, then nodes behind the accepted count (so that a second pass
    over the same buffers moves the same values)."""
    slots = rng.permutation(len(lens))
    table, pool, _ = _table(rng, -(-(starts + lens) // case["block"]), slots)
    count, depth = _accepted(case, lens), 8
    path = np.full((len(lens), depth), -1, np.int32)
    for r, (c, n) in enumerate(zip(count, lens)):
        later = 1 + np.arange(c - 1)
        if n - c >= c - 1:
            later = np.sort(rng.choice(np.arange(c, n), c - 1, replace=False))
            if c > 2 and rng.random() < 0.6:
                later[0] = 1
        path[r, :c] = np.concatenate([[0], later])
    return {"rows": _meta(starts, lens, slots), "table": _i32(table), "path": _i32(path),
            "n_accepted": _i32(count), **_pools(case, _gen(seed), pool, table)}


def _prepare_fork(case, seed, rng, starts, lens):
    """forks: (source row, new row, committed length, page for the partial block)."""
    n, block = len(lens), case["block"]
    slots = rng.permutation(2 * n)
    table, pool, fresh = _table(rng, np.concatenate([-(-starts // block), np.zeros(n, np.int64)]),
                                slots, spare=n)
    forks = np.stack([slots[:n], slots[n:], starts, np.where(starts % block, fresh, -1)],
                     1).astype(np.int32)
    return {"forks": forks, "table": _i32(table), **_pools(case, _gen(seed), pool, table)}


def prepare(case, seed):
    starts, lens = _rows(case)
    rng = np.random.default_rng(int(seed))
    s = {"attn": _prepare_attn, "layout": _prepare_layout, "verify": _prepare_verify,
         "compact": _prepare_compact, "fork": _prepare_fork}[case["kind"]](case, seed, rng, starts,
                                                                           lens)
    return {"case": case, **s}


# ---------------------------------------------------------------- plain forms

def _padded(rows):
    """For rows (slot, start, len, ctx) on the host: their columns on the GPU,
    the packed index of node j of each row (clamped inside the row), and which
    of the [rows, longest] places are nodes."""
    slot, start, n, ctx = _i32(rows).long().unbind(1)
    j = torch.arange(int(rows[:, 2].max()), device=DEV)
    first = torch.cumsum(n, 0) - n
    real = j < n[:, None]
    return slot, start, n, ctx, first[:, None] + torch.minimum(j, n[:, None] - 1), real


def _plain_attn(s):
    kc, vc, q = s["kc"], s["vc"], s["q"]
    (t, hq, d), (_, hkv, block, _) = q.shape, kc.shape
    g, rows = hq // hkv, s["rows"]
    slot, start, n, ctx, node, real = _padded(rows)
    r, m = node.shape
    keys = -(-int(rows[:, 3].max()) // block) * block
    pages = s["table"][slot, :keys // block].long()
    k = kc[pages].float().permute(0, 2, 1, 3, 4).reshape(r, hkv, keys, d)
    v = vc[pages].float().permute(0, 2, 1, 4, 3).reshape(r, hkv, keys, d)
    i = torch.arange(keys, device=DEV)
    # stale slots past a row's keys may hold anything
    v = torch.where((i < ctx[:, None])[:, None, :, None], v, 0.0)
    qf = q[node].float().view(r, m, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(r, hkv, m * g, d)
    scores = torch.matmul(qf, k.transpose(2, 3)) * s["scale"]
    at = i - start[:, None]                                      # [r, keys]: index in the tree
    drafted = at.clamp(0, 64 * s["mask"].shape[1] - 1)[:, None, :].expand(r, m, keys)
    bits = (torch.gather(s["mask"][node], 2, drafted >> 6) >> (drafted & 63)) & 1
    seen = ((at < 0)[:, None, :] | ((bits != 0) & (at < n[:, None])[:, None, :])).view(r, 1, m, 1, keys)
    scores = scores.view(r, hkv, m, g, keys).masked_fill(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    w = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    total = w.sum(-1)
    o = torch.matmul(w.view(r, hkv, m * g, keys), v).view(r, hkv, m, g, d)
    o = o / torch.where(total == 0, 1.0, total)[..., None]
    o = o.permute(0, 2, 1, 3, 4).reshape(r, m, hq, d).to(q.dtype)
    # places past a row's nodes repeat its last node
    s["out"][node.reshape(-1)] = o.reshape(-1, hq, d)
    return {"out": s["out"]}


def _closure(parents, real):
    """anc[r, j, k]: k is j or an ancestor of j."""
    r, m = parents.shape
    eye = torch.eye(m, device=DEV)
    up = (parents[..., None] == torch.arange(m, device=DEV)) & real[..., None]
    a = eye + up.float()
    steps = max(1, math.ceil(math.log2(m + 1)))
    return reduce(lambda x, _: (torch.matmul(x, x) > 0).float(), range(steps), a) > 0


def _plain_layout(s):
    slot, start, n, ctx, node, real = _padded(s["rows"])
    words = s["mask"].shape[1]
    anc = _closure(s["parents"][node], real)
    r, m, _ = anc.shape
    bits = torch.zeros(r, m, words * 64, dtype=torch.int64, device=DEV)
    bits[..., :m] = anc
    mask = (bits.view(r, m, words, 64) << torch.arange(64, device=DEV)).sum(-1)
    pos = start[:, None] + anc.sum(-1) - 1
    at = node.reshape(-1)
    last = real.sum(-1, keepdim=True) - 1                        # padded places repeat the last node
    j = torch.minimum(torch.arange(m, device=DEV), last)
    s["mask"][at] = torch.gather(mask, 1, j[..., None].expand_as(mask)).reshape(-1, words)
    s["positions"][at] = torch.gather(pos, 1, j).reshape(-1).int()
    return {"mask": s["mask"], "positions": s["positions"]}


def _plain_verify(s):
    x = s["logits"].float()
    vocab = x.shape[1]
    v = torch.arange(vocab, device=DEV, dtype=torch.int32)
    target = torch.where(x == x.amax(1, keepdim=True), v, vocab).amin(1).int()
    slot, start, n, ctx, node, real = _padded(s["rows"])
    r, m = node.shape
    par, tok, tgt = s["parents"][node].long(), s["tokens"][node], target[node]
    j = torch.arange(m, device=DEV)
    fits = real & (j > 0) & (par >= 0) & (tok == torch.gather(tgt, 1, par.clamp(min=0)))
    same = (par[:, :, None] == par[:, None, :]) & fits[:, None, :] & (j < j[:, None])
    fits = (fits & ~same.any(-1)) | (j == 0)                     # the first child that agrees
    anc = _closure(par, real)
    taken = real & ~(anc & ~fits[:, None, :]).any(-1)
    depth = anc.sum(-1) - 1
    most = s["path"].shape[1]
    taken &= depth < most
    path = torch.full((r, most + 1), -1, dtype=torch.int64, device=DEV)
    path.scatter_(1, torch.where(taken, depth, most), j.expand(r, m))
    count = taken.sum(-1)
    last = torch.gather(path, 1, (count - 1)[:, None])
    s["target"].copy_(target)
    s["path"].copy_(path[:, :most])
    s["n_accepted"].copy_(count)
    s["next_token"].copy_(torch.gather(tgt, 1, last)[:, 0])
    return _verified(s)


def _verified(s):
    return {k: s[k] for k in ("target", "path", "n_accepted", "next_token")}


def _plain_compact(s):
    slot, start, n, ctx = _i32(s["rows"]).long().unbind(1)
    path, block = s["path"].long(), s["case"]["block"]
    i = torch.arange(path.shape[1], device=DEV)
    moves = i < s["n_accepted"][:, None]

    def place(node):                                             # of no move: the root's, onto itself
        p = (start[:, None] + torch.where(moves, node, 0))
        return s["table"][slot[:, None], p // block].long().reshape(-1), (p % block).reshape(-1)

    (sb, ss), (db, ds) = place(path), place(i.expand_as(path))
    k, v = s["k_pools"], s["v_pools"]
    k[:, db, :, ds] = k[:, sb, :, ss]
    v[:, db, :, :, ds] = v[:, sb, :, :, ss]
    return _bits(s)


def _bits(s):
    """The pools as the bit patterns that they hold: these calls only move them."""
    return {"k": s["k_pools"].view(torch.int16), "v": s["v_pools"].view(torch.int16)}


def _plain_fork(s):
    block = s["case"]["block"]
    src, dst, ctx, page = _i32(s["forks"]).long().unbind(1)
    table = s["table"]
    col, full = torch.arange(table.shape[1], device=DEV), (ctx // block)[:, None]
    partial = (ctx % block != 0)[:, None]
    old = table[src]
    table[dst] = torch.where(col < full, old, torch.where((col == full) & partial,
                                                          page[:, None].int(), table[dst]))
    part = torch.from_numpy(np.nonzero(s["forks"][:, 3] >= 0)[0]).to(DEV)
    frm, to = old[part, full[part, 0]].long(), page[part]
    s["k_pools"][:, to] = s["k_pools"][:, frm]
    s["v_pools"][:, to] = s["v_pools"][:, frm]
    return {"table": table, **_bits(s)}


# ---------------------------------------------------------------- one pass

def _own(s):
    from paper_2606_09061_amd import tree
    kind = s["case"]["kind"]
    if kind == "attn":
        tree.attn(s["desc"], s["q"], s["kc"], s["vc"], s["table"], s["mask"], s["rows"], s["out"],
                  s["ws"])
        return {"out": s["out"]}
    if kind == "layout":
        tree.layout(s["parents"], s["rows"], s["mask"], s["positions"])
        return {"mask": s["mask"], "positions": s["positions"]}
    if kind == "verify":
        tree.verify(s["logits"], s["tokens"], s["parents"], s["rows"], s["target"], s["path"],
                    s["n_accepted"], s["next_token"], s["ws"])
        return _verified(s)
    if kind == "compact":
        tree.kv_compact(s["layers"], s["table"], s["rows"], s["path"], s["n_accepted"])
        return _bits(s)
    tree.kv_fork(s["layers"], s["table"], s["forks"])
    return {"table": s["table"], **_bits(s)}


def run(s):
    if own:
        return _own(s)
    return {"attn": _plain_attn, "layout": _plain_layout, "verify": _plain_verify,
            "compact": _plain_compact, "fork": _plain_fork}[s["case"]["kind"]](s)


# ---------------------------------------------------------------- 64-bit results

def _exact_attn(s):
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    hkv, at = s["kc"].shape[1], 0
    g, scale = s["q"].shape[1] // hkv, s["scale"]
    block, mask = s["kc"].shape[2], s["mask"].cpu().numpy().view(np.uint64)
    for slot, start, n, ctx in s["rows"].tolist():
        b = s["table"][slot, :-(-ctx // block)].long()
        words = mask[at:at + n]
        vis = np.ones((n, ctx), bool)
        for j in range(n):
            vis[:, start + j] = (words[:, j // 64] >> np.uint64(j % 64)) & np.uint64(1)
        vis = torch.from_numpy(vis).to(DEV)
        for h in range(hkv):
            k = s["kc"][b, h].double().reshape(-1, s["q"].shape[2])[:ctx]
            v = s["vc"][b, h].double().transpose(1, 2).reshape(-1, s["q"].shape[2])[:ctx]
            for e in range(g):
                x = s["q"][at:at + n, h * g + e].double() @ k.t() * scale
                w = torch.where(vis, torch.exp(x - x.max(1, keepdim=True).values), 0.0)
                total = w.sum(1, keepdim=True)
                out[at:at + n, h * g + e] = w @ v / torch.where(total == 0, 1.0, total)
        at += n
    return {"out": out}


def _exact_layout(s):
    mask, pos, at = np.zeros(tuple(s["mask"].shape), np.uint64), [], 0
    parents = s["parents"].cpu().numpy()
    for _, start, n, _ in s["rows"].tolist():
        for j in range(n):
            k, depth = j, -1
            while k >= 0:
                mask[at + j, k // 64] |= np.uint64(1 << (k % 64))
                k, depth = int(parents[at + k]), depth + 1
            pos.append(start + depth)
        at += n
    return {"mask": mask.view(np.int64), "positions": np.array(pos, np.int32)}


def _exact_verify(s):
    x = s["logits"]
    target = np.empty(x.shape[0], np.int32)
    for t in range(x.shape[0]):
        y = x[t].double()
        target[t] = int((y == y.max()).nonzero()[0, 0])
    parents, tokens = s["parents"].cpu().numpy(), s["tokens"].cpu().numpy()
    path = np.full(tuple(s["path"].shape), -1, np.int32)
    count, after, at = [], [], 0
    for r, (_, _, n, _) in enumerate(s["rows"].tolist()):
        cur, c = 0, 1
        path[r, 0] = 0
        while c < path.shape[1]:
            good = [j for j in range(1, n)
                    if parents[at + j] == cur and tokens[at + j] == target[at + cur]]
            if not good:
                break
            cur = good[0]
            path[r, c] = cur
            c += 1
        count.append(c)
        after.append(target[at + cur])
        at += n
    return {"target": target, "path": path, "n_accepted": np.array(count, np.int32),
            "next_token": np.array(after, np.int32)}


def _exact_compact(s):
    table, path, block = s["table"].cpu().numpy(), s["path"].cpu().numpy(), s["case"]["block"]
    count = s["n_accepted"].cpu().numpy()
    for r, (slot, start, _, _) in enumerate(s["rows"].tolist()):
        for i in range(count[r]):
            a, b = start + int(path[r, i]), start + i
            x, y = int(table[slot, a // block]), int(table[slot, b // block])
            s["k_pools"][:, y, :, b % block] = s["k_pools"][:, x, :, a % block].clone()
            s["v_pools"][:, y, :, :, b % block] = s["v_pools"][:, x, :, :, a % block].clone()
    return _bits(s)


def _exact_fork(s):
    table, block = s["table"].cpu().numpy().copy(), s["case"]["block"]
    for src, dst, ctx, page in s["forks"].tolist():
        full = ctx // block
        table[dst, :full] = table[src, :full]
        if ctx % block:
            x = int(table[src, full])
            table[dst, full] = page
            s["k_pools"][:, page] = s["k_pools"][:, x].clone()
            s["v_pools"][:, page] = s["v_pools"][:, x].clone()
    return {"table": table, **_bits(s)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"attn": _exact_attn, "layout": _exact_layout, "verify": _exact_verify,
            "compact": _exact_compact, "fork": _exact_fork}[case["kind"]](s)
