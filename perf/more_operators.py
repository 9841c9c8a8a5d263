"""Operators of long and shared contexts over the paged cache.

Five kinds, each one call of the framework:

* ``append``  the fused projection's queries and keys normalised and rotated,
              keys and values written straight into their pages.
* ``bounds``  the smallest and largest value of every feature over the keys of
              the pages that a batch wrote.
* ``select``  the pages that a token reads: the first and the last ones, and of
              the others those whose bounds promise the largest scores.
* ``pages``   attention over the selected pages.
* ``prefix``  attention of requests that have their first tokens in common,
              whose keys and values are read once for all of them.

``own`` chooses between the framework's calls and their plain forms in
elementary torch operations.  A case is a dict of plain values; row lengths
follow from it (``rows_seed``), tensor contents from the seed.
"""

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
THETA, EPS = 1e6, 1e-6


# ---------------------------------------------------------------- the cases

def _append(hq, hkv, d, block, decodes, chunks, chunk, median, rows_seed):
    """``decodes`` requests of one new token behind contexts of log-normal length
    (median), and ``chunks`` ones of ``chunk`` new tokens."""
    return {"kind": "append", "hq": hq, "hkv": hkv, "d": d, "block": block, "decodes": decodes,
            "chunks": chunks, "chunk": chunk, "median": median, "spread": 0.5, "longest": 8192,
            "rows_seed": rows_seed}


def _bounds(hkv, d, block, decodes, chunks, chunk, median, rows_seed):
    return {"kind": "bounds", "hq": hkv, "hkv": hkv, "d": d, "block": block, "decodes": decodes,
            "chunks": chunks, "chunk": chunk, "median": median, "spread": 0.5, "longest": 8192,
            "rows_seed": rows_seed}


def _sparse(kind, hq, hkv, d, block, reqs, most, median, spread, longest, budget, rows_seed):
    """``reqs`` requests of 1 to ``most`` new tokens, each token on ``budget`` pages."""
    return {"kind": kind, "hq": hq, "hkv": hkv, "d": d, "block": block, "decodes": reqs,
            "chunks": 0, "chunk": 0, "most": most, "median": median, "spread": spread,
            "longest": longest, "budget": budget, "rows_seed": rows_seed}


def _prefix(hq, hkv, d, block, groups, reqs, most, common, spread, tail, rows_seed):
    """``groups`` prompts of log-normal length (median ``common``), each continued by
    ``reqs`` requests that have some ``tail`` tokens of their own and 1 to ``most``
    new ones."""
    return {"kind": "prefix", "hq": hq, "hkv": hkv, "d": d, "block": block, "groups": groups,
            "reqs": reqs, "most": most, "common": common, "spread": spread, "tail": tail,
            "rows_seed": rows_seed}


def listed():
    return [
        # one short request's next token on few heads: latency
        {"name": "append-1", **_append(4, 2, 64, 16, 1, 0, 0, 300, 1)},
        # a decode round of the 32/8-head layer
        {"name": "append-64", **_append(32, 8, 128, 16, 64, 0, 0, 1000, 2)},
        # a round of 2,048 tokens: decodes beside two prompt chunks, 64/8 heads
        {"name": "append-2k", **_append(64, 8, 128, 32, 48, 2, 1000, 500, 3)},
        # the pages that a decode round wrote to
        {"name": "bounds-64", **_bounds(8, 128, 16, 64, 0, 0, 500, 4)},
        # long prompts, all their pages
        {"name": "bounds-32k", **_bounds(8, 128, 16, 0, 4, 8192, 500, 5)},
        # one request of a few thousand tokens: latency
        {"name": "select-1", **_sparse("select", 32, 8, 128, 16, 1, 1, 4096, 0.1, 8192, 32, 6)},
        # a decode round over very long contexts: the bounds are the traffic
        {"name": "select-32", **_sparse("select", 32, 8, 128, 16, 32, 1, 32768, 0.3, 50000, 128, 7)},
        # one request's next token on a thousand of its keys
        {"name": "pages-1", **_sparse("pages", 32, 8, 128, 16, 1, 1, 30000, 0.1, 40000, 64, 8)},
        # a decode round of the 64/8-head layer on four thousand keys each
        {"name": "pages-48", **_sparse("pages", 64, 8, 128, 16, 48, 1, 8192, 0.3, 16384, 256, 9)},
        # a few samples of one short prompt on few heads: latency
        {"name": "prefix-4", **_prefix(4, 2, 64, 16, 1, 4, 1, 500, 0.1, 20, 10)},
        # a decode round of requests behind one long system prompt
        {"name": "prefix-32", **_prefix(32, 8, 128, 16, 1, 32, 1, 8192, 0.1, 200, 11)},
        # parallel samples of several prompts on the 64/8-head layer
        {"name": "prefix-8x16", **_prefix(64, 8, 128, 32, 8, 16, 1, 4096, 0.3, 300, 12)},
    ]


HEADS = [(4, 2, 64, 16), (16, 16, 64, 32), (32, 8, 128, 16), (32, 8, 128, 16), (64, 8, 128, 32),
         (8, 1, 128, 32), (16, 8, 128, 32)]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    kind = rng.choice(["append", "append", "bounds", "select", "select", "pages", "pages",
                       "prefix", "prefix"])
    most = {c["kind"]: work(c) for c in listed()}                # the last one of a kind is its largest
    while True:
        hq, hkv, d, block = rng.choice(HEADS)
        seed = rng.randrange(1 << 30)
        if kind == "append":
            case = _append(hq, hkv, d, block, _log_int(rng, 1, 150), rng.choice([0, 0, 1, 2, 3]),
                           _log_int(rng, 2, 1500), _log_int(rng, 20, 2000), seed)
        elif kind == "bounds":
            case = _bounds(hkv, d, block, _log_int(rng, 1, 150), rng.choice([0, 0, 1, 2, 3]),
                           _log_int(rng, 2, 8000), _log_int(rng, 20, 2000), seed)
        elif kind == "prefix":
            case = _prefix(hq, hkv, d, block, _log_int(rng, 1, 12), _log_int(rng, 1, 48),
                           rng.choice([1, 1, 1, 4]), _log_int(rng, 20, 16000),
                           rng.choice([0.1, 0.5]), _log_int(rng, 1, 1000), seed)
        else:
            case = _sparse(kind, hq, hkv, d, block, _log_int(rng, 1, 64), rng.choice([1, 1, 1, 4]),
                           _log_int(rng, 16, 40000), rng.choice([0.1, 0.5, 1.0]), 60000,
                           _log_int(rng, 3, 300), seed)
        w, padded = work(case), 0.0
        if kind in ("select", "pages", "prefix"):                # what the plain form holds at a time
            starts, lens = _rows(case)
            ctx = int((starts + lens).max())
            keys = {"select": ctx / block * 4, "pages": min(case.get("budget", 0) * block, ctx) * 2,
                    "prefix": ctx * 2}[kind]
            padded = hkv * d * keys * (len(lens) if kind == "prefix" else float(lens.sum()))
        if w["bytes"] <= most[kind]["bytes"] and w["flops"] <= most[kind]["flops"] and padded <= 1.5e9:
            return case


# ---------------------------------------------------------------- rows and work

def _rows(case):
    """(cached tokens, new tokens) of every row."""
    rng = np.random.default_rng(case["rows_seed"])
    if case["kind"] == "prefix":
        n = case["groups"] * case["reqs"]
        tail = rng.integers(max(0, case["tail"] // 2), case["tail"] + 1, n)
        return np.repeat(_common(case), case["reqs"]) + tail, rng.integers(1, case["most"] + 1, n)
    n = case["decodes"] + case["chunks"]
    starts = np.round(rng.lognormal(math.log(case["median"]), case["spread"], n)).astype(np.int64)
    lens = rng.integers(1, case.get("most", 1) + 1, n)
    lens[case["decodes"]:] = case["chunk"]
    return np.clip(starts, 1, case["longest"]), lens


def _common(case):
    """Tokens that the requests of each group have in common."""
    rng = np.random.default_rng(case["rows_seed"] + 1)
    return np.maximum(1, np.round(rng.lognormal(math.log(case["common"]), case["spread"],
                                                case["groups"]))).astype(np.int64)


def _last_page(starts, lens, block):
    """The page of every token's own position."""
    return np.concatenate([(s + np.arange(n)) // block for s, n in zip(starts, lens)])


def work(case):
    starts, lens = _rows(case)
    kind, hq, hkv, d, block = (case[k] for k in ("kind", "hq", "hkv", "d", "block"))
    t = float(lens.sum())
    if kind == "append":
        return {"bytes": t * (hq + 2 * hkv) * d * 4.0 + 4.0 * d, "flops": 0.0}
    if kind == "bounds":
        first = starts // block * block                          # a page begun earlier is read again
        pages = (starts + lens - 1) // block - starts // block + 1
        return {"bytes": 2.0 * hkv * d * float((starts + lens - first).sum())
                + 4.0 * hkv * d * float(pages.sum()), "flops": 0.0}
    if kind == "select":
        pages = _last_page(starts, lens, block) + 1.0
        held = (starts + lens - 1) // block + 1.0
        return {"bytes": 4.0 * hkv * d * float(held.sum()) + t * (2.0 * hq * d + 4.0 * hkv * case["budget"]),
                "flops": 4.0 * hq * d * float(pages.sum())}
    if kind == "pages":
        pages = _last_page(starts, lens, block) + 1
        keys = float((np.minimum(pages, case["budget"]) * block).sum())
        return {"bytes": 4.0 * hkv * d * keys + t * (4.0 * hq * d + 4.0 * hkv * case["budget"]),
                "flops": 4.0 * hq * d * keys}
    common, own_keys = _common(case), starts + lens - np.repeat(_common(case), case["reqs"])
    return {"bytes": 4.0 * hkv * d * float(common.sum() + own_keys.sum()) + t * 4.0 * hq * d,
            "flops": 4.0 * hq * d * float((lens * (starts + (lens + 1) / 2)).sum())}


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.bfloat16)


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).to(DEV)


def _empty(*shape, dtype=torch.bfloat16):
    return torch.empty(*shape, dtype=dtype, device=DEV)


def _bytes(n):
    return _empty(max(n, 256), dtype=torch.uint8)


def _table(rng, need, slots):
    """A block table over a pool of sum(need) + 1 pages in random order: row
    slots[i] names need[i] of them, the other entries the last page."""
    pool = int(sum(need)) + 1
    perm = rng.permutation(pool).astype(np.int32)
    table = np.full((int(max(slots)) + 1, int(max(need)) + 1), perm[-1], np.int32)
    at = 0
    for slot, n in zip(slots, need):
        table[slot, :n] = perm[at:at + n]
        at += n
    return table, pool


def _desc(hq, hkv, d, block, pool, table):
    from paper_2606_09061_amd import binding
    return binding.make_desc(hq, hkv, d, block, pool, table.shape[1], table.shape[0],
                             1.0 / math.sqrt(d))


def _keys(g, pool, hkv, block, d):
    """Keys whose pages differ, as those of a text do."""
    return (_randn(g, pool, hkv, 1, d) * 0.7 + _randn(g, pool, hkv, block, d) * 0.7).contiguous()


def _prepare_append(s, g, pool):
    case, t = s["case"], s["t"]
    hq, hkv, d, block = (case[k] for k in ("hq", "hkv", "d", "block"))
    s |= {"qkv": _randn(g, t, (hq + 2 * hkv) * d), "qw": 1 + 0.1 * _randn(g, d),
          "kw": 1 + 0.1 * _randn(g, d), "q": _empty(t, hq, d),
          "kc": _randn(g, pool, hkv, block, d), "vc": _randn(g, pool, hkv, d, block)}


def _prepare_bounds(s, g, pool):
    case = s["case"]
    hkv, d, block = (case[k] for k in ("hkv", "d", "block"))
    s |= {"kc": _keys(g, pool, hkv, block, d),
          "bounds": torch.zeros(pool, hkv, 2, d, dtype=torch.bfloat16, device=DEV)}


def _prepare_select(s, g, pool):
    case, t = s["case"], s["t"]
    hq, hkv, d, block = (case[k] for k in ("hq", "hkv", "d", "block"))
    k = _keys(g, pool, hkv, block, d)
    s |= {"q": _randn(g, t, hq, d), "bounds": torch.stack([k.amin(2), k.amax(2)], 2).contiguous(),
          "pages": _empty(t, hkv, case["budget"], dtype=torch.int32)}
    if own:
        from paper_2606_09061_amd import cache
        s["ws"] = _bytes(cache.page_select_workspace_bytes(s["desc"], s["rows"], case["budget"]))


def _prepare_pages(s, g, pool):
    """The first page, the last one and a random part of those between, rising."""
    case, t = s["case"], s["t"]
    hq, hkv, d, block, budget = (case[k] for k in ("hq", "hkv", "d", "block", "budget"))
    last = torch.from_numpy(_last_page(s["rows"][:, 1], s["rows"][:, 2], block)).to(DEV)
    width = max(int(last.max()) + 1, budget)
    i = torch.arange(width, device=DEV)
    rank = torch.rand(t, hkv, width, generator=g, device=DEV)
    rank = torch.where((i == 0) | (i == last[:, None, None]), 2.0, rank)
    rank = torch.where(i > last[:, None, None], -1.0, rank)
    top, at = rank.topk(budget, -1)
    at = torch.where(top < 0, width, at).sort(-1).values
    s |= {"q": _randn(g, t, hq, d), "kc": _keys(g, pool, hkv, block, d),
          "vc": _randn(g, pool, hkv, d, block), "out": _empty(t, hq, d),
          "pages": torch.where(at == width, -1, at).int().contiguous()}
    if own:
        from paper_2606_09061_amd import cache
        s["ws"] = _bytes(cache.page_attn_workspace_bytes(s["desc"], s["rows"], budget))


def _prepare_prefix(s, g, pool):
    case, t = s["case"], s["t"]
    hq, hkv, d, block = (case[k] for k in ("hq", "hkv", "d", "block"))
    s |= {"q": _randn(g, t, hq, d), "kc": _keys(g, pool, hkv, block, d),
          "vc": _randn(g, pool, hkv, d, block), "out": _empty(t, hq, d),
          "groups": np.stack([np.arange(case["groups"]) * case["reqs"],
                              np.full(case["groups"], case["reqs"]), _common(case)],
                             1).astype(np.int32)}
    if own:
        from paper_2606_09061_amd import cache
        s["ws"] = _bytes(cache.prefix_attn_workspace_bytes(s["desc"], s["rows"], s["groups"]))


def prepare(case, seed):
    starts, lens = _rows(case)
    rng, n, block = np.random.default_rng(int(seed)), len(lens), case["block"]
    slots, need = rng.permutation(n), -(-(starts + lens) // block)
    if case["kind"] == "prefix":                                 # full pages in common are shared
        shared = _common(case) // block
        first = np.arange(n) % case["reqs"] == 0
        keep = np.repeat(shared, case["reqs"])
        table, pool = _table(rng, np.concatenate([need - np.where(first, 0, keep), [0]]),
                             np.concatenate([slots, [n - 1]]))
        wide = np.full((n, int(need.max()) + 1), table[0, -1], np.int32)
        for r, slot in enumerate(slots):
            if first[r]:
                wide[slot, :need[r]] = table[slot, :need[r]]
            else:
                wide[slot, :keep[r]] = table[slots[r - r % case["reqs"]], :keep[r]]
                wide[slot, keep[r]:need[r]] = table[slot, :need[r] - keep[r]]
        table = wide
    else:
        table, pool = _table(rng, need, slots)
    rows = np.stack([slots, starts, lens, starts + lens], 1).astype(np.int32)
    s = {"case": case, "rows": rows, "table": _i32(table), "t": int(lens.sum()),
         "scale": 1.0 / math.sqrt(case["d"])}
    if own:
        s["desc"] = _desc(case["hq"], case["hkv"], case["d"], block, pool, table)
    {"append": _prepare_append, "bounds": _prepare_bounds, "select": _prepare_select,
     "pages": _prepare_pages, "prefix": _prepare_prefix}[case["kind"]](s, _gen(seed), pool)
    return s


# ---------------------------------------------------------------- plain forms

def _tokens(rows):
    """(row, position) of every new token, on the GPU."""
    start, n = rows[:, 1].astype(np.int64), rows[:, 2].astype(np.int64)
    row = np.repeat(np.arange(len(rows)), n)
    at = np.arange(int(n.sum())) - np.repeat(np.cumsum(n) - n, n)
    return torch.from_numpy(row).to(DEV), torch.from_numpy(start[row] + at).to(DEV)


def _rotated(x, w, pos):
    """x [T, H, D] normalised per head and rotated, in 32 bits; angles in 64."""
    half = x.shape[-1] // 2
    x = x.float()
    x = x / (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * w.float()
    turn = THETA ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
    angle = pos.double()[:, None, None] * turn
    c, s = angle.cos().float(), angle.sin().float()
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * c - b * s, b * c + a * s], -1).bfloat16()


def _plain_append(s):
    hq, hkv, d, block = (s["case"][k] for k in ("hq", "hkv", "d", "block"))
    row, pos = _tokens(s["rows"])
    q, k, v = s["qkv"].view(-1, hq + 2 * hkv, d).split([hq, hkv, hkv], 1)
    page = s["table"][_i32(s["rows"][:, 0]).long()[row], pos // block].long()
    s["q"].copy_(_rotated(q, s["qw"], pos))
    s["kc"][page, :, pos % block] = _rotated(k, s["kw"], pos)
    s["vc"][page, :, :, pos % block] = v
    return {"q": s["q"], "k": s["kc"], "v": s["vc"]}


def _plain_bounds(s):
    block = s["case"]["block"]
    slot, start, _, ctx = _i32(s["rows"]).long().unbind(1)
    first, pages = start // block, (ctx - 1) // block - start // block + 1
    n = int(((s["rows"][:, 3] - 1) // block - s["rows"][:, 1] // block + 1).max())
    page = first[:, None] + torch.arange(n, device=DEV)
    real = torch.arange(n, device=DEV) < pages[:, None]
    page = torch.where(real, page, first[:, None])[real]
    slot, ctx = slot[:, None].expand_as(real)[real], ctx[:, None].expand_as(real)[real]
    at = s["table"][slot, page].long()
    k = s["kc"][at].float()
    held = (page[:, None] * block + torch.arange(block, device=DEV) < ctx[:, None])[:, None, :, None]
    lo, hi = k.masked_fill(~held, math.inf).amin(2), k.masked_fill(~held, -math.inf).amax(2)
    s["bounds"][at] = torch.stack([lo, hi], 2).bfloat16()
    return {"bounds": s["bounds"]}


def _plain_select(s):
    hq, hkv, d, block, budget = (s["case"][k] for k in ("hq", "hkv", "d", "block", "budget"))
    row, pos = _tokens(s["rows"])
    n = int((s["rows"][:, 3].max() - 1) // block) + 1
    at = s["table"][_i32(s["rows"][:, 0]).long()[row], :n].long()
    lo, hi = s["bounds"][at].double().permute(0, 2, 3, 4, 1).unbind(2)   # [T, hkv, d, n]
    q = s["q"].double().view(-1, hkv, hq // hkv, d)
    score = torch.matmul(q.clamp(min=0), hi.contiguous()) + torch.matmul(q.clamp(max=0), lo.contiguous())
    score = score.amax(2)
    i, last = torch.arange(n, device=DEV), (pos // block)[:, None, None]
    score = torch.where((i == 0) | (i == last), math.inf, score).masked_fill(i > last, -math.inf)
    value, order = score.sort(dim=-1, descending=True, stable=True)
    chosen = torch.where(value == -math.inf, n, order)[..., :budget].sort(-1).values
    s["pages"].fill_(-1)
    s["pages"][..., :chosen.shape[-1]] = torch.where(chosen == n, -1, chosen).int()
    return {"pages": s["pages"]}


def _attention(q, k, v, seen, scale):
    """q [N, hkv, M, D], k and v [N, hkv, keys, D], seen broadcastable to the scores."""
    x = (torch.matmul(q, k.transpose(2, 3).contiguous()) * scale).masked_fill(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    w = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = w.sum(-1, keepdim=True)
    return torch.matmul(w, v) / torch.where(total == 0, 1.0, total)


def _plain_pages(s):
    hq, hkv, d, block, budget = (s["case"][k] for k in ("hq", "hkv", "d", "block", "budget"))
    row, pos = _tokens(s["rows"])
    slot, t = _i32(s["rows"][:, 0]).long()[row], s["t"]
    page = s["pages"].long()
    at = s["table"][slot[:, None, None], page.clamp(min=0)].long()
    h = torch.arange(hkv, device=DEV)[:, None]
    k = s["kc"][at, h].float().view(t, hkv, budget * block, d)
    v = s["vc"][at, h].float().transpose(3, 4).reshape(t, hkv, budget * block, d)
    key = page[..., None] * block + torch.arange(block, device=DEV)
    seen = ((page >= 0)[..., None] & (key <= pos[:, None, None, None])).view(t, hkv, 1, -1)
    v = torch.where(seen.transpose(2, 3), v, 0.0)
    o = _attention(s["q"].float().view(t, hkv, -1, d), k, v, seen, s["scale"])
    s["out"].copy_(o.reshape(t, hq, d))
    return {"out": s["out"]}


def _plain_prefix(s):
    hq, hkv, d, block = (s["case"][k] for k in ("hq", "hkv", "d", "block"))
    slot, start, n, ctx = _i32(s["rows"]).long().unbind(1)
    m, keys = int(s["rows"][:, 2].max()), -(-int(s["rows"][:, 3].max()) // block) * block
    j, first = torch.arange(m, device=DEV), torch.cumsum(n, 0) - n
    j = torch.minimum(j, n[:, None] - 1)                         # places past a row repeat its last token
    node, r = first[:, None] + j, len(s["rows"])
    at = s["table"][slot, :keys // block].long()
    k = s["kc"][at].float().permute(0, 2, 1, 3, 4).reshape(r, hkv, keys, d)
    v = s["vc"][at].float().permute(0, 2, 1, 4, 3).reshape(r, hkv, keys, d)
    i, g = torch.arange(keys, device=DEV), hq // hkv
    v = torch.where((i < ctx[:, None])[:, None, :, None], v, 0.0)
    q = s["q"][node].float().view(r, m, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(r, hkv, m * g, d)
    seen = (i <= (start[:, None] + j)[..., None]).repeat_interleave(g, 1)[:, None]
    o = _attention(q, k, v, seen, s["scale"])
    o = o.view(r, hkv, m, g, d).permute(0, 2, 1, 3, 4).reshape(-1, hq, d)
    s["out"][node.reshape(-1)] = o.bfloat16()
    return {"out": s["out"]}


# ---------------------------------------------------------------- one pass

def _own(s):
    from paper_2606_09061_amd import cache
    kind = s["case"]["kind"]
    if kind == "append":
        cache.qkv_append(s["desc"], s["qkv"], s["qw"], s["kw"], s["rows"], s["q"], s["kc"], s["vc"],
                         s["table"], THETA, EPS)
        return {"q": s["q"], "k": s["kc"], "v": s["vc"]}
    if kind == "bounds":
        cache.page_bounds(s["desc"], s["kc"], s["table"], s["rows"], s["bounds"])
        return {"bounds": s["bounds"]}
    if kind == "select":
        cache.page_select(s["desc"], s["q"], s["bounds"], s["table"], s["rows"], s["pages"], 1, 1,
                          s["ws"])
        return {"pages": s["pages"]}
    if kind == "pages":
        cache.page_attn(s["desc"], s["q"], s["kc"], s["vc"], s["table"], s["pages"], s["rows"],
                        s["out"], s["ws"])
        return {"out": s["out"]}
    cache.prefix_attn(s["desc"], s["q"], s["kc"], s["vc"], s["table"], s["rows"], s["groups"],
                      s["out"], s["ws"])
    return {"out": s["out"]}


def run(s):
    if own:
        return _own(s)
    return {"append": _plain_append, "bounds": _plain_bounds, "select": _plain_select,
            "pages": _plain_pages, "prefix": _plain_prefix}[s["case"]["kind"]](s)


# ---------------------------------------------------------------- 64-bit results

def _turned(x, w, pos):
    """One head row [H, D] in 64 bits: norm, then the rotation as a complex product."""
    x = x.double()
    x = x * w.double() * torch.rsqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS)
    half = x.shape[-1] // 2
    power = torch.arange(half, dtype=torch.float64, device=x.device) * (-2.0 / x.shape[-1])
    z = torch.complex(x[..., :half], x[..., half:])
    z = z * torch.polar(torch.ones_like(power), pos * torch.exp(power * math.log(THETA)))
    return torch.cat([z.real, z.imag], -1)


def _exact_append(s):
    hq, hkv, d, block = (s["case"][k] for k in ("hq", "hkv", "d", "block"))
    x = s["qkv"].view(-1, hq + 2 * hkv, d)
    q = torch.empty(s["t"], hq, d, dtype=torch.float64, device=DEV)
    k, v, t = s["kc"].double(), s["vc"].double(), 0
    table = s["table"].cpu().numpy()
    for slot, start, n, _ in s["rows"].tolist():
        for p in range(start, start + n):
            q[t] = _turned(x[t, :hq], s["qw"], float(p))
            b = int(table[slot, p // block])
            k[b, :, p % block] = _turned(x[t, hq:hq + hkv], s["kw"], float(p))
            v[b, :, :, p % block] = x[t, hq + hkv:].double()
            t += 1
    return {"q": q, "k": k, "v": v}


def _exact_bounds(s):
    block, table = s["case"]["block"], s["table"].cpu().numpy()
    out = s["bounds"].double()
    for slot, start, _, ctx in s["rows"].tolist():
        for p in range(start // block, (ctx - 1) // block + 1):
            b = int(table[slot, p])
            k = s["kc"][b, :, :min(block, ctx - p * block)].double()
            out[b, :, 0], out[b, :, 1] = k.min(1).values, k.max(1).values
    return {"bounds": out}


def _exact_select(s):
    hq, hkv, d, block, budget = (s["case"][k] for k in ("hq", "hkv", "d", "block", "budget"))
    out, t, table = np.full((s["t"], hkv, budget), -1, np.int32), 0, s["table"].cpu().numpy()
    for slot, start, n, _ in s["rows"].tolist():
        for p in range(start, start + n):
            last = p // block
            b = torch.from_numpy(table[slot, :last + 1].astype(np.int64)).to(DEV)
            for h in range(hkv):
                lo, hi = s["bounds"][b, h].double().unbind(1)
                best = [torch.maximum(x * lo, x * hi).sum(1)
                        for x in s["q"][t, h * hq // hkv:(h + 1) * hq // hkv].double()]
                score = torch.stack(best).max(0).values.cpu().numpy()
                score[0] = score[last] = np.inf
                order = np.lexsort((np.arange(last + 1), -score))[:budget]
                out[t, h, :len(order)] = np.sort(order)
            t += 1
    return {"pages": out}


def _head(q, k, v, scale):
    x = k.double() @ q.double() * scale
    w = torch.exp(x - x.max())
    return (w[:, None] * v.double()).sum(0) / w.sum()


def _exact_pages(s):
    hq, hkv, d, block = (s["case"][k] for k in ("hq", "hkv", "d", "block"))
    out, t = torch.zeros(s["t"], hq, d, dtype=torch.float64, device=DEV), 0
    pages, table = s["pages"].cpu().numpy(), s["table"].cpu().numpy()
    for slot, start, n, _ in s["rows"].tolist():
        for p in range(start, start + n):
            for h in range(hkv):
                mine = pages[t, h][pages[t, h] >= 0]
                b = torch.from_numpy(table[slot, mine].astype(np.int64)).to(DEV)
                there = torch.from_numpy(
                    ((mine[:, None] * block + np.arange(block)) <= p).reshape(-1)).to(DEV)
                k = s["kc"][b, h].reshape(-1, d)[there]
                v = s["vc"][b, h].transpose(1, 2).reshape(-1, d)[there]
                for e in range(h * hq // hkv, (h + 1) * hq // hkv):
                    out[t, e] = _head(s["q"][t, e], k, v, s["scale"])
            t += 1
    return {"out": out}


def _exact_prefix(s):
    hq, hkv, d, block = (s["case"][k] for k in ("hq", "hkv", "d", "block"))
    out, t = torch.zeros(s["t"], hq, d, dtype=torch.float64, device=DEV), 0
    for slot, start, n, ctx in s["rows"].tolist():
        b = s["table"][slot, :-(-ctx // block)].long()
        for h in range(hkv):
            k = s["kc"][b, h].reshape(-1, d)
            v = s["vc"][b, h].transpose(1, 2).reshape(-1, d)
            for j in range(n):
                seen = start + j + 1
                for e in range(h * hq // hkv, (h + 1) * hq // hkv):
                    out[t + j, e] = _head(s["q"][t + j, e], k[:seen], v[:seen], s["scale"])
        t += n
    return {"out": out}


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "bounds": _exact_bounds, "select": _exact_select,
            "pages": _exact_pages, "prefix": _exact_prefix}[case["kind"]](s)
