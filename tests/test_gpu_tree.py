"""Drafted trees and forks on the GPU against the 64-bit oracle (oracle/tree.py)."""

import math

import numpy as np
import pytest
import torch

import paper_2606_09061_amd as cp
from oracle import tree as ref
from paper_2606_09061_amd import tree

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN = float("nan")


def bf16(x):
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16)


def f64(t):
    return t.detach().cpu().double().numpy()


def parents_of(lens, rng, kind="random"):
    out = []
    for n in lens:
        j = np.arange(n)
        if kind == "chain":
            p = j - 1
        elif kind == "star":
            p = np.where(j == 0, -1, 0)
        else:
            p = np.where(j == 0, -1, np.floor(rng.random(n) * np.maximum(j, 1)))
        out.append(p.astype(np.int32))
    return np.concatenate(out) if out else np.zeros(0, np.int32)


class Case:
    """Rows [(start, nodes)] over randomly placed pages; every slot that no row
    owns, and every page that none names, holds NaN."""

    def __init__(self, hq, hkv, d, block, rows, seed, spare=3, kind="random"):
        rng = self.rng = np.random.default_rng(seed)
        self.hq, self.hkv, self.d, self.block = hq, hkv, d, block
        n = len(rows)
        slots = rng.permutation(n + 2)[:n]
        self.rows = np.array([(s, a, c, a + c) for s, (a, c) in zip(slots, rows)], np.int32)
        need = [-(-(a + c) // block) for a, c in rows]
        nb = sum(need) + spare
        perm = rng.permutation(nb).astype(np.int32)
        self.table = np.full((n + 2, max(need + [1]) + 1), perm[-1], np.int32)
        self.free = perm[sum(need):]
        k = np.full((nb, hkv, block, d), NAN, np.float32)
        v = np.full((nb, hkv, d, block), NAN, np.float32)
        at = 0
        for i, (a, c) in enumerate(rows):
            b = perm[at:at + need[i]]
            self.table[slots[i], :need[i]] = b
            at += need[i]
            kk = rng.standard_normal((need[i], hkv, block, d)).astype(np.float32)
            vv = rng.standard_normal((need[i], hkv, d, block)).astype(np.float32)
            past = (np.arange(need[i] * block) >= a + c).reshape(need[i], block)
            kk[np.broadcast_to(past[:, None, :, None], kk.shape)] = NAN
            vv[np.broadcast_to(past[:, None, None, :], vv.shape)] = NAN
            k[b], v[b] = kk, vv
        self.t = int(self.rows[:, 2].sum())
        self.words = max(1, -(-max([c for _, c in rows] + [1]) // 64))
        self.parents = parents_of(self.rows[:, 2], rng, kind)
        self.mask, self.pos = ref.layout(self.parents, self.rows, self.words)
        self.q = bf16(rng.standard_normal((self.t, hq, d)))
        self.k, self.v = bf16(k), bf16(v)
        self.scale = 1.0 / math.sqrt(d)

    def desc(self):
        return cp.make_desc(self.hq, self.hkv, self.d, self.block, self.k.shape[0],
                            self.table.shape[1], self.table.shape[0], self.scale)

    def gpu(self):
        return dict(q=self.q.to(DEV), k=self.k.to(DEV), v=self.v.to(DEV),
                    bt=torch.from_numpy(self.table).to(DEV),
                    mask=torch.from_numpy(self.mask.view(np.int64)).to(DEV))

    def run(self, g=None, ws=None, out=None, stream=None):
        g = g or self.gpu()
        if out is None:
            out = torch.full((self.t, self.hq, self.d), 7.0, dtype=torch.bfloat16, device=DEV)
        tree.attn(self.desc(), g["q"], g["k"], g["v"], g["bt"], g["mask"], self.rows, out, ws,
                  stream)
        return out

    def check(self, out, what=""):
        """|out - o| <= 2^-8 |o| (the output's rounding) + 2^-8 (1 + 2^-7) spread (the
        weights', summed as rounded) + the fp32 part: a score is a sum of d
        products whose sizes add up to at most top = |q| |k| scale, so it is off
        by (d + 8) 2^-23 top with the factors' own roundings, which moves the
        weights by as much, relatively; sums of ctx weighted values in fp32, and
        the exponentials' and the merge's few ulps."""
        o, spread, size = ref.attn(f64(self.q), f64(self.k), f64(self.v), self.table, self.mask,
                                   self.rows, self.scale)
        got = f64(out)
        fine = np.isfinite(o)
        assert np.array_equal(np.isfinite(got), fine), what
        assert np.array_equal(np.isnan(got), np.isnan(o)), what
        assert np.array_equal(got[~fine & ~np.isnan(o)], o[~fine & ~np.isnan(o)]), what
        def longest(x, axis):                       # of the finite vectors along axis
            n = np.linalg.norm(x, axis=axis)
            return n[np.isfinite(n)].max(initial=0)

        top = longest(f64(self.q), -1) * longest(f64(self.k), -1) * self.scale
        ctx = int(self.rows[:, 3].max(initial=0))
        tol = (2.0 ** -8 * np.abs(o) + 2.0 ** -8 * (1 + 2.0 ** -7) * spread
               + 2 * (self.d + 8) * 2.0 ** -23 * top * spread
               + (2 * ctx + 64) * 2.0 ** -23 * size + 1e-30)
        with np.errstate(invalid="ignore"):
            bad = fine & (np.abs(got - o) > tol)
        with np.errstate(invalid="ignore"):
            worst = np.nanmax(np.where(fine, np.abs(got - o) / tol, 0), initial=0)
        print(f"  {what}: worst error {worst:.3f} of the bound", flush=True)
        assert not bad.any(), (what, worst, np.argwhere(bad)[:5])


HEADS = [(1, 1), (4, 2), (8, 2), (8, 1), (5, 5), (16, 2), (12, 3)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("hq,hkv", HEADS)
def test_attn_matches_the_oracle(hq, hkv, d, block):
    rows = [(37, 5), (0, 1), (0, 9), (64, 17), (300, 2), (1, 40), (31, 0), (15, 1), (129, 64)]
    c = Case(hq, hkv, d, block, rows, 100 * hq + hkv + d + block)
    c.check(c.run(), f"{hq}/{hkv} d {d} block {block}")


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127,
                               128, 129, 200, 255, 256])
@pytest.mark.parametrize("hq,hkv,d,block", [(4, 1, 128, 16), (8, 1, 64, 32), (2, 2, 128, 32)])
def test_attn_tree_sizes(n, hq, hkv, d, block):
    c = Case(hq, hkv, d, block, [(70, n), (0, n)], n)
    c.check(c.run(), f"{n} nodes")


@pytest.mark.parametrize("ctx", [1, 2, 15, 16, 17, 31, 32, 33, 47, 63, 64, 65, 127, 128, 129, 255,
                                 256, 257, 511, 513, 1000, 2047, 4100])
@pytest.mark.parametrize("n", [1, 6, 30])
def test_attn_context_lengths(ctx, n):
    c = Case(8, 2, 128, 16, [(ctx, n)], ctx + n)
    c.check(c.run(), f"context {ctx}, {n} nodes")


@pytest.mark.parametrize("hq,hkv,d,block,n", [(4, 1, 128, 16, 3), (8, 1, 128, 32, 70),
                                              (1, 1, 64, 16, 1), (2, 1, 64, 32, 20)])
def test_attn_long_context_few_rows(hq, hkv, d, block, n):
    c = Case(hq, hkv, d, block, [(40000, n), (9, 2)], n)
    c.check(c.run(), f"{n} nodes after 40,000 keys")


@pytest.mark.parametrize("kind", ["chain", "star"])
def test_attn_chains_and_stars(kind):
    c = Case(8, 2, 128, 16, [(50, 70), (3, 33), (0, 200)], 5, kind=kind)
    c.check(c.run(), kind)


def test_attn_any_mask_and_nodes_that_see_nothing():
    """Masks that are no tree, bits past the row's nodes, nodes without a key
    (zeros) next to others in the same tile."""
    c = Case(8, 2, 128, 16, [(0, 40), (20, 70), (0, 1), (0, 130), (0, 3)], 6)
    c.mask = c.rng.integers(0, 1 << 63, c.mask.shape, dtype=np.int64).view(np.uint64) * np.uint64(2)
    c.mask ^= c.rng.integers(0, 2, c.mask.shape).astype(np.uint64)
    c.mask[0:40:3] = 0
    c.mask[110] = 0
    c.mask[113:240:2] = 0
    c.mask[-2] = 0
    out = c.run()
    c.check(out, "masks")
    assert (out[0:40:3] == 0).all() and (out[113:240:2] == 0).all()


@pytest.mark.parametrize("start", [0, 5, 100, 700])
@pytest.mark.parametrize("hq,hkv,n", [(4, 1, 5), (8, 1, 60), (2, 2, 100)])
def test_attn_what_a_node_does_not_see_does_not_touch_it(start, hq, hkv, n):
    """NaN and infinities in the K and V of some nodes reach those that see them only."""
    c = Case(hq, hkv, 128, 16, [(start, n), (33, 4)], start + n)
    bad = c.rng.choice(np.arange(1, n), max(1, n // 6), replace=False)
    values = [NAN, math.inf, -math.inf]
    for i, j in enumerate(bad):
        p = start + int(j)
        b = int(c.table[c.rows[0, 0], p // 16])
        if i % 4 == 3:
            c.k[b, :, p % 16, i % 128] = values[i // 4 % 3]
        else:
            c.v[b, :, (7 * i) % 128, p % 16] = values[i % 3]
            c.v[b, :, 3, p % 16] = values[(i + 1) % 3]
    o, _, _ = ref.attn(f64(c.q), f64(c.k), f64(c.v), c.table, c.mask, c.rows, c.scale)
    assert np.isfinite(o).any() and not np.isfinite(o).all()
    c.check(c.run(), "poisoned nodes")


@pytest.mark.parametrize("scale", [30.0, 1e-3, 1000.0])
def test_attn_large_scores(scale):
    """Scores far apart: the running maximum moves, most weights vanish.  (The
    scale enters the bound through the scores' own rounding.)"""
    c = Case(8, 2, 64, 16, [(500, 12), (0, 5)], 8)
    c.scale = scale / 8
    c.check(c.run(), f"scale {scale}")


def test_attn_rising_scores_move_the_maximum():
    c = Case(4, 1, 128, 16, [(600, 6)], 9)
    k = f64(c.k)
    b = c.table[c.rows[0, 0]]
    for p in range(606):
        k[b[p // 16], :, p % 16] *= 0.01 * p if p < 300 else 0.01 * (606 - p)
    c.k = bf16(k)
    c.q = bf16(np.abs(f64(c.q)) * 4)
    c.check(c.run(), "rising")


def test_attn_batches_of_many_rows():
    rng = np.random.default_rng(10)
    rows = [(int(rng.integers(0, 200)), int(rng.integers(0, 12))) for _ in range(300)]
    c = Case(4, 2, 64, 16, rows, 11)
    c.check(c.run(), "300 rows")


@pytest.mark.parametrize("n", [2, 70])
def test_attn_splits_behind_a_full_launch(n):
    """More rows than travel in one launch, the long ones, whose ranges are split
    and merged, at its end and behind it."""
    rng = np.random.default_rng(n)
    rows = [(int(rng.integers(0, 40)), 1) for _ in range(118)]
    for r, a in ((3, 5000), (111, 9000), (112, 7001), (117, 6000)):
        rows[r] = (a, n)
    c = Case(4, 1, 128, 16, rows, 21)
    c.check(c.run(), "118 rows")


@pytest.mark.parametrize("lens", [[1] * 7, [1] * 8, [1] * 9, [0, 4] * 8, [0] * 9 + [5]])
def test_attn_numbers_of_rows_around_the_short_argument_block(lens):
    c = Case(8, 2, 64, 16, [(11 * i, n) for i, n in enumerate(lens)], 22)
    c.check(c.run(), f"{len(lens)} rows")


def test_attn_mixed_tree_sizes():
    rows = [(int(a), int(n)) for a, n in zip([10, 900, 0, 333, 77, 2500, 31, 500, 64],
                                             [256, 1, 100, 16, 8, 60, 33, 2, 128])]
    c = Case(16, 2, 128, 32, rows, 12)
    c.check(c.run(), "mixed sizes")


def test_attn_repeats_bit_for_bit_and_reads_no_stale_workspace():
    c = Case(8, 2, 128, 16, [(3000, 20), (5, 3), (900, 90)], 13)
    g = c.gpu()
    need = tree.attn_workspace_bytes(c.desc(), c.rows)
    first = None
    for fill in (0, 255, 127):
        ws = torch.full((need,), fill, dtype=torch.uint8, device=DEV)
        out = c.run(g, ws).view(torch.int16)
        first = out if first is None else first
        assert torch.equal(out, first)


def test_attn_writes_its_rows_only():
    c = Case(8, 2, 128, 16, [(70, 20), (5, 3)], 14)
    need = tree.attn_workspace_bytes(c.desc(), c.rows)
    big = torch.full((c.t + 40, 8, 128), 5.0, dtype=torch.bfloat16, device=DEV)
    ws = torch.full((need + 4096,), 77, dtype=torch.uint8, device=DEV)
    c.check(c.run(ws=ws[:need], out=big[20:20 + c.t]), "inside a larger tensor")
    assert (big[:20] == 5).all() and (big[20 + c.t:] == 5).all() and (ws[need:] == 77).all()


def test_attn_on_another_stream_and_two_at_once():
    a, b = Case(8, 2, 128, 16, [(2000, 30)], 15), Case(4, 1, 64, 32, [(1500, 9), (3, 70)], 16)
    ga, gb = a.gpu(), b.gpu()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    outs = []
    for _ in range(3):
        outs = [a.run(ga, stream=streams[0], out=torch.empty_like(ga["q"])),
                b.run(gb, stream=streams[1].cuda_stream, out=torch.empty_like(gb["q"]))]
    torch.cuda.synchronize()
    a.check(outs[0], "stream 0")
    b.check(outs[1], "stream 1")


def test_attn_from_two_threads():
    """The host's side of a call keeps nothing that another thread's could meet."""
    import threading
    cases = [Case(8, 2, 128, 16, [(3000, 20), (40, 5)], 23), Case(4, 1, 64, 32, [(900, 70)], 24),
             Case(32, 8, 128, 16, [(60 * i, 3) for i in range(30)], 25)]
    gpu = [c.gpu() for c in cases]
    want = [c.run(g) for c, g in zip(cases, gpu)]
    torch.cuda.synchronize()
    bad = []

    def work(c, g, w):
        s = torch.cuda.Stream()
        for _ in range(40):
            out = torch.empty_like(g["q"])
            c.run(g, out=out, stream=s)
            s.synchronize()
            if not torch.equal(out.view(torch.int16), w.view(torch.int16)):
                bad.append(c)

    threads = [threading.Thread(target=work, args=x) for x in zip(cases, gpu, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


@pytest.mark.parametrize("words", [1, 2, 3, 4])
@pytest.mark.parametrize("rows", [[(700, 3), (40, 30)], [(300, 64), (90, 33), (5, 1)]])
def test_attn_masks_wider_than_the_trees(rows, words):
    """Narrow and wide kernels; the words behind a tree's nodes may hold anything."""
    c = Case(8, 1, 128, 16, rows, 26)
    mask = np.full((c.t, words), (1 << 64) - 1, np.uint64)
    mask[:, :1] = c.mask
    for t, n in enumerate(np.repeat(c.rows[:, 2], c.rows[:, 2]).tolist()):
        if n < 64:
            mask[t, 0] |= np.uint64(((1 << 64) - 1) >> n << n)
    g = c.gpu()
    g["mask"] = torch.from_numpy(mask.view(np.int64)).to(DEV)
    c.check(c.run(g), f"{words} words")


def test_attn_in_a_graph():
    """Captured once, replayed on new contents of the same buffers."""
    c, other = (Case(8, 2, 128, 16, [(2000, 30), (40, 5)], 17) for _ in range(2))
    other.q, other.k, other.v = (bf16(-0.5 * f64(x)) for x in (c.q, c.k.flip(1), c.v.flip(1)))
    other.mask = np.roll(c.mask, 1, 0)
    g = c.gpu()
    ws = torch.empty(tree.attn_workspace_bytes(c.desc(), c.rows), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(g["q"])
    c.run(g, ws, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(g, ws, out)
    for i in range(4):
        now = (c, other)[i % 2]
        for name, x in now.gpu().items():
            g[name].copy_(x)
        out.fill_(3)
        eager = now.run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), eager.view(torch.int16)), i
        now.check(out, f"replay {i}")


def test_attn_offsets_beyond_32_bits():
    """A pool of more than 2^32 bytes, the request's pages at its end."""
    hkv, d, block = 8, 128, 16
    nb = (1 << 32) // (hkv * d * block * 2) * 2 + 300       # 8.6 GB each of K and V
    c = Case(32, hkv, d, block, [(250, 9)], 19)
    used = c.k.shape[0]
    g = c.gpu()
    k = torch.empty(nb, hkv, block, d, dtype=torch.bfloat16, device=DEV)
    v = torch.empty(nb, hkv, d, block, dtype=torch.bfloat16, device=DEV)
    k[nb - used:], v[nb - used:] = g["k"], g["v"]
    desc = cp.make_desc(32, hkv, d, block, nb, c.table.shape[1], c.table.shape[0], c.scale)
    out = torch.empty_like(g["q"])
    tree.attn(desc, g["q"], k, v, g["bt"] + (nb - used), g["mask"], c.rows, out)
    c.check(out, "far pages")
    # the same pages compacted: node 8 becomes node 1
    layers = tree.kv_layers(desc, [k], [v])
    path = torch.tensor([[0, 8]], dtype=torch.int32, device=DEV)
    tree.kv_compact(layers, g["bt"] + (nb - used), c.rows, path,
                    torch.tensor([2], dtype=torch.int32, device=DEV))
    wk, wv = ref.compact(f64(c.k), f64(c.v), c.table, c.rows, np.array([[0, 8]]), [2])
    assert np.array_equal(f64(k[nb - used:]), wk, equal_nan=True)
    assert np.array_equal(f64(v[nb - used:]), wv, equal_nan=True)


def test_attn_agrees_with_the_mixed_step_on_chains():
    """A chain is a causal chunk: both kernels within their bounds of the oracle,
    and one node is a decode row."""
    c = Case(32, 8, 128, 16, [(500, 20), (90, 1)], 20, kind="chain")
    g = c.gpu()
    ws = torch.empty(cp.workspace_bytes(c.desc(), c.rows), dtype=torch.uint8, device=DEV)
    mixed = torch.empty_like(g["q"])
    cp.attn_mixed(c.desc(), g["q"], g["k"], g["v"], g["bt"], c.rows, mixed, ws)
    c.check(mixed, "mixed step")
    c.check(c.run(g), "tree")


def test_attn_refuses_other_tensors():
    c = Case(8, 2, 128, 16, [(70, 20)], 21)
    g, out = c.gpu(), torch.empty(20, 8, 128, dtype=torch.bfloat16, device=DEV)
    bad = [("q", g["q"].half()), ("q", g["q"][:19]), ("k", g["k"].transpose(2, 3)),
           ("mask", g["mask"].int()), ("mask", g["mask"][:, 0]), ("bt", g["bt"].long()),
           ("q", g["q"].cpu()), ("mask", torch.cat([g["mask"]] * 2, 1)[:, ::2])]
    for name, x in bad:
        with pytest.raises(cp.CpError):
            c.run({**g, name: x}, out=out)
    with pytest.raises(cp.CpError):
        c.run(g, ws=torch.empty(16, dtype=torch.uint8, device=DEV), out=out)
    # a buffer that is not 16-byte aligned
    q = torch.empty(20 * 8 * 128 + 8, dtype=torch.bfloat16, device=DEV)[4:4 + 20 * 8 * 128]
    with pytest.raises(cp.CpError):
        c.run({**g, "q": q.view(20, 8, 128)}, out=out)


def test_bad_pages_are_refused_under_debug(monkeypatch):
    monkeypatch.setenv("CP_DEBUG", "1")
    c = Case(8, 2, 128, 16, [(70, 20)], 22)
    c.check(c.run(), "debug")
    g = c.gpu()
    for page in (-1, c.k.shape[0]):
        bt = g["bt"].clone()
        bt[int(c.rows[0, 0]), 2] = page
        with pytest.raises(cp.CpError) as e:
            c.run({**g, "bt": bt})
        assert e.value.code == -2


# ---------------------------------------------------------------- layout

@pytest.mark.parametrize("lens,words", [([1], 1), ([8], 1), ([64, 1, 0, 63], 1), ([65, 3], 2),
                                        ([256, 255, 1, 129], 4), ([5] * 600, 1), ([0, 0], 1),
                                        ([40, 7], 4)])
@pytest.mark.parametrize("kind", ["random", "chain"])
def test_layout(lens, words, kind):
    rng = np.random.default_rng(sum(lens) + words)
    par = parents_of(lens, rng, kind)
    if kind == "random" and len(par) > 7:        # parents that are none
        par[rng.integers(0, len(par), 4)] = [-7, 300, 255, 1 << 30]
    rows = np.array([(0, a, n, a + n) for a, n in zip(rng.integers(0, 5000, len(lens)), lens)],
                    np.int32)
    t = len(par)
    mask = torch.full((t + 8, words), 99, dtype=torch.int64, device=DEV)
    pos = torch.full((t + 8,), 99, dtype=torch.int32, device=DEV)
    tree.layout(torch.from_numpy(par).to(DEV), rows, mask[:t], pos[:t])
    want = ref.layout(par, rows, words)
    assert np.array_equal(mask[:t].cpu().numpy().view(np.uint64), want[0])
    assert np.array_equal(pos[:t].cpu().numpy(), want[1])
    assert (mask[t:] == 99).all() and (pos[t:] == 99).all()


# ---------------------------------------------------------------- verify

class Drafts:
    def __init__(self, lens, vocab, seed, liked=0.7):
        rng = self.rng = np.random.default_rng(seed)
        self.rows = np.array([(0, 3, n, 3 + n) for n in lens], np.int32).reshape(-1, 4)
        self.t, self.vocab = int(sum(lens)), vocab
        self.parents = parents_of(lens, rng)
        self.tokens = rng.integers(0, max(1, min(vocab, 1000)), self.t).astype(np.int32)
        self.logits = rng.standard_normal((self.t, vocab)).astype(np.float32)
        at = 0
        for n in lens:
            for j in range(1, n):
                if rng.random() < liked:
                    self.logits[at + self.parents[at + j], self.tokens[at + j]] = 9
            at += n
        self.logits = f64(bf16(self.logits))

    def run(self, max_path, logits=None, ws=None, stream=None):
        if logits is None:
            logits = bf16(self.logits).to(DEV)
        R = len(self.rows)
        self.t_ok = torch.full((self.t + 5,), 55, dtype=torch.int32, device=DEV)
        self.out = dict(target=self.t_ok[:self.t],
                        path=torch.full((R, max_path), 55, dtype=torch.int32, device=DEV),
                        n_accepted=torch.full((R,), 55, dtype=torch.int32, device=DEV),
                        next_token=torch.full((R,), 55, dtype=torch.int32, device=DEV))
        tree.verify(logits, torch.from_numpy(self.tokens).to(DEV),
                    torch.from_numpy(self.parents).to(DEV), self.rows, **self.out, ws=ws,
                    stream=stream)
        return self.out

    def check(self, out, max_path):
        want = ref.verify(self.logits, self.tokens, self.parents, self.rows.tolist(), max_path)
        for name, w in zip(("target", "path", "n_accepted", "next_token"), want):
            assert np.array_equal(out[name].cpu().numpy(), w), name
        assert (self.t_ok[self.t:] == 55).all()


@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 63, 1000, 4097, 8191, 8192, 32001, 151936])
@pytest.mark.parametrize("lens", [[1], [8], [5, 0, 12]])
def test_verify_vocabularies(vocab, lens):
    d = Drafts(lens, vocab, vocab + len(lens))
    d.check(d.run(6), 6)


@pytest.mark.parametrize("lens,max_path", [([256, 200, 1], 256), ([64] * 20, 3), ([1] * 300, 1),
                                           ([3, 0, 0, 9] * 80, 5), ([0, 0], 4)])
def test_verify_trees(lens, max_path):
    d = Drafts(lens, 777, len(lens) + max_path, liked=0.9)
    if d.t > 20:
        d.parents[d.rng.integers(0, d.t, 5)] = [-3, 400, 255, 1 << 30, -1]
    d.check(d.run(max_path), max_path)


def test_verify_long_chains_are_followed_to_the_end():
    d = Drafts([256], 500, 3, liked=0)
    d.parents = np.arange(256, dtype=np.int32) - 1
    d.logits[:] = 0
    d.logits[np.arange(255), d.tokens[1:]] = 1
    out = d.run(256)
    d.check(out, 256)
    assert int(out["n_accepted"][0]) == 256
    d.check(d.run(100), 100)


def test_verify_ties_zeros_infinities_and_nan():
    d = Drafts([12], 5003, 4)
    x = d.logits
    x[0] = -math.inf
    x[1] = 0.0
    x[1, :4000] = -0.0                       # equal to +0: the lowest index
    x[2, [900, 4999, 17]] = 30               # ties
    x[3, [4000, 77]] = NAN
    x[4] = NAN
    x[5, 5002] = math.inf
    x[6, 0] = math.inf
    x[7] = -math.inf
    x[7, 5002] = -1e38
    x[8, 4096] = -NAN
    x[9, [100, 200]] = math.inf
    x[10, 3] = NAN
    x[10, 2] = math.inf
    d.logits = f64(bf16(x))
    g = bf16(x).to(DEV)
    g.view(torch.int16)[8, 4096] = -1        # a NaN with its sign bit set
    out = d.run(4, g)
    d.check(out, 4)
    t = out["target"].tolist()
    assert t[:11] == [0, 0, 17, 77, 0, 5002, 0, 5002, 4096, 100, 3]


@pytest.mark.parametrize("shift", range(8))
@pytest.mark.parametrize("pad", [0, 1, 5, 8])
def test_verify_strides_and_alignments(shift, pad):
    d = Drafts([9, 4], 1003, shift + pad)
    flat = torch.full((13 * (1003 + pad) + 16,), 100.0, dtype=torch.bfloat16, device=DEV)
    g = torch.as_strided(flat, (13, 1003), (1003 + pad, 1), shift)
    g.copy_(bf16(d.logits))
    d.check(d.run(5, g), 5)


def test_verify_is_repeatable_on_a_stream_and_in_a_graph():
    d = Drafts([30, 5], 20000, 6)
    g = bf16(d.logits).to(DEV)
    ws = torch.full((tree.verify_workspace_bytes(d.t, d.vocab),), 255, dtype=torch.uint8, device=DEV)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    d.check(d.run(8, g, ws, s), 8)
    torch.cuda.synchronize()
    out = d.run(8, g, ws)
    tok, par = torch.from_numpy(d.tokens).to(DEV), torch.from_numpy(d.parents).to(DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tree.verify(g, tok, par, d.rows, **out, ws=ws)
    for i in range(3):
        d2 = Drafts([30, 5], 20000, 60 + i)
        g.copy_(bf16(d2.logits))
        tok.copy_(torch.from_numpy(d2.tokens))
        par.copy_(torch.from_numpy(d2.parents))
        for x in out.values():
            x.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        d2.t_ok = d.t_ok
        d.t_ok[d.t:] = 55
        d2.check(out, 8)


@pytest.mark.parametrize("rows", [7, 8, 9, 256, 257])
def test_layout_and_verify_numbers_of_rows(rows):
    """Around the short argument block and the full one; two verifications at
    once, on streams of their own, each with its own workspace."""
    lens = [1 + r % 3 for r in range(rows)]
    a, b = Drafts(lens, 40, rows), Drafts(lens[::-1], 40, rows + 1)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    outs = []
    for x, s in zip((a, b), streams):
        with torch.cuda.stream(s):
            outs.append(x.run(4))
    torch.cuda.synchronize()
    a.check(outs[0], 4)
    b.check(outs[1], 4)


def test_verify_of_the_smallest_numbers():
    """Denormal logits differ, and the smallest one is above both zeros."""
    g = torch.zeros(4, 30, dtype=torch.int16)
    g[0, 7] = 1                     # the smallest positive value
    g[1, :] = -32768                # -0 ...
    g[1, 9] = 0                     # ... equals +0: the first one wins
    g[2, :] = -32768 + 2            # negative denormals
    g[2, 11] = -32768 + 1
    g[3, 4], g[3, 20] = 0x7f, 0x80  # the largest denormal, the smallest normal number
    rows = np.array([(0, 0, 1, 1)] * 4, np.int32)
    i32 = dict(dtype=torch.int32, device=DEV)
    target, count, after = (torch.empty(4, **i32) for _ in range(3))
    tree.verify(g.to(DEV).view(torch.bfloat16), torch.zeros(4, **i32), torch.full((4,), -1, **i32),
                rows, target, torch.empty(4, 2, **i32), count, after)
    assert target.tolist() == after.tolist() == [7, 0, 11, 20] and count.tolist() == [1] * 4


# ---------------------------------------------------------------- the pools

def _layers_of(c, n, seed):
    """Copies of a case's pools with other contents, bits compared as integers."""
    g = torch.Generator().manual_seed(seed)
    ks = [torch.randint(-32768, 32768, c.k.shape, generator=g).to(torch.int16) for _ in range(n)]
    vs = [torch.randint(-32768, 32768, c.v.shape, generator=g).to(torch.int16) for _ in range(n)]
    dev = [[x.to(DEV).view(torch.bfloat16) for x in p] for p in (ks, vs)]
    return ks, vs, dev


def _same(dev, want):
    for x, w in zip(dev, want):
        assert np.array_equal(x.view(torch.int16).cpu().numpy(), w)


@pytest.mark.parametrize("hkv,d,block,layers", [(2, 128, 16, 3), (1, 64, 32, 1), (3, 64, 16, 2),
                                                (2, 128, 32, 70)])
def test_compact(hkv, d, block, layers):
    lens = [40, 1, 0, 256, 17, 33, 8, 20, 5]
    rows = [(int(a), n) for a, n in zip([0, 5, 7, 30, 100, 15, 31, 3, 64], lens)]
    if layers > 8:
        rows, lens = rows[:4], lens[:4]
    c = Case(hkv, hkv, d, block, rows, hkv + d + block)
    path = np.full((len(rows), 60), -1, np.int32)
    count = np.zeros(len(rows), np.int32)
    for r, n in enumerate(lens):
        k = min(60, max(0, n - r % 3))
        path[r, :k] = np.sort(c.rng.choice(n, k, replace=False)) if n else -1
        count[r] = k
    if len(rows) > 8:
        path[4, 3] = path[4, 2]          # does not rise: the path ends there
        path[5, 4] = 33                  # no node of the row
        path[6, 2] = -5
        count[7], count[8] = 1000, -3    # clamped
        path[7, :] = np.arange(60)       # ... and past the row's nodes
    ks, vs, (kd, vd) = _layers_of(c, layers, 7)
    tree.kv_compact(tree.kv_layers(c.desc(), kd, vd), torch.from_numpy(c.table).to(DEV), c.rows,
                    torch.from_numpy(path).to(DEV), torch.from_numpy(count).to(DEV))
    want = [ref.compact(k.numpy(), v.numpy(), c.table, c.rows.tolist(), path, count)
            for k, v in zip(ks, vs)]
    _same(kd, [w[0] for w in want])
    _same(vd, [w[1] for w in want])
    assert any((w[0] != k.numpy()).any() for w, k in zip(want, ks))


def test_compact_leaves_out_moves_over_bad_pages_and_takes_many_rows():
    rows = [(int(a), 6) for a in range(300)]
    c = Case(1, 1, 64, 16, rows, 30)
    path = np.tile(np.array([0, 2, 4, 5], np.int32), (300, 1))
    count = np.full(300, 4, np.int32)
    for r in range(0, 300, 7):
        c.table[c.rows[r, 0], (c.rows[r, 1] + 4) // 16] = [-1, c.k.shape[0], 1 << 30][r % 3]
    ks, vs, (kd, vd) = _layers_of(c, 2, 8)
    tree.kv_compact(tree.kv_layers(c.desc(), kd, vd), torch.from_numpy(c.table).to(DEV), c.rows,
                    torch.from_numpy(path).to(DEV), torch.from_numpy(count).to(DEV))
    want = [ref.compact(k.numpy(), v.numpy(), c.table, c.rows.tolist(), path, count)
            for k, v in zip(ks, vs)]
    _same(kd, [w[0] for w in want])
    _same(vd, [w[1] for w in want])


@pytest.mark.parametrize("hkv,d,block,layers", [(2, 128, 16, 3), (1, 64, 32, 1), (5, 64, 16, 2),
                                                (8, 128, 32, 2), (1, 64, 16, 70)])
def test_fork(hkv, d, block, layers):
    c = Case(hkv, hkv, d, block, [(100, 0), (block, 0), (3, 0), (200, 0)], 31 + layers, spare=8)
    slot = c.rows[:, 0].tolist()
    new = [r for r in range(c.table.shape[0]) if r not in slot]
    table = np.concatenate([c.table, np.full((4, c.table.shape[1]), 2, np.int32)])
    new += [6, 7, 8, 9]
    free = c.free.tolist()
    forks = np.array([(slot[0], new[0], 100, free[0]), (slot[0], new[1], 50, free[1]),
                      (slot[1], new[2], block, -9), (slot[2], new[3], 3, free[2]),
                      (slot[3], new[4], 0, -1), (slot[3], new[5], 199, free[3])], np.int32)
    desc = cp.make_desc(hkv, hkv, d, block, c.k.shape[0], table.shape[1], len(table), 0.1)
    ks, vs, (kd, vd) = _layers_of(c, layers, 9)
    bt = torch.from_numpy(table).to(DEV)
    tree.kv_fork(tree.kv_layers(desc, kd, vd), bt, forks)
    want = [ref.fork(k.numpy(), v.numpy(), table, forks.tolist()) for k, v in zip(ks, vs)]
    assert np.array_equal(bt.cpu().numpy(), want[0][2])
    _same(kd, [w[0] for w in want])
    _same(vd, [w[1] for w in want])


def test_many_forks_and_pages_that_are_none():
    n, block = 300, 16
    c = Case(1, 1, 64, block, [(20, 0)] * n, 32, spare=n)
    table = np.concatenate([c.table, np.zeros((n, c.table.shape[1]), np.int32)])
    for r in range(0, n, 5):
        table[c.rows[r, 0], 1] = [-1, c.k.shape[0]][r % 2]
    forks = np.array([(c.rows[r, 0], n + 2 + r, 20, c.free[r]) for r in range(n)], np.int32)
    desc = cp.make_desc(1, 1, 64, block, c.k.shape[0], table.shape[1], len(table), 0.1)
    ks, vs, (kd, vd) = _layers_of(c, 2, 10)
    bt = torch.from_numpy(table).to(DEV)
    tree.kv_fork(tree.kv_layers(desc, kd, vd), bt, forks)
    want = [ref.fork(k.numpy(), v.numpy(), table, forks.tolist()) for k, v in zip(ks, vs)]
    assert np.array_equal(bt.cpu().numpy(), want[0][2])
    _same(kd, [w[0] for w in want])
    _same(vd, [w[1] for w in want])


@pytest.mark.parametrize("d,block", [(128, 16), (64, 32), (64, 16), (128, 32)])
def test_compact_paths_of_more_than_a_wave(d, block):
    """Paths of up to 256 nodes, whole, with few or many gaps, and ended by an
    entry that does not rise at the border of two groups of 64."""
    rows = [(0, 256), (13, 256), (100, 256), (31, 200), (1, 130), (63, 66), (5, 256)]
    c = Case(2, 2, d, block, rows, d + block)
    n = c.rows[:, 2]
    path = np.full((len(rows), 256), -1, np.int32)
    count = np.zeros(len(rows), np.int32)
    for r, k in enumerate([256, 255, 129, 192, 128, 65, 200]):
        path[r, :k] = np.sort(c.rng.choice(n[r], k, replace=False))
        count[r] = k
    path[3, 64] = path[3, 63]            # the first of the second group does not rise
    path[4, 127] = path[4, 126] - 1      # nor does the last of it here
    path[6, 128:] = -1                   # ends between groups, though more are counted
    ks, vs, (kd, vd) = _layers_of(c, 2, 12)
    tree.kv_compact(tree.kv_layers(c.desc(), kd, vd), torch.from_numpy(c.table).to(DEV), c.rows,
                    torch.from_numpy(path).to(DEV), torch.from_numpy(count).to(DEV))
    want = [ref.compact(k.numpy(), v.numpy(), c.table, c.rows.tolist(), path, count)
            for k, v in zip(ks, vs)]
    _same(kd, [w[0] for w in want])
    _same(vd, [w[1] for w in want])


def test_moves_and_forks_in_a_graph_and_on_two_streams():
    """A fork and a compaction captured once and replayed on new contents, while
    another pair of pools goes through the same calls on a stream of its own."""
    def case(seed):
        c = Case(2, 2, 128, 16, [(21, 40), (70, 12)], 33, spare=6)
        src, new = int(c.rows[0, 0]), [r for r in range(4) if r not in c.rows[:, 0]]
        forks = np.array([(src, new[0], 10, c.free[0]), (src, new[1], 16, -1)], np.int32)
        rng = np.random.default_rng(seed)
        path = np.full((2, 12), -1, np.int32)
        for r, k in enumerate((12, 7)):
            path[r, :k] = np.sort(rng.choice(int(c.rows[r, 2]), k, replace=False))
        return c, forks, path, np.array([12, 7], np.int32), _layers_of(c, 3, seed)

    def expect(c, forks, path, count, pools):
        ks, vs, _ = pools
        bt = ref.fork(ks[0].numpy(), vs[0].numpy(), c.table, forks.tolist())[2]
        out = [ref.fork(k.numpy(), v.numpy(), c.table, forks.tolist())[:2] for k, v in zip(ks, vs)]
        out = [ref.compact(k, v, bt, c.rows.tolist(), path, count) for k, v in out]
        return bt, [o[0] for o in out], [o[1] for o in out]

    c, forks, path, count, (ks, vs, (kd, vd)) = case(1)
    handle = tree.kv_layers(c.desc(), kd, vd)
    bt, p, n = (torch.from_numpy(x).to(DEV) for x in (c.table, path, count))

    def both(handle, bt, p, n, stream=None):
        tree.kv_fork(handle, bt, forks, stream)
        tree.kv_compact(handle, bt, c.rows, p, n, stream)

    both(handle, bt, p, n)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(handle, bt, p, n)
    side = torch.cuda.Stream()
    for i in range(4):
        now, other = case(2 + i), case(20 + i)
        for dst, src in zip(kd + vd, now[4][2][0] + now[4][2][1]):
            dst.copy_(src)
        bt.copy_(torch.from_numpy(c.table))
        p.copy_(torch.from_numpy(now[2]))
        n.copy_(torch.from_numpy(now[3]))
        obt, op, on = (torch.from_numpy(x).to(DEV) for x in (c.table, other[2], other[3]))
        oh = tree.kv_layers(c.desc(), *other[4][2])
        torch.cuda.synchronize()
        graph.replay()
        both(oh, obt, op, on, side)
        torch.cuda.synchronize()
        for got, want in (((bt, kd, vd), expect(*now)), ((obt, *other[4][2]), expect(*other))):
            assert np.array_equal(got[0].cpu().numpy(), want[0]), i
            _same(got[1], want[1])
            _same(got[2], want[2])


def test_pools_that_share_memory_are_refused():
    c = Case(2, 2, 64, 16, [(20, 3)], 34)
    k = torch.zeros(2, *c.k.shape, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros(2, *c.v.shape, dtype=torch.bfloat16, device=DEV)
    tree.kv_layers(c.desc(), list(k), list(v))
    flat = k.view(-1)
    shifted = flat[8:8 + k[0].numel()].view(c.k.shape)
    for ks, vs in (([k[0], k[0]], list(v)), (list(k), [v[1], v[1]]),
                   ([k[0], shifted], list(v)), ([k[0]], [k[0].view(c.v.shape)])):
        with pytest.raises(cp.CpError):
            tree.kv_layers(c.desc(), ks, vs)


# ---------------------------------------------------------------- a round of them together

def test_a_drafted_round():
    """A request is forked; both draft a tree, which is laid out, appended,
    attended, verified and compacted; the next round attends over what was
    kept.  The second round's attention equals that over a cache which only
    ever held the accepted tokens."""
    hq, hkv, d, block, layers, start, vocab = 8, 2, 128, 16, 2, 45, 600
    rng = np.random.default_rng(40)
    lens, r2 = [12, 30], [(0, 45), (1, 45)]
    table = np.array([[3, 9, 1, 7, 12, 0], [0, 0, 0, 5, 2, 0]], np.int32)
    desc = cp.make_desc(hq, hkv, d, block, 14, 6, 2, d ** -0.5)
    ks = [bf16(rng.standard_normal((14, hkv, block, d))).to(DEV) for _ in range(layers)]
    vs = [bf16(rng.standard_normal((14, hkv, d, block))).to(DEV) for _ in range(layers)]
    handle, bt = tree.kv_layers(desc, ks, vs), torch.from_numpy(table).to(DEV)
    tree.kv_fork(handle, bt, [(0, 1, start, 11)])
    rows = np.array([(q, a, n, a + n) for (q, a), n in zip(r2, lens)], np.int32)
    t = sum(lens)
    dr = Drafts(lens, vocab, 41, liked=0.95)
    par, tok = torch.from_numpy(dr.parents).to(DEV), torch.from_numpy(dr.tokens).to(DEV)
    mask = torch.empty(t, 1, dtype=torch.int64, device=DEV)
    pos = torch.empty(t, dtype=torch.int32, device=DEV)
    tree.layout(par, rows, mask, pos)
    k_new, v_new, q = (bf16(rng.standard_normal((layers, t, h, d))).to(DEV)
                       for h in (hkv, hkv, hq))
    ws = torch.empty(cp.workspace_bytes(desc, rows), dtype=torch.uint8, device=DEV)
    outs = []
    for i in range(layers):
        cp.kv_append(desc, k_new[i], v_new[i], ks[i], vs[i], bt, rows, ws)
        outs.append(torch.empty(t, hq, d, dtype=torch.bfloat16, device=DEV))
        tree.attn(desc, q[i], ks[i], vs[i], bt, mask, rows, outs[i])
    got = dr.run(8)
    dr.check(got, 8)
    c = Case.__new__(Case)
    c.hq, c.hkv, c.d, c.block, c.rows, c.scale = hq, hkv, d, block, rows, d ** -0.5
    c.mask, c.table = ref.layout(dr.parents, rows, 1)[0], bt.cpu().numpy()
    for i in range(layers):
        c.q, c.k, c.v = q[i].cpu(), ks[i].cpu(), vs[i].cpu()
        c.check(outs[i], f"layer {i}")
    tree.kv_compact(handle, bt, rows, got["path"], got["n_accepted"])
    count, path = got["n_accepted"].tolist(), got["path"].cpu().numpy()
    assert max(count) > 2
    # the same tokens appended one after another to untouched copies of the pools
    ks2 = [x.clone() for x in ks]
    vs2 = [x.clone() for x in vs]
    first = np.cumsum([0] + lens)
    keep = np.concatenate([first[r] + path[r, :count[r]] for r in range(2)])
    rows3 = np.array([(r, start, count[r], start + count[r]) for r in range(2)], np.int32)
    for i in range(layers):
        cp.kv_append(desc, k_new[i][keep].contiguous(), v_new[i][keep].contiguous(), ks2[i],
                     vs2[i], bt, rows3, ws)
        assert torch.equal(ks[i].view(torch.int16), ks2[i].view(torch.int16))
        assert torch.equal(vs[i].view(torch.int16), vs2[i].view(torch.int16))
    lens2 = [4, 4]
    rows4 = np.array([(r, start + count[r], 4, start + count[r] + 4) for r in range(2)], np.int32)
    dr2 = Drafts(lens2, vocab, 42)
    mask2 = torch.empty(8, 1, dtype=torch.int64, device=DEV)
    tree.layout(torch.from_numpy(dr2.parents).to(DEV), rows4, mask2, pos[:8])
    q2, k2, v2 = (bf16(rng.standard_normal((8, h, d))).to(DEV) for h in (hq, hkv, hkv))
    out2 = torch.empty_like(q2)
    cp.kv_append(desc, k2, v2, ks[0], vs[0], bt, rows4, ws)
    tree.attn(desc, q2, ks[0], vs[0], bt, mask2, rows4, out2)
    c.rows, c.mask = rows4, ref.layout(dr2.parents, rows4, 1)[0]
    c.q, c.k, c.v = q2.cpu(), ks[0].cpu(), vs[0].cpu()
    c.check(out2, "next round")


def test_one_verify_workspace_for_all_batches():
    """Sized for 2,100 nodes, it serves fewer, whose vocabulary is cut into more pieces."""
    vocab = 20000
    ws = torch.empty(tree.verify_workspace_bytes(2100, vocab), dtype=torch.uint8, device=DEV)
    for lens in ([1], [7], [250] * 8, [256] * 8 + [52], [255, 256, 256, 256]):
        d = Drafts(lens, vocab, sum(lens))
        d.check(d.run(5, ws=ws), 5)


def test_all_calls_from_several_threads():
    """Each thread's attention and verification, 40 times, against what the same
    calls give alone; a worker's exception is the test's."""
    from concurrent.futures import ThreadPoolExecutor
    cases = [Case(8, 2, 128, 16, [(3000, 20), (40, 5)], 23), Case(4, 1, 64, 32, [(900, 70)], 24),
             Case(32, 8, 128, 16, [(60 * i, 3) for i in range(30)], 25)]
    work = []
    for i, c in enumerate(cases):
        d, g = Drafts([3, 9, 5 + i], 700 + i, i), c.gpu()
        work.append((c, g, c.run(g), d, {k: x.clone() for k, x in d.run(4).items()}))
    torch.cuda.synchronize()

    def loop(c, g, attended, d, verified):
        s, ends = torch.cuda.Stream(), 0
        logits, tok, par = (torch.as_tensor(x).to(DEV) for x in (bf16(d.logits), d.tokens, d.parents))
        torch.cuda.synchronize()
        for _ in range(40):
            with torch.cuda.stream(s):
                out = c.run(g, out=torch.empty_like(g["q"]))
                got = {k: torch.empty_like(x) for k, x in verified.items()}
                tree.verify(logits, tok, par, d.rows, **got)
            s.synchronize()
            assert torch.equal(out.view(torch.int16), attended.view(torch.int16))
            assert all(torch.equal(got[k], x) for k, x in verified.items())
            ends += 1
        return ends

    with ThreadPoolExecutor(len(work)) as pool:
        assert [f.result(60) for f in [pool.submit(loop, *w) for w in work]] == [40] * len(work)
