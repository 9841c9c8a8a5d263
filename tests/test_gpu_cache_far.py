"""Long and shared contexts past the sizes at which the kernels change: selection of
more pages than a workgroup holds, common prefixes that are read past the caches."""

import math

import numpy as np
import pytest
import torch

import paper_2606_09061_amd as cp
import test_gpu_cache as base
from paper_2606_09061_amd import cache
from test_gpu_cache import DEV, Case, Select, same_bits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pages", [16384, 16385, 16640, 40001])
@pytest.mark.parametrize("n_pages,n_first,n_last", [(1, 0, 0), (300, 1, 1), (64, 30, 34), (4096, 0, 3)])
@pytest.mark.parametrize("pool", [None, 40, 1], ids=["distinct", "shared", "equal"])
def test_select_of_more_pages_than_a_workgroup_holds(pages, n_pages, n_first, n_last, pool):
    """Beside rows that choose from few pages, and from none."""
    rows = [(16 * pages - 5, 1), (700, 3), (0, 1)]
    s = Select(4, 2, 64, 16, rows, pages + n_pages, pool=pool)
    s.table[0, 3::97] = -1
    s.table[0, 5::301] = s.bounds.shape[0]
    s.check(n_pages, n_first, n_last)


def _attn64(q, k, v, table, rows, scale, pages=None):
    """oracle.cache.attn over all keys with its sums on the GPU, in 64 bits."""
    assert pages is None
    q, k, v = (torch.from_numpy(x).to(DEV) for x in (q, k, v))
    hkv, block = k.shape[1], k.shape[2]
    group = q.shape[1] // hkv
    res = torch.zeros(3, *q.shape, dtype=torch.float64, device=DEV)
    for t, r, p in base.ref.tokens(rows):
        b = torch.from_numpy(table[rows[r][0], :p // block + 1]).to(DEV).long()
        for h in range(hkv):
            kk = k[b, h].reshape(-1, k.shape[3])[:p + 1]
            vv = v[b, h].transpose(1, 2).reshape(-1, k.shape[3])[:p + 1]
            for e in range(h * group, (h + 1) * group):
                w = torch.softmax((kk * q[t, e]).sum(1) * scale, 0)[:, None]
                o = (w * vv).sum(0)
                res[0, t, e], res[1, t, e] = o, (w * (vv - o).abs()).sum(0)
                res[2, t, e] = (w * vv.abs()).sum(0)
    return res.cpu().numpy()


def test_the_sums_on_the_gpu_are_the_oracles():
    c = Case(8, 2, 64, 16, [(70, 2), (90, 1)], 1, groups=[(0, 2, 64)])
    args = [base.f64(x) for x in (c.q, c.k, c.v)] + [c.table, c.rows.tolist(), c.scale]
    for a, b in zip(_attn64(*args), base.ref.attn(*args)):
        assert np.allclose(a, b, rtol=1e-11, atol=1e-14)


# Heads, and (rows, tokens in common) of three groups: more than 32 (token, q head) rows
# per kv head, which are read past the caches as all the common K and V are more than
# 64 MB; more than 128 of them, through the caches; and few.
LARGE = [(8, 1, 128, 16, [(5, 100000), (17, 20003), (3, 6001)]),
         (32, 4, 64, 32, [(6, 50001), (20, 10000), (4, 4005)]),
         (8, 8, 128, 32, [(40, 14000), (130, 1700), (3, 1800)]),
         (4, 2, 128, 16, [(31, 60003), (70, 3000), (5, 2040)])]


@pytest.mark.parametrize("hq,hkv,d,block,sizes", LARGE)
def test_prefix_attn_reads_large_prefixes_past_the_caches(hq, hkv, d, block, sizes, monkeypatch):
    """Scores four times as far apart as usual: a few dozen keys have most of a
    token's weight, so that an output is far above the bound of its sums' error."""
    assert sum(n // block * block for _, n in sizes) * hkv * d * 4 > 64e6
    rows, groups = [], []
    for n, common in sizes:
        groups.append((len(rows), n, common))
        rows += [(common + 11 * i % 40, 1 + (i == 1)) for i in range(n)]
    c = Case(hq, hkv, d, block, rows, d + block, groups=groups)
    c.scale = 4 / math.sqrt(d)
    monkeypatch.setattr(base.ref, "attn", _attn64)
    out = c.prefix()
    c.check(out, f"{hq}/{hkv} d {d} block {block}")
    assert same_bits([out], [c.prefix()])


def test_prefix_offsets_beyond_32_bits():
    """Pools of more than 2^31 values, groups of all three kinds at their end: the same
    bits as in small pools."""
    hq, hkv, d, block, far = 64, 8, 128, 16, 140000
    rows = ([(16000 + i, 1 + i % 2) for i in range(6)] + [(1700 + i, 1) for i in range(20)]
            + [(900, 2), (1500, 1)])
    c = Case(hq, hkv, d, block, rows, 17, groups=[(0, 6, 16000), (6, 20, 1700), (26, 2, 900)])
    g, results = c.gpu(), []
    k = torch.empty(far + len(g["k"]), hkv, block, d, dtype=torch.bfloat16, device=DEV)
    v = torch.empty(far + len(g["v"]), hkv, d, block, dtype=torch.bfloat16, device=DEV)
    assert k[:far].numel() > 1 << 31
    k[far:], v[far:] = g["k"], g["v"]
    for kk, vv, bt in ((g["k"], g["v"], g["bt"]), (k, v, g["bt"] + far)):
        desc = cp.make_desc(hq, hkv, d, block, len(kk), *c.table.shape[::-1], c.scale)
        out = c.new_out()
        cache.prefix_attn(desc, g["q"], kk, vv, bt, c.rows, c.groups, out)
        results.append(out)
    assert torch.isfinite(results[0].float()).all() and same_bits(results[:1], results[1:])
    del k, v
    torch.cuda.empty_cache()
