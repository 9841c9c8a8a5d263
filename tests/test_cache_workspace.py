"""What the workspaces of libcpcache have to hold for every batch of some sizes, as
include/cp_cache.h states it (host only)."""

import numpy as np
import pytest

import paper_2606_09061_amd as cp
from paper_2606_09061_amd import cache

HEADS = [(1, 1), (4, 2), (8, 1), (12, 3), (16, 16), (32, 8), (64, 8)]


def _desc(hq, hkv, d, block):
    return cp.make_desc(hq, hkv, d, block, 1000, 1 << 20, 2000, 0.1)


def _pages_bound(d, tokens, n_pages):
    return max(256, (4 * d.head_dim + 4) * d.num_q_heads * tokens
               * -(-n_pages * d.block_size // 256))


def _prefix_bound(d, tokens, keys, several):
    more = 16 * d.num_kv_heads // d.num_q_heads if several else 1
    return max(256, (4 * d.head_dim + 4) * d.num_q_heads * tokens * (keys // 256 + 2) * more)


def test_a_smaller_batch_can_need_more():
    """64 lists of 256 pages fill the CUs uncut; 13 or one are cut and merged."""
    d = _desc(32, 8, 128, 16)

    def need(n):
        rows = np.array([(r, 7999, 1, 8000) for r in range(n)], np.int32)
        return [cache.page_attn_workspace_bytes(d, rows, 256),
                cache.prefix_attn_workspace_bytes(d, rows, [])]
    most, few, one = need(64), need(13), need(1)
    assert all(a < b for a, b in zip(most, few)) and all(a < b for a, b in zip(most, one))
    for needs, n in ((most, 64), (few, 13), (one, 1)):
        assert needs[0] <= _pages_bound(d, n, 256) and needs[1] <= _prefix_bound(d, n, 8000, False)


@pytest.mark.parametrize("several", [False, True], ids=["decode", "chunks"])
@pytest.mark.parametrize("seed", range(6))
def test_the_stated_sizes_serve_every_batch(seed, several):
    r = np.random.default_rng(seed)

    def spread(lo, hi):
        return int(min(hi, lo * (hi / lo) ** r.random() + r.random()))
    for _ in range(300):
        d = _desc(*HEADS[r.integers(len(HEADS))], int(r.choice([64, 128])), int(r.choice([16, 32])))
        n, longest = spread(1, 300), spread(4, 1 << 20)
        rows, groups = [], []
        while len(rows) < n:
            count, common = min(n - len(rows), spread(1, 40)), int(r.integers(longest))
            if r.random() < 0.7:
                groups.append((len(rows), count, common))
            for _ in range(count):
                start = common + int(r.integers(longest)) // spread(1, longest)
                new = int(r.integers(2)) if r.random() < 0.9 or not several else spread(2, 1500)
                rows.append((len(rows), start, new, start + new))
        rows = np.array(rows, np.int32)
        tokens, keys = int(rows[:, 2].sum()), int(rows[rows[:, 2] > 0, 3].max(initial=0))
        n_pages = spread(1, cache.MAX_PAGES)
        need = cache.page_attn_workspace_bytes(d, rows, n_pages)
        assert need <= _pages_bound(d, tokens, n_pages)
        assert need <= _pages_bound(d, tokens, -(-keys // d.block_size))   # (no list is longer)
        assert cache.prefix_attn_workspace_bytes(d, rows, groups) <= _prefix_bound(d, tokens, keys,
                                                                                   several)
