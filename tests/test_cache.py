"""Long and shared contexts on the host: the oracle's own pins, the exported
symbols, and every refusal (the stand-in addresses are never dereferenced)."""

import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

import paper_2606_09061_amd as cp
from oracle import cache as ref
from paper_2606_09061_amd import binding, cache

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20
BAD, ARG, UNSUPPORTED = (binding.CP_ERR_BAD_META, binding.CP_ERR_INVALID_ARG,
                         binding.CP_ERR_UNSUPPORTED)


def test_library_exports_every_declared_function():
    src = open(os.path.join(ROOT, "include", "cp_cache.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    names = sorted(set(re.findall(r"\b(cp_(?:qkv|page|prefix)_[a-z_]+)\s*\(", src)))
    lib = cache.load()
    assert len(names) == 8 and sorted(cache.exported_symbols()) == names
    for n in names:
        assert hasattr(lib, n)


# ---------------------------------------------------------------- the oracle

def test_oracle_attention_of_listed_pages():
    rng = np.random.default_rng(0)
    k, v = rng.standard_normal((4, 1, 16, 64)), rng.standard_normal((4, 1, 64, 16))
    table, q = np.array([[2, 0, 3]]), rng.standard_normal((1, 1, 64))
    rows = [(0, 36, 1, 37)]
    keys = np.concatenate([k[2, 0], k[0, 0], k[3, 0, :5]])
    values = np.concatenate([v[2, 0].T, v[0, 0].T, v[3, 0, :, :5].T])
    for pages, use in ((None, range(37)), ([0, 2, -1], [*range(16), *range(32, 37)]),
                       ([1, 1, 2], range(16, 32)), ([-1, 0, 1], [])):
        p = None if pages is None else np.array([[pages]])
        out, spread, _ = ref.attn(q, k, v, table, rows, 0.2, p)
        use = np.array(list(use), int)
        if len(use) == 0:
            assert (out == 0).all()
            continue
        w = np.exp(keys[use] @ q[0, 0] * 0.2)
        assert np.allclose(out[0, 0], (w / w.sum()) @ values[use], rtol=1e-12)


def test_oracle_selection_of_known_scores():
    b = np.zeros((6, 1, 2, 2))
    b[:, 0, 0, 0] = [-1, 0, -4, 2, 0, 0]                 # lo of feature 0
    b[:, 0, 1, 0] = [1, 5, 3, 2, 0, 0]                   # hi
    q = np.array([[[1.0, 0.0], [-1.0, 0.0]]])            # max over both heads: 1 5 4 2 0 0
    table, rows = np.arange(6)[None], [(0, 5 * 16 + 3, 1, 84)]

    def pick(n, first, last):
        return ref.select(q, b, table, rows, 16, n, first, last)[0, 0].tolist()

    assert pick(2, 0, 0) == [1, 2] and pick(3, 0, 1) == [1, 2, 5] and pick(3, 1, 1) == [0, 1, 5]
    assert pick(5, 0, 0) == [0, 1, 2, 3, 4]              # of equal ones the lower
    assert pick(8, 1, 1) == [0, 1, 2, 3, 4, 5, -1, -1]


def test_oracle_bounds_and_append():
    k = np.arange(2 * 16, dtype=float).reshape(2, 1, 16, 1)
    out = ref.bounds(k, np.array([[1, 0]]), [(0, 14, 4, 18)], np.full((2, 1, 2, 1), 9.0))
    assert out[:, 0, :, 0].tolist() == [[0, 1], [16, 31]]
    out = ref.bounds(k, np.array([[1, 0]]), [(0, 16, 0, 16)], np.full((2, 1, 2, 1), 9.0))
    assert (out == 9).all()
    k[1, 0, 3, 0] = np.nan
    out = ref.bounds(k, np.array([[1, 0]]), [(0, 0, 16, 16)], np.full((2, 1, 2, 1), 9.0))
    assert out[1, 0, :, 0].tolist() == [-ref.LARGEST, ref.LARGEST]
    new = np.array([[[70.0]], [[71.0]]])
    kc, vc = ref.append(k, k.transpose(0, 1, 3, 2), new, new, np.array([[1, 0]]), [(0, 15, 2, 17)])
    assert kc[1, 0, 15, 0] == 70 and kc[0, 0, 0, 0] == 71 and vc[0, 0, 0, 0] == 71
    assert (kc != k).sum() == 3                          # (and the NaN)


def test_oracle_notices_a_planted_mistake():
    rng = np.random.default_rng(1)
    k, v = rng.standard_normal((4, 1, 16, 64)), rng.standard_normal((4, 1, 64, 16))
    q, rows = rng.standard_normal((1, 1, 64)), [(0, 50, 1, 51)]
    a = ref.attn(q, k, v, np.array([[2, 0, 3, 1]]), rows, 0.2)[0]
    b = ref.attn(q, k, v, np.array([[2, 0, 1, 3]]), rows, 0.2)[0]
    assert np.abs(a - b).max() > 0.05


# ---------------------------------------------------------------- refusals

def _desc(**kw):
    base = dict(num_q_heads=32, num_kv_heads=8, head_dim=128, block_size=16, num_blocks=100,
                max_blocks_per_req=20, num_reqs_in_table=4, sm_scale=0.088)
    base.update(kw)
    return cp.make_desc(**base)


def _rows(*rows):
    return np.array(rows, np.int32).reshape(-1, 4)


GOOD = _rows([0, 10, 5, 15], [1, 300, 1, 301])


def _args(names, kw):
    p = {n: FAKE for n in names}
    p.update(kw)
    return p


def _append(desc=None, rows=GOOD, theta=1e6, eps=1e-6, **kw):
    p = _args(("qkv", "qw", "kw", "pos", "q", "k", "v", "bt"), kw)
    return cache.load().cp_qkv_append(ctypes.byref(desc or _desc()), p["qkv"], p["qw"], p["kw"],
                                      p["pos"], theta, eps, p["q"], p["k"], p["v"], p["bt"],
                                      rows.ctypes.data, len(rows), None)


def _bounds(desc=None, rows=GOOD, **kw):
    p = _args(("k", "bt", "bounds"), kw)
    return cache.load().cp_page_bounds(ctypes.byref(desc or _desc()), p["k"], p["bt"],
                                       rows.ctypes.data, len(rows), p["bounds"], None)


def _select(desc=None, rows=GOOD, n_pages=4, first=1, last=1, ws_bytes=1 << 40, **kw):
    p = _args(("q", "bounds", "bt", "pages", "ws"), kw)
    return cache.load().cp_page_select(ctypes.byref(desc or _desc()), p["q"], p["bounds"], p["bt"],
                                       rows.ctypes.data, len(rows), n_pages, first, last,
                                       p["pages"], p["ws"], ws_bytes, None)


def _attn(desc=None, rows=GOOD, n_pages=4, ws_bytes=1 << 40, **kw):
    p = _args(("q", "k", "v", "bt", "pages", "out", "ws"), kw)
    return cache.load().cp_page_attn(ctypes.byref(desc or _desc()), p["q"], p["k"], p["v"], p["bt"],
                                     p["pages"], n_pages, rows.ctypes.data, len(rows), p["out"],
                                     p["ws"], ws_bytes, None)


def _prefix(desc=None, rows=GOOD, groups=((0, 2, 5),), ws_bytes=1 << 40, **kw):
    p = _args(("q", "k", "v", "bt", "out", "ws"), kw)
    groups = np.array(groups, np.int32).reshape(-1, 3)
    at = kw.get("groups_at", groups.ctypes.data)
    return cache.load().cp_prefix_attn(ctypes.byref(desc or _desc()), p["q"], p["k"], p["v"],
                                       p["bt"], rows.ctypes.data, len(rows), at,
                                       kw.get("n_groups", len(groups)), p["out"], p["ws"], ws_bytes,
                                       None)


ALL = (_append, _bounds, _select, _attn, _prefix)
QUERIES = (lambda d, r: cache.page_select_workspace_bytes(d, r, 4),
           lambda d, r: cache.page_attn_workspace_bytes(d, r, 4),
           lambda d, r: cache.prefix_attn_workspace_bytes(d, r, []))


def _refused(desc, rows, code):
    for call in ALL:
        assert call(desc, rows, **({"groups": ()} if call is _prefix else {})) == code, call
    for query in QUERIES:
        with pytest.raises(cp.CpError) as e:
            query(desc, rows)
        assert e.value.code == code


@pytest.mark.parametrize("rows", [
    _rows([0, 10, -1, 9]), _rows([0, -1, 2, 1]), _rows([0, 10, 5, 16]), _rows([0, 318, 3, 321]),
    _rows([4, 0, 1, 1]), _rows([-1, 0, 1, 1]), _rows([1, 3, 1, 4], [1, 0, 1, 1]),
])
def test_bad_rows_are_refused(rows):
    _refused(_desc(), rows, BAD)


@pytest.mark.parametrize("kw,code", [
    (dict(num_q_heads=0), ARG), (dict(num_blocks=0), ARG),
    (dict(num_q_heads=12), BAD), (dict(sm_scale=float("nan")), BAD),
    (dict(head_dim=96), UNSUPPORTED), (dict(block_size=8), UNSUPPORTED),
    (dict(num_q_heads=48, num_kv_heads=3), UNSUPPORTED),
    (dict(num_q_heads=2048, num_kv_heads=2048), UNSUPPORTED),
])
def test_geometries_are_refused(kw, code):
    _refused(_desc(**kw), GOOD, code)


@pytest.mark.parametrize("ctx", [(1 << 30) + 1, 2147483521])
def test_contexts_past_the_longest_are_refused(ctx):
    _refused(_desc(max_blocks_per_req=(1 << 27) - 1), _rows([0, ctx - 1, 1, ctx]), UNSUPPORTED)


@pytest.mark.parametrize("tokens,hq,hkv", [((1 << 23) + 1, 1, 1), ((1 << 20) + 1, 128, 16)])
def test_batches_of_too_many_tokens_are_refused(tokens, hq, hkv):
    d = _desc(num_q_heads=hq, num_kv_heads=hkv, max_blocks_per_req=1 << 20)
    _refused(d, _rows([0, 0, tokens, tokens]), UNSUPPORTED)


BUFFERS = {
    _append: [("qkv", 8), ("qw", 8), ("kw", 8), ("q", 8), ("k", 8), ("v", 8), ("bt", 2)],
    _bounds: [("k", 8), ("bt", 2), ("bounds", 8)],
    _select: [("q", 8), ("bounds", 8), ("bt", 2), ("pages", 2), ("ws", 128)],
    _attn: [("q", 8), ("k", 8), ("v", 8), ("bt", 2), ("pages", 2), ("out", 8), ("ws", 128)],
    _prefix: [("q", 8), ("k", 8), ("v", 8), ("bt", 2), ("out", 8), ("ws", 128)],
}


@pytest.mark.parametrize("call,name,step", [(c, *b) for c, bs in BUFFERS.items() for b in bs])
def test_missing_and_misaligned_buffers_are_refused(call, name, step):
    assert call(**{name: None}) == ARG
    assert call(**{name: FAKE + step}) == ARG


def test_append_refuses_positions_theta_and_eps():
    assert _append(pos=FAKE + 2) == ARG
    for kw in (dict(theta=1.0), dict(theta=float("nan")), dict(theta=float("inf")), dict(eps=0.0),
               dict(eps=float("nan"))):
        assert _append(**kw) == ARG


@pytest.mark.parametrize("n", [0, -1, 4097])
def test_numbers_of_pages_are_refused(n):
    assert _select(n_pages=n, first=0, last=0) == _attn(n_pages=n) == ARG
    for query in (cache.page_select_workspace_bytes, cache.page_attn_workspace_bytes):
        with pytest.raises(cp.CpError) as e:
            query(_desc(), GOOD, n)
        assert e.value.code == ARG


@pytest.mark.parametrize("first,last", [(-1, 0), (0, -1), (3, 2), (5, 0), (1 << 30, 1 << 30),
                                        ((1 << 31) - 1, (1 << 31) - 1)])
def test_more_fixed_pages_than_there_are_is_refused(first, last):
    assert _select(first=first, last=last) == ARG


@pytest.mark.parametrize("groups", [
    [(0, 3, 5)], [(-1, 2, 5)], [(0, -1, 5)], [(0, 2, -1)], [(0, 2, 11)],
    [(0, 2, 5), (1, 1, 5)],                            # overlap
    [(1, 1, 5), (0, 1, 5)],                            # fall
    [((1 << 31) - 1, (1 << 31) - 1, 0)],
])
def test_groups_are_refused(groups):
    assert _prefix(groups=groups) == BAD
    with pytest.raises(cp.CpError) as e:
        cache.prefix_attn_workspace_bytes(_desc(), GOOD, groups)
    assert e.value.code == BAD


def test_missing_groups_are_refused():
    assert _prefix(groups_at=None) == ARG
    assert _prefix(n_groups=-1) == ARG


def test_short_workspaces_are_refused():
    need = cache.page_select_workspace_bytes(_desc(), GOOD, 4)
    assert need == (19 * 8) * 8                          # the second row has 19 pages
    assert _select(ws_bytes=need - 1) == binding.CP_ERR_WORKSPACE
    d = _desc(max_blocks_per_req=4000)
    rows = _rows([0, 1300, 1, 1301], [1, 1200, 1, 1201])
    need = cache.prefix_attn_workspace_bytes(d, rows, [(0, 2, 1200)])
    assert need > 256 and _prefix(d, rows=rows, groups=[(0, 2, 1200)],
                                  ws_bytes=need - 1) == binding.CP_ERR_WORKSPACE
    rows = _rows([0, 40000, 1, 40001])
    need = cache.page_attn_workspace_bytes(d, rows, 600)
    assert need > 256 and _attn(d, rows, 600, need - 1) == binding.CP_ERR_WORKSPACE


def test_the_largest_batches_are_planned():
    """The longest rows and the most heads: queries answer, calls get as far as their
    workspace."""
    d = _desc(num_q_heads=8192, num_kv_heads=1024, max_blocks_per_req=(1 << 27) - 1)
    far = 1 << 30
    for rows in (_rows([0, far - 1, 1, far]), _rows([0, far - 16384, 16384, far])):
        need = cache.page_select_workspace_bytes(d, rows, 4)
        assert need >= 1024 * (1 << 26) * 8
        assert _select(d, rows, ws_bytes=need - 1) == binding.CP_ERR_WORKSPACE
        assert cache.page_attn_workspace_bytes(d, rows, 4) >= 256
        need = cache.prefix_attn_workspace_bytes(d, rows, [(0, 1, far - 16384)])
        assert _prefix(d, rows, [(0, 1, far - 16384)], ws_bytes=need - 1) == binding.CP_ERR_WORKSPACE
    rows = _rows([0, far - 16384, 16384, far])
    with pytest.raises(cp.CpError) as e:                 # partial rows past their index type
        cache.page_attn_workspace_bytes(d, rows, 4096)
    assert e.value.code == UNSUPPORTED and _attn(d, rows, 4096) == UNSUPPORTED


def test_a_select_workspace_serves_smaller_batches():
    d = _desc(max_blocks_per_req=4000)
    sizes = [cache.page_select_workspace_bytes(d, _rows([0, c, 2, c + 2], [1, 50, 1, 51]), 20)
             for c in range(0, 3000, 7)]
    assert sizes == sorted(sizes)


def test_empty_batches_are_fine_without_a_gpu():
    for rows in (_rows(), _rows([0, 10, 0, 10], [2, 0, 0, 0])):
        assert _append(rows=rows, qkv=None, k=None) == 0
        assert _bounds(rows=rows, k=None, bounds=None) == 0
        assert _select(rows=rows, q=None, ws=None) == 0
        assert _attn(rows=rows, q=None, ws=None) == 0
        assert _prefix(rows=rows, groups=(), q=None, ws=None) == 0
        for query in QUERIES:
            assert query(_desc(), rows) == 256
    assert _prefix(rows=_rows([0, 10, 0, 10]), groups=[(0, 1, 500)], q=None) == 0


def test_calls_want_tensors_on_a_gpu():
    import torch
    b16 = dict(dtype=torch.bfloat16)
    d, rows = _desc(), _rows([0, 10, 2, 12])
    q, qkv, w = torch.zeros(2, 32, 128, **b16), torch.zeros(2, 48 * 128, **b16), torch.zeros(128, **b16)
    k, v = torch.zeros(100, 8, 16, 128, **b16), torch.zeros(100, 8, 128, 16, **b16)
    bounds, bt = torch.zeros(100, 8, 2, 128, **b16), torch.zeros(4, 20, dtype=torch.int32)
    pages = torch.zeros(2, 8, 4, dtype=torch.int32)
    for call in (lambda: cache.qkv_append(d, qkv, w, w, rows, q, k, v, bt, 1e6, 1e-6),
                 lambda: cache.page_bounds(d, k, bt, rows, bounds),
                 lambda: cache.page_select(d, q, bounds, bt, rows, pages),
                 lambda: cache.page_attn(d, q, k, v, bt, pages, rows, q),
                 lambda: cache.prefix_attn(d, q, k, v, bt, rows, [], q)):
        with pytest.raises(cp.CpError) as e:
            call()
        assert e.value.code == ARG


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_plans_under_sanitizers(tmp_path):
    """Host C++: random batches through the plans (tests/native/cache_fuzz.cpp)."""
    csrc = os.path.join(ROOT, "paper_2606_09061_amd", "csrc")
    exe = str(tmp_path / "cache_fuzz")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    os.path.join(ROOT, "tests", "native", "cache_fuzz.cpp"),
                    os.path.join(csrc, "cache_plan.cpp"), "-o", exe], check=True, timeout=300)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.startswith("ok"), r.stderr[-2000:]


def test_barriers_wait_for_lds_writes(tmp_path):
    """test_lds_waits.py's walk over the device code, of this library's."""
    import test_lds_waits as waits
    if waits.OBJDUMP is None:
        pytest.skip("needs llvm-objdump")
    waits.test_barriers_wait_for_lds_writes("libcpcache.so", tmp_path)
