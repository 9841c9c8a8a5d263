"""Drafted trees and forks on the host: the oracle's own pins, the exported
symbols, and every refusal (the stand-in addresses are never dereferenced)."""

import ctypes
import os
import re

import numpy as np
import pytest

import paper_2606_09061_amd as cp
from oracle import tree as ref
from paper_2606_09061_amd import binding, tree

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20


def test_library_exports_every_declared_function():
    src = open(os.path.join(ROOT, "include", "cp_tree.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    names = sorted(set(re.findall(r"\b(cp_(?:tree|kv)_[a-z_]+)\s*\(", src)))
    lib = tree.load()
    assert len(names) == 7 and sorted(tree.exported_symbols()) == names
    for n in names:
        assert hasattr(lib, n)


# ---------------------------------------------------------------- the oracle

def test_oracle_layout_of_a_known_tree():
    #      0
    #     / \
    #    1   2
    #    |   |\
    #    3   4 5
    mask, pos = ref.layout(np.array([-1, 0, 0, 1, 2, 2]), [(0, 10, 6, 16)], 1)
    assert mask[:, 0].tolist() == [0b1, 0b11, 0b101, 0b1011, 0b10101, 0b100101]
    assert pos.tolist() == [10, 11, 11, 12, 12, 12]


def test_oracle_attention_of_a_chain_is_causal_and_of_one_key_is_its_value():
    rng = np.random.default_rng(0)
    n, d, start = 5, 64, 3
    k, v = rng.standard_normal((1, 1, 16, d)), rng.standard_normal((1, 1, d, 16))
    q = rng.standard_normal((n, 1, d))
    mask, _ = ref.layout(np.arange(n) - 1, [(0, start, n, start + n)], 1)
    out, _, _ = ref.attn(q, k, v, np.zeros((1, 1), int), mask, [(0, start, n, start + n)], 0.2)
    for j in range(n):
        s = k[0, 0, :start + j + 1] @ q[j, 0] * 0.2
        w = np.exp(s) / np.exp(s).sum()
        assert np.allclose(out[j, 0], v[0, 0, :, :start + j + 1] @ w, rtol=1e-12)
    only = np.array([[1 << 2]], np.uint64)   # no committed keys, one node seen
    out, spread, _ = ref.attn(q[:1], k, v, np.zeros((1, 1), int), np.repeat(only, 1, 0),
                              [(0, 0, 1, 1)], 0.2)
    assert (out == 0).all()                  # bit 2 is past the row's one node
    out, spread, _ = ref.attn(q[:3], k, v, np.zeros((1, 1), int), np.repeat(only, 3, 0),
                              [(0, 0, 3, 3)], 0.2)
    assert np.allclose(out[:, 0], v[0, 0, :, 2]) and np.allclose(spread, 0)


def test_oracle_notices_a_planted_mistake():
    """A mask shifted by one node changes the oracle's result."""
    rng = np.random.default_rng(1)
    k, v = rng.standard_normal((1, 1, 16, 64)), rng.standard_normal((1, 1, 64, 16))
    q, rows = rng.standard_normal((6, 1, 64)), [(0, 4, 6, 10)]
    mask, _ = ref.layout(np.array([-1, 0, 0, 1, 2, 2]), rows, 1)
    a, _, _ = ref.attn(q, k, v, np.zeros((1, 1), int), mask, rows, 0.2)
    b, _, _ = ref.attn(q, k, v, np.zeros((1, 1), int), np.roll(mask, 1, 0), rows, 0.2)
    assert np.abs(a - b).max() > 0.1


def test_oracle_verify_walks_to_the_lowest_child_that_agrees():
    logits = np.zeros((6, 8))
    logits[0, 3] = logits[2, 5] = logits[4, 1] = 1
    tokens = np.array([7, 2, 3, 3, 5, 5])
    parents = np.array([-1, 0, 0, 0, 2, 2])
    target, path, count, after = ref.verify(logits, tokens, parents, [(0, 0, 6, 6)], 4)
    assert target.tolist() == [3, 0, 5, 0, 1, 0]
    assert path.tolist() == [[0, 2, 4, -1]] and count.tolist() == [3] and after.tolist() == [1]
    _, path, count, after = ref.verify(logits, tokens, parents, [(0, 0, 6, 6)], 2)
    assert path.tolist() == [[0, 2]] and after.tolist() == [5]
    assert ref.argmax(np.array([1.0, np.nan, 2.0, np.nan])) == 1
    assert ref.argmax(np.array([-0.0, 0.0])) == 0


def test_oracle_compact_and_fork():
    k = np.arange(4 * 16, dtype=float).reshape(4, 1, 16, 1)
    v = k.transpose(0, 1, 3, 2).copy()
    table = np.array([[2, 0], [3, 3]])
    k2, v2 = ref.compact(k, v, table, [(0, 14, 5, 19)], np.array([[0, 2, 4]]), np.array([3]))
    assert k2[2, 0, 14:, 0].tolist() == [46, 0] and k2[0, 0, 0, 0] == 2
    assert (v2.transpose(0, 1, 3, 2) == k2).all() and (k2 != k).sum() == 2
    k3, v3, t3 = ref.fork(k, v, table, [(0, 1, 17, 1)])
    assert t3.tolist() == [[2, 0], [2, 1]] and (k3[1] == k[0]).all() and (v3[1] == v[0]).all()


# ---------------------------------------------------------------- refusals

def _desc(**kw):
    base = dict(num_q_heads=32, num_kv_heads=8, head_dim=128, block_size=16, num_blocks=100,
                max_blocks_per_req=20, num_reqs_in_table=4, sm_scale=0.088)
    base.update(kw)
    return cp.make_desc(**base)


GOOD = np.array([[0, 10, 5, 15], [1, 0, 1, 1]], np.int32)


def _rows(*rows):
    return np.array(rows, np.int32).reshape(-1, 4)


def _layout(parents=FAKE, rows=GOOD, mask=FAKE, words=1, positions=FAKE):
    return tree.load().cp_tree_layout(parents, rows.ctypes.data, len(rows), mask, words, positions,
                                      None)


def _attn(desc=None, rows=GOOD, words=1, ws_bytes=1 << 40, **kw):
    p = {n: FAKE for n in ("q", "k", "v", "bt", "mask", "out", "ws")}
    p.update(kw)
    return tree.load().cp_tree_attn(ctypes.byref(desc or _desc()), p["q"], p["k"], p["v"], p["bt"],
                                    p["mask"], words, rows.ctypes.data, len(rows), p["out"],
                                    p["ws"], ws_bytes, None)


def _verify(rows=GOOD, ld=1000, vocab=1000, max_path=8, ws_bytes=1 << 40, **kw):
    p = {n: FAKE for n in ("logits", "tokens", "parents", "target", "path", "n", "next", "ws")}
    p.update(kw)
    return tree.load().cp_tree_verify(p["logits"], ld, vocab, p["tokens"], p["parents"],
                                      rows.ctypes.data, len(rows), max_path, p["target"],
                                      p["path"], p["n"], p["next"], p["ws"], ws_bytes, None)


def _pools(n=2, address=FAKE):
    return (ctypes.c_void_p * n)(*[address] * n)


def _compact(desc=None, rows=GOOD, k=None, v=None, n_layers=2, max_path=8, **kw):
    p = {n: FAKE for n in ("bt", "path", "n")}
    p.update(kw)
    return tree.load().cp_kv_compact(ctypes.byref(desc or _desc()), _pools() if k is None else k,
                                     _pools() if v is None else v, n_layers, p["bt"],
                                     rows.ctypes.data, len(rows), p["path"], max_path, p["n"], None)


def _fork(forks, desc=None, k=None, n_layers=2, bt=FAKE):
    forks = _rows(*forks)
    return tree.load().cp_kv_fork(ctypes.byref(desc or _desc()), _pools() if k is None else k,
                                  _pools(), n_layers, bt, forks.ctypes.data, len(forks), None)


BAD_ROWS = [
    _rows([0, 10, -1, 9]), _rows([0, -1, 2, 1]), _rows([0, 10, 5, 16]),
    _rows([0, 10, 257, 267]),                                  # more nodes than a tree may have
]
BAD_TABLE_ROWS = [_rows([0, 318, 3, 321]), _rows([4, 0, 1, 1]), _rows([1, 3, 1, 4], [1, 0, 1, 1])]


@pytest.mark.parametrize("rows", BAD_ROWS)
def test_bad_rows_are_refused(rows):
    assert _layout(rows=rows, words=4) == binding.CP_ERR_BAD_META
    assert _verify(rows=rows) == binding.CP_ERR_BAD_META
    assert _attn(rows=rows, words=4) == binding.CP_ERR_BAD_META
    assert _compact(rows=rows) == binding.CP_ERR_BAD_META
    assert tree.load().cp_tree_attn_workspace_bytes(ctypes.byref(_desc()), rows.ctypes.data,
                                                    len(rows)) == 0
    with pytest.raises(cp.CpError) as e:
        tree.attn_workspace_bytes(_desc(), rows)
    assert e.value.code == binding.CP_ERR_BAD_META


@pytest.mark.parametrize("rows", BAD_TABLE_ROWS)
def test_rows_outside_the_table_are_refused(rows):
    assert _attn(rows=rows) == binding.CP_ERR_BAD_META
    assert _compact(rows=rows) == binding.CP_ERR_BAD_META


def test_more_nodes_than_the_mask_has_bits_are_refused():
    rows = _rows([0, 10, 65, 75])
    assert _attn(rows=rows) == _layout(rows=rows) == binding.CP_ERR_BAD_META
    for words in (0, 5, -1):
        assert _attn(words=words) == _layout(words=words) == binding.CP_ERR_INVALID_ARG


@pytest.mark.parametrize("kw,code", [
    (dict(num_q_heads=0), binding.CP_ERR_INVALID_ARG),
    (dict(num_q_heads=12), binding.CP_ERR_BAD_META),
    (dict(sm_scale=float("nan")), binding.CP_ERR_BAD_META),
    (dict(head_dim=96), binding.CP_ERR_UNSUPPORTED),
    (dict(block_size=8), binding.CP_ERR_UNSUPPORTED),
    (dict(num_q_heads=48, num_kv_heads=3), binding.CP_ERR_UNSUPPORTED),
    (dict(num_q_heads=2048, num_kv_heads=2048), binding.CP_ERR_UNSUPPORTED),
])
def test_geometries_are_refused(kw, code):
    d = _desc(**kw)
    assert _attn(d) == _compact(d) == _fork([(0, 1, 20, 5)], d) == code


@pytest.mark.parametrize("name,step", [("q", 8), ("k", 8), ("v", 8), ("out", 8), ("mask", 4),
                                       ("bt", 2), ("ws", 128)])
def test_attn_refuses_missing_and_misaligned_buffers(name, step):
    assert _attn(**{name: None}) == binding.CP_ERR_INVALID_ARG
    assert _attn(**{name: FAKE + step}) == binding.CP_ERR_INVALID_ARG


def test_short_workspaces_are_refused():
    need = tree.attn_workspace_bytes(_desc(), GOOD)
    assert _attn(ws_bytes=need - 1) == binding.CP_ERR_WORKSPACE
    need = tree.verify_workspace_bytes(6, 1000)
    assert _verify(ws_bytes=need - 1) == binding.CP_ERR_WORKSPACE
    for n, vocab in ((-1, 10), (1, 0), (1 << 40, 10)):
        with pytest.raises(cp.CpError):
            tree.verify_workspace_bytes(n, vocab)


@pytest.mark.parametrize("name,step", [("parents", 2), ("mask", 4), ("positions", 2)])
def test_layout_refuses_missing_and_misaligned_buffers(name, step):
    assert _layout(**{name: None}) == binding.CP_ERR_INVALID_ARG
    assert _layout(**{name: FAKE + step}) == binding.CP_ERR_INVALID_ARG


@pytest.mark.parametrize("name,step", [("logits", 1), ("tokens", 2), ("parents", 2),
                                       ("target", 2), ("path", 2), ("n", 2), ("next", 2),
                                       ("ws", 128)])
def test_verify_refuses_missing_and_misaligned_buffers(name, step):
    assert _verify(**{name: None}) == binding.CP_ERR_INVALID_ARG
    assert _verify(**{name: FAKE + step}) == binding.CP_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(vocab=0), dict(ld=999), dict(max_path=0), dict(max_path=257)])
def test_verify_refuses_sizes(kw):
    assert _verify(**kw) == binding.CP_ERR_INVALID_ARG


def test_compact_refuses():
    for name, step in (("bt", 2), ("path", 2), ("n", 2)):
        assert _compact(**{name: None}) == binding.CP_ERR_INVALID_ARG
        assert _compact(**{name: FAKE + step}) == binding.CP_ERR_INVALID_ARG
    for bad in (_pools(2, None), _pools(2, FAKE + 8)):
        assert _compact(k=bad) == _compact(v=bad) == binding.CP_ERR_INVALID_ARG
    assert _compact(n_layers=-1) == binding.CP_ERR_INVALID_ARG
    assert _compact(max_path=0) == _compact(max_path=257) == binding.CP_ERR_INVALID_ARG


@pytest.mark.parametrize("forks", [
    [(0, 4, 20, 5)], [(4, 0, 20, 5)], [(-1, 0, 20, 5)], [(0, 1, -1, 5)], [(0, 1, 321, 5)],
    [(0, 0, 20, 5)],                                 # onto itself
    [(0, 1, 20, 100)], [(0, 1, 20, -1)],             # no such page
    [(0, 1, 20, 5), (0, 1, 20, 6)],                  # a new row twice
    [(0, 1, 20, 5), (1, 2, 20, 6)],                  # a new row that is a source
    [(0, 1, 20, 5), (0, 2, 20, 5)],                  # a page twice
])
def test_fork_refuses(forks):
    assert _fork(forks) == binding.CP_ERR_BAD_META


def test_fork_refuses_missing_buffers():
    good = [(0, 1, 20, 5)]
    assert _fork(good, bt=None) == _fork(good, bt=FAKE + 2) == binding.CP_ERR_INVALID_ARG
    assert _fork(good, k=_pools(2, None)) == binding.CP_ERR_INVALID_ARG
    assert _fork(good, n_layers=-1) == binding.CP_ERR_INVALID_ARG


def test_empty_batches_are_fine_without_a_gpu():
    none, idle = _rows(), _rows([0, 10, 0, 10], [2, 0, 0, 0])
    for rows in (none, idle):
        assert _layout(rows=rows, parents=None, mask=None, positions=None) == 0
        assert _attn(rows=rows, q=None, ws=None) == 0
        assert _compact(rows=rows, path=None) == 0
        assert tree.attn_workspace_bytes(_desc(), rows) >= 256
    assert _verify(rows=none, logits=None, path=None) == 0
    assert _compact(n_layers=0) == 0
    assert _fork([]) == 0


def test_calls_want_tensors_on_a_gpu():
    import torch
    z = torch.zeros(6, dtype=torch.int32)
    with pytest.raises(cp.CpError):
        tree.layout(z, GOOD, torch.zeros(6, 1, dtype=torch.int64), z)
    with pytest.raises(cp.CpError):
        tree.kv_layers(_desc(), [torch.zeros(100, 8, 16, 128, dtype=torch.bfloat16)],
                       [torch.zeros(100, 8, 128, 16, dtype=torch.bfloat16)])


def test_plan_under_sanitizers(tmp_path):
    """Host C++: random batches through the plan (tests/native/tree_fuzz.cpp)."""
    import shutil
    import subprocess
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    csrc = os.path.join(ROOT, "paper_2606_09061_amd", "csrc")
    exe = str(tmp_path / "tree_fuzz")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    os.path.join(ROOT, "tests", "native", "tree_fuzz.cpp"),
                    os.path.join(csrc, "tree_plan.cpp"), "-o", exe], check=True, timeout=300)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.startswith("ok"), r.stderr[-2000:]


# ---------------------------------------------------------------- the longest contexts

LONGEST = 1 << 30   # keys of a row


def _far(ctx, n=3):
    return _desc(max_blocks_per_req=(1 << 27) - 1), _rows([0, ctx - n, n, ctx])


@pytest.mark.parametrize("ctx", [LONGEST + 1, 2147475000, 2147483521, 2147483632])
def test_contexts_past_the_longest_are_refused(ctx):
    """In a process of its own: the plan of such rows used to divide by zero."""
    import subprocess
    import sys
    code = (f"import test_tree as t\n"
            f"d, rows = t._far({ctx})\n"
            f"assert t._attn(d, rows) == t.binding.CP_ERR_UNSUPPORTED\n"
            f"try:\n    t.tree.attn_workspace_bytes(d, rows)\n"
            f"except t.cp.CpError as e:\n    assert e.code == t.binding.CP_ERR_UNSUPPORTED\n"
            f"else:\n    raise SystemExit('not refused')\n")
    env = dict(os.environ, PYTHONPATH=os.pathsep.join([ROOT, os.path.join(ROOT, "tests")]))
    r = subprocess.run([sys.executable, "-c", code], env=env, capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0, (r.returncode, r.stderr[-2000:])


def test_the_longest_context_is_planned():
    need = tree.attn_workspace_bytes(*_far(LONGEST))
    assert need > 1 << 20
    assert _attn(*_far(LONGEST), ws_bytes=need - 1) == binding.CP_ERR_WORKSPACE


def test_refusals_of_the_workspace_query_name_their_reason():
    for d, rows, code in ((_desc(), _rows([0, 10, 257, 267]), binding.CP_ERR_BAD_META),
                          (_desc(num_q_heads=2048, num_kv_heads=2048), GOOD,
                           binding.CP_ERR_UNSUPPORTED)):
        with pytest.raises(cp.CpError) as e:
            tree.attn_workspace_bytes(d, rows)
        assert e.value.code == code


def test_plan_at_the_ends_of_its_ranges(tmp_path):
    """Host C++: contexts of up to 2^30 keys, up to 1,024 kv heads and many rows,
    under sanitizers (tests/native/tree_bounds.cpp)."""
    import shutil
    import subprocess
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    csrc = os.path.join(ROOT, "paper_2606_09061_amd", "csrc")
    exe = str(tmp_path / "tree_bounds")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    os.path.join(ROOT, "tests", "native", "tree_bounds.cpp"),
                    os.path.join(csrc, "tree_plan.cpp"), "-o", exe], check=True, timeout=300)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.startswith("ok"), r.stderr[-2000:]


@pytest.mark.parametrize("vocab", [1, 1000, 16384, 20000, 151936, 1 << 30])
def test_a_verify_workspace_serves_fewer_nodes_too(vocab):
    """A server sizes its workspace once, for its largest batch."""
    sizes = [tree.verify_workspace_bytes(n, vocab) for n in range(4200)]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))
    assert sizes[-1] <= 8 * (4199 + 2047)                 # and is none too large
