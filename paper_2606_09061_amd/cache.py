"""Long and shared contexts over the paged cache (libcpcache.so).

The calls around a decode iteration's attention:

    qkv_append   the fused projection's q and k heads normalised and rotated,
                 K and V written straight into their pages
    page_bounds  per feature the extremes of the keys of the pages written to
    page_select  the pages that every token reads, by these bounds
    page_attn    attention over the selected pages
    prefix_attn  attention of requests with a common prefix (as tree.kv_fork
                 leaves them), which is read once for all of them

Rows are those of the attention step, ``(req, start, len, ctx)``.  The calls
check their tensors (dense, type, shape, one device) and raise
:class:`CpError`; outputs are written into the caller's tensors, on ``stream``
or the current stream of their device.
"""

from __future__ import annotations

import ctypes
import os

import numpy as np

from . import binding as cp
from .tree import _BF16, _I32, _call, _check, _device, _nodes, _ptr, _want, _workspace

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libcpcache.so")

MAX_KEYS = 1 << 30   # CP_CACHE_MAX_KEYS
MAX_PAGES = 4096     # CP_CACHE_MAX_PAGES

_lib = None


def load():
    """Loads libcpcache.so; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it first "
                           "(python -m paper_2606_09061_amd.build)")
    lib = ctypes.CDLL(LIB_PATH)
    P, I32, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    F, D = ctypes.c_float, ctypes.c_double
    lib.cp_qkv_append.argtypes = [P, P, P, P, P, D, F, P, P, P, P, P, I32, P]
    lib.cp_page_bounds.argtypes = [P, P, P, P, I32, P, P]
    lib.cp_page_select_workspace_bytes.argtypes = [P, P, I32, I32]
    lib.cp_page_select.argtypes = [P, P, P, P, P, I32, I32, I32, I32, P, P, SZ, P]
    lib.cp_page_attn_workspace_bytes.argtypes = [P, P, I32, I32]
    lib.cp_page_attn.argtypes = [P, P, P, P, P, P, I32, P, I32, P, P, SZ, P]
    lib.cp_prefix_attn_workspace_bytes.argtypes = [P, P, I32, P, I32]
    lib.cp_prefix_attn.argtypes = [P, P, P, P, P, P, I32, P, I32, P, P, SZ, P]
    for f in (lib.cp_page_select_workspace_bytes, lib.cp_page_attn_workspace_bytes,
              lib.cp_prefix_attn_workspace_bytes):
        f.restype = SZ
    for f in (lib.cp_qkv_append, lib.cp_page_bounds, lib.cp_page_select, lib.cp_page_attn,
              lib.cp_prefix_attn):
        f.restype = ctypes.c_int
    _lib = lib
    return lib


def exported_symbols():
    return ["cp_qkv_append", "cp_page_bounds", "cp_page_select_workspace_bytes", "cp_page_select",
            "cp_page_attn_workspace_bytes", "cp_page_attn", "cp_prefix_attn_workspace_bytes",
            "cp_prefix_attn"]


def _k_pool(desc, k_cache, dev, what):
    return _ptr(k_cache, _BF16,
                (desc.num_blocks, desc.num_kv_heads, desc.block_size, desc.head_dim), dev, what)


def _v_pool(desc, v_cache, dev, what):
    return _ptr(v_cache, _BF16,
                (desc.num_blocks, desc.num_kv_heads, desc.head_dim, desc.block_size), dev, what)


def _table(desc, block_tables, dev, what):
    return _ptr(block_tables, _I32, (desc.num_reqs_in_table, desc.max_blocks_per_req), dev, what)


def _bytes(n, reason, what):
    """A workspace query's answer, or the error that none stands for."""
    if n == 0:
        raise cp.CpError(reason(), what)
    return int(n)


def qkv_append(desc, qkv, q_norm_w, k_norm_w, rows, q, k_cache, v_cache, block_tables, theta, eps,
               positions=None, stream=None):
    """model.qkv_rope and binding.kv_append in one: qkv [T, (Hq + 2 Hkv) * D] gives
    q [T, Hq, D], its heads normalised and rotated, and the keys (normalised and
    rotated) and values in the rows' slots of the pools.  ``positions`` (int32
    [T], device): the rotary ones, where they are not the tokens' own."""
    what = "cp_qkv_append"
    rows = cp._rows(rows)
    dev, T = _device(qkv, what), _nodes(rows)
    hq, hkv, d = desc.num_q_heads, desc.num_kv_heads, desc.head_dim
    _check(_call(dev, stream, load().cp_qkv_append, ctypes.byref(desc),
                 _ptr(qkv, _BF16, (T, (hq + 2 * hkv) * d), dev, what),
                 _ptr(q_norm_w, _BF16, (d,), dev, what), _ptr(k_norm_w, _BF16, (d,), dev, what),
                 None if positions is None else _ptr(positions, _I32, (T,), dev, what),
                 float(theta), float(eps), _ptr(q, _BF16, (T, hq, d), dev, what),
                 _k_pool(desc, k_cache, dev, what), _v_pool(desc, v_cache, dev, what),
                 _table(desc, block_tables, dev, what), rows.tobytes(), rows.shape[0]), what)


def page_bounds(desc, k_cache, block_tables, rows, bounds, stream=None):
    """bounds [num_blocks, Hkv, 2, D] (bf16) of the pages that hold the rows' new
    tokens: per feature the least and the largest value of the page's keys."""
    what = "cp_page_bounds"
    rows = cp._rows(rows)
    dev = _device(k_cache, what)
    shape = (desc.num_blocks, desc.num_kv_heads, 2, desc.head_dim)
    _check(_call(dev, stream, load().cp_page_bounds, ctypes.byref(desc),
                 _k_pool(desc, k_cache, dev, what), _table(desc, block_tables, dev, what),
                 rows.tobytes(), rows.shape[0], _ptr(bounds, _BF16, shape, dev, what)), what)


def page_select_workspace_bytes(desc, rows, n_pages) -> int:
    rows, what = cp._rows(rows), "cp_page_select_workspace_bytes"
    lib, d, r, n = load(), ctypes.byref(desc), rows.tobytes(), rows.shape[0]
    _want(1 <= n_pages <= MAX_PAGES, f"{what}: 1 to {MAX_PAGES} pages")
    return _bytes(lib.cp_page_select_workspace_bytes(d, r, n, n_pages),
                  lambda: cp.check_batch(desc, rows) or cp.CP_ERR_UNSUPPORTED, what)


def page_select(desc, q, bounds, block_tables, rows, pages, n_first=1, n_last=1, ws=None,
                stream=None):
    """pages [T, Hkv, P] (int32): the P logical pages that every token reads, in
    rising order, -1 behind them: the first ``n_first``, the last ``n_last``, and of
    the others those whose bounds promise the largest product with a q head of
    the kv head's group.  ``ws``: uint8 of at least page_select_workspace_bytes
    (allocated here when None)."""
    what = "cp_page_select"
    rows = cp._rows(rows)
    dev, T = _device(q, what), _nodes(rows)
    hq, hkv, d = desc.num_q_heads, desc.num_kv_heads, desc.head_dim
    _want(pages.dim() == 3, "cp_page_select: pages is [T, Hkv, P]")
    P = pages.shape[2]
    ws, ws_ptr, ws_bytes = _workspace(ws, lambda: page_select_workspace_bytes(desc, rows, P), dev,
                                      stream, what)
    _check(_call(dev, stream, load().cp_page_select, ctypes.byref(desc),
                 _ptr(q, _BF16, (T, hq, d), dev, what),
                 _ptr(bounds, _BF16, (desc.num_blocks, hkv, 2, d), dev, what),
                 _table(desc, block_tables, dev, what), rows.tobytes(), rows.shape[0], P, n_first,
                 n_last, _ptr(pages, _I32, (T, hkv, P), dev, what), ws_ptr, ws_bytes), what)


def page_attn_workspace_bytes(desc, rows, n_pages) -> int:
    """Of this batch: a smaller one can need more (cp_cache.h states what serves all)."""
    rows, what = cp._rows(rows), "cp_page_attn_workspace_bytes"
    lib, d, r, n = load(), ctypes.byref(desc), rows.tobytes(), rows.shape[0]
    _want(1 <= n_pages <= MAX_PAGES, f"{what}: 1 to {MAX_PAGES} pages")
    return _bytes(lib.cp_page_attn_workspace_bytes(d, r, n, n_pages),
                  lambda: cp.check_batch(desc, rows) or cp.CP_ERR_UNSUPPORTED, what)


def page_attn(desc, q, k_cache, v_cache, block_tables, pages, rows, out, ws=None, stream=None):
    """out [T, Hq, D]: every token over the keys, up to its own, of the logical
    pages that pages [T, Hkv, P] (int32, as page_select writes them) names.
    ``ws``: uint8 of at least page_attn_workspace_bytes (allocated here when None)."""
    what = "cp_page_attn"
    rows = cp._rows(rows)
    dev, T = _device(q, what), _nodes(rows)
    hq, hkv, d = desc.num_q_heads, desc.num_kv_heads, desc.head_dim
    _want(pages.dim() == 3, "cp_page_attn: pages is [T, Hkv, P]")
    P = pages.shape[2]
    ws, ws_ptr, ws_bytes = _workspace(ws, lambda: page_attn_workspace_bytes(desc, rows, P), dev,
                                      stream, what)
    _check(_call(dev, stream, load().cp_page_attn, ctypes.byref(desc),
                 _ptr(q, _BF16, (T, hq, d), dev, what), _k_pool(desc, k_cache, dev, what),
                 _v_pool(desc, v_cache, dev, what),
                 _table(desc, block_tables, dev, what), _ptr(pages, _I32, (T, hkv, P), dev, what),
                 P, rows.tobytes(), rows.shape[0], _ptr(out, _BF16, (T, hq, d), dev, what), ws_ptr,
                 ws_bytes), what)


def _groups(groups):
    return np.ascontiguousarray(groups, dtype=np.int32).reshape(-1, 3)


def prefix_attn_workspace_bytes(desc, rows, groups) -> int:
    """Of this batch: a smaller one can need more (cp_cache.h states what serves all)."""
    rows, groups = cp._rows(rows), _groups(groups)
    lib, d = load(), ctypes.byref(desc)
    batch = rows.tobytes(), rows.shape[0], groups.tobytes(), groups.shape[0]

    def reason():   # the call's checks come before those of its buffers, of which it gets none
        rc = lib.cp_prefix_attn(d, *[None] * 4, *batch, None, None, 0, None)
        return cp.CP_ERR_UNSUPPORTED if rc == cp.CP_ERR_INVALID_ARG else rc
    return _bytes(lib.cp_prefix_attn_workspace_bytes(d, *batch),
                  lambda: cp.check_batch(desc, rows) or reason(),
                  "cp_prefix_attn_workspace_bytes")


def prefix_attn(desc, q, k_cache, v_cache, block_tables, rows, groups, out, ws=None, stream=None):
    """out [T, Hq, D]: causal attention of every token.  ``groups`` (host int32
    [n, 3]) are rows (first row, rows, tokens in common), rising: the full pages
    of the common tokens are the same in the group's rows of block_tables and
    are read once for all of them.  For decode rows and short chunks.  ``ws``:
    uint8 of at least prefix_attn_workspace_bytes (allocated here when None)."""
    what = "cp_prefix_attn"
    rows, groups = cp._rows(rows), _groups(groups)
    dev, T = _device(q, what), _nodes(rows)
    hq, d = desc.num_q_heads, desc.head_dim
    ws, ws_ptr, ws_bytes = _workspace(ws, lambda: prefix_attn_workspace_bytes(desc, rows, groups),
                                      dev, stream, what)
    _check(_call(dev, stream, load().cp_prefix_attn, ctypes.byref(desc),
                 _ptr(q, _BF16, (T, hq, d), dev, what), _k_pool(desc, k_cache, dev, what),
                 _v_pool(desc, v_cache, dev, what),
                 _table(desc, block_tables, dev, what), rows.tobytes(), rows.shape[0],
                 groups.tobytes(), groups.shape[0], _ptr(out, _BF16, (T, hq, d), dev, what), ws_ptr,
                 ws_bytes), what)
