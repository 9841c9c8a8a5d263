"""Speculative decoding and forked requests over the paged cache (libcptree.so).

A drafted row is a row of the attention step, ``(req, start, nodes, ctx)``:
its nodes are guessed tokens that hang together as a tree, node 0 the last
token known.  One iteration verifies all of them:

    layout       masks and rotary positions from the nodes' parents
    kv_append    (the attention step's) the nodes' K/V behind the committed keys
    attn         every node over the committed keys and its ancestors
    verify       each node's greedy token, and the path that agrees with it
    kv_compact   the accepted nodes' K/V moved up, in every layer
    kv_fork      requests that continue another one's tokens

The calls check their tensors (dense, type, shape, one device) and raise
:class:`CpError`; outputs are written into the caller's tensors, on ``stream``
or the current stream of their device.
"""

from __future__ import annotations

import contextlib
import ctypes
import os

import numpy as np

from . import binding as cp
from .model import _scratch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libcptree.so")

MAX_NODES = 256   # CP_TREE_MAX_NODES

_lib = None


def load():
    """Loads libcptree.so; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it first "
                           "(python -m paper_2606_09061_amd.build)")
    lib = ctypes.CDLL(LIB_PATH)
    P, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    lib.cp_tree_layout.argtypes = [P, P, I32, P, I32, P, P]
    lib.cp_tree_attn_workspace_bytes.argtypes = [P, P, I32]
    lib.cp_tree_attn_workspace_bytes.restype = SZ
    lib.cp_tree_attn.argtypes = [P, P, P, P, P, P, I32, P, I32, P, P, SZ, P]
    lib.cp_tree_verify_workspace_bytes.argtypes = [I64, I32]
    lib.cp_tree_verify_workspace_bytes.restype = SZ
    lib.cp_tree_verify.argtypes = [P, I64, I32, P, P, P, I32, I32, P, P, P, P, P, SZ, P]
    lib.cp_kv_compact.argtypes = [P, P, P, I32, P, P, I32, P, I32, P, P]
    lib.cp_kv_fork.argtypes = [P, P, P, I32, P, P, I32, P]
    for f in (lib.cp_tree_layout, lib.cp_tree_attn, lib.cp_tree_verify, lib.cp_kv_compact,
              lib.cp_kv_fork):
        f.restype = ctypes.c_int
    _lib = lib
    return lib


def exported_symbols():
    return ["cp_tree_layout", "cp_tree_attn_workspace_bytes", "cp_tree_attn",
            "cp_tree_verify_workspace_bytes", "cp_tree_verify", "cp_kv_compact", "cp_kv_fork"]


def _check(rc, what):
    if rc != cp.CP_OK:
        raise cp.CpError(rc, what)


def _want(ok, what):
    if not ok:
        raise cp.CpError(cp.CP_ERR_INVALID_ARG, what)


def _tensors(what, device, *wanted):
    """Each of ``wanted`` is (tensor, dtype, shape): a dense tensor like that on
    ``device``."""
    for t, dtype, shape in wanted:
        if (t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous()
                or t.device != device or t.is_neg()):
            raise cp.CpError(cp.CP_ERR_INVALID_ARG,
                             f"{what}: a dense {dtype} tensor {shape} on {device} is wanted, got "
                             f"{t.dtype} {tuple(t.shape)} on {t.device}")


def _device(t, what):
    _want(t.is_cuda, f"{what}: tensors on a GPU are wanted, got {t.device}")
    return t.device


def _at(device):
    """Makes ``device`` current for the launches of a call."""
    import torch
    if torch.cuda.current_device() == device.index:
        return contextlib.nullcontext()
    return torch.cuda.device(device)


def _nodes(rows):
    return int(rows[:, 2].sum()) if len(rows) else 0


def layout(parents, rows, mask, positions, stream=None):
    """mask [T, W] (int64, bit j of a node's W words: it sees node j of its row)
    and positions [T] (int32) of the drafted nodes whose parents (int32 [T],
    indexes inside their row, -1 for the root) are given."""
    import torch
    rows = cp._rows(rows)
    T = _nodes(rows)
    _want(mask.dim() == 2, "cp_tree_layout: mask is [T, W]")
    dev = _device(parents, "cp_tree_layout")
    _tensors("cp_tree_layout", dev, (parents, torch.int32, (T,)),
             (mask, torch.int64, (T, mask.shape[1])), (positions, torch.int32, (T,)))
    with _at(dev):
        _check(load().cp_tree_layout(parents.data_ptr(), rows.ctypes.data, rows.shape[0],
                                     mask.data_ptr(), mask.shape[1], positions.data_ptr(),
                                     cp._stream(stream)), "cp_tree_layout")


def attn_workspace_bytes(desc, rows) -> int:
    rows = cp._rows(rows)
    n = load().cp_tree_attn_workspace_bytes(ctypes.byref(desc), rows.ctypes.data, rows.shape[0])
    if n == 0:
        rc = cp.check_batch(desc, rows)
        raise cp.CpError(rc if rc != cp.CP_OK else cp.CP_ERR_BAD_META,
                         "cp_tree_attn_workspace_bytes")
    return int(n)


def attn(desc, q, k_cache, v_cache, block_tables, mask, rows, out, ws=None, stream=None):
    """out [T, Hq, D]: every drafted node over its request's committed keys and
    the nodes that its mask (int64 [T, W]) names.  ``ws``: uint8 of at least
    attn_workspace_bytes (allocated here when None)."""
    import torch
    rows = cp._rows(rows)
    T, bf16 = _nodes(rows), torch.bfloat16
    hq, hkv, d, b = desc.num_q_heads, desc.num_kv_heads, desc.head_dim, desc.block_size
    _want(mask.dim() == 2, "cp_tree_attn: mask is [T, W]")
    dev = _device(q, "cp_tree_attn")
    _tensors("cp_tree_attn", dev, (q, bf16, (T, hq, d)), (out, bf16, (T, hq, d)),
             (k_cache, bf16, (desc.num_blocks, hkv, b, d)),
             (v_cache, bf16, (desc.num_blocks, hkv, d, b)),
             (block_tables, torch.int32, (desc.num_reqs_in_table, desc.max_blocks_per_req)),
             (mask, torch.int64, (T, mask.shape[1])))
    if ws is None:
        ws = _scratch(attn_workspace_bytes(desc, rows), dev, stream)
        if ws is None:
            raise cp.CpError(cp.CP_ERR_WORKSPACE, "cp_tree_attn")
    _want(ws.device == dev and ws.is_contiguous(), "cp_tree_attn: ws is on another device")
    with _at(dev):
        _check(load().cp_tree_attn(ctypes.byref(desc), q.data_ptr(), k_cache.data_ptr(),
                                   v_cache.data_ptr(), block_tables.data_ptr(), mask.data_ptr(),
                                   mask.shape[1], rows.ctypes.data, rows.shape[0], out.data_ptr(),
                                   ws.data_ptr(), ws.numel() * ws.element_size(),
                                   cp._stream(stream)), "cp_tree_attn")


def verify_workspace_bytes(n_tokens, vocab) -> int:
    n = load().cp_tree_verify_workspace_bytes(int(n_tokens), int(vocab))
    if n == 0:
        raise cp.CpError(cp.CP_ERR_INVALID_ARG, "cp_tree_verify_workspace_bytes")
    return int(n)


def verify(logits, tokens, parents, rows, target, path, n_accepted, next_token, ws=None,
           stream=None):
    """Greedy verification of drafted trees.  logits [T, V] (bf16, rows dense, at
    any stride) and tokens, parents [T] (int32) give target [T], each node's
    greedy token; path [R, P], the accepted nodes of each row, -1 behind them;
    n_accepted [R] and next_token [R] (all int32)."""
    import torch
    rows = cp._rows(rows)
    T, R, i32 = _nodes(rows), rows.shape[0], torch.int32
    dev = _device(logits, "cp_tree_verify")
    _want(logits.dim() == 2 and logits.dtype == torch.bfloat16 and logits.shape[0] == T
          and (logits.stride(1) == 1 or logits.shape[1] == 1 or T == 0) and not logits.is_neg(),
          "cp_tree_verify: logits are bf16 [T, V] with dense rows")
    _want(path.dim() == 2, "cp_tree_verify: path is [R, P]")
    _tensors("cp_tree_verify", dev, (tokens, i32, (T,)), (parents, i32, (T,)),
             (target, i32, (T,)), (path, i32, (R, path.shape[1])), (n_accepted, i32, (R,)),
             (next_token, i32, (R,)))
    vocab = logits.shape[1]
    ld = logits.stride(0) if T > 1 else vocab
    if ws is None:
        ws = _scratch(verify_workspace_bytes(T, vocab), dev, stream)
        if ws is None:
            raise cp.CpError(cp.CP_ERR_WORKSPACE, "cp_tree_verify")
    _want(ws.device == dev and ws.is_contiguous(), "cp_tree_verify: ws is on another device")
    with _at(dev):
        _check(load().cp_tree_verify(logits.data_ptr(), ld, vocab, tokens.data_ptr(),
                                     parents.data_ptr(), rows.ctypes.data, R, path.shape[1],
                                     target.data_ptr(), path.data_ptr(), n_accepted.data_ptr(),
                                     next_token.data_ptr(), ws.data_ptr(),
                                     ws.numel() * ws.element_size(), cp._stream(stream)),
               "cp_tree_verify")


class KvLayers:
    """The K/V pools of a model's layers, as kv_compact and kv_fork take them:
    checked once, and kept alive by this handle."""

    def __init__(self, desc, k_caches, v_caches):
        import torch
        _want(len(k_caches) == len(v_caches) > 0, "kv_layers: one K and one V pool per layer")
        hkv, d, b = desc.num_kv_heads, desc.head_dim, desc.block_size
        self.device = _device(k_caches[0], "kv_layers")
        for k, v in zip(k_caches, v_caches):
            _tensors("kv_layers", self.device, (k, torch.bfloat16, (desc.num_blocks, hkv, b, d)),
                     (v, torch.bfloat16, (desc.num_blocks, hkv, d, b)))
        self.desc, self.n = desc, len(k_caches)
        self.pools = list(k_caches), list(v_caches)
        self.k, self.v = ((ctypes.c_void_p * self.n)(*(t.data_ptr() for t in p))
                          for p in self.pools)


def kv_layers(desc, k_caches, v_caches) -> KvLayers:
    return KvLayers(desc, k_caches, v_caches)


def _table(layers, block_tables, what):
    import torch
    d = layers.desc
    _tensors(what, layers.device,
             (block_tables, torch.int32, (d.num_reqs_in_table, d.max_blocks_per_req)))


def kv_compact(layers, block_tables, rows, path, n_accepted, stream=None):
    """Moves the K/V of each row's accepted nodes, path [R, P] and n_accepted [R]
    (int32, as verify writes them), to slots start, start + 1, ..., in every
    layer of ``layers`` (kv_layers)."""
    import torch
    rows = cp._rows(rows)
    R = rows.shape[0]
    _table(layers, block_tables, "cp_kv_compact")
    _want(path.dim() == 2, "cp_kv_compact: path is [R, P]")
    _tensors("cp_kv_compact", layers.device, (path, torch.int32, (R, path.shape[1])),
             (n_accepted, torch.int32, (R,)))
    with _at(layers.device):
        _check(load().cp_kv_compact(ctypes.byref(layers.desc), layers.k, layers.v, layers.n,
                                    block_tables.data_ptr(), rows.ctypes.data, R, path.data_ptr(),
                                    path.shape[1], n_accepted.data_ptr(), cp._stream(stream)),
               "cp_kv_compact")


def kv_fork(layers, block_tables, forks, stream=None):
    """Forks requests: ``forks`` (host int32 [n, 4]) are rows (source request, new
    request, tokens in common, free block for the partly filled page).  The
    new request's row of block_tables is filled in, and the page copied in
    every layer of ``layers`` (kv_layers)."""
    forks = np.ascontiguousarray(forks, dtype=np.int32).reshape(-1, 4)
    _table(layers, block_tables, "cp_kv_fork")
    with _at(layers.device):
        _check(load().cp_kv_fork(ctypes.byref(layers.desc), layers.k, layers.v, layers.n,
                                 block_tables.data_ptr(), forks.ctypes.data, forks.shape[0],
                                 cp._stream(stream)), "cp_kv_fork")
