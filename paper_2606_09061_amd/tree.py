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

import ctypes
import os

import numpy as np
import torch

from . import binding as cp
from .model import _scratch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libcptree.so")

MAX_NODES = 256      # CP_TREE_MAX_NODES
MAX_KEYS = 1 << 30   # CP_TREE_MAX_KEYS

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


def _ptr(t, dtype, shape, device, what):
    """The address of a dense tensor of this type and shape on this GPU (its
    index: comparing device objects costs as much as the other checks)."""
    if (t.dtype is not dtype or t.shape != shape or not t.is_contiguous()
            or t.get_device() != device or t.is_neg()):
        raise cp.CpError(cp.CP_ERR_INVALID_ARG,
                         f"{what}: a dense {dtype} tensor {tuple(shape)} on cuda:{device} is "
                         f"wanted, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _device(t, what):
    """The index of a tensor's GPU."""
    index = t.get_device()
    if index < 0:
        raise cp.CpError(cp.CP_ERR_INVALID_ARG,
                         f"{what}: tensors on a GPU are wanted, got {t.device}")
    return index


def _call(device, stream, f, *args):
    """f(*args, stream) with ``device`` current; the raw stream is looked up
    without the stream objects, which cost more than a launch."""
    if torch._C._cuda_getDevice() != device:
        with torch.cuda.device(device):
            return f(*args, cp._stream(stream))
    if stream is None:
        return f(*args, torch._C._cuda_getCurrentRawStream(device))
    return f(*args, cp._stream(stream))


def _workspace(ws, nbytes, device, stream, what):
    """(address, bytes) of ws, allocated for the stream when None (and returned,
    to be held until the launches are enqueued)."""
    if ws is None:
        ws = _scratch(nbytes(), torch.device("cuda", device), stream)
        if ws is None:
            raise cp.CpError(cp.CP_ERR_WORKSPACE, what)
    if ws.get_device() != device or not ws.is_contiguous():
        raise cp.CpError(cp.CP_ERR_INVALID_ARG, f"{what}: ws is dense and on cuda:{device}")
    return ws, ws.data_ptr(), ws.numel() * ws.element_size()


def _nodes(rows):
    n = rows[:, 2]
    return int(n.sum()) if len(n) > 32 else sum(n.tolist())   # (the faster of the two)


_I32, _I64, _BF16 = torch.int32, torch.int64, torch.bfloat16


def layout(parents, rows, mask, positions, stream=None):
    """mask [T, W] (int64, bit j of a node's W words: it sees node j of its row)
    and positions [T] (int32) of the drafted nodes whose parents (int32 [T],
    indexes inside their row, -1 for the root) are given."""
    what = "cp_tree_layout"
    rows = cp._rows(rows)
    dev, T = _device(parents, what), _nodes(rows)
    _want(mask.dim() == 2, "cp_tree_layout: mask is [T, W]")
    W = mask.shape[1]
    _check(_call(dev, stream, load().cp_tree_layout, _ptr(parents, _I32, (T,), dev, what),
                 rows.tobytes(), rows.shape[0], _ptr(mask, _I64, (T, W), dev, what), W,
                 _ptr(positions, _I32, (T,), dev, what)), what)


def attn_workspace_bytes(desc, rows) -> int:
    rows = cp._rows(rows)
    n = load().cp_tree_attn_workspace_bytes(ctypes.byref(desc), rows.tobytes(), rows.shape[0])
    if n == 0:
        rc = cp.check_batch(desc, rows)
        if rc == cp.CP_OK:   # what the tree attention checks beyond it
            rc = cp.CP_ERR_BAD_META if (rows[:, 2] > MAX_NODES).any() else cp.CP_ERR_UNSUPPORTED
        raise cp.CpError(rc, "cp_tree_attn_workspace_bytes")
    return int(n)


def attn(desc, q, k_cache, v_cache, block_tables, mask, rows, out, ws=None, stream=None):
    """out [T, Hq, D]: every drafted node over its request's committed keys and
    the nodes that its mask (int64 [T, W]) names, MAX_KEYS keys a row at most.
    ``ws``: uint8 of at least attn_workspace_bytes (allocated here when None)."""
    what = "cp_tree_attn"
    rows = cp._rows(rows)
    dev, T = _device(q, what), _nodes(rows)
    hq, hkv, d, b, nb = (desc.num_q_heads, desc.num_kv_heads, desc.head_dim, desc.block_size,
                         desc.num_blocks)
    _want(mask.dim() == 2, "cp_tree_attn: mask is [T, W]")
    W = mask.shape[1]
    ws, ws_ptr, ws_bytes = _workspace(ws, lambda: attn_workspace_bytes(desc, rows), dev, stream,
                                      what)
    _check(_call(dev, stream, load().cp_tree_attn, ctypes.byref(desc),
                 _ptr(q, _BF16, (T, hq, d), dev, what),
                 _ptr(k_cache, _BF16, (nb, hkv, b, d), dev, what),
                 _ptr(v_cache, _BF16, (nb, hkv, d, b), dev, what),
                 _ptr(block_tables, _I32, (desc.num_reqs_in_table, desc.max_blocks_per_req), dev,
                      what), _ptr(mask, _I64, (T, W), dev, what), W, rows.tobytes(),
                 rows.shape[0], _ptr(out, _BF16, (T, hq, d), dev, what), ws_ptr, ws_bytes), what)


def verify_workspace_bytes(n_tokens, vocab) -> int:
    """Bytes of verify's ``ws`` for batches of up to n_tokens nodes."""
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
    what = "cp_tree_verify"
    rows = cp._rows(rows)
    dev, T, R = _device(logits, what), _nodes(rows), rows.shape[0]
    _want(logits.dim() == 2 and logits.dtype == _BF16 and logits.shape[0] == T
          and (logits.stride(1) == 1 or logits.shape[1] == 1 or T == 0) and not logits.is_neg(),
          "cp_tree_verify: logits are bf16 [T, V] with dense rows")
    _want(path.dim() == 2, "cp_tree_verify: path is [R, P]")
    vocab, P = logits.shape[1], path.shape[1]
    ld = logits.stride(0) if T > 1 else vocab
    ws, ws_ptr, ws_bytes = _workspace(ws, lambda: verify_workspace_bytes(T, vocab), dev, stream,
                                      what)
    _check(_call(dev, stream, load().cp_tree_verify, logits.data_ptr(), ld, vocab,
                 _ptr(tokens, _I32, (T,), dev, what), _ptr(parents, _I32, (T,), dev, what),
                 rows.tobytes(), R, P, _ptr(target, _I32, (T,), dev, what),
                 _ptr(path, _I32, (R, P), dev, what), _ptr(n_accepted, _I32, (R,), dev, what),
                 _ptr(next_token, _I32, (R,), dev, what), ws_ptr, ws_bytes), what)


class KvLayers:
    """The K/V pools of a model's layers, as kv_compact and kv_fork take them:
    checked once (none may share memory with another: what is moved in one
    would move again in the next), and kept alive by this handle."""

    def __init__(self, desc, k_caches, v_caches):
        _want(len(k_caches) == len(v_caches) > 0, "kv_layers: one K and one V pool per layer")
        hkv, d, b = desc.num_kv_heads, desc.head_dim, desc.block_size
        self.device = _device(k_caches[0], "kv_layers")
        self.desc, self.n = cp.Desc.from_buffer_copy(desc), len(k_caches)
        self.pools = list(k_caches), list(v_caches)   # kept alive
        self.k, self.v = (
            (ctypes.c_void_p * self.n)(*(_ptr(t, _BF16, (desc.num_blocks, hkv, *page), self.device,
                                              "kv_layers") for t in pools))
            for pools, page in zip(self.pools, ((b, d), (d, b))))
        at = sorted([*self.k, *self.v])
        _want(all(y - x >= 2 * desc.num_blocks * hkv * d * b for x, y in zip(at, at[1:])),
              "kv_layers: no two pools share memory")

    def table(self, block_tables, what):
        d = self.desc
        return _ptr(block_tables, _I32, (d.num_reqs_in_table, d.max_blocks_per_req), self.device,
                    what)


def kv_layers(desc, k_caches, v_caches) -> KvLayers:
    return KvLayers(desc, k_caches, v_caches)


def kv_compact(layers, block_tables, rows, path, n_accepted, stream=None):
    """Moves the K/V of each row's accepted nodes, path [R, P] and n_accepted [R]
    (int32, as verify writes them), to slots start, start + 1, ..., in every
    layer of ``layers`` (kv_layers)."""
    what = "cp_kv_compact"
    rows = cp._rows(rows)
    dev, R = layers.device, rows.shape[0]
    _want(path.dim() == 2, "cp_kv_compact: path is [R, P]")
    P = path.shape[1]
    _check(_call(dev, stream, load().cp_kv_compact, ctypes.byref(layers.desc), layers.k, layers.v,
                 layers.n, layers.table(block_tables, what), rows.tobytes(), R,
                 _ptr(path, _I32, (R, P), dev, what), P, _ptr(n_accepted, _I32, (R,), dev, what)),
           what)


def kv_fork(layers, block_tables, forks, stream=None):
    """Forks requests: ``forks`` (host int32 [n, 4]) are rows (source request, new
    request, tokens in common, free block for the partly filled page).  The
    new request's row of block_tables is filled in, and the page copied in
    every layer of ``layers`` (kv_layers)."""
    forks = np.ascontiguousarray(forks, dtype=np.int32).reshape(-1, 4)
    what = "cp_kv_fork"
    _check(_call(layers.device, stream, load().cp_kv_fork, ctypes.byref(layers.desc), layers.k,
                 layers.v, layers.n, layers.table(block_tables, what), forks.tobytes(),
                 forks.shape[0]), what)
