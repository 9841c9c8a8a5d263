"""A Qwen3-style decoder stack around the attention step, on one GPU.

The paper's predictor and target latency T* refer to a whole model iteration
(Sec. 3.2.1; Sec. 4.4 uses Qwen3-8B with T* = 105 ms), so this module runs the
scheduler's batch through every layer of such a model with synthetic weights:

    embedding -> L x [RMSNorm -> QKV GEMM -> cpl_qkv_rope -> cp_kv_append ->
    cp_attn_mixed -> O GEMM (+ residual) -> RMSNorm -> gate/up GEMM ->
    cpl_swiglu -> down GEMM (+ residual)] -> RMSNorm -> LM head on each row's
    last token -> argmax

``Model.verify`` runs the same layers over trees of drafted tokens
(libcptree.so): every node's logits, the accepted path, its K/V moved up.

Every step runs in this package's HIP kernels (libcplayer.so for the
projections and the element-wise parts, libcpattn.so for append and
attention); the largest of the feed-forward's projections, and those of shapes
or tensors that the kernels do not take, run as library GEMMs (torch.mm /
addmm, i.e. hipBLASLt).  Each layer has
its own paged KV pool; all layers share one block table, whose row s maps
slot s's logical blocks to physical blocks (a random permutation, so pages
are scattered).  Weights are N(0, 0.02) in bf16, norms 1.
"""

from __future__ import annotations

import contextlib
import ctypes
import math
import os
from dataclasses import dataclass

import numpy as np

from . import binding as cp

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libcplayer.so")

_lib = None


def load():
    """Loads libcplayer.so; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it first "
                           "(python -m paper_2606_09061_amd.build)")
    lib = ctypes.CDLL(LIB_PATH)
    P, I32, F, D = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float, ctypes.c_double
    lib.cpl_rmsnorm.argtypes = [P, P, P, I32, I32, F, P]
    lib.cpl_qkv_rope.argtypes = [P, P, P, P, I32, I32, I32, I32, D, F, P, P, P, P]
    lib.cpl_swiglu.argtypes = [P, P, I32, I32, P]
    lib.cpl_gemm_skinny.argtypes = [P, P, P, P, I32, I32, I32, P]
    lib.cpl_gemm.argtypes = [P, P, P, P, I32, I32, I32, P, ctypes.c_size_t, P]
    lib.cpl_gemm_workspace_bytes.argtypes = [I32, I32, I32]
    lib.cpl_gemm_workspace_bytes.restype = ctypes.c_size_t
    for f in (lib.cpl_rmsnorm, lib.cpl_qkv_rope, lib.cpl_swiglu, lib.cpl_gemm_skinny, lib.cpl_gemm):
        f.restype = ctypes.c_int
    _lib = lib
    return lib


def exported_symbols():
    return ["cpl_rmsnorm", "cpl_qkv_rope", "cpl_swiglu", "cpl_gemm_skinny", "cpl_gemm",
            "cpl_gemm_workspace_bytes"]


def _check(rc, what):
    if rc != 0:
        raise cp.CpError(rc, what)


def _s(stream):
    return cp._stream(stream)


def _dense(*ts):
    for t in ts:
        if not t.is_contiguous():
            raise cp.CpError(cp.CP_ERR_INVALID_ARG, "layer kernels take dense tensors")


def rmsnorm(x, w, out, eps, stream=None):
    """out = RMSNorm(x) * w over the last axis (bf16 tensors; out may be x)."""
    _dense(x, w, out)
    n, width = x.shape[0], x.shape[-1]
    _check(load().cpl_rmsnorm(x.data_ptr(), w.data_ptr(), out.data_ptr(), n, width, eps,
                              _s(stream)), "cpl_rmsnorm")


def qkv_rope(qkv, q_norm_w, k_norm_w, positions, hq, hkv, head_dim, theta, eps, q, k, v,
             stream=None):
    """Splits qkv [T, (hq+2hkv)*D] into q [T, hq, D], k, v [T, hkv, D] with
    per-head RMSNorm and rotary embedding of q and k (positions: int32 [T])."""
    _dense(qkv, q_norm_w, k_norm_w, positions, q, k, v)
    _check(load().cpl_qkv_rope(qkv.data_ptr(), q_norm_w.data_ptr(), k_norm_w.data_ptr(),
                               positions.data_ptr(), qkv.shape[0], hq, hkv, head_dim,
                               float(theta), eps, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                               _s(stream)), "cpl_qkv_rope")


def swiglu(gu, out, stream=None):
    """out [T, I] = silu(gu[:, :I]) * gu[:, I:]."""
    _dense(gu, out)
    _check(load().cpl_swiglu(gu.data_ptr(), out.data_ptr(), gu.shape[0], out.shape[-1],
                             _s(stream)), "cpl_swiglu")


# Where the skinny kernel beats the library GEMM on MI355X.  Per launch, with
# the weights evicted from the caches beforehand (a model iteration streams
# 15 GB of weights), at one row: QKV 24.0 -> 14.2 us, O 21.0 -> 11.1, gate/up
# 79.3 -> 34.0, down 40.8 -> 23.5, LM head 288 -> 178; at 32 rows still
# 1.19-1.97x on all five.  A whole 36-layer decode iteration with this
# dispatch against the library alone: 1.29x at 1 row, 1.23x at 8, 1.18x at
# 16, 1.08x at 24, 1.03x at 32, even at 40 rows (each 32-column slice
# re-reads the activations), hence no skinny kernel above 32 rows.
def skinny_faster(m, n, k):
    if n % 32 or k % 256 or m < 1:
        return False
    return m <= 32


# Where, of those, the skinny kernel is the faster one too (skinny / tiled us a
# launch, weights from HBM, at the row counts named):
# * Up to 7 rows; where N is not a multiple of 128 there is only the skinny one.
# * Up to 32 M weights.  QKV (6144 x 4096) 11.4 / 13.0 at 1 row, 13.1 / 14.2 at
#   24, 14.8 / 14.6 at 32; 8192 x 4096 13.2 / 15.0 at 17, 14.8 / 15.6 at 28.
#   Below, a step of the layer waits for the host, and the split's second
#   launch and scratch cost more than the kernel gains (down 2048 x 6144 10.8 /
#   9.2 at 8 rows, but its feed-forward block 31 / 45; the projections around
#   the step at hidden 4,096, 32 rows, 34.3 / 37.7).
# * Up to 16 rows otherwise: gate/up (24576 x 4096) 33.7 / 35.8 at 16; each
#   slice of columns streams the activations again, so that it loses with more
#   rows (gate/up 36.8 / 36.3 at 20, 42.3 / 37.7 at 32; LM head, 151936 x 4096,
#   196 / 194 at 16, 209 / 196 at 20).  N below 8,192 lasts to 24 (7168 x 7168
#   20.0 / 20.8 at 17, 21.9 / 21.8 at 24).
# * Up to 20 rows where its slices of 32 columns fill the CUs' rounds and the
#   tiles of 64 do not: gate/up 33.7 / 36.0 at 17, 35.1 / 36.1 at 19; 22016 x
#   4096 32.8 / 35.7 at 17; but 16384 x 4096 (whole rounds of tiles) 24.4 / 22.9
#   at 20, and with longer rows 8192 x 8192 29.7 / 25.7 at 17.
# * Long rows (K > N) up to 12, if the slices fill the CUs: 8192 x 28672 69.5 /
#   73.8 at 8, 73.3 / 73.8 at 16; 8192 x 12288 33.6 / 34.5 at 12, 34.7 / 33.4 at
#   16.  Else they need more workgroups than the slices give, which the tiled
#   kernel's split over K has: 4096 x 12288 21.2 / 19.2 at 8, 31.8 / 20.8 at 32;
#   12288 x 14336 63.4 / 55.4 at 8.
def _skinny_fastest(m, n, k):
    if m > 32 or n % 32 or k % 256 or m < 1:
        return False
    if m < 8 or n * k <= 32 << 20 or n % 128 != 0:
        return True
    if k <= n and (m <= 16 or (m <= 24 and n < 8192)):
        return True

    def filled(workgroups):   # share of whole rounds of 256 CUs
        return workgroups / (-(-workgroups // 256) * 256)
    if filled(n // 32) < 8 / 9:
        return False
    return m <= 12 if k > n else m <= 20 and k <= 4096 and filled(n // 64) <= 0.75


def gemm_skinny(a, w, out, residual=None, stream=None):
    """out [M, N] = a [M, K] @ w [N, K]^T (+ residual, which may be out itself)."""
    _dense(a, w, out)
    if residual is not None:
        _dense(residual)
    M, K = a.shape
    N = w.shape[0]
    _check(load().cpl_gemm_skinny(a.data_ptr(), w.data_ptr(),
                                  residual.data_ptr() if residual is not None else None,
                                  out.data_ptr(), M, N, K, _s(stream)), "cpl_gemm_skinny")


def gemm_workspace_bytes(m, n, k):
    """Device bytes cpl_gemm uses to split K for this shape (0: no split)."""
    return int(load().cpl_gemm_workspace_bytes(m, n, k))


def _on(stream, device):
    """Makes a `stream` argument torch's current stream (None: it stays)."""
    import torch
    if stream is None or device.type != "cuda":
        return contextlib.nullcontext()
    if isinstance(stream, int):
        stream = (torch.cuda.ExternalStream(stream, device=device) if stream
                  else torch.cuda.default_stream(device))
    return torch.cuda.stream(stream)


def _scratch(nbytes, device, stream):
    """Device bytes that belong to the stream the kernels run on, so that the
    allocator hands them out again only behind those kernels; None when there
    are none to be had."""
    import torch
    try:
        with _on(stream, device):
            return torch.empty(nbytes, dtype=torch.uint8, device=device)
    except torch.cuda.OutOfMemoryError:
        return None


def gemm(a, w, out, residual=None, stream=None, ws=None):
    """out [M, N] = a [M, K] @ w [N, K]^T (+ residual, which may be out itself),
    on the package's LDS-tiled MFMA kernel (cpl_gemm).  ``ws``: a uint8 device
    tensor for the split over K (allocated here when None and needed)."""
    _dense(a, w, out)
    if residual is not None:
        _dense(residual)
    M, K = a.shape
    N = w.shape[0]
    if ws is None:
        need = gemm_workspace_bytes(M, N, K)
        if need:
            ws = _scratch(need, a.device, stream)
    _check(load().cpl_gemm(a.data_ptr(), w.data_ptr(),
                           residual.data_ptr() if residual is not None else None,
                           out.data_ptr(), M, N, K, ws.data_ptr() if ws is not None else None,
                           ws.numel() if ws is not None else 0, _s(stream)), "cpl_gemm")


def _aligned(*ts):
    return all(t is None or t.data_ptr() % 16 == 0 for t in ts)


def project_attn(a, w, out, residual=None, stream=None, ws=None):
    """The QKV and output projections around the attention step, always on
    the package's kernels: the skinny kernel for the smallest batches, the
    tiled MFMA GEMM above (``ws``: its split-K workspace, see gemm)."""
    M, K = a.shape
    N = w.shape[0]
    if _skinny_fastest(M, N, K) or (M <= 32 and skinny_faster(M, N, K)
                                    and not _aligned(out, residual, ws)):
        gemm_skinny(a, w, out, residual, stream)
    elif N % 128 == 0 and K % 32 == 0:
        gemm(a, w, out, residual, stream, ws)
    else:
        raise ValueError(f"projection {M}x{N}x{K}: the kernels need N % 128 == 0 and K % 32 == 0")


def _apart(x, y):
    """Whether two dense bf16 tensors share no byte."""
    px, py = x.data_ptr(), y.data_ptr()
    return px + 2 * x.numel() <= py or py + 2 * y.numel() <= px


def _function_mode():
    """Whether a torch function mode other than a default device's is active."""
    import torch
    from torch.utils._device import DeviceContext
    return any(type(torch._C._get_function_stack_at(i)) is not DeviceContext
               for i in range(torch._C._len_torch_function_stack()))


def _watched():
    """Whether torch has to see the operations of this call: under the compiler,
    in a trace, inside a dispatch or function mode (flop counters, tracers; the
    mode of a default device concerns only factories)."""
    import torch
    return (torch.compiler.is_compiling() or torch._C._get_tracing_state() is not None
            or torch._C._len_torch_dispatch_stack() > 0
            or (torch._C._len_torch_function_stack() > 0 and _function_mode()))


def _tiled_takes(a, w, out, residual):
    """Whether cpl_gemm can stand in for torch.mm / addmm here: plain dense
    bf16 matrices of matching shapes on the current GPU, 16-byte aligned, that
    autograd does not follow (backward, or forward: inside a dual level) and no
    function transform wraps, with no operand under out except a residual that
    is out, and nobody watching.  Everything else is left to torch, which
    computes or refuses it."""
    import torch
    if (_watched() or not a.is_cuda or torch.autograd.forward_ad._current_level >= 0
            or torch._C._are_functorch_transforms_active()
            or (out.is_inference() and not torch.is_inference_mode_enabled())):
        return False
    dev = torch.cuda.current_device()
    for t in (a, w, out) if residual is None else (a, w, out, residual):
        if (type(t) not in (torch.Tensor, torch.nn.Parameter) or t.dtype != torch.bfloat16
                or t.dim() != 2 or t.get_device() != dev or not t.is_contiguous()
                or t.is_neg() or t.data_ptr() % 16
                or (t.requires_grad and torch.is_grad_enabled())):
            return False
    M, K = a.shape
    N = w.shape[0]
    if (M == 0 or K == 0 or N == 0 or N % 128 or K % 32 or w.shape[1] != K
            or out.shape != (M, N) or not _apart(a, out) or not _apart(w, out)):
        return False
    return residual is None or (residual.shape == out.shape
                                and (residual.data_ptr() == out.data_ptr()
                                     or _apart(residual, out)))


# Above 32 rows, where the library beats the tiled kernel (us, library / tiled,
# weights from HBM).  Long rows (K >= N) gain from the split over K: 4096 x
# 12288 121 / 92 at 1,000 rows, 186 / 161 at 2,048; 2048 x 6144 99 / 88 still at
# 4,096; only large ones past 2,048 rows lose (4096 x 12288 205 / 219 at 2,560,
# 286 / 277 at 4,096; 8192 x 28672 940 / 996 at 2,560).  Wide ones are bound by
# the products, and large ones run at a higher rate in the library: 24576 x 4096
# 49 / 42 at 100 rows, 88 / 83 at 512, 167 / 160 at 1,000, 164 / 160 at 1,024,
# but 184 / 188 at 1,100, 279 / 290 at 2,048, 542 / 561 at 4,096; 12288 x 2048
# 90 / 86 at 2,048, 92 / 93 at 2,100, 147 / 153 at 4,096 (the library's own bad
# sizes in between, 24576 x 4096 558 / 465 at 3,072, follow no rule).  Past 512
# rows, tiles that leave much of a round of 256 CUs idle lose where padded rows
# are a good part of it: 22016 x 4096 115 / 136 at 600 rows (0.53 of two rounds
# of 192 x 256, 600 rows of 768), 28672 x 4096 134 / 152 (0.68); but 24576 x
# 4096 147 / 142 at 700 (0.68, 700 rows of 768), 145 / 145 at 768 (0.75).
def _library_fastest(m, n, k):
    large = m * n * k > 1024 * 24576 * 4096
    if k >= n:
        return m > 2048 and large
    if m <= 512:
        return False
    if m > 2048 or large:
        return True

    def busy(rows, columns):   # share of the CUs' rounds
        rounds = -(-(-(-m // rows) * (n // columns)) // 256)
        return m * n / (rounds * 256 * rows * columns)
    if m >= 0.85 * -(-m // 192) * 192 or m >= 0.85 * -(-m // 256) * 256:
        return False
    tiles = [t for t in ((256, 256), (192, 256), (256, 192)) if n % t[1] == 0]
    return bool(tiles) and max(busy(*t) for t in tiles) < 0.78


def project(a, w, out, residual=None, stream=None, ws=None):
    """a @ w^T into out (+ residual), on the package's kernels like
    project_attn where they take the shapes and tensors, else on the platform
    BLAS (_library_fastest, _tiled_takes).  The feed-forward and LM-head
    projections use it.  Without ``ws`` the split's partials are allocated here:
    fp32, at most 8 x rows x N (65 MB for 4096 x 12288 at 1,000 rows)."""
    import torch
    M, K = a.shape
    N = w.shape[0]
    if _skinny_fastest(M, N, K):
        gemm_skinny(a, w, out, residual, stream)
    elif not _library_fastest(M, N, K) and _tiled_takes(a, w, out, residual):
        gemm(a, w, out, residual, stream, ws)
        if not skinny_faster(M, N, K) and not out.is_inference():
            torch.autograd.graph.increment_version(out)   # as torch's product does
    elif skinny_faster(M, N, K):
        gemm_skinny(a, w, out, residual, stream)
    else:
        with _on(stream, a.device):
            if residual is None:
                torch.mm(a, w.t(), out=out)
            elif residual is out:
                out.addmm_(a, w.t())
            else:
                torch.addmm(residual, a, w.t(), out=out)


@dataclass
class ModelConfig:
    hidden: int = 4096
    layers: int = 36
    hq: int = 32
    hkv: int = 8
    head_dim: int = 128
    inter: int = 12288
    vocab: int = 151936
    eps: float = 1e-6
    theta: float = 1e6
    block_size: int = 16


QWEN3_8B = ModelConfig()


def positions_of(rows) -> np.ndarray:
    """Absolute position of every scheduled token, in row order."""
    rows = np.asarray(rows).reshape(-1, 4)
    lens = rows[:, 2].astype(np.int64)
    if lens.sum() == 0:
        return np.zeros(0, np.int32)
    base = np.repeat(rows[:, 1].astype(np.int64) - np.concatenate([[0], np.cumsum(lens)[:-1]]),
                     lens)
    return (base + np.arange(lens.sum())).astype(np.int32)


class Model:
    """Synthetic-weight decoder stack with per-layer paged KV pools."""

    def __init__(self, cfg: ModelConfig = QWEN3_8B, max_seqs=128, max_seq_len=4096,
                 max_tokens=2048, seed=0, device=None, lm_head=True, fill_caches=False):
        import torch
        from workloads.tensors import _randn_bf16

        self.cfg = c = cfg
        self.dev = device or torch.device("cuda", 0)
        self.max_tokens = max_tokens
        gen = torch.Generator(device=self.dev)
        gen.manual_seed(seed)

        def w(*shape):
            t = _randn_bf16(shape, gen, self.dev)
            return t.mul_(0.02)

        def ones(n):
            return torch.ones(n, dtype=torch.bfloat16, device=self.dev)

        H, D = c.hidden, c.head_dim
        nqkv = (c.hq + 2 * c.hkv) * D
        self.layers = [dict(in_norm=ones(H), qkv=w(nqkv, H), q_norm=ones(D), k_norm=ones(D),
                            o=w(H, c.hq * D), post_norm=ones(H), gate_up=w(2 * c.inter, H),
                            down=w(H, c.inter)) for _ in range(c.layers)]
        self.embed = w(c.vocab, H)
        self.final_norm = ones(H)
        self.lm_head = w(c.vocab, H) if lm_head else None
        mbr = -(-max_seq_len // c.block_size)
        nb = max_seqs * mbr
        rng = np.random.default_rng(seed)
        self.bt = torch.from_numpy(rng.permutation(nb).astype(np.int32).reshape(max_seqs, mbr)
                                   ).to(self.dev)
        # Serving writes every position before attention reads it, so pools may
        # start unwritten; fill_caches draws N(0,1) contents for benchmarks
        # that attend to context they never appended.
        if fill_caches:
            self.kc = [_randn_bf16((nb, c.hkv, c.block_size, D), gen, self.dev)
                       for _ in range(c.layers)]
            self.vc = [_randn_bf16((nb, c.hkv, D, c.block_size), gen, self.dev)
                       for _ in range(c.layers)]
        else:
            self.kc = [torch.empty(nb, c.hkv, c.block_size, D, dtype=torch.bfloat16,
                                   device=self.dev) for _ in range(c.layers)]
            self.vc = [torch.empty(nb, c.hkv, D, c.block_size, dtype=torch.bfloat16,
                                   device=self.dev) for _ in range(c.layers)]
        self.desc = cp.make_desc(c.hq, c.hkv, D, c.block_size, nb, mbr, max_seqs,
                                 1.0 / math.sqrt(D))
        T = max_tokens

        def buf(*shape):
            return torch.empty(*shape, dtype=torch.bfloat16, device=self.dev)

        self.x, self.h = buf(T, H), buf(T, H)
        self.qkv = buf(T, nqkv)
        self.q, self.k, self.v = buf(T, c.hq, D), buf(T, c.hkv, D), buf(T, c.hkv, D)
        self.attn = buf(T, c.hq, D)
        self.gu, self.act = buf(T, 2 * c.inter), buf(T, c.inter)
        self.pos_host = torch.zeros(T, dtype=torch.int32).pin_memory()
        self.pos_copied = torch.cuda.Event()   # the last upload out of pos_host is done
        self.pos = torch.zeros(T, dtype=torch.int32, device=self.dev)
        self.tokens = torch.randint(0, c.vocab, (T,), generator=gen, device=self.dev)
        self.ws = torch.empty(64 << 20, dtype=torch.uint8, device=self.dev)      # attention plan
        # split-K partials of the projections (grown on demand)
        self.ws_gemm = torch.empty(256, dtype=torch.uint8, device=self.dev)
        # an append item covers one row's tokens inside one block: at most
        # max_tokens + max_seqs items of 16 bytes, so the append never needs more
        self.ws_append = torch.empty(16 * (max_tokens + max_seqs) + 256, dtype=torch.uint8,
                                     device=self.dev)

    def forward(self, rows, stream=None):
        """Runs one iteration for the batch ``rows`` [(slot, start, len, ctx)];
        returns the greedy next token of every row (device int64 [n_rows]), or
        None when the model has no LM head."""
        import torch
        c = self.cfg
        rows = np.ascontiguousarray(np.asarray(rows, dtype=np.int32).reshape(-1, 4))
        T = int(rows[:, 2].sum())
        if T == 0:
            return None
        if T > self.max_tokens:
            raise ValueError(f"batch of {T} tokens exceeds the model's {self.max_tokens}")
        s = stream or torch.cuda.current_stream(self.dev)
        pos = positions_of(rows)
        self.pos_copied.synchronize()   # the previous iteration's upload has left pos_host
        self.pos_host[:T].numpy()[:] = pos
        with torch.cuda.stream(s):
            self.pos[:T].copy_(self.pos_host[:T], non_blocking=True)
            self.pos_copied.record(s)
            x = self.x[:T]
            torch.index_select(self.embed, 0, self.tokens[:T], out=x)
            # every layer attends with the same rows: plan once, run per layer
            # (the plan is built once per iteration; only a workspace that is
            # too small costs a second planning, to learn the size)
            try:
                plan = cp.attn_prepare(self.desc, rows, self.ws, stream=s)
            except cp.CpError as e:
                if e.code != cp.CP_ERR_WORKSPACE:
                    raise
                self.ws = torch.empty(cp.workspace_bytes(self.desc, rows), dtype=torch.uint8,
                                      device=self.dev)
                plan = cp.attn_prepare(self.desc, rows, self.ws, stream=s)
            self._layers(rows, T, int((rows[:, 2] > 0).sum()), s,
                         lambda q, kc, vc, out: cp.attn_run(plan, q, kc, vc, self.bt, out, self.ws,
                                                            stream=s))
            if self.lm_head is None:
                return None
            last = torch.from_numpy(np.cumsum(rows[:, 2]).astype(np.int64) - 1)
            last = last[rows[:, 2] > 0].to(self.dev, non_blocking=True)
            hl = torch.empty(len(last), c.hidden, dtype=torch.bfloat16, device=self.dev)
            rmsnorm(x.index_select(0, last), self.final_norm, hl, c.eps, s)
            logits = torch.empty(len(last), c.vocab, dtype=torch.bfloat16, device=self.dev)
            project(hl, self.lm_head, logits, None, s, self.ws_gemm)
            return torch.argmax(logits, dim=-1)

    def _layers(self, rows, T, n_head, s, attend):
        """The decoder layers over the embeddings in x[:T], whose positions are in
        pos[:T], on stream ``s``: K/V appended, ``attend(q, kc, vc, out)`` for the
        attention.  The projections' workspace is grown for ``n_head`` rows of
        the LM head too."""
        import torch
        c = self.cfg
        x, h, qkv, q, k, v = (b[:T] for b in (self.x, self.h, self.qkv, self.q, self.k, self.v))
        attn, gu, act = self.attn[:T], self.gu[:T], self.act[:T]
        need = max(gemm_workspace_bytes(T, qkv.shape[1], c.hidden),
                   gemm_workspace_bytes(T, c.hidden, c.hq * c.head_dim),
                   gemm_workspace_bytes(T, 2 * c.inter, c.hidden),
                   gemm_workspace_bytes(T, c.hidden, c.inter),
                   gemm_workspace_bytes(n_head, c.vocab, c.hidden)
                   if self.lm_head is not None else 0)
        if need > self.ws_gemm.numel():
            self.ws_gemm = torch.empty(need, dtype=torch.uint8, device=self.dev)
        for L, kc, vc in zip(self.layers, self.kc, self.vc):
            rmsnorm(x, L["in_norm"], h, c.eps, s)
            project_attn(h, L["qkv"], qkv, None, s, self.ws_gemm)
            qkv_rope(qkv, L["q_norm"], L["k_norm"], self.pos, c.hq, c.hkv, c.head_dim,
                     c.theta, c.eps, q, k, v, s)
            cp.kv_append(self.desc, k, v, kc, vc, self.bt, rows, self.ws_append, stream=s)
            attend(q, kc, vc, attn)
            project_attn(attn.view(T, c.hq * c.head_dim), L["o"], x, x, s, self.ws_gemm)
            rmsnorm(x, L["post_norm"], h, c.eps, s)
            project(h, L["gate_up"], gu, None, s, self.ws_gemm)
            swiglu(gu, act, s)
            project(act, L["down"], x, x, s, self.ws_gemm)

    def verify(self, rows, tokens, parents, max_path=16, stream=None):
        """One iteration over drafted trees: every row (slot, start, nodes, ctx)
        brings a tree of ``nodes`` guessed tokens, at most 256, node 0 the
        last token known (a decode row is a tree of one).  tokens (in [0, vocab))
        and parents: int32 device tensors [T], packed in row order, parents as
        indexes inside their row and -1 for node 0.

        The greedy token of every node is found, the path of drafted tokens that
        agrees with them accepted, and its K/V moved to the slots from ``start``
        on, in every layer: the row's next start is start + n_accepted, with
        next_token as its root.  Returns device int32 tensors (target [T], path
        [rows, max_path], n_accepted [rows], next_token [rows])."""
        import torch
        from . import tree
        c = self.cfg
        if self.lm_head is None:
            raise ValueError("verify needs a model with an LM head")
        rows = np.ascontiguousarray(np.asarray(rows, dtype=np.int32).reshape(-1, 4))
        T, R = int(rows[:, 2].sum()), len(rows)
        if T > self.max_tokens:
            raise ValueError(f"batch of {T} tokens exceeds the model's {self.max_tokens}")
        if (rows[:, 2] > tree.MAX_NODES).any() or not 1 <= max_path <= tree.MAX_NODES:
            raise ValueError(f"a tree has at most {tree.MAX_NODES} nodes, and so its path")
        for t in (tokens, parents):   # (index_select would resize its output to others)
            if (t.shape != (T,) or t.dtype != torch.int32 or t.device != self.x.device
                    or not t.is_contiguous()):
                raise cp.CpError(cp.CP_ERR_INVALID_ARG, "verify: tokens and parents are dense "
                                 f"int32 [{T}] on {self.x.device}")
        # (both check what they are given, before anything runs)
        need = tree.attn_workspace_bytes(self.desc, rows) if T > 0 else 0
        pools = tree.kv_layers(self.desc, self.kc, self.vc)
        s = stream or torch.cuda.current_stream(self.dev)
        with torch.cuda.stream(s):
            i32 = dict(dtype=torch.int32, device=self.dev)
            target, n_accepted, after = (torch.empty(n, **i32) for n in (T, R, R))
            path = torch.empty(R, max_path, **i32)
            logits = torch.empty(T, c.vocab, dtype=torch.bfloat16, device=self.dev)
            if T > 0:
                words = -(-int(rows[:, 2].max()) // 64)
                mask = torch.empty(T, words, dtype=torch.int64, device=self.dev)
                tree.layout(parents, rows, mask, self.pos[:T], s)
                if need > self.ws.numel():
                    self.ws = torch.empty(need, dtype=torch.uint8, device=self.dev)
                x, h = self.x[:T], self.h[:T]
                torch.index_select(self.embed, 0, tokens, out=x)
                self._layers(rows, T, T, s,
                             lambda q, kc, vc, out: tree.attn(self.desc, q, kc, vc, self.bt, mask,
                                                              rows, out, self.ws, s))
                rmsnorm(x, self.final_norm, h, c.eps, s)
                project(h, self.lm_head, logits, None, s, self.ws_gemm)
            tree.verify(logits, tokens, parents, rows, target, path, n_accepted, after, stream=s)
            if T > 0:
                tree.kv_compact(pools, self.bt, rows, path, n_accepted, s)
        return target, path, n_accepted, after


class ModelEngine:
    """StepEngine-compatible wrapper: one scheduler round = one model iteration."""

    def __init__(self, model: Model):
        import torch
        self.model = model
        self.max_tokens = model.max_tokens
        self.stream = torch.cuda.current_stream(model.dev)
        self.ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]

    def step(self, rows) -> float:
        rows = np.asarray(rows, dtype=np.int32).reshape(-1, 4)
        if int(rows[:, 2].sum()) == 0:
            return 0.0
        self.ev[0].record(self.stream)
        self.model.forward(rows, self.stream)
        self.ev[1].record(self.stream)
        self.ev[1].synchronize()
        return self.ev[0].elapsed_time(self.ev[1]) * 1e3
