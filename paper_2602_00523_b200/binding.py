"""Binding of libsage.so: argument marshalling only.

Every function below has the name of the C entry point it calls (include/sage.h),
takes torch CUDA tensors (PyTorch is used for device memory and streams, nothing
else), passes raw device pointers and sizes through the C ABI and returns the
output tensors.  Outputs and workspaces can be passed in (``out=`` dicts /
``ws=``) so that a caller can keep allocation out of its hot loop; what a call allocates
itself belongs to the stream that it goes to (``stream=``, else the current one).  The calls that
launch kernels are marshalled by the extension ``_native`` (csrc/binding.cpp), which
returns None when an output is still to be allocated.  ctypes (``lib()``) serves size
queries, settings and callers that bring raw pointers.  There is no CPU fallback: if
the shared library or the extension is missing, importing this module fails.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional

import torch

from .build import LIB_PATH, NATIVE_PATH

SAGE_OK = 0
SAGE_ERR_INVALID_ARG = 1
SAGE_ERR_UNSUPPORTED = 2
SAGE_ERR_WORKSPACE = 3
SAGE_ERR_CUDA = 4
SAGE_ERR_TOO_LARGE = 5
SAGE_STATIC_SCRATCH_BYTES = 1 << 20
SAGE_STATUS_BAD_TREE = 101
SAGE_STATUS_BAD_PAGE = 102
SAGE_STATUS_TIMEOUT = 103
SAGE_STATUS_BAD_PATH = 104
SAGE_MAX_NODES = 64
SAGE_MAX_TOPK = 16
SAGE_MAX_TEMPLATES = 8


class SagePolicy(ctypes.Structure):
    """Mirror of ``sage_tree_policy``."""
    _fields_ = [("n_templates", ctypes.c_int),
                ("alpha_thresholds", ctypes.c_float * SAGE_MAX_TEMPLATES),
                ("d_min", ctypes.c_float), ("d_max", ctypes.c_float),
                ("w_min", ctypes.c_float), ("w_max", ctypes.c_float)]


class SageHistoryPolicy(ctypes.Structure):
    """Mirror of ``sage_history_policy``."""
    _fields_ = [("window", ctypes.c_int), ("min_samples", ctypes.c_int),
                ("lower", ctypes.c_float), ("upper", ctypes.c_float), ("step", ctypes.c_float),
                ("d_lo", ctypes.c_float), ("d_hi", ctypes.c_float)]


class SageRopePolicy(ctypes.Structure):
    """Mirror of ``sage_rope_policy``."""
    _fields_ = [("inv_freq", ctypes.c_double * 64), ("axis", ctypes.c_uint8 * 64), ("scale", ctypes.c_float)]


class SageRopeRows(ctypes.Structure):
    """Mirror of ``sage_rope_rows``."""
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p)] + [
        (f"{t}_{d}_stride", ctypes.c_int64) for t in "qkv" for d in ("layer", "token")]


class SageSealedCache(ctypes.Structure):
    """Mirror of ``sage_sealed_cache``."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("layer_stride", ctypes.c_int64), ("k_exp", ctypes.c_void_p),
                ("v_exp", ctypes.c_void_p), ("n_pages", ctypes.c_int), ("page_table", ctypes.c_void_p),
                ("max_pages_per_seq", ctypes.c_int)]


class SageError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} (code {code})")


for _path in (LIB_PATH, NATIVE_PATH):
    if not os.path.exists(_path):
        raise ImportError(f"{_path} is missing: build it first (python -m paper_2602_00523_b200.build); "
                          "this package has no fallback path")

_lib = ctypes.CDLL(LIB_PATH)
from . import _native  # noqa: E402  (needs libsage.so and torch's libraries, loaded above)

_vp, _i, _i64, _f, _sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t

_lib.sage_expand_topk.restype = _i
_lib.sage_expand_topk.argtypes = [_vp, _i, _i, _i64, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp,
                                  _vp, _vp, _vp, _i, _vp, _vp, _vp, _sz, _vp, _vp]
_lib.sage_expand_topk_workspace_size.restype = _sz
_lib.sage_expand_topk_workspace_size.argtypes = [_i, _i]
_lib.sage_expand_topk_static.restype = _i
_lib.sage_expand_topk_static.argtypes = [_vp, _i, _i, _i64, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp,
                                         _vp, _vp, _vp, _i, _vp, _vp, _vp, _vp]
_lib.sage_select_tree.restype = _i
_lib.sage_select_tree.argtypes = [_vp, _vp, _i, ctypes.POINTER(SagePolicy), _vp, _vp, _vp,
                                  _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
_lib.sage_grow_tree.restype = _i
_lib.sage_grow_tree.argtypes = [_vp, _vp, _i, _vp, _vp, _i, ctypes.POINTER(SagePolicy), _i,
                                _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
_lib.sage_update_history.restype = _i
_lib.sage_update_history.argtypes = [_vp, _i, ctypes.POINTER(SageHistoryPolicy), _vp, _vp, _vp, _vp, _vp]
_lib.sage_build_ancestor_mask.restype = _i
_lib.sage_build_ancestor_mask.argtypes = [_vp, _vp, _i, _vp, _vp, _vp]
_lib.sage_tree_attention.restype = _i
_lib.sage_tree_attention.argtypes = [_vp, _vp, _vp, _i64, _i, _i, _vp, _i, _vp, _vp, _vp, _i, _i,
                                     _i, _i, _i, _i, _f, _vp, _vp, _sz, _vp, _vp]
_lib.sage_tree_attention_workspace_size.restype = _sz
_lib.sage_tree_attention_workspace_size.argtypes = [_i, _i, _i, _i, _i, _i, _i]
_lib.sage_accept.restype = _i
_lib.sage_accept.argtypes = [_vp, _vp, _vp, _vp, _i, _i, _vp, _vp, _vp, _vp, _vp]
_lib.sage_compact_kv.restype = _i
_lib.sage_compact_kv.argtypes = [_vp, _vp, _i64, _i, _i, _vp, _i, _vp, _vp, _vp, _i, _i, _i, _i, _i, _vp, _vp]
_lib.sage_rope_append.restype = _i
_lib.sage_rope_append.argtypes = [ctypes.POINTER(SageRopeRows), ctypes.POINTER(SageRopePolicy), _i, _i, _i, _i, _i, _vp, _vp, _vp,
                                  _vp, _vp, _vp, _i64, _i, _i, _vp, _i, _vp, _vp, _i, _vp, _vp]
_lib.sage_seal_kv.restype = _i
_lib.sage_seal_kv.argtypes = [_vp, _vp, _i64, _i, _i, _vp, _i, _vp, ctypes.POINTER(SageSealedCache), _vp, _i, _i, _i, _i, _vp, _vp]
_lib.sage_tree_attention_window.restype = _i
_lib.sage_tree_attention_window.argtypes = [_vp, _vp, _vp, _i64, _i, _i, _vp, _i, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _f, _i, _i,
                                            _vp, _vp, _sz, _vp, _vp]
_lib.sage_tree_attention_window_workspace_size.restype = _sz
_lib.sage_tree_attention_window_workspace_size.argtypes = [_i] * 9
_lib.sage_tree_attention_sealed.restype = _i
_lib.sage_tree_attention_sealed.argtypes = [_vp, _vp, _vp, _i64, _i, _i, _vp, _i, ctypes.POINTER(SageSealedCache), _vp, _vp, _vp, _vp,
                                            _i, _i, _i, _i, _i, _i, _f, _vp, _vp, _sz, _vp, _vp]
_lib.sage_tree_attention_sealed_workspace_size.restype = _sz
_lib.sage_tree_attention_sealed_workspace_size.argtypes = [_i] * 7
_lib.sage_debug_attention_waits.restype = None
_lib.sage_debug_attention_waits.argtypes = [ctypes.c_longlong, _i]
_lib.sage_debug_attention_schedule.restype = None
_lib.sage_debug_attention_schedule.argtypes = [_i]
_lib.sage_debug_attention_plan.restype = _i
_lib.sage_debug_attention_plan.argtypes = [_i, _i, _i, _i, _i, _i, ctypes.POINTER(_i)]
_lib.sage_status_string.restype = ctypes.c_char_p
_lib.sage_status_string.argtypes = [_i]


def lib() -> ctypes.CDLL:
    return _lib


def status_string(code: int) -> str:
    return _lib.sage_status_string(int(code)).decode()


def _check(code: int, where: str):
    if code != SAGE_OK:
        raise SageError(code, where)


def make_policy(thresholds, d_min=3.0, d_max=8.0, w_min=2.0, w_max=10.0) -> SagePolicy:
    p = SagePolicy()
    p.n_templates = len(thresholds) + 1
    for j, t in enumerate(thresholds):
        p.alpha_thresholds[j] = float(t)
    p.d_min, p.d_max, p.w_min, p.w_max = d_min, d_max, w_min, w_max
    return p


def new_status(device="cuda") -> torch.Tensor:
    return torch.zeros(1, dtype=torch.int32, device=device)


def sage_expand_topk_workspace_size(rows: int, vocab: int) -> int:
    return int(_lib.sage_expand_topk_workspace_size(rows, vocab))


def _made(make, stream) -> torch.Tensor:
    """What ``make`` allocates (and fills) for a call that goes to ``stream``: there and not on the current stream, whose later work
    may otherwise be given a workspace's bytes while the call still uses them, or fill an output behind the call.  The allocator
    holds it back, once it has been dropped, until what the current stream does with it has been done too."""
    if stream is None:
        return make()
    if not isinstance(stream, torch.cuda.Stream):
        # (0 is the default stream's handle, of which ExternalStream would make a new stream)
        stream = torch.cuda.ExternalStream(stream.cuda_stream) if stream.cuda_stream else torch.cuda.default_stream()
    with torch.cuda.stream(stream):
        t = make()
    if t.is_cuda:
        t.record_stream(torch.cuda.current_stream(t.device))
    return t


def _need(out: Dict[str, torch.Tensor], name: str, make, stream) -> None:
    if name not in out:
        out[name] = _made(make, stream)


def sage_expand_topk(logits: torch.Tensor, k: int, k_entropy: int, *, parent=None, rank=None,
                     node_offsets=None, root_token=None, out: Optional[Dict[str, torch.Tensor]] = None,
                     ws: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                     stream=None) -> Dict[str, torch.Tensor]:
    """logits fp32 [rows, vocab] (row stride = logits.stride(0)).  Returns a dict with
    topk_idx, topk_logprob, entropy_full, entropy_topk, alpha, lse and, when the tree
    arrays are given, draft_token."""
    o = {} if out is None else out
    code = _native.expand_topk(logits, k, k_entropy, parent, rank, node_offsets, root_token, o, ws, status, stream, False)
    if code is None:
        rows, vocab = logits.shape
        dev = logits.device
        _need(o, "topk_idx", lambda: torch.empty((rows, k), dtype=torch.int32, device=dev), stream)
        _need(o, "topk_logprob", lambda: torch.empty((rows, k), dtype=torch.float32, device=dev), stream)
        for name in ("entropy_full", "entropy_topk", "alpha", "lse"):
            _need(o, name, lambda: torch.empty(rows, dtype=torch.float32, device=dev), stream)
        if parent is not None:
            _need(o, "draft_token", lambda: torch.empty(parent.numel(), dtype=torch.int32, device=dev), stream)
        if ws is None:
            ws = _made(lambda: torch.empty(max(16, sage_expand_topk_workspace_size(rows, vocab)), dtype=torch.uint8, device=dev), stream)
        code = _native.expand_topk(logits, k, k_entropy, parent, rank, node_offsets, root_token, o, ws, status, stream, False)
    _check(code, "sage_expand_topk")
    return o


def sage_expand_topk_static(logits: torch.Tensor, k: int, k_entropy: int, *, parent=None, rank=None,
                            node_offsets=None, root_token=None, out: Dict[str, torch.Tensor],
                            status: Optional[torch.Tensor] = None, stream=None) -> Dict[str, torch.Tensor]:
    """sage_expand_topk without a workspace argument, for callers that cannot allocate device
    memory.  To honour that, this wrapper allocates nothing either -- every output tensor must
    already be in ``out`` (topk_idx, topk_logprob, entropy_full, entropy_topk, alpha, lse, and
    draft_token when the tree arrays are given).  Problems whose workspace would exceed
    SAGE_STATIC_SCRATCH_BYTES raise SageError(SAGE_ERR_TOO_LARGE)."""
    code = _native.expand_topk(logits, k, k_entropy, parent, rank, node_offsets, root_token, out, None, status, stream, True)
    if code is None:
        names = ["topk_idx", "topk_logprob", "entropy_full", "entropy_topk", "alpha", "lse"]
        raise KeyError(next((n for n in names if n not in out), "draft_token"))
    _check(code, "sage_expand_topk_static")
    return out


def sage_select_tree(alpha: torch.Tensor, policy: SagePolicy, *, alpha_row=None, batch: Optional[int] = None,
                     bank_parent=None, bank_rank=None, bank_n_nodes=None, handover: bool = False,
                     out: Optional[Dict[str, torch.Tensor]] = None, status=None, stream=None):
    """Returns template_id, depth_cont, width_cont (and next_parent / next_rank /
    next_node_offsets when ``handover``)."""
    o = {} if out is None else out
    code = _native.select_tree(alpha, alpha_row, batch, policy, o, bank_parent, bank_rank, bank_n_nodes, handover, status, stream)
    if code is None:
        dev = alpha.device
        n = batch if batch is not None else alpha_row.numel() if alpha_row is not None else alpha.numel()
        _need(o, "template_id", lambda: torch.empty(n, dtype=torch.int32, device=dev), stream)
        _need(o, "depth_cont", lambda: torch.empty(n, dtype=torch.float32, device=dev), stream)
        _need(o, "width_cont", lambda: torch.empty(n, dtype=torch.float32, device=dev), stream)
        if handover:
            _need(o, "next_parent", lambda: torch.full((n * SAGE_MAX_NODES,), -1, dtype=torch.int32, device=dev), stream)
            _need(o, "next_rank", lambda: torch.zeros(n * SAGE_MAX_NODES, dtype=torch.int32, device=dev), stream)
            _need(o, "next_node_offsets", lambda: torch.zeros(n + 1, dtype=torch.int32, device=dev), stream)
        code = _native.select_tree(alpha, alpha_row, batch, policy, o, bank_parent, bank_rank, bank_n_nodes, handover, status, stream)
    _check(code, "sage_select_tree")
    return o


def sage_grow_tree(topk_idx: torch.Tensor, topk_logprob: torch.Tensor, alpha: torch.Tensor, policy: SagePolicy,
                   tree: Dict[str, torch.Tensor], *, alpha_row=None, n_max: int = SAGE_MAX_NODES, d_max_seq=None,
                   status=None, stream=None) -> Dict[str, torch.Tensor]:
    """One level of dynamic tree construction, in place on ``tree`` (parent, rank, depth, token:
    int32 [batch * SAGE_MAX_NODES]; cum_logprob fp32 of the same length; n_nodes, frontier_begin:
    int32 [batch]).  topk_idx / topk_logprob: [batch * SAGE_MAX_NODES, k]."""
    code = _native.grow_tree(topk_idx, topk_logprob, alpha, policy, tree, alpha_row, n_max, d_max_seq, status, stream)
    if code is None:
        raise KeyError("tree needs parent, rank, depth, token, cum_logprob, n_nodes and frontier_begin")
    _check(code, "sage_grow_tree")
    return tree


def make_history_policy(window=10, min_samples=None, lower=2.0, upper=3.0, step=1.0, d_lo=3.0, d_hi=8.0):
    p = SageHistoryPolicy()
    p.window, p.min_samples = window, window if min_samples is None else min_samples
    p.lower, p.upper, p.step, p.d_lo, p.d_hi = lower, upper, step, d_lo, d_hi
    return p


def sage_update_history(path_len: torch.Tensor, policy: SageHistoryPolicy, window_buf: torch.Tensor,
                        count: torch.Tensor, d_max: torch.Tensor, *, status=None, stream=None):
    """In place: window_buf int32 [batch, window], count int32 [batch], d_max fp32 [batch]."""
    _check(_native.update_history(path_len, policy, window_buf, count, d_max, status, stream), "sage_update_history")
    return d_max


def sage_build_ancestor_mask(parent: torch.Tensor, node_offsets: torch.Tensor, *, out=None, status=None, stream=None):
    """Returns int64 [sum_nodes] holding the uint64 bitsets."""
    anc = out if out is not None else _made(lambda: torch.zeros(parent.numel(), dtype=torch.int64, device=parent.device), stream)
    _check(_native.build_ancestor_mask(parent, node_offsets, anc, status, stream), "sage_build_ancestor_mask")
    return anc


def sage_tree_attention_workspace_size(n_layers, batch, sum_nodes, n_q_heads, n_kv_heads, head_dim, max_pages) -> int:
    return int(_lib.sage_tree_attention_workspace_size(n_layers, batch, sum_nodes, n_q_heads, n_kv_heads,
                                                       head_dim, max_pages))


def sage_tree_attention(q: torch.Tensor, k_pool: torch.Tensor, v_pool: torch.Tensor, page_table: torch.Tensor,
                        seq_len: torch.Tensor, parent: torch.Tensor, node_offsets: torch.Tensor, sm_scale: float,
                        *, out=None, ws=None, status=None, stream=None) -> torch.Tensor:
    """q bf16 [layers, sum_nodes, Hq, d]; pools bf16 [layers, pages, Hkv, P, d];
    page_table int32 [B, max_pages].  Returns bf16 [layers, sum_nodes, Hq, d]."""
    if out is None:
        out = _made(lambda: torch.empty_like(q), stream)
    if ws is None:
        n_layers, sum_nodes, Hq, d = q.shape
        need = sage_tree_attention_workspace_size(n_layers, page_table.shape[0], sum_nodes, Hq, k_pool.shape[2], d,
                                                  page_table.shape[1])
        ws = _made(lambda: torch.empty(max(16, need), dtype=torch.uint8, device=q.device), stream)
    _check(_native.tree_attention(q, k_pool, v_pool, page_table, seq_len, parent, node_offsets, sm_scale, out, ws, status, stream),
           "sage_tree_attention")
    return out


def sage_tree_attention_window_workspace_size(n_layers, batch, sum_nodes, n_q_heads, n_kv_heads, head_dim, max_pages, window,
                                              sink) -> int:
    most = 2 ** 31 - 1
    return int(_lib.sage_tree_attention_window_workspace_size(n_layers, batch, sum_nodes, n_q_heads, n_kv_heads, head_dim, max_pages,
                                                              min(int(window), most), min(int(sink), most)))


def sage_tree_attention_window(q: torch.Tensor, k_pool: torch.Tensor, v_pool: torch.Tensor, page_table: torch.Tensor,
                               seq_len: torch.Tensor, parent: torch.Tensor, node_offsets: torch.Tensor, sm_scale: float,
                               window: int, sink: int = 0, *, out=None, ws=None, status=None, stream=None) -> torch.Tensor:
    """sage_tree_attention of rows that see the last ``window`` positions and the first ``sink`` ones only; shapes as there."""
    if out is None:
        out = _made(lambda: torch.empty_like(q), stream)
    if ws is None:
        n_layers, sum_nodes, Hq, d = q.shape
        need = sage_tree_attention_window_workspace_size(n_layers, page_table.shape[0], sum_nodes, Hq, k_pool.shape[2], d,
                                                         page_table.shape[1], window, sink)
        ws = _made(lambda: torch.empty(max(16, need), dtype=torch.uint8, device=q.device), stream)
    _check(_native.tree_attention_window(q, k_pool, v_pool, page_table, seq_len, parent, node_offsets, sm_scale, window, sink, out, ws,
                                         status, stream), "sage_tree_attention_window")
    return out


def make_rope_policy(base: float = 10000.0, sections=(64, 0, 0), *, interleaved: bool = False, scale: float = 1.0,
                     inv_freq=None) -> SageRopePolicy:
    """Frequencies base ** (-i / 64), i < 64 (or 64 given ones), and the axis of each: ``sections`` frequencies for time, height
    and width one after the other, or, ``interleaved``, in turn (time, height, width, time, ...) as long as an axis has some
    left.  The default is the ordinary one-axis rotation; ``scale`` multiplies the turned rows."""
    sections = [int(n) for n in sections]
    if len(sections) != 3 or min(sections) < 0 or sum(sections) != 64:
        raise ValueError("sections: three counts that sum to 64")
    if interleaved:
        left, axis = list(sections), []
        while len(axis) < 64:
            for a in range(3):
                if left[a]:
                    left[a] -= 1
                    axis.append(a)
    else:
        axis = [a for a, n in enumerate(sections) for _ in range(n)]
    freq = [float(base) ** (-i / 64.0) for i in range(64)] if inv_freq is None else [float(f) for f in inv_freq]
    if len(freq) != 64:
        raise ValueError("inv_freq: 64 values")
    p = SageRopePolicy()
    for i in range(64):
        p.inv_freq[i], p.axis[i] = freq[i], axis[i]
    p.scale = float(scale)
    return p


def sage_rope_append(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, policy: SageRopePolicy, k_pool: torch.Tensor,
                     v_pool: torch.Tensor, page_table: torch.Tensor, seq_len: torch.Tensor, node_offsets: torch.Tensor, *, pos=None,
                     parent=None, next_pos=None, out=None, status=None, stream=None) -> torch.Tensor:
    """q bf16 [layers, tokens, Hq, d], k and v [layers, tokens, Hkv, d]: the heads of a token side by side, tokens and layers at
    any distance (parts of a fused projection's rows).  Returns the turned queries (``out``, contiguous) and writes turned keys, and
    values, behind each sequence's prefix into the pools.  Positions: ``pos`` int32 [3, tokens], or ``parent`` and ``next_pos`` [B]."""
    if out is None:
        out = _made(lambda: torch.empty(q.shape, dtype=q.dtype, device=q.device), stream)
    _check(_native.rope_append(q, k, v, policy, k_pool, v_pool, page_table, seq_len, node_offsets, pos, parent, next_pos, out, status,
                               stream), "sage_rope_append")
    return out


def new_sealed_cache(n_layers: int, n_pages: int, n_kv_heads: int, page_table: torch.Tensor, *, page_size: int = 64,
                     head_dim: int = 128) -> Dict[str, torch.Tensor]:
    """An empty 8-bit cache for pages that are full: k, v (e4m3 [layers, pages, Hkv, P, d]), k_exp, v_exp (bytes [layers, pages,
    Hkv]) and the page table (int32 [B, max_pages], ids of these pools) that it goes by."""
    dev = page_table.device
    shape = (n_layers, n_pages, n_kv_heads)
    cache = {"page_table": page_table}
    for name in ("k", "v"):
        cache[name] = torch.zeros(shape + (page_size, head_dim), dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)
        cache[name + "_exp"] = torch.full(shape, 127, dtype=torch.uint8, device=dev)
    return cache


def _sealed(code, where: str):
    if code is None:
        raise KeyError("cache needs k, v, k_exp, v_exp and page_table")
    _check(code, where)


def sage_seal_kv(k_pool: torch.Tensor, v_pool: torch.Tensor, page_table: torch.Tensor, seq_len: torch.Tensor, sealed: torch.Tensor,
                 cache: Dict[str, torch.Tensor], *, status=None, stream=None) -> Dict[str, torch.Tensor]:
    """Full pages of the prefix that are not sealed yet move into ``cache`` (see new_sealed_cache); ``sealed`` int32 [B], in
    place: the number of each sequence's first pages that are held there."""
    _sealed(_native.seal_kv(k_pool, v_pool, page_table, seq_len, sealed, cache, status, stream), "sage_seal_kv")
    return cache


def sage_tree_attention_sealed_workspace_size(n_layers, batch, sum_nodes, n_q_heads, n_kv_heads, head_dim, max_pages) -> int:
    return int(_lib.sage_tree_attention_sealed_workspace_size(n_layers, batch, sum_nodes, n_q_heads, n_kv_heads, head_dim, max_pages))


def sage_tree_attention_sealed(q: torch.Tensor, k_pool: torch.Tensor, v_pool: torch.Tensor, page_table: torch.Tensor,
                               cache: Dict[str, torch.Tensor], sealed: torch.Tensor, seq_len: torch.Tensor, parent: torch.Tensor,
                               node_offsets: torch.Tensor, sm_scale: float, *, out=None, ws=None, status=None,
                               stream=None) -> torch.Tensor:
    """sage_tree_attention over a cache whose first ``sealed[b]`` pages lie in ``cache`` and whose others, with the tree's rows, lie
    in the bf16 pools; shapes as there."""
    if out is None:
        out = _made(lambda: torch.empty_like(q), stream)
    if ws is None:
        n_layers, sum_nodes, Hq, d = q.shape
        need = sage_tree_attention_sealed_workspace_size(n_layers, page_table.shape[0], sum_nodes, Hq, k_pool.shape[2], d,
                                                         page_table.shape[1])
        ws = _made(lambda: torch.empty(max(16, need), dtype=torch.uint8, device=q.device), stream)
    _sealed(_native.tree_attention_sealed(q, k_pool, v_pool, page_table, cache, sealed, seq_len, parent, node_offsets, sm_scale, out, ws,
                                          status, stream), "sage_tree_attention_sealed")
    return out


def sage_debug_attention_waits(wait_cycles: int = 0, producer_off: bool = False) -> None:
    """Cycle budget of the attention kernel's on-device waits (0 = default) and, for tests of the
    time-out path, a switch that keeps its copy warp from issuing anything."""
    _lib.sage_debug_attention_waits(int(wait_cycles), 1 if producer_off else 0)


def sage_debug_attention_schedule(schedule: int = 0) -> None:
    """0: the library picks the attention schedule per launch; 1: streaming; 2: split."""
    _lib.sage_debug_attention_schedule(int(schedule))


def sage_debug_attention_plan(n_layers, batch, sum_nodes, n_q_heads, n_kv_heads, max_pages) -> dict:
    """What sage_tree_attention would do with a launch of these sizes: the schedule, 1 streaming or 2 split, the split one's
    context slices, and whether their merge is brought up while they are still being worked on."""
    plan = (_i * 3)()
    _check(_lib.sage_debug_attention_plan(n_layers, batch, sum_nodes, n_q_heads, n_kv_heads, max_pages, plan), "sage_debug_attention_plan")
    return {"schedule": plan[0], "slices": plan[1], "merge_overlaps": bool(plan[2])}


def sage_accept(parent, draft_token, target_argmax, node_offsets, max_path: int, *, out=None, status=None, stream=None):
    o = {} if out is None else out
    code = _native.accept(parent, draft_token, target_argmax, node_offsets, max_path, o, status, stream)
    if code is None:
        batch, dev = node_offsets.numel() - 1, parent.device
        _need(o, "path", lambda: torch.empty((batch, max_path), dtype=torch.int32, device=dev), stream)
        _need(o, "path_len", lambda: torch.empty(batch, dtype=torch.int32, device=dev), stream)
        _need(o, "bonus_token", lambda: torch.empty(batch, dtype=torch.int32, device=dev), stream)
        code = _native.accept(parent, draft_token, target_argmax, node_offsets, max_path, o, status, stream)
    _check(code, "sage_accept")
    return o


def sage_compact_kv(k_pool, v_pool, page_table, seq_len, path, path_len, *, status=None, stream=None):
    """In place on k_pool, v_pool ([layers, pages, Hkv, P, d] bf16) and seq_len."""
    _check(_native.compact_kv(k_pool, v_pool, page_table, seq_len, path, path_len, status, stream), "sage_compact_kv")
