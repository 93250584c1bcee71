"""ctypes binding of libpps (include/pps.h): same entry-point names, argument
marshalling only.  Torch supplies device memory and the current stream; every
step of the computation runs in the library's CUDA kernels.  There is no CPU
fallback: a missing or unloadable libpps.so raises immediately.
"""
from __future__ import annotations

import contextlib
import ctypes
import importlib.util
import os
import struct
import threading

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))


def library_path(rounds: int = 10) -> str:
    """The build of libpps whose keyed source is Philox4x32 with `rounds` rounds: 10
    (libpps.so, the default) or 7 (libpps_r7.so)."""
    if rounds not in (7, 10):
        raise ValueError("libpps is built for Philox4x32-10 and Philox4x32-7 only")
    return os.path.join(_HERE, "_lib", "libpps.so" if rounds == 10 else "libpps_r7.so")


# PPS_PHILOX_ROUNDS=7 in the environment selects the Philox4x32-7 build at import
LIB_PATH = library_path(int(os.environ.get("PPS_PHILOX_ROUNDS", "10")))

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA, ERR_SIZE = 0, 1, 2, 3, 4, 5
NOALLOC_MAX_ROWS = 4096  # PPS_NOALLOC_MAX_ROWS of include/pps.h (tests/test_abi.py checks the two agree)
F32, BF16, F16 = 0, 1, 2
DISTINCT, IID = 0, 1
FLAG_GUARD, FLAG_LOGIT_RANGE, FLAG_TREE, FLAG_TIMEOUT, FLAG_INDEX = 1, 2, 4, 8, 16
MAX_K = 32
MAX_TOP_K = 64
MAX_BLOCKS = 32
LMHEAD_MAX_K = 8

_lock = threading.Lock()
_lib = None
_fast = None  # pps_torch, bound to the loaded library


class RowIds(ctypes.Structure):
    _fields_ = [("key", ctypes.c_void_p), ("ctx_hash", ctypes.c_void_p), ("pos", ctypes.c_void_p)]


class PPSError(RuntimeError):
    def __init__(self, fn, code):
        super().__init__(f"{fn} failed: {code} ({status_string(code)})")
        self.code = code


def use_library(rounds: int = 10):
    """Switch the binding to the build for Philox4x32-`rounds` (the next call loads it).
    Device memory (workspaces, outputs) carries over; results follow the new keyed source."""
    global _lib, _fast, LIB_PATH
    with _lock:
        LIB_PATH = library_path(rounds)
        _lib = _fast = None


def philox_rounds() -> int:
    """Rounds of the keyed source of the loaded library (pps_philox_rounds)."""
    return int(lib().pps_philox_rounds())


def lib():
    """Load libpps.so (raises if it was not built)."""
    global _lib
    loaded = _lib
    if loaded is not None:
        return loaded
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise RuntimeError(f"libpps.so not found at {LIB_PATH}; build it with "
                                   "`python -c 'import __graft_entry__ as g; g.build()'`")
            L = ctypes.CDLL(LIB_PATH)
            vp, i64, i32, f32, u64, sz = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float,
                                          ctypes.c_uint64, ctypes.c_size_t)
            L.pps_version.restype = ctypes.c_char_p
            L.pps_philox_rounds.argtypes = []
            L.pps_philox_rounds.restype = ctypes.c_int
            L.pps_status_string.argtypes = [ctypes.c_int]
            L.pps_status_string.restype = ctypes.c_char_p
            L.pps_workspace_size.argtypes = [i64, i64, i32, i32]
            L.pps_workspace_size.restype = sz
            L.pps_workspace_clear.argtypes = [vp, sz, vp]
            L.pps_workspace_clear.restype = ctypes.c_int
            L.pps_draft_list.argtypes = [vp, ctypes.c_int, i64, i64, i64, RowIds, f32, i32, vp, ctypes.c_int,
                                         vp, vp, vp, vp, vp, vp, vp, sz, vp]
            L.pps_draft_list.restype = ctypes.c_int
            L.pps_verify_tree.argtypes = [vp, ctypes.c_int, i64, i64, i64, RowIds, f32, i32, i32, vp, vp, i64, vp,
                                          vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
            L.pps_verify_tree.restype = ctypes.c_int
            L.pps_draft_list_trunc.argtypes = [vp, ctypes.c_int, i64, i64, i64, RowIds, f32, i32, f32, i32, vp,
                                               ctypes.c_int, vp, vp, vp, vp, vp, vp, vp, sz, vp]
            L.pps_draft_list_trunc.restype = ctypes.c_int
            L.pps_verify_tree_trunc.argtypes = [vp, ctypes.c_int, i64, i64, i64, RowIds, f32, i32, f32, i32, i32, vp,
                                                vp, i64, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
            L.pps_verify_tree_trunc.restype = ctypes.c_int
            L.pps_draft_list_noalloc.argtypes = [vp, ctypes.c_int, i64, i64, i64, RowIds, f32, i32, vp, ctypes.c_int,
                                                 vp, vp, vp, vp, vp, vp, vp]
            L.pps_draft_list_noalloc.restype = ctypes.c_int
            L.pps_wm_score.argtypes = [vp, RowIds, i64, i32, vp, vp, vp, vp]
            L.pps_tree_expand.argtypes = [i32, i32, i32, i32, vp, vp, vp, RowIds, vp, vp, vp, vp, vp, vp, vp, vp,
                                          vp, vp]
            L.pps_tree_expand.restype = ctypes.c_int
            L.pps_wm_detect.argtypes = [vp, RowIds, i64, i32, vp, ctypes.c_int, ctypes.c_double, vp, vp, vp, vp]
            L.pps_wm_detect.restype = ctypes.c_int
            L.pps_wm_score.restype = ctypes.c_int
            L.pps_draft_hetero.argtypes = [vp, ctypes.c_int, i64, i64, i64, RowIds, f32, vp, i32, vp, vp, vp, vp,
                                           sz, vp]
            L.pps_draft_hetero.restype = ctypes.c_int
            L.pps_draft_hetero_trunc.argtypes = [vp, ctypes.c_int, i64, i64, i64, RowIds, f32, i32, f32, vp, i32, vp,
                                                 vp, vp, vp, sz, vp]
            L.pps_draft_hetero_trunc.restype = ctypes.c_int
            L.pps_hetero_expand.argtypes = [i32, i32, i32, i32, vp, RowIds, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                            vp, vp]
            L.pps_hetero_expand.restype = ctypes.c_int
            L.pps_hetero_block.argtypes = [vp, RowIds, i64, i32, vp, vp]
            L.pps_hetero_block.restype = ctypes.c_int
            L.pps_lmhead_workspace_size.argtypes = [i64, i32]
            L.pps_lmhead_workspace_size.restype = sz
            L.pps_lmhead_logits.argtypes = [vp, i64, vp, i64, i64, i64, i64, vp, i64, vp]
            L.pps_lmhead_logits.restype = ctypes.c_int
            L.pps_lmhead_draft_list.argtypes = [vp, i64, vp, i64, i64, i64, i64, RowIds, f32, i32, vp, ctypes.c_int,
                                                vp, vp, vp, vp, vp, vp, vp, sz, vp]
            L.pps_lmhead_draft_list.restype = ctypes.c_int
            L.pps_lmhead_verify_tree.argtypes = [vp, i64, vp, i64, i64, i64, i64, RowIds, f32, i32, i32, vp, vp, i64,
                                                 vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
            L.pps_lmhead_verify_tree.restype = ctypes.c_int
            for fn in (L.pps_kv_append, L.pps_paged_attention, L.pps_verify_chain):
                fn.argtypes, fn.restype = [ctypes.c_char_p, vp], ctypes.c_int
            L.pps_attention_workspace_size.argtypes = [i64, i32, i32, i32]
            L.pps_attention_workspace_size.restype = sz
            L.pps_chain_workspace_size.argtypes = [i64, i64, i32]
            L.pps_chain_workspace_size.restype = sz
            L.pps_philox_words.argtypes = [RowIds, i64, i64, i32, vp, vp]
            L.pps_philox_words.restype = ctypes.c_int
            L.pps_selftest_philox_rate.argtypes = [u64, vp, i32, vp]
            L.pps_selftest_philox_rate.restype = ctypes.c_int
            L.pps_selftest_lg2_error.argtypes = [f32, f32, vp, vp]
            L.pps_selftest_lg2_error.restype = ctypes.c_int
            L.pps_selftest_key_error.argtypes = [u64, u64, vp, vp]
            L.pps_selftest_key_error.restype = ctypes.c_int
            _lib = L
    return _lib


def version() -> str:
    return lib().pps_version().decode()


def status_string(code: int) -> str:
    return lib().pps_status_string(int(code)).decode()


def _check(fn, code):
    if code != OK:
        raise PPSError(fn, code)


# Host cost of a call.  A step of few rows runs two launches of about 20 us, and its two calls took
# 47 us of Python (tensor checks 14, stream object 4, device guard 3, ids 4, pointer objects 6), so
# the binding keeps every check but makes the common outcome cheap: one expression per tensor, raw
# pointers and stream handles instead of wrapper objects, and a device switch only when it is needed.

def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream, dev=None):
    """The stream's handle; with no stream, the current stream of `dev` (the tensors' device)."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if dev is None else dev.index)
    if dev is not None and stream.device != dev:
        raise ValueError(f"stream is on {stream.device}, the tensors on {dev}")
    return stream.cuda_stream


_HERE_ALREADY = contextlib.nullcontext()


def _on(dev):
    """A context in which `dev` is the current device."""
    return _HERE_ALREADY if torch.cuda.current_device() == dev.index else torch.cuda.device(dev)


def _need(name, t, dev, dtype, numel=0, contiguous=True):
    """Raise unless tensor `t` (skipped when None) is on `dev` with `dtype` and holds at least
    `numel` elements: the library writes and reads through plain pointers, so a short or
    misplaced buffer must be refused here, before anything is launched."""
    if t is None or (isinstance(t, torch.Tensor) and t.is_cuda and t.get_device() == dev.index and t.dtype is dtype
                     and t.numel() >= numel and (not contiguous or t.is_contiguous())):
        return
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.device != dev:
        raise TypeError(f"{name} must be a CUDA tensor on {dev}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if contiguous and not t.is_contiguous():
        raise TypeError(f"{name} must be contiguous")
    if t.numel() < numel:
        raise ValueError(f"{name} holds {t.numel()} elements; the call needs {numel}")


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise TypeError(f"logits must be bfloat16 or float32, got {t.dtype}")


def _ids(key, ctx, pos, n=0, dev=None):
    """Row ids (bit patterns of the unsigned key, context label and position), n of each."""
    for name, t, dt in (("key", key, torch.int64), ("ctx", ctx, torch.int64), ("pos", pos, torch.int32)):
        if not t.is_cuda or t.dtype is not dt or not t.is_contiguous():
            raise TypeError(f"{name} must be a contiguous CUDA {dt} tensor (bit pattern of the unsigned id)")
        if (dev is not None and t.get_device() != dev.index) or t.numel() < n:
            _need(name, t, dev if dev is not None else t.device, dt, n)
    return RowIds(key.data_ptr(), ctx.data_ptr(), pos.data_ptr())


def _need_out(out: dict, spec, dev):
    for name, dt, numel in spec:
        _need(name, out.get(name), dev, dt, numel)


def _rows(logits):
    if not logits.is_cuda or logits.dim() != 2 or logits.stride(1) != 1:
        raise TypeError("logits must be a 2-D CUDA tensor with unit stride along the vocabulary")
    return logits.shape[0], logits.shape[1], logits.stride(0)


def workspace_size(n_rows: int, vocab: int = 0, K: int = 1, n_seq: int = 0) -> int:
    return int(lib().pps_workspace_size(n_rows, vocab, K, n_seq))


def workspace(n_rows: int, n_seq: int = 0, device=None) -> torch.Tensor:
    """A zeroed workspace (reusable across calls of the same or smaller size)."""
    nb = workspace_size(n_rows, 0, 1, n_seq)
    return torch.zeros(nb, dtype=torch.uint8, device=device or "cuda")


def workspace_clear(ws: torch.Tensor, stream=None):
    _need("ws", ws, ws.device, torch.uint8)
    with _on(ws.device):
        _check("pps_workspace_clear", lib().pps_workspace_clear(_ptr(ws), ws.numel(), _stream(stream, ws.device)))


def _need_draft(out, n, K, row_k, status, dev):
    _need_out(out, [("tok", torch.int32, n * K), ("key", torch.float32, n * K), ("mult", torch.int32, n * K),
                    ("ndist", torch.int32, n), ("samples", torch.int32, n * K)], dev)
    for name in ("tok", "mult", "ndist"):
        if out.get(name) is None:
            raise TypeError(f"out[{name!r}] is required")
    _need("row_k", row_k, dev, torch.int32, n)
    _need("status", status, dev, torch.int32, 1)


def draft_list(q_logits, key, ctx, pos, K: int, row_k=None, mode: int = DISTINCT, temperature: float = 1.0,
               ws=None, status=None, out=None, keys: bool = True, samples: bool = True, stream=None,
               top_k: int = 0, top_p: float = 1.0):
    """pps_draft_list (pps_draft_list_trunc when top_k > 0).  Returns dict(tok, key, mult, ndist, samples)."""
    n, V, stride = _rows(q_logits)
    dev = q_logits.device
    if out is None:
        out = dict(tok=torch.empty(n, K, dtype=torch.int32, device=dev),
                   key=torch.empty(n, K, dtype=torch.float32, device=dev) if keys else None,
                   mult=torch.empty(n, K, dtype=torch.int32, device=dev),
                   ndist=torch.empty(n, dtype=torch.int32, device=dev),
                   samples=torch.empty(n, K, dtype=torch.int32, device=dev) if samples else None)
    if ws is None:
        ws = workspace(n, 0, dev)
    _need_draft(out, n, K, row_k, status, dev)
    _need("ws", ws, dev, torch.uint8)
    ids = _ids(key, ctx, pos, n, dev)
    with _on(dev):
        if top_k > 0:
            code = lib().pps_draft_list_trunc(_ptr(q_logits), _dtype_code(q_logits), n, V, stride, ids,
                                              float(temperature), int(top_k), float(top_p), int(K), _ptr(row_k),
                                              int(mode), _ptr(out["tok"]), _ptr(out.get("key")), _ptr(out["mult"]),
                                              _ptr(out["ndist"]), _ptr(out.get("samples")), _ptr(status), _ptr(ws),
                                              ws.numel(), _stream(stream, dev))
            _check("pps_draft_list_trunc", code)
            return out
        code = lib().pps_draft_list(_ptr(q_logits), _dtype_code(q_logits), n, V, stride, ids, float(temperature),
                                    int(K), _ptr(row_k), int(mode), _ptr(out["tok"]), _ptr(out.get("key")),
                                    _ptr(out["mult"]), _ptr(out["ndist"]), _ptr(out.get("samples")), _ptr(status),
                                    _ptr(ws), ws.numel(), _stream(stream, dev))
    _check("pps_draft_list", code)
    return out


def draft_list_noalloc(q_logits, key, ctx, pos, K: int, row_k=None, mode: int = DISTINCT, temperature: float = 1.0,
                       status=None, out=None, keys: bool = True, samples: bool = True, stream=None):
    """pps_draft_list_noalloc: pps_draft_list without a workspace, for callers
    that cannot allocate device memory per call (the library's built-in
    scratch serves up to NOALLOC_MAX_ROWS rows; calls must not overlap on the GPU)."""
    n, V, stride = _rows(q_logits)
    dev = q_logits.device
    if out is None:
        out = dict(tok=torch.empty(n, K, dtype=torch.int32, device=dev),
                   key=torch.empty(n, K, dtype=torch.float32, device=dev) if keys else None,
                   mult=torch.empty(n, K, dtype=torch.int32, device=dev),
                   ndist=torch.empty(n, dtype=torch.int32, device=dev),
                   samples=torch.empty(n, K, dtype=torch.int32, device=dev) if samples else None)
    _need_draft(out, n, K, row_k, status, dev)
    ids = _ids(key, ctx, pos, n, dev)
    with _on(dev):
        code = lib().pps_draft_list_noalloc(_ptr(q_logits), _dtype_code(q_logits), n, V, stride, ids,
                                            float(temperature), int(K), _ptr(row_k), int(mode), _ptr(out["tok"]),
                                            _ptr(out.get("key")), _ptr(out["mult"]), _ptr(out["ndist"]),
                                            _ptr(out.get("samples")), _ptr(status), _stream(stream, dev))
    _check("pps_draft_list_noalloc", code)
    return out


def verify_tree(p_logits, key, ctx, pos, gamma: int, seq_off, node_draft_row, draft_tok, draft_ndist, child_node,
                temperature: float = 1.0, ws=None, status=None, out=None, stream=None, top_k: int = 0,
                top_p: float = 1.0):
    """pps_verify_tree (pps_verify_tree_trunc when top_k > 0).
    Returns dict(winner, word, accept_len, n_emitted, emitted, score, score_sum)."""
    n, V, stride = _rows(p_logits)
    dev = p_logits.device
    n_seq = seq_off.numel() - 1
    K = draft_tok.shape[1]
    W = gamma + 1
    if out is None:
        out = dict(winner=torch.empty(n, dtype=torch.int32, device=dev),
                   word=torch.empty(n, dtype=torch.int32, device=dev),
                   accept_len=torch.empty(n_seq, dtype=torch.int32, device=dev),
                   n_emitted=torch.empty(n_seq, dtype=torch.int32, device=dev),
                   emitted=torch.empty(n_seq, W, dtype=torch.int32, device=dev),
                   score=torch.empty(n_seq, W, dtype=torch.float32, device=dev),
                   score_sum=torch.empty(n_seq, dtype=torch.float64, device=dev))
    if ws is None:
        ws = workspace(n, n_seq, dev)
    n_draft = draft_tok.shape[0]
    for name, t, numel in (("seq_off", seq_off, n_seq + 1), ("node_draft_row", node_draft_row, n),
                           ("draft_tok", draft_tok, n_draft * K), ("draft_ndist", draft_ndist, n_draft),
                           ("child_node", child_node, n_draft * K)):
        _need(name, t, dev, torch.int32, numel)
    _need_out(out, [("winner", torch.int32, n), ("word", torch.int32, n), ("accept_len", torch.int32, n_seq),
                    ("n_emitted", torch.int32, n_seq), ("emitted", torch.int32, n_seq * W),
                    ("score", torch.float32, n_seq * W), ("score_sum", torch.float64, n_seq)], dev)
    _need("status", status, dev, torch.int32, 1)
    _need("ws", ws, dev, torch.uint8)
    ids = _ids(key, ctx, pos, n, dev)
    with _on(dev):
        if top_k > 0:
            code = lib().pps_verify_tree_trunc(_ptr(p_logits), _dtype_code(p_logits), n, V, stride, ids,
                                               float(temperature), int(top_k), float(top_p), n_seq, int(gamma),
                                               _ptr(seq_off), _ptr(node_draft_row), n_draft, _ptr(draft_tok),
                                               _ptr(draft_ndist), int(K), _ptr(child_node), _ptr(out["winner"]),
                                               _ptr(out["word"]), _ptr(out["accept_len"]), _ptr(out["n_emitted"]),
                                               _ptr(out["emitted"]), _ptr(out["score"]), _ptr(out["score_sum"]),
                                               _ptr(status), _ptr(ws), ws.numel(), _stream(stream, dev))
            _check("pps_verify_tree_trunc", code)
            return out
        code = lib().pps_verify_tree(_ptr(p_logits), _dtype_code(p_logits), n, V, stride, ids, float(temperature),
                                     n_seq, int(gamma), _ptr(seq_off), _ptr(node_draft_row), n_draft,
                                     _ptr(draft_tok), _ptr(draft_ndist), int(K), _ptr(child_node),
                                     _ptr(out["winner"]), _ptr(out["word"]), _ptr(out["accept_len"]),
                                     _ptr(out["n_emitted"]), _ptr(out["emitted"]), _ptr(out["score"]),
                                     _ptr(out["score_sum"]), _ptr(status), _ptr(ws), ws.numel(),
                                     _stream(stream, dev))
    _check("pps_verify_tree", code)
    return out


def _need_detector(tokens, seg_off, n, n_seg, dev):
    if not isinstance(tokens, torch.Tensor) or tokens.dtype != torch.int32 or not tokens.is_cuda:
        raise TypeError("tokens must be a CUDA int32 tensor")
    _need("tokens", tokens, dev, torch.int32, n)
    if seg_off is not None and (seg_off.dtype != torch.int64 or not seg_off.is_cuda):
        raise TypeError("seg_off must be a CUDA int64 tensor")
    _need("seg_off", seg_off, dev, torch.int64, n_seg + 1)


def wm_score(tokens, key, ctx, pos, seg_off=None, out_score=None, out_sum=None, want_scores=True, stream=None):
    """pps_wm_score.  Returns (scores or None, sums)."""
    n = tokens.numel()
    dev = tokens.device
    n_seg = seg_off.numel() - 1 if seg_off is not None else 1
    if out_score is None and want_scores:
        out_score = torch.empty(n, dtype=torch.float32, device=dev)
    if out_sum is None:
        out_sum = torch.empty(n_seg, dtype=torch.float64, device=dev)
    _need_detector(tokens, seg_off, n, n_seg, dev)
    _need("out_score", out_score, dev, torch.float32, n)
    _need("out_sum", out_sum, dev, torch.float64, n_seg)
    ids = _ids(key, ctx, pos, n, dev)
    with _on(dev):
        code = lib().pps_wm_score(_ptr(tokens), ids, n, n_seg, _ptr(seg_off), _ptr(out_score), _ptr(out_sum),
                                  _stream(stream, dev))
    _check("pps_wm_score", code)
    return out_score, out_sum


def tree_expand(K: int, gamma: int, depth: int, draft, rows_key, rows_ctx, rows_pos, row_k, nxt: dict, child_node,
                nodes: dict, stream=None):
    """pps_tree_expand: children of depth `depth`'s rows (dynamic IID tree).  `draft` = the
    pps_draft_list (IID) outputs of those rows; writes nxt = dict(key, ctx, pos, k) of the next
    depth's rows, child_node and nodes = dict(key, ctx, pos) in place."""
    n_seq = nxt["k"].numel() // K
    dev = nxt["k"].device
    ids = _ids(rows_key, rows_ctx, rows_pos, 0, dev)
    with _on(dev):
        code = lib().pps_tree_expand(n_seq, int(K), int(gamma), int(depth), _ptr(draft["tok"]), _ptr(draft["mult"]),
                                     _ptr(draft["ndist"]), ids, _ptr(row_k), _ptr(nxt["key"]), _ptr(nxt["ctx"]),
                                     _ptr(nxt["pos"]), _ptr(nxt["k"]), _ptr(child_node), _ptr(nodes["key"]),
                                     _ptr(nodes["ctx"]), _ptr(nodes["pos"]), _stream(stream, dev))
    _check("pps_tree_expand", code)


def draft_hetero(q_logits, key, ctx, pos, row_block, n_blocks: int, temperature: float = 1.0, ws=None, status=None,
                 out_tok=None, out_key=None, stream=None, top_k: int = 0, top_p: float = 1.0):
    """pps_draft_hetero (pps_draft_hetero_trunc when top_k > 0): proposal row_block[r] of
    n_blocks at each row (non-identical proposals on the augmented source).  Returns the
    [n_rows] int32 tokens."""
    n, V, stride = _rows(q_logits)
    dev = q_logits.device
    if out_tok is None:
        out_tok = torch.empty(n, dtype=torch.int32, device=dev)
    if ws is None:
        ws = workspace(n, 0, dev)
    if row_block.dtype != torch.int32 or not row_block.is_cuda or not row_block.is_contiguous():
        raise TypeError("row_block must be a contiguous CUDA int32 tensor")
    _need("row_block", row_block, dev, torch.int32, n)
    _need("out_tok", out_tok, dev, torch.int32, n)
    _need("out_key", out_key, dev, torch.float32, n)
    _need("status", status, dev, torch.int32, 1)
    _need("ws", ws, dev, torch.uint8)
    ids = _ids(key, ctx, pos, n, dev)
    with _on(dev):
        if top_k > 0:
            code = lib().pps_draft_hetero_trunc(_ptr(q_logits), _dtype_code(q_logits), n, V, stride, ids,
                                                float(temperature), int(top_k), float(top_p), _ptr(row_block),
                                                int(n_blocks), _ptr(out_tok), _ptr(out_key), _ptr(status), _ptr(ws),
                                                ws.numel(), _stream(stream, dev))
            _check("pps_draft_hetero_trunc", code)
            return out_tok
        code = lib().pps_draft_hetero(_ptr(q_logits), _dtype_code(q_logits), n, V, stride, ids, float(temperature),
                                      _ptr(row_block), int(n_blocks), _ptr(out_tok), _ptr(out_key), _ptr(status),
                                      _ptr(ws), ws.numel(), _stream(stream, dev))
    _check("pps_draft_hetero", code)
    return out_tok


def hetero_expand(n_blocks: int, gamma: int, depth: int, draft_tok, rows_key, rows_ctx, rows_pos, row_owner,
                  nxt, lists: dict, nodes: dict, stream=None):
    """pps_hetero_expand: depth `depth` of the tree of n_blocks proposals.  Writes
    lists = dict(tok, ndist, child) of the depth's nodes, nodes = dict(key, ctx, pos) of
    the next depth's nodes and nxt = dict(key, ctx, pos, owner) of the next depth's
    proposal rows (None at the last depth) in place."""
    n_seq = row_owner.numel() // n_blocks
    nx = nxt or {}
    dev = row_owner.device
    ids = _ids(rows_key, rows_ctx, rows_pos, 0, dev)
    with _on(dev):
        code = lib().pps_hetero_expand(n_seq, int(n_blocks), int(gamma), int(depth), _ptr(draft_tok), ids,
                                       _ptr(row_owner), _ptr(nx.get("key")), _ptr(nx.get("ctx")), _ptr(nx.get("pos")),
                                       _ptr(nx.get("owner")), _ptr(lists["tok"]), _ptr(lists["ndist"]),
                                       _ptr(lists["child"]), _ptr(nodes["key"]), _ptr(nodes["ctx"]),
                                       _ptr(nodes["pos"]), _stream(stream, dev))
    _check("pps_hetero_expand", code)


def hetero_block(tokens, key, ctx, pos, n_blocks: int, out=None, stream=None):
    """pps_hetero_block: the block J of the target's augmented point for each token."""
    n = tokens.numel()
    dev = tokens.device
    if out is None:
        out = torch.empty(n, dtype=torch.int32, device=dev)
    _need_detector(tokens, None, n, 0, dev)
    _need("out", out, dev, torch.int32, n)
    ids = _ids(key, ctx, pos, n, dev)
    with _on(dev):
        code = lib().pps_hetero_block(_ptr(tokens), ids, n, int(n_blocks), _ptr(out), _stream(stream, dev))
    _check("pps_hetero_block", code)
    return out


SCORE_AARONSON, SCORE_U, SCORE_LI, SCORE_POWER_LAW = 0, 1, 2, 3


def wm_detect(tokens, key, ctx, pos, seg_off=None, kind: int = SCORE_AARONSON, param: float = 0.0,
              want_scores: bool = True, want_logp: bool = True, stream=None):
    """pps_wm_detect.  Returns (scores or None, sums, log p-values or None)."""
    n = tokens.numel()
    dev = tokens.device
    n_seg = seg_off.numel() - 1 if seg_off is not None else 1
    out_score = torch.empty(n, dtype=torch.float32, device=dev) if want_scores else None
    out_sum = torch.empty(n_seg, dtype=torch.float64, device=dev)
    out_logp = torch.empty(n_seg, dtype=torch.float64, device=dev) if want_logp else None
    _need_detector(tokens, seg_off, n, n_seg, dev)
    ids = _ids(key, ctx, pos, n, dev)
    with _on(dev):
        code = lib().pps_wm_detect(_ptr(tokens), ids, n, n_seg, _ptr(seg_off), int(kind), float(param),
                                   _ptr(out_score), _ptr(out_sum), _ptr(out_logp), _stream(stream, dev))
    _check("pps_wm_detect", code)
    return out_score, out_sum, out_logp


def philox_words(key, ctx, pos, vocab: int, arrival: int = 1, stream=None):
    n = key.numel()
    dev = key.device
    out = torch.empty(n, vocab, dtype=torch.int32, device=dev)
    ids = _ids(key, ctx, pos, n, dev)
    with _on(dev):
        _check("pps_philox_words", lib().pps_philox_words(ids, n, vocab, arrival, _ptr(out), _stream(stream, dev)))
    return out


def selftest_key_error(w_begin: int = 0, w_end: int = 1 << 32, stream=None) -> float:
    out = torch.zeros(1, dtype=torch.float32, device="cuda")
    _check("pps_selftest_key_error", lib().pps_selftest_key_error(w_begin, w_end, _ptr(out), _stream(stream)))
    return float(out.item())


def selftest_lg2_error(x_lo: float = 2.0 ** -40, x_hi: float = 2.0 ** 7, stream=None) -> float:
    """Largest |lg2.approx(x) - log2 x| over every fp32 x in [x_lo, x_hi)."""
    out = torch.zeros(1, dtype=torch.float32, device="cuda")
    _check("pps_selftest_lg2_error", lib().pps_selftest_lg2_error(float(x_lo), float(x_hi), _ptr(out),
                                                                  _stream(stream)))
    return float(out.item())


def selftest_philox_rate(n_blocks: int, out_len: int, stream=None):
    """Launch the Philox-only throughput kernel (returns the folded words)."""
    out = torch.empty(out_len, dtype=torch.int32, device="cuda")
    _check("pps_selftest_philox_rate", lib().pps_selftest_philox_rate(n_blocks, _ptr(out), out_len, _stream(stream)))
    return out


# ---------------------------------------------------------------- LM head (the race fused into the GEMM)

def _lm_operands(hidden, weight):
    """Shapes and strides of the bf16 hidden states [n, d] and LM-head matrix [V, d]."""
    for name, t in (("hidden", hidden), ("weight", weight)):
        if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dim() != 2 or t.stride(1) != 1:
            raise TypeError(f"{name} must be a 2-D CUDA tensor with unit stride along d")
        if t.dtype != torch.bfloat16:
            raise TypeError(f"{name} must be bfloat16, got {t.dtype}")
    if hidden.device != weight.device:
        raise ValueError("hidden and weight must be on the same device")
    if hidden.shape[1] != weight.shape[1]:
        raise ValueError(f"hidden has d={hidden.shape[1]}, weight d={weight.shape[1]}")
    return hidden.shape[0], weight.shape[0], hidden.shape[1], hidden.stride(0), weight.stride(0)


def lmhead_workspace(n_rows: int, n_seq: int = 0, device=None) -> torch.Tensor:
    """A zeroed workspace for the fused LM-head calls."""
    nb = int(lib().pps_lmhead_workspace_size(n_rows, n_seq))
    return torch.zeros(nb, dtype=torch.uint8, device=device or "cuda")


def lmhead_logits(hidden, weight, out=None, stream=None):
    """pps_lmhead_logits: fp32 logits = hidden @ weight^T on the tensor cores (the unfused path)."""
    n, V, d, ldh, ldw = _lm_operands(hidden, weight)
    dev = hidden.device
    if out is None:
        out = torch.empty(n, V, dtype=torch.float32, device=dev)
    if out.dtype != torch.float32 or out.device != dev or out.dim() != 2 or out.stride(1) != 1 or \
            out.shape[0] < n or out.shape[1] < V:
        raise TypeError("out must be a float32 [n_rows, >= vocab] tensor on the operands' device")
    with _on(dev):
        code = lib().pps_lmhead_logits(_ptr(hidden), ldh, _ptr(weight), ldw, n, V, d, _ptr(out), out.stride(0),
                                       _stream(stream, dev))
    _check("pps_lmhead_logits", code)
    return out


def lmhead_draft_list(hidden, weight, key, ctx, pos, K: int, row_k=None, mode: int = DISTINCT,
                      temperature: float = 1.0, ws=None, status=None, out=None, keys: bool = True,
                      samples: bool = True, stream=None):
    """pps_lmhead_draft_list: the draft lists of pps_draft_list, computed in the LM-head GEMM's epilogue."""
    n, V, d, ldh, ldw = _lm_operands(hidden, weight)
    dev = hidden.device
    if out is None:
        out = dict(tok=torch.empty(n, K, dtype=torch.int32, device=dev),
                   key=torch.empty(n, K, dtype=torch.float32, device=dev) if keys else None,
                   mult=torch.empty(n, K, dtype=torch.int32, device=dev),
                   ndist=torch.empty(n, dtype=torch.int32, device=dev),
                   samples=torch.empty(n, K, dtype=torch.int32, device=dev) if samples else None)
    if ws is None:
        ws = lmhead_workspace(n, 0, dev)
    _need_draft(out, n, K, row_k, status, dev)
    _need("ws", ws, dev, torch.uint8)
    ids = _ids(key, ctx, pos, n, dev)
    with _on(dev):
        code = lib().pps_lmhead_draft_list(_ptr(hidden), ldh, _ptr(weight), ldw, n, V, d, ids, float(temperature),
                                           int(K), _ptr(row_k), int(mode), _ptr(out["tok"]), _ptr(out.get("key")),
                                           _ptr(out["mult"]), _ptr(out["ndist"]), _ptr(out.get("samples")),
                                           _ptr(status), _ptr(ws), ws.numel(), _stream(stream, dev))
    _check("pps_lmhead_draft_list", code)
    return out


def lmhead_verify_tree(hidden, weight, key, ctx, pos, gamma: int, seq_off, node_draft_row, draft_tok, draft_ndist,
                       child_node, temperature: float = 1.0, ws=None, status=None, out=None, stream=None):
    """pps_lmhead_verify_tree: the target race of every node, the tree walk and the scores of
    pps_verify_tree, computed in the LM-head GEMM's epilogue."""
    n, V, d, ldh, ldw = _lm_operands(hidden, weight)
    dev = hidden.device
    n_seq = seq_off.numel() - 1
    K = draft_tok.shape[1]
    W = gamma + 1
    if out is None:
        out = dict(winner=torch.empty(n, dtype=torch.int32, device=dev),
                   word=torch.empty(n, dtype=torch.int32, device=dev),
                   accept_len=torch.empty(n_seq, dtype=torch.int32, device=dev),
                   n_emitted=torch.empty(n_seq, dtype=torch.int32, device=dev),
                   emitted=torch.empty(n_seq, W, dtype=torch.int32, device=dev),
                   score=torch.empty(n_seq, W, dtype=torch.float32, device=dev),
                   score_sum=torch.empty(n_seq, dtype=torch.float64, device=dev))
    if ws is None:
        ws = lmhead_workspace(n, n_seq, dev)
    n_draft = draft_tok.shape[0]
    for name, t, numel in (("seq_off", seq_off, n_seq + 1), ("node_draft_row", node_draft_row, n),
                           ("draft_tok", draft_tok, n_draft * K), ("draft_ndist", draft_ndist, n_draft),
                           ("child_node", child_node, n_draft * K)):
        _need(name, t, dev, torch.int32, numel)
    _need_out(out, [("winner", torch.int32, n), ("word", torch.int32, n), ("accept_len", torch.int32, n_seq),
                    ("n_emitted", torch.int32, n_seq), ("emitted", torch.int32, n_seq * W),
                    ("score", torch.float32, n_seq * W), ("score_sum", torch.float64, n_seq)], dev)
    _need("status", status, dev, torch.int32, 1)
    _need("ws", ws, dev, torch.uint8)
    ids = _ids(key, ctx, pos, n, dev)
    with _on(dev):
        code = lib().pps_lmhead_verify_tree(_ptr(hidden), ldh, _ptr(weight), ldw, n, V, d, ids, float(temperature),
                                            n_seq, int(gamma), _ptr(seq_off), _ptr(node_draft_row), n_draft,
                                            _ptr(draft_tok), _ptr(draft_ndist), int(K), _ptr(child_node),
                                            _ptr(out["winner"]), _ptr(out["word"]), _ptr(out["accept_len"]),
                                            _ptr(out["n_emitted"]), _ptr(out["emitted"]), _ptr(out["score"]),
                                            _ptr(out["score_sum"]), _ptr(status), _ptr(ws), ws.numel(),
                                            _stream(stream, dev))
    _check("pps_lmhead_verify_tree", code)
    return out


# ---------------------------------------------------------------- target side of a step
#
# Host cost: a model makes these calls once per layer, some of them for a few tokens (kv_append of 8 tokens: one launch of
# 3 us), and checks and marshalling in Python take 10 to 27 us.  So each call first goes to pps_torch (csrc/pps_torch.cpp),
# which makes the common call, on the current stream, from C++; what it does not take (None) is checked and made below.

_HALVES = {torch.bfloat16: BF16, torch.float16: F16}

# the layouts of pps_append_args, pps_attention_args and pps_chain_args ("0q": padded to the struct's alignment)
_CACHE_FIELDS = "PPqiiiqqq"
_APPEND_ARGS = struct.Struct("@N" + "Pqq" * 4 + _CACHE_FIELDS + "PPPPPP" + "qq" + "iiiif" + "0q")
_ATTENTION_ARGS = struct.Struct("@N" + "Pqq" * 2 + _CACHE_FIELDS + "PPPPPPPN" + "qq" + "iiiiif" + "0q")
_CHAIN_ARGS = struct.Struct("@N" + "P" * 13 + "N" + "q" * 6 + "iiif" + "0q")


def _load_fast():
    """The extension that makes the common call (csrc/pps_torch.cpp; raises if it was not built), bound to the library."""
    global _fast
    L = lib()
    with _lock:
        if _fast is None:
            path = os.path.join(_HERE, "_lib", "pps_torch.so")
            if not os.path.exists(path):
                raise RuntimeError(f"pps_torch.so not found at {path}; build it with "
                                   "`python -c 'import __graft_entry__ as g; g.build()'`")
            spec = importlib.util.spec_from_file_location("pps_torch", path)
            ext = importlib.util.module_from_spec(spec)
            spec.loader.exec_module(ext)
            ext.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
                L.pps_kv_append, L.pps_paged_attention, L.pps_verify_chain, L.pps_attention_workspace_size,
                L.pps_chain_workspace_size)))
            _fast = ext
    return _fast


def _own_memory(stream):
    """A context for the tensors a call allocates itself: on the stream it is given they come from that
    stream's pool, so that neither pending nor later work of the current stream shares their memory."""
    return _HERE_ALREADY if stream is None else torch.cuda.stream(stream)


def _done(fn, x):
    """What the extension returned: a result, or the status code of a call that the library refused."""
    if x.__class__ is int:
        _check(fn, x)
    return x


class _Scratch:
    """`nbytes` of the caching allocator's memory, for the work that is queued on the stream `handle` while it is held:
    the next to be given it comes later on that stream.  (A tensor for it costs 2 us more.)"""

    def __init__(self, nbytes, handle):
        self.nbytes = nbytes
        self.address = torch._C._cuda_cudaCachingAllocator_raw_alloc(max(nbytes, 1), handle)

    def __del__(self):
        address, self.address = getattr(self, "address", 0), 0
        if address:
            torch._C._cuda_cudaCachingAllocator_raw_delete(address)


def _handle(stream, di):
    """The stream's handle; with no stream, the current stream of device di (the tensors')."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(di)
    if stream.device.index != di:
        raise ValueError(f"stream is on {stream.device}, the tensors on cuda:{di}")
    return stream.cuda_stream


def _strided(name, t, di, dt, shape, what):
    """Strides of tensor `t` of dtype `dt` on device di: contiguous along its last dimension, its sizes those of
    `shape` (None: any)."""
    if isinstance(t, torch.Tensor) and t.get_device() == di and t.dtype is dt and t.shape == shape:
        st = t.stride()
        if st[-1] == 1:
            return st
    _required(name, t, di)
    if t.dtype is not dt:
        raise TypeError(f"{name} must be {dt}, got {t.dtype}")
    have, st = t.shape, t.stride()
    if len(have) != len(shape) or (st[-1] != 1 and have[-1] > 1):
        raise TypeError(f"{name} must be {what} with unit stride along the last dimension")
    for x, y in zip(have, shape):
        if y is not None and x != y:
            raise ValueError(f"{name} is {list(have)}; the call needs {list(shape)} ({what})")
    return st


def _flat(name, t, di, dt, numel):
    """Address of a contiguous tensor of at least numel elements (0 when it is None)."""
    if t is None:
        return 0
    if isinstance(t, torch.Tensor) and t.get_device() == di and t.dtype is dt and t.is_contiguous() and t.numel() >= numel:
        return t.data_ptr()
    _need(name, t, torch.device("cuda", di), dt, numel)
    return t.data_ptr()


def _required(name, t, di):
    """Raise unless t is a tensor of device di."""
    if not isinstance(t, torch.Tensor) or t.get_device() != di:
        raise TypeError(f"{name} must be a CUDA tensor on cuda:{di}")
    return t


def _half_rows(q):
    """Device index, dtype and dtype code of the queries."""
    if not isinstance(q, torch.Tensor) or not q.is_cuda:
        raise TypeError("q must be a CUDA tensor")
    if q.dtype not in _HALVES:
        raise TypeError(f"q must be bfloat16 or float16, got {q.dtype}")
    if q.dim() != 3:
        raise TypeError("q must be [tokens, heads, channels]")
    return q.get_device(), q.dtype, _HALVES[q.dtype]


_HEADS = "[tokens, heads, channels]"
_CACHE = "[pages, page_size, heads, channels]"


def _cache(k, v, di, dt, d):
    """The fields of pps_kv_cache of the two halves of a paged cache, which have the same strides."""
    st = _strided("k_cache", k, di, dt, (None, None, None, d), _CACHE)
    n, page, heads, _ = shape = k.shape
    if _strided("v_cache", v, di, dt, shape, _CACHE) != st:
        raise ValueError("k_cache and v_cache must have the same strides")
    return k.data_ptr(), v.data_ptr(), n, page, heads, d, st[0], st[1], st[2]


def rope_table(max_pos: int, rot: int, base: float = 10000.0, device=None) -> torch.Tensor:
    """The [max_pos, rot] fp32 table of kv_append: cosines of position * base^(-2i / rot), i < rot / 2, then
    the sines (formed in 64 bits)."""
    if rot < 2 or rot % 2:
        raise ValueError(f"rot must be even and positive, got {rot}")
    dev = device or "cuda"
    freq = float(base) ** (-torch.arange(0, rot, 2, device=dev, dtype=torch.float64) / rot)
    t = torch.arange(max_pos, device=dev, dtype=torch.float64)[:, None] * freq
    return torch.cat([t.cos(), t.sin()], dim=1).float()


def kv_append(q, k, v, pos, slot, k_cache, v_cache, rope, q_norm=None, k_norm=None, eps: float = 1e-6,
              interleaved: bool = False, out=None, status=None, stream=None):
    """pps_kv_append: norm (optional) and rotate the queries and keys of new tokens, write keys and values to
    their cache slots.  Returns the queries (`out`, which may be q).  q [n, heads, d]; k, v [n, kv heads, d];
    k_cache, v_cache [pages, page_size, kv heads, d]; rope: rope_table or None (no rotation); slot int64, < 0:
    not written."""
    if stream is None:
        done = (_fast or _load_fast()).kv_append(q, k, v, pos, slot, k_cache, v_cache, rope, q_norm, k_norm, eps,
                                                 interleaved, out, status)
        if done is not None:
            return _done("pps_kv_append", done)
    di, dt, code = _half_rows(q)
    n, heads, d = shape = q.shape
    cache = _cache(k_cache, v_cache, di, dt, d)
    kv_shape = (n, cache[4], d)
    sq = _strided("q", q, di, dt, shape, _HEADS)
    sk = _strided("k", k, di, dt, kv_shape, _HEADS)
    sv = _strided("v", v, di, dt, kv_shape, _HEADS)
    rot = max_pos = table = at = 0
    if rope is not None:
        if _required("rope", rope, di).dim() != 2:
            raise TypeError("rope must be [max_pos, rot]")
        max_pos, rot = rope.shape
        table, at = _flat("rope", rope, di, torch.float32, 0), _flat("pos", _required("pos", pos, di), di, torch.int32, n)
    slots = _flat("slot", _required("slot", slot, di), di, torch.int64, n)
    wq, wk = _flat("q_norm", q_norm, di, dt, d), _flat("k_norm", k_norm, di, dt, d)
    flags = _flat("status", status, di, torch.int32, 1)
    if torch._C._cuda_getDevice() != di:
        with torch.cuda.device(di):
            return kv_append(q, k, v, pos, slot, k_cache, v_cache, rope, q_norm, k_norm, eps, interleaved, out, status,
                             stream)
    if out is None:
        with _own_memory(stream):
            out = torch.empty(n, heads, d, dtype=dt, device=q.device)
    so = _strided("out", out, di, dt, shape, _HEADS)
    args = _APPEND_ARGS.pack(_APPEND_ARGS.size, q.data_ptr(), sq[0], sq[1], k.data_ptr(), sk[0], sk[1], v.data_ptr(),
                             sv[0], sv[1], out.data_ptr(), so[0], so[1], *cache, wq, wk, table, at, slots, flags, n,
                             max_pos, code, heads, rot, 1 if interleaved else 0, eps)
    _check("pps_kv_append", lib().pps_kv_append(args, _handle(stream, di)))
    return out


def attention_workspace(n_tok: int, n_heads: int, n_kv_heads: int, head_dim: int, device=None) -> torch.Tensor:
    """A workspace for paged_attention calls of up to n_tok tokens (not shared by concurrent calls)."""
    nb = int(lib().pps_attention_workspace_size(n_tok, n_heads, n_kv_heads, head_dim))
    return torch.empty(nb, dtype=torch.uint8, device=device or "cuda")


def paged_attention(q, k_cache, v_cache, pages, kv_len, q_off, mask=None, scale=None, out=None, lse=None, ws=None,
                    status=None, stream=None):
    """pps_paged_attention: the newest tokens of each sequence (q [n, heads, d], those of sequence s in
    q_off[s] .. q_off[s+1]-1) attend to the paged cache.  pages [n_seq, columns] int32, kv_len [n_seq] int32
    (the new tokens' own keys included); mask [n, words] int32 tree masks, None: causal; scale None: 1/sqrt(d);
    lse: an optional [n, heads] float32 output.  Returns out (tokens that belong to no sequence are not written)."""
    if stream is None:
        done = (_fast or _load_fast()).paged_attention(q, k_cache, v_cache, pages, kv_len, q_off, mask, scale, out, lse,
                                                       ws, status)
        if done is not None:
            return _done("pps_paged_attention", done)
    di, dt, code = _half_rows(q)
    n, heads, d = shape = q.shape
    cache = _cache(k_cache, v_cache, di, dt, d)
    sq = _strided("q", q, di, dt, shape, _HEADS)
    i32 = torch.int32
    n_seq = _required("kv_len", kv_len, di).numel()
    sp = _strided("pages", pages, di, i32, (n_seq, None), "[n_seq, columns]")
    columns = pages.shape[1]
    lens = _flat("kv_len", kv_len, di, i32, 0)
    offs = _flat("q_off", _required("q_off", q_off, di), di, i32, n_seq + 1)
    words = bits = 0
    if mask is not None:
        if _required("mask", mask, di).dim() != 2 or mask.shape[0] != n or mask.shape[1] < 1:
            raise ValueError(f"mask must be [{n}, words]")
        words, bits = mask.shape[1], _flat("mask", mask, di, i32, 0)
    sums, flags = _flat("lse", lse, di, torch.float32, n * heads), _flat("status", status, di, i32, 1)
    work = _flat("ws", ws, di, torch.uint8, 0)
    if torch._C._cuda_getDevice() != di:
        with torch.cuda.device(di):
            return paged_attention(q, k_cache, v_cache, pages, kv_len, q_off, mask, scale, out, lse, ws, status, stream)
    if out is None:
        with _own_memory(stream):
            out = torch.empty(n, heads, d, dtype=dt, device=q.device)
    so = _strided("out", out, di, dt, shape, _HEADS)
    L, handle = lib(), _handle(stream, di)
    if ws is None:
        scratch = _Scratch(L.pps_attention_workspace_size(n, heads, cache[4], d), handle)
        work, room = scratch.address, scratch.nbytes
    else:
        room = ws.numel()
    # of one sequence, the table's row stride has no meaning; else one below the columns is the library's to refuse
    args = _ATTENTION_ARGS.pack(_ATTENTION_ARGS.size, q.data_ptr(), sq[0], sq[1], out.data_ptr(), so[0], so[1], *cache,
                                pages.data_ptr(), lens, offs, bits, sums, flags, work, room, n,
                                sp[0] if n_seq > 1 else columns, code, heads, columns, n_seq, words,
                                d ** -0.5 if scale is None else scale)
    _check("pps_paged_attention", L.pps_paged_attention(args, handle))
    return out


def chain_workspace(n_nodes: int, n_draft: int, n_seq: int, device=None) -> torch.Tensor:
    """A workspace for verify_chain calls of up to these sizes (not shared by concurrent calls)."""
    nb = int(lib().pps_chain_workspace_size(n_nodes, n_draft, n_seq))
    return torch.empty(nb, dtype=torch.uint8, device=device or "cuda")


def verify_chain(p_logits, q_logits, gamma: int, seq_off, node_draft_row, draft_tok, u, noise, temperature: float = 1.0,
                 ws=None, out=None, status=None, stream=None):
    """pps_verify_chain: the token-level maximal coupling along drafted chains of up to gamma tokens, from the
    uniforms u [n_draft] and exponentials noise [n_seq, >= V].  Returns dict(accept_len, n_emitted, emitted,
    accept_prob [n_draft], 0 for rows that no chain names); `out` may leave accept_prob out."""
    if stream is None and out is None:
        done = (_fast or _load_fast()).verify_chain(p_logits, q_logits, gamma, seq_off, node_draft_row, draft_tok, u, noise,
                                                    temperature, ws, status)
        if done is not None:
            return _done("pps_verify_chain", done)
    if not isinstance(p_logits, torch.Tensor) or not p_logits.is_cuda:
        raise TypeError("p_logits must be a CUDA tensor")
    di, dt, code = p_logits.get_device(), p_logits.dtype, _dtype_code(p_logits)
    rows = "[rows, vocabulary]"
    p_stride = _strided("p_logits", p_logits, di, dt, (None, None), rows)[0]
    n, V = p_logits.shape
    q_stride = _strided("q_logits", q_logits, di, _required("q_logits", q_logits, di).dtype, (None, V), rows)[0]
    if q_logits.dtype is not dt:
        raise ValueError("p_logits and q_logits must have the same dtype")
    n_draft = q_logits.shape[0]
    i32, f32 = torch.int32, torch.float32
    n_seq = _required("seq_off", seq_off, di).numel() - 1
    noise_stride = _strided("noise", noise, di, f32, (None, None), "[n_seq, >= vocabulary]")[0]
    if noise.shape[0] < n_seq or noise.shape[1] < V:
        raise ValueError(f"noise is {list(noise.shape)}; the call needs [{n_seq}, >= {V}]")
    # (a tensor that is not read may be None)
    inputs = [_flat(name, t if numel == 0 else _required(name, t, di), di, dtype, numel) for name, t, dtype, numel in (
        ("seq_off", seq_off, i32, n_seq + 1), ("node_draft_row", node_draft_row, i32, n),
        ("draft_tok", draft_tok, i32, n_draft), ("u", u, f32, n_draft))]
    flags, work = _flat("status", status, di, i32, 1), _flat("ws", ws, di, torch.uint8, 0)
    if torch._C._cuda_getDevice() != di:
        with torch.cuda.device(di):
            return verify_chain(p_logits, q_logits, gamma, seq_off, node_draft_row, draft_tok, u, noise, temperature, ws,
                                out, status, stream)
    W = gamma + 1
    if out is None:
        with _own_memory(stream):
            e, dev = torch.empty, p_logits.device
            out = dict(accept_len=e(n_seq, dtype=i32, device=dev), n_emitted=e(n_seq, dtype=i32, device=dev),
                       emitted=e((n_seq, W), dtype=i32, device=dev), accept_prob=e(n_draft, dtype=f32, device=dev))
    L, handle = lib(), _handle(stream, di)
    if ws is None:
        scratch = _Scratch(L.pps_chain_workspace_size(n, n_draft, n_seq), handle)
        work, room = scratch.address, scratch.nbytes
    else:
        room = ws.numel()
    for name in ("accept_len", "n_emitted", "emitted"):
        if out.get(name) is None:
            raise TypeError(f"out[{name!r}] is required")
    # rows of one sequence or one row have no stride
    args = _CHAIN_ARGS.pack(_CHAIN_ARGS.size, p_logits.data_ptr(), q_logits.data_ptr(), *inputs, noise.data_ptr(),
                            _flat("accept_len", out["accept_len"], di, i32, n_seq),
                            _flat("n_emitted", out["n_emitted"], di, i32, n_seq),
                            _flat("emitted", out["emitted"], di, i32, n_seq * W),
                            _flat("accept_prob", out.get("accept_prob"), di, f32, n_draft), flags, work, room, n,
                            n_draft, V, p_stride if n > 1 else V, q_stride if n_draft > 1 else V,
                            noise_stride if n_seq > 1 else V, code, n_seq, gamma, temperature)
    _check("pps_verify_chain", L.pps_verify_chain(args, handle))
    return out
