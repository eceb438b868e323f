"""Thin Python binding of the AVTP C ABI (``include/avtp.h``).

Argument marshalling only: every step of the pruning stage runs in the CUDA
kernels of ``libavtp.so``. torch supplies device memory and streams. There is
no CPU fallback: if the library is missing or a call fails, this module raises.

Function names follow the C ABI (``score``, ``allocate``, ``select``,
``compact``, ``prune``, ``workspace_size``, ``kept_count_host``,
``read_device_status``); each takes torch tensors and calls the entry point of
the same name.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
from ctypes import POINTER, c_double, c_float, c_int, c_int32, c_int64, c_size_t, c_void_p
from dataclasses import dataclass, field
from typing import Dict, Iterable, List, Optional, Sequence, Tuple

import numpy as np
import torch

from . import build as _build

OK = 0
ERR_INVALID_ARG = 1
ERR_UNSUPPORTED = 2
ERR_RANGE = 3
ERR_CUDA = 4
ERR_TIMEOUT = 5
ERR_DEVICE_INPUT = 6
ERR_WORKSPACE = 7

CRIT_HIDDEN_VARIATION = 0
CRIT_TEXT_ATTENTION = 1
MAX_ROW_SETS = 8
N_STEP_EVENTS = 5

_CRITERIA = {"hidden_variation": CRIT_HIDDEN_VARIATION, "text_attention": CRIT_TEXT_ATTENTION}
# avtp_query_set_t and avtp_attn_path_t
QUERIES_TEXT, QUERIES_LAST = 0, 1
ROPE_HALF, ROPE_INTERLEAVED = 0, 1
PATH_AUTO, PATH_TENSOR, PATH_CUDA = 0, 1, 2
_QUERY_SETS = {"text": QUERIES_TEXT, "last": QUERIES_LAST}
_ROPE_STYLES = {"half": ROPE_HALF, "interleaved": ROPE_INTERLEAVED}
_ROPE_SCALES = {None: 0, "linear": 1, "ntk": 2, "yarn": 3}
_PATHS = {"auto": PATH_AUTO, "tensor": PATH_TENSOR, "cuda": PATH_CUDA}


class AVTPError(RuntimeError):
    """A non-OK status from the library: ``code`` (an avtp_status_t value) and the call it came from."""
    def __init__(self, code: int, where: str):
        self.code = int(code)
        super().__init__(f"{where}: {status_string(code)} (status {code})")


# ---------------------------------------------------------------- C structs
class _Layout(ctypes.Structure):
    _fields_ = [("n_requests", c_int32), ("n_images", c_int32), ("n_tokens", c_int64),
                ("cu_seqlens", c_void_p), ("img_cu", c_void_p), ("img_start", c_void_p), ("img_len", c_void_p)]


class _ScoreArgs(ctypes.Structure):
    _fields_ = [("criterion", c_int), ("h_cur", c_void_p), ("h_prior", c_void_p), ("hidden", c_int32),
                ("h_cur_stride", c_int64), ("h_prior_stride", c_int64), ("q", c_void_p), ("k", c_void_p),
                ("n_q_heads", c_int32), ("n_kv_heads", c_int32), ("head_dim", c_int32), ("q_stride", c_int64),
                ("k_stride", c_int64), ("softmax_scale", c_float), ("lse", c_void_p), ("lse_stride", c_int64),
                ("max_text_tokens", c_int64), ("query_set", c_int32), ("path", c_int32)]


class _AllocArgs(ctypes.Structure):
    _fields_ = [("keep_ratio", c_void_p), ("alpha", c_float), ("r_min", c_float), ("r_max", c_float),
                ("relative", c_int32)]


class _Rows(ctypes.Structure):
    _fields_ = [("in_", c_void_p), ("out", c_void_p), ("row_bytes", c_int64), ("in_stride", c_int64),
                ("out_stride", c_int64)]


class _Cache(ctypes.Structure):
    _fields_ = [("k", c_void_p), ("v", c_void_p), ("n_pages", c_int64), ("page_size", c_int32),
                ("n_kv_heads", c_int32), ("head_dim", c_int32), ("k_page_stride", c_int64),
                ("k_token_stride", c_int64), ("k_head_stride", c_int64), ("v_page_stride", c_int64),
                ("v_token_stride", c_int64), ("v_head_stride", c_int64)]


class _CacheSlotsArgs(ctypes.Structure):
    _fields_ = [("n_requests", c_int32), ("n_tokens", c_int64), ("page_size", c_int32), ("n_pages", c_int64),
                ("max_pages", c_int32), ("table_stride", c_int64), ("cu_new", c_void_p), ("past_len", c_void_p),
                ("free_pages", c_void_p), ("n_free", c_int64), ("free_head", c_void_p), ("block_table", c_void_p),
                ("seq_len", c_void_p), ("slot_map", c_void_p), ("free_head_out", c_void_p)]


class _CacheWriteArgs(ctypes.Structure):
    _fields_ = [("k", c_void_p), ("v", c_void_p), ("k_stride", c_int64), ("v_stride", c_int64), ("n_rows", c_int64),
                ("kept_idx", c_void_p), ("slot_map", c_void_p), ("n", c_int64)]


class _RopeArgs(ctypes.Structure):
    _fields_ = [("n_tokens", c_int64), ("n_q_heads", c_int32), ("n_kv_heads", c_int32), ("head_dim", c_int32),
                ("q", c_void_p), ("q_stride", c_int64), ("q_out", c_void_p), ("q_out_stride", c_int64),
                ("k", c_void_p), ("k_stride", c_int64), ("k_out", c_void_p), ("k_out_stride", c_int64),
                ("v", c_void_p), ("v_stride", c_int64), ("slot_map", c_void_p), ("rot_dim", c_int32),
                ("style", c_int32), ("inv_freq", c_void_p), ("pos", c_void_p), ("pos_stride", c_int64),
                ("n_planes", c_int32), ("pair_plane", c_void_p), ("attn_factor", c_float), ("q_norm", c_void_p),
                ("k_norm", c_void_p), ("eps", c_float)]


class _RopeFreqArgs(ctypes.Structure):
    _fields_ = [("rot_dim", c_int32), ("scale", c_int32), ("base", c_double), ("factor", c_double),
                ("original_len", c_double), ("slow", c_double), ("fast", c_double)]


class _CacheAttnArgs(ctypes.Structure):
    _fields_ = [("n_requests", c_int32), ("n_tokens", c_int64), ("max_new", c_int32), ("n_q_heads", c_int32),
                ("q", c_void_p), ("q_stride", c_int64), ("cu_new", c_void_p), ("seq_len", c_void_p),
                ("block_table", c_void_p), ("max_pages", c_int32), ("table_stride", c_int64),
                ("softmax_scale", c_float), ("o", c_void_p), ("o_stride", c_int64), ("lse", c_void_p),
                ("lse_stride", c_int64)]


class _CacheWindow(ctypes.Structure):
    _fields_ = [("window", c_int32), ("n_sinks", c_int32)]


class _CacheCompactArgs(ctypes.Structure):
    _fields_ = [("n_requests", c_int32), ("n_kept", c_int64), ("keep_cu", c_void_p), ("keep_idx", c_void_p),
                ("base_cu", c_void_p), ("seq_len", c_void_p), ("block_table", c_void_p), ("max_pages", c_int32),
                ("table_stride", c_int64), ("dst_table", c_void_p), ("dst_max_pages", c_int32), ("dst_stride", c_int64),
                ("shared", c_void_p), ("window", c_int32), ("n_sinks", c_int32), ("held_len", c_void_p),
                ("len_out", c_void_p)]


class _CacheForkArgs(ctypes.Structure):
    _fields_ = [("n_requests", c_int32), ("n_children", c_int32), ("page_size", c_int32), ("n_pages", c_int64),
                ("max_pages", c_int32), ("table_stride", c_int64), ("parent", c_void_p), ("child", c_void_p),
                ("fork_len", c_void_p), ("free_pages", c_void_p), ("n_free", c_int64), ("free_head", c_void_p),
                ("block_table", c_void_p), ("seq_len", c_void_p), ("shared", c_void_p), ("window", c_int32),
                ("n_sinks", c_int32), ("held_len", c_void_p), ("copy_src", c_void_p), ("copy_dst", c_void_p),
                ("free_head_out", c_void_p)]


class _CacheFreeArgs(ctypes.Structure):
    _fields_ = [("n_requests", c_int32), ("page_size", c_int32), ("n_pages", c_int64), ("max_pages", c_int32),
                ("table_stride", c_int64), ("seq_len", c_void_p), ("new_len", c_void_p), ("block_table", c_void_p),
                ("free_pages", c_void_p), ("n_free", c_int64), ("free_head", c_void_p), ("shared", c_void_p),
                ("window", c_int32), ("n_sinks", c_int32), ("held_len", c_void_p), ("seq_len_out", c_void_p),
                ("held_len_out", c_void_p), ("free_head_out", c_void_p)]


class _ForwardArgs(ctypes.Structure):
    _fields_ = [("v", c_void_p), ("v_stride", c_int64), ("o", c_void_p), ("o_stride", c_int64), ("lse", c_void_p),
                ("lse_stride", c_int64)]


# ---------------------------------------------------------------- library
_LIB = None

# name -> (restype, argtypes); every symbol the header declares
SIGNATURES = {
    "avtp_workspace_size": (c_int, [POINTER(_Layout), POINTER(_ScoreArgs), POINTER(c_size_t)]),
    "avtp_score": (c_int, [POINTER(_Layout), POINTER(_ScoreArgs), c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "avtp_forward_workspace_size": (c_int, [POINTER(_Layout), POINTER(_ScoreArgs), POINTER(_ForwardArgs),
                                            POINTER(c_size_t)]),
    "avtp_attn_forward": (c_int, [POINTER(_Layout), POINTER(_ScoreArgs), POINTER(_ForwardArgs), c_void_p, c_void_p,
                                  c_void_p, c_size_t, c_void_p]),
    "avtp_forward_timeline": (c_int, [c_void_p, c_int32]),
    "avtp_score_timeline": (c_int, [c_int32, c_void_p, c_int32]),
    "avtp_allocate": (c_int, [POINTER(_Layout), c_void_p, POINTER(_AllocArgs), c_void_p, c_void_p, c_void_p,
                              c_size_t, c_void_p]),
    "avtp_select": (c_int, [POINTER(_Layout), c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_void_p, c_size_t,
                            c_void_p]),
    "avtp_compact": (c_int, [c_void_p, c_int64, c_int64, POINTER(_Rows), c_int32, c_void_p, c_size_t, c_void_p]),
    "avtp_prune": (c_int, [POINTER(_Layout), POINTER(_ScoreArgs), POINTER(_AllocArgs), c_void_p, c_void_p, c_void_p,
                           c_void_p, c_void_p, c_int64, POINTER(_Rows), c_int32, c_void_p, c_size_t,
                           POINTER(c_void_p), c_void_p]),
    "avtp_select_noalloc": (c_int, [POINTER(_Layout), c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_void_p,
                                    c_void_p]),
    "avtp_kept_count_host": (c_int64, [c_void_p, c_void_p, c_void_p, c_void_p, c_int32]),
    "avtp_pruned_layout": (c_int, [POINTER(_Layout), c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "avtp_kept_count_vis_host": (c_int64, [c_void_p, c_void_p, c_void_p, c_int32, c_void_p, c_void_p]),
    "avtp_cache_slots_workspace_size": (c_int, [POINTER(_CacheSlotsArgs), POINTER(c_size_t)]),
    "avtp_cache_slots": (c_int, [POINTER(_CacheSlotsArgs), c_void_p, c_size_t, c_void_p]),
    "avtp_cache_write": (c_int, [POINTER(_Cache), POINTER(_CacheWriteArgs), c_void_p, c_size_t, c_void_p]),
    "avtp_rope": (c_int, [POINTER(_RopeArgs), POINTER(_Cache), c_void_p, c_size_t, c_void_p]),
    "avtp_rope_frequencies": (c_int, [POINTER(_RopeFreqArgs), POINTER(c_float), POINTER(c_float)]),
    "avtp_cache_attention_workspace_size": (c_int, [POINTER(_Cache), POINTER(_CacheAttnArgs), POINTER(c_size_t)]),
    "avtp_cache_attention": (c_int, [POINTER(_Cache), POINTER(_CacheAttnArgs), c_void_p, c_size_t, c_void_p]),
    "avtp_cache_window_attention_workspace_size": (c_int, [POINTER(_Cache), POINTER(_CacheAttnArgs),
                                                           POINTER(_CacheWindow), POINTER(c_size_t)]),
    "avtp_cache_window_attention": (c_int, [POINTER(_Cache), POINTER(_CacheAttnArgs), POINTER(_CacheWindow), c_void_p,
                                            c_size_t, c_void_p]),
    "avtp_cache_compact": (c_int, [POINTER(_Cache), POINTER(_CacheCompactArgs), c_void_p, c_size_t, c_void_p]),
    "avtp_cache_copy": (c_int, [POINTER(_Cache), c_void_p, c_void_p, c_int64, c_void_p, c_size_t, c_void_p]),
    "avtp_cache_fork_workspace_size": (c_int, [POINTER(_CacheForkArgs), POINTER(c_size_t)]),
    "avtp_cache_fork": (c_int, [POINTER(_CacheForkArgs), c_void_p, c_size_t, c_void_p]),
    "avtp_cache_free_workspace_size": (c_int, [POINTER(_CacheFreeArgs), POINTER(c_size_t)]),
    "avtp_cache_free": (c_int, [POINTER(_CacheFreeArgs), c_void_p, c_size_t, c_void_p]),
    "avtp_wait_selftest": (c_int, [c_int64, c_int32, c_void_p, c_size_t, c_void_p]),
    "avtp_layer_attention": (c_int, [POINTER(_Layout), c_void_p, c_void_p, c_int32, c_int32, c_void_p, c_size_t,
                                     c_void_p]),
    "avtp_layer_select": (c_int, [c_void_p, c_int32, c_int32, c_int32, c_void_p, c_void_p, c_void_p]),
    "avtp_read_device_status": (c_int, [c_void_p, c_void_p, POINTER(c_int32)]),
    "avtp_status_string": (ctypes.c_char_p, [c_int32]),
    "avtp_version": (c_int32, []),
}


def library_path() -> str:
    """Path of the in-tree libavtp.so that ``load()`` opens: the diagnostic timeline build
    when the environment sets AVTP_TIMELINE=1, the normal build otherwise."""
    return _build.TIMELINE_LIB_PATH if os.environ.get("AVTP_TIMELINE") == "1" else _build.LIB_PATH


def load() -> ctypes.CDLL:
    """Load libavtp.so (built by ``__graft_entry__.build()``); raise if it is missing."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = library_path()
    if not os.path.exists(path):
        if os.environ.get("AVTP_AUTOBUILD") == "1":
            _build.build(timeline=path == _build.TIMELINE_LIB_PATH)
        else:
            raise RuntimeError(f"libavtp.so is not built ({path}); run __graft_entry__.build() first")
    lib = ctypes.CDLL(path)
    for name, (res, args) in SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _LIB = lib
    return lib


TIMELINE_EVENTS = ("prep_begin", "prep_end", "score_begin", "score_end", "select_begin", "select_dry_end",
                   "select_waited", "rule_begin", "rule_end", "select_end", "compact_begin", "compact_waited",
                   "compact_end", "hist_done")


def timeline(workspace: torch.Tensor) -> Dict[str, Tuple[int, int]]:
    """Phase stamps of the last avtp_prune on ``workspace`` (timeline build only): event ->
    (earliest, latest) global-timer nanoseconds over the CTAs that reached it; events no CTA
    reached are left out. Synchronises the device."""
    torch.cuda.synchronize()
    n = len(TIMELINE_EVENTS)
    raw = workspace[16:16 + 16 * n].cpu().numpy().view(np.uint64)
    out = {}
    for i, name in enumerate(TIMELINE_EVENTS):
        lo, hi = int(raw[i]), int(raw[n + i])
        if lo != 2 ** 64 - 1:
            out[name] = (lo, hi)
    return out


def status_string(code: int) -> str:
    """avtp_status_string: static English text for a status code."""
    return load().avtp_status_string(int(code)).decode()


def _check(code: int, where: str) -> None:
    if code != OK:
        raise AVTPError(code, where)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else int(t.data_ptr())


# The current stream's handle without a torch.cuda.Stream object around it: 1 us of a call
# instead of 7 (torch's own generated code takes it this way).
_RAW_STREAM = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is None:
        if _RAW_STREAM is not None and torch.cuda.is_initialized():
            return int(_RAW_STREAM(torch._C._cuda_getDevice()))
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream) if hasattr(stream, "cuda_stream") else int(stream)


# ---------------------------------------------------------------- layout
@dataclass
class Layout:
    """A varlen-packed multi-image layout on the device (int32 tensors) plus host copies. A
    program may refill both for its next batch.

    A layout made by ``pruned_layout`` keeps its image spans on the device only: its
    host copy holds cu_seqlens, img_cu and the visual tokens per request (``n_vis``).
    """
    cu_seqlens: torch.Tensor
    img_cu: torch.Tensor
    img_start: torch.Tensor
    img_len: torch.Tensor
    host: Dict[str, np.ndarray]

    # what n_text counted last: the host arrays' bytes, and the visual tokens in them
    _counted: Tuple[Optional[tuple], int] = field(default=(None, 0), init=False, repr=False, compare=False)

    @staticmethod
    def from_host(cu_seqlens, img_cu, img_start, img_len, device="cuda") -> "Layout":
        """Copies host layout arrays (int32) to ``device`` and keeps the host copies."""
        host = {k: np.ascontiguousarray(np.asarray(v, dtype=np.int32))
                for k, v in dict(cu_seqlens=cu_seqlens, img_cu=img_cu, img_start=img_start, img_len=img_len).items()}
        dev = {k: torch.from_numpy(v.copy()).to(device) for k, v in host.items()}
        return Layout(host=host, **dev)

    @property
    def n_requests(self) -> int:
        """R, the number of varlen-packed requests."""
        return int(self.host["cu_seqlens"].shape[0] - 1)

    @property
    def n_images(self) -> int:
        """Images over all requests."""
        return int(self.host["img_cu"][-1])

    @property
    def n_tokens(self) -> int:
        """T, the packed tokens over all requests."""
        return int(self.host["cu_seqlens"][-1])

    @property
    def n_vis_per_request(self) -> np.ndarray:
        """Visual tokens of each request (int32 [R])."""
        if "n_vis" in self.host:
            return self.host["n_vis"]
        csum = np.concatenate([[0], np.cumsum(self.host["img_len"].astype(np.int64))])
        return (csum[self.host["img_cu"][1:]] - csum[self.host["img_cu"][:-1]]).astype(np.int32)

    @property
    def n_text(self) -> int:
        """Text tokens over all requests."""
        # counting takes 17 us of a scoring call (a plain sum of img_len 6), comparing the arrays
        # with those counted last 1 to 2
        h = self.host
        seen = (h["n_vis"].tobytes(),) if "n_vis" in h else (h["img_len"].tobytes(), h["img_cu"].tobytes())
        counted = self._counted
        if counted[0] != seen:
            counted = self._counted = (seen, int(self.n_vis_per_request.astype(np.int64).sum()))
        return self.n_tokens - counted[1]

    def c(self) -> _Layout:
        """The avtp_layout_t the C calls take (pointers into the device tensors)."""
        return _Layout(self.n_requests, self.n_images, self.n_tokens, _ptr(self.cu_seqlens), _ptr(self.img_cu),
                       _ptr(self.img_start) if self.n_images else None, _ptr(self.img_len) if self.n_images else None)


def _score_args(criterion, h_cur=None, h_prior=None, q=None, k=None, softmax_scale=None, lse=None,
                max_text_tokens=0, query_set="text", path="auto") -> _ScoreArgs:
    a = _ScoreArgs()
    a.max_text_tokens = int(max_text_tokens)
    a.query_set = _QUERY_SETS[query_set] if isinstance(query_set, str) else int(query_set)
    a.path = _PATHS[path] if isinstance(path, str) else int(path)
    a.criterion = _CRITERIA[criterion] if isinstance(criterion, str) else int(criterion)
    if a.criterion == CRIT_HIDDEN_VARIATION:
        for t in (h_cur, h_prior):
            if t is None or t.dtype != torch.bfloat16 or t.dim() != 2 or t.stride(1) != 1:
                raise ValueError("h_cur / h_prior must be bf16 [T, hidden] with a contiguous last dim")
        a.h_cur, a.h_prior = _ptr(h_cur), _ptr(h_prior)
        a.hidden = h_cur.shape[1]
        a.h_cur_stride, a.h_prior_stride = h_cur.stride(0), h_prior.stride(0)
    else:
        for t in (q, k):
            if t is None or t.dtype != torch.bfloat16 or t.dim() != 3 or t.stride(2) != 1 or t.stride(1) != t.shape[2]:
                raise ValueError("q / k must be bf16 [T, heads, head_dim] with contiguous heads")
        a.q, a.k = _ptr(q), _ptr(k)
        a.n_q_heads, a.n_kv_heads, a.head_dim = q.shape[1], k.shape[1], q.shape[2]
        a.q_stride, a.k_stride = q.stride(0), k.stride(0)
        a.softmax_scale = float(softmax_scale if softmax_scale is not None else q.shape[2] ** -0.5)
        if lse is not None:
            if lse.dtype != torch.float32 or lse.dim() != 2 or lse.stride(1) != 1:
                raise ValueError("lse must be fp32 [Hq, T] with a contiguous last dim")
            a.lse, a.lse_stride = _ptr(lse), lse.stride(0)
    return a


def _alloc_args(keep_ratio: torch.Tensor, alpha=1.0, r_min=0.05, r_max=0.95, relative=False) -> _AllocArgs:
    if keep_ratio.dtype != torch.float32 or not keep_ratio.is_cuda:
        raise ValueError("keep_ratio must be a float32 CUDA tensor [R]")
    return _AllocArgs(_ptr(keep_ratio), float(alpha), float(r_min), float(r_max), 1 if relative else 0)


def _row_sets(rows: Sequence[Tuple[torch.Tensor, torch.Tensor]]) -> Tuple[ctypes.Array, int]:
    """(in, out) pairs gathered along dim 0: row j of out = row kept_idx[j] of in."""
    arr = (_Rows * MAX_ROW_SETS)()
    if len(rows) > MAX_ROW_SETS:
        raise ValueError(f"at most {MAX_ROW_SETS} row sets")
    for i, (src, dst) in enumerate(rows):
        es = src.element_size()
        row_elems = int(np.prod(src.shape[1:])) if src.dim() > 1 else 1
        if src.dim() > 1 and not src[0].is_contiguous():
            raise ValueError("each row must be contiguous")
        arr[i] = _Rows(_ptr(src), _ptr(dst), row_elems * es, src.stride(0) * es, dst.stride(0) * es)
    return arr, len(rows)


def workspace_size(layout: Layout, criterion=None, **score_tensors) -> int:
    """avtp_workspace_size: bytes of workspace a call needs for this layout and scoring setup."""
    lay = layout.c()
    sa = _score_args(criterion, max_text_tokens=layout.n_text, **score_tensors) if criterion is not None else None
    out = c_size_t()
    _check(load().avtp_workspace_size(ctypes.byref(lay), ctypes.byref(sa) if sa is not None else None,
                                      ctypes.byref(out)), "avtp_workspace_size")
    return int(out.value)


def new_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    """A caller-owned workspace (torch allocations are 256-byte aligned)."""
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


# ---------------------------------------------------------------- entry points
def score(layout: Layout, criterion, *, h_cur=None, h_prior=None, q=None, k=None, softmax_scale=None, lse=None,
          query_set="text", path="auto", scores=None, img_sums=None, workspace=None, stream=None):
    """avtp_score: per-token scores (fp32 [T], text entries untouched) and fixed-point per-image sums.

    Text attention: ``query_set`` "text" (every text token) or "last" (the request's last
    token); ``path`` "auto", "tensor" (tcgen05) or "cuda" (CUDA cores)."""
    dev = layout.cu_seqlens.device
    sa = _score_args(criterion, h_cur, h_prior, q, k, softmax_scale, lse, max_text_tokens=layout.n_text,
                     query_set=query_set, path=path)
    if scores is None:
        scores = torch.zeros(layout.n_tokens, dtype=torch.float32, device=dev)
    if img_sums is None:
        img_sums = torch.empty(max(layout.n_images, 1), dtype=torch.int64, device=dev)
    if workspace is None:
        workspace = new_workspace(workspace_size(layout, criterion, h_cur=h_cur, h_prior=h_prior, q=q, k=k,
                                                 softmax_scale=softmax_scale, lse=lse, query_set=query_set,
                                                 path=path), dev)
    lay = layout.c()
    _check(load().avtp_score(ctypes.byref(lay), ctypes.byref(sa), _ptr(scores), _ptr(img_sums), _ptr(workspace),
                             workspace.numel(), _stream(stream)), "avtp_score")
    return scores, img_sums if img_sums.shape[0] == layout.n_images else img_sums[:layout.n_images]


def _forward_args(v: torch.Tensor, o: torch.Tensor, lse: torch.Tensor) -> _ForwardArgs:
    if v.dtype != torch.bfloat16 or v.dim() != 3 or v.stride(2) != 1 or v.stride(1) != v.shape[2]:
        raise ValueError("v must be bf16 [T, Hkv, head_dim] with contiguous heads")
    if o.dtype != torch.float32 or o.dim() != 3 or o.stride(2) != 1 or o.stride(1) != o.shape[2]:
        raise ValueError("o must be fp32 [T, Hq, head_dim] with contiguous heads")
    if lse.dtype != torch.float32 or lse.dim() != 2 or lse.stride(1) != 1:
        raise ValueError("lse must be fp32 [Hq, T] with a contiguous last dim")
    return _ForwardArgs(_ptr(v), v.stride(0), _ptr(o), o.stride(0), _ptr(lse), lse.stride(0))


class ForwardCall:
    """A prepared avtp_attn_forward call: arguments marshalled once, outputs and workspace
    allocated once, so that ``run()`` is the C call alone (for timing and graphs)."""

    def __init__(self, layout: Layout, *, q, k, v, softmax_scale=None, scores: bool = True, query_set="text",
                 path="auto", o=None, lse=None, workspace=None):
        dev = layout.cu_seqlens.device
        T, Hq, d = q.shape
        self.layout = layout
        self.o = o if o is not None else torch.empty(T, Hq, d, dtype=torch.float32, device=dev)
        self.lse = lse if lse is not None else torch.empty(Hq, max(T, 1), dtype=torch.float32, device=dev)
        self.scores = torch.zeros(T, dtype=torch.float32, device=dev) if scores else None
        self.img_sums = torch.empty(max(layout.n_images, 1), dtype=torch.int64, device=dev) if scores else None
        self._keep = (q, k, v)
        self._sa = _score_args(CRIT_TEXT_ATTENTION, q=q, k=k, softmax_scale=softmax_scale,
                               max_text_tokens=layout.n_text, query_set=query_set, path=path)
        self._fa = _forward_args(v, self.o, self.lse)
        self._lay = layout.c()
        lib = load()
        if workspace is None:
            n = c_size_t()
            _check(lib.avtp_forward_workspace_size(ctypes.byref(self._lay), ctypes.byref(self._sa),
                                                   ctypes.byref(self._fa), ctypes.byref(n)),
                   "avtp_forward_workspace_size")
            workspace = new_workspace(int(n.value), dev)
        self.workspace = workspace

    def run(self, stream=None):
        _check(load().avtp_attn_forward(ctypes.byref(self._lay), ctypes.byref(self._sa), ctypes.byref(self._fa),
                                        _ptr(self.scores), _ptr(self.img_sums), _ptr(self.workspace),
                                        self.workspace.numel(), _stream(stream)), "avtp_attn_forward")
        return self


FORWARD_TIMELINE_SLOTS = ("top", "s_ready", "half_done", "exp_done", "p_handed", "mma_s_entry", "mma_s_issued",
                          "mma_pv_entry", "mma_pv_ready", "mma_pv_issued")


def forward_timeline(n_blocks: int) -> np.ndarray:
    """avtp_forward_timeline: clock stamps int64 [n_blocks, 10] (FORWARD_TIMELINE_SLOTS) of the
    last forward call's first CTA; needs the timeline build (AVTP_TIMELINE=1)."""
    out = np.zeros((n_blocks, len(FORWARD_TIMELINE_SLOTS)), dtype=np.int64)
    _check(load().avtp_forward_timeline(out.ctypes.data, n_blocks), "avtp_forward_timeline")
    return out


SCORE_TIMELINE_SLOTS = ("load_issued", "mma_step", "mma_ready", "mma_issued", "acc_ready", "acc_released")


def score_timeline(pass_: int, n_steps: int) -> np.ndarray:
    """avtp_score_timeline: clock stamps int64 [n_steps, 6] (SCORE_TIMELINE_SLOTS) of the first
    CTA of criterion B's tensor-core pass 1 or 2; needs the timeline build (AVTP_TIMELINE=1)."""
    out = np.zeros((n_steps, len(SCORE_TIMELINE_SLOTS)), dtype=np.int64)
    _check(load().avtp_score_timeline(int(pass_), out.ctypes.data, n_steps), "avtp_score_timeline")
    return out


def attn_forward(layout: Layout, *, q, k, v, softmax_scale=None, scores: bool = True, query_set="text",
                 path="auto", stream=None):
    """avtp_attn_forward: the layer's causal attention forward, O (fp32 [T, Hq, d]) and the
    natural-log LSE (fp32 [Hq, T]), and with ``scores`` the text-attention scores and
    fixed-point image sums from that LSE. Returns (o, lse, scores, img_sums); the last
    two are None without ``scores``."""
    c = ForwardCall(layout, q=q, k=k, v=v, softmax_scale=softmax_scale, scores=scores, query_set=query_set,
                    path=path).run(stream)
    sums = c.img_sums[:layout.n_images] if c.img_sums is not None else None
    return c.o, c.lse[:, :layout.n_tokens], c.scores, sums


def allocate(layout: Layout, img_sums: torch.Tensor, keep_ratio: torch.Tensor, alpha=1.0, r_min=0.05, r_max=0.95,
             relative=False, budgets=None, out_cu_seqlens=None, workspace=None, stream=None):
    """avtp_allocate: per-image budgets (int32 [n_images]) and out_cu_seqlens (int32 [R+1])."""
    dev = layout.cu_seqlens.device
    aa = _alloc_args(keep_ratio, alpha, r_min, r_max, relative)
    if budgets is None:
        budgets = torch.empty(max(layout.n_images, 1), dtype=torch.int32, device=dev)
    if out_cu_seqlens is None:
        out_cu_seqlens = torch.empty(layout.n_requests + 1, dtype=torch.int32, device=dev)
    if workspace is None:
        workspace = new_workspace(workspace_size(layout), dev)
    lay = layout.c()
    _check(load().avtp_allocate(ctypes.byref(lay), _ptr(img_sums), ctypes.byref(aa), _ptr(budgets),
                                _ptr(out_cu_seqlens), _ptr(workspace), workspace.numel(), _stream(stream)),
           "avtp_allocate")
    return budgets[:layout.n_images], out_cu_seqlens


def select(layout: Layout, scores: torch.Tensor, budgets: torch.Tensor, out_cu_seqlens: torch.Tensor, n_kept: int,
           kept_idx=None, workspace=None, stream=None):
    """avtp_select: ascending packed positions of the kept tokens (int32 [n_kept])."""
    dev = layout.cu_seqlens.device
    if kept_idx is None:
        kept_idx = torch.empty(max(int(n_kept), 1), dtype=torch.int32, device=dev)
    if workspace is None:
        workspace = new_workspace(workspace_size(layout), dev)
    lay = layout.c()
    _check(load().avtp_select(ctypes.byref(lay), _ptr(scores), _ptr(budgets), _ptr(out_cu_seqlens), _ptr(kept_idx),
                              int(n_kept), _ptr(workspace), workspace.numel(), _stream(stream)), "avtp_select")
    return kept_idx[:int(n_kept)]


def select_noalloc(layout: Layout, scores: torch.Tensor, budgets: torch.Tensor, out_cu_seqlens: torch.Tensor,
                   kept_idx: torch.Tensor, n_kept: int, device_status: Optional[torch.Tensor] = None,
                   stream=None) -> torch.Tensor:
    """avtp_select_noalloc: avtp_select with the library's fixed scratch instead of a workspace.

    For callers that cannot allocate device memory at the call site; ``kept_idx``
    (int32, capacity >= n_kept) must be supplied by the caller.
    """
    lay = layout.c()
    _check(load().avtp_select_noalloc(ctypes.byref(lay), _ptr(scores), _ptr(budgets), _ptr(out_cu_seqlens),
                                      _ptr(kept_idx), int(n_kept), _ptr(device_status), _stream(stream)),
           "avtp_select_noalloc")
    return kept_idx[:int(n_kept)]


def compact(kept_idx: torch.Tensor, n_tokens: int, rows: Sequence[Tuple[torch.Tensor, torch.Tensor]],
            workspace=None, stream=None) -> None:
    """avtp_compact: for each (in, out) pair, out[j] = in[kept_idx[j]] along dim 0."""
    dev = kept_idx.device
    if workspace is None:
        workspace = new_workspace(256, dev)
    sets, n = _row_sets(rows)
    _check(load().avtp_compact(_ptr(kept_idx), kept_idx.numel(), int(n_tokens), sets, n, _ptr(workspace),
                               workspace.numel(), _stream(stream)), "avtp_compact")


def kept_count_vis_host(cu_seqlens: np.ndarray, n_vis: np.ndarray, keep_ratio: np.ndarray):
    """avtp_kept_count_vis_host: the pruned batch's size, host offsets and visual tokens per request."""
    cu = np.ascontiguousarray(np.asarray(cu_seqlens, dtype=np.int32))
    nv = np.ascontiguousarray(np.asarray(n_vis, dtype=np.int32))
    kr = np.ascontiguousarray(np.asarray(keep_ratio, dtype=np.float32))
    R = int(cu.shape[0] - 1)
    out_cu = np.zeros(R + 1, dtype=np.int32)
    out_nv = np.zeros(R, dtype=np.int32)
    n = load().avtp_kept_count_vis_host(cu.ctypes.data, nv.ctypes.data, kr.ctypes.data, R, out_cu.ctypes.data,
                                        out_nv.ctypes.data)
    if n < 0:
        raise AVTPError(ERR_INVALID_ARG, "avtp_kept_count_vis_host")
    return int(n), out_cu, out_nv


def pruned_layout(layout: Layout, keep_ratio_host: np.ndarray, budgets: torch.Tensor, out_cu_seqlens: torch.Tensor,
                  workspace=None, stream=None, into: Optional[Layout] = None) -> Layout:
    """avtp_pruned_layout: the layout of the batch that avtp_prune produced (device arrays).

    ``budgets`` and ``out_cu_seqlens`` are the prune call's device outputs; they are
    read on the device, so the pruned layout is usable in the same stream at once.
    ``into``: a layout returned by an earlier call whose device arrays are rewritten.
    """
    dev = layout.cu_seqlens.device
    NI = layout.n_images
    if into is not None:
        img_start, img_len = into.img_start, into.img_len
    else:
        img_start = torch.empty(max(NI, 1), dtype=torch.int32, device=dev)
        img_len = torch.empty(max(NI, 1), dtype=torch.int32, device=dev)
    if workspace is None:
        workspace = new_workspace(workspace_size(layout), dev)
    lay = layout.c()
    _check(load().avtp_pruned_layout(ctypes.byref(lay), _ptr(budgets), _ptr(img_start), _ptr(img_len),
                                     _ptr(workspace), workspace.numel(), _stream(stream)), "avtp_pruned_layout")
    if into is not None:
        return into
    _, cu_host, nv_host = kept_count_vis_host(layout.host["cu_seqlens"], layout.n_vis_per_request, keep_ratio_host)
    host = {"cu_seqlens": cu_host, "img_cu": layout.host["img_cu"].copy(), "n_vis": nv_host}
    return Layout(cu_seqlens=out_cu_seqlens[:layout.n_requests + 1], img_cu=layout.img_cu, img_start=img_start[:NI],
                  img_len=img_len[:NI], host=host)


def kept_count_host(layout_host: Dict[str, np.ndarray], keep_ratio: np.ndarray) -> int:
    """avtp_kept_count_host: sum_r floor(r_base*N_vis + 0.5) + N_txt over requests."""
    if "n_vis" in layout_host:  # a pruned layout: image lengths on the device only
        return kept_count_vis_host(layout_host["cu_seqlens"], layout_host["n_vis"], keep_ratio)[0]
    h = {k: np.ascontiguousarray(np.asarray(layout_host[k], dtype=np.int32))
         for k in ("cu_seqlens", "img_cu", "img_len")}
    kr = np.ascontiguousarray(np.asarray(keep_ratio, dtype=np.float32))
    img_len = h["img_len"] if h["img_len"].size else np.zeros(1, dtype=np.int32)
    n = load().avtp_kept_count_host(h["cu_seqlens"].ctypes.data, h["img_cu"].ctypes.data, img_len.ctypes.data,
                                    kr.ctypes.data, int(h["cu_seqlens"].shape[0] - 1))
    if n < 0:
        raise AVTPError(ERR_INVALID_ARG, "avtp_kept_count_host")
    return int(n)


def wait_selftest(limit_ns: int, arrive: bool, workspace: torch.Tensor, stream=None) -> None:
    """Runs the bounded-wait check kernel (``avtp_wait_selftest``); read the outcome
    with :func:`read_device_status` (``ERR_TIMEOUT`` when ``arrive`` is false)."""
    _check(load().avtp_wait_selftest(int(limit_ns), 1 if arrive else 0, _ptr(workspace),
                                     workspace.numel() * workspace.element_size(), _stream(stream)),
           "avtp_wait_selftest")


def layer_attention(layout: Layout, img_sums: torch.Tensor, A: torch.Tensor, layer: int, workspace=None,
                    stream=None) -> torch.Tensor:
    """avtp_layer_attention: column ``layer`` of A (int64 [R, n_layers]) <- each request's
    sum of text-attention image sums at that layer (pruning-layer selection, §3.3.2)."""
    if A.dtype != torch.int64 or A.dim() != 2 or not A.is_contiguous() or A.shape[0] != layout.n_requests:
        raise ValueError("A must be a contiguous int64 [R, n_layers] tensor")
    if workspace is None:
        workspace = new_workspace(workspace_size(layout), A.device)
    lay = layout.c()
    _check(load().avtp_layer_attention(ctypes.byref(lay), _ptr(img_sums), _ptr(A), A.shape[1], int(layer),
                                       _ptr(workspace), workspace.numel(), _stream(stream)), "avtp_layer_attention")
    return A


def layer_select(A: torch.Tensor, k: int, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """avtp_layer_select: (rank_sum int64 [n_layers], top_layers int32 [k]) from A [N, n_layers]."""
    if A.dtype != torch.int64 or A.dim() != 2 or not A.is_contiguous():
        raise ValueError("A must be a contiguous int64 [n_samples, n_layers] tensor")
    rank_sum = torch.empty(A.shape[1], dtype=torch.int64, device=A.device)
    top = torch.empty(int(k), dtype=torch.int32, device=A.device)
    _check(load().avtp_layer_select(_ptr(A), A.shape[0], A.shape[1], int(k), _ptr(rank_sum), _ptr(top),
                                    _stream(stream)), "avtp_layer_select")
    return rank_sum, top


def read_device_status(workspace: torch.Tensor, stream=None) -> int:
    """avtp_read_device_status: waits for ``stream`` and returns the workspace's status word."""
    out = c_int32()
    _check(load().avtp_read_device_status(_ptr(workspace), _stream(stream), ctypes.byref(out)),
           "avtp_read_device_status")
    return int(out.value)


@dataclass
class PruneBuffers:
    """Every buffer one avtp_prune call touches, allocated once for a fixed layout."""
    scores: torch.Tensor
    img_sums: torch.Tensor
    budgets: torch.Tensor
    out_cu_seqlens: torch.Tensor
    kept_idx: torch.Tensor
    workspace: torch.Tensor
    outputs: Dict[str, torch.Tensor]
    n_kept: int


def prune_buffers(layout: Layout, keep_ratio_host: np.ndarray, criterion, score_tensors: Dict[str, torch.Tensor],
                  rows: Dict[str, torch.Tensor], planes: Dict[str, torch.Tensor]) -> PruneBuffers:
    """Every output buffer and the workspace of an avtp_prune call, sized on the host (no device read)."""
    dev = layout.cu_seqlens.device
    n_kept = kept_count_host(layout.host, keep_ratio_host)
    outputs = {}
    for name, src in rows.items():
        outputs[name] = torch.empty((n_kept,) + tuple(src.shape[1:]), dtype=src.dtype, device=dev)
    for name, src in planes.items():
        outputs[name] = torch.empty((src.shape[0], n_kept), dtype=src.dtype, device=dev)
    ws = new_workspace(workspace_size(layout, criterion, **score_tensors), dev)
    return PruneBuffers(
        scores=torch.zeros(layout.n_tokens, dtype=torch.float32, device=dev),
        img_sums=torch.empty(max(layout.n_images, 1), dtype=torch.int64, device=dev),
        budgets=torch.empty(max(layout.n_images, 1), dtype=torch.int32, device=dev),
        out_cu_seqlens=torch.empty(layout.n_requests + 1, dtype=torch.int32, device=dev),
        kept_idx=torch.empty(max(n_kept, 1), dtype=torch.int32, device=dev),
        workspace=ws, outputs=outputs, n_kept=n_kept)


class PruneCall:
    """A prepared avtp_prune call: C structs built once, then launched with ``run()``.

    ``rows``: name -> [T, ...] tensors gathered along dim 0; ``planes``: name ->
    [P, T] tensors (e.g. M-RoPE position ids) gathered along dim 1.
    """

    def __init__(self, layout: Layout, criterion, *, keep_ratio: torch.Tensor, keep_ratio_host: np.ndarray,
                 alpha=1.0, r_min=0.05, r_max=0.95, relative=None, rows: Optional[Dict[str, torch.Tensor]] = None,
                 planes: Optional[Dict[str, torch.Tensor]] = None, buffers: Optional[PruneBuffers] = None,
                 **score_tensors):
        rows = rows or {}
        planes = planes or {}
        if relative is None:
            crit = _CRITERIA[criterion] if isinstance(criterion, str) else int(criterion)
            relative = crit == CRIT_TEXT_ATTENTION
        self.layout = layout
        self.buffers = buffers or prune_buffers(layout, keep_ratio_host, criterion, score_tensors, rows, planes)
        b = self.buffers
        self._lay = layout.c()
        self._sa = _score_args(criterion, max_text_tokens=layout.n_text, **score_tensors)
        self._aa = _alloc_args(keep_ratio, alpha, r_min, r_max, relative)
        pairs: List[Tuple[torch.Tensor, torch.Tensor]] = []
        for name, src in rows.items():
            pairs.append((src, b.outputs[name]))
        for name, src in planes.items():
            for p in range(src.shape[0]):
                pairs.append((src[p], b.outputs[name][p]))
        self._sets, self._n_sets = _row_sets(pairs)
        self._keep_alive = (keep_ratio, rows, planes, score_tensors)

    def run(self, stream=None, step_events: Optional[Sequence] = None) -> PruneBuffers:
        """Launches the prepared avtp_prune call on ``stream``; ``step_events`` (5 CUDA events) times its steps."""
        b = self.buffers
        ev = None
        if step_events is not None:  # 5 events: start, after validation, scoring, allocation+selection, compaction
            if len(step_events) != N_STEP_EVENTS:
                raise ValueError(f"step_events needs {N_STEP_EVENTS} events")
            ev = (c_void_p * N_STEP_EVENTS)(*[int(e.cuda_event) if hasattr(e, "cuda_event") else int(e)
                                              for e in step_events])
        _check(load().avtp_prune(ctypes.byref(self._lay), ctypes.byref(self._sa), ctypes.byref(self._aa),
                                 _ptr(b.scores), _ptr(b.img_sums), _ptr(b.budgets), _ptr(b.out_cu_seqlens),
                                 _ptr(b.kept_idx), b.n_kept, self._sets, self._n_sets, _ptr(b.workspace),
                                 b.workspace.numel(), ev, _stream(stream)), "avtp_prune")
        return b


def prune(layout: Layout, criterion, *, keep_ratio: torch.Tensor, keep_ratio_host: np.ndarray, alpha=1.0,
          r_min=0.05, r_max=0.95, relative=None, rows=None, planes=None, stream=None, **score_tensors) -> PruneBuffers:
    """avtp_prune: score -> allocate -> select -> compact in one call on one stream."""
    call = PruneCall(layout, criterion, keep_ratio=keep_ratio, keep_ratio_host=keep_ratio_host, alpha=alpha,
                     r_min=r_min, r_max=r_max, relative=relative, rows=rows, planes=planes, **score_tensors)
    return call.run(stream)


# ---------------------------------------------------------------- the paged cache
def _on_one_device(where: str, *tensors: Optional[torch.Tensor]) -> torch.device:
    """The tensors' device, which has to be the current one: the library launches there."""
    dev = None
    for t in tensors:
        if t is None:
            continue
        if not t.is_cuda or (dev is not None and t.device != dev):
            raise ValueError(f"{where}: every tensor must be on one CUDA device")
        dev = t.device
    if dev.index != torch.cuda.current_device():
        raise ValueError(f"{where}: the tensors are on {dev}, the current device is another")
    return dev


def _int32(where: str, name: str, t: Optional[torch.Tensor], shape: Tuple[int, ...]) -> None:
    if t is not None and (t.dtype != torch.int32 or tuple(t.shape) != shape or (t.numel() > 1 and not t.is_contiguous())):
        raise ValueError(f"{where}: {name} must be a contiguous int32 tensor of shape {list(shape)}")


def _int32_list(where: str, name: str, t: Optional[torch.Tensor]) -> None:
    if t is None or t.dim() != 1:
        raise ValueError(f"{where}: {name} must be a contiguous int32 tensor with one dimension")
    _int32(where, name, t, tuple(t.shape))


def _block_table(where: str, t: torch.Tensor, n_requests: int) -> Tuple[int, int]:
    """(max_pages, row stride) of a block table."""
    if t.dtype != torch.int32 or t.dim() != 2 or t.shape[0] != n_requests or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{where}: block_table must be int32 [R, max_pages] with a contiguous last dim")
    return t.shape[1], t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1)


def _on_stream(stream):
    """The stream as the current one, so that buffers made for a call on it come from its memory."""
    if stream is None:
        return contextlib.nullcontext()
    return torch.cuda.stream(stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream)))


class _CacheCall:
    """A prepared call of one entry point: what ``run`` passes is made once, so that a step's call costs
    the C call and little else (2 us of 6 for a small one). Buffers that it makes (outputs, the workspace)
    belong to the stream that is current then: to run it on another, order that stream behind it, and keep
    the call until it is through."""

    def _prepare(self, name: str, workspace: torch.Tensor, *structs) -> None:
        self.workspace = workspace
        self._name = name
        self._fn = getattr(load(), name)
        self._device = workspace.device.index
        self._args = tuple(ctypes.byref(x) if isinstance(x, ctypes.Structure) else x for x in structs) + (
            c_void_p(_ptr(workspace)), c_size_t(workspace.numel() * workspace.element_size()))

    def run(self, stream=None):
        """Launches the prepared call on ``stream`` (default: the current one); returns self."""
        if torch._C._cuda_getDevice() != self._device:
            raise ValueError(f"{self._name}: prepared for device {self._device}, the current device is another")
        code = self._fn(*self._args, _stream(stream))
        if code != OK:
            raise AVTPError(code, self._name)
        return self


@dataclass
class PagedCache:
    """One layer's keys and values in pages: bf16 [n_pages, page_size, Hkv, head_dim], the last
    dimension contiguous. Pages of another order are passed as views: a head-major pool
    [n_pages, Hkv, page_size, head_dim] as ``pool.transpose(1, 2)``."""
    k: torch.Tensor
    v: torch.Tensor

    def __post_init__(self):
        k, v = self.k, self.v
        for t in (k, v):
            if t.dtype != torch.bfloat16 or t.dim() != 4 or t.stride(3) != 1 or t.shape != k.shape:
                raise ValueError("k and v must be bf16 [n_pages, page_size, Hkv, head_dim] with a contiguous last dim")
        _on_one_device("PagedCache", k, v)

    @staticmethod
    def new(n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, device="cuda") -> "PagedCache":
        """A pool of ``n_pages`` pages, not initialised."""
        shape = (int(n_pages), int(page_size), int(n_kv_heads), int(head_dim))
        return PagedCache(*(torch.empty(shape, dtype=torch.bfloat16, device=device) for _ in range(2)))

    @property
    def n_pages(self) -> int:
        return self.k.shape[0]

    @property
    def page_size(self) -> int:
        return self.k.shape[1]

    def c(self) -> _Cache:
        """The avtp_cache_t the C calls take."""
        n, p, h, d = self.k.shape

        def strides(t):  # a dimension of one entry may carry any stride: one that the others allow
            head = t.stride(2) if h > 1 else d
            token = t.stride(1) if p > 1 else (h * d if h > 1 and head == d else max(head, d))
            return (t.stride(0) if n > 1 else max(head * h, token * p), token, head)

        return _Cache(_ptr(self.k), _ptr(self.v), n, p, h, d, *strides(self.k), *strides(self.v))


class CacheSlotsCall(_CacheCall):
    """A prepared avtp_cache_slots call: block-table entries, slots and lengths of a step's new
    tokens from ``cu_new`` (int32 [R+1], for example ``out_cu_seqlens`` of a prune) and the cached
    tokens ``past_len`` (int32 [R], default none). New pages come from ``free_pages`` (int32), from
    entry ``free_head`` (int32 [1], default 0) on. ``n_tokens``: at least ``cu_new[-1]``, the length
    of ``slot_map``. ``seq_len=past_len`` and ``free_head_out=free_head`` advance them in place, so
    that replays of a captured call append step after step. A refused call (read_device_status) writes
    nothing: outputs of its own hold -1, or what an earlier run left, and a ``cache_write`` behind that
    run writes to those slots again."""

    def __init__(self, cu_new: torch.Tensor, n_tokens: int, *, page_size: int, n_pages: int, block_table: torch.Tensor,
                 free_pages: torch.Tensor, free_head=None, past_len=None, seq_len=None, slot_map=None,
                 free_head_out=None, workspace=None):
        name = "cache_slots"
        _int32_list(name, "cu_new", cu_new)
        _int32_list(name, "free_pages", free_pages)
        R = cu_new.shape[0] - 1
        max_pages, stride = _block_table(name, block_table, R)
        dev = _on_one_device(name, cu_new, block_table, free_pages, free_head, past_len, seq_len, slot_map,
                             free_head_out, workspace)
        self.block_table = block_table
        # One buffer for the outputs that are made here, -1 until a call that is not refused writes them: a slot that
        # cache_write skips, a length and a head that the next call refuses.
        made = (0 if slot_map is not None else int(n_tokens), 0 if seq_len is not None else R,
                0 if free_head_out is not None else 1)
        made = torch.full((sum(made),), -1, dtype=torch.int32, device=dev).split(made)
        self.slot_map = slot_map if slot_map is not None else made[0]
        self.seq_len = seq_len if seq_len is not None else made[1]
        self.free_head_out = free_head_out if free_head_out is not None else made[2]
        for what, t, shape in (("past_len", past_len, (R,)), ("seq_len", self.seq_len, (R,)),
                               ("slot_map", self.slot_map, (int(n_tokens),)), ("free_head", free_head, (1,)),
                               ("free_head_out", self.free_head_out, (1,))):
            _int32(name, what, t, shape)
        self._keep = (cu_new, free_pages, free_head, past_len)
        self._a = _CacheSlotsArgs(R, int(n_tokens), int(page_size), int(n_pages), max_pages, stride, _ptr(cu_new),
                                  _ptr(past_len), _ptr(free_pages), free_pages.shape[0], _ptr(free_head),
                                  _ptr(block_table), _ptr(self.seq_len), _ptr(self.slot_map), _ptr(self.free_head_out))
        if workspace is None:
            n = c_size_t()
            _check(load().avtp_cache_slots_workspace_size(ctypes.byref(self._a), ctypes.byref(n)),
                   "avtp_cache_slots_workspace_size")
            workspace = new_workspace(int(n.value), dev)
        self._prepare("avtp_cache_slots", workspace, self._a)


def cache_slots(cu_new: torch.Tensor, n_tokens: int, *, page_size: int, n_pages: int, block_table: torch.Tensor,
                free_pages: torch.Tensor, free_head=None, past_len=None, stream=None, **buffers):
    """avtp_cache_slots: (slot_map int32 [n_tokens], seq_len int32 [R], free_head int32 [1]); the new
    pages' entries go into ``block_table``. See :class:`CacheSlotsCall`."""
    with _on_stream(stream):
        c = CacheSlotsCall(cu_new, n_tokens, page_size=page_size, n_pages=n_pages, block_table=block_table,
                           free_pages=free_pages, free_head=free_head, past_len=past_len, **buffers).run()
    return c.slot_map, c.seq_len, c.free_head_out


class CacheWriteCall(_CacheCall):
    """A prepared avtp_cache_write call: row ``kept_idx[j]`` (default j) of ``k`` and ``v`` (bf16
    [n_rows, Hkv, head_dim]) to slot ``slot_map[j]`` of the cache, -1 for none."""

    def __init__(self, cache: PagedCache, slot_map: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, kept_idx=None,
                 workspace=None):
        name = "cache_write"
        _int32_list(name, "slot_map", slot_map)
        n = slot_map.shape[0]
        if kept_idx is not None:
            _int32(name, "kept_idx", kept_idx, (n,))
        h, d = cache.k.shape[2:]
        for t in (k, v):
            if (t.dtype != torch.bfloat16 or t.dim() != 3 or tuple(t.shape[1:]) != (h, d) or t.stride(2) != 1
                    or (h > 1 and t.stride(1) != d) or t.shape[0] != k.shape[0]):
                raise ValueError(f"{name}: k / v must be bf16 [n_rows, Hkv, head_dim] with contiguous heads")
        if kept_idx is None and k.shape[0] < n:
            raise ValueError(f"{name}: fewer rows than slots")
        dev = _on_one_device(name, cache.k, slot_map, k, v, kept_idx, workspace)
        self.cache = cache
        self._keep = (slot_map, k, v, kept_idx)
        self._c = cache.c()
        self._a = _CacheWriteArgs(_ptr(k), _ptr(v), k.stride(0) if k.shape[0] > 1 else h * d,
                                  v.stride(0) if v.shape[0] > 1 else h * d, k.shape[0], _ptr(kept_idx), _ptr(slot_map), n)
        self._prepare("avtp_cache_write", workspace if workspace is not None else new_workspace(256, dev), self._c,
                      self._a)


def cache_write(cache: PagedCache, slot_map: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, kept_idx=None,
                workspace=None, stream=None) -> None:
    """avtp_cache_write: K and V rows to their slots; with a prune's ``kept_idx`` only the kept ones."""
    with _on_stream(stream):
        CacheWriteCall(cache, slot_map, k, v, kept_idx=kept_idx, workspace=workspace).run()


def rope_frequencies(rot_dim: int, base: float = 10000.0, scaling: Optional[str] = None, *, factor: float = 1.0,
                     original_len: float = 0.0, slow: float = 1.0, fast: float = 32.0) -> Tuple[np.ndarray, float]:
    """avtp_rope_frequencies: (inv_freq fp32 [rot_dim / 2], attn_factor) on the host, for ``scaling`` None,
    "linear", "ntk" or "yarn". The last ramps over the pairs' turns as its paper does: a checkpoint that was run with
    a ramp over the pair's index wants its own array for :class:`RopeCall`."""
    if scaling not in _ROPE_SCALES:
        raise ValueError(f"rope_frequencies: scaling must be one of {list(_ROPE_SCALES)}")
    out = np.empty(max(int(rot_dim) // 2, 1), dtype=np.float32)
    attn = c_float()
    a = _RopeFreqArgs(int(rot_dim), _ROPE_SCALES[scaling], float(base), float(factor), float(original_len), float(slow),
                      float(fast))
    _check(load().avtp_rope_frequencies(ctypes.byref(a), out.ctypes.data_as(POINTER(c_float)), ctypes.byref(attn)),
           "avtp_rope_frequencies")
    return out, float(attn.value)


class RopeCall(_CacheCall):
    """A prepared avtp_rope call: rotary positions of ``q`` and ``k`` (bf16 [T, H, head_dim]; either may be None), behind
    their norms of each head where ``q_norm`` / ``k_norm`` (bf16 [head_dim]) are given. ``pos``: int32 [T], or
    [n_planes, T] with ``pair_plane`` (int32 [rot_dim / 2]) naming each pair's plane; ``inv_freq``: fp32 [rot_dim /
    2] (:func:`rope_frequencies`). With ``cache``, ``v`` and ``slot_map`` the keys and values go to their slots, and
    to ``k_out`` only if one is given. ``q_out`` and ``k_out`` may be ``q`` and ``k`` themselves."""

    def __init__(self, pos: Optional[torch.Tensor], inv_freq: Optional[torch.Tensor], *, q=None, k=None, v=None, q_out=None,
                 k_out=None, style="half", pair_plane=None, attn_factor=1.0, q_norm=None, k_norm=None, eps=1e-6,
                 cache: Optional[PagedCache] = None, slot_map=None, workspace=None):
        name = "rope"
        some = q if q is not None else k
        if some is None or some.dim() != 3:
            raise ValueError(f"{name}: q or k must be bf16 [T, H, head_dim] with contiguous heads")
        T, d = some.shape[0], some.shape[2]
        if (cache is None) != (slot_map is None) or (cache is None) != (v is None) or (cache is not None and k is None):
            raise ValueError(f"{name}: cache, slot_map and v go together, with k")
        dev = _on_one_device(name, pos, inv_freq, q, k, v, q_out, k_out, pair_plane, q_norm, k_norm, slot_map, workspace,
                             cache.k if cache is not None else None)
        if q is not None and q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=dev)
        if k is not None and k_out is None and cache is None:
            k_out = torch.empty(k.shape, dtype=k.dtype, device=dev)
        for what, t, like in (("q", q, q), ("q_out", q_out, q), ("k", k, k), ("k_out", k_out, k), ("v", v, k)):
            if t is None:
                continue
            if (like is None or t.dtype != torch.bfloat16 or t.dim() != 3 or tuple(t.shape) != (T, like.shape[1], d)
                    or t.stride(2) != 1 or (t.shape[1] > 1 and t.stride(1) != d)):
                raise ValueError(f"{name}: {what} must be bf16 [T, H, head_dim] with contiguous heads")
        if cache is not None and tuple(cache.k.shape[2:]) != tuple(k.shape[1:]):
            raise ValueError(f"{name}: the cache has other heads than k")
        rot = 0 if inv_freq is None else 2 * inv_freq.numel()
        planes = 1
        if rot:
            if inv_freq.dtype != torch.float32 or inv_freq.dim() != 1 or not inv_freq.is_contiguous():
                raise ValueError(f"{name}: inv_freq must be a contiguous fp32 tensor with one dimension")
            if (pos is None or pos.dtype != torch.int32 or pos.dim() not in (1, 2) or pos.shape[-1] != T
                    or (T > 1 and pos.stride(-1) != 1)):
                raise ValueError(f"{name}: pos must be int32 [T] or [n_planes, T] with a contiguous last dim")
            planes = pos.shape[0] if pos.dim() == 2 else 1
            if pair_plane is not None:
                _int32(name, "pair_plane", pair_plane, (rot // 2,))
        for what, t in (("q_norm", q_norm), ("k_norm", k_norm)):
            if t is not None and (t.dtype != torch.bfloat16 or tuple(t.shape) != (d,) or not t.is_contiguous()):
                raise ValueError(f"{name}: {what} must be a contiguous bf16 tensor of shape [head_dim]")
        if slot_map is not None:
            _int32(name, "slot_map", slot_map, (T,))
        self.q_out, self.k_out, self.cache = q_out, k_out, cache
        self._keep = (pos, inv_freq, q, k, v, pair_plane, q_norm, k_norm, slot_map)

        def stride(t):
            return 0 if t is None else (t.stride(0) if T > 1 else t.shape[1] * d)

        self._c = cache.c() if cache is not None else None
        self._a = _RopeArgs(
            T, 0 if q is None else q.shape[1], 0 if k is None else k.shape[1], d, _ptr(q), stride(q), _ptr(q_out),
            stride(q_out), _ptr(k), stride(k), _ptr(k_out), stride(k_out), _ptr(v), stride(v), _ptr(slot_map), rot,
            _ROPE_STYLES[style] if isinstance(style, str) else int(style), _ptr(inv_freq), _ptr(pos),
            pos.stride(0) if rot and planes > 1 else T, planes, _ptr(pair_plane), float(attn_factor), _ptr(q_norm),
            _ptr(k_norm), float(eps))
        self._prepare("avtp_rope", workspace if workspace is not None else new_workspace(256, dev), self._a, self._c)


def rope(pos: Optional[torch.Tensor], inv_freq: Optional[torch.Tensor], *, q=None, k=None, stream=None, **more):
    """avtp_rope: (q_out, k_out) rotated, the keys and values in the cache where one is given. See
    :class:`RopeCall`."""
    with _on_stream(stream):
        c = RopeCall(pos, inv_freq, q=q, k=k, **more).run()
    return c.q_out, c.k_out


class CacheAttentionCall(_CacheCall):
    """A prepared avtp_cache_attention call: causal attention of a step's new tokens ``q`` (bf16 [T,
    Hq, head_dim], request r's rows ``cu_new[r] .. cu_new[r+1]``, at most ``max_new`` of them) over
    the cache, where each request has ``seq_len[r]`` tokens, the new ones among them. ``o`` (bf16, as
    q) and ``lse`` (fp32 [Hq, T]; False for none) are written for those rows alone. With ``window`` each token
    sees itself, the ``window`` - 1 tokens before it and the request's first ``sinks``
    (avtp_cache_window_attention)."""

    def __init__(self, cache: PagedCache, q: torch.Tensor, cu_new: torch.Tensor, seq_len: torch.Tensor,
                 block_table: torch.Tensor, *, max_new: int, softmax_scale=None, o=None, lse=None, window=None, sinks=0,
                 workspace=None):
        name = "cache_attention"
        _int32_list(name, "cu_new", cu_new)
        R = cu_new.shape[0] - 1
        _int32(name, "seq_len", seq_len, (R,))
        max_pages, stride = _block_table(name, block_table, R)
        d = cache.k.shape[3]
        if q.dim() != 3:
            raise ValueError(f"{name}: q must be bf16 [T, Hq, head_dim] with contiguous heads")
        T, Hq = q.shape[:2]
        dev = _on_one_device(name, cache.k, q, cu_new, seq_len, block_table, o, lse if lse is not False else None,
                             workspace)
        self.o = o if o is not None else torch.empty(T, Hq, d, dtype=torch.bfloat16, device=dev)
        for what, t in (("q", q), ("o", self.o)):
            if (t.dtype != torch.bfloat16 or tuple(t.shape) != (T, Hq, d) or t.stride(2) != 1
                    or (Hq > 1 and t.stride(1) != d)):
                raise ValueError(f"{name}: {what} must be bf16 [T, Hq, head_dim] with contiguous heads")
        self.lse = None if lse is False else (lse if lse is not None
                                              else torch.empty(Hq, T, dtype=torch.float32, device=dev))
        if self.lse is not None and (self.lse.dtype != torch.float32 or tuple(self.lse.shape) != (Hq, T)
                                     or (T > 1 and self.lse.stride(1) != 1)):
            raise ValueError(f"{name}: lse must be fp32 [Hq, T] with a contiguous last dim")
        self.cache = cache
        self._keep = (q, cu_new, seq_len, block_table)
        self._c = cache.c()
        self._a = _CacheAttnArgs(
            R, T, int(max_new), Hq, _ptr(q), q.stride(0) if T > 1 else Hq * d, _ptr(cu_new), _ptr(seq_len),
            _ptr(block_table), max_pages, stride, float(softmax_scale if softmax_scale is not None else d ** -0.5),
            _ptr(self.o), self.o.stride(0) if T > 1 else Hq * d, _ptr(self.lse),
            self.lse.stride(0) if self.lse is not None and Hq > 1 else max(T, 1))
        if window is None and int(sinks) != 0:
            raise ValueError(f"{name}: sinks go with a window")
        entry = "avtp_cache_attention" if window is None else "avtp_cache_window_attention"
        structs = (self._c, self._a) if window is None else (self._c, self._a, _CacheWindow(int(window), int(sinks)))
        if workspace is None:
            n = c_size_t()
            _check(getattr(load(), entry + "_workspace_size")(*(ctypes.byref(x) for x in structs), ctypes.byref(n)),
                   entry + "_workspace_size")
            workspace = new_workspace(int(n.value), dev)
        self._prepare(entry, workspace, *structs)


def cache_attention(cache: PagedCache, q: torch.Tensor, cu_new: torch.Tensor, seq_len: torch.Tensor,
                    block_table: torch.Tensor, *, max_new: int, softmax_scale=None, o=None, lse=None, window=None, sinks=0,
                    workspace=None, stream=None):
    """avtp_cache_attention, or with ``window`` avtp_cache_window_attention: (o, lse) of a chunk of new tokens, or a
    single one, a request over the paged cache. See :class:`CacheAttentionCall`."""
    with _on_stream(stream):
        c = CacheAttentionCall(cache, q, cu_new, seq_len, block_table, max_new=max_new, softmax_scale=softmax_scale,
                               o=o, lse=lse, window=window, sinks=sinks, workspace=workspace).run()
    return c.o, c.lse


# ---------------------------------------------------------------- upkeep of the pages
def _window(where: str, window: int, sinks: int, n_requests: int, held_len: Optional[torch.Tensor]) -> Tuple[int, int]:
    if int(window) > 0 and held_len is None:
        raise ValueError(f"{where}: a window goes with held_len")
    _int32(where, "held_len", held_len, (n_requests,))
    return int(window), int(sinks)


class CacheCompactCall(_CacheCall):
    """A prepared avtp_cache_compact call: the kept tokens of cached requests moved together in one layer's cache, to
    the pages of ``dst_table`` (int32 [R, columns]) or, without one, in place. ``keep_idx`` (int32): request r's kept
    positions at ``keep_cu[r] .. keep_cu[r+1]``, less ``base_cu[r]`` where that is given (a prune's ``kept_idx``,
    ``out_cu_seqlens`` and the batch's ``cu_seqlens``). ``len_out`` (int32 [R]) receives the kept tokens, or in place
    the whole length of a request that is refused and left as it was; the pages behind them go back with
    :class:`CacheFreeCall`. ``shared``, ``window``, ``sinks`` and ``held_len``: as there."""

    def __init__(self, cache: PagedCache, keep_cu: torch.Tensor, keep_idx: torch.Tensor, seq_len: torch.Tensor,
                 block_table: torch.Tensor, *, dst_table=None, base_cu=None, shared=None, window=0, sinks=0, held_len=None,
                 len_out=None, workspace=None):
        name = "cache_compact"
        _int32_list(name, "keep_cu", keep_cu)
        _int32_list(name, "keep_idx", keep_idx)
        R = keep_cu.shape[0] - 1
        max_pages, stride = _block_table(name, block_table, R)
        dst = _block_table(name, dst_table, R) if dst_table is not None else (0, 0)
        dev = _on_one_device(name, cache.k, keep_cu, keep_idx, seq_len, block_table, dst_table, base_cu, shared, held_len,
                             len_out, workspace)
        self.len_out = len_out if len_out is not None else torch.full((R,), -1, dtype=torch.int32, device=dev)
        if base_cu is not None:  # a batch's offsets: R of them, or with its end
            _int32_list(name, "base_cu", base_cu)
            if base_cu.shape[0] not in (R, R + 1):
                raise ValueError(f"{name}: base_cu must have an offset a request")
        for what, t, n in (("seq_len", seq_len, R), ("len_out", self.len_out, R), ("shared", shared, cache.n_pages)):
            _int32(name, what, t, (n,))
        window, sinks = _window(name, window, sinks, R, held_len)
        self.cache = cache
        self._keep = (keep_cu, keep_idx, seq_len, block_table, dst_table, base_cu, shared, held_len)
        self._c = cache.c()
        self._a = _CacheCompactArgs(R, keep_idx.shape[0], _ptr(keep_cu), _ptr(keep_idx), _ptr(base_cu), _ptr(seq_len),
                                    _ptr(block_table), max_pages, stride, _ptr(dst_table), *dst, _ptr(shared), window, sinks,
                                    _ptr(held_len), _ptr(self.len_out))
        self._prepare("avtp_cache_compact", workspace if workspace is not None else new_workspace(256, dev), self._c,
                      self._a)


def cache_compact(cache: PagedCache, keep_cu: torch.Tensor, keep_idx: torch.Tensor, seq_len: torch.Tensor,
                  block_table: torch.Tensor, *, stream=None, **more) -> torch.Tensor:
    """avtp_cache_compact: kept tokens together; returns the new lengths (int32 [R]). See :class:`CacheCompactCall`."""
    with _on_stream(stream):
        return CacheCompactCall(cache, keep_cu, keep_idx, seq_len, block_table, **more).run().len_out


class CacheCopyCall(_CacheCall):
    """A prepared avtp_cache_copy call: pages ``src[i]`` to pages ``dst[i]`` (int32; -1 in either: none) of one
    layer's cache."""

    def __init__(self, cache: PagedCache, src: torch.Tensor, dst: torch.Tensor, *, workspace=None):
        name = "cache_copy"
        _int32_list(name, "src", src)
        _int32(name, "dst", dst, tuple(src.shape))
        dev = _on_one_device(name, cache.k, src, dst, workspace)
        self.cache = cache
        self._keep = (src, dst)
        self._c = cache.c()
        self._prepare("avtp_cache_copy", workspace if workspace is not None else new_workspace(256, dev), self._c,
                      c_void_p(_ptr(src)), c_void_p(_ptr(dst)), c_int64(src.shape[0]))


def cache_copy(cache: PagedCache, src: torch.Tensor, dst: torch.Tensor, *, workspace=None, stream=None) -> None:
    """avtp_cache_copy: whole pages to other pages. See :class:`CacheCopyCall`."""
    with _on_stream(stream):
        CacheCopyCall(cache, src, dst, workspace=workspace).run()


class CacheForkCall(_CacheCall):
    """A prepared avtp_cache_fork call: rows ``child`` of ``block_table`` and ``seq_len`` go on from the cached tokens
    of rows ``parent`` (int32 [C] each), or the first ``fork_len`` of them. Full pages are shared (``shared``, int32
    [n_pages], zeros at first, counts the holders beyond the first); a last page that is not full is to be copied,
    from ``copy_src`` to ``copy_dst`` (:class:`CacheCopyCall`, once a layer), to a page of the free list. A
    refused call (read_device_status) writes nothing: copy lists of its own then hold -1."""

    def __init__(self, parent: torch.Tensor, child: torch.Tensor, seq_len: torch.Tensor, block_table: torch.Tensor, *,
                 page_size: int, n_pages: int, free_pages: torch.Tensor, shared: torch.Tensor, free_head=None, fork_len=None,
                 window=0, sinks=0, held_len=None, copy_src=None, copy_dst=None, free_head_out=None, workspace=None):
        name = "cache_fork"
        _int32_list(name, "parent", parent)
        _int32_list(name, "free_pages", free_pages)
        _int32_list(name, "seq_len", seq_len)
        C, R = parent.shape[0], seq_len.shape[0]
        max_pages, stride = _block_table(name, block_table, R)
        dev = _on_one_device(name, parent, child, seq_len, block_table, free_pages, shared, free_head, fork_len, held_len,
                             copy_src, copy_dst, free_head_out, workspace)
        made = torch.full((2 * C + 1,), -1, dtype=torch.int32, device=dev).split([C, C, 1])
        self.copy_src = copy_src if copy_src is not None else made[0]
        self.copy_dst = copy_dst if copy_dst is not None else made[1]
        self.free_head_out = free_head_out if free_head_out is not None else made[2]
        if shared is None:
            raise ValueError(f"{name}: shared is needed")
        for what, t, n in (("child", child, C), ("fork_len", fork_len, C), ("copy_src", self.copy_src, C),
                           ("copy_dst", self.copy_dst, C), ("shared", shared, int(n_pages)), ("free_head", free_head, 1),
                           ("free_head_out", self.free_head_out, 1)):
            _int32(name, what, t, (n,))
        window, sinks = _window(name, window, sinks, R, held_len)
        self.block_table, self.seq_len = block_table, seq_len
        self._keep = (parent, child, free_pages, shared, free_head, fork_len, held_len)
        self._a = _CacheForkArgs(R, C, int(page_size), int(n_pages), max_pages, stride, _ptr(parent), _ptr(child),
                                 _ptr(fork_len), _ptr(free_pages), free_pages.shape[0], _ptr(free_head), _ptr(block_table),
                                 _ptr(seq_len), _ptr(shared), window, sinks, _ptr(held_len), _ptr(self.copy_src),
                                 _ptr(self.copy_dst), _ptr(self.free_head_out))
        if workspace is None:
            n = c_size_t()
            _check(load().avtp_cache_fork_workspace_size(ctypes.byref(self._a), ctypes.byref(n)),
                   "avtp_cache_fork_workspace_size")
            workspace = new_workspace(int(n.value), dev)
        self._prepare("avtp_cache_fork", workspace, self._a)


def cache_fork(parent: torch.Tensor, child: torch.Tensor, seq_len: torch.Tensor, block_table: torch.Tensor, *, stream=None,
               **more):
    """avtp_cache_fork: (copy_src, copy_dst, free_head). See :class:`CacheForkCall`."""
    with _on_stream(stream):
        c = CacheForkCall(parent, child, seq_len, block_table, **more).run()
    return c.copy_src, c.copy_dst, c.free_head_out


class CacheFreeCall(_CacheCall):
    """A prepared avtp_cache_free call: requests go from ``seq_len`` to ``new_len`` tokens (int32 [R]; 0: done) and the
    pages that they need no more go back to ``free_pages``, before its entry ``free_head``. With ``shared``
    (:class:`CacheForkCall`) a page goes back with its last holder. With ``window`` (and ``sinks``, ``held_len`` int32
    [R], zeros at first) what a sliding window has left goes back too. ``seq_len_out=seq_len``,
    ``held_len_out=held_len`` and ``free_head_out=free_head`` advance them in place. A refused call
    (read_device_status) writes nothing: outputs of its own then hold -1."""

    def __init__(self, seq_len: torch.Tensor, new_len: torch.Tensor, block_table: torch.Tensor, *, page_size: int,
                 n_pages: int, free_pages: torch.Tensor, free_head: torch.Tensor, shared=None, window=0, sinks=0,
                 held_len=None, seq_len_out=None, held_len_out=None, free_head_out=None, workspace=None):
        name = "cache_free"
        _int32_list(name, "seq_len", seq_len)
        _int32_list(name, "free_pages", free_pages)
        _int32_list(name, "free_head", free_head)
        R = seq_len.shape[0]
        max_pages, stride = _block_table(name, block_table, R)
        dev = _on_one_device(name, seq_len, new_len, block_table, free_pages, free_head, shared, held_len, seq_len_out,
                             held_len_out, free_head_out, workspace)
        window, sinks = _window(name, window, sinks, R, held_len)
        made = torch.full((2 * R + 1,), -1, dtype=torch.int32, device=dev).split([R, R, 1])
        self.seq_len_out = seq_len_out if seq_len_out is not None else made[0]
        self.held_out = None if not window else (held_len_out if held_len_out is not None else made[1])
        self.free_head_out = free_head_out if free_head_out is not None else made[2]
        self.free_pages = free_pages
        for what, t, n in (("new_len", new_len, R), ("seq_len_out", self.seq_len_out, R), ("held_len_out", self.held_out, R),
                           ("shared", shared, int(n_pages)), ("free_head", free_head, 1),
                           ("free_head_out", self.free_head_out, 1)):
            _int32(name, what, t, (n,))
        self._keep = (seq_len, new_len, block_table, free_head, shared, held_len)
        self._a = _CacheFreeArgs(R, int(page_size), int(n_pages), max_pages, stride, _ptr(seq_len), _ptr(new_len),
                                 _ptr(block_table), _ptr(free_pages), free_pages.shape[0], _ptr(free_head), _ptr(shared),
                                 window, sinks, _ptr(held_len), _ptr(self.seq_len_out), _ptr(self.held_out),
                                 _ptr(self.free_head_out))
        if workspace is None:
            n = c_size_t()
            _check(load().avtp_cache_free_workspace_size(ctypes.byref(self._a), ctypes.byref(n)),
                   "avtp_cache_free_workspace_size")
            workspace = new_workspace(int(n.value), dev)
        self._prepare("avtp_cache_free", workspace, self._a)


def cache_free(seq_len: torch.Tensor, new_len: torch.Tensor, block_table: torch.Tensor, *, stream=None, **more):
    """avtp_cache_free: (seq_len, free_head), the pages in ``free_pages``. See :class:`CacheFreeCall`."""
    with _on_stream(stream):
        c = CacheFreeCall(seq_len, new_len, block_table, **more).run()
    return c.seq_len_out, c.free_head_out
