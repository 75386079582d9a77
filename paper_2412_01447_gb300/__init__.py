"""PLD+ drafting and greedy verification on GB300 (sm_103a).

Python binding of the C ABI in ``include/pldp.h``.  Every function here only
marshals torch tensors (device pointers, sizes, the current CUDA stream) into
the library call of the same name; all the work runs in the CUDA kernels of
``libpldp.so``.  There is no CPU fallback: if the library is missing the calls
raise.

PLD+ (arXiv 2412.01447), per decode step and per sequence:
  * ``pldp_find_candidates`` -- Eq. 1 (Sec. 4.2): earlier occurrences of the last
    token, narrowed to the longest matching suffix n-gram;
  * ``pldp_rank_hidden``     -- Eq. 3 (Sec. 4.2.2): cosine of hidden states;
  * ``pldp_rank_attention``  -- Eq. 2 (Sec. 4.2.1): max attention of selected heads;
  * ``pldp_extract_draft``   -- Sec. 4.3: the K tokens after the best occurrence;
  * ``pldp_verify_greedy``   -- Sec. 4.4: greedy accept against the target argmax;
  * ``pldp_verify_sample``   -- Sec. 4.4 with sampling, from caller uniforms.
The fused calls: ``pldp_draft_step`` (the first four in one, optionally
with the token index of ``pldp_index_build``), ``pldp_verify_greedy_draft`` and
``pldp_verify_sample_draft`` (verification, greedy or by sampling, then the next
step's draft).  Also ``pldp_rank_hidden_avg``
(App. B.2) and ``pldp_identify_heads`` / ``pldp_top_heads`` (Sec. 4.2.1).

Around the target model's forward pass over x_t and the draft, on a paged cache
(class ``pldp_cache``): ``pldp_cache_append``, ``pldp_attend_cache``,
``pldp_rank_cache`` (Eq. 2 from the cache), ``pldp_cache_read``; and
``pldp_token_logprobs`` on its logits.  Prompts of different lengths, packed:
``pldp_cache_append_prompt``, ``pldp_attend_prompt``.  The cache's pages (class
``pldp_page_table``): ``pldp_pages_reserve``, ``pldp_pages_fork``, ``pldp_pages_free``,
``pldp_pages_compact``, ``pldp_cache_copy_pages``.

The marshalling of the calls a decode step makes is native as well
(``csrc/host_calls.cpp``), with the Python below as its wording of errors.

Device buffers are passed as raw pointers, so the binding checks what the C
side cannot: every tensor is a CUDA tensor of the stated dtype, dense where
the call wants it, and holds at least the elements the call will touch.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
import threading
import warnings

import torch

from . import _build

__all__ = [
    "build", "library_path", "PldpError",
    "PLDP_F32", "PLDP_BF16", "PLDP_E4M3", "PLDP_AGG_MAX", "PLDP_AGG_SUM",
    "PLDP_ST_CAND_OVERFLOW", "PLDP_ST_TOKEN_RANGE", "PLDP_ST_CAPACITY", "PLDP_ST_SEQ_LEN",
    "PLDP_ST_DRAFT_LEN", "PLDP_ST_ROW_INDEX", "PLDP_ST_TIMEOUT", "PLDP_ST_PAGE",
    "PLDP_OK", "PLDP_ERR_INVALID_ARG", "PLDP_ERR_UNSUPPORTED", "PLDP_ERR_CUDA", "PLDP_ERR_TIMEOUT",
    "pldp_find_candidates", "pldp_rank_hidden", "pldp_rank_attention", "pldp_extract_draft",
    "pldp_verify_greedy", "pldp_verify_workspace_size", "pldp_verify_greedy_noalloc",
    "pldp_verify_sample", "pldp_verify_sample_workspace_size",
    "pldp_draft_step", "pldp_draft_step_args", "pldp_draft_workspace_size",
    "pldp_index_size", "pldp_index_build",
    "pldp_verify_greedy_draft", "pldp_verify_draft_args",
    "pldp_verify_sample_draft", "pldp_verify_sample_draft_args", "pldp_verify_sample_draft_workspace_size",
    "pldp_rank_hidden_avg", "pldp_identify_heads", "pldp_top_heads",
    "pldp_cache", "pldp_cache_args", "pldp_cache_append", "pldp_cache_append_args", "pldp_cache_read",
    "pldp_cache_read_args", "pldp_attend_cache", "pldp_attend_args", "pldp_attend_workspace_size",
    "pldp_rank_cache", "pldp_rank_cache_args", "pldp_token_logprobs", "pldp_token_logprobs_workspace_size",
    "pldp_cache_append_prompt", "pldp_cache_append_prompt_args", "pldp_attend_prompt", "pldp_attend_prompt_args",
    "pldp_attend_prompt_workspace_size", "pldp_page_table", "pldp_page_table_args", "pldp_pages_workspace_size",
    "pldp_pages_reserve", "pldp_pages_fork", "pldp_pages_free", "pldp_pages_compact", "pldp_cache_copy_pages",
    "pldp_version", "pldp_last_error",
]

PLDP_F32, PLDP_BF16, PLDP_E4M3 = 0, 1, 2
PLDP_AGG_MAX, PLDP_AGG_SUM = 0, 1
PLDP_ST_CAND_OVERFLOW = 1
PLDP_ST_TOKEN_RANGE = 2
PLDP_ST_CAPACITY = 4
PLDP_ST_SEQ_LEN = 8
PLDP_ST_DRAFT_LEN = 16
PLDP_ST_ROW_INDEX = 32
PLDP_ST_TIMEOUT = 64
PLDP_ST_PAGE = 128

PLDP_OK = 0
PLDP_ERR_INVALID_ARG = 1
PLDP_ERR_UNSUPPORTED = 2
PLDP_ERR_CUDA = 3
PLDP_ERR_TIMEOUT = 4

_STATUS_NAMES = {1: "PLDP_ERR_INVALID_ARG", 2: "PLDP_ERR_UNSUPPORTED", 3: "PLDP_ERR_CUDA",
                 4: "PLDP_ERR_TIMEOUT"}


class PldpError(RuntimeError):
    def __init__(self, fn, code, msg):
        super().__init__(f"{fn}: {_STATUS_NAMES.get(code, code)}: {msg}")
        self.code = code


_lock = threading.Lock()
_lib = None
_calls = None            # the native checks and marshalling (csrc/host_calls.cpp), once loaded


class pldp_draft_step_args(ctypes.Structure):
    """Mirror of the C argument block of pldp_draft_step (include/pldp.h)."""
    _fields_ = [
        ("ids", ctypes.c_void_p), ("ids_stride", ctypes.c_int64), ("seq_len", ctypes.c_void_p),
        ("B", ctypes.c_int), ("T_cap", ctypes.c_int64), ("ngram_min", ctypes.c_int),
        ("ngram_max", ctypes.c_int), ("cand_pos", ctypes.c_void_p), ("C_cap", ctypes.c_int),
        ("cand_count", ctypes.c_void_p), ("match_len", ctypes.c_void_p),
        ("H", ctypes.c_void_p), ("h_dtype", ctypes.c_int), ("d", ctypes.c_int64),
        ("h_seq_stride", ctypes.c_int64), ("threshold", ctypes.c_float), ("h_scores", ctypes.c_void_p),
        ("best_h", ctypes.c_void_p), ("best_h_score", ctypes.c_void_p),
        ("A", ctypes.c_void_p), ("a_dtype", ctypes.c_int), ("R", ctypes.c_int),
        ("a_row_stride", ctypes.c_int64), ("a_key_stride", ctypes.c_int64), ("a_seq_stride", ctypes.c_int64),
        ("row_idx", ctypes.c_void_p),
        ("n_sel", ctypes.c_int), ("agg", ctypes.c_int), ("a_scores", ctypes.c_void_p),
        ("best_a", ctypes.c_void_p), ("best_a_score", ctypes.c_void_p),
        ("draft_from", ctypes.c_int), ("K", ctypes.c_int), ("draft", ctypes.c_void_p),
        ("draft_len", ctypes.c_void_p), ("status", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
        ("index", ctypes.c_void_p), ("index_bytes", ctypes.c_size_t), ("V", ctypes.c_int),
    ]


class pldp_verify_sample_draft_args(ctypes.Structure):
    """Mirror of the C argument block of pldp_verify_sample_draft (include/pldp.h)."""
    _fields_ = [
        ("logits", ctypes.c_void_p), ("dtype", ctypes.c_int), ("V", ctypes.c_int),
        ("temperature", ctypes.c_float), ("uniforms", ctypes.c_void_p),
        ("draft", ctypes.c_void_p), ("draft_len", ctypes.c_void_p), ("sampled", ctypes.c_void_p),
        ("accept_len", ctypes.c_void_p), ("next_token", ctypes.c_void_p), ("kv_keep_len", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t), ("next", pldp_draft_step_args),
    ]


class pldp_verify_draft_args(ctypes.Structure):
    """Mirror of the C argument block of pldp_verify_greedy_draft (include/pldp.h)."""
    _fields_ = [
        ("logits", ctypes.c_void_p), ("dtype", ctypes.c_int), ("V", ctypes.c_int),
        ("draft", ctypes.c_void_p), ("draft_len", ctypes.c_void_p), ("argmax", ctypes.c_void_p),
        ("accept_len", ctypes.c_void_p), ("next_token", ctypes.c_void_p), ("kv_keep_len", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t), ("next", pldp_draft_step_args),
    ]


class pldp_cache_args(ctypes.Structure):
    """Mirror of the C description of a paged cache, pldp_cache (include/pldp.h)."""
    _fields_ = [
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("dtype", ctypes.c_int),
        ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
        ("n_pages", ctypes.c_int), ("page_size", ctypes.c_int), ("heads", ctypes.c_int), ("head_dim", ctypes.c_int),
        ("page_stride", ctypes.c_int64), ("pos_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
        ("pages", ctypes.c_void_p), ("pages_stride", ctypes.c_int64), ("max_pages", ctypes.c_int),
    ]


_STRIDES = ctypes.c_int64 * 3


class pldp_cache_append_args(ctypes.Structure):
    """Mirror of the C argument block of pldp_cache_append (include/pldp.h)."""
    _fields_ = [
        ("cache", pldp_cache_args), ("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("dtype", ctypes.c_int), ("B", ctypes.c_int), ("n", ctypes.c_int), ("q_heads", ctypes.c_int),
        ("q_strides", _STRIDES), ("k_strides", _STRIDES), ("v_strides", _STRIDES),
        ("q_norm", ctypes.c_void_p), ("k_norm", ctypes.c_void_p), ("eps", ctypes.c_float),
        ("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p), ("rot", ctypes.c_int), ("interleaved", ctypes.c_int),
        ("rot_rows", ctypes.c_int64), ("seq_len", ctypes.c_void_p), ("draft_len", ctypes.c_void_p),
        ("q_out", ctypes.c_void_p), ("q_out_strides", _STRIDES), ("status", ctypes.c_void_p),
    ]


class pldp_cache_read_args(ctypes.Structure):
    """Mirror of the C argument block of pldp_cache_read (include/pldp.h)."""
    _fields_ = [
        ("cache", pldp_cache_args), ("start", ctypes.c_void_p), ("count", ctypes.c_void_p), ("B", ctypes.c_int),
        ("n", ctypes.c_int), ("dtype", ctypes.c_int), ("k_out", ctypes.c_void_p), ("v_out", ctypes.c_void_p),
        ("out_strides", _STRIDES), ("status", ctypes.c_void_p),
    ]


class pldp_attend_args(ctypes.Structure):
    """Mirror of the C argument block of pldp_attend_cache (include/pldp.h)."""
    _fields_ = [
        ("cache", pldp_cache_args), ("q", ctypes.c_void_p), ("B", ctypes.c_int), ("n", ctypes.c_int),
        ("q_heads", ctypes.c_int), ("q_strides", _STRIDES), ("seq_len", ctypes.c_void_p),
        ("draft_len", ctypes.c_void_p), ("scale", ctypes.c_float), ("out", ctypes.c_void_p),
        ("out_strides", _STRIDES), ("lse", ctypes.c_void_p), ("status", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
    ]


class pldp_rank_cache_args(ctypes.Structure):
    """Mirror of the C argument block of pldp_rank_cache (include/pldp.h)."""
    _fields_ = [
        ("cache", pldp_cache_args), ("q", ctypes.c_void_p), ("B", ctypes.c_int), ("n", ctypes.c_int),
        ("q_heads", ctypes.c_int), ("q_strides", _STRIDES), ("row", ctypes.c_void_p), ("kv_len", ctypes.c_void_p),
        ("lse", ctypes.c_void_p), ("heads", ctypes.c_void_p), ("n_sel", ctypes.c_int), ("agg", ctypes.c_int),
        ("accumulate", ctypes.c_int), ("scale", ctypes.c_float), ("cand_pos", ctypes.c_void_p),
        ("cand_count", ctypes.c_void_p), ("C_cap", ctypes.c_int), ("scores", ctypes.c_void_p),
        ("best_pos", ctypes.c_void_p), ("best_score", ctypes.c_void_p), ("status", ctypes.c_void_p),
    ]


_ROW_STRIDES = ctypes.c_int64 * 2


class pldp_cache_append_prompt_args(ctypes.Structure):
    """Mirror of the C argument block of pldp_cache_append_prompt (include/pldp.h)."""
    _fields_ = [
        ("cache", pldp_cache_args), ("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("dtype", ctypes.c_int), ("B", ctypes.c_int), ("R", ctypes.c_int), ("q_heads", ctypes.c_int),
        ("q_strides", _ROW_STRIDES), ("k_strides", _ROW_STRIDES), ("v_strides", _ROW_STRIDES),
        ("q_norm", ctypes.c_void_p), ("k_norm", ctypes.c_void_p), ("eps", ctypes.c_float),
        ("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p), ("rot", ctypes.c_int), ("interleaved", ctypes.c_int),
        ("rot_rows", ctypes.c_int64), ("rows", ctypes.c_void_p), ("start", ctypes.c_void_p),
        ("q_out", ctypes.c_void_p), ("q_out_strides", _ROW_STRIDES), ("status", ctypes.c_void_p),
    ]


class pldp_attend_prompt_args(ctypes.Structure):
    """Mirror of the C argument block of pldp_attend_prompt (include/pldp.h)."""
    _fields_ = [
        ("cache", pldp_cache_args), ("q", ctypes.c_void_p), ("B", ctypes.c_int), ("R", ctypes.c_int),
        ("q_heads", ctypes.c_int), ("q_strides", _ROW_STRIDES), ("rows", ctypes.c_void_p), ("start", ctypes.c_void_p),
        ("scale", ctypes.c_float), ("out", ctypes.c_void_p), ("out_strides", _ROW_STRIDES), ("lse", ctypes.c_void_p),
        ("status", ctypes.c_void_p), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
    ]


class pldp_page_table_args(ctypes.Structure):
    """Mirror of the C description of a page table, pldp_page_table (include/pldp.h)."""
    _fields_ = [
        ("pages", ctypes.c_void_p), ("pages_stride", ctypes.c_int64), ("B", ctypes.c_int), ("max_pages", ctypes.c_int),
        ("page_size", ctypes.c_int), ("refs", ctypes.c_void_p), ("n_pages", ctypes.c_int),
    ]


def library_path() -> str:
    return _build.LIB


def build(force: bool = False) -> str:
    """Compile libpldp.so for sm_103a (in-tree) if it is missing or stale."""
    return _build.build(force=force)


# The entry points _calls makes, in the order of its `Library`.
_CALLS = ("pldp_find_candidates", "pldp_rank_hidden", "pldp_rank_attention", "pldp_extract_draft", "pldp_draft_step",
          "pldp_index_build", "pldp_verify_greedy", "pldp_verify_greedy_draft", "pldp_verify_sample",
          "pldp_verify_sample_draft", "pldp_identify_heads", "pldp_top_heads")


# ... and of its `CacheLibrary`.
_CACHE_CALLS = ("pldp_cache_append", "pldp_cache_read", "pldp_attend_cache", "pldp_rank_cache", "pldp_token_logprobs")

# ... and of its `PromptLibrary`.
_PROMPT_CALLS = ("pldp_cache_append_prompt", "pldp_attend_prompt", "pldp_pages_reserve", "pldp_pages_fork", "pldp_pages_free",
                 "pldp_pages_compact", "pldp_cache_copy_pages")


def _load_calls(lib):
    """The native form of the calls below, bound to the loaded library.  Each takes a
    call's arguments, makes its checks and returns the library's status, or None when a
    check does not pass or an argument is of a kind it does not handle; the Python that
    follows then does the same and words the error."""
    path = _build.calls_path()
    if not os.path.exists(path):
        return None
    try:
        spec = importlib.util.spec_from_file_location("_pldp_calls", path)
        m = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(m)
        m.bind(tuple(ctypes.cast(getattr(lib, f), ctypes.c_void_p).value for f in _CALLS))
        m.bind_cache(tuple(ctypes.cast(getattr(lib, f), ctypes.c_void_p).value for f in _CACHE_CALLS))
        m.bind_prompt(tuple(ctypes.cast(getattr(lib, f), ctypes.c_void_p).value for f in _PROMPT_CALLS))
    except Exception as e:                               # the Python below makes every call by itself
        warnings.warn(f"{os.path.basename(path)} does not load, the binding's calls go through ctypes: {e}",
                      RuntimeWarning, stacklevel=2)
        return None
    return m


def _load():
    global _lib, _calls
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(_build.LIB):
                raise RuntimeError("libpldp.so is not built: call paper_2412_01447_gb300.build() "
                                   "(needs nvcc); there is no CPU fallback")
            lib = ctypes.CDLL(_build.LIB)
            P, i32, i64, f32, sz = (ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float,
                                    ctypes.c_size_t)
            lib.pldp_find_candidates.argtypes = [P, i64, P, i32, i64, i32, i32, P, i32, P, P, P, P]
            lib.pldp_rank_hidden.argtypes = [P, i32, i64, i64, P, i32, i64, P, P, i32, f32, P, P, P,
                                             P, P]
            lib.pldp_identify_heads.argtypes = [P, i64, P, i32, i64, i32, P, i32, i32, i64, i64, P, P, P, P]
            lib.pldp_identify_heads.restype = ctypes.c_int
            lib.pldp_top_heads.argtypes = [P, i32, i32, P, P]
            lib.pldp_top_heads.restype = ctypes.c_int
            lib.pldp_rank_hidden_avg.argtypes = [P, i32, i64, i64, i32, P, i32, i64, P, P, i32, f32, P, P,
                                                 P, P, P]
            lib.pldp_rank_hidden_avg.restype = ctypes.c_int
            lib.pldp_rank_attention.argtypes = [P, i32, i32, i64, i64, i64, P, i32, i32, P, i32, i64, P,
                                                P, i32, P, P, P, P, P]
            lib.pldp_extract_draft.argtypes = [P, i64, P, i64, P, i32, i32, P, P, P]
            lib.pldp_verify_greedy.argtypes = [P, i32, i32, i32, i32, P, P, P, P, P, P, i64, P, i64,
                                               P, P, P, sz, P]
            for f in ("pldp_find_candidates", "pldp_rank_hidden", "pldp_rank_attention",
                      "pldp_extract_draft", "pldp_verify_greedy"):
                getattr(lib, f).restype = ctypes.c_int
            lib.pldp_draft_step.argtypes = [ctypes.POINTER(pldp_draft_step_args), P]
            lib.pldp_draft_step.restype = ctypes.c_int
            lib.pldp_verify_greedy_draft.argtypes = [ctypes.POINTER(pldp_verify_draft_args), P]
            lib.pldp_verify_greedy_draft.restype = ctypes.c_int
            lib.pldp_verify_sample_draft.argtypes = [ctypes.POINTER(pldp_verify_sample_draft_args), P]
            lib.pldp_verify_sample_draft.restype = ctypes.c_int
            lib.pldp_verify_sample_draft_workspace_size.argtypes = [i32, i32, i32, i32]
            lib.pldp_verify_sample_draft_workspace_size.restype = sz
            lib.pldp_draft_workspace_size.argtypes = [i32]
            lib.pldp_draft_workspace_size.restype = sz
            lib.pldp_index_size.argtypes = [i32, i32]
            lib.pldp_index_size.restype = sz
            lib.pldp_index_build.argtypes = [P, i64, P, i32, i64, i32, P, sz, P, P]
            lib.pldp_index_build.restype = ctypes.c_int
            lib.pldp_verify_greedy_noalloc.argtypes = [P, i32, i32, i32, i32, P, P, P, P, P, P, i64,
                                                       P, i64, P, P, P]
            lib.pldp_verify_greedy_noalloc.restype = ctypes.c_int
            lib.pldp_verify_workspace_size.argtypes = [i32, i32, i32]
            lib.pldp_verify_workspace_size.restype = sz
            lib.pldp_verify_sample.argtypes = [P, i32, i32, i32, i32, f32, P, P, P, P, P, P, P, i64, P,
                                               i64, P, P, P, sz, P]
            lib.pldp_verify_sample.restype = ctypes.c_int
            lib.pldp_verify_sample_workspace_size.argtypes = [i32, i32, i32, i32]
            lib.pldp_verify_sample_workspace_size.restype = sz
            for f, block in (("pldp_cache_append", pldp_cache_append_args), ("pldp_cache_read", pldp_cache_read_args),
                             ("pldp_attend_cache", pldp_attend_args), ("pldp_rank_cache", pldp_rank_cache_args),
                             ("pldp_cache_append_prompt", pldp_cache_append_prompt_args),
                             ("pldp_attend_prompt", pldp_attend_prompt_args)):
                getattr(lib, f).argtypes = [ctypes.POINTER(block), P]
                getattr(lib, f).restype = ctypes.c_int
            lib.pldp_attend_workspace_size.argtypes = [i32, i32, i32, i32, i32]
            lib.pldp_attend_workspace_size.restype = sz
            lib.pldp_token_logprobs.argtypes = [P, i32, i64, i32, f32, P, P, P, i32, P, P, P, sz, P]
            lib.pldp_token_logprobs.restype = ctypes.c_int
            lib.pldp_token_logprobs_workspace_size.argtypes = [i64, i32]
            lib.pldp_token_logprobs_workspace_size.restype = sz
            lib.pldp_attend_prompt_workspace_size.argtypes = [i32, i32, i32]
            lib.pldp_attend_prompt_workspace_size.restype = sz
            table = ctypes.POINTER(pldp_page_table_args)
            lib.pldp_pages_workspace_size.argtypes = [i32, i32, i32]
            lib.pldp_pages_workspace_size.restype = sz
            lib.pldp_pages_reserve.argtypes = [table, P, P, i32, P, P, P, sz, P]
            lib.pldp_pages_fork.argtypes = [table, P, P, P, P]
            lib.pldp_pages_free.argtypes = [table, P, P]
            lib.pldp_pages_compact.argtypes = [table, P, i32, P, P, P, sz, P]
            lib.pldp_cache_copy_pages.argtypes = [ctypes.POINTER(pldp_cache_args), P, i32, P, P]
            for f in ("pldp_pages_reserve", "pldp_pages_fork", "pldp_pages_free", "pldp_pages_compact", "pldp_cache_copy_pages"):
                getattr(lib, f).restype = ctypes.c_int
            lib.pldp_last_error.argtypes = []
            lib.pldp_last_error.restype = ctypes.c_char_p
            lib.pldp_version.argtypes = []
            lib.pldp_version.restype = ctypes.c_int
            _calls = _load_calls(lib)
            _lib = lib
    return _lib


# ----------------------------------------------------------------------------
# marshalling helpers
# ----------------------------------------------------------------------------
def _stream(stream):
    if stream is None:
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    if isinstance(stream, torch.cuda.Stream):
        return ctypes.c_void_p(stream.cuda_stream)
    return ctypes.c_void_p(int(stream))


def _dev(t, name, dtype=None, allow_none=False):
    if t is None:
        if allow_none:
            return None
        raise ValueError(f"{name} is required")
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    return ctypes.c_void_p(t.data_ptr())


_WORD = (torch.int32, getattr(torch, "uint32", torch.int32))


def _dev_or_pinned(t, name):
    """A CUDA tensor, or a page-locked (pinned) host tensor, which the device reads in
    place through unified addressing."""
    if isinstance(t, torch.Tensor) and not t.is_cuda and t.is_pinned():
        return ctypes.c_void_p(t.data_ptr())
    return _dev(t, name)


def _dense(t, name, dtype=None, allow_none=False, n=None):
    """A contiguous tensor of at least n elements (the call reads or writes n).
    dtype _WORD: any 4-byte integer type (status bits, counts)."""
    if t is not None:
        if not isinstance(t, torch.Tensor):
            raise ValueError(f"{name} must be a CUDA tensor")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        if n is not None and t.numel() < n:
            raise ValueError(f"{name} needs {n} elements, has {t.numel()}")
        if dtype is _WORD:
            if t.dtype not in _WORD:
                raise ValueError(f"{name} must be int32 or uint32, got {t.dtype}")
            dtype = None
    return _dev(t, name, dtype, allow_none)


def _rows(t, name, B=None, T_cap=None):
    """A [B, T] int32 tensor whose rows may be strided (unit inner stride), with at
    least B rows; returns (pointer, row stride, T_cap), T_cap at most T (default T)."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2 or t.stride(1) != 1:
        raise ValueError(f"{name} must be 2-D with unit inner stride")
    if B is not None and t.shape[0] < B:
        raise ValueError(f"{name} has {t.shape[0]} rows, the call needs {B}")
    if T_cap is None:
        T_cap = t.shape[1]
    elif not 0 <= T_cap <= t.shape[1]:
        raise ValueError(f"T_cap = {T_cap} is outside [0, {name}.shape[1] = {t.shape[1]}]")
    return _dev(t, name, torch.int32), t.stride(0), int(T_cap)


def _code(x):
    if x in (torch.float32, "f32", PLDP_F32):
        return PLDP_F32
    if x in (torch.bfloat16, "bf16", PLDP_BF16):
        return PLDP_BF16
    raise ValueError(f"unsupported dtype {x}")


def _done(fn, rc):
    """Whether a native call was made (rc is not None); raises when it failed."""
    if rc:
        _check(fn, rc)
    return rc is not None


def _check(fn, rc):
    if rc != 0:
        raise PldpError(fn, rc, _load().pldp_last_error().decode())


# ----------------------------------------------------------------------------
# the C ABI, one call each
# ----------------------------------------------------------------------------
def pldp_find_candidates(ids, seq_len, ngram_min, ngram_max, cand_pos, cand_count, match_len,
                         status=None, T_cap=None, stream=None):
    """Eq. 1 with the longest-suffix n-gram rule.  ids: int32 [B, T] (rows may be
    strided), seq_len int32 [B]; outputs cand_pos int32 [B, C_cap], cand_count and
    match_len int32 [B], status uint32-as-int32 [B] (optional)."""
    if _calls is not None and _done("pldp_find_candidates", _calls.find_candidates(
            ids, seq_len, ngram_min, ngram_max, cand_pos, cand_count, match_len, status, T_cap, stream)):
        return
    p_ids, stride, T = _rows(ids, "ids", T_cap=T_cap)
    B = ids.shape[0]
    C_cap = cand_pos.shape[1] if cand_pos is not None and cand_pos.dim() == 2 else 0
    _check("pldp_find_candidates", _load().pldp_find_candidates(
        p_ids, stride, _dense(seq_len, "seq_len", torch.int32, n=B), B, T,
        ngram_min, ngram_max, _dense(cand_pos, "cand_pos", torch.int32, allow_none=True, n=B * C_cap), C_cap,
        _dense(cand_count, "cand_count", torch.int32, n=B), _dense(match_len, "match_len", torch.int32, n=B),
        _dense(status, "status", _WORD, allow_none=True, n=B), _stream(stream)))


def pldp_rank_hidden(H, seq_len, cand_pos, cand_count, best_pos, scores=None, best_score=None,
                     threshold=float("-inf"), status=None, stream=None):
    """Eq. 3.  H: [B, T_cap, d] float32/bfloat16 (the chosen layer), contiguous rows;
    cand_pos int32 [B, C_cap]; outputs best_pos int32 [B], scores float32 [B, C_cap]
    and best_score float32 [B] (optional)."""
    if _calls is not None and _done("pldp_rank_hidden", _calls.rank_hidden(
            H, seq_len, cand_pos, cand_count, best_pos, scores, best_score, threshold, status, stream)):
        return
    if H.dim() != 3 or H.stride(2) != 1 or H.stride(1) != H.shape[2]:
        raise ValueError("H must be [B, T_cap, d] with contiguous rows")
    B, T_cap, d = H.shape
    C_cap = cand_pos.shape[1]
    _check("pldp_rank_hidden", _load().pldp_rank_hidden(
        _dev(H, "H"), _code(H.dtype), d, H.stride(0), _dense(seq_len, "seq_len", torch.int32, n=B), B,
        T_cap, _dense(cand_pos, "cand_pos", torch.int32, n=B * C_cap), _dense(cand_count, "cand_count", torch.int32, n=B),
        C_cap, float(threshold), _dense(scores, "scores", torch.float32, allow_none=True, n=B * C_cap),
        _dense(best_pos, "best_pos", torch.int32, n=B),
        _dense(best_score, "best_score", torch.float32, allow_none=True, n=B),
        _dense(status, "status", _WORD, allow_none=True, n=B), _stream(stream)))


def pldp_rank_hidden_avg(H, seq_len, cand_pos, cand_count, best_pos, m, scores=None, best_score=None,
                         threshold=float("-inf"), status=None, stream=None):
    """App. B.2: Eq. 3 on the means of the m rows ending at each position.  Same
    arguments as pldp_rank_hidden plus the window length m >= 1."""
    if H.dim() != 3 or H.stride(2) != 1 or H.stride(1) != H.shape[2]:
        raise ValueError("H must be [B, T_cap, d] with contiguous rows")
    B, T_cap, d = H.shape
    C_cap = cand_pos.shape[1]
    _check("pldp_rank_hidden_avg", _load().pldp_rank_hidden_avg(
        _dev(H, "H"), _code(H.dtype), d, H.stride(0), int(m), _dense(seq_len, "seq_len", torch.int32, n=B), B,
        T_cap, _dense(cand_pos, "cand_pos", torch.int32, n=B * C_cap), _dense(cand_count, "cand_count", torch.int32, n=B),
        C_cap, float(threshold), _dense(scores, "scores", torch.float32, allow_none=True, n=B * C_cap),
        _dense(best_pos, "best_pos", torch.int32, n=B),
        _dense(best_score, "best_score", torch.float32, allow_none=True, n=B),
        _dense(status, "status", _WORD, allow_none=True, n=B), _stream(stream)))


def pldp_identify_heads(ids, pos, A, counts, max_suffix=64, r_star=None, status=None, stream=None):
    """Sec. 4.2.1 head identification.  ids int32 [B, T_cap]; pos int32 [B] (the
    generated token's position p); A [B, R, T_cap] float32/bfloat16, the attention
    rows of query p-1 (unit inner stride); counts int32/uint32 [R] CUDA tensor,
    added to.  r_star int32 [B] out (optional)."""
    if _calls is not None and _done("pldp_identify_heads", _calls.identify_heads(
            ids, pos, A, counts, max_suffix, r_star, status, stream)):
        return
    if A.dim() != 3 or A.stride(2) != 1:
        raise ValueError("A must be [B, R, T_cap] with unit inner stride")
    B, R = A.shape[0], A.shape[1]
    p_ids, stride, T_cap = _rows(ids, "ids", B)
    if A.shape[2] < T_cap:
        raise ValueError("A must cover the T_cap = ids.shape[1] key positions")
    _check("pldp_identify_heads", _load().pldp_identify_heads(
        p_ids, stride, _dense(pos, "pos", torch.int32, n=B), B, T_cap, int(max_suffix), _dev(A, "A"), _code(A.dtype),
        R, A.stride(1), A.stride(0), _dense(counts, "counts", _WORD, n=R),
        _dense(r_star, "r_star", torch.int32, allow_none=True, n=B),
        _dense(status, "status", _WORD, allow_none=True, n=B), _stream(stream)))


def pldp_top_heads(counts, k, row_idx, stream=None):
    """The k rows with the most counts (ties to the smaller index) into row_idx int32 [k]."""
    if _calls is not None and _done("pldp_top_heads", _calls.top_heads(counts, k, row_idx, stream)):
        return
    _check("pldp_top_heads", _load().pldp_top_heads(_dense(counts, "counts", _WORD), counts.numel(), int(k),
                                                    _dense(row_idx, "row_idx", torch.int32, n=int(k)),
                                                    _stream(stream)))


def pldp_rank_attention(A, seq_len, cand_pos, cand_count, best_pos, row_idx=None, agg=PLDP_AGG_MAX,
                        scores=None, best_score=None, status=None, stream=None):
    """Eq. 2.  A: [B, R, T_cap] float32/bfloat16, attention of query t-1 for each of R
    (layer, head) rows, with contiguous keys (each row dense) or key-major (the R values
    of a key dense: e.g. a [B, T_cap, R] tensor transposed to [B, R, T_cap]), on the
    device or in pinned host memory (read in place: only the selected rows' values at the
    candidate keys cross the link); row_idx int32 [n_sel] device or None (all)."""
    if _calls is not None and _done("pldp_rank_attention", _calls.rank_attention(
            A, seq_len, cand_pos, cand_count, best_pos, row_idx, agg, scores, best_score, status, stream)):
        return
    if A.dim() != 3:
        raise ValueError("A must be [B, R, T_cap]")
    B, R, T_cap = A.shape
    C_cap = cand_pos.shape[1]
    n_sel = R if row_idx is None else row_idx.numel()
    _check("pldp_rank_attention", _load().pldp_rank_attention(
        _dev_or_pinned(A, "A"), _code(A.dtype), R, A.stride(1), A.stride(2), A.stride(0),
        _dense(row_idx, "row_idx", torch.int32, allow_none=True), n_sel, int(agg),
        _dense(seq_len, "seq_len", torch.int32, n=B), B, T_cap, _dense(cand_pos, "cand_pos", torch.int32, n=B * C_cap),
        _dense(cand_count, "cand_count", torch.int32, n=B), C_cap,
        _dense(scores, "scores", torch.float32, allow_none=True, n=B * C_cap),
        _dense(best_pos, "best_pos", torch.int32, n=B),
        _dense(best_score, "best_score", torch.float32, allow_none=True, n=B),
        _dense(status, "status", _WORD, allow_none=True, n=B), _stream(stream)))


def pldp_extract_draft(ids, seq_len, best_pos, draft, draft_len, T_cap=None, stream=None):
    """Sec. 4.3.  draft int32 [B, K] and draft_len int32 [B] are written."""
    if _calls is not None and _done("pldp_extract_draft", _calls.extract_draft(ids, seq_len, best_pos, draft, draft_len, T_cap, stream)):
        return
    B, K = draft.shape
    p_ids, stride, T = _rows(ids, "ids", B, T_cap)
    _check("pldp_extract_draft", _load().pldp_extract_draft(
        p_ids, stride, _dense(seq_len, "seq_len", torch.int32, n=B), T,
        _dense(best_pos, "best_pos", torch.int32, n=B), B, K, _dense(draft, "draft", torch.int32, n=B * K),
        _dense(draft_len, "draft_len", torch.int32, n=B), _stream(stream)))


def pldp_draft_workspace_size(B) -> int:
    return int(_load().pldp_draft_workspace_size(B))


def _draft_args(ids, seq_len, ngram_min, ngram_max, cand_pos, cand_count, match_len, K, draft,
                draft_len, workspace, H=None, best_h=None, h_scores=None, best_h_score=None,
                threshold=float("-inf"), A=None, best_a=None, row_idx=None, agg=PLDP_AGG_MAX,
                a_scores=None, best_a_score=None, draft_from="hidden", status=None, T_cap=None,
                index=None, V=None):
    """The argument block of pldp_draft_step (marshalling only)."""
    p_ids, stride, T = _rows(ids, "ids", T_cap=T_cap)
    B = ids.shape[0]
    a = pldp_draft_step_args()
    a.ids, a.ids_stride, a.seq_len, a.B = p_ids, stride, _dense(seq_len, "seq_len", torch.int32, n=B), B
    a.T_cap = T
    a.ngram_min, a.ngram_max = ngram_min, ngram_max
    a.C_cap = C_cap = cand_pos.shape[1] if cand_pos is not None and cand_pos.dim() == 2 else 0
    a.cand_pos = _dense(cand_pos, "cand_pos", torch.int32, allow_none=True, n=B * C_cap)
    a.cand_count = _dense(cand_count, "cand_count", torch.int32, n=B)
    a.match_len = _dense(match_len, "match_len", torch.int32, n=B)
    if H is not None:
        if H.dim() != 3 or H.stride(2) != 1 or H.stride(1) != H.shape[2]:
            raise ValueError("H must be [B, T_cap, d] with contiguous rows")
        if H.shape[0] < B or H.shape[1] < T:
            raise ValueError(f"H must cover [B, T_cap] = [{B}, {T}] positions")
        a.H, a.h_dtype, a.d, a.h_seq_stride = _dev(H, "H"), _code(H.dtype), H.shape[2], H.stride(0)
        a.threshold = float(threshold)
        a.h_scores = _dense(h_scores, "h_scores", torch.float32, allow_none=True, n=B * C_cap)
        a.best_h = _dense(best_h, "best_h", torch.int32, n=B)
        a.best_h_score = _dense(best_h_score, "best_h_score", torch.float32, allow_none=True, n=B)
    if A is not None:
        if A.dim() != 3:
            raise ValueError("A must be [B, R, T_cap]")
        if A.shape[0] < B or A.shape[2] < T:
            raise ValueError(f"A must cover [B, T_cap] = [{B}, {T}] positions")
        a.A, a.a_dtype, a.R = _dev_or_pinned(A, "A"), _code(A.dtype), A.shape[1]
        a.a_row_stride, a.a_key_stride, a.a_seq_stride = A.stride(1), A.stride(2), A.stride(0)
        a.row_idx = _dense(row_idx, "row_idx", torch.int32, allow_none=True)
        a.n_sel = A.shape[1] if row_idx is None else row_idx.numel()
        a.agg = int(agg)
        a.a_scores = _dense(a_scores, "a_scores", torch.float32, allow_none=True, n=B * C_cap)
        a.best_a = _dense(best_a, "best_a", torch.int32, n=B)
        a.best_a_score = _dense(best_a_score, "best_a_score", torch.float32, allow_none=True, n=B)
    a.draft_from = {"hidden": 0, "attention": 1, 0: 0, 1: 1}[draft_from]
    a.K = K
    a.draft = _dense(draft, "draft", torch.int32, n=B * K)
    a.draft_len = _dense(draft_len, "draft_len", torch.int32, n=B)
    a.status = _dense(status, "status", _WORD, allow_none=True, n=B)
    if workspace is not None:
        a.workspace = _dense(workspace, "workspace")
        a.workspace_bytes = workspace.numel() * workspace.element_size()
    if index is not None:
        if V is None:
            raise ValueError("an index needs V")
        a.index = _dense(index, "index")
        a.index_bytes = index.numel() * index.element_size()
        a.V = int(V)
    return a


def pldp_draft_step(ids, seq_len, ngram_min, ngram_max, cand_pos, cand_count, match_len, K, draft,
                    draft_len, workspace, stream=None, **kw):
    """Candidate search, ranking (hidden and/or attention) and draft in one call; the
    arguments mean what they mean in the separate calls.  workspace: a uint8 CUDA
    tensor of pldp_draft_workspace_size(B) bytes, zeroed once before first use (may be
    None with an index).  index: a uint8 CUDA tensor of pldp_index_size(B, V) bytes
    built by pldp_index_build (token ids in [0, V)); the step then looks occurrences
    up instead of scanning, with the same results.  Keyword arguments: H, best_h,
    h_scores, best_h_score, threshold, A, best_a, row_idx, agg, a_scores,
    best_a_score, draft_from, status, T_cap, index, V."""
    if _calls is not None and _done("pldp_draft_step", _calls.draft_step(
            ids, seq_len, ngram_min, ngram_max, cand_pos, cand_count, match_len, K, draft, draft_len, workspace, stream, kw)):
        return
    a = _draft_args(ids, seq_len, ngram_min, ngram_max, cand_pos, cand_count, match_len, K, draft,
                    draft_len, workspace, **kw)
    _check("pldp_draft_step", _load().pldp_draft_step(ctypes.byref(a), _stream(stream)))


def pldp_verify_greedy_draft(logits, draft, draft_len, accept_len, next_token, workspace, ids, seq_len,
                             ngram_min, ngram_max, cand_pos, cand_count, match_len, next_draft,
                             next_draft_len, index, argmax=None, kv_keep_len=None, stream=None, **kw):
    """Greedy verification of this step (as pldp_verify_greedy, appending to ids and
    seq_len) followed by the next step's drafting with the token index (as
    pldp_draft_step on the extended context), in one call.  next_draft /
    next_draft_len receive the next draft (they may be draft / draft_len).  Keyword
    arguments are pldp_draft_step's (H, best_h, A, best_a, status, ...)."""
    if _calls is not None and _done("pldp_verify_greedy_draft", _calls.verify_greedy_draft(
            logits, draft, draft_len, accept_len, next_token, workspace, ids, seq_len, ngram_min, ngram_max, cand_pos,
            cand_count, match_len, next_draft, next_draft_len, index, argmax, kv_keep_len, stream, kw)):
        return
    B, K1, V = logits.shape
    K = K1 - 1
    if draft.shape != (B, K) or next_draft.shape != (B, K):
        raise ValueError("draft and next_draft must be [B, K] with K = logits.shape[1] - 1")
    if not isinstance(ids, torch.Tensor) or ids.dim() != 2 or ids.shape[0] != B:
        raise ValueError("ids must be [B, T_cap] with B = logits.shape[0]")
    a = pldp_verify_draft_args()
    a.next = _draft_args(ids, seq_len, ngram_min, ngram_max, cand_pos, cand_count, match_len, K, next_draft,
                         next_draft_len, None, index=index, V=V, **kw)
    a.logits, a.dtype, a.V = _dense(logits, "logits"), _code(logits.dtype), V
    a.draft = _dense(draft, "draft", torch.int32, n=B * K)
    a.draft_len = _dense(draft_len, "draft_len", torch.int32, n=B)
    a.argmax = _dense(argmax, "argmax", torch.int32, allow_none=True, n=B * K1)
    a.accept_len = _dense(accept_len, "accept_len", torch.int32, n=B)
    a.next_token = _dense(next_token, "next_token", torch.int32, n=B)
    a.kv_keep_len = _dense(kv_keep_len, "kv_keep_len", torch.int32, allow_none=True, n=B)
    a.workspace = _dense(workspace, "workspace")
    a.workspace_bytes = workspace.numel() * workspace.element_size()
    _check("pldp_verify_greedy_draft", _load().pldp_verify_greedy_draft(ctypes.byref(a), _stream(stream)))


def pldp_verify_sample_draft_workspace_size(B, K, V, dtype=torch.bfloat16) -> int:
    return int(_load().pldp_verify_sample_draft_workspace_size(B, K, V, _code(dtype)))


def pldp_verify_sample_draft(logits, uniforms, draft, draft_len, accept_len, next_token, workspace, ids, seq_len,
                             ngram_min, ngram_max, cand_pos, cand_count, match_len, next_draft, next_draft_len,
                             index, temperature=1.0, sampled=None, kv_keep_len=None, stream=None, **kw):
    """Sampling verification of this step (as pldp_verify_sample at ``temperature``
    with ``uniforms`` [B, K+1], appending to ids and seq_len) followed by the next
    step's drafting with the token index (as pldp_draft_step on the extended
    context), in one call.  workspace: uint8 CUDA tensor of
    pldp_verify_sample_draft_workspace_size(B, K, V, dtype) bytes.  Other arguments
    as pldp_verify_greedy_draft."""
    if _calls is not None and _done("pldp_verify_sample_draft", _calls.verify_sample_draft(
            logits, uniforms, draft, draft_len, accept_len, next_token, workspace, ids, seq_len, ngram_min, ngram_max,
            cand_pos, cand_count, match_len, next_draft, next_draft_len, index, temperature, sampled, kv_keep_len, stream,
            kw)):
        return
    B, K1, V = logits.shape
    K = K1 - 1
    if draft.shape != (B, K) or next_draft.shape != (B, K):
        raise ValueError("draft and next_draft must be [B, K] with K = logits.shape[1] - 1")
    if uniforms.shape != (B, K1):
        raise ValueError("uniforms must be [B, K+1]")
    if not isinstance(ids, torch.Tensor) or ids.dim() != 2 or ids.shape[0] != B:
        raise ValueError("ids must be [B, T_cap] with B = logits.shape[0]")
    a = pldp_verify_sample_draft_args()
    a.next = _draft_args(ids, seq_len, ngram_min, ngram_max, cand_pos, cand_count, match_len, K, next_draft,
                         next_draft_len, None, index=index, V=V, **kw)
    a.logits, a.dtype, a.V = _dense(logits, "logits"), _code(logits.dtype), V
    a.temperature = float(temperature)
    a.uniforms = _dense(uniforms, "uniforms", torch.float32, n=B * K1)
    a.draft = _dense(draft, "draft", torch.int32, n=B * K)
    a.draft_len = _dense(draft_len, "draft_len", torch.int32, n=B)
    a.sampled = _dense(sampled, "sampled", torch.int32, allow_none=True, n=B * K1)
    a.accept_len = _dense(accept_len, "accept_len", torch.int32, n=B)
    a.next_token = _dense(next_token, "next_token", torch.int32, n=B)
    a.kv_keep_len = _dense(kv_keep_len, "kv_keep_len", torch.int32, allow_none=True, n=B)
    a.workspace = _dense(workspace, "workspace")
    a.workspace_bytes = workspace.numel() * workspace.element_size()
    _check("pldp_verify_sample_draft", _load().pldp_verify_sample_draft(ctypes.byref(a), _stream(stream)))


def pldp_index_size(B, V) -> int:
    return int(_load().pldp_index_size(B, V))


def pldp_index_build(ids, seq_len, V, index, status=None, T_cap=None, stream=None):
    """Builds the incremental token index of pldp_draft_step over positions
    0 .. seq_len[b]-2 of every sequence.  index: uint8 CUDA tensor of
    pldp_index_size(B, V) bytes (cleared by the call)."""
    if _calls is not None and _done("pldp_index_build", _calls.index_build(ids, seq_len, V, index, status, T_cap, stream)):
        return
    p_ids, stride, T = _rows(ids, "ids", T_cap=T_cap)
    B = ids.shape[0]
    _check("pldp_index_build", _load().pldp_index_build(
        p_ids, stride, _dense(seq_len, "seq_len", torch.int32, n=B), B, T, int(V),
        _dense(index, "index"), index.numel() * index.element_size(),
        _dense(status, "status", _WORD, allow_none=True, n=B), _stream(stream)))


def pldp_verify_workspace_size(B, K, V) -> int:
    return int(_load().pldp_verify_workspace_size(B, K, V))


def pldp_verify_greedy(logits, draft, draft_len, accept_len, next_token, workspace, argmax=None,
                       ids=None, seq_len=None, kv_keep_len=None, status=None, T_cap=None,
                       stream=None):
    """Sec. 4.4 (greedy).  logits [B, K+1, V] float32/bfloat16 contiguous; workspace a
    uint8 CUDA tensor of pldp_verify_workspace_size(B, K, V) bytes, zeroed once before
    first use (every call leaves it zeroed).  ids/seq_len (optional, modified in place)
    get the accepted tokens and the bonus token appended."""
    if _calls is not None and _done("pldp_verify_greedy", _calls.verify_greedy(
            logits, draft, draft_len, accept_len, next_token, workspace, argmax, ids, seq_len, kv_keep_len, status, T_cap,
            stream)):
        return
    B, K1, V = logits.shape
    K = K1 - 1
    if draft.shape != (B, K):
        raise ValueError("draft must be [B, K] with K = logits.shape[1] - 1")
    p_ids, stride, T = (None, 0, 0) if ids is None else _rows(ids, "ids", B, T_cap)
    if T_cap is None:
        T_cap = T
    _check("pldp_verify_greedy", _load().pldp_verify_greedy(
        _dense(logits, "logits"), _code(logits.dtype), B, K, V, _dense(draft, "draft", torch.int32, n=B * K),
        _dense(draft_len, "draft_len", torch.int32, n=B),
        _dense(argmax, "argmax", torch.int32, allow_none=True, n=B * K1),
        _dense(accept_len, "accept_len", torch.int32, n=B), _dense(next_token, "next_token", torch.int32, n=B),
        p_ids, stride, _dense(seq_len, "seq_len", torch.int32, allow_none=True, n=B), T_cap,
        _dense(kv_keep_len, "kv_keep_len", torch.int32, allow_none=True, n=B),
        _dense(status, "status", _WORD, allow_none=True, n=B), _dense(workspace, "workspace"),
        workspace.numel() * workspace.element_size(), _stream(stream)))


def pldp_verify_sample_workspace_size(B, K, V, dtype=torch.bfloat16) -> int:
    return int(_load().pldp_verify_sample_workspace_size(B, K, V, _code(dtype)))


def pldp_verify_sample(logits, uniforms, draft, draft_len, accept_len, next_token, workspace,
                       temperature=1.0, sampled=None, ids=None, seq_len=None, kv_keep_len=None,
                       status=None, T_cap=None, stream=None):
    """Sec. 4.4 with sampling at ``temperature``: position i of sequence b draws the
    smallest v whose cumulative softmax(logits / T) probability exceeds uniforms[b, i]
    (float32 [B, K+1] CUDA tensor); acceptance and bookkeeping as pldp_verify_greedy.
    workspace: uint8 CUDA tensor of pldp_verify_sample_workspace_size(B, K, V, dtype) bytes."""
    if _calls is not None and _done("pldp_verify_sample", _calls.verify_sample(
            logits, uniforms, draft, draft_len, accept_len, next_token, workspace, temperature, sampled, ids, seq_len,
            kv_keep_len, status, T_cap, stream)):
        return
    B, K1, V = logits.shape
    K = K1 - 1
    if draft.shape != (B, K):
        raise ValueError("draft must be [B, K] with K = logits.shape[1] - 1")
    if uniforms.shape != (B, K1):
        raise ValueError("uniforms must be [B, K+1]")
    p_ids, stride, T = (None, 0, 0) if ids is None else _rows(ids, "ids", B, T_cap)
    if T_cap is None:
        T_cap = T
    _check("pldp_verify_sample", _load().pldp_verify_sample(
        _dense(logits, "logits"), _code(logits.dtype), B, K, V, float(temperature),
        _dense(uniforms, "uniforms", torch.float32), _dense(draft, "draft", torch.int32, n=B * K),
        _dense(draft_len, "draft_len", torch.int32, n=B), _dense(sampled, "sampled", torch.int32, allow_none=True, n=B * K1),
        _dense(accept_len, "accept_len", torch.int32, n=B), _dense(next_token, "next_token", torch.int32, n=B),
        p_ids, stride, _dense(seq_len, "seq_len", torch.int32, allow_none=True, n=B), T_cap,
        _dense(kv_keep_len, "kv_keep_len", torch.int32, allow_none=True, n=B),
        _dense(status, "status", _WORD, allow_none=True, n=B), _dense(workspace, "workspace"),
        workspace.numel() * workspace.element_size(), _stream(stream)))


def pldp_verify_greedy_noalloc(logits, draft, draft_len, accept_len, next_token, argmax=None,
                               ids=None, seq_len=None, kv_keep_len=None, status=None, T_cap=None,
                               stream=None):
    """pldp_verify_greedy for callers that cannot allocate a workspace: the library
    uses its own fixed scratch area (see include/pldp.h for the size limit and for
    why overlapping calls on one device must be serialised)."""
    B, K1, V = logits.shape
    K = K1 - 1
    if draft.shape != (B, K):
        raise ValueError("draft must be [B, K] with K = logits.shape[1] - 1")
    p_ids, stride, T = (None, 0, 0) if ids is None else _rows(ids, "ids", B, T_cap)
    if T_cap is None:
        T_cap = T
    _check("pldp_verify_greedy_noalloc", _load().pldp_verify_greedy_noalloc(
        _dense(logits, "logits"), _code(logits.dtype), B, K, V, _dense(draft, "draft", torch.int32, n=B * K),
        _dense(draft_len, "draft_len", torch.int32, n=B),
        _dense(argmax, "argmax", torch.int32, allow_none=True, n=B * K1),
        _dense(accept_len, "accept_len", torch.int32, n=B), _dense(next_token, "next_token", torch.int32, n=B),
        p_ids, stride, _dense(seq_len, "seq_len", torch.int32, allow_none=True, n=B), T_cap,
        _dense(kv_keep_len, "kv_keep_len", torch.int32, allow_none=True, n=B),
        _dense(status, "status", _WORD, allow_none=True, n=B), _stream(stream)))


# ----------------------------------------------------------------------------
# the target model's cache around a step
# ----------------------------------------------------------------------------
class pldp_cache:
    """One layer's paged cache, for the calls below: the description of pldp_cache in
    include/pldp.h, made and checked once (it keeps the tensors alive).

    k_cache, v_cache   CUDA tensors seen as [n_pages, page_size, heads, head_dim], bfloat16 or
                       float8_e4m3fn, of the same shape and strides with unit inner stride
                       (a pool held as [n_pages, heads, page_size, head_dim] is passed
                       as ``pool.permute(0, 2, 1, 3)``).
    pages              int32 [B, max_pages], rows may be strided.
    k_scale, v_scale   float32 [n_pages, heads, page_size], contiguous, for float8_e4m3fn.
    """

    def __init__(self, k_cache, v_cache, pages, k_scale=None, v_scale=None):
        kinds = {torch.bfloat16: PLDP_BF16, torch.float8_e4m3fn: PLDP_E4M3}
        for t, name in ((k_cache, "k_cache"), (v_cache, "v_cache")):
            _dev(t, name)
            if t.dim() != 4 or t.stride(3) != 1 or t.dtype not in kinds:
                raise ValueError(f"{name} must be [n_pages, page_size, heads, head_dim] with unit inner stride, bfloat16 or "
                                 "float8_e4m3fn")
        if k_cache.shape != v_cache.shape or k_cache.stride() != v_cache.stride() or k_cache.dtype != v_cache.dtype:
            raise ValueError("k_cache and v_cache must have the same shape, strides and dtype")
        n_pages, page_size, heads, head_dim = k_cache.shape
        p_pages, stride, max_pages = _rows(pages, "pages")
        a = self.args = pldp_cache_args()
        a.k, a.v, a.dtype = _dev(k_cache, "k_cache"), _dev(v_cache, "v_cache"), kinds[k_cache.dtype]
        if a.dtype == PLDP_E4M3:
            for t, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
                if t is None or tuple(t.shape) != (n_pages, heads, page_size):
                    raise ValueError(f"{name} must be [n_pages, heads, page_size] for a float8_e4m3fn cache")
            a.k_scale, a.v_scale = _dense(k_scale, "k_scale", torch.float32), _dense(v_scale, "v_scale", torch.float32)
        elif k_scale is not None or v_scale is not None:
            raise ValueError("k_scale and v_scale belong to a float8_e4m3fn cache")
        a.n_pages, a.page_size, a.heads, a.head_dim = n_pages, page_size, heads, head_dim
        a.page_stride, a.pos_stride, a.head_stride = k_cache.stride()[:3]
        a.pages, a.pages_stride, a.max_pages = p_pages, stride, max_pages
        self.B, self.heads, self.head_dim, self.dtype = pages.shape[0], heads, head_dim, k_cache.dtype
        self.address = ctypes.addressof(a)                   # for the native calls
        self.tensors = (k_cache, v_cache, pages, k_scale, v_scale)


def _vectors(t, name, shape, dtypes):
    """A [sequences, tokens, heads, head_dim] tensor of `shape` (None: any) with unit inner
    stride; returns (pointer, its three strides)."""
    p = _dev(t, name)
    if t.dim() != 4 or t.stride(3) != 1 or t.dtype not in dtypes:
        raise ValueError(f"{name} must be [B, n, heads, head_dim] of {' or '.join(map(str, dtypes))} with unit inner stride")
    if any(w is not None and w != g for w, g in zip(shape, t.shape)):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, the call needs {shape}")
    return p, _STRIDES(*t.stride()[:3])


def _step_cache(cache, B):
    if not isinstance(cache, pldp_cache):
        raise ValueError("cache must be a pldp_cache")
    if B > cache.B:
        raise ValueError(f"the cache's page table has {cache.B} rows, the call needs {B}")
    return cache.args


def pldp_cache_append(cache, q, k, v, seq_len, q_out, draft_len=None, q_norm=None, k_norm=None, eps=1e-6, cos=None,
                      sin=None, interleaved=False, status=None, stream=None):
    """Norms (q_norm / k_norm [head_dim], optional) and rotates (cos / sin float32 [positions,
    rot/2], optional) the queries and keys of a step's tokens, x_t and the draft at positions
    seq_len[b]-1 .. seq_len[b]-1+draft_len[b], writes the queries to q_out (bfloat16) and the keys
    and values to the cache.  q [B, n, q_heads, head_dim], k and v [B, n, heads, head_dim], float32
    or bfloat16, any strides of whole 16 bytes with unit inner stride (slices of one projection)."""
    if _calls is not None and type(cache) is pldp_cache and _done("pldp_cache_append", _calls.cache_append(
            cache.address, cache.B, q, k, v, seq_len, q_out, draft_len, q_norm, k_norm, eps, cos, sin, interleaved, status,
            stream)):
        return
    kinds = (torch.float32, torch.bfloat16)
    a = pldp_cache_append_args()
    a.q, a.q_strides = _vectors(q, "q", (None,) * 4, kinds)
    B, n, Hq, D = q.shape
    a.cache = _step_cache(cache, B)
    if D != cache.head_dim:
        raise ValueError(f"q has head_dim {D}, the cache {cache.head_dim}")
    a.k, a.k_strides = _vectors(k, "k", (B, n, cache.heads, D), (q.dtype,))
    a.v, a.v_strides = _vectors(v, "v", (B, n, cache.heads, D), (q.dtype,))
    a.q_out, a.q_out_strides = _vectors(q_out, "q_out", (B, n, Hq, D), (torch.bfloat16,))
    a.dtype, a.B, a.n, a.q_heads, a.eps = _code(q.dtype), B, n, Hq, float(eps)
    a.q_norm = _dense(q_norm, "q_norm", q.dtype, allow_none=True, n=D)
    a.k_norm = _dense(k_norm, "k_norm", q.dtype, allow_none=True, n=D)
    if cos is not None or sin is not None:
        if cos is None or sin is None or cos.dim() != 2 or cos.shape != sin.shape:
            raise ValueError("cos and sin must both be [positions, rot/2]")
        a.cos, a.sin = _dense(cos, "cos", torch.float32), _dense(sin, "sin", torch.float32)
        if cos.numel() == 0:                             # an empty tensor's null pointer would mean no rotation
            raise PldpError("pldp_cache_append", PLDP_ERR_INVALID_ARG, "rot must be even, 2..head_dim, and rot_rows >= 1")
        a.rot_rows, a.rot = cos.shape[0], 2 * cos.shape[1]
    a.interleaved = int(bool(interleaved))
    a.seq_len = _dense(seq_len, "seq_len", torch.int32, n=B)
    a.draft_len = _dense(draft_len, "draft_len", torch.int32, allow_none=True, n=B)
    a.status = _dense(status, "status", _WORD, allow_none=True, n=B)
    _check("pldp_cache_append", _load().pldp_cache_append(ctypes.byref(a), _stream(stream)))


def pldp_cache_read(cache, start, count, k_out, v_out, status=None, stream=None):
    """Positions start[b] .. start[b]+count[b]-1 (start None: from 0) of every sequence into rows
    0 .. count[b]-1 of k_out and v_out [B, n, heads, head_dim], float32 or bfloat16 and of the same
    strides; either may be None."""
    if _calls is not None and type(cache) is pldp_cache and _done("pldp_cache_read", _calls.cache_read(
            cache.address, cache.B, start, count, k_out, v_out, status, stream)):
        return
    one = k_out if k_out is not None else v_out
    a = pldp_cache_read_args()
    p, a.out_strides = _vectors(one, "k_out" if one is k_out else "v_out", (None,) * 4, (torch.float32, torch.bfloat16))
    B, n = one.shape[:2]
    a.cache = _step_cache(cache, B)
    shape = (B, n, cache.heads, cache.head_dim)
    for name, t in (("k_out", k_out), ("v_out", v_out)):
        if t is not None:
            setattr(a, name, _vectors(t, name, shape, (one.dtype,))[0])
            if t.stride() != one.stride():
                raise ValueError("k_out and v_out must have the same strides")
    a.start = _dense(start, "start", torch.int32, allow_none=True, n=B)
    a.count = _dense(count, "count", torch.int32, n=B)
    a.B, a.n, a.dtype = B, n, _code(one.dtype)
    a.status = _dense(status, "status", _WORD, allow_none=True, n=B)
    _check("pldp_cache_read", _load().pldp_cache_read(ctypes.byref(a), _stream(stream)))


def pldp_attend_workspace_size(B, n, q_heads, heads, head_dim) -> int:
    return int(_load().pldp_attend_workspace_size(B, n, q_heads, heads, head_dim))


def pldp_attend_cache(cache, q, seq_len, out, workspace, draft_len=None, lse=None, scale=None, status=None, stream=None):
    """Attention of a step's tokens (x_t and the draft, appended before) over the cache.  q and
    out bfloat16 [B, n, q_heads, head_dim]; lse float32 [B, n, q_heads] (optional); scale default
    1/sqrt(head_dim).  workspace: uint8 CUDA tensor of pldp_attend_workspace_size(B, n, q_heads,
    heads, head_dim) bytes, zeroed once before first use; one of the largest size does for calls of
    any shapes that follow one another."""
    if _calls is not None and type(cache) is pldp_cache and _done("pldp_attend_cache", _calls.attend_cache(
            cache.address, cache.B, q, seq_len, out, workspace, draft_len, lse, scale, status, stream)):
        return
    a = pldp_attend_args()
    a.q, a.q_strides = _vectors(q, "q", (None,) * 4, (torch.bfloat16,))
    B, n, Hq, D = q.shape
    a.cache = _step_cache(cache, B)
    if D != cache.head_dim:
        raise ValueError(f"q has head_dim {D}, the cache {cache.head_dim}")
    a.out, a.out_strides = _vectors(out, "out", (B, n, Hq, D), (torch.bfloat16,))
    a.B, a.n, a.q_heads = B, n, Hq
    a.scale = D ** -0.5 if scale is None else float(scale)
    a.seq_len = _dense(seq_len, "seq_len", torch.int32, n=B)
    a.draft_len = _dense(draft_len, "draft_len", torch.int32, allow_none=True, n=B)
    a.lse = _dense(lse, "lse", torch.float32, allow_none=True, n=B * n * Hq)
    a.status = _dense(status, "status", _WORD, allow_none=True, n=B)
    a.workspace = _dense(workspace, "workspace")
    a.workspace_bytes = workspace.numel() * workspace.element_size()
    _check("pldp_attend_cache", _load().pldp_attend_cache(ctypes.byref(a), _stream(stream)))


def pldp_rank_cache(cache, q, row, kv_len, lse, cand_pos, cand_count, best_pos, heads=None, agg=PLDP_AGG_MAX, scale=None,
                    scores=None, best_score=None, accumulate=False, status=None, stream=None):
    """Eq. 2 from one layer's cache: candidate j scores the max (or sum) over the selected query
    heads (int32 `heads`, None: all) of the attention probability exp(scale q.k_j - lse) of query
    row[b] (None: 0) of the step, with q and lse as pldp_attend_cache had and wrote them.  After
    verification row is accept_len and kv_len is kv_keep_len.  accumulate: scores holds other
    layers' scores and takes the larger (or the sum)."""
    agg = {"max": PLDP_AGG_MAX, "sum": PLDP_AGG_SUM}.get(agg, agg)
    if _calls is not None and type(cache) is pldp_cache and _done("pldp_rank_cache", _calls.rank_cache(
            cache.address, cache.B, q, row, kv_len, lse, cand_pos, cand_count, best_pos, heads, agg, scale, scores, best_score,
            accumulate, status, stream)):
        return
    a = pldp_rank_cache_args()
    a.q, a.q_strides = _vectors(q, "q", (None,) * 4, (torch.bfloat16,))
    B, n, Hq, D = q.shape
    a.cache = _step_cache(cache, B)
    if D != cache.head_dim:
        raise ValueError(f"q has head_dim {D}, the cache {cache.head_dim}")
    if not isinstance(cand_pos, torch.Tensor) or cand_pos.dim() != 2 or cand_pos.shape[0] < B:
        raise ValueError("cand_pos must be [B, C_cap]")
    a.B, a.n, a.q_heads, a.C_cap = B, n, Hq, cand_pos.shape[1]
    a.row = _dense(row, "row", torch.int32, allow_none=True, n=B)
    a.kv_len = _dense(kv_len, "kv_len", torch.int32, n=B)
    a.lse = _dense(lse, "lse", torch.float32, n=B * n * Hq)
    a.heads = _dense(heads, "heads", torch.int32, allow_none=True)
    a.n_sel = 0 if heads is None else heads.numel()
    if heads is not None and a.n_sel < 1:                # an empty tensor's null pointer would mean all heads
        raise PldpError("pldp_rank_cache", PLDP_ERR_INVALID_ARG, "n_sel < 1")
    a.agg = agg
    a.accumulate = int(bool(accumulate))
    a.scale = D ** -0.5 if scale is None else float(scale)
    a.cand_pos = _dense(cand_pos, "cand_pos", torch.int32)
    a.cand_count = _dense(cand_count, "cand_count", torch.int32, n=B)
    a.scores = _dense(scores, "scores", torch.float32, allow_none=True, n=B * cand_pos.shape[1])
    a.best_pos = _dense(best_pos, "best_pos", torch.int32, n=B)
    a.best_score = _dense(best_score, "best_score", torch.float32, allow_none=True, n=B)
    a.status = _dense(status, "status", _WORD, allow_none=True, n=B)
    _check("pldp_rank_cache", _load().pldp_rank_cache(ctypes.byref(a), _stream(stream)))


def pldp_token_logprobs_workspace_size(rows, V) -> int:
    return int(_load().pldp_token_logprobs_workspace_size(rows, V))


def pldp_token_logprobs(logits, tokens, logprob, workspace, entropy=None, top_id=None, top_logprob=None, temperature=1.0,
                        stream=None):
    """Log probabilities under softmax(logits / temperature) of tokens (int32 [...], logprob float32
    [...]; both None for neither), the entropy (float32 [...], optional) and the likeliest
    alternatives (top_id int32 and top_logprob float32 [..., top], optional, top <= 32) of every row
    of logits [..., V] (float32 or bfloat16, contiguous).  workspace: uint8 CUDA tensor of
    pldp_token_logprobs_workspace_size(rows, V) bytes."""
    if _calls is not None and _done("pldp_token_logprobs", _calls.token_logprobs(
            logits, tokens, logprob, workspace, entropy, top_id, top_logprob, temperature, stream)):
        return
    p = _dense(logits, "logits")
    if logits.dim() < 1 or logits.shape[-1] < 1:
        raise ValueError("logits must be [..., V]")
    V = logits.shape[-1]
    rows = logits.numel() // V
    tops = {t.shape[-1] if t.dim() else 0 for t in (top_id, top_logprob) if t is not None}
    if len(tops) > 1:
        raise ValueError("top_id and top_logprob must have the same last dimension")
    top = tops.pop() if tops else 0
    _check("pldp_token_logprobs", _load().pldp_token_logprobs(
        p, _code(logits.dtype), rows, V, float(temperature),
        _dense(tokens, "tokens", torch.int32, allow_none=True, n=rows),
        _dense(logprob, "logprob", torch.float32, allow_none=True, n=rows),
        _dense(entropy, "entropy", torch.float32, allow_none=True, n=rows), top,
        _dense(top_id, "top_id", torch.int32, allow_none=True, n=rows * top),
        _dense(top_logprob, "top_logprob", torch.float32, allow_none=True, n=rows * top),
        _dense(workspace, "workspace"), workspace.numel() * workspace.element_size(), _stream(stream)))


# ----------------------------------------------------------------------------
# prompts, packed
# ----------------------------------------------------------------------------
def _packed(t, name, shape, dtypes):
    """A [rows, heads, head_dim] tensor of `shape` (None: any) with unit inner stride; returns
    (pointer, its two strides)."""
    p = _dev(t, name)
    if t.dim() != 3 or t.stride(2) != 1 or t.dtype not in dtypes:
        raise ValueError(f"{name} must be [rows, heads, head_dim] of {' or '.join(map(str, dtypes))} with unit inner stride")
    if any(w is not None and w != g for w, g in zip(shape, t.shape)):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, the call needs {shape}")
    return p, _ROW_STRIDES(*t.stride()[:2])


def _sequences(cache, rows, q):
    """The number of sequences of `rows`, and the cache's description."""
    p = _dense(rows, "rows", torch.int32)
    if rows.dim() != 1 or rows.numel() < 1:
        raise ValueError("rows must be [B + 1]")
    args = _step_cache(cache, rows.numel() - 1)
    if q.shape[2] != cache.head_dim:
        raise ValueError(f"q has head_dim {q.shape[2]}, the cache {cache.head_dim}")
    return p, rows.numel() - 1, args


def pldp_cache_append_prompt(cache, q, k, v, rows, q_out, start=None, q_norm=None, k_norm=None, eps=1e-6, cos=None, sin=None,
                             interleaved=False, status=None, stream=None):
    """pldp_cache_append of prompts packed behind one another: rows rows[b] .. rows[b+1]-1 (int32
    [B + 1]) of q [rows, q_heads, head_dim] and of k and v [rows, heads, head_dim] are sequence b's
    tokens at positions start[b] (int32 [B], None: 0) and on.  Other arguments as pldp_cache_append."""
    if _calls is not None and type(cache) is pldp_cache and _done("pldp_cache_append_prompt", _calls.cache_append_prompt(
            cache.address, cache.B, q, k, v, rows, q_out, start, q_norm, k_norm, eps, cos, sin, interleaved, status, stream)):
        return
    kinds = (torch.float32, torch.bfloat16)
    a = pldp_cache_append_prompt_args()
    a.q, a.q_strides = _packed(q, "q", (None,) * 3, kinds)
    R, Hq, D = q.shape
    a.rows, a.B, a.cache = _sequences(cache, rows, q)
    a.k, a.k_strides = _packed(k, "k", (R, cache.heads, D), (q.dtype,))
    a.v, a.v_strides = _packed(v, "v", (R, cache.heads, D), (q.dtype,))
    a.q_out, a.q_out_strides = _packed(q_out, "q_out", (R, Hq, D), (torch.bfloat16,))
    a.dtype, a.R, a.q_heads, a.eps = _code(q.dtype), R, Hq, float(eps)
    a.q_norm = _dense(q_norm, "q_norm", q.dtype, allow_none=True, n=D)
    a.k_norm = _dense(k_norm, "k_norm", q.dtype, allow_none=True, n=D)
    if cos is not None or sin is not None:
        if cos is None or sin is None or cos.dim() != 2 or cos.shape != sin.shape:
            raise ValueError("cos and sin must both be [positions, rot/2]")
        a.cos, a.sin = _dense(cos, "cos", torch.float32), _dense(sin, "sin", torch.float32)
        if cos.numel() == 0:                             # an empty tensor's null pointer would mean no rotation
            raise PldpError("pldp_cache_append_prompt", PLDP_ERR_INVALID_ARG, "rot must be even, 2..head_dim, and rot_rows >= 1")
        a.rot_rows, a.rot = cos.shape[0], 2 * cos.shape[1]
    a.interleaved = int(bool(interleaved))
    a.start = _dense(start, "start", torch.int32, allow_none=True, n=a.B)
    a.status = _dense(status, "status", _WORD, allow_none=True, n=a.B)
    _check("pldp_cache_append_prompt", _load().pldp_cache_append_prompt(ctypes.byref(a), _stream(stream)))


def pldp_attend_prompt_workspace_size(q_heads, heads, head_dim) -> int:
    return int(_load().pldp_attend_prompt_workspace_size(q_heads, heads, head_dim))


def pldp_attend_prompt(cache, q, rows, out, workspace, start=None, lse=None, scale=None, status=None, stream=None):
    """Causal attention over the cache of prompts packed behind one another (appended before): rows
    rows[b] .. rows[b+1]-1 (int32 [B + 1]) of q and out, bfloat16 [rows, q_heads, head_dim], are
    sequence b's tokens at positions start[b] (int32 [B], None: 0) and on, behind whatever the cache
    holds of it before.  lse float32 [rows, q_heads] (optional); scale default 1/sqrt(head_dim).
    workspace: uint8 CUDA tensor of pldp_attend_prompt_workspace_size(q_heads, heads, head_dim)
    bytes, 256-byte aligned; calls of any lengths that follow one another may share it."""
    if _calls is not None and type(cache) is pldp_cache and _done("pldp_attend_prompt", _calls.attend_prompt(
            cache.address, cache.B, q, rows, out, workspace, start, lse, scale, status, stream)):
        return
    a = pldp_attend_prompt_args()
    a.q, a.q_strides = _packed(q, "q", (None,) * 3, (torch.bfloat16,))
    R, Hq, D = q.shape
    a.rows, a.B, a.cache = _sequences(cache, rows, q)
    a.out, a.out_strides = _packed(out, "out", (R, Hq, D), (torch.bfloat16,))
    a.R, a.q_heads = R, Hq
    a.scale = D ** -0.5 if scale is None else float(scale)
    a.start = _dense(start, "start", torch.int32, allow_none=True, n=a.B)
    a.lse = _dense(lse, "lse", torch.float32, allow_none=True, n=R * Hq)
    a.status = _dense(status, "status", _WORD, allow_none=True, n=a.B)
    a.workspace = _dense(workspace, "workspace")
    a.workspace_bytes = workspace.numel() * workspace.element_size()
    _check("pldp_attend_prompt", _load().pldp_attend_prompt(ctypes.byref(a), _stream(stream)))


# ----------------------------------------------------------------------------
# the pages of a cache
# ----------------------------------------------------------------------------
class pldp_page_table:
    """The page table of a cache (one for all layers) with the number of entries that hold each
    page: the description of pldp_page_table in include/pldp.h, made and checked once (it keeps
    the tensors alive).

    pages       int32 [B, max_pages], rows may be strided; -1: no page.
    refs        int32 [n_pages], contiguous.
    page_size   positions of a page.
    """

    def __init__(self, pages, refs, page_size):
        p, stride, max_pages = _rows(pages, "pages")
        a = self.args = pldp_page_table_args()
        a.pages, a.pages_stride, a.B, a.max_pages, a.page_size = p, stride, pages.shape[0], max_pages, int(page_size)
        if not isinstance(refs, torch.Tensor) or refs.dim() != 1:
            raise ValueError("refs must be an int32 CUDA tensor [n_pages]")
        a.refs, a.n_pages = _dense(refs, "refs", torch.int32), refs.numel()
        self.B, self.max_pages, self.page_size, self.n_pages = a.B, max_pages, int(page_size), a.n_pages
        self.address = ctypes.addressof(a)                   # for the native calls
        self.tensors = (pages, refs)


def _table(table):
    if not isinstance(table, pldp_page_table):
        raise ValueError("table must be a pldp_page_table")
    return ctypes.byref(table.args)


def _pairs(copies, name="copies", n=None):
    """int32 [n, 2], contiguous: (pointer, n)."""
    p = _dense(copies, name, torch.int32)
    if copies.dim() != 2 or copies.shape[1] != 2 or (n is not None and copies.shape[0] != n):
        raise ValueError(f"{name} must be [{'n' if n is None else n}, 2]")
    return p, copies.shape[0]


def pldp_pages_workspace_size(table) -> int:
    _table(table)
    return int(_load().pldp_pages_workspace_size(table.B, table.max_pages, table.n_pages))


def pldp_pages_reserve(table, start, copies, workspace, n, count=None, status=None, stream=None):
    """Makes positions start[b] .. start[b]+count[b]-1 (int32 [B]; count None: n, which is the most)
    of every sequence ones that may be written: the lowest free pages for those that have none, and
    for pages that others hold too.  copies int32 [B, 2]: the page that pldp_cache_copy_pages then has
    to copy in every layer, and where to.  workspace: uint8 CUDA tensor of
    pldp_pages_workspace_size(table) bytes."""
    if _calls is not None and type(table) is pldp_page_table and _done("pldp_pages_reserve", _calls.pages_reserve(
            table.address, start, copies, workspace, n, count, status, stream)):
        return
    t = _table(table)
    _check("pldp_pages_reserve", _load().pldp_pages_reserve(
        t, _dense(start, "start", torch.int32, n=table.B), _dense(count, "count", torch.int32, allow_none=True, n=table.B), int(n),
        _pairs(copies, n=table.B)[0], _dense(status, "status", _WORD, allow_none=True, n=table.B), _dense(workspace, "workspace"),
        workspace.numel() * workspace.element_size(), _stream(stream)))


def pldp_pages_fork(table, parent, len, status=None, stream=None):
    """Row b of the table becomes those of row parent[b]'s entries that hold its first len[b]
    positions, shared with it (int32 [B]; parent -1: the row stays as it is)."""
    if _calls is not None and type(table) is pldp_page_table and _done("pldp_pages_fork", _calls.pages_fork(
            table.address, parent, len, status, stream)):
        return
    t = _table(table)
    _check("pldp_pages_fork", _load().pldp_pages_fork(
        t, _dense(parent, "parent", torch.int32, n=table.B), _dense(len, "len", torch.int32, n=table.B),
        _dense(status, "status", _WORD, allow_none=True, n=table.B), _stream(stream)))


def pldp_pages_free(table, keep_len, stream=None):
    """Gives back the pages past each sequence's first keep_len[b] positions (int32 [B]; 0: all of
    them, negative: none)."""
    if _calls is not None and type(table) is pldp_page_table and _done("pldp_pages_free", _calls.pages_free(
            table.address, keep_len, stream)):
        return
    t = _table(table)
    _check("pldp_pages_free", _load().pldp_pages_free(t, _dense(keep_len, "keep_len", torch.int32, n=table.B), _stream(stream)))


def pldp_pages_compact(table, copies, n_copies, workspace, used=None, stream=None):
    """Moves the held pages to the front of the pool in the table and refs; copies int32 [at least
    n_pages // 2, 2] and n_copies int32 [1] are what pldp_cache_copy_pages then has to copy in every
    layer, used (int32 [1], optional) the number of held pages."""
    if _calls is not None and type(table) is pldp_page_table and _done("pldp_pages_compact", _calls.pages_compact(
            table.address, copies, n_copies, workspace, used, stream)):
        return
    t = _table(table)
    p, cap = _pairs(copies)
    _check("pldp_pages_compact", _load().pldp_pages_compact(
        t, p, cap, _dense(n_copies, "n_copies", torch.int32, n=1), _dense(used, "used", torch.int32, allow_none=True, n=1),
        _dense(workspace, "workspace"), workspace.numel() * workspace.element_size(), _stream(stream)))


def pldp_cache_copy_pages(cache, copies, n_copies=None, stream=None):
    """Copies pages of one layer's cache, copies[i, 0] to copies[i, 1] (int32 [n, 2]; pairs with an
    entry that is no page are skipped), the first n_copies[0] pairs (int32 [1], None: all)."""
    if _calls is not None and type(cache) is pldp_cache and _done("pldp_cache_copy_pages", _calls.cache_copy_pages(
            cache.address, copies, n_copies, stream)):
        return
    if not isinstance(cache, pldp_cache):
        raise ValueError("cache must be a pldp_cache")
    p, n = _pairs(copies)
    _check("pldp_cache_copy_pages", _load().pldp_cache_copy_pages(
        ctypes.byref(cache.args), p, n, _dense(n_copies, "n_copies", torch.int32, allow_none=True, n=1), _stream(stream)))


def pldp_version() -> int:
    return int(_load().pldp_version())


def pldp_last_error() -> str:
    return _load().pldp_last_error().decode()
