"""ctypes binding of libcaote.so: argument marshalling only, every step runs in the CUDA kernels.

The functions mirror the C entry points one to one and take torch tensors (device memory) in place
of raw pointers. There is no CPU fallback: if the library is missing it is built with nvcc, and if
that fails the import raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

from . import build as _build

BF16, F32 = 0, 1
BASE_MODES = {"last_query": 0, "chunk_sum": 1, "accum": 2, "external": 3}
COMPACT_MODES = {"fill": 0, "stable": 1}

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_CUDA, ERR_TIMEOUT, ERR_BAD_LENGTH, ERR_OVERFLOW = 0, -1, -2, -3, -4, -5, -6
ERR_TOO_LARGE, ERR_BAD_PAGE = -7, -8
STATIC_SCRATCH_BYTES = 16 << 20


class Params(ctypes.Structure):
    """Mirror of caote_params_t."""

    _fields_ = [
        ("batch", ctypes.c_int32),
        ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("capacity", ctypes.c_int32),
        ("n_new", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("base_mode", ctypes.c_int32),
        ("flags", ctypes.c_int32),
    ]


class PagedParams(ctypes.Structure):
    """Mirror of caote_paged_params_t."""

    _fields_ = [
        ("batch", ctypes.c_int32),
        ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("n_pages", ctypes.c_int32),
        ("max_pages", ctypes.c_int32),
        ("total_new", ctypes.c_int32),
        ("max_new", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("flags", ctypes.c_int32),
    ]


class TraceEntry(ctypes.Structure):
    """Mirror of caote_trace_entry_t."""

    _fields_ = [("name", ctypes.c_char * 48), ("launches", ctypes.c_int64), ("total_ms", ctypes.c_double)]


class CaoteError(RuntimeError):
    def __init__(self, fn: str, code: int):
        msg = lib().caote_status_string(code).decode()
        detail = lib().caote_last_cuda_error().decode()
        super().__init__(f"{fn}: {msg} ({code})" + (f": {detail}" if code == ERR_CUDA and detail else ""))
        self.code = code


_lib = None


def library_path() -> str:
    return _build.LIB


def lib() -> ctypes.CDLL:
    """Load (building first if needed) the CUDA library; raises if it cannot be had."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.build()
    if not os.path.exists(path):
        raise ImportError(f"CAOTE CUDA library not found at {path}")
    L = ctypes.CDLL(path)
    vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
    pp = ctypes.POINTER(Params)
    L.caote_workspace_bytes.restype = sz
    L.caote_workspace_bytes.argtypes = [pp]
    L.caote_append.restype = ctypes.c_int
    L.caote_append.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.caote_score.restype = ctypes.c_int
    L.caote_score.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.caote_score_static.restype = ctypes.c_int
    L.caote_score_static.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    L.caote_select_evict.restype = ctypes.c_int
    L.caote_select_evict.argtypes = [pp, vp, vp, vp, vp, vp, i32, vp, vp, sz, vp]
    L.caote_compact.restype = ctypes.c_int
    L.caote_compact.argtypes = [pp, vp, vp, vp, vp, vp, vp, i32, vp, i32, vp, sz, vp]
    L.caote_step.restype = ctypes.c_int
    L.caote_step.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, i32, vp, sz, vp]
    L.caote_step_sum_errors.restype = ctypes.c_int
    L.caote_step_sum_errors.argtypes = L.caote_step.argtypes
    L.caote_step_post_evict.restype = ctypes.c_int
    L.caote_step_post_evict.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, i32, vp, sz, vp]
    L.caote_vsum.restype = ctypes.c_int
    L.caote_vsum.argtypes = [pp, vp, vp, vp, vp]
    L.caote_score_fast.restype = ctypes.c_int
    L.caote_score_fast.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.caote_step_fast.restype = ctypes.c_int
    L.caote_step_fast.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, i32, vp, sz, vp]
    L.caote_score_sum_errors.restype = ctypes.c_int
    L.caote_score_sum_errors.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.caote_post_evict_output.restype = ctypes.c_int
    L.caote_post_evict_output.argtypes = [pp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp]
    L.caote_post_evict_output_ws.restype = ctypes.c_int
    L.caote_post_evict_output_ws.argtypes = [pp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, sz, vp]
    L.caote_read_status.restype = ctypes.c_int
    L.caote_read_status.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_int32)]
    L.caote_status_string.restype = ctypes.c_char_p
    L.caote_status_string.argtypes = [ctypes.c_int]
    L.caote_last_cuda_error.restype = ctypes.c_char_p
    L.caote_last_cuda_error.argtypes = []
    L.caote_trace_enable.restype = ctypes.c_int
    L.caote_trace_enable.argtypes = [ctypes.c_int]
    L.caote_trace_collect.restype = ctypes.c_int
    L.caote_trace_collect.argtypes = [ctypes.POINTER(TraceEntry), i32, ctypes.POINTER(ctypes.c_int32)]
    L.caote_select_evict_greedy.restype = ctypes.c_int
    L.caote_select_evict_greedy.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, sz, vp]
    gp, i64 = ctypes.POINTER(PagedParams), ctypes.c_int64
    L.caote_paged_workspace_bytes.restype = sz
    L.caote_paged_workspace_bytes.argtypes = [gp]
    L.caote_prompt_attend.restype = ctypes.c_int
    L.caote_prompt_attend.argtypes = [gp, vp, i64, vp, vp, i64, vp, vp, vp, vp, vp, sz, vp]
    L.caote_paged_append.restype = ctypes.c_int
    L.caote_paged_append.argtypes = [gp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, vp, vp, vp, sz, vp]
    L.caote_paged_attend.restype = ctypes.c_int
    L.caote_paged_attend.argtypes = [gp, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.caote_paged_evict.restype = ctypes.c_int
    L.caote_paged_evict.argtypes = [gp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, vp, i32, vp, vp, sz, vp]
    L.caote_launch_count.restype = ctypes.c_int64
    L.caote_launch_count.argtypes = []
    L.caote_set_option.restype = ctypes.c_int
    L.caote_set_option.argtypes = [ctypes.c_int32, ctypes.c_int64]
    _lib = L
    return L


def make_params(batch, n_q_heads, n_kv_heads, head_dim, capacity, n_new, dtype, scale, base_mode) -> Params:
    if isinstance(dtype, torch.dtype):
        dtype = {torch.bfloat16: BF16, torch.float32: F32}[dtype]
    if isinstance(base_mode, str):
        base_mode = BASE_MODES[base_mode]
    return Params(batch, n_q_heads, n_kv_heads, head_dim, capacity, n_new, dtype, float(scale), base_mode, 0)


# A step of a small cache takes the GPU some 15 us, so what is done here per call counts: addresses go to ctypes as plain
# integers (the declared argument types convert them) and the library's functions are looked up once. One caote_step call:
# 6.4 us with c_void_p objects made for every pointer, 3.8 us so.
def _p(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


# (torch.cuda.current_stream() makes a Stream object on every call: 3.3 us; the handle alone: 0.2 us.)
def _stream(stream) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check(fn: str, rc: int):
    if rc != 0:
        raise CaoteError(fn, rc)


class _Functions:
    """The library's entry points as attributes; loads the library at the first use of one."""

    def __getattr__(self, name):
        f = getattr(lib(), name)
        setattr(self, name, f)
        return f


_fn = _Functions()


def caote_workspace_bytes(p: Params) -> int:
    return int(_fn.caote_workspace_bytes(ctypes.byref(p)))


def alloc_workspace(p: Params, device) -> torch.Tensor:
    """A zeroed uint8 workspace of the size the library asks for."""
    n = caote_workspace_bytes(p)
    if n == 0:
        raise CaoteError("caote_workspace_bytes", ERR_INVALID_ARG)
    return torch.zeros(n, dtype=torch.uint8, device=device)


def caote_append(p, K, V, base, pos, lens, n_seen, k_new, v_new, workspace, stream=None):
    _check("caote_append", _fn.caote_append(ctypes.byref(p), _p(K), _p(V), _p(base), _p(pos), _p(lens),
                                            _p(n_seen), _p(k_new), _p(v_new), _p(workspace),
                                            workspace.numel(), _stream(stream)))


def caote_score(p, q, K, V, lens, base, o, scores, workspace, stream=None):
    _check("caote_score", _fn.caote_score(ctypes.byref(p), _p(q), _p(K), _p(V), _p(lens), _p(base), _p(o),
                                          _p(scores), _p(workspace), workspace.numel(), _stream(stream)))


def caote_score_static(p, q, K, V, lens, base, o, scores, status_out=None, stream=None):
    """caote_score on the library's built-in scratch array: for callers that may not allocate device
    memory (no workspace argument). ``status_out``: optional int32 device tensor of one element."""
    _check("caote_score_static",
           _fn.caote_score_static(ctypes.byref(p), _p(q), _p(K), _p(V), _p(lens), _p(base), _p(o), _p(scores),
                                  _p(status_out), _stream(stream)))


def caote_select_evict(p, scores, lens, budget, pos, evict_idx, n_evict, workspace, stream=None):
    _check("caote_select_evict",
           _fn.caote_select_evict(ctypes.byref(p), _p(scores), _p(lens), _p(budget), _p(pos), _p(evict_idx),
                                  evict_idx.shape[-1], _p(n_evict), _p(workspace), workspace.numel(),
                                  _stream(stream)))


def caote_select_evict_greedy(p, V, h, lens, budget, pos, evict_idx, order, n_evict, workspace, stream=None):
    _check("caote_select_evict_greedy", _fn.caote_select_evict_greedy(
        ctypes.byref(p), _p(V), _p(h), _p(lens), _p(budget), _p(pos), _p(evict_idx), _p(order), evict_idx.shape[-1],
        _p(n_evict), _p(workspace), workspace.numel() * workspace.element_size(), _stream(stream)))


def caote_compact(p, K, V, base, pos, lens, evict_idx, n_evict, mode, workspace, stream=None):
    if isinstance(mode, str):
        mode = COMPACT_MODES[mode]
    _check("caote_compact",
           _fn.caote_compact(ctypes.byref(p), _p(K), _p(V), _p(base), _p(pos), _p(lens), _p(evict_idx),
                             evict_idx.shape[-1], _p(n_evict), mode, _p(workspace), workspace.numel(),
                             _stream(stream)))


def caote_step(p, q, k_new, v_new, K, V, base, pos, lens, n_seen, budget, o, scores, evict_idx, n_evict, mode,
               workspace, stream=None):
    if isinstance(mode, str):
        mode = COMPACT_MODES[mode]
    _check("caote_step",
           _fn.caote_step(ctypes.byref(p), _p(q), _p(k_new), _p(v_new), _p(K), _p(V), _p(base), _p(pos),
                          _p(lens), _p(n_seen), _p(budget), _p(o), _p(scores), _p(evict_idx),
                          evict_idx.shape[-1], _p(n_evict), mode, _p(workspace), workspace.numel(),
                          _stream(stream)))


def caote_vsum(p, V, lens, vsum, stream=None):
    """vsum[u, :] = sum of the unit's valid V rows (FastCAOTE, Sec. 3.3)."""
    _check("caote_vsum", _fn.caote_vsum(ctypes.byref(p), _p(V), _p(lens), _p(vsum), _stream(stream)))


def caote_score_fast(p, q, K, V, lens, base, vsum, o, scores, workspace, stream=None):
    _check("caote_score_fast",
           _fn.caote_score_fast(ctypes.byref(p), _p(q), _p(K), _p(V), _p(lens), _p(base), _p(vsum), _p(o),
                                _p(scores), _p(workspace), workspace.numel(), _stream(stream)))


def caote_step_fast(p, q, k_new, v_new, K, V, base, pos, lens, n_seen, budget, vsum, o, scores, evict_idx, n_evict,
                    mode, workspace, stream=None):
    if isinstance(mode, str):
        mode = COMPACT_MODES[mode]
    _check("caote_step_fast",
           _fn.caote_step_fast(ctypes.byref(p), _p(q), _p(k_new), _p(v_new), _p(K), _p(V), _p(base), _p(pos),
                               _p(lens), _p(n_seen), _p(budget), _p(vsum), _p(o), _p(scores), _p(evict_idx),
                               evict_idx.shape[-1], _p(n_evict), mode, _p(workspace), workspace.numel(),
                               _stream(stream)))


def caote_score_sum_errors(p, q, K, V, lens, o, scores, workspace, stream=None):
    """Scores as the sum over the counted query rows of the exact single-query eviction errors."""
    _check("caote_score_sum_errors",
           _fn.caote_score_sum_errors(ctypes.byref(p), _p(q), _p(K), _p(V), _p(lens), _p(o), _p(scores),
                                      _p(workspace), workspace.numel(), _stream(stream)))


def caote_step_sum_errors(p, q, k_new, v_new, K, V, base, pos, lens, n_seen, budget, o, scores, evict_idx, n_evict, mode,
                          workspace, stream=None):
    """caote_step with caote_score_sum_errors in the place of caote_score."""
    if isinstance(mode, str):
        mode = COMPACT_MODES[mode]
    _check("caote_step_sum_errors",
           _fn.caote_step_sum_errors(ctypes.byref(p), _p(q), _p(k_new), _p(v_new), _p(K), _p(V), _p(base), _p(pos),
                                     _p(lens), _p(n_seen), _p(budget), _p(o), _p(scores), _p(evict_idx),
                                     evict_idx.shape[-1], _p(n_evict), mode, _p(workspace), workspace.numel(),
                                     _stream(stream)))


def caote_step_post_evict(p, q, k_new, v_new, K, V, base, pos, lens, n_seen, budget, o, o_post, scores, evict_idx,
                          n_evict, mode, workspace, stream=None):
    """caote_step with caote_post_evict_output_ws between selection and compaction."""
    if isinstance(mode, str):
        mode = COMPACT_MODES[mode]
    _check("caote_step_post_evict",
           _fn.caote_step_post_evict(ctypes.byref(p), _p(q), _p(k_new), _p(v_new), _p(K), _p(V), _p(base), _p(pos),
                                     _p(lens), _p(n_seen), _p(budget), _p(o), _p(o_post), _p(scores), _p(evict_idx),
                                     evict_idx.shape[-1], _p(n_evict), mode, _p(workspace), workspace.numel(),
                                     _stream(stream)))


def caote_post_evict_output(p, q, K, V, lens, evict_idx, n_evict, o, o_post, stream=None):
    """Attention output over the retained tokens (call between caote_select_evict and caote_compact)."""
    _check("caote_post_evict_output",
           _fn.caote_post_evict_output(ctypes.byref(p), _p(q), _p(K), _p(V), _p(lens), _p(evict_idx),
                                       evict_idx.shape[-1], _p(n_evict), _p(o), _p(o_post), _stream(stream)))


def caote_post_evict_output_ws(p, q, K, V, lens, evict_idx, n_evict, o, o_post, workspace, stream=None):
    """The same from the softmax statistics the scoring call left in `workspace`, where it left any."""
    _check("caote_post_evict_output_ws",
           _fn.caote_post_evict_output_ws(ctypes.byref(p), _p(q), _p(K), _p(V), _p(lens), _p(evict_idx),
                                          evict_idx.shape[-1], _p(n_evict), _p(o), _p(o_post), _p(workspace),
                                          workspace.numel(), _stream(stream)))


# ---- packed prompts and the paged cache (caote_paged.h) ----------------------------------------------------------
def make_paged_params(batch, n_q_heads, n_kv_heads, head_dim, page_size, n_pages, max_pages, total_new, max_new, dtype,
                      scale) -> PagedParams:
    """Prompts alone: page_size, n_pages and max_pages are 0."""
    if isinstance(dtype, torch.dtype):
        dtype = {torch.bfloat16: BF16, torch.float32: F32}[dtype]
    return PagedParams(batch, n_q_heads, n_kv_heads, head_dim, page_size, n_pages, max_pages, total_new, max_new, dtype,
                       float(scale), 0)


def caote_paged_workspace_bytes(p: PagedParams) -> int:
    return int(_fn.caote_paged_workspace_bytes(ctypes.byref(p)))


def alloc_paged_workspace(p: PagedParams, device) -> torch.Tensor:
    """A zeroed uint8 workspace of the size the library asks for; one for the largest total_new and max_new serves all."""
    n = caote_paged_workspace_bytes(p)
    if n == 0:
        raise CaoteError("caote_paged_workspace_bytes", ERR_INVALID_ARG)
    return torch.zeros(n, dtype=torch.uint8, device=device)


_IO = {BF16: torch.bfloat16, F32: torch.float32}


# What the library cannot see behind a bare address: a tensor's type, size, layout and device. The calls below look for
# themselves, in one expression and without a call per tensor (11 tensors: 3 us; a loop over their descriptions: 8 us, as
# long as the smallest calls take the GPU), and say what was wrong only when something was.
def _refuse(fn, workspace, io, rows, f32, i32):
    """The message for whatever is wrong: groups of {name: (tensor or None, elements)} by type; rows may be packed."""
    here = torch._C._cuda_getDevice()
    if workspace.get_device() != here:
        raise ValueError(f"{fn}: the workspace has to be on the current CUDA device, it is on {workspace.device}")
    for dtype, group in ((io, rows), (torch.float32, f32), (torch.int32, i32)):
        for name, (t, n) in group.items():
            if t is None:
                continue
            if t.get_device() != here:
                raise ValueError(f"{fn}: {name} has to be on the current CUDA device, it is on {t.device}")
            if t.dtype is not dtype or t.numel() != n or (dtype is not io and not t.is_contiguous()):
                raise ValueError(f"{fn}: {name} has to be a contiguous {dtype} tensor of {n} elements, "
                                 f"not {t.dtype} {tuple(t.shape)} with strides {t.stride()}")
    raise ValueError(f"{fn}: pools and outputs have to be contiguous")


def _token_stride(fn, name, t):
    """Elements from one token to the next of a [T, heads, d] tensor that may be a slice of a wider one."""
    T, heads, d = t.shape if t.dim() == 3 else (0, 0, 0)
    s = t.stride()
    if T < 1 or s[2] != 1 or (s[1] != d and heads != 1) or (s[0] <= 0 and T > 1):
        raise ValueError(f"{fn}: {name} needs dense rows [T, heads, d], its shape is {tuple(t.shape)} with strides {s}")
    return s[0] if T > 1 else heads * d


def _pair_stride(fn, k, v):
    """The same for k and v, which have one stride between them."""
    s = _token_stride(fn, "k", k)
    if _token_stride(fn, "v", v) != s:
        raise ValueError(f"{fn}: k and v need the same token stride")
    return s


def check_packed_rows(fn, workspace, q, k, v):
    """Refuses now what the calls below would refuse about q, k and v [T, heads, d] by and by: for callers that make several."""
    if workspace.is_cuda:
        if workspace.get_device() != torch._C._cuda_getDevice():
            raise ValueError(f"{fn}: the current CUDA device has to be {workspace.device}")
        if torch.cuda.is_current_stream_capturing():
            raise ValueError(f"{fn}: cannot be captured into a graph")
    for name, t in (("q", q), ("k", k), ("v", v)):
        s, (_, heads, d) = _token_stride(fn, name, t), t.shape
        if t.data_ptr() % 16 or s * t.element_size() % 16 or not heads * d <= s < 1 << 31:
            raise ValueError(f"{fn}: {name} needs a 16-byte address and a token stride of {heads * d} elements or more, a multiple of "
                             f"16 bytes; it is at {t.data_ptr():#x} with a stride of {s} elements")
    _pair_stride(fn, k, v)


def caote_prompt_attend(p, q, k, v, cu, o, lse, mass, workspace, stream=None):
    """Causal attention inside packed prompts. lse [T, Hq], mass [T, Hkv]: None if not wanted."""
    fn, io, f32, here = "caote_prompt_attend", _IO.get(p.dtype), torch.float32, torch._C._cuda_getDevice()
    nq, nk = p.total_new * p.n_q_heads, p.total_new * p.n_kv_heads
    d, B1 = p.head_dim, p.batch + 1
    if not (workspace.get_device() == here
            and q.dtype is io and q.numel() == nq * d and q.get_device() == here
            and k.dtype is io and k.numel() == nk * d and k.get_device() == here
            and v.dtype is io and v.numel() == nk * d and v.get_device() == here
            and o.dtype is io and o.numel() == nq * d and o.get_device() == here and o.is_contiguous()
            and cu.dtype is torch.int32 and cu.numel() == B1 and cu.get_device() == here and cu.is_contiguous()
            and (lse is None or (lse.dtype is f32 and lse.numel() == nq and lse.get_device() == here and lse.is_contiguous()))
            and (mass is None or (mass.dtype is f32 and mass.numel() == nk and mass.get_device() == here
                                  and mass.is_contiguous()))):
        _refuse(fn, workspace, io, {"q": (q, nq * d), "k": (k, nk * d), "v": (v, nk * d), "o": (o, nq * d)},
                {"lse": (lse, nq), "mass": (mass, nk)}, {"cu": (cu, B1)})
    qs = 0 if q.is_contiguous() else _token_stride(fn, "q", q)
    ks = 0 if k.is_contiguous() and v.is_contiguous() else _pair_stride(fn, k, v)
    _check(fn, _fn.caote_prompt_attend(ctypes.byref(p), q.data_ptr(), qs, k.data_ptr(), v.data_ptr(), ks, cu.data_ptr(),
                                       o.data_ptr(), None if lse is None else lse.data_ptr(),
                                       None if mass is None else mass.data_ptr(), workspace.data_ptr(), workspace.numel(),
                                       _stream(stream)))


def caote_paged_append(p, K, V, mass, pos, page_table, lens, n_seen, k_new, v_new, mass_new, cu, workspace, stream=None):
    """New rows, their positions and their first weights (mass_new [T, Hkv], None: 0) into the pages."""
    fn, io, f32, i32 = "caote_paged_append", _IO.get(p.dtype), torch.float32, torch.int32
    here, B, d = torch._C._cuda_getDevice(), p.batch, p.head_dim
    nk, slots, npt = p.total_new * p.n_kv_heads, p.n_pages * p.n_kv_heads * p.page_size, B * p.max_pages
    if not (workspace.get_device() == here
            and K.dtype is io and K.numel() == slots * d and K.get_device() == here and K.is_contiguous()
            and V.dtype is io and V.numel() == slots * d and V.get_device() == here and V.is_contiguous()
            and (mass is None or (mass.dtype is f32 and mass.numel() == slots and mass.get_device() == here
                                  and mass.is_contiguous()))
            and (pos is None or (pos.dtype is i32 and pos.numel() == slots and pos.get_device() == here and pos.is_contiguous()))
            and page_table.dtype is i32 and page_table.numel() == npt and page_table.get_device() == here
            and page_table.is_contiguous()
            and lens.dtype is i32 and lens.numel() == B and lens.get_device() == here and lens.is_contiguous()
            and (n_seen is None or (n_seen.dtype is i32 and n_seen.numel() == B and n_seen.get_device() == here
                                    and n_seen.is_contiguous()))
            and k_new.dtype is io and k_new.numel() == nk * d and k_new.get_device() == here
            and v_new.dtype is io and v_new.numel() == nk * d and v_new.get_device() == here
            and (mass_new is None or (mass_new.dtype is f32 and mass_new.numel() == nk and mass_new.get_device() == here
                                      and mass_new.is_contiguous()))
            and cu.dtype is i32 and cu.numel() == B + 1 and cu.get_device() == here and cu.is_contiguous()):
        _refuse(fn, workspace, io, {"K": (K, slots * d), "V": (V, slots * d), "k_new": (k_new, nk * d), "v_new": (v_new, nk * d)},
                {"mass": (mass, slots), "mass_new": (mass_new, nk)},
                {"pos": (pos, slots), "page_table": (page_table, npt), "lens": (lens, B), "n_seen": (n_seen, B), "cu": (cu, B + 1)})
    ks = 0 if k_new.is_contiguous() and v_new.is_contiguous() else _pair_stride(fn, k_new, v_new)
    _check(fn, _fn.caote_paged_append(ctypes.byref(p), K.data_ptr(), V.data_ptr(), None if mass is None else mass.data_ptr(),
                                      None if pos is None else pos.data_ptr(), page_table.data_ptr(), lens.data_ptr(),
                                      None if n_seen is None else n_seen.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), ks,
                                      None if mass_new is None else mass_new.data_ptr(), cu.data_ptr(), workspace.data_ptr(),
                                      workspace.numel(), _stream(stream)))


def caote_paged_attend(p, q, K, V, mass, page_table, lens, cu, o, lse, workspace, stream=None):
    """Attention of the new tokens, the last ones of their sequences' pages. mass (None: not wanted) is added to."""
    fn, io, f32, i32 = "caote_paged_attend", _IO.get(p.dtype), torch.float32, torch.int32
    here, B, d = torch._C._cuda_getDevice(), p.batch, p.head_dim
    nq, slots, npt = p.total_new * p.n_q_heads, p.n_pages * p.n_kv_heads * p.page_size, B * p.max_pages
    if not (workspace.get_device() == here
            and q.dtype is io and q.numel() == nq * d and q.get_device() == here
            and K.dtype is io and K.numel() == slots * d and K.get_device() == here and K.is_contiguous()
            and V.dtype is io and V.numel() == slots * d and V.get_device() == here and V.is_contiguous()
            and (mass is None or (mass.dtype is f32 and mass.numel() == slots and mass.get_device() == here
                                  and mass.is_contiguous()))
            and page_table.dtype is i32 and page_table.numel() == npt and page_table.get_device() == here
            and page_table.is_contiguous()
            and lens.dtype is i32 and lens.numel() == B and lens.get_device() == here and lens.is_contiguous()
            and cu.dtype is i32 and cu.numel() == B + 1 and cu.get_device() == here and cu.is_contiguous()
            and o.dtype is io and o.numel() == nq * d and o.get_device() == here and o.is_contiguous()
            and (lse is None or (lse.dtype is f32 and lse.numel() == nq and lse.get_device() == here and lse.is_contiguous()))):
        _refuse(fn, workspace, io, {"q": (q, nq * d), "K": (K, slots * d), "V": (V, slots * d), "o": (o, nq * d)},
                {"mass": (mass, slots), "lse": (lse, nq)},
                {"page_table": (page_table, npt), "lens": (lens, B), "cu": (cu, B + 1)})
    qs = 0 if q.is_contiguous() else _token_stride(fn, "q", q)
    _check(fn, _fn.caote_paged_attend(ctypes.byref(p), q.data_ptr(), qs, K.data_ptr(), V.data_ptr(),
                                      None if mass is None else mass.data_ptr(), page_table.data_ptr(), lens.data_ptr(),
                                      cu.data_ptr(), o.data_ptr(), None if lse is None else lse.data_ptr(),
                                      workspace.data_ptr(), workspace.numel(), _stream(stream)))


def caote_paged_evict(p, K, V, mass, pos, page_table, lens, n_seen, budget, sinks, recent, evict_idx, n_evict, workspace,
                      stream=None):
    """The lightest tokens beyond the budget leave the pages; the first `sinks` and the `recent` newest go last."""
    fn, io, f32, i32 = "caote_paged_evict", _IO.get(p.dtype), torch.float32, torch.int32
    here, B, Hkv = torch._C._cuda_getDevice(), p.batch, p.n_kv_heads
    slots, npt, most = p.n_pages * Hkv * p.page_size, B * p.max_pages, evict_idx.shape[-1]
    rows, picks = slots * p.head_dim, B * Hkv * most
    if not (workspace.get_device() == here
            and K.dtype is io and K.numel() == rows and K.get_device() == here and K.is_contiguous()
            and V.dtype is io and V.numel() == rows and V.get_device() == here and V.is_contiguous()
            and mass.dtype is f32 and mass.numel() == slots and mass.get_device() == here and mass.is_contiguous()
            and pos.dtype is i32 and pos.numel() == slots and pos.get_device() == here and pos.is_contiguous()
            and page_table.dtype is i32 and page_table.numel() == npt and page_table.get_device() == here
            and page_table.is_contiguous()
            and lens.dtype is i32 and lens.numel() == B and lens.get_device() == here and lens.is_contiguous()
            and n_seen.dtype is i32 and n_seen.numel() == B and n_seen.get_device() == here and n_seen.is_contiguous()
            and budget.dtype is i32 and budget.numel() == B and budget.get_device() == here and budget.is_contiguous()
            and evict_idx.dtype is i32 and evict_idx.numel() == picks and evict_idx.get_device() == here
            and evict_idx.is_contiguous()
            and n_evict.dtype is i32 and n_evict.numel() == B and n_evict.get_device() == here and n_evict.is_contiguous()):
        _refuse(fn, workspace, io, {"K": (K, rows), "V": (V, rows)}, {"mass": (mass, slots)},
                {"pos": (pos, slots), "page_table": (page_table, npt), "lens": (lens, B), "n_seen": (n_seen, B),
                 "budget": (budget, B), "evict_idx": (evict_idx, picks), "n_evict": (n_evict, B)})
    _check(fn, _fn.caote_paged_evict(ctypes.byref(p), K.data_ptr(), V.data_ptr(), mass.data_ptr(), pos.data_ptr(),
                                     page_table.data_ptr(), lens.data_ptr(), n_seen.data_ptr(), budget.data_ptr(), sinks, recent,
                                     evict_idx.data_ptr(), most, n_evict.data_ptr(), workspace.data_ptr(), workspace.numel(),
                                     _stream(stream)))


def caote_read_status(workspace, stream=None) -> int:
    out = ctypes.c_int32(0)
    _check("caote_read_status", _fn.caote_read_status(_p(workspace), _stream(stream), ctypes.byref(out)))
    return int(out.value)


def caote_status_string(code: int) -> str:
    return _fn.caote_status_string(code).decode()


def caote_trace_enable(on: bool) -> None:
    _check("caote_trace_enable", _fn.caote_trace_enable(1 if on else 0))


def caote_trace_collect(max_entries: int = 32) -> dict:
    """{kernel name: (launches, total_ms)} since the last collect."""
    buf = (TraceEntry * max_entries)()
    n = ctypes.c_int32(0)
    _check("caote_trace_collect", _fn.caote_trace_collect(buf, max_entries, ctypes.byref(n)))
    return {buf[i].name.decode(): (int(buf[i].launches), float(buf[i].total_ms)) for i in range(n.value)}


OPT_WAIT_CYCLES, OPT_DECODE_CLUSTER, OPT_SIDE_BY_SIDE = 1, 2, 3


def caote_set_option(option: int, value: int) -> None:
    _check("caote_set_option", _fn.caote_set_option(int(option), int(value)))


def caote_launch_count() -> int:
    return int(_fn.caote_launch_count())
