"""Binding of libgsd.so with the same names as the C ABI (include/gsd.h).  The calls of a serving
iteration go through a CPython extension (csrc/gsd_native.cpp) when their arguments are the plain
case, and through ctypes otherwise; both load the same library.

The functions take torch tensors (CUDA tensors for the device calls, CPU tensors for the
host-buffer step), check dtype / shape / contiguity, and pass raw pointers, sizes and the
current CUDA stream.  PyTorch is used for memory and streams only.
"""
from __future__ import annotations

import ctypes
import os
import warnings
from typing import Optional, Sequence, Tuple

import torch

GSD_ATTN_AUTO, GSD_ATTN_MMA, GSD_ATTN_TCGEN05 = 0, 1, 2
GSD_ATTN_SPLIT_BALANCED = -1      # num_splits: equal shares of key tiles per CTA, dealt out on the device
GSD_ATTN_SPLIT_PER_SEQUENCE = -2  # num_splits: a split count per sequence, chosen on the device

GSD_ROTARY_HALVES, GSD_ROTARY_NEIGHBOURS = 0, 1

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libgsd.so")
_lib: Optional[ctypes.CDLL] = None


class GsdError(RuntimeError):
    """A negative gsd_status returned by the library."""

    def __init__(self, code: int, what: str):
        super().__init__(what)
        self.code = code


class AttnParams(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("N", ctypes.c_int32), ("Hq", ctypes.c_int32),
                ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32), ("Lmax", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float), ("num_splits", ctypes.c_int32),
                ("kernel", ctypes.c_int32)]


class CommitParams(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("N", ctypes.c_int32), ("Hkv", ctypes.c_int32),
                ("D", ctypes.c_int32), ("Lmax", ctypes.c_int32), ("Tcap", ctypes.c_int32)]


class AcceptParams(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("N", ctypes.c_int32), ("V", ctypes.c_int32),
                ("Ecap", ctypes.c_int32), ("Tcap", ctypes.c_int32)]


class DraftParams(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("F", ctypes.c_int32), ("V", ctypes.c_int32),
                ("Ncap", ctypes.c_int32), ("k", ctypes.c_int32), ("tau", ctypes.c_int32),
                ("theta_prob", ctypes.c_float), ("theta_sib", ctypes.c_float)]


class Kv8Params(ctypes.Structure):
    _fields_ = [("format", ctypes.c_int32), ("block", ctypes.c_int32)]


class AppendParams(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("T", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32),
                ("Lmax", ctypes.c_int32)]


class PageParams(ctypes.Structure):
    _fields_ = [("page", ctypes.c_int32), ("num_pages", ctypes.c_int32), ("max_pages", ctypes.c_int32)]


class Rotation(ctypes.Structure):
    _fields_ = [("pairs", ctypes.c_int32), ("layout", ctypes.c_int32), ("axes", ctypes.c_int32), ("axis", ctypes.c_uint8 * 64)]


class RotaryParams(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("T", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32),
                ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64)]


class AppendPagedParams(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("T", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32),
                ("Lmax", ctypes.c_int32), ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64)]


class LogprobsParams(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("N", ctypes.c_int32), ("V", ctypes.c_int32), ("T", ctypes.c_int32),
                ("k", ctypes.c_int32)]


EXPORTS = ["gsd_version", "gsd_status_string", "gsd_last_cuda_error", "gsd_debug_attn_wait", "gsd_verify_attn",
           "gsd_verify_attn_workspace_bytes", "gsd_verify_attn_num_splits", "gsd_accept",
           "gsd_accept_workspace_bytes", "gsd_accept_static", "gsd_accept_sampled",
           "gsd_accept_sampled_workspace_bytes", "gsd_draft_expand", "gsd_draft_expand_workspace_bytes",
           "gsd_commit_kv", "gsd_build_mask", "gsd_unmerge_tree", "gsd_verify_step_host",
           "gsd_verify_step_host_arena_bytes", "gsd_verify_attn_q8", "gsd_verify_attn_q8_workspace_bytes",
           "gsd_commit_kv_q8", "gsd_append_kv_q8", "gsd_token_logprobs", "gsd_token_logprobs_workspace_bytes",
           "gsd_verify_attn_paged", "gsd_verify_attn_paged_workspace_bytes", "gsd_commit_kv_paged", "gsd_append_kv_paged",
           "gsd_rotary"]


def library_path() -> str:
    return _LIB_PATH


def lib() -> ctypes.CDLL:
    """Load libgsd.so (built in-tree by paper_2407_16207_b200/build.py). No fallback."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise GsdError(-100, f"{_LIB_PATH} is missing: run `python -m paper_2407_16207_b200.build` "
                                 "(there is no CPU fallback)")
        L = ctypes.CDLL(_LIB_PATH)
        vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
        L.gsd_version.restype = i32
        L.gsd_status_string.restype = ctypes.c_char_p
        L.gsd_status_string.argtypes = [i32]
        L.gsd_last_cuda_error.restype = ctypes.c_char_p
        L.gsd_debug_attn_wait.restype = None
        L.gsd_debug_attn_wait.argtypes = [ctypes.c_uint64, ctypes.c_int32]
        L.gsd_verify_attn.restype = i32
        L.gsd_verify_attn.argtypes = [vp] * 8 + [ctypes.POINTER(AttnParams), vp, sz, vp, vp]
        L.gsd_verify_attn_workspace_bytes.restype = sz
        L.gsd_verify_attn_workspace_bytes.argtypes = [ctypes.POINTER(AttnParams)]
        L.gsd_verify_attn_num_splits.restype = i32
        L.gsd_verify_attn_num_splits.argtypes = [ctypes.POINTER(AttnParams)]
        L.gsd_accept.restype = i32
        L.gsd_accept.argtypes = [vp] * 7 + [ctypes.POINTER(AcceptParams), vp, sz, vp, vp]
        L.gsd_accept_sampled.restype = i32
        L.gsd_accept_sampled.argtypes = [vp] * 11 + [ctypes.POINTER(AcceptParams), vp, sz, vp, vp]
        L.gsd_accept_sampled_workspace_bytes.restype = sz
        L.gsd_accept_sampled_workspace_bytes.argtypes = [ctypes.POINTER(AcceptParams)]
        L.gsd_draft_expand.restype = i32
        L.gsd_draft_expand.argtypes = [vp] * 11 + [ctypes.POINTER(DraftParams), vp, sz, vp, vp]
        L.gsd_draft_expand_workspace_bytes.restype = sz
        L.gsd_draft_expand_workspace_bytes.argtypes = [ctypes.POINTER(DraftParams)]
        L.gsd_accept_static.restype = i32
        L.gsd_accept_static.argtypes = [vp] * 7 + [ctypes.POINTER(AcceptParams), vp, vp]
        L.gsd_build_mask.restype = i32
        L.gsd_build_mask.argtypes = [vp, vp, vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, vp, vp]
        L.gsd_unmerge_tree.restype = i32
        L.gsd_unmerge_tree.argtypes = [vp] * 7 + [ctypes.c_int32] * 5 + [vp, vp]
        L.gsd_commit_kv.restype = i32
        L.gsd_commit_kv.argtypes = [vp] * 7 + [ctypes.POINTER(CommitParams), vp, vp]
        L.gsd_accept_workspace_bytes.restype = sz
        L.gsd_accept_workspace_bytes.argtypes = [ctypes.POINTER(AcceptParams)]
        L.gsd_verify_step_host.restype = i32
        L.gsd_verify_step_host.argtypes = ([vp] * 8 + [ctypes.POINTER(AttnParams)] + [vp] * 7
                                           + [ctypes.POINTER(AcceptParams), vp, sz, vp, vp])
        L.gsd_verify_step_host_arena_bytes.restype = sz
        L.gsd_verify_step_host_arena_bytes.argtypes = [ctypes.POINTER(AttnParams),
                                                       ctypes.POINTER(AcceptParams)]
        kv8 = ctypes.POINTER(Kv8Params)
        L.gsd_verify_attn_q8.restype = i32
        L.gsd_verify_attn_q8.argtypes = [vp] * 10 + [ctypes.POINTER(AttnParams), kv8, vp, sz, vp, vp]
        L.gsd_verify_attn_q8_workspace_bytes.restype = sz
        L.gsd_verify_attn_q8_workspace_bytes.argtypes = [ctypes.POINTER(AttnParams), kv8]
        L.gsd_commit_kv_q8.restype = i32
        L.gsd_commit_kv_q8.argtypes = [vp] * 9 + [ctypes.POINTER(CommitParams), kv8, vp, vp]
        L.gsd_append_kv_q8.restype = i32
        L.gsd_append_kv_q8.argtypes = [vp] * 8 + [ctypes.POINTER(AppendParams), kv8, vp, vp]
        L.gsd_token_logprobs.restype = i32
        L.gsd_token_logprobs.argtypes = [vp] * 8 + [ctypes.POINTER(LogprobsParams), vp, sz, vp, vp]
        L.gsd_token_logprobs_workspace_bytes.restype = sz
        L.gsd_token_logprobs_workspace_bytes.argtypes = [ctypes.POINTER(LogprobsParams)]
        page, rot = ctypes.POINTER(PageParams), ctypes.POINTER(Rotation)
        L.gsd_verify_attn_paged.restype = i32
        L.gsd_verify_attn_paged.argtypes = [vp] * 9 + [ctypes.POINTER(AttnParams), page, vp, sz, vp, vp]
        L.gsd_verify_attn_paged_workspace_bytes.restype = sz
        L.gsd_verify_attn_paged_workspace_bytes.argtypes = [ctypes.POINTER(AttnParams), page]
        L.gsd_commit_kv_paged.restype = i32
        L.gsd_commit_kv_paged.argtypes = [vp] * 8 + [ctypes.POINTER(CommitParams), page, vp, vp]
        L.gsd_append_kv_paged.restype = i32
        L.gsd_append_kv_paged.argtypes = [vp] * 10 + [ctypes.POINTER(AppendPagedParams), page, rot, vp, vp]
        L.gsd_rotary.restype = i32
        L.gsd_rotary.argtypes = [vp] * 7 + [ctypes.POINTER(RotaryParams), rot, vp]
        _lib = L
    return _lib


# The library's functions the extension calls, in the order of its table.
_NATIVE_CALLS = ("gsd_verify_attn", "gsd_verify_attn_workspace_bytes", "gsd_accept", "gsd_accept_workspace_bytes",
                 "gsd_accept_sampled", "gsd_accept_sampled_workspace_bytes", "gsd_binding_draft_expand",
                 "gsd_draft_expand_workspace_bytes", "gsd_build_mask", "gsd_commit_kv", "gsd_verify_attn_q8",
                 "gsd_verify_attn_q8_workspace_bytes", "gsd_commit_kv_q8", "gsd_append_kv_q8", "gsd_token_logprobs",
                 "gsd_token_logprobs_workspace_bytes", "gsd_verify_attn_paged", "gsd_verify_attn_paged_workspace_bytes",
                 "gsd_commit_kv_paged", "gsd_append_kv_paged", "gsd_rotary")
_native = None
_native_lib: Optional[ctypes.CDLL] = None      # the library the extension is bound to


def native():
    """The CPython extension (built in-tree beside the library), bound to the loaded library."""
    global _native, _native_lib
    L = lib()
    if _native is None:
        try:
            from . import _native as module
        except ImportError as e:
            raise GsdError(-100, f"the extension _native.so is missing or does not load ({e}): run "
                                 "`python -m paper_2407_16207_b200.build`") from e
        if module.torch_version != torch.__version__:
            raise GsdError(-100, f"the extension _native.so was built against torch {module.torch_version}, this is "
                                 f"{torch.__version__}: run `python -m paper_2407_16207_b200.build`")
        _native = module
    if _native_lib is not L:
        _native.bind(*(ctypes.cast(getattr(L, name), ctypes.c_void_p).value for name in _NATIVE_CALLS))
        _native_lib = L
    return _native


class _Declines:
    """In the extension's place where it cannot be loaded: takes no call."""

    def __getattr__(self, name):
        return lambda *args: None


_declines: Optional[_Declines] = None


def _marshal():
    """What the calls try first: the extension, or nothing but the ctypes path if it does not load (the
    library and its kernels are the same, a call takes 20 us longer)."""
    global _declines
    if _native is not None and _lib is not None and _lib is _native_lib:
        return _native
    if _declines is None:
        lib()                                   # (a missing library is an error)
        try:
            return native()
        except GsdError as e:
            _declines = _Declines()
            warnings.warn(f"{e}; the calls go through ctypes", RuntimeWarning, stacklevel=3)
    return _declines


def _check(rc: int) -> None:
    if rc != 0:
        L = lib()
        msg = L.gsd_status_string(rc).decode()
        detail = L.gsd_last_cuda_error().decode()
        if rc == -5 or (rc == -4 and detail.startswith("gsd_accept_static")):
            msg += ": " + detail
        raise GsdError(rc, f"gsd error {rc}: {msg}")


def gsd_version() -> int:
    return int(lib().gsd_version())


def gsd_debug_attn_wait(limit_ns: int = 0, withhold_first_k: bool = False) -> None:
    """Test hook for the bounded in-kernel waits of the tcgen05 attention kernel; see
    gsd_debug_attn_wait in include/gsd.h.  (0, False) restores the defaults."""
    lib().gsd_debug_attn_wait(int(limit_ns), 1 if withhold_first_k else 0)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _want(t: torch.Tensor, dtype, shape, name: str, cuda: bool) -> None:
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name}: expected contiguous {dtype} {tuple(shape)}, got {t.dtype} "
                         f"{tuple(t.shape)}")
    if t.is_cuda != cuda:
        raise ValueError(f"{name}: expected a {'CUDA' if cuda else 'CPU'} tensor")


def _stream(t: torch.Tensor) -> int:
    return torch.cuda.current_stream(t.device).cuda_stream


def _attn_params(q, k_cache, draft_k, softmax_scale, num_splits, kernel) -> AttnParams:
    B, N, Hq, D = q.shape
    Lmax, Hkv = k_cache.shape[1], k_cache.shape[2]
    return AttnParams(B, N, Hq, Hkv, D, Lmax, float(softmax_scale), int(num_splits), int(kernel))


def _check_attn_tensors(q, k_cache, v_cache, draft_k, draft_v, ancestor_mask, seq_lens, cuda):
    bf = torch.bfloat16
    if q.dim() != 4 or k_cache.dim() != 4:
        raise ValueError("q must be [B,N,Hq,D] and k_cache [B,Lmax,Hkv,D]")
    B, N, Hq, D = q.shape
    Lmax, Hkv = k_cache.shape[1], k_cache.shape[2]
    _want(q, bf, (B, N, Hq, D), "q", cuda)
    _want(k_cache, bf, (B, Lmax, Hkv, D), "k_cache", cuda)
    _want(v_cache, bf, (B, Lmax, Hkv, D), "v_cache", cuda)
    _want(draft_k, bf, (B, N, Hkv, D), "draft_k", cuda)
    _want(draft_v, bf, (B, N, Hkv, D), "draft_v", cuda)
    if ancestor_mask.dtype not in (torch.int32, torch.uint32):
        raise ValueError("ancestor_mask must hold 32-bit words (int32 or uint32)")
    _want(ancestor_mask, ancestor_mask.dtype, (B, N, (N + 31) // 32), "ancestor_mask", cuda)
    _want(seq_lens, torch.int32, (B,), "seq_lens", cuda)


def gsd_verify_attn_num_splits(B, N, Hq, Hkv, D, Lmax, num_splits=0, kernel=GSD_ATTN_AUTO) -> int:
    p = AttnParams(B, N, Hq, Hkv, D, Lmax, 0.0, num_splits, kernel)
    return int(lib().gsd_verify_attn_num_splits(ctypes.byref(p)))


def gsd_verify_attn_workspace_bytes(B, N, Hq, Hkv, D, Lmax, num_splits=0,
                                    kernel=GSD_ATTN_AUTO) -> int:
    p = AttnParams(B, N, Hq, Hkv, D, Lmax, 0.0, num_splits, kernel)
    return int(lib().gsd_verify_attn_workspace_bytes(ctypes.byref(p)))


def gsd_verify_attn(q, k_cache, v_cache, draft_k, draft_v, ancestor_mask, seq_lens,
                    out: Optional[torch.Tensor] = None, *, softmax_scale: float = 0.0,
                    num_splits: int = 0, kernel: int = GSD_ATTN_AUTO,
                    workspace: Optional[torch.Tensor] = None,
                    status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """DAG-masked attention of the draft nodes; see gsd_verify_attn in include/gsd.h.
    Enqueued on the current stream; returns `out` [B,N,Hq,D] bf16."""
    fast = _native if _lib is not None and _lib is _native_lib else _marshal()
    r = fast.verify_attn(q, k_cache, v_cache, draft_k, draft_v, ancestor_mask, seq_lens, out, softmax_scale, num_splits, kernel,
                         workspace, status)
    if r is not None:
        if r.__class__ is int:
            _check(r)
        return r
    _check_attn_tensors(q, k_cache, v_cache, draft_k, draft_v, ancestor_mask, seq_lens, True)
    if out is None:
        out = torch.empty_like(q)
    _want(out, torch.bfloat16, q.shape, "out", True)
    p = _attn_params(q, k_cache, draft_k, softmax_scale, num_splits, kernel)
    L = lib()
    with torch.cuda.device(q.device):
        need = int(L.gsd_verify_attn_workspace_bytes(ctypes.byref(p)))
        if workspace is None and need:
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        _check(L.gsd_verify_attn(q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                                 draft_k.data_ptr(), draft_v.data_ptr(), ancestor_mask.data_ptr(),
                                 seq_lens.data_ptr(), out.data_ptr(), ctypes.byref(p),
                                 _ptr(workspace), ws_bytes, _ptr(status), _stream(q)))
    return out


def gsd_accept_workspace_bytes(B, N, V=1, Ecap=1, Tcap=1) -> int:
    p = AcceptParams(B, N, V, Ecap, Tcap)
    return int(lib().gsd_accept_workspace_bytes(ctypes.byref(p)))


def gsd_accept(logits, draft_tokens, parent_ptr, parent_idx, *, Tcap: int = 0,
               want_nodes: bool = True, workspace: Optional[torch.Tensor] = None,
               status: Optional[torch.Tensor] = None,
               out: Optional[Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]] = None
               ) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """Greedy verification + longest accepted path; see gsd_accept in include/gsd.h.
    Returns (accepted_tokens [B,Tcap], accepted_len [B], accepted_nodes [B,Tcap] or None)."""
    if out is None:
        fast = _native if _lib is not None and _lib is _native_lib else _marshal()
        r = fast.accept(logits, draft_tokens, parent_ptr, parent_idx, Tcap, want_nodes, workspace, status)
        if r is not None:
            if r.__class__ is int:
                _check(r)
            return r
    if logits.dim() != 3:
        raise ValueError("logits must be [B,N,V]")
    B, N, V = logits.shape
    _want(logits, torch.float32, (B, N, V), "logits", True)
    _want(draft_tokens, torch.int32, (B, N), "draft_tokens", True)
    _want(parent_ptr, torch.int32, (B, N + 1), "parent_ptr", True)
    if parent_idx.dim() != 2:
        raise ValueError("parent_idx must be [B,Ecap]")
    Ecap = parent_idx.shape[1]
    _want(parent_idx, torch.int32, (B, Ecap), "parent_idx", True)
    Tcap = Tcap or N
    if out is None:
        toks = torch.empty((B, Tcap), dtype=torch.int32, device=logits.device)
        lens = torch.empty((B,), dtype=torch.int32, device=logits.device)
        nodes = torch.empty((B, Tcap), dtype=torch.int32, device=logits.device) if want_nodes else None
    else:
        toks, lens, nodes = out
    p = AcceptParams(B, N, V, Ecap, Tcap)
    L = lib()
    with torch.cuda.device(logits.device):
        need = int(L.gsd_accept_workspace_bytes(ctypes.byref(p)))
        if workspace is None:
            workspace = torch.empty(max(need, 8), dtype=torch.uint8, device=logits.device)
        _check(L.gsd_accept(logits.data_ptr(), draft_tokens.data_ptr(), parent_ptr.data_ptr(),
                            parent_idx.data_ptr(), toks.data_ptr(), lens.data_ptr(), _ptr(nodes),
                            ctypes.byref(p), workspace.data_ptr(),
                            workspace.numel() * workspace.element_size(), _ptr(status),
                            _stream(logits)))
    return toks, lens, nodes


def gsd_accept_sampled_workspace_bytes(B, N) -> int:
    p = AcceptParams(B, N, 1, 1, 1)
    return int(lib().gsd_accept_sampled_workspace_bytes(ctypes.byref(p)))


def gsd_accept_sampled(logits, draft_tokens, parent_ptr, parent_idx, draft_q, u_accept, u_sample, *,
                       draft_logits: Optional[torch.Tensor] = None,
                       Tcap: int = 0, want_nodes: bool = True, workspace: Optional[torch.Tensor] = None,
                       status: Optional[torch.Tensor] = None,
                       out: Optional[Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]] = None
                       ) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """Non-deterministic verification with the random numbers passed in; see gsd_accept_sampled in
    include/gsd.h.  `draft_logits` [B,N,V] (optional) makes the regenerated token come from the
    residual max(0, P - Q).  Returns (accepted_tokens [B,Tcap], accepted_len [B], accepted_nodes
    or None)."""
    if out is None:
        fast = _native if _lib is not None and _lib is _native_lib else _marshal()
        r = fast.accept_sampled(logits, draft_tokens, parent_ptr, parent_idx, draft_q, u_accept, u_sample, draft_logits, Tcap,
                                want_nodes, workspace, status)
        if r is not None:
            if r.__class__ is int:
                _check(r)
            return r
    if logits.dim() != 3:
        raise ValueError("logits must be [B,N,V]")
    B, N, V = logits.shape
    _want(logits, torch.float32, (B, N, V), "logits", True)
    _want(draft_tokens, torch.int32, (B, N), "draft_tokens", True)
    _want(parent_ptr, torch.int32, (B, N + 1), "parent_ptr", True)
    if parent_idx.dim() != 2:
        raise ValueError("parent_idx must be [B,Ecap]")
    Ecap = parent_idx.shape[1]
    _want(parent_idx, torch.int32, (B, Ecap), "parent_idx", True)
    _want(draft_q, torch.float32, (B, N), "draft_q", True)
    _want(u_accept, torch.float32, (B, N), "u_accept", True)
    _want(u_sample, torch.float32, (B,), "u_sample", True)
    if draft_logits is not None:
        _want(draft_logits, torch.float32, (B, N, V), "draft_logits", True)
    Tcap = Tcap or N
    if out is None:
        toks = torch.empty((B, Tcap), dtype=torch.int32, device=logits.device)
        lens = torch.empty((B,), dtype=torch.int32, device=logits.device)
        nodes = torch.empty((B, Tcap), dtype=torch.int32, device=logits.device) if want_nodes else None
    else:
        toks, lens, nodes = out
        _want(toks, torch.int32, (B, Tcap), "accepted_tokens", True)
        _want(lens, torch.int32, (B,), "accepted_len", True)
    p = AcceptParams(B, N, V, Ecap, Tcap)
    L = lib()
    with torch.cuda.device(logits.device):
        need = int(L.gsd_accept_sampled_workspace_bytes(ctypes.byref(p)))
        if workspace is None:
            workspace = torch.empty(max(need, 8), dtype=torch.uint8, device=logits.device)
        _check(L.gsd_accept_sampled(logits.data_ptr(), draft_tokens.data_ptr(), parent_ptr.data_ptr(),
                                    parent_idx.data_ptr(), _ptr(draft_logits), draft_q.data_ptr(),
                                    u_accept.data_ptr(),
                                    u_sample.data_ptr(), toks.data_ptr(), lens.data_ptr(), _ptr(nodes),
                                    ctypes.byref(p), workspace.data_ptr(),
                                    workspace.numel() * workspace.element_size(), _ptr(status),
                                    _stream(logits)))
    return toks, lens, nodes


def gsd_draft_expand(logits, frontier, frontier_len, tokens, tree_parent, merge_to, leaf, prob, num_nodes, *,
                     k: int, tau: int, theta_prob: float, theta_sib: float,
                     workspace: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                     out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None
                     ) -> Tuple[torch.Tensor, torch.Tensor]:
    """One growth step of the draft token graph, in place; see gsd_draft_expand in include/gsd.h.
    Returns (new_frontier [B,F*k], new_frontier_len [B])."""
    if out is None:
        fast = _native if _lib is not None and _lib is _native_lib else _marshal()
        r = fast.draft_expand(logits, frontier, frontier_len, tokens, tree_parent, merge_to, leaf, prob, num_nodes, k, tau,
                              theta_prob, theta_sib, workspace, status)
        if r is not None:
            if r.__class__ is int:
                _check(r)
            return r
    if logits.dim() != 3:
        raise ValueError("logits must be [B,F,V]")
    B, F, V = logits.shape
    Ncap = tokens.shape[1]
    _want(logits, torch.float32, (B, F, V), "logits", True)
    _want(frontier, torch.int32, (B, F), "frontier", True)
    _want(frontier_len, torch.int32, (B,), "frontier_len", True)
    for name, t, dt in (("tokens", tokens, torch.int32), ("tree_parent", tree_parent, torch.int32),
                        ("merge_to", merge_to, torch.int32), ("leaf", leaf, torch.uint8), ("prob", prob, torch.float32)):
        _want(t, dt, (B, Ncap), name, True)
    _want(num_nodes, torch.int32, (B,), "num_nodes", True)
    if out is None:
        nf = torch.full((B, F * k), -1, dtype=torch.int32, device=logits.device)
        nfl = torch.zeros((B,), dtype=torch.int32, device=logits.device)
    else:
        nf, nfl = out
        _want(nf, torch.int32, (B, F * k), "new_frontier", True)
        _want(nfl, torch.int32, (B,), "new_frontier_len", True)
    p = DraftParams(B, F, V, Ncap, int(k), int(tau), float(theta_prob), float(theta_sib))
    L = lib()
    with torch.cuda.device(logits.device):
        need = int(L.gsd_draft_expand_workspace_bytes(ctypes.byref(p)))
        if workspace is None:
            workspace = torch.empty(max(need, 8), dtype=torch.uint8, device=logits.device)
        _check(L.gsd_draft_expand(logits.data_ptr(), frontier.data_ptr(), frontier_len.data_ptr(),
                                  tokens.data_ptr(), tree_parent.data_ptr(), merge_to.data_ptr(), leaf.data_ptr(),
                                  prob.data_ptr(), num_nodes.data_ptr(), nf.data_ptr(), nfl.data_ptr(),
                                  ctypes.byref(p), workspace.data_ptr(),
                                  workspace.numel() * workspace.element_size(), _ptr(status), _stream(logits)))
    return nf, nfl


def gsd_build_mask(parent_ptr, parent_idx, out: Optional[torch.Tensor] = None, *,
                   status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Ancestor bitmask [B,N,ceil(N/32)] (int32 words) from the parent CSR; see gsd_build_mask in
    include/gsd.h.  Enqueued on the current stream."""
    fast = _native if _lib is not None and _lib is _native_lib else _marshal()
    r = fast.build_mask(parent_ptr, parent_idx, out, status)
    if r is not None:
        if r.__class__ is int:
            _check(r)
        return r
    B, N1 = parent_ptr.shape
    N = N1 - 1
    Ecap = parent_idx.shape[1]
    _want(parent_ptr, torch.int32, (B, N + 1), "parent_ptr", True)
    _want(parent_idx, torch.int32, (B, Ecap), "parent_idx", True)
    if out is None:
        out = torch.empty((B, N, (N + 31) // 32), dtype=torch.int32, device=parent_ptr.device)
    _want(out, out.dtype, (B, N, (N + 31) // 32), "ancestor_mask", True)
    with torch.cuda.device(parent_ptr.device):
        _check(lib().gsd_build_mask(parent_ptr.data_ptr(), parent_idx.data_ptr(), out.data_ptr(),
                                    B, N, Ecap, _ptr(status), _stream(parent_ptr)))
    return out


def gsd_unmerge_tree(draft_tokens, parent_ptr, parent_idx, *, Ucap: int, max_depth: int,
                     status: Optional[torch.Tensor] = None,
                     out: Optional[Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]] = None
                     ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """The token graph unfolded into a tree (one node per root path); see gsd_unmerge_tree in
    include/gsd.h.  Returns (tree_tokens, tree_parent, tree_source [B,Ucap], tree_count [B])."""
    B, N = draft_tokens.shape
    Ecap = parent_idx.shape[1]
    _want(draft_tokens, torch.int32, (B, N), "draft_tokens", True)
    _want(parent_ptr, torch.int32, (B, N + 1), "parent_ptr", True)
    _want(parent_idx, torch.int32, (B, Ecap), "parent_idx", True)
    dev = draft_tokens.device
    if out is None:
        tt = torch.empty((B, Ucap), dtype=torch.int32, device=dev)
        tp = torch.empty((B, Ucap), dtype=torch.int32, device=dev)
        ts = torch.empty((B, Ucap), dtype=torch.int32, device=dev)
        cnt = torch.empty((B,), dtype=torch.int32, device=dev)
    else:
        tt, tp, ts, cnt = out
        for name, t in (("tree_tokens", tt), ("tree_parent", tp), ("tree_source", ts)):
            _want(t, torch.int32, (B, Ucap), name, True)
        _want(cnt, torch.int32, (B,), "tree_count", True)
    with torch.cuda.device(dev):
        _check(lib().gsd_unmerge_tree(draft_tokens.data_ptr(), parent_ptr.data_ptr(), parent_idx.data_ptr(),
                                      tt.data_ptr(), tp.data_ptr(), ts.data_ptr(), cnt.data_ptr(), B, N, Ecap,
                                      int(Ucap), int(max_depth), _ptr(status), _stream(draft_tokens)))
    return tt, tp, ts, cnt


def gsd_commit_kv(k_cache, v_cache, draft_k, draft_v, accepted_nodes, accepted_len, seq_lens, *,
                  status: Optional[torch.Tensor] = None) -> None:
    """Append the draft K/V rows of the accepted path to the cache in place and advance
    seq_lens; see gsd_commit_kv in include/gsd.h.  Enqueued on the current stream."""
    fast = _native if _lib is not None and _lib is _native_lib else _marshal()
    r = fast.commit_kv(k_cache, v_cache, draft_k, draft_v, accepted_nodes, accepted_len, seq_lens, status)
    if r is not None:
        return _check(r)
    B, Lmax, Hkv, D = k_cache.shape
    N = draft_k.shape[1]
    Tcap = accepted_nodes.shape[1]
    bf = torch.bfloat16
    _want(k_cache, bf, (B, Lmax, Hkv, D), "k_cache", True)
    _want(v_cache, bf, (B, Lmax, Hkv, D), "v_cache", True)
    _want(draft_k, bf, (B, N, Hkv, D), "draft_k", True)
    _want(draft_v, bf, (B, N, Hkv, D), "draft_v", True)
    _want(accepted_nodes, torch.int32, (B, Tcap), "accepted_nodes", True)
    _want(accepted_len, torch.int32, (B,), "accepted_len", True)
    _want(seq_lens, torch.int32, (B,), "seq_lens", True)
    p = CommitParams(B, N, Hkv, D, Lmax, Tcap)
    with torch.cuda.device(k_cache.device):
        _check(lib().gsd_commit_kv(k_cache.data_ptr(), v_cache.data_ptr(), draft_k.data_ptr(),
                                   draft_v.data_ptr(), accepted_nodes.data_ptr(),
                                   accepted_len.data_ptr(), seq_lens.data_ptr(), ctypes.byref(p),
                                   _ptr(status), _stream(k_cache)))


GSD_KV8_E4M3, GSD_KV8_INT8 = 0, 1
GSD_KV8_EXP_MIN, GSD_KV8_EXP_MAX = -117, 119
_KV8_FORMATS = {torch.float8_e4m3fn: GSD_KV8_E4M3, torch.int8: GSD_KV8_INT8}


def _check_kv8(k_cache, v_cache, k_exp, v_exp, block) -> Kv8Params:
    """The 8-bit cache: codes [B,Lmax,Hkv,D] of float8_e4m3fn or int8, exponents [B,ceil(Lmax/block),Hkv] int8."""
    if k_cache.dim() != 4:
        raise ValueError("k_cache must be [B,Lmax,Hkv,D]")
    if k_cache.dtype not in _KV8_FORMATS:
        raise ValueError(f"k_cache: expected torch.float8_e4m3fn or torch.int8, got {k_cache.dtype}")
    if block not in (16, 32, 64, 128):
        raise ValueError(f"block must be 16, 32, 64 or 128, got {block}")
    B, Lmax, Hkv, D = k_cache.shape
    _want(k_cache, k_cache.dtype, (B, Lmax, Hkv, D), "k_cache", True)
    _want(v_cache, k_cache.dtype, (B, Lmax, Hkv, D), "v_cache", True)
    nb = (Lmax + block - 1) // block
    _want(k_exp, torch.int8, (B, nb, Hkv), "k_exp", True)
    _want(v_exp, torch.int8, (B, nb, Hkv), "v_exp", True)
    return Kv8Params(_KV8_FORMATS[k_cache.dtype], int(block))


def gsd_verify_attn_q8_workspace_bytes(B, N, Hq, Hkv, D, Lmax, *, block, num_splits=0, kernel=GSD_ATTN_AUTO) -> int:
    p = AttnParams(B, N, Hq, Hkv, D, Lmax, 0.0, num_splits, kernel)
    c = Kv8Params(GSD_KV8_E4M3, block)
    return int(lib().gsd_verify_attn_q8_workspace_bytes(ctypes.byref(p), ctypes.byref(c)))


def gsd_verify_attn_q8(q, k_cache, v_cache, k_exp, v_exp, draft_k, draft_v, ancestor_mask, seq_lens,
                       out: Optional[torch.Tensor] = None, *, block: int, softmax_scale: float = 0.0,
                       num_splits: int = 0, kernel: int = GSD_ATTN_AUTO,
                       workspace: Optional[torch.Tensor] = None,
                       status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """gsd_verify_attn over a cache held in 8 bits (codes float8_e4m3fn or int8, int8 exponents of a scale for each
    `block` tokens and kv head); see gsd_verify_attn_q8 in include/gsd.h.  Enqueued on the current stream; returns
    `out` [B,N,Hq,D] bf16."""
    fast = _native if _lib is not None and _lib is _native_lib else _marshal()
    r = fast.verify_attn_q8(q, k_cache, v_cache, k_exp, v_exp, draft_k, draft_v, ancestor_mask, seq_lens, out, block,
                            softmax_scale, num_splits, kernel, workspace, status)
    if r is not None:
        if r.__class__ is int:
            _check(r)
        return r
    if q.dim() != 4:
        raise ValueError("q must be [B,N,Hq,D]")
    c = _check_kv8(k_cache, v_cache, k_exp, v_exp, block)
    bf = torch.bfloat16
    B, N, Hq, D = q.shape
    Lmax, Hkv = k_cache.shape[1], k_cache.shape[2]
    _want(q, bf, (B, N, Hq, D), "q", True)
    _want(k_cache, k_cache.dtype, (B, Lmax, Hkv, D), "k_cache", True)
    _want(draft_k, bf, (B, N, Hkv, D), "draft_k", True)
    _want(draft_v, bf, (B, N, Hkv, D), "draft_v", True)
    if ancestor_mask.dtype not in (torch.int32, torch.uint32):
        raise ValueError("ancestor_mask must hold 32-bit words (int32 or uint32)")
    _want(ancestor_mask, ancestor_mask.dtype, (B, N, (N + 31) // 32), "ancestor_mask", True)
    _want(seq_lens, torch.int32, (B,), "seq_lens", True)
    _same_device(q, k_cache, v_cache, k_exp, v_exp, draft_k, draft_v, ancestor_mask, seq_lens, out, workspace, status)
    if out is None:
        out = torch.empty_like(q)
    _want(out, bf, q.shape, "out", True)
    p = _attn_params(q, k_cache, draft_k, softmax_scale, num_splits, kernel)
    L = lib()
    with torch.cuda.device(q.device):
        need = int(L.gsd_verify_attn_q8_workspace_bytes(ctypes.byref(p), ctypes.byref(c)))
        if workspace is None and need:
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        _check(L.gsd_verify_attn_q8(q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), k_exp.data_ptr(), v_exp.data_ptr(),
                                    draft_k.data_ptr(), draft_v.data_ptr(), ancestor_mask.data_ptr(), seq_lens.data_ptr(),
                                    out.data_ptr(), ctypes.byref(p), ctypes.byref(c), _ptr(workspace), ws_bytes, _ptr(status),
                                    _stream(q)))
    return out


def _same_device(first, *others) -> None:
    for t in others:
        if t is not None and t.device != first.device:
            raise ValueError(f"tensors on {first.device} and {t.device}")


def gsd_commit_kv_q8(k_cache, v_cache, k_exp, v_exp, draft_k, draft_v, accepted_nodes, accepted_len, seq_lens, *,
                     block: int, status: Optional[torch.Tensor] = None) -> None:
    """Round the draft K/V rows of the accepted path into the 8-bit cache in place and advance seq_lens; see
    gsd_commit_kv_q8 in include/gsd.h.  Enqueued on the current stream."""
    fast = _native if _lib is not None and _lib is _native_lib else _marshal()
    r = fast.commit_kv_q8(k_cache, v_cache, k_exp, v_exp, draft_k, draft_v, accepted_nodes, accepted_len, seq_lens, block, status)
    if r is not None:
        return _check(r)
    c = _check_kv8(k_cache, v_cache, k_exp, v_exp, block)
    B, Lmax, Hkv, D = k_cache.shape
    if draft_k.dim() != 4 or accepted_nodes.dim() != 2:
        raise ValueError("draft_k must be [B,N,Hkv,D] and accepted_nodes [B,Tcap]")
    N, Tcap = draft_k.shape[1], accepted_nodes.shape[1]
    _want(draft_k, torch.bfloat16, (B, N, Hkv, D), "draft_k", True)
    _want(draft_v, torch.bfloat16, (B, N, Hkv, D), "draft_v", True)
    _want(accepted_nodes, torch.int32, (B, Tcap), "accepted_nodes", True)
    _want(accepted_len, torch.int32, (B,), "accepted_len", True)
    _want(seq_lens, torch.int32, (B,), "seq_lens", True)
    _same_device(k_cache, v_cache, k_exp, v_exp, draft_k, draft_v, accepted_nodes, accepted_len, seq_lens, status)
    p = CommitParams(B, N, Hkv, D, Lmax, Tcap)
    with torch.cuda.device(k_cache.device):
        _check(lib().gsd_commit_kv_q8(k_cache.data_ptr(), v_cache.data_ptr(), k_exp.data_ptr(), v_exp.data_ptr(),
                                      draft_k.data_ptr(), draft_v.data_ptr(), accepted_nodes.data_ptr(),
                                      accepted_len.data_ptr(), seq_lens.data_ptr(), ctypes.byref(p), ctypes.byref(c),
                                      _ptr(status), _stream(k_cache)))


def gsd_append_kv_q8(k_cache, v_cache, k_exp, v_exp, k, v, counts, seq_lens, *, block: int,
                     status: Optional[torch.Tensor] = None) -> None:
    """Round the first counts[b] rows of k / v [B,T,Hkv,D] into the 8-bit cache behind seq_lens[b] in place and advance
    seq_lens; see gsd_append_kv_q8 in include/gsd.h.  Enqueued on the current stream."""
    fast = _native if _lib is not None and _lib is _native_lib else _marshal()
    r = fast.append_kv_q8(k_cache, v_cache, k_exp, v_exp, k, v, counts, seq_lens, block, status)
    if r is not None:
        return _check(r)
    c = _check_kv8(k_cache, v_cache, k_exp, v_exp, block)
    B, Lmax, Hkv, D = k_cache.shape
    if k.dim() != 4:
        raise ValueError("k must be [B,T,Hkv,D]")
    T = k.shape[1]
    _want(k, torch.bfloat16, (B, T, Hkv, D), "k", True)
    _want(v, torch.bfloat16, (B, T, Hkv, D), "v", True)
    _want(counts, torch.int32, (B,), "counts", True)
    _want(seq_lens, torch.int32, (B,), "seq_lens", True)
    _same_device(k_cache, v_cache, k_exp, v_exp, k, v, counts, seq_lens, status)
    p = AppendParams(B, T, Hkv, D, Lmax)
    with torch.cuda.device(k_cache.device):
        _check(lib().gsd_append_kv_q8(k_cache.data_ptr(), v_cache.data_ptr(), k_exp.data_ptr(), v_exp.data_ptr(),
                                      k.data_ptr(), v.data_ptr(), counts.data_ptr(), seq_lens.data_ptr(), ctypes.byref(p),
                                      ctypes.byref(c), _ptr(status), _stream(k_cache)))


_PAGED_LMAX = 1 << 30


def _check_pages(k_pages, v_pages, page_table, B) -> PageParams:
    """The paged cache: pools [num_pages,page,Hkv,D] bf16 and a table [B,max_pages] int32."""
    if k_pages.dim() != 4 or page_table.dim() != 2:
        raise ValueError("k_pages must be [num_pages,page,Hkv,D] and page_table [B,max_pages]")
    P, page, Hkv, D = k_pages.shape
    if page not in (16, 32, 64, 128, 256):
        raise ValueError(f"pages must have 16, 32, 64, 128 or 256 rows, got {page}")
    _want(k_pages, torch.bfloat16, (P, page, Hkv, D), "k_pages", True)
    _want(v_pages, torch.bfloat16, (P, page, Hkv, D), "v_pages", True)
    _want(page_table, torch.int32, (B, page_table.shape[1]), "page_table", True)
    return PageParams(page, P, page_table.shape[1])


def _paged_lmax(c: PageParams) -> int:
    return min(c.max_pages * c.page, _PAGED_LMAX)


def gsd_verify_attn_paged_workspace_bytes(B, N, Hq, Hkv, D, page, max_pages, *, max_len=0, num_splits=0, kernel=GSD_ATTN_AUTO) -> int:
    c = PageParams(page, 1, max_pages)
    p = AttnParams(B, N, Hq, Hkv, D, int(max_len) or _paged_lmax(c), 0.0, num_splits, kernel)
    return int(lib().gsd_verify_attn_paged_workspace_bytes(ctypes.byref(p), ctypes.byref(c)))


def gsd_verify_attn_paged(q, k_pages, v_pages, page_table, draft_k, draft_v, ancestor_mask, seq_lens,
                          out: Optional[torch.Tensor] = None, *, max_len: int = 0, softmax_scale: float = 0.0,
                          num_splits: int = 0, kernel: int = GSD_ATTN_AUTO, workspace: Optional[torch.Tensor] = None,
                          status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """gsd_verify_attn over a cache in pages: pools k_pages / v_pages [num_pages,page,Hkv,D], page_table [B,max_pages] int32;
    `max_len` is a length no sequence exceeds (0: the room in the table).  See gsd_verify_attn_paged in include/gsd.h.
    Enqueued on the current stream; returns `out` [B,N,Hq,D] bf16."""
    fast = _native if _lib is not None and _lib is _native_lib else _marshal()
    r = fast.verify_attn_paged(q, k_pages, v_pages, page_table, draft_k, draft_v, ancestor_mask, seq_lens, out, max_len,
                               softmax_scale, num_splits, kernel, workspace, status)
    if r is not None:
        if r.__class__ is int:
            _check(r)
        return r
    if q.dim() != 4:
        raise ValueError("q must be [B,N,Hq,D]")
    bf = torch.bfloat16
    B, N, Hq, D = q.shape
    c = _check_pages(k_pages, v_pages, page_table, B)
    Hkv = k_pages.shape[2]
    _want(q, bf, (B, N, Hq, D), "q", True)
    _want(k_pages, bf, (c.num_pages, c.page, Hkv, D), "k_pages", True)
    _want(draft_k, bf, (B, N, Hkv, D), "draft_k", True)
    _want(draft_v, bf, (B, N, Hkv, D), "draft_v", True)
    if ancestor_mask.dtype not in (torch.int32, torch.uint32):
        raise ValueError("ancestor_mask must hold 32-bit words (int32 or uint32)")
    _want(ancestor_mask, ancestor_mask.dtype, (B, N, (N + 31) // 32), "ancestor_mask", True)
    _want(seq_lens, torch.int32, (B,), "seq_lens", True)
    _same_device(q, k_pages, v_pages, page_table, draft_k, draft_v, ancestor_mask, seq_lens, out, workspace, status)
    if out is None:
        out = torch.empty_like(q)
    _want(out, bf, q.shape, "out", True)
    p = AttnParams(B, N, Hq, Hkv, D, int(max_len) or _paged_lmax(c), float(softmax_scale), int(num_splits), int(kernel))
    L = lib()
    with torch.cuda.device(q.device):
        need = int(L.gsd_verify_attn_paged_workspace_bytes(ctypes.byref(p), ctypes.byref(c)))
        if workspace is None and need:
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        _check(L.gsd_verify_attn_paged(q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), page_table.data_ptr(),
                                       draft_k.data_ptr(), draft_v.data_ptr(), ancestor_mask.data_ptr(), seq_lens.data_ptr(),
                                       out.data_ptr(), ctypes.byref(p), ctypes.byref(c), _ptr(workspace), ws_bytes,
                                       _ptr(status), _stream(q)))
    return out


def gsd_commit_kv_paged(k_pages, v_pages, page_table, draft_k, draft_v, accepted_nodes, accepted_len, seq_lens, *,
                        status: Optional[torch.Tensor] = None) -> None:
    """Copy the draft K/V rows of the accepted path behind the sequences' ends in a paged cache and advance seq_lens; see
    gsd_commit_kv_paged in include/gsd.h.  Enqueued on the current stream."""
    fast = _native if _lib is not None and _lib is _native_lib else _marshal()
    r = fast.commit_kv_paged(k_pages, v_pages, page_table, draft_k, draft_v, accepted_nodes, accepted_len, seq_lens, status)
    if r is not None:
        return _check(r)
    if draft_k.dim() != 4 or accepted_nodes.dim() != 2:
        raise ValueError("draft_k must be [B,N,Hkv,D] and accepted_nodes [B,Tcap]")
    B, N, Hkv, D = draft_k.shape
    c = _check_pages(k_pages, v_pages, page_table, B)
    Tcap = accepted_nodes.shape[1]
    _want(k_pages, torch.bfloat16, (c.num_pages, c.page, Hkv, D), "k_pages", True)
    _want(draft_k, torch.bfloat16, (B, N, Hkv, D), "draft_k", True)
    _want(draft_v, torch.bfloat16, (B, N, Hkv, D), "draft_v", True)
    _want(accepted_nodes, torch.int32, (B, Tcap), "accepted_nodes", True)
    _want(accepted_len, torch.int32, (B,), "accepted_len", True)
    _want(seq_lens, torch.int32, (B,), "seq_lens", True)
    _same_device(k_pages, v_pages, page_table, draft_k, draft_v, accepted_nodes, accepted_len, seq_lens, status)
    p = CommitParams(B, N, Hkv, D, _paged_lmax(c), Tcap)
    with torch.cuda.device(k_pages.device):
        _check(lib().gsd_commit_kv_paged(k_pages.data_ptr(), v_pages.data_ptr(), page_table.data_ptr(), draft_k.data_ptr(),
                                         draft_v.data_ptr(), accepted_nodes.data_ptr(), accepted_len.data_ptr(),
                                         seq_lens.data_ptr(), ctypes.byref(p), ctypes.byref(c), _ptr(status), _stream(k_pages)))


def _token_stride(x: torch.Tensor, name: str) -> int:
    """Elements from a token's rows to the next token's in x [B,T,H,D] bf16, whose rows of a token are contiguous."""
    if x.dim() != 4 or x.dtype != torch.bfloat16:
        raise ValueError(f"{name}: expected bfloat16 [B,T,H,D], got {x.dtype} {tuple(x.shape)}")
    if not x.is_cuda:
        raise ValueError(f"{name}: expected a CUDA tensor")
    B, T, H, D = x.shape
    s = x.stride(1) if T > 1 else x.stride(0) if B > 1 else H * D
    if (x.stride(3) != 1 and D > 1) or (H > 1 and x.stride(2) != D) or (B > 1 and x.stride(0) != T * s):
        raise ValueError(f"{name}: the rows of a token must be contiguous and the tokens a fixed distance apart, got strides "
                         f"{tuple(x.stride())} for {tuple(x.shape)}")
    return s


def _rotation(freqs, positions, offsets, axes, pairs, B, T) -> Rotation:
    if freqs.dim() != 1:
        raise ValueError("freqs must be [pairs]")
    n = freqs.shape[0]
    _want(freqs, torch.float32, (n,), "freqs", True)
    if positions is not None:
        if positions.dim() != 3:
            raise ValueError("positions must be [axes,B,T]")
        _want(positions, torch.int32, (positions.shape[0], B, T), "positions", True)
    if offsets is not None:
        _want(offsets, torch.int32, (B,), "offsets", True)
    axes = [0] * n if axes is None else [int(a) for a in axes]
    count = positions.shape[0] if positions is not None else max(axes, default=0) + 1
    if len(axes) != n or any(a < 0 or a >= count for a in axes):
        raise ValueError(f"axes: expected an axis below {count} for each of {n} pairs")
    return Rotation(n, GSD_ROTARY_NEIGHBOURS if pairs else GSD_ROTARY_HALVES, count, (ctypes.c_uint8 * 64)(*axes[:64]))


def gsd_append_kv_paged(k_pages, v_pages, page_table, k, v, counts, seq_lens, *, freqs: Optional[torch.Tensor] = None,
                        positions: Optional[torch.Tensor] = None, offsets: Optional[torch.Tensor] = None,
                        axes: Optional[Sequence[int]] = None, pairs: bool = False,
                        status: Optional[torch.Tensor] = None) -> None:
    """Write the first counts[b] rows of k / v [B,T,Hkv,D] behind the sequences' ends in a paged cache, K rotated by position on
    the way if `freqs` is given (positions [axes,B,T]; None: the place in the sequence), and advance seq_lens; see
    gsd_append_kv_paged in include/gsd.h and gsd_rotary.  k and v may be slices of a projection's output.  Enqueued on the
    current stream."""
    fast = _native if _lib is not None and _lib is _native_lib else _marshal()
    r = fast.append_kv_paged(k_pages, v_pages, page_table, k, v, counts, seq_lens, freqs, positions, offsets, axes, pairs, status)
    if r is not None:
        return _check(r)
    ks, vs = _token_stride(k, "k"), _token_stride(v, "v")
    B, T, Hkv, D = k.shape
    if v.shape != k.shape:
        raise ValueError(f"v: expected {tuple(k.shape)}, got {tuple(v.shape)}")
    c = _check_pages(k_pages, v_pages, page_table, B)
    _want(k_pages, torch.bfloat16, (c.num_pages, c.page, Hkv, D), "k_pages", True)
    _want(counts, torch.int32, (B,), "counts", True)
    _want(seq_lens, torch.int32, (B,), "seq_lens", True)
    if freqs is None and not (positions is None and offsets is None and axes is None):
        raise ValueError("positions, offsets and axes need freqs")
    rot = None if freqs is None else _rotation(freqs, positions, offsets, axes, pairs, B, T)
    _same_device(k_pages, v_pages, page_table, k, v, counts, seq_lens, freqs, positions, offsets, status)
    p = AppendPagedParams(B, T, Hkv, D, _paged_lmax(c), ks, vs)
    with torch.cuda.device(k_pages.device):
        _check(lib().gsd_append_kv_paged(k_pages.data_ptr(), v_pages.data_ptr(), page_table.data_ptr(), k.data_ptr(),
                                         v.data_ptr(), counts.data_ptr(), seq_lens.data_ptr(), _ptr(freqs), _ptr(positions),
                                         _ptr(offsets), ctypes.byref(p), ctypes.byref(c),
                                         None if rot is None else ctypes.byref(rot), _ptr(status), _stream(k_pages)))


def gsd_rotary(q, k, freqs, positions, *, offsets: Optional[torch.Tensor] = None, axes: Optional[Sequence[int]] = None,
               pairs: bool = False, out: Optional[Tuple[torch.Tensor, Optional[torch.Tensor]]] = None
               ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Rotary positions of q [B,T,Hq,D] and k [B,T,Hkv,D] (or None): pair i of the first 2 * len(freqs) columns turns by
    (positions[axes[i],b,t] + offsets[b]) * freqs[i].  `axes` names the position axis of each pair (None: the first), `pairs`
    says that neighbouring columns form a pair, else column i and i + len(freqs) do.  q and k may be slices of a projection's
    output.  Returns new dense tensors, or `out`, which may be (q, k) themselves if those are dense.  See gsd_rotary in
    include/gsd.h.  Enqueued on the current stream."""
    fast = _native if _lib is not None and _lib is _native_lib else _marshal()
    r = fast.rotary(q, k, freqs, positions, offsets, axes, pairs, out)
    if r is not None:
        if r.__class__ is int:
            _check(r)
        return r
    qs = _token_stride(q, "q")
    B, T, Hq, D = q.shape
    ks, Hkv = 0, 0
    if k is not None:
        ks, Hkv = _token_stride(k, "k"), k.shape[2]
        if tuple(k.shape) != (B, T, Hkv, D):
            raise ValueError(f"k: expected [{B},{T},Hkv,{D}], got {tuple(k.shape)}")
    if positions is None:
        raise ValueError("positions must be [axes,B,T]")
    rot = _rotation(freqs, positions, offsets, axes, pairs, B, T)
    if out is None:
        out = (torch.empty((B, T, Hq, D), dtype=q.dtype, device=q.device),
               None if k is None else torch.empty((B, T, Hkv, D), dtype=q.dtype, device=q.device))
    qo, ko = out
    _want(qo, torch.bfloat16, (B, T, Hq, D), "q_out", True)
    if (k is None) != (ko is None):
        raise ValueError("out: k and its place go together")
    if ko is not None:
        _want(ko, torch.bfloat16, (B, T, Hkv, D), "k_out", True)
    _same_device(q, k, freqs, positions, offsets, qo, ko)
    p = RotaryParams(B, T, Hq, Hkv, D, qs, ks)
    with torch.cuda.device(q.device):
        _check(lib().gsd_rotary(q.data_ptr(), _ptr(k), freqs.data_ptr(), positions.data_ptr(), _ptr(offsets), qo.data_ptr(),
                                _ptr(ko), ctypes.byref(p), ctypes.byref(rot), _stream(q)))
    return qo, ko


def gsd_token_logprobs_workspace_bytes(B, N, V, T, k=0) -> int:
    p = LogprobsParams(B, N, V, T, k)
    return int(lib().gsd_token_logprobs_workspace_bytes(ctypes.byref(p)))


def gsd_token_logprobs(logits, nodes, tokens, lens, *, k: int = 0, workspace: Optional[torch.Tensor] = None,
                       status: Optional[torch.Tensor] = None,
                       out: Optional[Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]] = None
                       ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """Log probabilities of the tokens [B,T] under the logits rows of the nodes [B,T], entropy of these rows and their k
    best entries; see gsd_token_logprobs in include/gsd.h.  Takes accepted_nodes, accepted_tokens, accepted_len of the
    acceptance calls.  Returns (logprobs [B,T], entropy [B,T], top_tokens [B,T,k], top_logprobs [B,T,k])."""
    if out is None:
        fast = _native if _lib is not None and _lib is _native_lib else _marshal()
        r = fast.token_logprobs(logits, nodes, tokens, lens, k, workspace, status)
        if r is not None:
            if r.__class__ is int:
                _check(r)
            return r
    if logits.dim() != 3 or nodes.dim() != 2:
        raise ValueError("logits must be [B,N,V] and nodes [B,T]")
    B, N, V = logits.shape
    T = nodes.shape[1]
    _want(logits, torch.float32, (B, N, V), "logits", True)
    _want(nodes, torch.int32, (B, T), "nodes", True)
    _want(tokens, torch.int32, (B, T), "tokens", True)
    _want(lens, torch.int32, (B,), "lens", True)
    dev = logits.device
    if out is None:
        n = max(int(k), 0)
        out = (torch.empty((B, T), dtype=torch.float32, device=dev), torch.empty((B, T), dtype=torch.float32, device=dev),
               torch.empty((B, T, n), dtype=torch.int32, device=dev), torch.empty((B, T, n), dtype=torch.float32, device=dev))
    lp, ent, top, val = out
    _want(lp, torch.float32, (B, T), "logprobs", True)
    _want(ent, torch.float32, (B, T), "entropy", True)
    _want(top, torch.int32, (B, T, max(int(k), 0)), "top_tokens", True)
    _want(val, torch.float32, (B, T, max(int(k), 0)), "top_logprobs", True)
    _same_device(logits, nodes, tokens, lens, lp, ent, top, val, workspace, status)
    p = LogprobsParams(B, N, V, T, int(k))
    L = lib()
    with torch.cuda.device(dev):
        need = int(L.gsd_token_logprobs_workspace_bytes(ctypes.byref(p)))
        if workspace is None:
            workspace = torch.empty(max(need, 8), dtype=torch.uint8, device=dev)
        _check(L.gsd_token_logprobs(logits.data_ptr(), nodes.data_ptr(), tokens.data_ptr(), lens.data_ptr(), lp.data_ptr(),
                                    ent.data_ptr(), _ptr(top) if k else None, _ptr(val) if k else None, ctypes.byref(p),
                                    workspace.data_ptr(), workspace.numel() * workspace.element_size(), _ptr(status),
                                    _stream(logits)))
    return lp, ent, top, val


GSD_STATIC_MAX_ROWS = 16384


def gsd_accept_static(logits, draft_tokens, parent_ptr, parent_idx, *, Tcap: int = 0,
                      want_nodes: bool = True, status: Optional[torch.Tensor] = None
                      ) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """gsd_accept for callers that cannot provide scratch memory: the library's own fixed
    array is used instead (B * N <= GSD_STATIC_MAX_ROWS; calls on one device must not overlap).
    The C call allocates nothing; this wrapper only allocates the result tensors it returns.
    See gsd_accept_static in include/gsd.h."""
    B, N, V = logits.shape
    _want(logits, torch.float32, (B, N, V), "logits", True)
    _want(draft_tokens, torch.int32, (B, N), "draft_tokens", True)
    _want(parent_ptr, torch.int32, (B, N + 1), "parent_ptr", True)
    Ecap = parent_idx.shape[1]
    _want(parent_idx, torch.int32, (B, Ecap), "parent_idx", True)
    Tcap = Tcap or N
    toks = torch.empty((B, Tcap), dtype=torch.int32, device=logits.device)
    lens = torch.empty((B,), dtype=torch.int32, device=logits.device)
    nodes = torch.empty((B, Tcap), dtype=torch.int32, device=logits.device) if want_nodes else None
    p = AcceptParams(B, N, V, Ecap, Tcap)
    with torch.cuda.device(logits.device):
        _check(lib().gsd_accept_static(logits.data_ptr(), draft_tokens.data_ptr(),
                                       parent_ptr.data_ptr(), parent_idx.data_ptr(),
                                       toks.data_ptr(), lens.data_ptr(), _ptr(nodes),
                                       ctypes.byref(p), _ptr(status), _stream(logits)))
    return toks, lens, nodes


def gsd_verify_step_host_arena_bytes(B, N, Hq, Hkv, D, Lmax, V, Ecap, Tcap, num_splits=0,
                                     kernel=GSD_ATTN_AUTO) -> int:
    ap = AttnParams(B, N, Hq, Hkv, D, Lmax, 0.0, num_splits, kernel)
    cp = AcceptParams(B, N, V, Ecap, Tcap)
    return int(lib().gsd_verify_step_host_arena_bytes(ctypes.byref(ap), ctypes.byref(cp)))


def gsd_verify_step_host(q, k_cache, v_cache, draft_k, draft_v, ancestor_mask, seq_lens, logits,
                         draft_tokens, parent_ptr, parent_idx, arena: torch.Tensor, *,
                         out=None, accepted=None, Tcap: int = 0, softmax_scale: float = 0.0,
                         num_splits: int = 0, kernel: int = GSD_ATTN_AUTO):
    """One whole verification step from HOST tensors through a caller-owned device arena;
    see gsd_verify_step_host in include/gsd.h.  Synchronises the current stream.
    Returns (out [B,N,Hq,D] bf16 CPU, accepted_tokens, accepted_len, accepted_nodes, status)."""
    _check_attn_tensors(q, k_cache, v_cache, draft_k, draft_v, ancestor_mask, seq_lens, False)
    B, N, V = logits.shape
    Ecap = parent_idx.shape[1]
    _want(logits, torch.float32, (B, N, V), "logits", False)
    _want(draft_tokens, torch.int32, (B, N), "draft_tokens", False)
    _want(parent_ptr, torch.int32, (B, N + 1), "parent_ptr", False)
    _want(parent_idx, torch.int32, (B, Ecap), "parent_idx", False)
    Tcap = Tcap or N
    if out is None:
        out = torch.empty_like(q)
    if accepted is None:
        accepted = (torch.empty((B, Tcap), dtype=torch.int32), torch.empty((B,), dtype=torch.int32),
                    torch.empty((B, Tcap), dtype=torch.int32))
    toks, lens, nodes = accepted
    ap = _attn_params(q, k_cache, draft_k, softmax_scale, num_splits, kernel)
    cp = AcceptParams(B, N, V, Ecap, Tcap)
    dev_status = ctypes.c_int32(0)
    if not arena.is_cuda:
        raise ValueError("arena must be a CUDA tensor")
    with torch.cuda.device(arena.device):
        _check(lib().gsd_verify_step_host(
            q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), draft_k.data_ptr(),
            draft_v.data_ptr(), ancestor_mask.data_ptr(), seq_lens.data_ptr(), out.data_ptr(),
            ctypes.byref(ap), logits.data_ptr(), draft_tokens.data_ptr(), parent_ptr.data_ptr(),
            parent_idx.data_ptr(), toks.data_ptr(), lens.data_ptr(), _ptr(nodes), ctypes.byref(cp),
            arena.data_ptr(), arena.numel() * arena.element_size(),
            ctypes.addressof(dev_status), _stream(arena)))
    return out, toks, lens, nodes, int(dev_status.value)
