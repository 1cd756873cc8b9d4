"""Python binding of libdreams.so (C ABI in include/dreams.h).

Argument marshalling only: every step runs in the library's HIP kernels.  PyTorch supplies device memory
and the current stream.  The library must be built (``python -m paper_2606_00535_amd.build``); if it is
missing every call raises -- there is no fallback.
"""
from __future__ import annotations

import ctypes
import math
import os
import threading
from typing import Optional, Tuple

import torch

LIBRARY = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libdreams.so")

DREAMS_OK, DREAMS_ERR_INVALID_ARG, DREAMS_ERR_UNSUPPORTED, DREAMS_ERR_WORKSPACE, DREAMS_ERR_HIP = 0, -1, -2, -3, -4
DREAMS_ERR_DEVICE = -5
DREAMS_F32, DREAMS_BF16, DREAMS_E4M3 = 0, 1, 2

# every symbol include/dreams.h declares
EXPORTS = (
    "dreams_tree_verify_attn_workspace_size", "dreams_tree_verify_attn", "dreams_tree_accept_workspace_size",
    "dreams_tree_accept", "dreams_kv_commit", "dreams_status_string", "dreams_last_error_message",
    "dreams_check_tree_host", "dreams_stream_read", "dreams_tree_verify_attn_entropy", "dreams_attn_entropy_mean",
    "dreams_attn_entropy_select", "dreams_visual_importance_workspace_size", "dreams_visual_importance",
    "dreams_visual_topk", "dreams_visual_gather", "dreams_tree_accept_sampled_workspace_size",
    "dreams_tree_accept_sampled", "dreams_tree_accept_lm_head_workspace_size", "dreams_tree_accept_lm_head",
    "dreams_workspace_status", "dreams_tree_verify_attn_splits", "dreams_tree_verify_attn_noalloc",
    "dreams_set_wait_limit", "dreams_prefill_attn_stats", "dreams_prefill_attn_entropy_mean",
    "dreams_prefill_visual_importance", "dreams_prefill_visual_importance_workspace_size",
    "dreams_paged_verify_attn", "dreams_paged_verify_attn_workspace_size", "dreams_paged_prompt_attn",
    "dreams_paged_prompt_attn_workspace_size", "dreams_paged_append", "dreams_paged_kv_commit", "dreams_pages_reserve",
    "dreams_pages_fork", "dreams_pages_release", "dreams_rope_frequencies", "dreams_rope", "dreams_paged_append_rope",
    "dreams_paged_append_e4m3", "dreams_paged_kv_commit_e4m3", "dreams_paged_read_e4m3", "dreams_pages_fork_e4m3",
    "dreams_paged_verify_attn_e4m3", "dreams_paged_verify_attn_e4m3_workspace_size", "dreams_paged_prompt_attn_e4m3",
    "dreams_paged_prompt_attn_e4m3_workspace_size",
)


class DreamsError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("%s (status %d)" % (message, status))
        self.status = status


class AttnDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("num_nodes", ctypes.c_int32), ("cache_capacity", ctypes.c_int32),
                ("max_kv_len", ctypes.c_int32), ("num_splits", ctypes.c_int32), ("dtype", ctypes.c_int),
                ("scale", ctypes.c_float)]


class PrefillDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("num_rows", ctypes.c_int32), ("cache_capacity", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class PagedDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "num_q_heads", "num_kv_heads", "head_dim", "num_rows", "num_pages",
                                              "page_size", "table_width", "max_kv_len", "num_splits", "window", "sinks")]
    _fields_ += [("dtype", ctypes.c_int), ("scale", ctypes.c_float), ("page_stride", ctypes.c_int64)]


class PagePool(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("num_layers", "batch", "num_kv_heads", "head_dim", "num_pages", "page_size",
                                              "table_width")]
    _fields_ += [("dtype", ctypes.c_int), ("layer_stride", ctypes.c_int64), ("page_stride", ctypes.c_int64)]


class Rope(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("frequencies", ctypes.c_void_p),
                ("positions", ctypes.c_void_p), ("parent", ctypes.c_void_p), ("amplitude", ctypes.c_float)]


class RopeQueries(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("out", ctypes.c_void_p), ("num_q_heads", ctypes.c_int32),
                ("strides", ctypes.c_int64 * 3)]


class PageScales(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("layer_stride", ctypes.c_int64),
                ("page_stride", ctypes.c_int64)]


_lib = None
_lib_lock = threading.Lock()


def library_path() -> str:
    return LIBRARY


def lib():
    """The loaded library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        with _lib_lock:
            if _lib is None:
                if not os.path.exists(LIBRARY):
                    raise RuntimeError("libdreams.so is not built (run: python -m paper_2606_00535_amd.build)")
                L = ctypes.CDLL(LIBRARY)
                P, I32, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
                L.dreams_tree_verify_attn_workspace_size.argtypes = [ctypes.POINTER(AttnDesc), ctypes.POINTER(SZ)]
                L.dreams_tree_verify_attn.argtypes = [ctypes.POINTER(AttnDesc), P, P, P, P, P, P, P, P, P, SZ, P]
                L.dreams_tree_accept_workspace_size.argtypes = [I32, I32, I32, ctypes.POINTER(SZ)]
                L.dreams_tree_accept.argtypes = [I32, I32, I32, P, P, P, P, P, P, P, P, SZ, P]
                L.dreams_kv_commit.argtypes = [I32, ctypes.c_int64, I32, I32, I32, I32, ctypes.c_int, P, P, P, P, P,
                                               I32, P, P]
                L.dreams_status_string.argtypes = [ctypes.c_int]
                L.dreams_status_string.restype = ctypes.c_char_p
                L.dreams_last_error_message.argtypes = []
                L.dreams_last_error_message.restype = ctypes.c_char_p
                L.dreams_check_tree_host.argtypes = [P, I32]
                L.dreams_stream_read.argtypes = [P, SZ, P, P]
                L.dreams_tree_verify_attn_entropy.argtypes = [ctypes.POINTER(AttnDesc), P, P, P, P, P, P, P, P, P, P,
                                                              SZ, P]
                L.dreams_attn_entropy_mean.argtypes = [ctypes.c_int64, P, P, P]
                L.dreams_attn_entropy_select.argtypes = [I32, P, P, P]
                L.dreams_visual_importance_workspace_size.argtypes = [I32, I32, I32, ctypes.POINTER(SZ)]
                L.dreams_prefill_visual_importance_workspace_size.argtypes = [I32, I32, I32, ctypes.POINTER(SZ)]
                L.dreams_visual_importance.argtypes = [ctypes.POINTER(AttnDesc), P, P, P, P, I32, I32, P, P, SZ, P]
                L.dreams_visual_topk.argtypes = [I32, I32, I32, P, P, P]
                L.dreams_tree_accept_sampled_workspace_size.argtypes = [I32, I32, I32, ctypes.POINTER(SZ)]
                L.dreams_tree_accept_sampled.argtypes = [I32, I32, I32, ctypes.c_double, P, P, P, P, P, P, P, P, P,
                                                         SZ, P]
                L.dreams_tree_accept_lm_head_workspace_size.argtypes = [I32, I32, I32, I32, ctypes.POINTER(SZ)]
                L.dreams_tree_accept_lm_head.argtypes = [I32, I32, I32, I32, P, P, P, P, P, P, P, P, P, SZ, P]
                L.dreams_visual_gather.argtypes = [I32, I32, I32, I32, ctypes.c_int, P, P, I32, P, I32, P, P, P]
                L.dreams_workspace_status.argtypes = [P, SZ, P]
                L.dreams_set_wait_limit.argtypes = [ctypes.c_double]
                L.dreams_tree_verify_attn_noalloc.argtypes = [ctypes.POINTER(AttnDesc), P, P, P, P, P, P, P, P, P]
                L.dreams_tree_verify_attn_splits.argtypes = [ctypes.POINTER(AttnDesc), ctypes.POINTER(I32)]
                L.dreams_prefill_attn_stats.argtypes = [ctypes.POINTER(PrefillDesc), P, P, P, P, P, P]
                L.dreams_prefill_attn_entropy_mean.argtypes = [I32, I32, I32, P, P, P, P]
                L.dreams_prefill_visual_importance.argtypes = [ctypes.POINTER(PrefillDesc), P, P, P, P, I32, I32, P, P,
                                                               SZ, P]
                PD, PP = ctypes.POINTER(PagedDesc), ctypes.POINTER(PagePool)
                L.dreams_paged_verify_attn_workspace_size.argtypes = [PD, ctypes.POINTER(SZ)]
                L.dreams_paged_prompt_attn_workspace_size.argtypes = [PD, ctypes.POINTER(SZ)]
                L.dreams_paged_verify_attn.argtypes = [PD, P, P, P, P, P, P, P, P, P, P, SZ, P]
                L.dreams_paged_prompt_attn.argtypes = [PD, P, P, P, P, P, P, P, P, P, SZ, P]
                L.dreams_paged_append.argtypes = [PP, P, P, I32, ctypes.POINTER(ctypes.c_int64), P, P, P, P, P, P]
                L.dreams_paged_kv_commit.argtypes = [PP, P, P, P, P, P, P, I32, P, P]
                L.dreams_pages_reserve.argtypes = [PP, P, P, P, P, P, P]
                L.dreams_pages_fork.argtypes = [PP, P, P, P, P, P, P, I32, P, P, P, P]
                L.dreams_pages_release.argtypes = [PP, P, P, P, P, I32, P, I32, P]
                RP, QP, SP, I64P = (ctypes.POINTER(t) for t in (Rope, RopeQueries, PageScales, ctypes.c_int64))
                F64 = ctypes.c_double
                L.dreams_rope_frequencies.argtypes = [I32, F64, ctypes.c_int, F64, F64, F64, F64, P]
                L.dreams_rope.argtypes = [RP, I32, I32, I32, I32, ctypes.c_int, P, I64P, P, P, I64P, P]
                L.dreams_paged_append_rope.argtypes = [PP, RP, QP, P, P, I32, I64P, P, P, P, P, P, P]
                L.dreams_paged_append_e4m3.argtypes = [PP, SP, RP, QP, ctypes.c_int, P, P, I32, I64P, P, P, P, P, P, P]
                L.dreams_paged_kv_commit_e4m3.argtypes = [PP, SP, P, P, P, P, P, P, I32, P, P]
                L.dreams_paged_read_e4m3.argtypes = [PP, SP, P, P, P, P, I32, P, P, P]
                L.dreams_paged_verify_attn_e4m3_workspace_size.argtypes = [PD, ctypes.POINTER(SZ)]
                L.dreams_paged_prompt_attn_e4m3_workspace_size.argtypes = [PD, ctypes.POINTER(SZ)]
                L.dreams_paged_verify_attn_e4m3.argtypes = [PD, P, P, P, SP, P, P, P, P, P, P, P, SZ, P]
                L.dreams_paged_prompt_attn_e4m3.argtypes = [PD, P, P, P, SP, P, P, P, P, P, P, SZ, P]
                L.dreams_pages_fork_e4m3.argtypes = [PP, SP, P, P, P, P, P, P, I32, P, P, P, P]
                for f in ("dreams_tree_verify_attn_workspace_size", "dreams_tree_verify_attn",
                          "dreams_tree_accept_workspace_size", "dreams_tree_accept", "dreams_kv_commit",
                          "dreams_check_tree_host", "dreams_stream_read", "dreams_tree_verify_attn_entropy",
                          "dreams_attn_entropy_mean", "dreams_attn_entropy_select",
                          "dreams_visual_importance_workspace_size", "dreams_visual_importance", "dreams_visual_topk",
                          "dreams_visual_gather", "dreams_workspace_status", "dreams_tree_verify_attn_splits",
                          "dreams_tree_verify_attn_noalloc", "dreams_set_wait_limit", "dreams_prefill_attn_stats",
                          "dreams_prefill_attn_entropy_mean", "dreams_prefill_visual_importance",
                          "dreams_prefill_visual_importance_workspace_size"):
                    getattr(L, f).restype = ctypes.c_int
                _lib = L
    return _lib


def _check(status: int):
    if status != DREAMS_OK:
        msg = lib().dreams_last_error_message().decode() or lib().dreams_status_string(status).decode()
        raise DreamsError(status, msg)


# Addresses and streams go to the library as plain integers (every prototype declares them as pointers, so ctypes
# converts them): boxing each in a c_void_p and the current stream in a torch.cuda.Stream took 3 of a small call's 13 us.
def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


# (not part of torch's documented interface: without it, the Stream object)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _need(t: torch.Tensor, name: str, dtype, device=None, ndim=None):
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.is_cuda and t.is_contiguous()
            and (ndim is None or t.dim() == ndim) and (device is None or t.device == device)):
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if device is not None and t.device != device:
        raise ValueError("%s is on %s, expected %s" % (name, t.device, device))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if ndim is not None and t.dim() != ndim:
        raise ValueError("%s must have %d dimensions" % (name, ndim))


# A call on a given stream runs with it as the current one, so that its outputs and its workspace (and that one's first
# fill) belong to the stream that uses them.
# Workspaces: one per (device, stream, verb), zero-filled when created and left zero by every call.
_ws = {}
_ws_lock = threading.Lock()


def _workspace(kind: str, nbytes: int, device: torch.device, stream: int) -> Optional[torch.Tensor]:
    if nbytes == 0:
        return None
    key = (kind, device.index, stream)
    with _ws_lock:
        t = _ws.get(key)
        if t is None or t.numel() < nbytes:
            t = torch.zeros(nbytes, dtype=torch.uint8, device=device)
            _ws[key] = t
        return t


def attn_desc(q: torch.Tensor, k_cache: torch.Tensor, num_splits: int = 0, max_kv_len: int = 0,
              scale: Optional[float] = None) -> AttnDesc:
    B, Hq, T, D = q.shape
    Hkv, S_cap = k_cache.shape[1], k_cache.shape[2]
    dtype = DREAMS_BF16 if q.dtype == torch.bfloat16 else DREAMS_F32
    return AttnDesc(B, Hq, Hkv, D, T, S_cap, max_kv_len, num_splits, dtype,
                    1.0 / math.sqrt(D) if scale is None else float(scale))


def tree_verify_attn_workspace_size(desc: AttnDesc) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().dreams_tree_verify_attn_workspace_size(ctypes.byref(desc), ctypes.byref(n)))
    return n.value


def tree_verify_attn_splits(desc: AttnDesc) -> int:
    """dreams_tree_verify_attn_splits: pieces of the key axis the library uses for `desc`."""
    n = ctypes.c_int32(0)
    _check(lib().dreams_tree_verify_attn_splits(ctypes.byref(desc), ctypes.byref(n)))
    return n.value


def workspace_status(workspace: torch.Tensor, stream=None) -> None:
    """dreams_workspace_status: raises DreamsError (DREAMS_ERR_DEVICE) if a kernel flagged a failure in
    `workspace` since the last check; clears the flags."""
    _need(workspace, "workspace", torch.uint8, workspace.device)
    _check(lib().dreams_workspace_status(_ptr(workspace), workspace.numel(), _stream(stream)))


def set_wait_limit(seconds: float) -> None:
    """dreams_set_wait_limit: bound on every in-kernel wait for another workgroup (default 0.2 s)."""
    _check(lib().dreams_set_wait_limit(float(seconds)))


def cached_workspaces():
    """The workspaces the binding created (one per device, stream and verb)."""
    with _ws_lock:
        return list(_ws.values())


def tree_verify_attn(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, kv_len: torch.Tensor,
                     parent: Optional[torch.Tensor] = None, tree_mask: Optional[torch.Tensor] = None,
                     scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                     lse: Optional[torch.Tensor] = None, with_lse: bool = True, max_kv_len: int = 0,
                     num_splits: int = 0, workspace: Optional[torch.Tensor] = None,
                     stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """dreams_tree_verify_attn.  q [B,Hq,T,D]; k_cache/v_cache [B,Hkv,S_cap,D] (bf16 or fp32, same as q);
    kv_len [B] int32; parent [B,T] int32 or tree_mask [B,T,ceil(T/64)] int64 (bit patterns).
    Returns (out [B,Hq,T,D], lse [B,Hq,T] float32 or None)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return tree_verify_attn(q, k_cache, v_cache, kv_len, parent, tree_mask, scale, out, lse, with_lse,
                                    max_kv_len, num_splits, workspace)
    out, lse, _ = _verify_attn(q, k_cache, v_cache, kv_len, parent, tree_mask, scale, out, lse, with_lse,
                               max_kv_len, num_splits, workspace, stream, None)
    return out, lse


def tree_verify_attn_entropy(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, kv_len: torch.Tensor,
                             parent: Optional[torch.Tensor] = None, tree_mask: Optional[torch.Tensor] = None,
                             scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                             lse: Optional[torch.Tensor] = None, with_lse: bool = True,
                             entropy: Optional[torch.Tensor] = None, max_kv_len: int = 0, num_splits: int = 0,
                             workspace: Optional[torch.Tensor] = None, stream=None):
    """dreams_tree_verify_attn_entropy: as tree_verify_attn, plus every row's attention entropy (nats).
    Returns (out, lse or None, entropy [B,Hq,T] float32)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return tree_verify_attn_entropy(q, k_cache, v_cache, kv_len, parent, tree_mask, scale, out, lse, with_lse,
                                            entropy, max_kv_len, num_splits, workspace)
    B, Hq, T, _ = q.shape
    if entropy is None:
        entropy = torch.empty((B, Hq, T), dtype=torch.float32, device=q.device)
    else:
        _need(entropy, "entropy", torch.float32, q.device)
        if tuple(entropy.shape) != (B, Hq, T):
            raise ValueError("entropy must be [B, Hq, T]")
    return _verify_attn(q, k_cache, v_cache, kv_len, parent, tree_mask, scale, out, lse, with_lse, max_kv_len,
                        num_splits, workspace, stream, entropy)


def attn_entropy_mean(entropy: torch.Tensor, ae: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """dreams_attn_entropy_mean: AE of one layer from its row entropies (any shape).  Returns a [1] float32."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return attn_entropy_mean(entropy, ae)
    _need(entropy, "entropy", torch.float32, entropy.device)
    if ae is None:
        ae = torch.empty(1, dtype=torch.float32, device=entropy.device)
    _check(lib().dreams_attn_entropy_mean(entropy.numel(), _ptr(entropy), _ptr(ae), _stream(stream)))
    return ae


def attn_entropy_select(ae: torch.Tensor, best: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """dreams_attn_entropy_select: the distillation layer from per-layer AE [NL].  Returns a [1] int32."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return attn_entropy_select(ae, best)
    _need(ae, "ae", torch.float32, ae.device, 1)
    if best is None:
        best = torch.empty(1, dtype=torch.int32, device=ae.device)
    _check(lib().dreams_attn_entropy_select(ae.numel(), _ptr(ae), _ptr(best), _stream(stream)))
    return best


VISUAL_MAX_TOKENS = 8192


def visual_importance_workspace_size(batch: int, num_kv_heads: int, vis_count: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().dreams_visual_importance_workspace_size(batch, num_kv_heads, vis_count, ctypes.byref(n)))
    return n.value


def visual_importance(q: torch.Tensor, k_cache: torch.Tensor, kv_len: torch.Tensor, lse: torch.Tensor,
                      vis_begin: int, vis_count: int, scale: Optional[float] = None,
                      importance: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                      stream=None) -> torch.Tensor:
    """dreams_visual_importance (Eq. 2): q [B,Hq,T,D] and k_cache [B,Hkv,S_cap,D] bf16, kv_len [B] int32, lse
    [B,Hq,T] float32 from the attention call on the same rows.  Returns importance [B, vis_count] float32."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return visual_importance(q, k_cache, kv_len, lse, vis_begin, vis_count, scale, importance, workspace)
    dev = q.device
    _need(q, "q", torch.bfloat16, dev, 4)
    _need(k_cache, "k_cache", torch.bfloat16, dev, 4)
    _need(kv_len, "kv_len", torch.int32, dev, 1)
    _need(lse, "lse", torch.float32, dev, 3)
    B, Hq, T, D = q.shape
    desc = attn_desc(q, k_cache, 0, 0, scale)
    if importance is None:
        importance = torch.empty((B, vis_count), dtype=torch.float32, device=dev)
    else:
        _need(importance, "importance", torch.float32, dev)
    nbytes = visual_importance_workspace_size(B, k_cache.shape[1], vis_count)
    st = _stream(stream)
    if workspace is None:
        workspace = _workspace("visual", nbytes, dev, st)
    _check(lib().dreams_visual_importance(ctypes.byref(desc), _ptr(q), _ptr(k_cache), _ptr(kv_len), _ptr(lse),
                                          vis_begin, vis_count, _ptr(importance), _ptr(workspace),
                                          0 if workspace is None else workspace.numel() * workspace.element_size(),
                                          st))
    return importance


def prefill_desc(q: torch.Tensor, k_cache: torch.Tensor, scale: Optional[float] = None) -> PrefillDesc:
    B, Hq, N, D = q.shape
    return PrefillDesc(B, Hq, k_cache.shape[1], D, N, k_cache.shape[2],
                       float(1.0 / math.sqrt(D) if scale is None else scale))


def prefill_attn_stats(q: torch.Tensor, k_cache: torch.Tensor, prompt_len: torch.Tensor, scale: Optional[float] = None,
                       lse: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None,
                       with_lse: bool = True, with_entropy: bool = True, stream=None):
    """dreams_prefill_attn_stats: the causal attention of a prompt's own rows (row i sees slots 0..i).  q
    [B,Hq,N,D] and k_cache [B,Hkv,S_cap,D] bf16, prompt_len [B] int32.  Returns (lse, entropy), each [B,Hq,N]
    float32 or None."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return prefill_attn_stats(q, k_cache, prompt_len, scale, lse, entropy, with_lse, with_entropy)
    dev = q.device
    _need(q, "q", torch.bfloat16, dev, 4)
    _need(k_cache, "k_cache", torch.bfloat16, dev, 4)
    _need(prompt_len, "prompt_len", torch.int32, dev, 1)
    B, Hq, N, D = q.shape
    if with_lse and lse is None:
        lse = torch.empty((B, Hq, N), dtype=torch.float32, device=dev)
    if with_entropy and entropy is None:
        entropy = torch.empty((B, Hq, N), dtype=torch.float32, device=dev)
    for t, nm in ((lse, "lse"), (entropy, "entropy")):
        if t is not None:
            _need(t, nm, torch.float32, dev, 3)
    desc = prefill_desc(q, k_cache, scale)
    _check(lib().dreams_prefill_attn_stats(ctypes.byref(desc), _ptr(q), _ptr(k_cache), _ptr(prompt_len), _ptr(lse),
                                           _ptr(entropy), _stream(stream)))
    return lse, entropy


def prefill_attn_entropy_mean(entropy: torch.Tensor, prompt_len: torch.Tensor, ae: Optional[torch.Tensor] = None,
                              stream=None) -> torch.Tensor:
    """dreams_prefill_attn_entropy_mean: AE of one layer over prompts from entropy [B,Hq,N].  Returns [1] float32."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return prefill_attn_entropy_mean(entropy, prompt_len, ae)
    _need(entropy, "entropy", torch.float32, entropy.device, 3)
    _need(prompt_len, "prompt_len", torch.int32, entropy.device, 1)
    if ae is None:
        ae = torch.empty(1, dtype=torch.float32, device=entropy.device)
    B, Hq, N = entropy.shape
    _check(lib().dreams_prefill_attn_entropy_mean(B, Hq, N, _ptr(entropy), _ptr(prompt_len), _ptr(ae),
                                                  _stream(stream)))
    return ae


def prefill_visual_importance_workspace_size(batch: int, num_kv_heads: int, vis_count: int) -> int:
    """Bytes that hold the partial sums of every piece a prompt's rows are cut into; a workspace of
    visual_importance_workspace_size bytes serves too, with fewer pieces."""
    n = ctypes.c_size_t(0)
    _check(lib().dreams_prefill_visual_importance_workspace_size(batch, num_kv_heads, vis_count, ctypes.byref(n)))
    return n.value


def prefill_visual_importance(q: torch.Tensor, k_cache: torch.Tensor, prompt_len: torch.Tensor, lse: torch.Tensor,
                              vis_begin: int, vis_count: int, scale: Optional[float] = None,
                              importance: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                              stream=None) -> torch.Tensor:
    """dreams_prefill_visual_importance (Eq. 2 over the prompt's causal attention): lse [B,Hq,N] from
    prefill_attn_stats.  Returns importance [B, vis_count] float32."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return prefill_visual_importance(q, k_cache, prompt_len, lse, vis_begin, vis_count, scale, importance,
                                             workspace)
    dev = q.device
    _need(q, "q", torch.bfloat16, dev, 4)
    _need(k_cache, "k_cache", torch.bfloat16, dev, 4)
    _need(prompt_len, "prompt_len", torch.int32, dev, 1)
    _need(lse, "lse", torch.float32, dev, 3)
    B = q.shape[0]
    if importance is None:
        importance = torch.empty((B, vis_count), dtype=torch.float32, device=dev)
    else:
        _need(importance, "importance", torch.float32, dev)
    st = _stream(stream)
    if workspace is None:
        workspace = _workspace("visual", prefill_visual_importance_workspace_size(B, k_cache.shape[1], vis_count), dev, st)
    desc = prefill_desc(q, k_cache, scale)
    _check(lib().dreams_prefill_visual_importance(ctypes.byref(desc), _ptr(q), _ptr(k_cache), _ptr(prompt_len),
                                                  _ptr(lse), vis_begin, vis_count, _ptr(importance), _ptr(workspace),
                                                  0 if workspace is None else workspace.numel() * workspace.element_size(),
                                                  st))
    return importance


def visual_topk(importance: torch.Tensor, keep_count: int, keep: Optional[torch.Tensor] = None,
                stream=None) -> torch.Tensor:
    """dreams_visual_topk: importance [B, n] float32 -> keep [B, keep_count] int32 (increasing token order)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return visual_topk(importance, keep_count, keep)
    _need(importance, "importance", torch.float32, importance.device, 2)
    B, n = importance.shape
    if keep is None:
        keep = torch.empty((B, keep_count), dtype=torch.int32, device=importance.device)
    else:
        _need(keep, "keep", torch.int32, importance.device, 2)
    _check(lib().dreams_visual_topk(B, n, keep_count, _ptr(importance), _ptr(keep), _stream(stream)))
    return keep


def visual_gather(k_cache: torch.Tensor, v_cache: torch.Tensor, vis_begin: int, keep: torch.Tensor,
                  k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None, stream=None):
    """dreams_visual_gather: the kept visual tokens' K/V rows -> (k_out, v_out) [B, Hkv, keep_count, D]."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return visual_gather(k_cache, v_cache, vis_begin, keep, k_out, v_out)
    dt = k_cache.dtype
    dev = k_cache.device
    _need(k_cache, "k_cache", dt, dev, 4)
    _need(v_cache, "v_cache", dt, dev, 4)
    _need(keep, "keep", torch.int32, dev, 2)
    B, Hkv, S, D = k_cache.shape
    r = keep.shape[1]
    if k_out is None:
        k_out = torch.empty((B, Hkv, r, D), dtype=dt, device=dev)
    if v_out is None:
        v_out = torch.empty((B, Hkv, r, D), dtype=dt, device=dev)
    _check(lib().dreams_visual_gather(B, Hkv, D, S, DREAMS_BF16 if dt == torch.bfloat16 else DREAMS_F32,
                                      _ptr(k_cache), _ptr(v_cache), vis_begin, _ptr(keep), r, _ptr(k_out),
                                      _ptr(v_out), _stream(stream)))
    return k_out, v_out


def _verify_attn(q, k_cache, v_cache, kv_len, parent, tree_mask, scale, out, lse, with_lse, max_kv_len, num_splits,
                 workspace, stream, entropy):
    dt = q.dtype
    if dt not in (torch.bfloat16, torch.float32):
        raise TypeError("q must be bfloat16 or float32")
    dev = q.device
    _need(q, "q", dt, dev, 4)
    _need(k_cache, "k_cache", dt, dev, 4)
    _need(v_cache, "v_cache", dt, dev, 4)
    _need(kv_len, "kv_len", torch.int32, dev, 1)
    if k_cache.shape != v_cache.shape:
        raise ValueError("k_cache and v_cache shapes differ")
    B, Hq, T, D = q.shape
    if k_cache.shape[0] != B or k_cache.shape[3] != D or kv_len.shape[0] != B:
        raise ValueError("batch / head_dim mismatch between q, caches and kv_len")
    if parent is not None:
        _need(parent, "parent", torch.int32, dev, 2)
        if tuple(parent.shape) != (B, T):
            raise ValueError("parent must be [B, T]")
    if tree_mask is not None:
        _need(tree_mask, "tree_mask", torch.int64, dev, 3)
        if tuple(tree_mask.shape) != (B, T, (T + 63) // 64):
            raise ValueError("tree_mask must be [B, T, ceil(T/64)]")
    desc = attn_desc(q, k_cache, num_splits, max_kv_len, scale)
    if out is None:
        out = torch.empty_like(q)
    else:
        _need(out, "out", dt, dev)
        if out.shape != q.shape:
            raise ValueError("out must have q's shape")
    if lse is None and with_lse:
        lse = torch.empty((B, Hq, T), dtype=torch.float32, device=dev)
    elif lse is not None:
        _need(lse, "lse", torch.float32, dev)
        if tuple(lse.shape) != (B, Hq, T):
            raise ValueError("lse must be [B, Hq, T]")
    st = _stream(stream)
    nbytes = tree_verify_attn_workspace_size(desc)
    if workspace is None:
        workspace = _workspace("attn", nbytes, dev, st)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if entropy is None:
        _check(lib().dreams_tree_verify_attn(ctypes.byref(desc), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(kv_len),
                                             _ptr(parent), _ptr(tree_mask), _ptr(out), _ptr(lse), _ptr(workspace),
                                             ws_bytes, st))
    else:
        _check(lib().dreams_tree_verify_attn_entropy(ctypes.byref(desc), _ptr(q), _ptr(k_cache), _ptr(v_cache),
                                                     _ptr(kv_len), _ptr(parent), _ptr(tree_mask), _ptr(out), _ptr(lse),
                                                     _ptr(entropy), _ptr(workspace), ws_bytes, st))
    return out, lse, entropy


def tree_verify_attn_noalloc(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, kv_len: torch.Tensor,
                             parent: Optional[torch.Tensor] = None, tree_mask: Optional[torch.Tensor] = None,
                             scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                             lse: Optional[torch.Tensor] = None, with_lse: bool = True, max_kv_len: int = 0,
                             num_splits: int = 0, stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """dreams_tree_verify_attn_noalloc: tree_verify_attn without a workspace (the library's fixed scratch array
    instead).  `out` and `lse` may be passed in so that nothing is allocated here either."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return tree_verify_attn_noalloc(q, k_cache, v_cache, kv_len, parent, tree_mask, scale, out, lse, with_lse,
                                            max_kv_len, num_splits)
    dt = q.dtype
    if dt not in (torch.bfloat16, torch.float32):
        raise TypeError("q must be bfloat16 or float32")
    dev = q.device
    for t, name in ((q, "q"), (k_cache, "k_cache"), (v_cache, "v_cache")):
        _need(t, name, dt, dev, 4)
    _need(kv_len, "kv_len", torch.int32, dev, 1)
    if parent is not None:
        _need(parent, "parent", torch.int32, dev, 2)
    if tree_mask is not None:
        _need(tree_mask, "tree_mask", torch.int64, dev, 3)
    B, Hq, T, D = q.shape
    desc = attn_desc(q, k_cache, num_splits, max_kv_len, scale)
    if out is None:
        out = torch.empty_like(q)
    _need(out, "out", dt, dev)
    if out.shape != q.shape:
        raise ValueError("out must have q's shape")
    if lse is None and with_lse:
        lse = torch.empty((B, Hq, T), dtype=torch.float32, device=dev)
    if lse is not None:
        _need(lse, "lse", torch.float32, dev)
        if tuple(lse.shape) != (B, Hq, T):
            raise ValueError("lse must be [B, Hq, T]")
    _check(lib().dreams_tree_verify_attn_noalloc(ctypes.byref(desc), _ptr(q), _ptr(k_cache), _ptr(v_cache),
                                                 _ptr(kv_len), _ptr(parent), _ptr(tree_mask), _ptr(out), _ptr(lse),
                                                 _stream(stream)))
    return out, lse


def tree_accept_workspace_size(batch: int, num_nodes: int, vocab: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().dreams_tree_accept_workspace_size(batch, num_nodes, vocab, ctypes.byref(n)))
    return n.value


def tree_accept(target_logits: torch.Tensor, draft_tokens: torch.Tensor, parent: torch.Tensor,
                want_target_argmax: bool = False, outputs=None, workspace: Optional[torch.Tensor] = None,
                stream=None):
    """dreams_tree_accept.  target_logits [B,T,V] float32, draft_tokens / parent [B,T] int32.
    Returns (accept_len [B], accept_path [B,T], next_token [B], target_argmax [B,T] or None), all int32.
    `outputs` may pass preallocated (accept_len, accept_path, next_token, target_argmax-or-None)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return tree_accept(target_logits, draft_tokens, parent, want_target_argmax, outputs, workspace)
    dev = target_logits.device
    _need(target_logits, "target_logits", torch.float32, dev, 3)
    B, T, V = target_logits.shape
    _need(draft_tokens, "draft_tokens", torch.int32, dev, 2)
    _need(parent, "parent", torch.int32, dev, 2)
    if tuple(draft_tokens.shape) != (B, T) or tuple(parent.shape) != (B, T):
        raise ValueError("draft_tokens and parent must be [B, T]")
    if outputs is None:
        alen = torch.empty(B, dtype=torch.int32, device=dev)
        path = torch.empty((B, T), dtype=torch.int32, device=dev)
        nxt = torch.empty(B, dtype=torch.int32, device=dev)
        am = torch.empty((B, T), dtype=torch.int32, device=dev) if want_target_argmax else None
    else:
        alen, path, nxt, am = outputs
        for t, nm, shp in ((alen, "accept_len", (B,)), (path, "accept_path", (B, T)), (nxt, "next_token", (B,))):
            _need(t, nm, torch.int32, dev)
            if tuple(t.shape) != shp:
                raise ValueError("%s has the wrong shape" % nm)
        if am is not None:
            _need(am, "target_argmax", torch.int32, dev)
    st = _stream(stream)
    nbytes = tree_accept_workspace_size(B, T, V)
    if workspace is None:
        workspace = _workspace("accept", nbytes, dev, st)
    _check(lib().dreams_tree_accept(B, T, V, _ptr(target_logits), _ptr(draft_tokens), _ptr(parent), _ptr(alen),
                                    _ptr(path), _ptr(nxt), _ptr(am), _ptr(workspace),
                                    0 if workspace is None else workspace.numel(), st))
    return alen, path, nxt, am


def tree_accept_sampled_workspace_size(batch: int, num_nodes: int, vocab: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().dreams_tree_accept_sampled_workspace_size(batch, num_nodes, vocab, ctypes.byref(n)))
    return n.value


def tree_accept_sampled(target_logits: torch.Tensor, draft_logits: torch.Tensor, draft_tokens: torch.Tensor,
                        parent: torch.Tensor, uniforms: torch.Tensor, temperature: float = 1.0, outputs=None,
                        workspace: Optional[torch.Tensor] = None, stream=None):
    """dreams_tree_accept_sampled.  target_logits / draft_logits [B,T,V] float32, draft_tokens / parent [B,T]
    int32, uniforms [B,T] float32 in [0, 1).  Returns (accept_len [B], accept_path [B,T], next_token [B]), int32.
    `outputs` may pass preallocated (accept_len, accept_path, next_token)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return tree_accept_sampled(target_logits, draft_logits, draft_tokens, parent, uniforms, temperature,
                                       outputs, workspace)
    dev = target_logits.device
    _need(target_logits, "target_logits", torch.float32, dev, 3)
    B, T, V = target_logits.shape
    _need(draft_logits, "draft_logits", torch.float32, dev, 3)
    if tuple(draft_logits.shape) != (B, T, V):
        raise ValueError("draft_logits must have the shape of target_logits")
    _need(draft_tokens, "draft_tokens", torch.int32, dev, 2)
    _need(parent, "parent", torch.int32, dev, 2)
    _need(uniforms, "uniforms", torch.float32, dev, 2)
    if tuple(draft_tokens.shape) != (B, T) or tuple(parent.shape) != (B, T) or tuple(uniforms.shape) != (B, T):
        raise ValueError("draft_tokens, parent and uniforms must be [B, T]")
    if outputs is None:
        alen = torch.empty(B, dtype=torch.int32, device=dev)
        path = torch.empty((B, T), dtype=torch.int32, device=dev)
        nxt = torch.empty(B, dtype=torch.int32, device=dev)
    else:
        alen, path, nxt = outputs
        for t, nm, shp in ((alen, "accept_len", (B,)), (path, "accept_path", (B, T)), (nxt, "next_token", (B,))):
            _need(t, nm, torch.int32, dev)
            if tuple(t.shape) != shp:
                raise ValueError("%s has the wrong shape" % nm)
    st = _stream(stream)
    nbytes = tree_accept_sampled_workspace_size(B, T, V)
    if workspace is None:
        workspace = _workspace("accept_sampled", nbytes, dev, st)
    _check(lib().dreams_tree_accept_sampled(B, T, V, float(temperature), _ptr(target_logits), _ptr(draft_logits),
                                            _ptr(draft_tokens), _ptr(parent), _ptr(uniforms), _ptr(alen),
                                            _ptr(path), _ptr(nxt), _ptr(workspace),
                                            0 if workspace is None else workspace.numel(), st))
    return alen, path, nxt


def tree_accept_lm_head_workspace_size(batch: int, num_nodes: int, hidden: int, vocab: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().dreams_tree_accept_lm_head_workspace_size(batch, num_nodes, hidden, vocab, ctypes.byref(n)))
    return n.value


def tree_accept_lm_head(hidden_states: torch.Tensor, lm_weight: torch.Tensor, draft_tokens: torch.Tensor,
                        parent: torch.Tensor, want_target_argmax: bool = False, outputs=None,
                        workspace: Optional[torch.Tensor] = None, stream=None):
    """dreams_tree_accept_lm_head.  hidden_states [B,T,H] bfloat16, lm_weight [V,H] bfloat16, draft_tokens /
    parent [B,T] int32.  Returns (accept_len [B], accept_path [B,T], next_token [B], target_argmax [B,T] or
    None), all int32.  `outputs` may pass preallocated (accept_len, accept_path, next_token, target_argmax)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return tree_accept_lm_head(hidden_states, lm_weight, draft_tokens, parent, want_target_argmax, outputs,
                                       workspace)
    dev = hidden_states.device
    _need(hidden_states, "hidden_states", torch.bfloat16, dev, 3)
    B, T, H = hidden_states.shape
    _need(lm_weight, "lm_weight", torch.bfloat16, dev, 2)
    V = lm_weight.shape[0]
    if lm_weight.shape[1] != H:
        raise ValueError("lm_weight must be [V, H] with the hidden size of hidden_states")
    _need(draft_tokens, "draft_tokens", torch.int32, dev, 2)
    _need(parent, "parent", torch.int32, dev, 2)
    if tuple(draft_tokens.shape) != (B, T) or tuple(parent.shape) != (B, T):
        raise ValueError("draft_tokens and parent must be [B, T]")
    if outputs is None:
        alen = torch.empty(B, dtype=torch.int32, device=dev)
        path = torch.empty((B, T), dtype=torch.int32, device=dev)
        nxt = torch.empty(B, dtype=torch.int32, device=dev)
        am = torch.empty((B, T), dtype=torch.int32, device=dev) if want_target_argmax else None
    else:
        alen, path, nxt, am = outputs
        for t, nm, shp in ((alen, "accept_len", (B,)), (path, "accept_path", (B, T)), (nxt, "next_token", (B,))):
            _need(t, nm, torch.int32, dev)
            if tuple(t.shape) != shp:
                raise ValueError("%s has the wrong shape" % nm)
        if am is not None:
            _need(am, "target_argmax", torch.int32, dev)
    st = _stream(stream)
    nbytes = tree_accept_lm_head_workspace_size(B, T, H, V)
    if workspace is None:
        workspace = _workspace("accept_lm_head", nbytes, dev, st)
    _check(lib().dreams_tree_accept_lm_head(B, T, H, V, _ptr(hidden_states), _ptr(lm_weight), _ptr(draft_tokens),
                                            _ptr(parent), _ptr(alen), _ptr(path), _ptr(nxt), _ptr(am),
                                            _ptr(workspace), 0 if workspace is None else workspace.numel(), st))
    return alen, path, nxt, am


def kv_commit(k_cache: torch.Tensor, v_cache: torch.Tensor, kv_len_in: torch.Tensor, accept_path: torch.Tensor,
              accept_len: torch.Tensor, kv_len_out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """dreams_kv_commit, in place on k_cache / v_cache of shape [NL, B, Hkv, S_cap, D] (or [B, Hkv, S_cap, D]
    for one layer).  Returns kv_len_out [B] int32."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return kv_commit(k_cache, v_cache, kv_len_in, accept_path, accept_len, kv_len_out)
    dt = k_cache.dtype
    if dt not in (torch.bfloat16, torch.float32):
        raise TypeError("caches must be bfloat16 or float32")
    dev = k_cache.device
    _need(k_cache, "k_cache", dt, dev)
    _need(v_cache, "v_cache", dt, dev)
    if k_cache.shape != v_cache.shape or k_cache.dim() not in (4, 5):
        raise ValueError("caches must share a [NL,]B,Hkv,S_cap,D shape")
    shp = k_cache.shape if k_cache.dim() == 5 else (1,) + tuple(k_cache.shape)
    NL, B, Hkv, S_cap, D = shp
    _need(kv_len_in, "kv_len_in", torch.int32, dev, 1)
    _need(accept_path, "accept_path", torch.int32, dev, 2)
    _need(accept_len, "accept_len", torch.int32, dev, 1)
    if kv_len_out is None:
        kv_len_out = torch.empty(B, dtype=torch.int32, device=dev)
    _need(kv_len_out, "kv_len_out", torch.int32, dev, 1)
    if kv_len_in.shape[0] != B or accept_len.shape[0] != B or accept_path.shape[0] != B or kv_len_out.shape[0] != B:
        raise ValueError("length / path arrays must have the cache's batch size")
    _check(lib().dreams_kv_commit(NL, B * Hkv * S_cap * D, B, Hkv, D, S_cap,
                                  DREAMS_BF16 if dt == torch.bfloat16 else DREAMS_F32, _ptr(k_cache), _ptr(v_cache),
                                  _ptr(kv_len_in), _ptr(accept_path), _ptr(accept_len), accept_path.shape[1],
                                  _ptr(kv_len_out), _stream(stream)))
    return kv_len_out


def check_tree_host(parent) -> None:
    """dreams_check_tree_host on a host int32 array; raises DreamsError if it is not a valid parent array."""
    import numpy as np
    p = np.ascontiguousarray(parent, dtype=np.int32)
    _check(lib().dreams_check_tree_host(p.ctypes.data_as(ctypes.c_void_p), int(p.shape[0])))


STREAM_READ_SINK_WORDS = 2048


def stream_read(src: torch.Tensor, sink: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """dreams_stream_read: one plain read of every byte of `src` (a contiguous device tensor whose size is a
    multiple of 16 bytes), for measuring read bandwidth.  Returns the sink words."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return stream_read(src, sink)
    if not src.is_contiguous():
        raise ValueError("src must be contiguous")
    if sink is None:
        sink = torch.empty(STREAM_READ_SINK_WORDS, dtype=torch.int32, device=src.device)
    _check(lib().dreams_stream_read(_ptr(src), src.numel() * src.element_size(), _ptr(sink), _stream(stream)))
    return sink


# ---------------------------------------------------------------------------------------------------- paged cache
PAGES_MAX, PAGES_MAX_SEQUENCES = 524288, 4096

# (small calls take as long as the host does: torch's calls without their wrappers, where it has them)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_capturing = getattr(torch._C, "_cuda_isCurrentStreamCapturing", torch.cuda.is_current_stream_capturing)


def _stream_on(stream, at) -> int:
    """_stream, where `at` is the current device: a stream of another one would run the kernels there."""
    if stream is None:
        return _raw_stream(at) if _raw_stream is not None else _stream(None)
    if stream.device.index != at:
        raise ValueError("stream is on %s, not on the current device" % (stream.device,))
    return stream.cuda_stream


def _new(t: torch.Tensor, stream, shape=None, dtype=None) -> torch.Tensor:
    """An output like t, allocated on the stream that writes it: memory of the current stream's may still be in use there."""
    if stream is None:
        return torch.empty_like(t) if shape is None else t.new_empty(shape, dtype=dtype)
    captured = _capturing()
    with torch.cuda.stream(stream):
        if captured and not _capturing():
            raise ValueError("a call on another stream than the captured one needs a workspace and its outputs given")
        return _new(t, None, shape, dtype)


def _dense_like(t: torch.Tensor, stream) -> torch.Tensor:
    """A dense output of t's shape and type (_new)."""
    if stream is None:
        return torch.empty_like(t, memory_format=torch.contiguous_format)
    return _new(t, stream, t.shape, t.dtype)


def _code(dtype, what: str = "pages") -> int:
    if dtype is torch.bfloat16:
        return DREAMS_BF16
    if dtype is torch.float32:
        return DREAMS_F32
    raise TypeError("%s must be bfloat16 or float32" % what)


def _current(t: torch.Tensor, name: str, dtype=None) -> int:
    """The tensor's device index.  Kernels are launched on the current device: its tensors only."""
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if dtype is not None and t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    at = t.get_device()
    if at < 0:
        raise ValueError("%s must be a device tensor" % name)
    if at != _current_device():
        raise ValueError("%s is on %s, not on the current device" % (name, t.device))
    return at


def _need_on(t: torch.Tensor, name: str, dtype, at: int, shape=None, ndim=None):
    """As _need, for a device index, a whole shape or a number of dimensions."""
    try:
        if (t.dtype is dtype and t.get_device() == at and t.is_contiguous() and (shape is None or t.shape == shape)
                and (ndim is None or t.dim() == ndim)):
            return
    except AttributeError:
        pass
    _need(t, name, dtype, torch.device("cuda", at), ndim)
    raise ValueError("%s must be %s, got %s" % (name, list(shape), list(t.shape)))


def _page_strides(k_pages: torch.Tensor, v_pages: torch.Tensor):
    """(shape, layer stride, page stride) of a pool [NL, P, Hkv, page_size, D] or [P, Hkv, page_size, D] whose pages are
    dense (a page's K and V may lie side by side in one buffer); strides in elements."""
    for t, name in ((k_pages, "k_pages"), (v_pages, "v_pages")):
        if not isinstance(t, torch.Tensor):
            raise TypeError("%s must be a torch.Tensor" % name)
    shape = k_pages.shape
    if k_pages.dtype is not v_pages.dtype:
        raise TypeError("k_pages and v_pages differ in dtype")
    if k_pages.get_device() != v_pages.get_device():
        raise ValueError("k_pages and v_pages are on different devices")
    if shape != v_pages.shape:
        raise ValueError("k_pages and v_pages differ in shape")
    n = len(shape)
    if n not in (4, 5):
        raise ValueError("k_pages and v_pages must be [NL,] num_pages, Hkv, page_size, D")
    P, H, S, D = shape[-4:]
    if k_pages.is_contiguous() and v_pages.is_contiguous():      # (most pools: nothing else to look at)
        return shape, P * H * S * D if n == 5 and shape[0] > 1 else 0, H * S * D
    st, vst = k_pages.stride(), v_pages.stride()
    # (a stride along an axis of one entry is not used)
    if st != vst and any(shape[i] > 1 and st[i] != vst[i] for i in range(n)):
        raise ValueError("k_pages and v_pages differ in layout")
    if st[-3:] != (S * D, D, 1) and any(shape[i] > 1 and st[i] != dense
                                       for i, dense in ((n - 1, 1), (n - 2, D), (n - 3, S * D))):
        raise ValueError("pages must be dense [Hkv, page_size, D]")
    if (P > 1 and st[-4] == 0) or (n == 5 and shape[0] > 1 and st[0] == 0):   # (0 means dense below)
        raise ValueError("pages or layers share memory (expanded views)")
    return shape, st[0] if n == 5 and shape[0] > 1 else 0, st[-4] if P > 1 else H * S * D


def _pool(k_pages, v_pages, page_table, code=None):
    """(PagePool, device index)"""
    shape, layer, page = _page_strides(k_pages, v_pages)
    at = _current(k_pages, "k_pages")
    _need_on(page_table, "page_table", torch.int32, at, None, 2)
    P, H, S, D = shape[-4:]
    B, width = page_table.shape
    return PagePool(shape[0] if len(shape) == 5 else 1, B, H, D, P, S, width,
                    _code(k_pages.dtype) if code is None else code, layer, page), at


def _table_pool(page_table, page_count, refcount, page_size):
    """(PagePool, device index)"""
    at = _current(page_table, "page_table", torch.int32)
    if not 0 < page_size < 2 ** 31:
        raise ValueError("page_size must be in [1, 2^31)")
    _need_on(page_table, "page_table", torch.int32, at, None, 2)
    B, width = page_table.shape
    _need_on(page_count, "page_count", torch.int32, at, (B,))
    _need_on(refcount, "refcount", torch.int32, at, None, 1)
    return PagePool(1, B, 1, 64, refcount.shape[0], page_size, width, DREAMS_BF16, 0, 0), at


def paged_desc(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor, window: int = 0,
               sinks: int = 0, max_kv_len: int = 0, num_splits: int = 0, scale: Optional[float] = None) -> PagedDesc:
    """The description of an attention call over pages; checks the tensors' types, devices and shapes."""
    return _paged_desc(q, k_pages, v_pages, page_table, getattr(k_pages, "dtype", None), window, sinks, max_kv_len, num_splits,
                       scale)


def _paged_desc(q, k_pages, v_pages, page_table, dt, window, sinks, max_kv_len, num_splits, scale) -> PagedDesc:
    """... with queries of type dt."""
    shape, _, page = _page_strides(k_pages, v_pages)
    if len(shape) != 4:
        raise ValueError("attention takes one layer's pages: [num_pages, Hkv, page_size, D]")
    code = _code(dt)
    at = _current(q, "q")
    if k_pages.get_device() != at:
        raise ValueError("k_pages is on %s, expected %s" % (k_pages.device, q.device))
    _need_on(q, "q", dt, at, None, 4)
    _need_on(page_table, "page_table", torch.int32, at, None, 2)
    if not (-1 < window < 2 ** 31 and -1 < sinks < 2 ** 31 and -1 < max_kv_len < 2 ** 31 and -1 < num_splits < 2 ** 31):
        raise ValueError("window, sinks, max_kv_len and num_splits must be in [0, 2^31)")
    B, Hq, T, D = q.shape
    P, H, S, Dk = shape
    Bt, width = page_table.shape
    if Dk != D or Bt != B:
        raise ValueError("batch / head_dim mismatch between q, the pages and page_table")
    return PagedDesc(B, Hq, H, D, T, P, S, width, max_kv_len, num_splits, window, sinks, code,
                     1.0 / math.sqrt(D) if scale is None else scale, page)


WORKSPACE_COUNTER_BYTES = 65536


def _call_paged(call, size, desc, tensors, workspace, at, stream):
    """An attention call with the caller's workspace, or the binding's own (one per device and stream; under capture one
    that belongs to the graph, its counters cleared by every replay, so that no two graphs share one)."""
    st = _stream_on(stream, at)
    if workspace is not None:
        if workspace.get_device() != at or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous tensor on the call's device")
        _check(call(desc, *tensors, _ptr(workspace), workspace.numel() * workspace.element_size(), st))
        return
    capturing = _capturing()
    if stream is not None and stream.cuda_stream != torch.cuda.current_stream().cuda_stream:
        with torch.cuda.stream(stream):
            capturing |= _capturing()
        if capturing:
            raise ValueError("a call captured on another stream than the current one needs a workspace")
    if capturing:
        device = torch.device("cuda", at)
        n = ctypes.c_size_t(0)
        _check(size(desc, ctypes.byref(n)))
        ws = None
        if n.value:
            ws = torch.empty(n.value, dtype=torch.uint8, device=device)
            ws[:WORKSPACE_COUNTER_BYTES].zero_()
        _check(call(desc, *tensors, _ptr(ws), n.value, st))
        return
    ws = _ws.get(("paged", at, st))
    status = call(desc, *tensors, _ptr(ws), 0 if ws is None else ws.numel(), st)
    if status == DREAMS_ERR_WORKSPACE:      # (nothing was enqueued: the first call, or the first of this size)
        n = ctypes.c_size_t(0)
        _check(size(desc, ctypes.byref(n)))
        device = torch.device("cuda", at)
        if stream is None:
            ws = _workspace("paged", n.value, device, st)
        else:
            with torch.cuda.stream(stream):
                ws = _workspace("paged", n.value, device, st)
        status = call(desc, *tensors, _ptr(ws), ws.numel(), st)
    _check(status)


def _paged_outputs(q, out, lse, with_lse, stream):
    at = q.get_device()
    if out is None:
        out = torch.empty_like(q) if stream is None else _new(q, stream)
    else:
        _need_on(out, "out", q.dtype, at, q.shape)
    if lse is not None:
        _need_on(lse, "lse", torch.float32, at, q.shape[:3])
    elif with_lse:
        B, H, T, _ = q.shape
        lse = q.new_empty(B, H, T, dtype=torch.float32) if stream is None else _new(q, stream, (B, H, T), torch.float32)
    return out, lse


def paged_verify_attn_workspace_size(desc: PagedDesc) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().dreams_paged_verify_attn_workspace_size(ctypes.byref(desc), ctypes.byref(n)))
    return n.value


def paged_prompt_attn_workspace_size(desc: PagedDesc) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().dreams_paged_prompt_attn_workspace_size(ctypes.byref(desc), ctypes.byref(n)))
    return n.value


def paged_verify_attn(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor,
                      kv_len: torch.Tensor, parent: Optional[torch.Tensor] = None,
                      tree_mask: Optional[torch.Tensor] = None, window: int = 0, sinks: int = 0,
                      scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                      lse: Optional[torch.Tensor] = None, with_lse: bool = True, max_kv_len: int = 0, num_splits: int = 0,
                      workspace: Optional[torch.Tensor] = None,
                      stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """dreams_paged_verify_attn.  q [B,Hq,T,D]; k_pages/v_pages [num_pages,Hkv,page_size,D] (bf16 or fp32, same as q;
    dense pages, any page stride); page_table [B,width] and kv_len [B] int32; parent [B,T] int32 and/or tree_mask
    [B,T,ceil(T/64)] int64 (bit patterns; a window needs parent).  Keys more than `window` - 1 positions before a node are
    out of its sight, but for the first `sinks` (window 0: none is).  max_kv_len bounds kv_len for the plan (0: the table's
    width; max(1, longest) where it is known, 1 without a prefix).  A row's own slots hold finite values.  Returns (out, lse
    [B,Hq,T] float32 or None); what a call over pages allocates belongs to the stream it runs on."""
    desc = _paged_desc(q, k_pages, v_pages, page_table, getattr(k_pages, "dtype", None), window, sinks, max_kv_len, num_splits,
                       scale)
    B, T, at = desc.batch, desc.num_rows, q.get_device()
    _need_on(kv_len, "kv_len", torch.int32, at, (B,))
    if parent is not None:
        _need_on(parent, "parent", torch.int32, at, (B, T))
    if tree_mask is not None:
        _need_on(tree_mask, "tree_mask", torch.int64, at, (B, T, (T + 63) // 64))
    out, lse = _paged_outputs(q, out, lse, with_lse, stream)
    L = lib()
    _call_paged(L.dreams_paged_verify_attn, L.dreams_paged_verify_attn_workspace_size, ctypes.byref(desc),
                (q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), page_table.data_ptr(), kv_len.data_ptr(),
                 _ptr(parent), _ptr(tree_mask), out.data_ptr(), _ptr(lse)), workspace, at, stream)
    return out, lse


def paged_prompt_attn(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor,
                      kv_len: torch.Tensor, row_len: Optional[torch.Tensor] = None, window: int = 0, sinks: int = 0,
                      scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                      lse: Optional[torch.Tensor] = None, with_lse: bool = True, max_kv_len: int = 0, num_splits: int = 0,
                      workspace: Optional[torch.Tensor] = None,
                      stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """dreams_paged_prompt_attn: causal attention of prompt rows at positions kv_len[b] + i, whose K/V the pages hold
    already.  q [B,Hq,N,D]; row_len [B] int32 live rows (None: N each; the others give 0 and -inf); the rest as for
    paged_verify_attn.  Returns (out, lse [B,Hq,N] float32 or None)."""
    desc = _paged_desc(q, k_pages, v_pages, page_table, getattr(k_pages, "dtype", None), window, sinks, max_kv_len, num_splits,
                       scale)
    B, at = desc.batch, q.get_device()
    _need_on(kv_len, "kv_len", torch.int32, at, (B,))
    if row_len is not None:
        _need_on(row_len, "row_len", torch.int32, at, (B,))
    out, lse = _paged_outputs(q, out, lse, with_lse, stream)
    L = lib()
    _call_paged(L.dreams_paged_prompt_attn, L.dreams_paged_prompt_attn_workspace_size, ctypes.byref(desc),
                (q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), page_table.data_ptr(), kv_len.data_ptr(),
                 _ptr(row_len), out.data_ptr(), _ptr(lse)), workspace, at, stream)
    return out, lse


_Strides = ctypes.c_int64 * 4


def _new_rows(k_new, v_new, k_pages, pool, at, dt, kv_len, row_len):
    """The strides of new rows of type dt, once they and their lengths are checked against the pool."""
    B, n = pool.batch, k_pages.dim()
    try:
        shape, st = k_new.shape, k_new.stride()
        plain = (k_new.dtype is dt and v_new.dtype is dt and k_new.get_device() == at == v_new.get_device()
                 and shape == v_new.shape and st == v_new.stride() and len(shape) == n and st[-1] == 1
                 and shape[-4] == B and shape[-3] == pool.num_kv_heads and shape[-1] == pool.head_dim
                 and (n == 4 or shape[0] == pool.num_layers))
    except AttributeError:
        plain = False
    if not plain:
        _check_new_rows(k_new, v_new, k_pages, pool, at, dt, n)
    _need_on(kv_len, "kv_len", torch.int32, at, (B,))
    if row_len is not None:
        _need_on(row_len, "row_len", torch.int32, at, (B,))
    return _Strides(0, st[0], st[1], st[2]) if n == 4 else _Strides(*st[:4])


def _check_new_rows(k_new, v_new, k_pages, pool, at, dt, n):
    B = pool.batch
    for t, name in ((k_new, "k_new"), (v_new, "v_new")):
        if not isinstance(t, torch.Tensor):
            raise TypeError("%s must be a torch.Tensor" % name)
        if t.dtype is not dt:
            raise TypeError("%s must be %s, got %s" % (name, dt, t.dtype))
        if t.get_device() != at:
            raise ValueError("%s is on %s, expected %s" % (name, t.device, k_pages.device))
    shape, st, vst = k_new.shape, k_new.stride(), v_new.stride()
    if len(shape) != n or shape[-4:-2] != (B, pool.num_kv_heads) or shape[-1] != pool.head_dim or (
            n == 5 and shape[0] != pool.num_layers):
        raise ValueError("k_new must be [NL,] B, Hkv, N, D like the pages")
    if shape != v_new.shape or (st != vst and any(shape[i] > 1 and st[i] != vst[i] for i in range(n))):
        raise ValueError("k_new and v_new differ in shape or layout")
    if shape[-1] > 1 and st[-1] != 1:
        raise ValueError("the rows of k_new and v_new must be dense")


def paged_append(k_new: torch.Tensor, v_new: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor,
                 page_table: torch.Tensor, kv_len: torch.Tensor, row_len: Optional[torch.Tensor] = None,
                 stream=None) -> None:
    """dreams_paged_append, in place on k_pages / v_pages [NL,num_pages,Hkv,page_size,D] (or one layer's, without NL):
    rows of k_new / v_new [NL,B,Hkv,N,D] (or without NL), of any strides with dense rows (a transposed view of a
    projection's [B,N,Hkv,D] serves), go to the slots kv_len[b] .. of every sequence; row_len [B] int32 of them (None: N)."""
    pool, at = _pool(k_pages, v_pages, page_table)
    strides = _new_rows(k_new, v_new, k_pages, pool, at, k_pages.dtype, kv_len, row_len)
    _check(lib().dreams_paged_append(ctypes.byref(pool), k_new.data_ptr(), v_new.data_ptr(), k_new.shape[-2], strides,
                                     page_table.data_ptr(), kv_len.data_ptr(), _ptr(row_len), k_pages.data_ptr(),
                                     v_pages.data_ptr(), _stream_on(stream, at)))


def _commit_lengths(B, at, kv_len_in, accept_path, accept_len, kv_len_out, stream):
    """kv_len_out, the caller's or a new one, once the lengths and the path are checked."""
    _need_on(kv_len_in, "kv_len_in", torch.int32, at, (B,))
    _need_on(accept_path, "accept_path", torch.int32, at, None, 2)
    if accept_path.shape[0] != B:
        raise ValueError("accept_path must have page_table's batch size")
    _need_on(accept_len, "accept_len", torch.int32, at, (B,))
    if kv_len_out is None:
        return _new(kv_len_in, stream)
    _need_on(kv_len_out, "kv_len_out", torch.int32, at, (B,))
    return kv_len_out


def paged_kv_commit(k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor, kv_len_in: torch.Tensor,
                    accept_path: torch.Tensor, accept_len: torch.Tensor, kv_len_out: Optional[torch.Tensor] = None,
                    stream=None) -> torch.Tensor:
    """dreams_paged_kv_commit, in place on k_pages / v_pages [NL,num_pages,Hkv,page_size,D] (or one layer's).  Returns
    kv_len_out [B] int32."""
    pool, at = _pool(k_pages, v_pages, page_table)
    kv_len_out = _commit_lengths(pool.batch, at, kv_len_in, accept_path, accept_len, kv_len_out, stream)
    _check(lib().dreams_paged_kv_commit(ctypes.byref(pool), k_pages.data_ptr(), v_pages.data_ptr(),
                                        page_table.data_ptr(), kv_len_in.data_ptr(), accept_path.data_ptr(),
                                        accept_len.data_ptr(), accept_path.shape[1],
                                        kv_len_out.data_ptr(), _stream_on(stream, at)))
    return kv_len_out


def pages_reserve(page_table: torch.Tensor, page_count: torch.Tensor, refcount: torch.Tensor, want_len: torch.Tensor,
                  page_size: int, granted: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """dreams_pages_reserve, in place on page_table [B,width], page_count [B] and refcount [num_pages] (int32): every
    sequence gets pages for want_len[b] slots, lowest free first.  Returns granted [B] int32 (1 or 0)."""
    pool, at = _table_pool(page_table, page_count, refcount, page_size)
    B = pool.batch
    _need_on(want_len, "want_len", torch.int32, at, (B,))
    if granted is None:
        granted = _new(want_len, stream)
    else:
        _need_on(granted, "granted", torch.int32, at, (B,))
    _check(lib().dreams_pages_reserve(ctypes.byref(pool), page_table.data_ptr(), page_count.data_ptr(),
                                      refcount.data_ptr(), want_len.data_ptr(), granted.data_ptr(), _stream_on(stream, at)))
    return granted


def _fork(call, head, pool, at, k_pages, v_pages, page_table, page_count, kv_len, refcount, src, dst, granted, stream):
    B = pool.batch
    _need_on(page_count, "page_count", torch.int32, at, (B,))
    _need_on(kv_len, "kv_len", torch.int32, at, (B,))
    _need_on(refcount, "refcount", torch.int32, at, (pool.num_pages,))
    _need_on(src, "src", torch.int32, at, None, 1)
    n = src.shape[0]
    _need_on(dst, "dst", torch.int32, at, (n,))
    if granted is None:
        granted = _new(src, stream)
    else:
        _need_on(granted, "granted", torch.int32, at, (n,))
    _check(call(*head, k_pages.data_ptr(), v_pages.data_ptr(), page_table.data_ptr(), page_count.data_ptr(),
                kv_len.data_ptr(), refcount.data_ptr(), n, src.data_ptr(), dst.data_ptr(), granted.data_ptr(),
                _stream_on(stream, at)))
    if B == 0:      # (no sequence to copy: the library has not written granted)
        with torch.cuda.stream(stream):
            granted.zero_()
    return granted


def pages_fork(k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor, page_count: torch.Tensor,
               kv_len: torch.Tensor, refcount: torch.Tensor, src: torch.Tensor, dst: torch.Tensor,
               granted: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """dreams_pages_fork, in place: sequence dst[i] (without pages) becomes a copy of sequence src[i]; whole pages are
    shared, the rows of a partly filled one copied in every layer.  Returns granted [n] int32 (1 or 0)."""
    pool, at = _pool(k_pages, v_pages, page_table)
    return _fork(lib().dreams_pages_fork, (ctypes.byref(pool),), pool, at, k_pages, v_pages, page_table, page_count, kv_len,
                 refcount, src, dst, granted, stream)


def pages_release(page_table: torch.Tensor, page_count: torch.Tensor, kv_len: torch.Tensor, refcount: torch.Tensor,
                  seqs: torch.Tensor, page_size: int, trim: bool = False, stream=None) -> None:
    """dreams_pages_release, in place: the sequences seqs [n] int32 give up all their pages (kv_len becomes 0) or, with
    trim, those past the ones that their kv_len slots need."""
    pool, at = _table_pool(page_table, page_count, refcount, page_size)
    _need_on(kv_len, "kv_len", torch.int32, at, (pool.batch,))
    _need_on(seqs, "seqs", torch.int32, at, None, 1)
    _check(lib().dreams_pages_release(ctypes.byref(pool), page_table.data_ptr(), page_count.data_ptr(),
                                      kv_len.data_ptr(), refcount.data_ptr(), seqs.shape[0], seqs.data_ptr(),
                                      1 if trim else 0, _stream_on(stream, at)))


# ------------------------------------------------------------------------------------------- rotary positions
ROPE_SCALINGS = {None: 0, "linear": 1, "parts": 2}
_Strides3 = ctypes.c_int64 * 3


def rope_frequencies(rotary_dim: int, base: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0,
                     trained_len: float = 0.0, low: float = 1.0, high: float = 32.0, device=None) -> torch.Tensor:
    """dreams_rope_frequencies: radians a position of every pair, [rotary_dim / 2] float64 on `device` (None: the current
    one).  scaling: None, "linear" (all slowed by `factor`) or "parts" (those that make fewer than `low` turns within
    trained_len positions slowed by it, those that make more than `high` kept, in between in part)."""
    if scaling not in ROPE_SCALINGS:
        raise ValueError("scaling must be one of None, 'linear', 'parts'")
    if not 1 < rotary_dim < 2 ** 31:
        raise ValueError("rotary_dim must be even and >= 2")
    f = torch.empty(rotary_dim // 2, dtype=torch.float64)
    _check(lib().dreams_rope_frequencies(rotary_dim, base, ROPE_SCALINGS[scaling], factor, trained_len, low, high,
                                         f.data_ptr()))
    return f.to(torch.device("cuda") if device is None else device)


def _rope(frequencies, positions, parent, shape, at, interleaved, amplitude) -> Rope:
    """The rotation of rows [B, N], checked."""
    _need_on(frequencies, "frequencies", torch.float64, at, None, 1)
    if positions is not None:
        _need_on(positions, "positions", torch.int32, at, shape)
    if parent is not None:
        _need_on(parent, "parent", torch.int32, at, shape)
    return Rope(2 * frequencies.shape[0], 1 if interleaved else 0, frequencies.data_ptr(), _ptr(positions), _ptr(parent),
                amplitude)


def rope(x: torch.Tensor, frequencies: torch.Tensor, kv_len: Optional[torch.Tensor] = None,
         positions: Optional[torch.Tensor] = None, parent: Optional[torch.Tensor] = None, interleaved: bool = False,
         amplitude: float = 1.0, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """dreams_rope.  x [B,H,N,D] bf16 or fp32 of any strides with dense rows (a transposed view of a projection's [B,N,H,D]
    serves); frequencies [R/2] float64 (rope_frequencies, or any others) for its first R columns; the rows' positions are
    positions [B,N] int32, or kv_len[b] ([B] int32) plus the depth by parent [B,N] int32, or plus 0, 1, ...  out: like x
    (None: a dense [B,H,N,D]; x itself: in place).  Returns out."""
    at = _current(x, "x")
    code = _code(x.dtype, "x")
    shape, st = x.shape, x.stride()
    if len(shape) != 4:
        raise ValueError("x must have 4 dimensions")
    B, H, N, D = shape
    if D > 1 and st[3] != 1:
        raise ValueError("the rows of x must be dense")
    r = _rope(frequencies, positions, parent, (B, N), at, interleaved, amplitude)
    if kv_len is not None:
        _need_on(kv_len, "kv_len", torch.int32, at, (B,))
    if out is None:
        out = _dense_like(x, stream)
        to = _Strides3(H * N * D, N * D, D)
    else:
        if not isinstance(out, torch.Tensor):
            raise TypeError("out must be a torch.Tensor")
        if out.dtype is not x.dtype or out.get_device() != at or out.shape != shape or (D > 1 and out.stride(3) != 1):
            raise ValueError("out must be like x, with dense rows")
        to = _Strides3(*out.stride()[:3])
    status = lib().dreams_rope(ctypes.byref(r), B, H, N, D, code, x.data_ptr(), _Strides3(st[0], st[1], st[2]), _ptr(kv_len),
                               out.data_ptr(), to, _stream_on(stream, at))
    if status:
        _check(status)
    return out


def _queries(q, q_out, like, batch, rows, head_dim, at, stream):
    """(RopeQueries or None, its output)"""
    if q is None:
        if q_out is not None:
            raise ValueError("q_out needs q")
        return None, None
    if not isinstance(q, torch.Tensor):
        raise TypeError("q must be a torch.Tensor")
    if q.dtype is not like.dtype:
        raise TypeError("q must be %s, got %s" % (like.dtype, q.dtype))
    if q.get_device() != at:
        raise ValueError("q is on %s, expected %s" % (q.device, like.device))
    shape, st = q.shape, q.stride()
    if len(shape) != 4 or shape[0] != batch or shape[2] != rows or shape[3] != head_dim:
        raise ValueError("q must be [B,Hq,N,D] for the new rows")
    if head_dim > 1 and st[3] != 1:
        raise ValueError("the rows of q must be dense")
    if q_out is None:
        q_out = _dense_like(q, stream)
    else:
        _need_on(q_out, "q_out", q.dtype, at, shape)
    return RopeQueries(q.data_ptr(), q_out.data_ptr(), shape[1], _Strides3(st[0], st[1], st[2])), q_out


def paged_append_rope(k_new: torch.Tensor, v_new: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor,
                      page_table: torch.Tensor, kv_len: torch.Tensor, frequencies: torch.Tensor,
                      row_len: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None,
                      positions: Optional[torch.Tensor] = None, parent: Optional[torch.Tensor] = None,
                      interleaved: bool = False, amplitude: float = 1.0, q_out: Optional[torch.Tensor] = None,
                      stream=None) -> Optional[torch.Tensor]:
    """dreams_paged_append_rope: paged_append with the keys rotated (as in rope, from kv_len on) on their way, and, in the
    same launch, the rows' queries q [B,Hq,N,D] (any strides with dense rows; one layer's rows only).  Returns the rotated
    queries, dense [B,Hq,N,D] (0 in rows from row_len on), or None."""
    pool, at = _pool(k_pages, v_pages, page_table)
    strides = _new_rows(k_new, v_new, k_pages, pool, at, k_pages.dtype, kv_len, row_len)
    B, N = pool.batch, k_new.shape[-2]
    r = _rope(frequencies, positions, parent, (B, N), at, interleaved, amplitude)
    queries, q_out = _queries(q, q_out, k_new, B, N, pool.head_dim, at, stream)
    _check(lib().dreams_paged_append_rope(ctypes.byref(pool), ctypes.byref(r),
                                          None if queries is None else ctypes.byref(queries), k_new.data_ptr(),
                                          v_new.data_ptr(), N, strides, page_table.data_ptr(), kv_len.data_ptr(),
                                          _ptr(row_len), k_pages.data_ptr(), v_pages.data_ptr(), _stream_on(stream, at)))
    return q_out


# --------------------------------------------------------------------------------------------- pages of 8 bits
_E4M3, _E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _scale_strides(k_scales, v_scales, shape, at):
    """(layer stride, page stride) of the scales [NL, P, Hkv, page_size / 16] of pages of this shape."""
    P, H, S = shape[-4], shape[-3], shape[-2] // 16
    want = (P, H, S) if len(shape) == 4 else (shape[0], P, H, S)
    try:
        if (k_scales.dtype is _E8M0 and v_scales.dtype is _E8M0 and k_scales.get_device() == at == v_scales.get_device()
                and k_scales.shape == want == v_scales.shape and k_scales.is_contiguous() and v_scales.is_contiguous()):
            return P * H * S if len(want) == 4 and want[0] > 1 else 0, H * S
    except AttributeError:
        pass
    for t, name in ((k_scales, "k_scales"), (v_scales, "v_scales")):
        if not isinstance(t, torch.Tensor):
            raise TypeError("%s must be a torch.Tensor" % name)
        if t.dtype is not _E8M0:
            raise TypeError("%s must be torch.float8_e8m0fnu, got %s" % (name, t.dtype))
        if t.get_device() != at:
            raise ValueError("%s is on %s, not with the pages" % (name, t.device))
        if t.shape != want:
            raise ValueError("%s must be %s, got %s" % (name, list(want), list(t.shape)))
    n, st, vst = len(want), k_scales.stride(), v_scales.stride()
    if any(want[i] > 1 and st[i] != vst[i] for i in range(n)):
        raise ValueError("k_scales and v_scales differ in layout")
    if (S > 1 and st[-1] != 1) or (H > 1 and st[-2] != S):
        raise ValueError("a page's scales must be dense [Hkv, page_size / 16]")
    if (P > 1 and st[-3] == 0) or (n == 4 and want[0] > 1 and st[0] == 0):
        raise ValueError("scales of pages or layers share memory (expanded views)")
    return st[0] if n == 4 and want[0] > 1 else 0, st[-3] if P > 1 else H * S


def _dense8(k_pages, v_pages, k_scales, v_scales, page_table, shape, at) -> bool:
    """Whether a pool of 8 bits is all dense tensors on the current device, as most are: nothing else is to be looked at."""
    try:
        scales = shape[:-2] + (shape[-2] // 16,)
        return (k_pages.dtype is _E4M3 is v_pages.dtype and k_scales.dtype is _E8M0 is v_scales.dtype
                and page_table.dtype is torch.int32 and len(page_table.shape) == 2 and shape == v_pages.shape
                and scales == k_scales.shape == v_scales.shape and at >= 0
                and at == v_pages.get_device() == k_scales.get_device() == v_scales.get_device()
                == page_table.get_device() == _current_device()
                and k_pages.is_contiguous() and v_pages.is_contiguous() and k_scales.is_contiguous()
                and v_scales.is_contiguous() and page_table.is_contiguous())
    except AttributeError:
        return False


def _pool8(k_pages, v_pages, k_scales, v_scales, page_table):
    """(PagePool, PageScales, device index) of pages of 8 bits"""
    if isinstance(k_pages, torch.Tensor):
        if k_pages.dtype is not _E4M3:
            raise TypeError("k_pages must be torch.float8_e4m3fn, got %s" % k_pages.dtype)
        shape, at = k_pages.shape, k_pages.get_device()
        if len(shape) in (4, 5) and _dense8(k_pages, v_pages, k_scales, v_scales, page_table, shape, at):
            P, H, S, D = shape[-4:]
            B, width = page_table.shape
            return (PagePool(shape[0] if len(shape) == 5 else 1, B, H, D, P, S, width, DREAMS_E4M3, 0, 0),
                    PageScales(k_scales.data_ptr(), v_scales.data_ptr(), 0, 0), at)
    pool, at = _pool(k_pages, v_pages, page_table, DREAMS_E4M3)
    layer, page = _scale_strides(k_scales, v_scales, k_pages.shape, at)
    return pool, PageScales(k_scales.data_ptr(), v_scales.data_ptr(), layer, page), at


def paged_append_e4m3(k_new: torch.Tensor, v_new: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor,
                      k_scales: torch.Tensor, v_scales: torch.Tensor, page_table: torch.Tensor, kv_len: torch.Tensor,
                      row_len: Optional[torch.Tensor] = None, frequencies: Optional[torch.Tensor] = None,
                      q: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
                      parent: Optional[torch.Tensor] = None, interleaved: bool = False, amplitude: float = 1.0,
                      q_out: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """dreams_paged_append_e4m3, in place on k_pages / v_pages [NL,num_pages,Hkv,page_size,D] float8_e4m3fn and k_scales /
    v_scales [NL,num_pages,Hkv,page_size/16] float8_e8m0fnu (or one layer's): new rows, bf16 or fp32, as in paged_append;
    with frequencies, keys and queries are rotated as in paged_append_rope.  A block of 16 slots takes the least power of
    two that holds its rows.  Returns the rotated queries or None."""
    pool, scales, at = _pool8(k_pages, v_pages, k_scales, v_scales, page_table)
    code = _code(k_new.dtype if isinstance(k_new, torch.Tensor) else None, "new rows")
    strides = _new_rows(k_new, v_new, k_pages, pool, at, k_new.dtype, kv_len, row_len)
    B, N = pool.batch, k_new.shape[-2]
    if frequencies is None:
        if q is not None or positions is not None or parent is not None:
            raise ValueError("q, positions and parent need frequencies")
        r = None
    else:
        r = _rope(frequencies, positions, parent, (B, N), at, interleaved, amplitude)
    queries, q_out = _queries(q, q_out, k_new, B, N, pool.head_dim, at, stream)
    _check(lib().dreams_paged_append_e4m3(ctypes.byref(pool), ctypes.byref(scales), None if r is None else ctypes.byref(r),
                                          None if queries is None else ctypes.byref(queries), code, k_new.data_ptr(),
                                          v_new.data_ptr(), N, strides, page_table.data_ptr(), kv_len.data_ptr(),
                                          _ptr(row_len), k_pages.data_ptr(), v_pages.data_ptr(), _stream_on(stream, at)))
    return q_out


def paged_kv_commit_e4m3(k_pages: torch.Tensor, v_pages: torch.Tensor, k_scales: torch.Tensor, v_scales: torch.Tensor,
                         page_table: torch.Tensor, kv_len_in: torch.Tensor, accept_path: torch.Tensor,
                         accept_len: torch.Tensor, kv_len_out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """dreams_paged_kv_commit_e4m3, in place on pages and scales (as paged_append_e4m3).  Returns kv_len_out [B] int32."""
    pool, scales, at = _pool8(k_pages, v_pages, k_scales, v_scales, page_table)
    kv_len_out = _commit_lengths(pool.batch, at, kv_len_in, accept_path, accept_len, kv_len_out, stream)
    _check(lib().dreams_paged_kv_commit_e4m3(ctypes.byref(pool), ctypes.byref(scales), k_pages.data_ptr(),
                                             v_pages.data_ptr(), page_table.data_ptr(), kv_len_in.data_ptr(),
                                             accept_path.data_ptr(), accept_len.data_ptr(), accept_path.shape[1],
                                             kv_len_out.data_ptr(), _stream_on(stream, at)))
    return kv_len_out


def paged_read_e4m3(k_pages: torch.Tensor, v_pages: torch.Tensor, k_scales: torch.Tensor, v_scales: torch.Tensor,
                    page_table: torch.Tensor, kv_len: torch.Tensor, num_slots: int, k_out: Optional[torch.Tensor] = None,
                    v_out: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """dreams_paged_read_e4m3: the first num_slots slots of every sequence as values, (k_out, v_out) bfloat16
    [NL,B,Hkv,num_slots,D] (without NL for one layer's pages), 0 from kv_len[b] on."""
    pool, scales, at = _pool8(k_pages, v_pages, k_scales, v_scales, page_table)
    _need_on(kv_len, "kv_len", torch.int32, at, (pool.batch,))
    if not -1 < num_slots < 2 ** 31:
        raise ValueError("num_slots must be in [0, 2^31)")
    shape = k_pages.shape[:-4] + (pool.batch, pool.num_kv_heads, num_slots, pool.head_dim)
    if k_out is None:
        k_out = kv_len.new_empty(*shape, dtype=torch.bfloat16) if stream is None else _new(kv_len, stream, shape, torch.bfloat16)
    else:
        _need_on(k_out, "k_out", torch.bfloat16, at, shape)
    if v_out is None:
        v_out = _dense_like(k_out, stream)
    else:
        _need_on(v_out, "v_out", torch.bfloat16, at, shape)
    _check(lib().dreams_paged_read_e4m3(ctypes.byref(pool), ctypes.byref(scales), k_pages.data_ptr(), v_pages.data_ptr(),
                                        page_table.data_ptr(), kv_len.data_ptr(), num_slots, k_out.data_ptr(),
                                        v_out.data_ptr(), _stream_on(stream, at)))
    return k_out, v_out


def pages_fork_e4m3(k_pages: torch.Tensor, v_pages: torch.Tensor, k_scales: torch.Tensor, v_scales: torch.Tensor,
                    page_table: torch.Tensor, page_count: torch.Tensor, kv_len: torch.Tensor, refcount: torch.Tensor,
                    src: torch.Tensor, dst: torch.Tensor, granted: Optional[torch.Tensor] = None,
                    stream=None) -> torch.Tensor:
    """dreams_pages_fork_e4m3: pages_fork over pages of 8 bits, whose scales go with the copied rows."""
    pool, scales, at = _pool8(k_pages, v_pages, k_scales, v_scales, page_table)
    call, L = (ctypes.byref(pool), ctypes.byref(scales)), lib()
    return _fork(L.dreams_pages_fork_e4m3, call, pool, at, k_pages, v_pages, page_table, page_count, kv_len, refcount, src,
                 dst, granted, stream)


def _paged_desc8(q, k_pages, v_pages, k_scales, v_scales, page_table, window, sinks, max_kv_len, num_splits, scale):
    """(PagedDesc, PageScales) of an attention call over pages of 8 bits"""
    if isinstance(k_pages, torch.Tensor):
        if k_pages.dtype is not _E4M3:
            raise TypeError("k_pages must be torch.float8_e4m3fn, got %s" % k_pages.dtype)
        shape, at = k_pages.shape, k_pages.get_device()
        if (len(shape) == 4 and _dense8(k_pages, v_pages, k_scales, v_scales, page_table, shape, at)
                and isinstance(q, torch.Tensor) and q.dtype is torch.bfloat16 and q.get_device() == at and q.is_contiguous()
                and -1 < window < 2 ** 31 and -1 < sinks < 2 ** 31 and -1 < max_kv_len < 2 ** 31 and -1 < num_splits < 2 ** 31):
            rows, table = q.shape, page_table.shape
            if len(rows) == 4 and rows[0] == table[0] and rows[3] == shape[3]:
                return (PagedDesc(rows[0], rows[1], shape[1], rows[3], rows[2], shape[0], shape[2], table[1], max_kv_len,
                                  num_splits, window, sinks, DREAMS_BF16, 1.0 / math.sqrt(rows[3]) if scale is None else scale,
                                  0), PageScales(k_scales.data_ptr(), v_scales.data_ptr(), 0, 0))
    desc = _paged_desc(q, k_pages, v_pages, page_table, torch.bfloat16, window, sinks, max_kv_len, num_splits, scale)
    _, page = _scale_strides(k_scales, v_scales, k_pages.shape, q.get_device())
    return desc, PageScales(k_scales.data_ptr(), v_scales.data_ptr(), 0, page)


def paged_verify_attn_e4m3(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, k_scales: torch.Tensor,
                           v_scales: torch.Tensor, page_table: torch.Tensor, kv_len: torch.Tensor,
                           parent: Optional[torch.Tensor] = None, tree_mask: Optional[torch.Tensor] = None, window: int = 0,
                           sinks: int = 0, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                           lse: Optional[torch.Tensor] = None, with_lse: bool = True, max_kv_len: int = 0,
                           num_splits: int = 0, workspace: Optional[torch.Tensor] = None,
                           stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """dreams_paged_verify_attn_e4m3: paged_verify_attn with bf16 queries over one layer's pages of 8 bits: k_pages / v_pages
    [num_pages,Hkv,page_size,D] float8_e4m3fn, k_scales / v_scales [num_pages,Hkv,page_size/16] float8_e8m0fnu, as
    paged_append_e4m3 writes them.  Returns (out, lse or None)."""
    desc, scales = _paged_desc8(q, k_pages, v_pages, k_scales, v_scales, page_table, window, sinks, max_kv_len, num_splits,
                                scale)
    B, T, at = desc.batch, desc.num_rows, q.get_device()
    _need_on(kv_len, "kv_len", torch.int32, at, (B,))
    if parent is not None:
        _need_on(parent, "parent", torch.int32, at, (B, T))
    if tree_mask is not None:
        _need_on(tree_mask, "tree_mask", torch.int64, at, (B, T, (T + 63) // 64))
    out, lse = _paged_outputs(q, out, lse, with_lse, stream)
    L = lib()
    _call_paged(L.dreams_paged_verify_attn_e4m3, L.dreams_paged_verify_attn_e4m3_workspace_size, ctypes.byref(desc),
                (q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), ctypes.byref(scales), page_table.data_ptr(),
                 kv_len.data_ptr(), _ptr(parent), _ptr(tree_mask), out.data_ptr(), _ptr(lse)), workspace, at, stream)
    return out, lse


def paged_prompt_attn_e4m3(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, k_scales: torch.Tensor,
                           v_scales: torch.Tensor, page_table: torch.Tensor, kv_len: torch.Tensor,
                           row_len: Optional[torch.Tensor] = None, window: int = 0, sinks: int = 0,
                           scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                           lse: Optional[torch.Tensor] = None, with_lse: bool = True, max_kv_len: int = 0,
                           num_splits: int = 0, workspace: Optional[torch.Tensor] = None,
                           stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """dreams_paged_prompt_attn_e4m3: paged_prompt_attn with bf16 queries over one layer's pages of 8 bits (as in
    paged_verify_attn_e4m3).  Returns (out, lse or None)."""
    desc, scales = _paged_desc8(q, k_pages, v_pages, k_scales, v_scales, page_table, window, sinks, max_kv_len, num_splits,
                                scale)
    B, at = desc.batch, q.get_device()
    _need_on(kv_len, "kv_len", torch.int32, at, (B,))
    if row_len is not None:
        _need_on(row_len, "row_len", torch.int32, at, (B,))
    out, lse = _paged_outputs(q, out, lse, with_lse, stream)
    L = lib()
    _call_paged(L.dreams_paged_prompt_attn_e4m3, L.dreams_paged_prompt_attn_e4m3_workspace_size, ctypes.byref(desc),
                (q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), ctypes.byref(scales), page_table.data_ptr(),
                 kv_len.data_ptr(), _ptr(row_len), out.data_ptr(), _ptr(lse)), workspace, at, stream)
    return out, lse
