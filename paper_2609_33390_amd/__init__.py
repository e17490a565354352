"""BRISK-DLM decoding hot path on MI355X (gfx950).

Thin Python binding of ``libbrisk.so``: it checks tensor metadata, allocates
outputs and workspaces with torch, and passes raw device pointers and the
current HIP stream to the C ABI declared in ``include/brisk.h``.  Every step of
the computation runs in the library's HIP kernels; there is no CPU fallback,
and a missing or unloadable library raises.

Entry points (same names as the C ABI):

* :func:`propose_block` - LM-head logits and ordered top-K candidates;
* :func:`rerank` - the prefix-conditioned corrector over the candidates;
* :func:`verify_accept` - greedy verification: accept length and correction;
* :func:`rerank_verify` - :func:`rerank` and :func:`verify_accept` in one call;
* :func:`propose_verify` - one LM-head pass for proposal rows (top-K) and
  verifier rows (argmax);
* :func:`verify_commit` - greedy verification and the committed tokens;
* :func:`corrector_loss` - the corrector's training loss on reached positions;
* :func:`spec_verify` - stochastic speculative verification with residual draws;
* :func:`accept_profile` - acceptance profile, tokens per forward and the
  risk-reward position weights from many blocks' accept lengths.

Every call is queued on ``stream`` (a torch stream or a handle), by default the
current one, and takes an optional ``workspace``.  Without one it uses scratch
of its own for that stream, or of the graph when the stream is being captured;
a workspace that the caller passes must not serve two calls at once.  Tensors
that are made or freed on another stream than the call's are the caller's to
order, as with every torch operation.

Around the step, on a :class:`KVCache` of paged keys and values:

* :func:`block_attention` - attention of every block (or single token) over a
  prefix shared by the batch and its own cache;
* :func:`cache_score` - the attention weight that every cached key received;
* :func:`cache_evict` - eviction by that weight, in place;
* :func:`draft_verify` - verification of drafted tokens against given
  probabilities, with the random numbers given.

On a :class:`KVCache4`, whose keys and values are held in 4 bits:

* :func:`kv4_write` - new tokens' keys and values into it;
* :func:`kv4_read` - what it holds, as 2-byte keys and values;
* :func:`kv4_attention` - :func:`block_attention` over it.
"""
from __future__ import annotations

import ctypes
import functools
import os
import threading
from typing import Dict, Optional, Tuple

import torch

__all__ = ["BriskError", "Corrector", "propose_block", "propose_block_noalloc", "propose_lmhead", "propose_merge", "rerank", "rerank_verify", "rerank_hoist", "rerank_finish", "verify_accept", "accept_profile",
           "propose_verify", "verify_commit", "corrector_loss", "spec_verify",
           "KVCache", "block_attention", "cache_score", "cache_evict", "draft_verify",
           "KVCache4", "kv4_page_bytes", "kv4_write", "kv4_read", "kv4_attention",
           "lib", "LIB_PATH", "ABI_SYMBOLS", "propose_workspace_size", "rerank_workspace_size"]

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libbrisk.so")
ABI_SYMBOLS = ("brisk_status_str", "brisk_abi_version", "brisk_propose_workspace_size",
               "brisk_propose_block", "brisk_propose_block_noalloc", "brisk_propose_lmhead",
               "brisk_propose_merge",
               "brisk_rerank_workspace_size", "brisk_rerank", "brisk_rerank_verify",
               "brisk_rerank_hoist", "brisk_rerank_finish",
               "brisk_verify_accept", "brisk_propose_verify_workspace_size", "brisk_propose_verify",
               "brisk_verify_commit", "brisk_spec_verify_workspace_size", "brisk_spec_verify",
               "brisk_corrector_loss", "brisk_accept_profile_workspace_size",
               "brisk_accept_profile", "brisk_corrector_tables_size", "brisk_corrector_prepare",
               "brisk_block_attention_workspace_size", "brisk_block_attention", "brisk_cache_score",
               "brisk_cache_evict_workspace_size", "brisk_cache_evict",
               "brisk_draft_verify_workspace_size", "brisk_draft_verify",
               "brisk_kv4_page_bytes", "brisk_kv4_write", "brisk_kv4_read",
               "brisk_kv4_attention_workspace_size", "brisk_kv4_attention")
PSI_FIELDS = ("A_h", "A_e", "P_h", "P_e", "pos_emb", "P_phi", "W_z", "W_h", "W_s", "W_c", "w_g")

_p = ctypes.c_void_p
_i32 = ctypes.c_int32
_sz = ctypes.c_size_t


class BriskError(RuntimeError):
    """A non-zero status returned by the library."""

    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: status {status} ({_status_str(status)})")


class _CorrectorC(ctypes.Structure):
    _fields_ = ([(n, _i32) for n in ("d_state", "d_hproj", "d_tproj", "d_pos", "d_feat", "rank", "max_L")]
                + [(n, _p) for n in PSI_FIELDS]
                + [("alpha", ctypes.c_float), ("b_g", ctypes.c_float), ("tables", _p), ("tables_V", _i32)])


class _KVCacheC(ctypes.Structure):
    _fields_ = ([(n, _i32) for n in ("dtype", "n_kv_heads", "d_head", "page_size", "n_pages", "max_pages")]
                + [(n, ctypes.c_int64) for n in ("page_stride", "slot_stride", "head_stride")]
                + [(n, _p) for n in ("k_pages", "v_pages", "block_table", "seq_len")])


class _KVCache4C(ctypes.Structure):
    _fields_ = ([(n, _i32) for n in ("dtype", "n_kv_heads", "d_head", "page_size", "n_pages", "max_pages")]
                + [(n, ctypes.c_int64) for n in ("page_stride", "head_stride")]
                + [(n, _p) for n in ("pages", "block_table", "seq_len")])


class _KVPrefixC(ctypes.Structure):
    _fields_ = [("len", _i32), ("slot_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("k", _p), ("v", _p)]


_lib = None
_lib_lock = threading.Lock()


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it has not been built."""
    global _lib, _several_devices
    if _lib is not None:
        return _lib
    with _lib_lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                                   "`python -m paper_2609_33390_amd.build`")
            L = ctypes.CDLL(LIB_PATH)
            L.brisk_status_str.restype = ctypes.c_char_p
            L.brisk_status_str.argtypes = [ctypes.c_int]
            L.brisk_abi_version.restype = ctypes.c_int
            L.brisk_abi_version.argtypes = []
            L.brisk_propose_workspace_size.restype = ctypes.c_int
            L.brisk_propose_workspace_size.argtypes = [_i32, _i32, _i32, _i32, ctypes.POINTER(_sz)]
            L.brisk_propose_block.restype = ctypes.c_int
            L.brisk_propose_block.argtypes = [_p, _p, _i32, _i32, _i32, _i32, _p, _p, _p, _sz, _p]
            L.brisk_propose_block_noalloc.restype = ctypes.c_int
            L.brisk_propose_block_noalloc.argtypes = [_p, _p, _i32, _i32, _i32, _i32, _p, _p, _p]
            L.brisk_propose_lmhead.restype = ctypes.c_int
            L.brisk_propose_lmhead.argtypes = [_p, _p, _i32, _i32, _i32, _i32, _p, _sz, _p]
            L.brisk_propose_merge.restype = ctypes.c_int
            L.brisk_propose_merge.argtypes = [_i32, _i32, _i32, _p, _p, _p, _sz, _p]
            L.brisk_rerank_workspace_size.restype = ctypes.c_int
            L.brisk_rerank_workspace_size.argtypes = [ctypes.POINTER(_CorrectorC), _i32, _i32, _i32,
                                                      ctypes.POINTER(_sz)]
            L.brisk_rerank.restype = ctypes.c_int
            L.brisk_rerank.argtypes = [ctypes.POINTER(_CorrectorC), _p, _p, _p, _p, _p, _p, _p,
                                       _i32, _i32, _i32, _i32, _i32, _p, _p, _p, _p, _p, _sz, _p]
            L.brisk_rerank_verify.restype = ctypes.c_int
            L.brisk_rerank_verify.argtypes = [ctypes.POINTER(_CorrectorC), _p, _p, _p, _p, _p, _p, _p, _p,
                                              _i32, _i32, _i32, _i32, _i32, _p, _p, _p, _p, _p, _p,
                                              _p, _sz, _p]
            L.brisk_rerank_hoist.restype = ctypes.c_int
            L.brisk_rerank_hoist.argtypes = [ctypes.POINTER(_CorrectorC), _p, _p, _p, _p,
                                             _i32, _i32, _i32, _i32, _i32, _p, _sz, _p]
            L.brisk_rerank_finish.restype = ctypes.c_int
            L.brisk_rerank_finish.argtypes = L.brisk_rerank_verify.argtypes
            L.brisk_verify_accept.restype = ctypes.c_int
            L.brisk_verify_accept.argtypes = [_p, _p, _i32, _i32, _p, _p, _p]
            L.brisk_propose_verify_workspace_size.restype = ctypes.c_int
            L.brisk_propose_verify_workspace_size.argtypes = [_i32, _i32, _i32, _i32, _i32,
                                                              ctypes.POINTER(_sz)]
            L.brisk_propose_verify.restype = ctypes.c_int
            L.brisk_propose_verify.argtypes = [_p, _p, _i32, _i32, _i32, _i32, _i32, _p, _p, _p, _p,
                                               _sz, _p]
            L.brisk_verify_commit.restype = ctypes.c_int
            L.brisk_verify_commit.argtypes = [_p, _p, _i32, _i32, _p, _p, _p, _p]
            L.brisk_spec_verify_workspace_size.restype = ctypes.c_int
            L.brisk_spec_verify_workspace_size.argtypes = [_i32, _i32, _i32, _i32, ctypes.POINTER(_sz)]
            L.brisk_spec_verify.restype = ctypes.c_int
            L.brisk_spec_verify.argtypes = [_p, _p, _p, _p, _p, _p, ctypes.c_uint64, ctypes.c_float,
                                            _i32, _i32, _i32, _i32, _i32, _p, _p, _p, _p, _p, _sz, _p]
            L.brisk_corrector_loss.restype = ctypes.c_int
            L.brisk_corrector_loss.argtypes = [_p, _p, _p, _p, _p, _p, _i32, _i32, _i32, _i32, _i32,
                                               ctypes.c_float, _p, _p, _p, _p, _p]
            L.brisk_accept_profile_workspace_size.restype = ctypes.c_int
            L.brisk_accept_profile_workspace_size.argtypes = [_i32, _i32, ctypes.POINTER(_sz)]
            L.brisk_accept_profile.restype = ctypes.c_int
            L.brisk_accept_profile.argtypes = [_p, _i32, _i32, ctypes.c_double, _p, _p, _p, _p, _p,
                                               _sz, _p]
            L.brisk_corrector_tables_size.restype = ctypes.c_int
            L.brisk_corrector_tables_size.argtypes = [ctypes.POINTER(_CorrectorC), _i32, ctypes.POINTER(_sz),
                                                      ctypes.POINTER(_sz)]
            L.brisk_corrector_prepare.restype = ctypes.c_int
            L.brisk_corrector_prepare.argtypes = [ctypes.POINTER(_CorrectorC), _p, _p, _i32, _i32, _p, _sz, _p,
                                                  _sz, _p]
            _i64, _f32, _szp = ctypes.c_int64, ctypes.c_float, ctypes.POINTER(_sz)
            _cache = ctypes.POINTER(_KVCacheC)
            L.brisk_block_attention_workspace_size.restype = ctypes.c_int
            L.brisk_block_attention_workspace_size.argtypes = [_i32] * 7 + [_szp]
            L.brisk_block_attention.restype = ctypes.c_int
            L.brisk_block_attention.argtypes = [_cache, ctypes.POINTER(_KVPrefixC), _p, _i64, _i64, _p, _i32, _i32,
                                                _i32, _i32, _f32, _p, _p, _p, _sz, _p]
            L.brisk_cache_score.restype = ctypes.c_int
            L.brisk_cache_score.argtypes = [_cache, _p, _i64, _i64, _p, _p, _i32, _i32, _i32, _f32, _f32, _p, _p,
                                            _i32, _p]
            L.brisk_cache_evict_workspace_size.restype = ctypes.c_int
            L.brisk_cache_evict_workspace_size.argtypes = [_i32] * 4 + [_szp]
            L.brisk_cache_evict.restype = ctypes.c_int
            L.brisk_cache_evict.argtypes = [_cache, _i32, _p, _p, _i32, _p, _i32, _i32, _p, _p, _p, _p, _sz, _p]
            L.brisk_draft_verify_workspace_size.restype = ctypes.c_int
            L.brisk_draft_verify_workspace_size.argtypes = [_i32, _i32, _szp]
            L.brisk_draft_verify.restype = ctypes.c_int
            L.brisk_draft_verify.argtypes = [_p, _i64, _p, _i64, _p, _p, _p, _p, _i64, _i32, _i32, _i32, _p, _p, _p,
                                             _sz, _p]
            _cache4 = ctypes.POINTER(_KVCache4C)
            L.brisk_kv4_page_bytes.restype = ctypes.c_int
            L.brisk_kv4_page_bytes.argtypes = [_i32, _i32, _szp]
            L.brisk_kv4_write.restype = ctypes.c_int
            L.brisk_kv4_write.argtypes = [_cache4, _p, _p, _i64, _i64, _i64, _i32, _i32, _p, _p, _p]
            L.brisk_kv4_read.restype = ctypes.c_int
            L.brisk_kv4_read.argtypes = [_cache4, _i32, _i32, _p, _p, _p, _p]
            L.brisk_kv4_attention_workspace_size.restype = ctypes.c_int
            L.brisk_kv4_attention_workspace_size.argtypes = [_i32] * 7 + [_szp]
            L.brisk_kv4_attention.restype = ctypes.c_int
            L.brisk_kv4_attention.argtypes = [_cache4] + L.brisk_block_attention.argtypes[1:]
            _several_devices = torch.cuda.device_count() > 1
            _lib = L
        return _lib


def _status_str(status: int) -> str:
    try:
        return lib().brisk_status_str(status).decode()
    except Exception:  # pragma: no cover - message only
        return "?"


def _check(status: int, where: str) -> None:
    if status != 0:
        raise BriskError(status, where)


def _dev_tensor(t: torch.Tensor, name: str, dtype: torch.dtype, ndim: Optional[int] = None, *,
                shape: Optional[Tuple[int, ...]] = None, device: Optional[torch.device] = None) -> None:
    """Checks a tensor before its pointer goes to the library: type, dtype,
    dimension count or exact shape, contiguity, a HIP device, and (when
    ``device`` is given) the same device as the call's other tensors.  A
    wrong shape would otherwise let a kernel read or write past the buffer."""
    if (type(t) is torch.Tensor and t.dtype is dtype and t.is_cuda and t.is_contiguous()
            and (t.shape == shape if shape is not None else ndim is None or t.dim() == ndim)
            and (device is None or t.device == device)):
        return                                     # nothing to object to: most calls end here
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None:
        if tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    elif ndim is not None and t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dims, got shape {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must live on a HIP device, got {t.device}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, the call's other tensors on {device}")


def _ws_bytes(ws: torch.Tensor, device: torch.device, need: int, name: str = "workspace") -> int:
    """Size in bytes of a caller's workspace, after checking that it is a
    contiguous tensor on the call's device and holds at least ``need`` bytes."""
    if not isinstance(ws, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not ws.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if not ws.is_cuda:
        raise ValueError(f"{name} must live on a HIP device, got {ws.device}")
    if ws.device != device:
        raise ValueError(f"{name} is on {ws.device}, the call's other tensors on {device}")
    nbytes = ws.nbytes
    if nbytes < need:
        raise ValueError(f"{name} holds {nbytes} bytes, the call needs {need}")
    return nbytes


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


# The current stream's handle without a Stream object around it, where torch offers that.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
# The current device's number, the same way, and whether there is another one (known once the library is loaded).
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_several_devices = False


def _stream_ptr(device: torch.device, stream) -> Optional[int]:
    """The handle of the stream that a call queues on.  Every device's default stream has the handle 0, which
    means the current device's: with tensors of another device that is refused."""
    if stream is None and _raw_stream is not None and device.index is not None:
        handle = _raw_stream(device.index)
    else:
        stream = torch.cuda.current_stream(device) if stream is None else stream
        handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    if _several_devices and not handle and device.type == "cuda" and device.index not in (None, _current_device()):
        raise ValueError(f"the tensors are on {device}, the default stream is that of cuda:{_current_device()}: call "
                         f"under torch.cuda.device({device.index}), or on another stream of {device}")
    return handle


_ws: Dict[Tuple[Optional[int], str, Optional[int]], torch.Tensor] = {}
# Whether the current stream is being captured, without the Python around it.
_capturing = getattr(torch._C, "_cuda_isCurrentStreamCapturing", torch.cuda.is_current_stream_capturing)


def _workspace(device: torch.device, nbytes: int, tag: str, stream) -> torch.Tensor:
    """Scratch of a call on ``stream`` (as the entry points take it): a buffer of
    the device, entry point and stream, grown on demand, so that calls on
    different streams share none.  It is allocated on the stream that uses it,
    so a smaller one is given back in that stream's order.  A call under
    capture gets memory of the graph instead: replays must not share a buffer
    with other calls, and it must live as long as the graph."""
    if stream is not None and _stream_ptr(device, stream) != _stream_ptr(device, None):
        if not hasattr(stream, "cuda_stream"):     # a handle; 0 is the default stream
            stream = torch.cuda.ExternalStream(int(stream), device) if int(stream) else torch.cuda.default_stream(device)
        with torch.cuda.stream(stream):
            return _workspace(device, nbytes, tag, None)
    if _capturing():
        return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
    key = (device.index, tag, _stream_ptr(device, None))  # a tensor's device has its index
    buf = _ws.get(key)
    if buf is None or buf.numel() < nbytes:
        buf = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
        _ws[key] = buf
    return buf


# ----------------------------------------------------------------- propose
def _lmhead_operands(hidden: torch.Tensor, lm_head: torch.Tensor):
    """(rows, d, V, device) of a hidden-state block and an LM head, checked."""
    _dev_tensor(hidden, "hidden", torch.bfloat16, 2)
    dev = hidden.device
    _dev_tensor(lm_head, "lm_head", torch.bfloat16, 2, device=dev)
    rows, d = hidden.shape
    if lm_head.shape[1] != d:
        raise ValueError("hidden and lm_head disagree on d")
    return rows, d, lm_head.shape[0], dev


def propose_workspace_size(rows: int, d: int, V: int, K: int) -> int:
    out = _sz()
    _check(lib().brisk_propose_workspace_size(rows, d, V, K, ctypes.byref(out)),
           "brisk_propose_workspace_size")
    return out.value


def propose_block(hidden: torch.Tensor, lm_head: torch.Tensor, K: int, *,
                  cand_logit: Optional[torch.Tensor] = None, cand_id: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None, stream=None
                  ) -> Tuple[torch.Tensor, torch.Tensor]:
    """Ordered top-K candidates of every row: (cand_logit [rows,K] fp32, cand_id [rows,K] int32)."""
    rows, d, V, dev = _lmhead_operands(hidden, lm_head)
    if cand_logit is None:
        cand_logit = torch.empty(rows, K, dtype=torch.float32, device=dev)
    if cand_id is None:
        cand_id = torch.empty(rows, K, dtype=torch.int32, device=dev)
    _dev_tensor(cand_logit, "cand_logit", torch.float32, shape=(rows, K), device=dev)
    _dev_tensor(cand_id, "cand_id", torch.int32, shape=(rows, K), device=dev)
    need = propose_workspace_size(rows, d, V, K)
    ws = workspace if workspace is not None else _workspace(dev, need, "propose", stream)
    st = lib().brisk_propose_block(_ptr(hidden), _ptr(lm_head), rows, d, V, K, _ptr(cand_logit),
                                   _ptr(cand_id), _ptr(ws), _ws_bytes(ws, dev, need),
                                   _stream_ptr(dev, stream))
    _check(st, "brisk_propose_block")
    return cand_logit, cand_id


def propose_block_noalloc(hidden: torch.Tensor, lm_head: torch.Tensor, K: int, cand_logit: torch.Tensor,
                          cand_id: torch.Tensor, *, stream=None) -> None:
    """:func:`propose_block` on the library's fixed per-device scratch: the
    library allocates nothing; the caller passes the [rows, K] outputs.  Calls
    that overlap in time on one GPU race (they share the scratch)."""
    rows, d, V, dev = _lmhead_operands(hidden, lm_head)
    _dev_tensor(cand_logit, "cand_logit", torch.float32, shape=(rows, K), device=dev)
    _dev_tensor(cand_id, "cand_id", torch.int32, shape=(rows, K), device=dev)
    st = lib().brisk_propose_block_noalloc(_ptr(hidden), _ptr(lm_head), rows, d, V, K, _ptr(cand_logit),
                                           _ptr(cand_id), _stream_ptr(dev, stream))
    _check(st, "brisk_propose_block_noalloc")


def propose_lmhead(hidden: torch.Tensor, lm_head: torch.Tensor, K: int, workspace: torch.Tensor, *,
                   stream=None) -> None:
    """The LM-head pass of propose_block alone: per-share ordered keys into ``workspace``."""
    rows, d, V, dev = _lmhead_operands(hidden, lm_head)
    need = propose_workspace_size(rows, d, V, K)
    st = lib().brisk_propose_lmhead(_ptr(hidden), _ptr(lm_head), rows, d, V, K, _ptr(workspace),
                                    _ws_bytes(workspace, dev, need), _stream_ptr(dev, stream))
    _check(st, "brisk_propose_lmhead")


def propose_merge(rows: int, V: int, K: int, workspace: torch.Tensor, cand_logit: torch.Tensor,
                  cand_id: torch.Tensor, *, stream=None) -> None:
    """The merge of propose_block alone: candidates from the keys a propose_lmhead left."""
    _dev_tensor(cand_logit, "cand_logit", torch.float32, shape=(rows, K))
    dev = cand_logit.device
    _dev_tensor(cand_id, "cand_id", torch.int32, shape=(rows, K), device=dev)
    need = propose_workspace_size(rows, 8, V, K)   # the key layout does not depend on d
    st = lib().brisk_propose_merge(rows, V, K, _ptr(cand_logit), _ptr(cand_id), _ptr(workspace),
                                   _ws_bytes(workspace, dev, need), _stream_ptr(dev, stream))
    _check(st, "brisk_propose_merge")


# ----------------------------------------------------------------- rerank
class Corrector:
    """Corrector parameters psi: bf16 device tensors plus the two gate scalars."""

    def __init__(self, tensors: Dict[str, torch.Tensor], alpha: float, b_g: float):
        missing = [n for n in PSI_FIELDS if n not in tensors]
        if missing:
            raise ValueError(f"missing corrector tensors: {missing}")
        for n in PSI_FIELDS:
            v = tensors[n]
            if not isinstance(v, torch.Tensor) or v.dim() != (1 if n == "w_g" else 2):
                raise ValueError(f"{n} must be a {1 if n == 'w_g' else 2}-d tensor")
        self.t = {n: tensors[n].contiguous() for n in PSI_FIELDS}
        self.alpha, self.b_g = float(alpha), float(b_g)
        t = self.t
        ds, self.d = t["A_h"].shape
        self.device = t["A_h"].device
        self.dims = dict(d_state=ds, d_hproj=t["P_h"].shape[0], d_tproj=t["P_e"].shape[0],
                         d_pos=t["pos_emb"].shape[1], d_feat=t["P_phi"].shape[0],
                         rank=t["W_s"].shape[0], max_L=t["pos_emb"].shape[0])
        dm = self.dims
        d_in = dm["d_hproj"] + dm["d_tproj"] + dm["d_pos"] + dm["d_feat"]
        want = {"A_h": (ds, self.d), "A_e": (ds, self.d), "P_h": (dm["d_hproj"], self.d),
                "P_e": (dm["d_tproj"], self.d), "pos_emb": (dm["max_L"], dm["d_pos"]),
                "P_phi": (dm["d_feat"], 5), "W_z": (ds, d_in), "W_h": (ds, d_in),
                "W_s": (dm["rank"], ds), "W_c": (dm["rank"], self.d), "w_g": (ds + 5,)}
        for n in PSI_FIELDS:        # every shape first, then dtypes and devices
            if tuple(t[n].shape) != want[n]:
                raise ValueError(f"{n} must have shape {want[n]}, got {tuple(t[n].shape)}")
        for n in PSI_FIELDS:
            _dev_tensor(t[n], n, torch.bfloat16, shape=want[n], device=self.device)
        self._c = _CorrectorC(**self.dims, **{n: _ptr(self.t[n]) for n in PSI_FIELDS},
                              alpha=self.alpha, b_g=self.b_g, tables=None, tables_V=0)
        self.tables: Optional[torch.Tensor] = None

    @property
    def c_struct(self) -> _CorrectorC:
        return self._c

    def prepare(self, lm_head: torch.Tensor, tok_embed: torch.Tensor, *, stream=None) -> torch.Tensor:
        """Compute the per-token tables (brisk_corrector_prepare) for this LM
        head and input embedding; later rerank calls read the candidates' and
        anchors' lifts from them.  Returns the [3, V, max(256, d_state)] fp32
        tables, which the corrector keeps."""
        _dev_tensor(lm_head, "lm_head", torch.bfloat16, 2, device=self.device)
        V, d = lm_head.shape
        if d != self.d:
            raise ValueError(f"lm_head has d = {d}, the corrector d = {self.d}")
        _dev_tensor(tok_embed, "tok_embed", torch.bfloat16, shape=(V, d), device=self.device)
        tb, wb = _sz(), _sz()
        _check(lib().brisk_corrector_tables_size(ctypes.byref(self._c), V, ctypes.byref(tb), ctypes.byref(wb)),
               "brisk_corrector_tables_size")
        vs = max(256, self.dims["d_state"])
        tables = torch.empty(3, V, vs, dtype=torch.float32, device=self.device)
        ws = torch.empty(wb.value, dtype=torch.uint8, device=self.device)
        _check(lib().brisk_corrector_prepare(ctypes.byref(self._c), _ptr(lm_head), _ptr(tok_embed), V, d,
                                             _ptr(tables), tables.numel() * 4, _ptr(ws), wb.value,
                                             _stream_ptr(self.device, stream)),
               "brisk_corrector_prepare")
        self.tables = tables
        self._c.tables = _ptr(tables)
        self._c.tables_V = V
        return tables

    def drop_tables(self) -> None:
        """Forget the per-token tables: rerank projects the embedding rows again."""
        self.tables = None
        self._c.tables = None
        self._c.tables_V = 0


def rerank_workspace_size(corr: Corrector, B: int, L: int, K: int) -> int:
    out = _sz()
    _check(lib().brisk_rerank_workspace_size(ctypes.byref(corr.c_struct), B, L, K, ctypes.byref(out)),
           "brisk_rerank_workspace_size")
    return out.value


def _rerank_args(corr, hidden, ctx_hidden, anchor_tok, lm_head, tok_embed, cand_logit, cand_id, B, L,
                 want_scores, selected, refined, gamma, resid, workspace, stream):
    rows = B * L
    _dev_tensor(hidden, "hidden", torch.bfloat16, 2)
    dev = hidden.device
    if hidden.shape[0] != rows:
        raise ValueError(f"hidden has {hidden.shape[0]} rows, B*L = {rows}")
    d = hidden.shape[1]
    if d != corr.d or corr.device != dev:
        raise ValueError(f"the corrector was built for d = {corr.d} on {corr.device}, "
                         f"the hidden states have d = {d} on {dev}")
    _dev_tensor(ctx_hidden, "ctx_hidden", torch.bfloat16, shape=(B, d), device=dev)
    _dev_tensor(anchor_tok, "anchor_tok", torch.int32, shape=(B,), device=dev)
    _dev_tensor(lm_head, "lm_head", torch.bfloat16, 2, device=dev)
    V = lm_head.shape[0]
    if lm_head.shape[1] != d:
        raise ValueError("hidden and lm_head disagree on d")
    _dev_tensor(tok_embed, "tok_embed", torch.bfloat16, shape=(V, d), device=dev)
    _dev_tensor(cand_id, "cand_id", torch.int32, 2, device=dev)
    K = cand_id.shape[1]
    _dev_tensor(cand_id, "cand_id", torch.int32, shape=(rows, K), device=dev)
    _dev_tensor(cand_logit, "cand_logit", torch.float32, shape=(rows, K), device=dev)
    if selected is None:
        selected = torch.empty(B, L, dtype=torch.int32, device=dev)
    if want_scores:
        if refined is None:
            refined = torch.empty(rows, K, dtype=torch.float32, device=dev)
        if gamma is None:
            gamma = torch.empty(rows, dtype=torch.float32, device=dev)
        if resid is None:
            resid = torch.empty(rows, K, dtype=torch.float32, device=dev)
    _dev_tensor(selected, "selected", torch.int32, shape=(B, L), device=dev)
    for name, t, shp in (("refined", refined, (rows, K)), ("gamma", gamma, (rows,)), ("resid", resid, (rows, K))):
        if t is not None:
            _dev_tensor(t, name, torch.float32, shape=shp, device=dev)
    need = rerank_workspace_size(corr, B, L, K)
    ws = workspace if workspace is not None else _workspace(dev, need, "rerank", stream)
    ws_n = _ws_bytes(ws, dev, need)
    out = {"selected": selected}
    for k, v in (("refined", refined), ("gamma", gamma), ("resid", resid)):
        if v is not None:
            out[k] = v
    return K, d, V, dev, ws, ws_n, out


def rerank(corr: Corrector, hidden: torch.Tensor, ctx_hidden: torch.Tensor, anchor_tok: torch.Tensor,
           lm_head: torch.Tensor, tok_embed: torch.Tensor, cand_logit: torch.Tensor,
           cand_id: torch.Tensor, B: int, L: int, *, want_scores: bool = False,
           selected: Optional[torch.Tensor] = None, refined: Optional[torch.Tensor] = None,
           gamma: Optional[torch.Tensor] = None, resid: Optional[torch.Tensor] = None,
           workspace: Optional[torch.Tensor] = None, stream=None) -> Dict[str, torch.Tensor]:
    """Run the corrector; returns {"selected": [B,L] int32} plus "refined", "gamma",
    "resid" when ``want_scores`` (or when the caller passes those buffers)."""
    K, d, V, dev, ws, ws_n, out = _rerank_args(corr, hidden, ctx_hidden, anchor_tok, lm_head, tok_embed,
                                               cand_logit, cand_id, B, L, want_scores, selected, refined,
                                               gamma, resid, workspace, stream)
    st = lib().brisk_rerank(ctypes.byref(corr.c_struct), _ptr(hidden), _ptr(ctx_hidden),
                            _ptr(anchor_tok), _ptr(lm_head), _ptr(tok_embed), _ptr(cand_logit),
                            _ptr(cand_id), B, L, K, d, V, _ptr(out["selected"]), _ptr(out.get("refined")),
                            _ptr(out.get("gamma")), _ptr(out.get("resid")), _ptr(ws), ws_n,
                            _stream_ptr(dev, stream))
    _check(st, "brisk_rerank")
    return out


def rerank_verify(corr: Corrector, hidden: torch.Tensor, ctx_hidden: torch.Tensor, anchor_tok: torch.Tensor,
                  lm_head: torch.Tensor, tok_embed: torch.Tensor, cand_logit: torch.Tensor,
                  cand_id: torch.Tensor, verifier: torch.Tensor, B: int, L: int, *,
                  want_scores: bool = False, selected: Optional[torch.Tensor] = None,
                  refined: Optional[torch.Tensor] = None, gamma: Optional[torch.Tensor] = None,
                  resid: Optional[torch.Tensor] = None, accept_len: Optional[torch.Tensor] = None,
                  correction: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                  stream=None) -> Dict[str, torch.Tensor]:
    """:func:`rerank` then :func:`verify_accept` on its selections, in one call.
    Returns the rerank outputs plus "accept_len" and "correction" [B] int32."""
    K, d, V, dev, ws, ws_n, out = _rerank_args(corr, hidden, ctx_hidden, anchor_tok, lm_head, tok_embed,
                                               cand_logit, cand_id, B, L, want_scores, selected, refined,
                                               gamma, resid, workspace, stream)
    _dev_tensor(verifier, "verifier", torch.int32, shape=(B, L), device=dev)
    if accept_len is None:
        accept_len = torch.empty(B, dtype=torch.int32, device=dev)
    if correction is None:
        correction = torch.empty(B, dtype=torch.int32, device=dev)
    _dev_tensor(accept_len, "accept_len", torch.int32, shape=(B,), device=dev)
    _dev_tensor(correction, "correction", torch.int32, shape=(B,), device=dev)
    st = lib().brisk_rerank_verify(ctypes.byref(corr.c_struct), _ptr(hidden), _ptr(ctx_hidden),
                                   _ptr(anchor_tok), _ptr(lm_head), _ptr(tok_embed), _ptr(cand_logit),
                                   _ptr(cand_id), _ptr(verifier), B, L, K, d, V, _ptr(out["selected"]),
                                   _ptr(out.get("refined")), _ptr(out.get("gamma")), _ptr(out.get("resid")),
                                   _ptr(accept_len), _ptr(correction), _ptr(ws), ws_n,
                                   _stream_ptr(dev, stream))
    _check(st, "brisk_rerank_verify")
    out["accept_len"] = accept_len
    out["correction"] = correction
    return out


def rerank_hoist(corr: Corrector, hidden: torch.Tensor, ctx_hidden: torch.Tensor, anchor_tok: torch.Tensor,
                 tok_embed: torch.Tensor, B: int, L: int, K: int, workspace: torch.Tensor, *,
                 stream=None) -> None:
    """The part of :func:`rerank` that does not read the candidates, queued on
    ``stream`` into ``workspace`` (which :func:`rerank_finish` then completes);
    it may run while the LM-head pass that makes the candidates streams."""
    _dev_tensor(hidden, "hidden", torch.bfloat16, 2)
    dev = hidden.device
    rows, d = hidden.shape
    if rows != B * L:
        raise ValueError(f"hidden has {rows} rows, B*L = {B * L}")
    if d != corr.d or corr.device != dev:
        raise ValueError(f"the corrector was built for d = {corr.d} on {corr.device}, "
                         f"the hidden states have d = {d} on {dev}")
    _dev_tensor(ctx_hidden, "ctx_hidden", torch.bfloat16, shape=(B, d), device=dev)
    _dev_tensor(anchor_tok, "anchor_tok", torch.int32, shape=(B,), device=dev)
    _dev_tensor(tok_embed, "tok_embed", torch.bfloat16, 2, device=dev)
    if tok_embed.shape[1] != d:
        raise ValueError("hidden and tok_embed disagree on d")
    V = tok_embed.shape[0]
    need = rerank_workspace_size(corr, B, L, K)
    st = lib().brisk_rerank_hoist(ctypes.byref(corr.c_struct), _ptr(hidden), _ptr(ctx_hidden),
                                  _ptr(anchor_tok), _ptr(tok_embed), B, L, K, d, V, _ptr(workspace),
                                  _ws_bytes(workspace, dev, need), _stream_ptr(dev, stream))
    _check(st, "brisk_rerank_hoist")


def rerank_finish(corr: Corrector, hidden: torch.Tensor, ctx_hidden: torch.Tensor, anchor_tok: torch.Tensor,
                  lm_head: torch.Tensor, tok_embed: torch.Tensor, cand_logit: torch.Tensor,
                  cand_id: torch.Tensor, B: int, L: int, workspace: torch.Tensor, *,
                  verifier: Optional[torch.Tensor] = None, want_scores: bool = False,
                  selected: Optional[torch.Tensor] = None, refined: Optional[torch.Tensor] = None,
                  gamma: Optional[torch.Tensor] = None, resid: Optional[torch.Tensor] = None,
                  accept_len: Optional[torch.Tensor] = None, correction: Optional[torch.Tensor] = None,
                  stream=None) -> Dict[str, torch.Tensor]:
    """The rest of :func:`rerank` (``verifier`` None) or :func:`rerank_verify`
    on a ``workspace`` that :func:`rerank_hoist` filled with the same inputs;
    returns what that call returns."""
    K, d, V, dev, ws, ws_n, out = _rerank_args(corr, hidden, ctx_hidden, anchor_tok, lm_head, tok_embed,
                                               cand_logit, cand_id, B, L, want_scores, selected, refined,
                                               gamma, resid, workspace, stream)
    if verifier is not None:
        _dev_tensor(verifier, "verifier", torch.int32, shape=(B, L), device=dev)
        if accept_len is None:
            accept_len = torch.empty(B, dtype=torch.int32, device=dev)
        if correction is None:
            correction = torch.empty(B, dtype=torch.int32, device=dev)
        _dev_tensor(accept_len, "accept_len", torch.int32, shape=(B,), device=dev)
        _dev_tensor(correction, "correction", torch.int32, shape=(B,), device=dev)
    st = lib().brisk_rerank_finish(ctypes.byref(corr.c_struct), _ptr(hidden), _ptr(ctx_hidden),
                                   _ptr(anchor_tok), _ptr(lm_head), _ptr(tok_embed), _ptr(cand_logit),
                                   _ptr(cand_id), _ptr(verifier), B, L, K, d, V, _ptr(out["selected"]),
                                   _ptr(out.get("refined")), _ptr(out.get("gamma")), _ptr(out.get("resid")),
                                   _ptr(accept_len), _ptr(correction), _ptr(ws), ws_n,
                                   _stream_ptr(dev, stream))
    _check(st, "brisk_rerank_finish")
    if verifier is not None:
        out["accept_len"] = accept_len
        out["correction"] = correction
    return out


# ----------------------------------------------------------------- verify
def verify_accept(proposal: torch.Tensor, verifier: torch.Tensor, *,
                  accept_len: Optional[torch.Tensor] = None, correction: Optional[torch.Tensor] = None,
                  stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(accept_len [B] int32, correction [B] int32; -1 where the block is fully accepted)."""
    _dev_tensor(proposal, "proposal", torch.int32, 2)
    B, L = proposal.shape
    dev = proposal.device
    _dev_tensor(verifier, "verifier", torch.int32, shape=(B, L), device=dev)
    if accept_len is None:
        accept_len = torch.empty(B, dtype=torch.int32, device=dev)
    if correction is None:
        correction = torch.empty(B, dtype=torch.int32, device=dev)
    _dev_tensor(accept_len, "accept_len", torch.int32, shape=(B,), device=dev)
    _dev_tensor(correction, "correction", torch.int32, shape=(B,), device=dev)
    st = lib().brisk_verify_accept(_ptr(proposal), _ptr(verifier), B, L, _ptr(accept_len),
                                   _ptr(correction), _stream_ptr(dev, stream))
    _check(st, "brisk_verify_accept")
    return accept_len, correction


def accept_profile(accept_len: torch.Tensor, M: int, *, eps: float = 0.0,
                   workspace: Optional[torch.Tensor] = None, stream=None) -> Dict[str, torch.Tensor]:
    """Acceptance profile of verified blocks: ``a``, ``w_raw``, ``w`` [M] and
    ``tpf_fpt`` [2], all float64 on the device of ``accept_len``."""
    _dev_tensor(accept_len, "accept_len", torch.int32, 1)
    n = accept_len.shape[0]
    dev = accept_len.device
    nbytes = _sz(0)
    _check(lib().brisk_accept_profile_workspace_size(n, M, ctypes.byref(nbytes)),
           "brisk_accept_profile_workspace_size")
    if workspace is None:
        workspace = _workspace(dev, nbytes.value, "profile", stream)
    ws_n = _ws_bytes(workspace, dev, nbytes.value)
    out = {k: torch.empty(M, dtype=torch.float64, device=dev) for k in ("a", "w_raw", "w")}
    out["tpf_fpt"] = torch.empty(2, dtype=torch.float64, device=dev)
    st = lib().brisk_accept_profile(_ptr(accept_len) if n > 0 else None, n, M, float(eps),
                                    _ptr(out["a"]), _ptr(out["w_raw"]), _ptr(out["w"]),
                                    _ptr(out["tpf_fpt"]), _ptr(workspace), ws_n,
                                    _stream_ptr(dev, stream))
    _check(st, "brisk_accept_profile")
    return out


def propose_verify(hidden: torch.Tensor, lm_head: torch.Tensor, rows_prop: int, K: int, *,
                   cand_logit: Optional[torch.Tensor] = None, cand_id: Optional[torch.Tensor] = None,
                   ver_token: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                   stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """One LM-head pass: the first ``rows_prop`` rows of ``hidden`` get ordered
    top-K candidates, the remaining rows their argmax token.
    Returns (cand_logit [rows_prop, K], cand_id [rows_prop, K], ver_token [rows_ver])."""
    rows, d, V, dev = _lmhead_operands(hidden, lm_head)
    rows_ver = rows - rows_prop
    if rows_prop < 0 or rows_ver < 0:
        raise ValueError("rows_prop must lie in [0, hidden rows]")
    if cand_logit is None:
        cand_logit = torch.empty(rows_prop, K, dtype=torch.float32, device=dev)
    if cand_id is None:
        cand_id = torch.empty(rows_prop, K, dtype=torch.int32, device=dev)
    if ver_token is None:
        ver_token = torch.empty(rows_ver, dtype=torch.int32, device=dev)
    _dev_tensor(cand_logit, "cand_logit", torch.float32, shape=(rows_prop, K), device=dev)
    _dev_tensor(cand_id, "cand_id", torch.int32, shape=(rows_prop, K), device=dev)
    _dev_tensor(ver_token, "ver_token", torch.int32, shape=(rows_ver,), device=dev)
    nbytes = _sz(0)
    _check(lib().brisk_propose_verify_workspace_size(rows_prop, rows_ver, d, V, K, ctypes.byref(nbytes)),
           "brisk_propose_verify_workspace_size")
    ws = workspace if workspace is not None else _workspace(dev, nbytes.value, "propose", stream)
    st = lib().brisk_propose_verify(_ptr(hidden), _ptr(lm_head), rows_prop, rows_ver, d, V, K,
                                    _ptr(cand_logit) if rows_prop else None,
                                    _ptr(cand_id) if rows_prop else None,
                                    _ptr(ver_token) if rows_ver else None, _ptr(ws),
                                    _ws_bytes(ws, dev, nbytes.value), _stream_ptr(dev, stream))
    _check(st, "brisk_propose_verify")
    return cand_logit, cand_id, ver_token


def verify_commit(proposal: torch.Tensor, verifier: torch.Tensor, *, stream=None
                  ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(accept_len [B], committed [B, L + 1] padded with -1, n_committed [B])."""
    _dev_tensor(proposal, "proposal", torch.int32, 2)
    B, L = proposal.shape
    dev = proposal.device
    _dev_tensor(verifier, "verifier", torch.int32, shape=(B, L), device=dev)
    acc = torch.empty(B, dtype=torch.int32, device=dev)
    committed = torch.empty(B, L + 1, dtype=torch.int32, device=dev)
    n = torch.empty(B, dtype=torch.int32, device=dev)
    st = lib().brisk_verify_commit(_ptr(proposal), _ptr(verifier), B, L, _ptr(acc), _ptr(committed),
                                   _ptr(n), _stream_ptr(dev, stream))
    _check(st, "brisk_verify_commit")
    return acc, committed, n


def corrector_loss(ver_hidden: torch.Tensor, lm_head: torch.Tensor, cand_id: torch.Tensor,
                   cand_logit: torch.Tensor, refined: torch.Tensor, accept_len: torch.Tensor,
                   B: int, L: int, *, beta: float = 0.01, stream=None) -> Dict[str, torch.Tensor]:
    """Per-position losses ``loss_pos``, ``ce``, ``kl`` [B*L] and ``loss_mean``
    [2] = (mean over reached positions, their count)."""
    rows = B * L
    nrows, d, V, dev = _lmhead_operands(ver_hidden, lm_head)
    if nrows != rows:
        raise ValueError(f"ver_hidden has {nrows} rows, B*L = {rows}")
    _dev_tensor(cand_id, "cand_id", torch.int32, 2, device=dev)
    K = cand_id.shape[1]
    _dev_tensor(cand_id, "cand_id", torch.int32, shape=(rows, K), device=dev)
    _dev_tensor(cand_logit, "cand_logit", torch.float32, shape=(rows, K), device=dev)
    _dev_tensor(refined, "refined", torch.float32, shape=(rows, K), device=dev)
    _dev_tensor(accept_len, "accept_len", torch.int32, shape=(B,), device=dev)
    out = {k: torch.empty(rows, dtype=torch.float32, device=dev) for k in ("loss_pos", "ce", "kl")}
    out["loss_mean"] = torch.empty(2, dtype=torch.float32, device=dev)
    st = lib().brisk_corrector_loss(_ptr(ver_hidden), _ptr(lm_head), _ptr(cand_id), _ptr(cand_logit),
                                    _ptr(refined), _ptr(accept_len), B, L, K, d, V, float(beta),
                                    _ptr(out["loss_pos"]), _ptr(out["ce"]), _ptr(out["kl"]),
                                    _ptr(out["loss_mean"]), _stream_ptr(dev, stream))
    _check(st, "brisk_corrector_loss")
    return out


def spec_verify(ver_hidden: torch.Tensor, lm_head: torch.Tensor, proposal: torch.Tensor,
                cand_id: torch.Tensor, cand_prob: Optional[torch.Tensor], u_accept: torch.Tensor, seed: int,
                temperature: float = 1.0, *, workspace: Optional[torch.Tensor] = None,
                stream=None) -> Dict[str, torch.Tensor]:
    """Stochastic verification: ``accept_len``, ``correction`` [B] and the
    per-position ``row_accept``, ``row_resample`` [B*L].  ``cand_prob=None``
    is the greedy proposer (pi = point mass at the proposal)."""
    rows, d, V, dev = _lmhead_operands(ver_hidden, lm_head)
    _dev_tensor(proposal, "proposal", torch.int32, 2, device=dev)
    B, L = proposal.shape
    if B * L != rows:
        raise ValueError(f"proposal is [{B}, {L}], ver_hidden has {rows} rows")
    _dev_tensor(cand_id, "cand_id", torch.int32, 2, device=dev)
    K = cand_id.shape[1]
    _dev_tensor(cand_id, "cand_id", torch.int32, shape=(rows, K), device=dev)
    if cand_prob is not None:
        _dev_tensor(cand_prob, "cand_prob", torch.float32, shape=(rows, K), device=dev)
    _dev_tensor(u_accept, "u_accept", torch.float32, shape=(rows,), device=dev)
    nbytes = _sz(0)
    _check(lib().brisk_spec_verify_workspace_size(B, L, V, K, ctypes.byref(nbytes)),
           "brisk_spec_verify_workspace_size")
    ws = workspace if workspace is not None else _workspace(dev, nbytes.value, "spec", stream)
    ws_n = _ws_bytes(ws, dev, nbytes.value)
    out = {"accept_len": torch.empty(B, dtype=torch.int32, device=dev),
           "correction": torch.empty(B, dtype=torch.int32, device=dev),
           "row_accept": torch.empty(B * L, dtype=torch.int32, device=dev),
           "row_resample": torch.empty(B * L, dtype=torch.int32, device=dev)}
    st = lib().brisk_spec_verify(_ptr(ver_hidden), _ptr(lm_head), _ptr(proposal), _ptr(cand_id),
                                 _ptr(cand_prob), _ptr(u_accept), int(seed) & ((1 << 64) - 1),
                                 float(temperature), B, L, K, d, V, _ptr(out["accept_len"]),
                                 _ptr(out["correction"]), _ptr(out["row_accept"]),
                                 _ptr(out["row_resample"]), _ptr(ws), ws_n, _stream_ptr(dev, stream))
    _check(st, "brisk_spec_verify")
    return out


# ------------------------------------------------- attention, cache and drafts
_HALF = {torch.bfloat16: 0, torch.float16: 1}


class KVCache:
    """Paged keys and values of a batch of sequences.

    ``k_pages`` and ``v_pages`` are [n_pages, page_size, n_kv_heads, d_head] in
    bfloat16 or float16 with the same strides; any strides with contiguous
    heads will do, so head-major pages are passed as a transposed view.
    ``block_table`` [B, max_pages] int32 lists each sequence's pages and
    ``seq_len`` [B] int32 the slots it holds, the block in flight included.
    The tensors stay the caller's: lengths and pages may be written between
    calls.  Which tensors they are is fixed (the library has their addresses):
    new lengths are copied into ``seq_len``, and an attribute assigned is refused."""

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor, block_table: torch.Tensor, seq_len: torch.Tensor):
        for t, n in ((k_pages, "k_pages"), (v_pages, "v_pages")):
            _half_tensor(t, n, 4)
        if v_pages.shape != k_pages.shape or _steps(v_pages) != _steps(k_pages) or v_pages.dtype != k_pages.dtype:
            raise ValueError("k_pages and v_pages must agree in shape, strides and dtype")
        dev = k_pages.device
        if v_pages.device != dev:
            raise ValueError(f"v_pages is on {v_pages.device}, k_pages on {dev}")
        _dev_tensor(block_table, "block_table", torch.int32, 2, device=dev)
        _dev_tensor(seq_len, "seq_len", torch.int32, shape=(block_table.shape[0],), device=dev)
        self.k_pages, self.v_pages, self.block_table, self.seq_len = k_pages, v_pages, block_table, seq_len
        self.device, self.dtype = dev, k_pages.dtype
        n_pages, self.page_size, self.n_kv_heads, self.d_head = k_pages.shape
        self.B, max_pages = block_table.shape
        self.max_seq_len = max_pages * self.page_size
        page, slot, head, _ = _steps(k_pages)
        self._c = _KVCacheC(_HALF[self.dtype], self.n_kv_heads, self.d_head, self.page_size, n_pages, max_pages, page,
                            slot, head, _ptr(k_pages), _ptr(v_pages), _ptr(block_table), _ptr(seq_len))
        self._ref = ctypes.byref(self._c)
        self._fixed = True

    def __setattr__(self, name: str, value) -> None:
        if getattr(self, "_fixed", False):
            raise AttributeError(f"{name}: a KVCache keeps its tensors; copy into them or make another cache")
        object.__setattr__(self, name, value)

    @property
    def c_struct(self) -> _KVCacheC:
        return self._c


def _steps(t: torch.Tensor) -> Tuple[int, ...]:
    """Strides, where a dimension of one element, whose stride nothing uses, has 0."""
    return tuple([0 if n == 1 else s for n, s in zip(t.shape, t.stride())])


def _half_tensor(t: torch.Tensor, name: str, ndim: int, like: Optional[KVCache] = None) -> None:
    """A 2-byte tensor on a HIP device whose last dimension is contiguous."""
    if (like is not None and type(t) is torch.Tensor and t.dtype is like.dtype and t.is_cuda and t.dim() == ndim
            and t.device == like.device and t.stride(-1) == 1):
        return                                     # nothing to object to: most calls end here
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype not in _HALF if like is None else t.dtype != like.dtype:
        raise TypeError(f"{name} must be {'bfloat16 or float16' if like is None else like.dtype}, got {t.dtype}")
    if t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dims, got shape {tuple(t.shape)}")
    if t.numel() and t.stride(-1) != 1:
        raise ValueError(f"{name} must be contiguous in its last dimension")
    if not t.is_cuda:
        raise ValueError(f"{name} must live on a HIP device, got {t.device}")
    if like is not None and t.device != like.device:
        raise ValueError(f"{name} is on {t.device}, the cache on {like.device}")


def _block_queries(q: torch.Tensor, cache: KVCache, block_mask: Optional[torch.Tensor]):
    """(B, L, H, row stride, head stride) of a block's queries, checked against the cache."""
    _half_tensor(q, "q", 4, cache)
    B, L, H, D = q.shape
    if B != cache.B or D != cache.d_head:
        raise ValueError(f"q is {tuple(q.shape)}, the cache holds {cache.B} sequences of {cache.d_head}-wide heads")
    sb, sl, sh, _ = q.stride()
    if B > 1 and L > 1 and sb != L * sl:
        raise ValueError("the rows of q must be evenly spaced: stride(0) == L * stride(1)")
    if block_mask is not None:
        _dev_tensor(block_mask, "block_mask", torch.int64, shape=(B, L), device=cache.device)
    return B, L, H, (sl if L > 1 else sb if B > 1 else 0), (sh if H > 1 else 0)


def block_attention(q: torch.Tensor, cache: KVCache, *, prefix: Optional[Tuple[torch.Tensor, torch.Tensor]] = None,
                    block_mask: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                    max_seq_len: Optional[int] = None, out: Optional[torch.Tensor] = None,
                    lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None
                    ) -> Tuple[torch.Tensor, torch.Tensor]:
    """Attention of every sequence's block over the shared prefix and its own cache.

    ``q`` [B, L, H, D] (L = 1: single tokens; rows and heads may be strided, as
    in a fused projection's output), ``prefix`` = (k, v) [P, n_kv_heads, D]
    held once for the whole batch, ``block_mask`` [B, L] int64 whose bit t lets
    position i see the block's position t, ``scale`` 1/sqrt(D) by default,
    ``max_seq_len`` a host bound of the lengths.  Returns (out [B, L, H, D],
    lse [B, L, H] fp32); a row that sees no key gets zeros and -inf."""
    B, L, H, row, head = _block_queries(q, cache, block_mask)
    return _attend(lib().brisk_block_attention, "brisk_block_attention", block_attention_workspace_size, "attention", q,
                   cache, prefix, block_mask, scale, max_seq_len, out, lse, workspace, stream, (B, L, H, row, head))


def _attend(entry, where, workspace_size, tag, q, cache, prefix, block_mask, scale, max_seq_len, out, lse, workspace,
            stream, rows) -> Tuple[torch.Tensor, torch.Tensor]:
    """Attention over either cache: the arguments past the queries checked, outputs and scratch made, the call."""
    B, L, H, row, head = rows
    dev, D = cache.device, cache.d_head
    pre, P = None, 0
    if prefix is not None:
        k, v = prefix
        for t, n in ((k, "prefix keys"), (v, "prefix values")):
            _half_tensor(t, n, 3, cache)
        P = k.shape[0]
        if k.shape[1:] != (cache.n_kv_heads, D) or v.shape != k.shape or (P and _steps(v) != _steps(k)):
            raise ValueError(f"prefix must be two tensors [P, {cache.n_kv_heads}, {D}] of the same strides")
        if P:
            pre = _KVPrefixC(P, *_steps(k)[:2], _ptr(k), _ptr(v))
    if out is None:
        out = torch.empty(B, L, H, D, dtype=cache.dtype, device=dev)
    else:
        _dev_tensor(out, "out", cache.dtype, shape=(B, L, H, D), device=dev)
    if lse is None:
        lse = torch.empty(B, L, H, dtype=torch.float32, device=dev)
    else:
        _dev_tensor(lse, "lse", torch.float32, shape=(B, L, H), device=dev)
    most = cache.max_seq_len if max_seq_len is None else max_seq_len
    need = workspace_size(B, L, H, cache.n_kv_heads, D, P, most)
    if workspace is not None:
        ws, nbytes = workspace.data_ptr(), _ws_bytes(workspace, dev, need)
    else:
        ws, nbytes = (_workspace(dev, need, tag, stream).data_ptr(), need) if need else (None, 0)
    st = entry(cache._ref, None if pre is None else ctypes.byref(pre), q.data_ptr(), row, head, _ptr(block_mask), B, L, H,
               most, D ** -0.5 if scale is None else scale, out.data_ptr(), lse.data_ptr(), ws, nbytes,
               _stream_ptr(dev, stream))
    _check(st, where)
    return out, lse


@functools.lru_cache(maxsize=1024)
def block_attention_workspace_size(B: int, L: int, n_heads: int, n_kv_heads: int, d_head: int, prefix_len: int,
                                   max_seq_len: int) -> int:
    out = _sz()
    _check(lib().brisk_block_attention_workspace_size(B, L, n_heads, n_kv_heads, d_head, prefix_len, max_seq_len,
                                                      ctypes.byref(out)), "brisk_block_attention_workspace_size")
    return out.value


def cache_score(q: torch.Tensor, lse: torch.Tensor, cache: KVCache, score: torch.Tensor, *,
                block_mask: Optional[torch.Tensor] = None, scale: Optional[float] = None, decay: float = 1.0,
                out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """``decay * score`` plus the attention weight every cached key received from
    the block's rows: [B, n_kv_heads, cap] fp32, zero past a sequence's length.
    ``q``, ``block_mask`` and ``scale`` as in :func:`block_attention`, ``lse``
    as it returned it.  ``out`` may be ``score`` itself."""
    B, L, H, row, head = _block_queries(q, cache, block_mask)
    dev = cache.device
    _dev_tensor(lse, "lse", torch.float32, shape=(B, L, H), device=dev)
    _dev_tensor(score, "score", torch.float32, 3, device=dev)
    cap = score.shape[2]
    shape = (B, cache.n_kv_heads, cap)
    _dev_tensor(score, "score", torch.float32, shape=shape, device=dev)
    if out is None:
        out = torch.empty_like(score)
    else:
        _dev_tensor(out, "out", torch.float32, shape=shape, device=dev)
    st = lib().brisk_cache_score(cache._ref, _ptr(q), row, head, _ptr(block_mask), _ptr(lse), B, L, H,
                                 cache.d_head ** -0.5 if scale is None else scale, decay, _ptr(score), _ptr(out), cap,
                                 _stream_ptr(dev, stream))
    _check(st, "brisk_cache_score")
    return out


def cache_evict(cache: KVCache, score: torch.Tensor, pos: torch.Tensor, next_pos: torch.Tensor, budget: int,
                recent: int, *, score_out: Optional[torch.Tensor] = None, pos_out: Optional[torch.Tensor] = None,
                new_len: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None
                ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Cuts every sequence's cache to ``budget`` slots, in place: each head keeps
    the slots whose ``pos`` is among the ``recent`` latest before ``next_pos``
    [B], then those of the largest ``score``.  ``score`` fp32 and ``pos`` int32
    are [B, n_kv_heads, cap]; returns (score, pos, new_len [B]) of the slots as
    they lie afterwards.  The cache's ``seq_len`` is left to the caller: workgroups
    read it while others write ``new_len``, which is therefore another tensor, copied into it afterwards."""
    dev = cache.device
    _dev_tensor(score, "score", torch.float32, 3, device=dev)
    cap = score.shape[2]
    shape = (cache.B, cache.n_kv_heads, cap)
    _dev_tensor(score, "score", torch.float32, shape=shape, device=dev)
    _dev_tensor(pos, "pos", torch.int32, shape=shape, device=dev)
    _dev_tensor(next_pos, "next_pos", torch.int32, shape=(cache.B,), device=dev)
    if score_out is None:
        score_out = torch.empty_like(score)
    if pos_out is None:
        pos_out = torch.empty_like(pos)
    if new_len is None:
        new_len = torch.empty(cache.B, dtype=torch.int32, device=dev)
    _dev_tensor(score_out, "score_out", torch.float32, shape=shape, device=dev)
    _dev_tensor(pos_out, "pos_out", torch.int32, shape=shape, device=dev)
    _dev_tensor(new_len, "new_len", torch.int32, shape=(cache.B,), device=dev)
    if _overlap(score, score_out) or _overlap(pos, pos_out):
        raise ValueError("score_out and pos_out must not overlap score and pos")
    if _overlap(new_len, cache.seq_len) or _overlap(new_len, next_pos):
        raise ValueError("new_len must not overlap the cache's seq_len (copy it there after the call) or next_pos")
    need = _evict_workspace_size(cache.B, cache.n_kv_heads, cap, budget)
    if workspace is None:
        workspace = _workspace(dev, need, "evict", stream)
    st = lib().brisk_cache_evict(cache._ref, cache.B, _ptr(score), _ptr(pos), cap, _ptr(next_pos),
                                 budget, recent, _ptr(score_out), _ptr(pos_out), _ptr(new_len), _ptr(workspace),
                                 _ws_bytes(workspace, dev, need), _stream_ptr(dev, stream))
    _check(st, "brisk_cache_evict")
    return score_out, pos_out, new_len


@functools.lru_cache(maxsize=1024)
def _evict_workspace_size(B: int, n_kv_heads: int, cap: int, budget: int) -> int:
    out = _sz()
    _check(lib().brisk_cache_evict_workspace_size(B, n_kv_heads, cap, budget, ctypes.byref(out)),
           "brisk_cache_evict_workspace_size")
    return out.value


def _overlap(a: torch.Tensor, b: torch.Tensor) -> bool:
    """Whether two contiguous tensors share memory."""
    pa, pb = a.data_ptr(), b.data_ptr()
    return pa < pb + b.numel() * b.element_size() and pb < pa + a.numel() * a.element_size()


def _prob_rows(t: torch.Tensor, name: str, shape: Tuple[int, ...], device: torch.device) -> int:
    """Row stride of fp32 rows [..., V] that may be spaced wider than V."""
    if (type(t) is torch.Tensor and t.dtype is torch.float32 and t.shape == shape and t.device == device
            and t.is_contiguous()):
        return shape[-1]
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != torch.float32:
        raise TypeError(f"{name} must be torch.float32, got {t.dtype}")
    if tuple(t.shape) != shape:
        raise ValueError(f"{name} must have shape {shape}, got {tuple(t.shape)}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the call's other tensors on {device}")
    if shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name} must be contiguous in its last dimension")
    if len(shape) == 2:
        return t.stride(0) if shape[0] > 1 else shape[1]
    if shape[0] > 1 and shape[1] > 1 and t.stride(0) != shape[1] * t.stride(1):
        raise ValueError(f"the rows of {name} must be evenly spaced: stride(0) == {shape[1]} * stride(1)")
    return t.stride(1) if shape[1] > 1 else t.stride(0) if shape[0] > 1 else shape[2]


@functools.lru_cache(maxsize=1024)
def _draft_workspace_size(B: int, V: int) -> int:
    out = _sz()
    _check(lib().brisk_draft_verify_workspace_size(B, V, ctypes.byref(out)), "brisk_draft_verify_workspace_size")
    return out.value


def draft_verify(target_prob: torch.Tensor, draft_prob: torch.Tensor, draft_tok: torch.Tensor, u_accept: torch.Tensor,
                 noise: torch.Tensor, *, draft_len: Optional[torch.Tensor] = None,
                 accept_len: Optional[torch.Tensor] = None, token: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Verifies drafted tokens against given probabilities with given random numbers.

    ``target_prob`` [B, L + 1, V] and ``draft_prob`` [B, L, V] fp32 (rows may be
    padded), ``draft_tok`` [B, L] int32, ``u_accept`` [B, L] uniforms, ``noise``
    [B, V] Exp(1) variates, ``draft_len`` [B] for drafts of different lengths.
    Returns (accept_len [B], token [B]) int32: the accepted prefix of each draft
    and the token after it, drawn from [p - q]_+ after a rejection and from the
    target's next row after a full acceptance (-1 if no weight over its variate is positive)."""
    _dev_tensor(draft_tok, "draft_tok", torch.int32, 2)
    B, L = draft_tok.shape
    dev = draft_tok.device
    if not isinstance(target_prob, torch.Tensor) or target_prob.dim() != 3:
        raise ValueError("target_prob must be a [B, L + 1, V] tensor")
    V = target_prob.shape[2]
    t_stride = _prob_rows(target_prob, "target_prob", (B, L + 1, V), dev)
    d_stride = _prob_rows(draft_prob, "draft_prob", (B, L, V), dev) if L else V
    n_stride = _prob_rows(noise, "noise", (B, V), dev)
    _dev_tensor(u_accept, "u_accept", torch.float32, shape=(B, L), device=dev)
    if draft_len is not None:
        _dev_tensor(draft_len, "draft_len", torch.int32, shape=(B,), device=dev)
    if accept_len is None:
        accept_len = torch.empty(B, dtype=torch.int32, device=dev)
    else:
        _dev_tensor(accept_len, "accept_len", torch.int32, shape=(B,), device=dev)
    if token is None:
        token = torch.empty(B, dtype=torch.int32, device=dev)
    else:
        _dev_tensor(token, "token", torch.int32, shape=(B,), device=dev)
    need = _draft_workspace_size(B, V)
    if workspace is None:
        workspace = _workspace(dev, need, "draft", stream)
    st = lib().brisk_draft_verify(_ptr(target_prob), t_stride, _ptr(draft_prob) if L else None, d_stride,
                                  _ptr(draft_tok) if L else None, _ptr(draft_len), _ptr(u_accept) if L else None,
                                  _ptr(noise), n_stride, B, L, V, _ptr(accept_len), _ptr(token), _ptr(workspace),
                                  _ws_bytes(workspace, dev, need), _stream_ptr(dev, stream))
    _check(st, "brisk_draft_verify")
    return accept_len, token


# ------------------------------------------------------- the cache in 4 bits
@functools.lru_cache(maxsize=1024)
def kv4_page_bytes(page_size: int, d_head: int) -> int:
    """Bytes of a page's part for one head: the last dimension of a :class:`KVCache4`'s pages."""
    out = _sz()
    _check(lib().brisk_kv4_page_bytes(page_size, d_head, ctypes.byref(out)), "brisk_kv4_page_bytes")
    return out.value


class KVCache4:
    """Paged keys and values of a batch of sequences, held in 4 bits.

    ``pages`` is [n_pages, n_kv_heads, kv4_page_bytes(page_size, d_head)] uint8,
    contiguous in its last dimension (pages and heads may lie further apart);
    ``dtype`` (bfloat16 or float16) is that of the keys and values written and
    read and of the queries.  A slot of a head takes 72 bytes up to 64 elements and
    136 beyond, so heads of 16 and 8 take more than in 2 bytes.  ``block_table`` [B, max_pages] int32 lists each
    sequence's pages and ``seq_len`` [B] int32 the slots it holds, the block in
    flight included.  The tensors stay the caller's, as with :class:`KVCache`:
    lengths and pages may be written between calls, which tensors they are is
    fixed."""

    def __init__(self, pages: torch.Tensor, block_table: torch.Tensor, seq_len: torch.Tensor, d_head: int,
                 dtype: torch.dtype = torch.bfloat16):
        if not isinstance(pages, torch.Tensor):
            raise TypeError("pages must be a torch.Tensor")
        if pages.dtype != torch.uint8:
            raise TypeError(f"pages must be torch.uint8, got {pages.dtype}")
        if dtype not in _HALF:
            raise TypeError(f"dtype must be bfloat16 or float16, got {dtype}")
        if pages.dim() != 3:
            raise ValueError(f"pages must have 3 dims, got shape {tuple(pages.shape)}")
        if pages.numel() and pages.stride(-1) != 1:
            raise ValueError("pages must be contiguous in its last dimension")
        if not pages.is_cuda:
            raise ValueError(f"pages must live on a HIP device, got {pages.device}")
        n_pages, self.n_kv_heads, part = pages.shape
        slot = kv4_page_bytes(16, d_head) // 16
        if part % slot or kv4_page_bytes(part // slot, d_head) != part:
            raise ValueError(f"pages of {part} bytes a head hold no whole number of slots of {slot} bytes")
        dev = pages.device
        _dev_tensor(block_table, "block_table", torch.int32, 2, device=dev)
        _dev_tensor(seq_len, "seq_len", torch.int32, shape=(block_table.shape[0],), device=dev)
        self.pages, self.block_table, self.seq_len = pages, block_table, seq_len
        self.device, self.dtype, self.d_head, self.page_size = dev, dtype, d_head, part // slot
        self.B, max_pages = block_table.shape
        self.max_seq_len = max_pages * self.page_size
        self._c = _KVCache4C(_HALF[dtype], self.n_kv_heads, d_head, self.page_size, n_pages, max_pages,
                             *_steps(pages)[:2], _ptr(pages), _ptr(block_table), _ptr(seq_len))
        self._ref = ctypes.byref(self._c)
        self._fixed = True

    def __setattr__(self, name: str, value) -> None:
        if getattr(self, "_fixed", False):
            raise AttributeError(f"{name}: a KVCache4 keeps its tensors; copy into them or make another cache")
        object.__setattr__(self, name, value)

    @property
    def c_struct(self) -> _KVCache4C:
        return self._c


def _cache4(cache) -> None:
    if type(cache) is not KVCache4 and not isinstance(cache, KVCache4):
        raise TypeError(f"cache must be a KVCache4, got {type(cache).__name__}")


def kv4_write(k: torch.Tensor, v: torch.Tensor, cache: KVCache4, first: torch.Tensor, *,
              count: Optional[torch.Tensor] = None, stream=None) -> None:
    """Quantises new tokens into the cache: token t < ``count[b]`` (all T without
    it) of ``k``, ``v`` [B, T, n_kv_heads, d_head] goes to slot ``first[b]`` + t.
    ``k`` and ``v`` may be strided, as columns of a fused projection, by the same
    strides.  ``first`` and ``count`` are [B] int32.  Slots that the table does
    not address are passed over; the cache's ``seq_len`` is neither read nor written."""
    _cache4(cache)
    for t, n in ((k, "k"), (v, "v")):
        _half_tensor(t, n, 4, cache)
    B, T, Hkv, D = k.shape
    if B != cache.B or Hkv != cache.n_kv_heads or D != cache.d_head:
        raise ValueError(f"k is {tuple(k.shape)}, the cache holds {cache.B} sequences of {cache.n_kv_heads} heads of "
                         f"{cache.d_head}")
    if v.shape != k.shape or (v.stride() != k.stride() and _steps(v) != _steps(k)):
        raise ValueError("k and v must agree in shape and strides")
    seq, row, head, _ = _steps(k) if B == 1 or T == 1 or Hkv == 1 else k.stride()
    dev = cache.device
    _dev_tensor(first, "first", torch.int32, shape=(B,), device=dev)
    if count is not None:
        _dev_tensor(count, "count", torch.int32, shape=(B,), device=dev)
    st = lib().brisk_kv4_write(cache._ref, k.data_ptr(), v.data_ptr(), seq, row, head, B, T, first.data_ptr(), _ptr(count),
                               _stream_ptr(dev, stream))
    _check(st, "brisk_kv4_write")


def kv4_read(cache: KVCache4, T: int, *, first: Optional[torch.Tensor] = None, k: Optional[torch.Tensor] = None,
             v: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Keys and values [B, T, n_kv_heads, d_head] as the cache holds them, of slots
    ``first[b]`` (0 without it) to ``first[b]`` + T - 1; zeros for slots that a
    sequence does not hold."""
    _cache4(cache)
    dev, dtype, shape = cache.device, cache.dtype, (cache.B, T, cache.n_kv_heads, cache.d_head)
    if first is not None:
        _dev_tensor(first, "first", torch.int32, shape=(cache.B,), device=dev)
    if k is None:
        k = torch.empty(shape, dtype=dtype, device=dev)
    else:
        _dev_tensor(k, "k", dtype, shape=shape, device=dev)
    if v is None:
        v = torch.empty_like(k)
    else:
        _dev_tensor(v, "v", dtype, shape=shape, device=dev)
    st = lib().brisk_kv4_read(cache._ref, cache.B, T, _ptr(first), k.data_ptr(), v.data_ptr(), _stream_ptr(dev, stream))
    _check(st, "brisk_kv4_read")
    return k, v


def kv4_attention(q: torch.Tensor, cache: KVCache4, *, prefix: Optional[Tuple[torch.Tensor, torch.Tensor]] = None,
                  block_mask: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                  max_seq_len: Optional[int] = None, out: Optional[torch.Tensor] = None,
                  lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None
                  ) -> Tuple[torch.Tensor, torch.Tensor]:
    """:func:`block_attention` over a cache held in 4 bits: the same arguments and
    results; the prefix is in the cache's 2-byte type."""
    _cache4(cache)
    return _attend(lib().brisk_kv4_attention, "brisk_kv4_attention", _kv4_workspace_size, "attention4", q, cache, prefix,
                   block_mask, scale, max_seq_len, out, lse, workspace, stream, _block_queries(q, cache, block_mask))


@functools.lru_cache(maxsize=1024)
def _kv4_workspace_size(B: int, L: int, n_heads: int, n_kv_heads: int, d_head: int, prefix_len: int,
                        max_seq_len: int) -> int:
    out = _sz()
    _check(lib().brisk_kv4_attention_workspace_size(B, L, n_heads, n_kv_heads, d_head, prefix_len, max_seq_len,
                                                    ctypes.byref(out)), "brisk_kv4_attention_workspace_size")
    return out.value
