"""ctypes binding of libnpd (C ABI in ``include/npd.h``): argument marshalling only.

Every function takes torch tensors that already live on the GPU, passes their device pointers and
the current HIP stream to the library, and raises ``NpdError`` on a non-zero status.  There is no
fallback: without the built library these calls fail.
"""
import ctypes
import importlib.util
import os
import warnings
from typing import Optional

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
# NPD_LIB_PATH overrides the in-tree library (e.g. to try a differently tuned build, or an older one: version 118 and later)
LIB_PATH = os.environ.get("NPD_LIB_PATH") or os.path.join(HERE, "libnpd.so")
HOST_PATH = os.path.join(HERE, "npd_host.so")

NPD_TEACHER_DENSE_BF16, NPD_TEACHER_TOPK, NPD_TEACHER_NONE = 0, 1, 2
NPD_FLAG_FWD_ONLY, NPD_FLAG_INPLACE_GRAD, NPD_FLAG_NO_WORKSPACE = 1, 2, 4
NPD_DIV_FORWARD_KL, NPD_DIV_REVERSE_KL, NPD_DIV_SKEW_KL, NPD_DIV_SKEW_REVERSE_KL = 0, 1, 2, 3
NPD_DEV_BAD_LABEL, NPD_DEV_BAD_TOPK_INDEX, NPD_DEV_BAD_CU_SEQLENS, NPD_DEV_GANG_TIMEOUT = 1, 2, 4, 8
NPD_DEV_BAD_SAMPLING, NPD_DEV_BAD_LOGITS = 16, 32
NPD_ZONE_DEGENERATE, NPD_ZONE_PROXIMAL, NPD_ZONE_DISCONNECT, NPD_ZONE_INVALID = 0, 1, 2, 3
NPD_IFD_REQUIRE_TEACHER_LE_1 = 1
NPD_TOPK_LOG_PROBS = 1
NPD_HEAD_GRAD_HIDDEN, NPD_HEAD_GRAD_WEIGHT, NPD_HEAD_GRAD_BIAS, NPD_HEAD_ACCUMULATE, NPD_HEAD_UNALIGNED = 1, 2, 4, 8, 16
NPD_HEAD_LOSS, NPD_HEAD_LOGITS, NPD_HEAD_LOGITS_BWD, NPD_HEAD_LOGITS_INT8 = 0, 1, 2, 3
NPD_NORM_RMS, NPD_NORM_GRAD_X, NPD_NORM_GRAD_WEIGHT, NPD_NORM_GRAD_BIAS, NPD_NORM_ACCUMULATE = 1, 2, 4, 8, 16
NOALLOC_WORKSPACE_BYTES = 16 << 20   # NPD_NOALLOC_WORKSPACE_BYTES

EXPORTS = ("npd_version", "npd_status_string", "npd_workspace_bytes", "npd_kd_loss_fwd_bwd",
           "npd_segment_reduce", "npd_delta_ifd_score", "npd_teacher_topk", "npd_debug_gang_spin_limit",
           "npd_kd_loss_fwd_bwd_noalloc", "npd_policy_lag", "npd_segment_ppl", "npd_kd_kernel_name",
           "npd_forward_scratch_bytes", "npd_kd_loss_forward", "npd_workspace_bytes_preferred",
           "npd_kept_workspace_bytes", "npd_kd_loss_fwd_bwd_kept", "npd_head_workspace_bytes",
           "npd_head_workspace_bytes_preferred", "npd_head_loss_fwd_bwd", "npd_head_logits", "npd_head_logits_bwd",
           "npd_layer_norm", "npd_layer_norm_bwd", "npd_layer_norm_workspace_bytes", "npd_quantize_rows", "npd_head_logits_int8",
           "npd_sample_tokens", "npd_sample_workspace_bytes")


class NpdError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"libnpd status {status}: {message}")
        self.status = status


class KdDesc(ctypes.Structure):
    """Mirror of ``npd_kd_desc``."""
    _fields_ = [("n_tokens", ctypes.c_int64), ("vocab", ctypes.c_int32), ("teacher_kind", ctypes.c_int32),
                ("student_stride", ctypes.c_int64), ("teacher_stride", ctypes.c_int64),
                ("topk", ctypes.c_int32), ("flags", ctypes.c_uint32),
                ("tau", ctypes.c_float), ("grad_scale", ctypes.c_float), ("ce_grad_scale", ctypes.c_float),
                ("divergence", ctypes.c_int32), ("skew_alpha", ctypes.c_float)]


class HeadDesc(ctypes.Structure):
    """Mirror of ``npd_head_desc``."""
    _fields_ = [("n_tokens", ctypes.c_int64), ("vocab", ctypes.c_int32), ("width", ctypes.c_int32),
                ("hidden_stride", ctypes.c_int64), ("weight_stride", ctypes.c_int64),
                ("grad_hidden_stride", ctypes.c_int64), ("grad_weight_stride", ctypes.c_int64),
                ("logits_stride", ctypes.c_int64), ("topk", ctypes.c_int32), ("flags", ctypes.c_uint32),
                ("tau", ctypes.c_float), ("grad_scale", ctypes.c_float), ("ce_grad_scale", ctypes.c_float),
                ("softcap", ctypes.c_float)]


class NormDesc(ctypes.Structure):
    """Mirror of ``npd_norm_desc``."""
    _fields_ = [("n_tokens", ctypes.c_int64), ("x_stride", ctypes.c_int64), ("y_stride", ctypes.c_int64),
                ("grad_x_stride", ctypes.c_int64), ("width", ctypes.c_int32), ("flags", ctypes.c_uint32), ("eps", ctypes.c_float)]


class SampleDesc(ctypes.Structure):
    """Mirror of ``npd_sample_desc``."""
    _fields_ = [("n_tokens", ctypes.c_int64), ("logits_stride", ctypes.c_int64), ("vocab", ctypes.c_int32),
                ("flags", ctypes.c_uint32), ("temperature", ctypes.c_float), ("top_k", ctypes.c_int32),
                ("top_p", ctypes.c_float), ("min_p", ctypes.c_float)]


_lib = None
# native marshalling of the ordinary call (csrc/npd_host.cpp), there once the library is loaded; None without it (the Python
# code below makes every call then).  Its functions return libnpd's status, or -1 for a call that is left to the Python code.
_host = None
_vp = ctypes.c_void_p


def load() -> ctypes.CDLL:
    """Load ``libnpd.so`` (built beforehand by ``paper_2605_05940_amd/build.py``); raises if it is missing."""
    global _lib, _host
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built: run `python -m paper_2605_05940_amd.build` "
                               "(or __graft_entry__.build()) first")
        L = ctypes.CDLL(LIB_PATH)
        L.npd_version.restype = ctypes.c_int
        L.npd_status_string.restype = ctypes.c_char_p
        L.npd_status_string.argtypes = [ctypes.c_int]
        L.npd_debug_gang_spin_limit.restype = ctypes.c_int
        L.npd_debug_gang_spin_limit.argtypes = [ctypes.c_int]
        L.npd_kd_kernel_name.restype = ctypes.c_char_p
        L.npd_kd_kernel_name.argtypes = [ctypes.POINTER(KdDesc)]
        L.npd_workspace_bytes.restype = ctypes.c_size_t
        L.npd_workspace_bytes.argtypes = [ctypes.POINTER(KdDesc)]
        L.npd_kd_loss_fwd_bwd.restype = ctypes.c_int
        L.npd_kd_loss_fwd_bwd.argtypes = [ctypes.POINTER(KdDesc)] + [_vp] * 13 + [ctypes.c_size_t, _vp]
        L.npd_kd_loss_fwd_bwd_noalloc.restype = ctypes.c_int
        L.npd_kd_loss_fwd_bwd_noalloc.argtypes = [ctypes.POINTER(KdDesc)] + [_vp] * 13
        L.npd_segment_reduce.restype = ctypes.c_int
        L.npd_segment_reduce.argtypes = [ctypes.c_int64, ctypes.c_int32] + [_vp] * 9
        L.npd_delta_ifd_score.restype = ctypes.c_int
        L.npd_delta_ifd_score.argtypes = ([ctypes.c_int32, ctypes.c_int32] + [_vp] * 5 +
                                          [ctypes.c_float, ctypes.c_float, ctypes.c_uint32] + [_vp] * 7)
        L.npd_policy_lag.restype = ctypes.c_int
        L.npd_policy_lag.argtypes = [ctypes.c_int64, ctypes.c_int32] + [_vp] * 3 + [ctypes.c_float] + [_vp] * 7
        L.npd_segment_ppl.restype = ctypes.c_int
        L.npd_segment_ppl.argtypes = [ctypes.c_int32] + [_vp] * 4
        L.npd_teacher_topk.restype = ctypes.c_int
        L.npd_teacher_topk.argtypes = ([ctypes.c_int64, ctypes.c_int32, ctypes.c_int64, ctypes.c_int32,
                                        ctypes.c_uint32] + [_vp] * 5)
        # entry points that a library of another build (NPD_LIB_PATH) may not have yet; its calls are made without them, by
        # native code if it has those of the first group
        newer = {"npd_forward_scratch_bytes": (ctypes.c_size_t, []),
                 "npd_workspace_bytes_preferred": (ctypes.c_size_t, []),
                 "npd_kd_loss_forward": (ctypes.c_int, [_vp] * 12 + [ctypes.c_size_t, _vp])}
        newest = {"npd_kept_workspace_bytes": (ctypes.c_size_t, [_vp]),
                  "npd_kd_loss_fwd_bwd_kept": (ctypes.c_int, [_vp] * 13 + [ctypes.c_size_t, _vp])}
        head = {"npd_head_workspace_bytes": (ctypes.c_size_t, [ctypes.c_int]),
                "npd_head_workspace_bytes_preferred": (ctypes.c_size_t, [ctypes.c_int]),
                "npd_head_loss_fwd_bwd": (ctypes.c_int, [_vp] * 15 + [ctypes.c_size_t, _vp]),
                "npd_head_logits": (ctypes.c_int, [_vp] * 5 + [ctypes.c_size_t, _vp]),
                "npd_head_logits_bwd": (ctypes.c_int, [_vp] * 8 + [ctypes.c_size_t, _vp])}
        here = os.path.realpath(LIB_PATH) == os.path.realpath(os.path.join(HERE, "libnpd.so"))
        native = here or all(hasattr(L, name) for name in newer)
        for name, (result, more) in {**newer, **newest}.items():
            if here or hasattr(L, name):
                getattr(L, name).restype = result
                getattr(L, name).argtypes = [ctypes.POINTER(KdDesc)] + more
        for name, (result, more) in head.items():
            if here or hasattr(L, name):
                getattr(L, name).restype = result
                getattr(L, name).argtypes = [ctypes.POINTER(HeadDesc)] + more
        i64, i32, size = ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
        around = {"npd_layer_norm": (ctypes.c_int, [ctypes.POINTER(NormDesc)] + [_vp] * 7),
                  "npd_layer_norm_bwd": (ctypes.c_int, [ctypes.POINTER(NormDesc)] + [_vp] * 9 + [size, _vp]),
                  "npd_layer_norm_workspace_bytes": (size, [ctypes.POINTER(NormDesc)]),
                  "npd_quantize_rows": (ctypes.c_int, [i64, i32, i64, i64] + [_vp] * 4),
                  "npd_head_logits_int8": (ctypes.c_int, [ctypes.POINTER(HeadDesc)] + [_vp] * 7 + [size, _vp]),
                  "npd_sample_tokens": (ctypes.c_int, [ctypes.POINTER(SampleDesc)] + [_vp] * 13 + [size, _vp]),
                  "npd_sample_workspace_bytes": (size, [ctypes.POINTER(SampleDesc)])}
        for name, (result, arguments) in around.items():
            if here or hasattr(L, name):
                getattr(L, name).restype = result
                getattr(L, name).argtypes = arguments
        _host = _load_host(L) if native else None
        _lib = L
    return _lib


def _load_host(L):
    if _raw_stream is None:
        return None
    try:
        spec = importlib.util.spec_from_file_location("npd_host", HOST_PATH)
        host = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(host)
    except (ImportError, OSError) as e:  # not built, or built against another torch
        warnings.warn(f"{HOST_PATH} cannot be loaded ({e}): calls are marshalled by Python code, which is slower; "
                      "`python -m paper_2605_05940_amd.build` builds it", RuntimeWarning)
        return None
    entries = [L.npd_workspace_bytes, L.npd_workspace_bytes_preferred, L.npd_forward_scratch_bytes, L.npd_kd_loss_fwd_bwd,
               L.npd_kd_loss_forward, L.npd_segment_reduce, L.npd_delta_ifd_score, L.npd_teacher_topk, L.npd_policy_lag]
    kept = [getattr(L, name, None) for name in ("npd_kept_workspace_bytes", "npd_kd_loss_fwd_bwd_kept")]
    addresses = [ctypes.cast(f, _vp).value for f in entries + (kept if all(kept) else [])]
    host.bind(_raw_stream, _workspaces, tuple(addresses + [0] * (11 - len(addresses))))
    around = [getattr(L, name, None) for name in (
        "npd_layer_norm", "npd_layer_norm_bwd", "npd_layer_norm_workspace_bytes", "npd_quantize_rows", "npd_head_logits_int8",
        "npd_head_workspace_bytes", "npd_sample_tokens", "npd_sample_workspace_bytes")]
    host.bind_around_head(tuple(ctypes.cast(f, _vp).value for f in around) if all(around) else (0,) * len(around))
    return host


def _check(status: int) -> None:
    if status != 0:
        raise NpdError(status, load().npd_status_string(status).decode())


def _ptr(t: Optional[torch.Tensor], dtype=None):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("libnpd takes device tensors")
    if dtype is not None and t.dtype is not dtype:
        raise ValueError(f"expected {dtype}, got {t.dtype}")
    return t.data_ptr()


def _array(name: str, t: Optional[torch.Tensor], n: int, dtype):
    """Device pointer of a contiguous array of ``n`` elements, None if it is absent."""
    if t is None:
        return None
    if t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous with {n} elements")
    if not t.is_cuda:
        raise ValueError("libnpd takes device tensors")
    if t.dtype is not dtype:
        raise ValueError(f"expected {dtype}, got {t.dtype}")
    return t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def version() -> int:
    return int(load().npd_version())


def _row_stride(x: torch.Tensor) -> int:
    if x.dim() != 2 or x.stride(1) != 1:
        raise ValueError("logits must be 2-D with unit stride along the vocabulary")
    return x.stride(0)


def npd_kd_loss_fwd_bwd(student_logits: torch.Tensor, loss_mask: torch.Tensor, *,
                        teacher_dense: Optional[torch.Tensor] = None,
                        teacher_idx: Optional[torch.Tensor] = None, teacher_val: Optional[torch.Tensor] = None,
                        labels: Optional[torch.Tensor] = None, tau: float = 1.0, grad_scale: float = 1.0,
                        ce_grad_scale: float = 0.0, divergence: int = NPD_DIV_FORWARD_KL, skew_alpha: float = 0.0,
                        grad_out: Optional[torch.Tensor] = None, kd_tok: Optional[torch.Tensor] = None,
                        nll_tok: Optional[torch.Tensor] = None, teacher_nll_tok: Optional[torch.Tensor] = None,
                        lse_tok: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None, no_workspace: bool = False,
                        noalloc: bool = False) -> None:
    """Enqueue the fused KD loss / gradient on the current stream (see ``npd_kd_loss_fwd_bwd`` in npd.h).

    The teacher kind follows from which teacher tensors are given; ``grad_out is None`` means forward
    only; ``grad_out`` sharing storage with ``student_logits`` means the in-place gradient.  ``workspace``:
    a uint8 tensor of at least ``npd_workspace_bytes`` bytes, better of ``npd_workspace_bytes_preferred``.  If it is None the
    native marshalling takes a record that it keeps per device and stream (``npd_kd_loss_fwd_bwd_kept``; eight of 32 MB at
    most, given back by ``release_records``), or for calls that need more a block allocated for the call.  Under capture, and
    where the Python code makes the call, one is taken from ``workspace_for`` (a per-device tensor that this module keeps and
    grows, for calls ordered on one stream) or, with a CE term at tau != 1, for rows that are not 16-byte aligned and for calls
    that prefer more than is kept, allocated for the call; the results are the same.  Forward-only calls allocate a block of
    their own where splitting rows pays (those of up to 512 rows are one launch on such a record), and run without it where
    there is no memory for it.  Blocks of a call go back to torch's allocator when it returns, so a capture that is not
    ``torch.cuda.graph``'s should set ``no_workspace`` (``NPD_FLAG_NO_WORKSPACE``: no scratch memory at all) or bring a
    workspace.  ``noalloc`` calls ``npd_kd_loss_fwd_bwd_noalloc`` instead (the library's built-in scratch array; no workspace
    argument).
    """
    if _host is not None and not noalloc:
        st = _host.kd(student_logits, loss_mask, teacher_dense, teacher_idx, teacher_val, labels, tau, grad_scale,
                      ce_grad_scale, divergence, skew_alpha, grad_out, kd_tok, nll_tok, teacher_nll_tok, lse_tok, dev_status,
                      workspace, no_workspace)
        if st >= 0:
            return _check(st)
    T, V = shape = student_logits.shape
    student_stride, teacher_stride, topk = _row_stride(student_logits), 0, 0
    if teacher_dense is not None:
        kind, teacher_stride = NPD_TEACHER_DENSE_BF16, _row_stride(teacher_dense)
        if teacher_dense.shape != shape:
            raise ValueError("teacher_dense must be [T, V]")
    elif teacher_idx is not None:
        kind, topk = NPD_TEACHER_TOPK, teacher_idx.shape[1]
        if not (teacher_idx.is_contiguous() and teacher_val.is_contiguous() and teacher_val.shape == teacher_idx.shape
                and teacher_idx.shape[0] == T):
            raise ValueError("teacher_idx / teacher_val must be contiguous [T, k]")
    else:
        kind = NPD_TEACHER_NONE
    flags = 0
    if grad_out is None:
        flags |= NPD_FLAG_FWD_ONLY
    else:
        if grad_out.shape != shape or _row_stride(grad_out) != student_stride:
            raise ValueError("grad_out must have the shape and row stride of student_logits")
        if grad_out.data_ptr() == student_logits.data_ptr():
            flags |= NPD_FLAG_INPLACE_GRAD
    if no_workspace:
        flags |= NPD_FLAG_NO_WORKSPACE
    desc = ctypes.byref(KdDesc(T, V, kind, student_stride, teacher_stride, topk, flags, tau, grad_scale, ce_grad_scale,
                               divergence, skew_alpha))
    L = load()
    scratch = None
    if workspace is None and not no_workspace and not noalloc and grad_out is None:
        need = L.npd_forward_scratch_bytes(desc) if hasattr(L, "npd_forward_scratch_bytes") else 0
        if need:  # rows to be split over several workgroups; without the block they are not
            scratch = _own_block(need)
    elif workspace is None and not no_workspace and not noalloc:
        # a CE term at tau != 1 and rows that are not 16-byte aligned: these calls can run without any scratch and may run
        # beside others on several streams, so they share none
        own = ce_grad_scale != 0.0 and tau != 1.0 or (student_logits.data_ptr() | 2 * student_stride) & 15
        workspace = _workspace(L, desc, own, student_logits.device)
    args = (desc, _ptr(student_logits, torch.bfloat16), _ptr(teacher_dense, torch.bfloat16),
            _ptr(teacher_idx, torch.int32), _ptr(teacher_val, torch.float32),
            _array("labels", labels, T, torch.int32), _array("loss_mask", loss_mask, T, torch.uint8),
            _ptr(grad_out, torch.bfloat16), _array("kd_tok", kd_tok, T, torch.float32),
            _array("nll_tok", nll_tok, T, torch.float32), _array("teacher_nll_tok", teacher_nll_tok, T, torch.float32),
            _array("lse_tok", lse_tok, T, torch.float32), _ptr(dev_status, torch.int32))
    if noalloc:
        if workspace is not None:
            raise ValueError("the no-allocation entry point takes no workspace")
        _check(L.npd_kd_loss_fwd_bwd_noalloc(*args, _stream()))
        return
    if scratch is not None:
        _check(L.npd_kd_loss_forward(*args[:7], *args[8:], scratch.data_ptr(), scratch.numel(), _stream()))
        return
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(L.npd_kd_loss_fwd_bwd(*args, _ptr(workspace), ws_bytes, _stream()))


def _own_block(n_bytes: int) -> Optional[torch.Tensor]:
    """Scratch of one call, from torch's stream-ordered allocator (reused only behind this call on its stream: the current
    device's, where the kernels run); None where there is no memory for it."""
    try:
        return torch.empty(n_bytes, dtype=torch.uint8, device="cuda")
    except torch.cuda.OutOfMemoryError:
        return None


_workspaces = {}


def _workspace(L, desc, own: bool, device) -> Optional[torch.Tensor]:
    """The scratch of a gradient call that brings none: as much as it prefers, so that what it runs does not depend on earlier
    calls.  The kept buffer is replaced only by a call that cannot run with it; one that prefers more gets a block."""
    need = L.npd_workspace_bytes(desc)
    if not need:
        return None
    want = getattr(L, "npd_workspace_bytes_preferred", L.npd_workspace_bytes)(desc)
    kept = None if own else _workspaces.get(torch.device(device).index or 0)
    if not own and (kept is None or kept.numel() < need):
        return workspace_for(want, device)
    if kept is not None and kept.numel() >= want:
        return kept
    block = _own_block(want)
    if block is None:
        block = kept if kept is not None else torch.empty(need, dtype=torch.uint8, device="cuda")
    return block


# what a kept buffer holds at least: more than any call of few rows prefers (1,400 slices of 64 bytes and the words behind them)
_KEPT_BYTES = 1 << 17


def workspace_for(n_bytes: int, device) -> Optional[torch.Tensor]:
    """A device buffer of at least ``n_bytes`` bytes (None for 0), kept per device and grown on demand, for callers
    that do not manage the workspace of ``npd_kd_loss_fwd_bwd`` themselves.  Calls that share it must be ordered on
    one stream."""
    if n_bytes == 0:
        return None
    key = torch.device(device).index or 0
    ws = _workspaces.get(key)
    if ws is None or ws.numel() < n_bytes:
        ws = torch.empty(max(n_bytes, _KEPT_BYTES), dtype=torch.uint8, device=device)
        _workspaces[key] = ws
    return ws


def release_records() -> None:
    """Give the scratch records that the native marshalling keeps (one per device and stream, eight of 32 MB at most) back to
    torch's allocator.  Calls that are under way keep theirs; later ones make new ones."""
    if _host is not None:
        _host.release()


def npd_workspace_bytes(n_tokens: int, vocab: int, teacher_kind: int = NPD_TEACHER_DENSE_BF16, topk: int = 0,
                        flags: int = 0, tau: float = 1.0) -> int:
    d = KdDesc()
    d.n_tokens, d.vocab, d.teacher_kind, d.topk, d.flags = n_tokens, vocab, teacher_kind, topk, flags
    d.student_stride = d.teacher_stride = vocab
    d.tau, d.grad_scale, d.ce_grad_scale = tau, 1.0, 0.0
    return int(load().npd_workspace_bytes(ctypes.byref(d)))


def npd_segment_reduce(values: Optional[torch.Tensor], loss_mask: torch.Tensor, cu_seqlens: torch.Tensor, *,
                       seg_sum: Optional[torch.Tensor] = None, seg_count: Optional[torch.Tensor] = None,
                       seg_mean: Optional[torch.Tensor] = None, token_to_sample: Optional[torch.Tensor] = None,
                       dev_status: Optional[torch.Tensor] = None) -> None:
    """Enqueue the per-sample reduction on the current stream (see ``npd_segment_reduce`` in npd.h)."""
    if _host is not None:
        st = _host.segment_reduce(values, loss_mask, cu_seqlens, seg_sum, seg_count, seg_mean, token_to_sample, dev_status)
        if st >= 0:
            return _check(st)
    T = loss_mask.numel()
    S = cu_seqlens.numel() - 1
    _check(load().npd_segment_reduce(
        T, S, _array("values", values, T, torch.float32), _ptr(loss_mask, torch.uint8), _ptr(cu_seqlens, torch.int32),
        _array("seg_sum", seg_sum, S, torch.float32), _array("seg_count", seg_count, S, torch.int32),
        _array("seg_mean", seg_mean, S, torch.float32), _array("token_to_sample", token_to_sample, T, torch.int32),
        _ptr(dev_status, torch.int32), _stream()))


def npd_delta_ifd_score(mean_nll_student: torch.Tensor, mean_nll_teacher: torch.Tensor, seg_count: torch.Tensor,
                        pair_cond: torch.Tensor, pair_uncond: torch.Tensor, lo: float, hi: float, *, flags: int = 0,
                        ifd_student: Optional[torch.Tensor] = None, ifd_teacher: Optional[torch.Tensor] = None,
                        delta: Optional[torch.Tensor] = None, zone: Optional[torch.Tensor] = None,
                        keep: Optional[torch.Tensor] = None, keep_count: Optional[torch.Tensor] = None) -> None:
    """Enqueue the Delta-IFD score on the current stream (see ``npd_delta_ifd_score`` in npd.h)."""
    if _host is not None:
        st = _host.delta_ifd(mean_nll_student, mean_nll_teacher, seg_count, pair_cond, pair_uncond, lo, hi, flags, ifd_student,
                             ifd_teacher, delta, zone, keep, keep_count)
        if st >= 0:
            return _check(st)
    S = mean_nll_student.numel()
    P = pair_cond.numel()
    if mean_nll_teacher.numel() != S or seg_count.numel() != S or pair_uncond.numel() != P:
        raise ValueError("inconsistent sizes")
    for name, t in (("ifd_student", ifd_student), ("ifd_teacher", ifd_teacher), ("delta", delta), ("zone", zone),
                    ("keep", keep)):
        if t is not None and (t.numel() != P or not t.is_contiguous()):
            raise ValueError(f"{name} must be contiguous with {P} elements")
    _check(load().npd_delta_ifd_score(
        P, S, _ptr(mean_nll_student, torch.float32), _ptr(mean_nll_teacher, torch.float32),
        _ptr(seg_count, torch.int32), _ptr(pair_cond, torch.int32), _ptr(pair_uncond, torch.int32),
        lo, hi, flags, _ptr(ifd_student, torch.float32), _ptr(ifd_teacher, torch.float32),
        _ptr(delta, torch.float32), _ptr(zone, torch.uint8), _ptr(keep, torch.uint8),
        _ptr(keep_count, torch.int32), _stream()))


def npd_teacher_topk(teacher_logits: torch.Tensor, k: int, *, topk_idx: torch.Tensor, topk_val: torch.Tensor,
                     loss_mask: Optional[torch.Tensor] = None, log_probs: bool = True) -> None:
    """Enqueue the teacher-side top-k extraction on the current stream (see ``npd_teacher_topk`` in npd.h)."""
    if _host is not None:
        st = _host.teacher_topk(teacher_logits, k, topk_idx, topk_val, loss_mask, log_probs)
        if st >= 0:
            return _check(st)
    T, V = teacher_logits.shape
    for name, t in (("topk_idx", topk_idx), ("topk_val", topk_val)):
        if t.shape != (T, k) or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous [T, k]")
    if loss_mask is not None and (loss_mask.numel() != T or not loss_mask.is_contiguous()):
        raise ValueError("loss_mask must be contiguous with T elements")
    _check(load().npd_teacher_topk(T, V, _row_stride(teacher_logits), k, NPD_TOPK_LOG_PROBS if log_probs else 0,
                                   _ptr(teacher_logits, torch.bfloat16), _ptr(loss_mask, torch.uint8),
                                   _ptr(topk_idx, torch.int32), _ptr(topk_val, torch.float32), _stream()))


def npd_policy_lag(kl_tok: torch.Tensor, loss_mask: torch.Tensor, cu_seqlens: torch.Tensor, epsilon: float = 0.10, *,
                   seg_kl_mean: Optional[torch.Tensor] = None, seg_count: Optional[torch.Tensor] = None,
                   batch_kl_mean: Optional[torch.Tensor] = None, batch_count: Optional[torch.Tensor] = None,
                   lag_exceeded: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None) -> None:
    """Enqueue the policy-latency monitor on the current stream (see ``npd_policy_lag`` in npd.h)."""
    if _host is not None:
        st = _host.policy_lag(kl_tok, loss_mask, cu_seqlens, epsilon, seg_kl_mean, seg_count, batch_kl_mean, batch_count,
                              lag_exceeded, dev_status)
        if st >= 0:
            return _check(st)
    T = loss_mask.numel()
    S = cu_seqlens.numel() - 1
    for name, t, n in (("kl_tok", kl_tok, T), ("seg_kl_mean", seg_kl_mean, S), ("seg_count", seg_count, S),
                       ("batch_kl_mean", batch_kl_mean, 1), ("batch_count", batch_count, 1),
                       ("lag_exceeded", lag_exceeded, 1)):
        if t is not None and (t.numel() != n or not t.is_contiguous()):
            raise ValueError(f"{name} must be contiguous with {n} elements")
    _check(load().npd_policy_lag(
        T, S, _ptr(kl_tok, torch.float32), _ptr(loss_mask, torch.uint8), _ptr(cu_seqlens, torch.int32), epsilon,
        _ptr(seg_kl_mean, torch.float32), _ptr(seg_count, torch.int32), _ptr(batch_kl_mean, torch.float32),
        _ptr(batch_count, torch.int32), _ptr(lag_exceeded, torch.int32), _ptr(dev_status, torch.int32), _stream()))


def npd_segment_ppl(seg_mean_nll: torch.Tensor, seg_count: torch.Tensor, seg_ppl: torch.Tensor) -> None:
    """Enqueue PPL = exp(mean NLL) per sample on the current stream (see ``npd_segment_ppl`` in npd.h)."""
    S = seg_mean_nll.numel()
    if seg_count.numel() != S or seg_ppl.numel() != S:
        raise ValueError("inconsistent sizes")
    _check(load().npd_segment_ppl(S, _ptr(seg_mean_nll, torch.float32), _ptr(seg_count, torch.int32),
                                  _ptr(seg_ppl, torch.float32), _stream()))


# ------------------------------------------------------------------------------------------------------------- the head

def _matrix(name: str, t: Optional[torch.Tensor], shape, dtype=torch.bfloat16):
    """Device pointer of a matrix of ``shape`` with unit stride along its rows (None if it is absent)."""
    if t is None:
        return None
    if t.shape != shape or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be {list(shape)} with unit stride along its rows")
    return _ptr(t, dtype)


def _pitch(t: Optional[torch.Tensor]) -> int:
    """Elements between the rows of a matrix (of one row, where torch keeps any stride: its width)."""
    return 0 if t is None else t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _head_desc(T: int, V: int, D: int, *rest):
    """A descriptor by reference.  Its vocabulary and width are 32 bits wide: what does not fit stays too large to be taken."""
    return ctypes.byref(HeadDesc(T, min(V, 0x7fffffff), min(D, 0x7fffffff), *rest))


def _head_flags(grad_hidden, grad_weight, grad_bias, accumulate, *inputs) -> int:
    return ((NPD_HEAD_GRAD_HIDDEN if grad_hidden is not None else 0) | (NPD_HEAD_GRAD_WEIGHT if grad_weight is not None else 0) |
            (NPD_HEAD_GRAD_BIAS if grad_bias is not None else 0) | (NPD_HEAD_ACCUMULATE if accumulate else 0) |
            (NPD_HEAD_UNALIGNED if any(t is not None and t.data_ptr() & 15 for t in inputs) else 0))


def _head_workspace(L, desc, op: int, workspace: Optional[torch.Tensor]):
    """(pointer, bytes) of a call's workspace: the caller's, or a block from torch's stream-ordered allocator, which it goes
    back to when the call has been enqueued (smaller where there is no memory for what the call prefers)."""
    if workspace is not None:
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        return workspace, _ptr(workspace), workspace.numel() * workspace.element_size()
    want = L.npd_head_workspace_bytes_preferred(desc, op)
    if not want:
        return None, None, 0
    block = _own_block(want)
    if block is None:
        want = L.npd_head_workspace_bytes(desc, op)
        block = torch.empty(want, dtype=torch.uint8, device="cuda")
    return block, block.data_ptr(), want


def npd_head_workspace_bytes(op: int, n_tokens: int, vocab: int, width: int, *, topk: int = 0, flags: int = 0, softcap: float = 0.0,
                             hidden_stride: Optional[int] = None, weight_stride: Optional[int] = None,
                             logits_stride: Optional[int] = None, preferred: bool = False) -> int:
    """Bytes of workspace that a call of a head operator (``op``: ``NPD_HEAD_LOSS``, ``NPD_HEAD_LOGITS``,
    ``NPD_HEAD_LOGITS_BWD`` or ``NPD_HEAD_LOGITS_INT8``) takes: the least, or as many as it can make use of.  ``flags``: ``NPD_HEAD_GRAD_*`` of the gradients
    that it is given, ``NPD_HEAD_UNALIGNED`` where hidden, weight or grad_logits do not begin on 16 bytes (a view; torch's
    allocations do).  Strides are in elements between rows and default to rows without gaps (a matrix of one row has none)."""
    hidden_stride, logits_stride = (hidden_stride, logits_stride) if n_tokens > 1 else (None, None)
    weight_stride = weight_stride if vocab > 1 else None
    grads = flags & (NPD_HEAD_GRAD_HIDDEN | NPD_HEAD_GRAD_WEIGHT | NPD_HEAD_GRAD_BIAS)
    desc = _head_desc(n_tokens, vocab, width, hidden_stride or width, weight_stride or width, width, width, logits_stride or vocab, topk,
                      flags, 1.0, 1.0, 1.0 if grads and not topk else 0.0, softcap)
    L = load()
    return int((L.npd_head_workspace_bytes_preferred if preferred else L.npd_head_workspace_bytes)(desc, op))


def _on_current_device(*tensors: Optional[torch.Tensor]) -> None:
    """Every tensor of a call: the kernels run on the current device, which need not reach another one's memory."""
    current = None
    for t in tensors:
        if t is None or not t.is_cuda:
            continue
        if current is None:
            current = torch.cuda.current_device()
        if t.device.index != current:
            raise ValueError(f"a tensor is on {t.device}, kernels run on the current device: make it current first")


def npd_head_loss_fwd_bwd(hidden: torch.Tensor, weight: torch.Tensor, loss_mask: torch.Tensor, *,
                          bias: Optional[torch.Tensor] = None, softcap: float = 0.0,
                          labels: Optional[torch.Tensor] = None, teacher_idx: Optional[torch.Tensor] = None,
                          teacher_val: Optional[torch.Tensor] = None, tau: float = 1.0, grad_scale: float = 1.0,
                          ce_grad_scale: float = 0.0, grad_hidden: Optional[torch.Tensor] = None,
                          grad_weight: Optional[torch.Tensor] = None, grad_bias: Optional[torch.Tensor] = None,
                          accumulate: bool = False, kd_tok: Optional[torch.Tensor] = None,
                          nll_tok: Optional[torch.Tensor] = None, lse_tok: Optional[torch.Tensor] = None,
                          dev_status: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> None:
    """Enqueue the loss of ``npd_kd_loss_fwd_bwd`` on logits ``hidden @ weight.T + bias`` that are not stored, with the
    gradients that are given a tensor (see ``npd_head_loss_fwd_bwd`` in npd.h); with none of them the call is forward only.
    ``accumulate``: the gradients of weight and bias are added to what their tensors hold.  ``workspace``: a uint8 tensor of
    at least ``npd_head_workspace_bytes(NPD_HEAD_LOSS, ...)`` bytes; without it the call takes a block from torch's allocator
    for as long as it is being enqueued.
    """
    T, D = hidden.shape
    V = weight.shape[0]
    k = 0
    if teacher_idx is not None:
        k = min(teacher_idx.shape[1], 0x7fffffff) if teacher_idx.dim() == 2 else 0
        if teacher_val is None or k == 0 or not (
                teacher_idx.is_contiguous() and teacher_val.is_contiguous() and teacher_val.shape == teacher_idx.shape
                and teacher_idx.shape[0] == T):
            raise ValueError("teacher_idx / teacher_val must be contiguous [T, k]")
    _on_current_device(hidden, weight, loss_mask, bias, labels, teacher_idx, teacher_val, grad_hidden, grad_weight, grad_bias, kd_tok,
                       nll_tok, lse_tok, dev_status, workspace)
    desc = _head_desc(T, V, D, _pitch(hidden), _pitch(weight), _pitch(grad_hidden), _pitch(grad_weight), 0, k,
                      _head_flags(grad_hidden, grad_weight, grad_bias, accumulate, hidden, weight), tau, grad_scale, ce_grad_scale, softcap)
    args = (desc, _matrix("hidden", hidden, (T, D)), _matrix("weight", weight, (V, D)),
            _array("bias", bias, V, torch.bfloat16), _array("labels", labels, T, torch.int32),
            _ptr(teacher_idx, torch.int32), _ptr(teacher_val, torch.float32),
            _array("loss_mask", loss_mask, T, torch.uint8), _matrix("grad_hidden", grad_hidden, (T, D)),
            _matrix("grad_weight", grad_weight, (V, D)), _array("grad_bias", grad_bias, V, torch.bfloat16),
            _array("kd_tok", kd_tok, T, torch.float32), _array("nll_tok", nll_tok, T, torch.float32),
            _array("lse_tok", lse_tok, T, torch.float32), _array("dev_status", dev_status, 1, torch.int32))
    L = load()
    _block, ws, n = _head_workspace(L, desc, NPD_HEAD_LOSS, workspace)
    _check(L.npd_head_loss_fwd_bwd(*args, ws, n, _stream()))


def npd_head_logits(hidden: torch.Tensor, weight: torch.Tensor, *, logits_out: torch.Tensor,
                    bias: Optional[torch.Tensor] = None, softcap: float = 0.0,
                    workspace: Optional[torch.Tensor] = None) -> None:
    """Enqueue ``logits_out = hidden @ weight.T + bias``, soft-capped, rounded to bf16 once (see ``npd_head_logits`` in npd.h)."""
    T, D = hidden.shape
    V = weight.shape[0]
    _on_current_device(hidden, weight, logits_out, bias, workspace)
    desc = _head_desc(T, V, D, _pitch(hidden), _pitch(weight), 0, 0, _pitch(logits_out), 0,
                      _head_flags(None, None, None, False, hidden, weight), 1.0, 0.0, 0.0, softcap)
    args = (desc, _matrix("hidden", hidden, (T, D)), _matrix("weight", weight, (V, D)),
            _array("bias", bias, V, torch.bfloat16), _matrix("logits_out", logits_out, (T, V)))
    L = load()
    _block, ws, n = _head_workspace(L, desc, NPD_HEAD_LOGITS, workspace)
    _check(L.npd_head_logits(*args, ws, n, _stream()))


def npd_head_logits_bwd(grad_logits: torch.Tensor, hidden: torch.Tensor, weight: torch.Tensor, *,
                        logits: Optional[torch.Tensor] = None, softcap: float = 0.0,
                        grad_hidden: Optional[torch.Tensor] = None, grad_weight: Optional[torch.Tensor] = None,
                        grad_bias: Optional[torch.Tensor] = None, accumulate: bool = False,
                        workspace: Optional[torch.Tensor] = None) -> None:
    """Enqueue the backward pass of ``npd_head_logits`` from the bf16 gradient of its logits (see ``npd_head_logits_bwd`` in
    npd.h); ``logits`` are its outputs, needed with a soft cap (and ignored without)."""
    T, D = hidden.shape
    V = weight.shape[0]
    if softcap == 0.0:
        logits = None
    elif logits is not None and logits.shape == grad_logits.shape and _pitch(logits) != _pitch(grad_logits):
        raise ValueError("logits must have the row stride of grad_logits")
    _on_current_device(grad_logits, hidden, weight, logits, grad_hidden, grad_weight, grad_bias, workspace)
    desc = _head_desc(T, V, D, _pitch(hidden), _pitch(weight), _pitch(grad_hidden), _pitch(grad_weight), _pitch(grad_logits), 0,
                      _head_flags(grad_hidden, grad_weight, grad_bias, accumulate, grad_logits, hidden, weight), 1.0, 0.0, 0.0, softcap)
    args = (desc, _matrix("grad_logits", grad_logits, (T, V)), _matrix("logits", logits, (T, V)),
            _matrix("hidden", hidden, (T, D)), _matrix("weight", weight, (V, D)),
            _matrix("grad_hidden", grad_hidden, (T, D)), _matrix("grad_weight", grad_weight, (V, D)),
            _array("grad_bias", grad_bias, V, torch.bfloat16))
    L = load()
    _block, ws, n = _head_workspace(L, desc, NPD_HEAD_LOGITS_BWD, workspace)
    _check(L.npd_head_logits_bwd(*args, ws, n, _stream()))


# ------------------------------------------------------------------------------------------------- on either side of the head

def _width32(n: int) -> int:
    """A size for a field of 32 bits: what does not fit stays too large to be taken."""
    return min(n, 0x7fffffff)


def npd_layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, *, y_out: torch.Tensor,
                   bias: Optional[torch.Tensor] = None, eps: float = 1e-5, rms: bool = False,
                   mean_out: Optional[torch.Tensor] = None, rstd_out: Optional[torch.Tensor] = None) -> None:
    """Enqueue ``y_out = (x - mean) * rstd * weight + bias`` of every row of a bf16 matrix (``rms``: without the mean), and the
    row statistics that the backward pass takes (see ``npd_layer_norm`` in npd.h)."""
    if _host is not None:
        st = _host.layer_norm(x, weight, y_out, bias, eps, rms, mean_out, rstd_out)
        if st >= 0:
            return _check(st)
    T, D = x.shape
    _on_current_device(x, weight, bias, y_out, mean_out, rstd_out)
    desc = NormDesc(T, _pitch(x), _pitch(y_out), 0, _width32(D), NPD_NORM_RMS if rms else 0, eps)
    _check(load().npd_layer_norm(
        ctypes.byref(desc), _matrix("x", x, (T, D)), _array("weight", weight, D, torch.bfloat16), _array("bias", bias, D, torch.bfloat16),
        _matrix("y_out", y_out, (T, D)), _array("mean_out", mean_out, T, torch.float32), _array("rstd_out", rstd_out, T, torch.float32),
        _stream()))


def _norm_grad_desc(T, D, strides, rms, grad_x, grad_weight, grad_bias, accumulate):
    flags = ((NPD_NORM_RMS if rms else 0) | (NPD_NORM_GRAD_X if grad_x else 0) | (NPD_NORM_GRAD_WEIGHT if grad_weight else 0) |
             (NPD_NORM_GRAD_BIAS if grad_bias else 0) | (NPD_NORM_ACCUMULATE if accumulate else 0))
    return NormDesc(T, *strides, _width32(D), flags, 0.0)


def npd_layer_norm_workspace_bytes(n_tokens: int, width: int, *, grad_weight: bool = True, grad_bias: bool = False) -> int:
    """Bytes of workspace that ``npd_layer_norm_bwd`` takes for the gradients of the norm's parameters that it is asked for."""
    if not (grad_weight or grad_bias):
        return 0
    desc = _norm_grad_desc(n_tokens, width, (width, width, width), False, False, grad_weight, grad_bias, False)
    return int(load().npd_layer_norm_workspace_bytes(ctypes.byref(desc)))


def npd_layer_norm_bwd(grad_y: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor] = None, *, rstd: torch.Tensor,
                       mean: Optional[torch.Tensor] = None, rms: bool = False, grad_x: Optional[torch.Tensor] = None,
                       grad_weight: Optional[torch.Tensor] = None, grad_bias: Optional[torch.Tensor] = None,
                       accumulate: bool = False, workspace: Optional[torch.Tensor] = None) -> None:
    """Enqueue the backward pass of ``npd_layer_norm`` from the statistics that it left, for the gradients that are given a tensor
    (see ``npd_layer_norm_bwd`` in npd.h).  ``accumulate``: the gradients of weight and bias are added to what their tensors
    hold.  ``workspace``: a uint8 tensor of at least ``npd_layer_norm_workspace_bytes`` bytes; without it the call takes a block
    from torch's allocator for as long as it is being enqueued."""
    if _host is not None:
        st = _host.layer_norm_bwd(grad_y, x, weight, rstd, mean, rms, grad_x, grad_weight, grad_bias, accumulate, workspace)
        if st >= 0:
            return _check(st)
    T, D = x.shape
    _on_current_device(grad_y, x, weight, rstd, mean, grad_x, grad_weight, grad_bias, workspace)
    desc = _norm_grad_desc(T, D, (_pitch(x), _pitch(grad_y), _pitch(grad_x)), rms, grad_x is not None, grad_weight is not None,
                           grad_bias is not None, accumulate)
    args = (_matrix("grad_y", grad_y, (T, D)), _matrix("x", x, (T, D)), _array("weight", weight, D, torch.bfloat16),
            _array("mean", mean, T, torch.float32), _array("rstd", rstd, T, torch.float32), _matrix("grad_x", grad_x, (T, D)),
            _array("grad_weight", grad_weight, D, torch.bfloat16), _array("grad_bias", grad_bias, D, torch.bfloat16))
    L = load()
    ref = ctypes.byref(desc)
    _block, ws, n = _given_or_own(workspace, lambda: L.npd_layer_norm_workspace_bytes(ref))
    _check(L.npd_layer_norm_bwd(ref, *args, ws, n, _stream()))


def _given_or_own(workspace: Optional[torch.Tensor], bytes_of):
    """(tensor, pointer, bytes) of a call's workspace: the caller's, or a block from torch's stream-ordered allocator."""
    if workspace is not None:
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        return workspace, _ptr(workspace), workspace.numel() * workspace.element_size()
    want = bytes_of()
    if not want:
        return None, None, 0
    block = torch.empty(want, dtype=torch.uint8, device="cuda")
    return block, block.data_ptr(), want


def npd_quantize_rows(x: torch.Tensor, *, q_out: torch.Tensor, scale_out: torch.Tensor) -> None:
    """Enqueue ``scale_out = max|x| / 127`` and ``q_out = round(x / scale_out)`` of every row of a bf16 matrix, as 8-bit integers
    (see ``npd_quantize_rows`` in npd.h).  ``npd_head_logits_int8`` copies rows of a width or stride that is no multiple of 16, in
    calls of more than 64 positions.  It reads them as they are if they are laid out in rows of the next multiple, zeros behind the
    width (``q_out`` is the view without these), and it is given those whole rows: zeros add nothing to a sum."""
    if _host is not None:
        st = _host.quantize_rows(x, q_out, scale_out)
        if st >= 0:
            return _check(st)
    R, D = x.shape
    _on_current_device(x, q_out, scale_out)
    _check(load().npd_quantize_rows(R, _width32(D), _pitch(x), _pitch(q_out), _matrix("x", x, (R, D)),
                                    _matrix("q_out", q_out, (R, D), torch.int8), _array("scale_out", scale_out, R, torch.float32),
                                    _stream()))


def npd_head_logits_int8(hidden: torch.Tensor, hidden_scale: torch.Tensor, weight: torch.Tensor, weight_scale: torch.Tensor, *,
                         logits_out: torch.Tensor, bias: Optional[torch.Tensor] = None, softcap: float = 0.0,
                         workspace: Optional[torch.Tensor] = None) -> None:
    """Enqueue ``npd_head_logits`` of 8-bit hidden states and weights with a scale for each of their rows (see
    ``npd_head_logits_int8`` in npd.h)."""
    if _host is not None:
        st = _host.head_logits_int8(hidden, hidden_scale, weight, weight_scale, logits_out, bias, softcap, workspace)
        if st >= 0:
            return _check(st)
    T, D = hidden.shape
    V = weight.shape[0]
    _on_current_device(hidden, hidden_scale, weight, weight_scale, logits_out, bias, workspace)
    desc = _head_desc(T, V, D, _pitch(hidden), _pitch(weight), 0, 0, _pitch(logits_out), 0,
                      _head_flags(None, None, None, False, hidden, weight), 1.0, 0.0, 0.0, softcap)
    args = (desc, _matrix("hidden", hidden, (T, D), torch.int8), _array("hidden_scale", hidden_scale, T, torch.float32),
            _matrix("weight", weight, (V, D), torch.int8), _array("weight_scale", weight_scale, V, torch.float32),
            _array("bias", bias, V, torch.bfloat16), _matrix("logits_out", logits_out, (T, V)))
    L = load()
    _block, ws, n = _given_or_own(workspace, lambda: L.npd_head_workspace_bytes(desc, NPD_HEAD_LOGITS_INT8))
    _check(L.npd_head_logits_int8(*args, ws, n, _stream()))


def npd_sample_workspace_bytes(n_tokens: int, vocab: int) -> int:
    """Bytes of workspace with which ``npd_sample_tokens`` shares the rows of a call of few among several workgroups (0: it does not)."""
    return int(load().npd_sample_workspace_bytes(ctypes.byref(SampleDesc(n_tokens, _width32(vocab), _width32(vocab), 0, 1.0, 0, 1.0, 0.0))))


def npd_sample_tokens(logits: torch.Tensor, uniform: torch.Tensor, *, tokens_out: torch.Tensor, temperature=1.0, top_k=0,
                      top_p=1.0, min_p=0.0, loss_mask: Optional[torch.Tensor] = None, logprob_out: Optional[torch.Tensor] = None,
                      nll_out: Optional[torch.Tensor] = None, kept_out: Optional[torch.Tensor] = None,
                      dev_status: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> None:
    """Enqueue the drawing of a token from every row of bf16 logits by the random numbers ``uniform`` in [0, 1) (see
    ``npd_sample_tokens`` in npd.h).  ``temperature``, ``top_p``, ``min_p`` (numbers, or fp32 tensors of one per row) and ``top_k``
    (int32) truncate the distribution; 0 or None for no ``top_k``, 1 for no ``top_p``, 0 for no ``min_p``, temperature 0 for the largest
    logit.  ``workspace``: a uint8 tensor (``npd_sample_workspace_bytes``; a smaller one is not used); without it the call takes a block
    from torch's allocator for as long as it is being enqueued."""
    top_k = 0 if top_k is None else top_k
    if _host is not None:
        st = _host.sample_tokens(logits, uniform, tokens_out, temperature, top_k, top_p, min_p, loss_mask, logprob_out, nll_out, kept_out,
                                 dev_status, workspace)
        if st >= 0:
            return _check(st)
    T, V = logits.shape
    settings = (temperature, top_k, top_p, min_p)
    rows = [s if isinstance(s, torch.Tensor) else None for s in settings]
    numbers = [n if r is None else 0 for n, r in zip(settings, rows)]
    _on_current_device(logits, uniform, tokens_out, *rows, loss_mask, logprob_out, nll_out, kept_out, dev_status, workspace)
    desc = ctypes.byref(SampleDesc(T, _pitch(logits), _width32(V), 0, numbers[0], max(-1, _width32(numbers[1])), numbers[2], numbers[3]))
    f32, i32 = torch.float32, torch.int32
    args = (desc, _matrix("logits", logits, (T, V)), _array("uniform", uniform, T, f32),
            _array("loss_mask", loss_mask, T, torch.uint8), _array("temperature", rows[0], T, f32), _array("top_k", rows[1], T, i32),
            _array("top_p", rows[2], T, f32), _array("min_p", rows[3], T, f32), _array("tokens_out", tokens_out, T, i32),
            _array("logprob_out", logprob_out, T, f32), _array("nll_out", nll_out, T, f32), _array("kept_out", kept_out, T, i32),
            _array("dev_status", dev_status, 1, i32))
    L = load()
    _block, ws, n = _given_or_own(workspace, lambda: L.npd_sample_workspace_bytes(desc))
    _check(L.npd_sample_tokens(*args, ws, n, _stream()))
