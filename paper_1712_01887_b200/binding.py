"""Thin ctypes binding of the C ABI in include/dgc.h: argument marshalling only.

Every step of the path runs in the CUDA library; there is no CPU fallback.
Importing this module without the built library raises ImportError.
PyTorch supplies device memory and streams: tensors are passed as raw device
pointers, `stream` arguments default to torch's current stream.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import struct
from typing import Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdgc.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_1712_01887_b200.build` "
        "(there is no CPU fallback)")

_lib = ctypes.CDLL(LIB_PATH)

OK, EINVAL, ENOMEM, ECAPACITY, ECUDA, ESTATE = 0, -1, -2, -3, -4, -5
FLAG_NONFINITE_NORM, FLAG_FULL_SELECT, FLAG_CAND_OVERFLOW, FLAG_CAND_SHORT = 1, 2, 4, 8
FLAG_TIE_FILL = 16
ARENA_ALIGN = 512
MAX_DECODE_WORKERS = 64


class Config(ctypes.Structure):
    _fields_ = [("num_tensors", ctypes.c_int32), ("num_workers", ctypes.c_int32),
                ("tensor_numel", ctypes.POINTER(ctypes.c_int64)), ("momentum", ctypes.c_float),
                ("clip_threshold", ctypes.c_float), ("sparsity", ctypes.c_double),
                ("sample_ratio", ctypes.c_double), ("seed", ctypes.c_uint64),
                ("device", ctypes.c_int32), ("debug_sample_rank", ctypes.c_int32),
                ("nesterov", ctypes.c_int32), ("select_mode", ctypes.c_int32),
                ("clip_scope", ctypes.c_int32)]


class Status(ctypes.Structure):
    _fields_ = [("grad_norm", ctypes.c_double), ("clip_coef", ctypes.c_float),
                ("flags", ctypes.c_int32), ("iterations", ctypes.c_int64),
                ("full_select_last", ctypes.c_int64), ("candidates_last", ctypes.c_int64)]


_vp = ctypes.c_void_p
_i64p = ctypes.POINTER(ctypes.c_int64)
_sigs = {
    "dgc_state_create": (ctypes.c_int32, [ctypes.POINTER(Config), ctypes.POINTER(_vp)]),
    "dgc_state_destroy": (ctypes.c_int32, [_vp]),
    "dgc_set_sparsity": (ctypes.c_int32, [_vp, ctypes.c_double]),
    "dgc_warmup_sparsity": (ctypes.c_int32, [ctypes.c_int32, ctypes.POINTER(ctypes.c_double)]),
    "dgc_max_nnz": (ctypes.c_int64, [_vp]),
    "dgc_layout": (ctypes.c_int32, [_vp, _i64p, _i64p, _i64p, _i64p]),
    "dgc_compress": (ctypes.c_int32, [_vp, _vp, _vp, _vp, ctypes.c_int64, _vp]),
    "dgc_compress_batch": (ctypes.c_int32, [ctypes.c_int32, ctypes.POINTER(_vp),
                                            ctypes.POINTER(_vp), ctypes.POINTER(_vp),
                                            ctypes.POINTER(_vp), _i64p, _vp]),
    "dgc_compress_host": (ctypes.c_int32, [_vp, _vp, _vp, _vp, ctypes.c_int64, _vp]),
    "dgc_compress_host_batch": (ctypes.c_int32, [ctypes.c_int32, ctypes.POINTER(_vp),
                                                 ctypes.POINTER(_vp), ctypes.POINTER(_vp),
                                                 ctypes.POINTER(_vp), _i64p, _vp]),
    "dgc_decode_accumulate": (ctypes.c_int32, [ctypes.c_int32, ctypes.POINTER(_vp),
                                               ctypes.POINTER(_vp), _i64p, _vp, ctypes.c_int64,
                                               _vp, ctypes.c_int64, _vp]),
    "dgc_decode_workspace_bytes": (ctypes.c_int64, [ctypes.c_int32, ctypes.c_int64]),
    "dgc_decode_accumulate_static": (ctypes.c_int32, [ctypes.c_int32, ctypes.POINTER(_vp),
                                                      ctypes.POINTER(_vp), _i64p, _vp,
                                                      ctypes.c_int64, _vp]),
    "dgc_decode_rejected": (ctypes.c_int32, [ctypes.c_int32, ctypes.c_int64, _vp, _vp, _i64p]),
    "dgc_apply_sgd": (ctypes.c_int32, [_vp, _vp, ctypes.c_int64, ctypes.c_float, _vp]),
    "dgc_decode_accumulate_sgd": (ctypes.c_int32, [ctypes.c_int32, ctypes.POINTER(_vp),
                                                   ctypes.POINTER(_vp), _i64p, _vp, _vp,
                                                   ctypes.c_int64, ctypes.c_float, _vp,
                                                   ctypes.c_int64, _vp]),
    "dgc_decode_apply_sgd": (ctypes.c_int32, [ctypes.c_int32, ctypes.POINTER(_vp),
                                              ctypes.POINTER(_vp), _i64p, _vp, ctypes.c_int64,
                                              ctypes.c_float, _vp, ctypes.c_int64, _vp]),
    "dgc_encode_runlength": (ctypes.c_int32, [_vp, _vp, ctypes.c_int64, _vp, _vp, ctypes.c_int64,
                                              _vp, _vp, ctypes.c_int64, _vp]),
    "dgc_decode_runlength": (ctypes.c_int32, [_vp, _vp, ctypes.c_int64, _vp, _vp, _vp, _vp,
                                              ctypes.c_int64, _vp]),
    "dgc_runlength_max_entries": (ctypes.c_int64, [ctypes.c_int64, ctypes.c_int64]),
    "dgc_runlength_workspace_bytes": (ctypes.c_int64, [ctypes.c_int64]),
    "dgc_get_nnz": (ctypes.c_int32, [_vp, _vp, _i64p, _i64p]),
    "dgc_get_status": (ctypes.c_int32, [_vp, _vp, ctypes.POINTER(Status)]),
    "dgc_get_thresholds": (ctypes.c_int32, [_vp, _vp, _vp, _vp]),
    "dgc_get_clip": (ctypes.c_int32, [_vp, _vp, _vp, _vp]),
    "dgc_state_read": (ctypes.c_int32, [_vp, _vp, _vp, _vp]),
    "dgc_state_write": (ctypes.c_int32, [_vp, _vp, _vp, _vp]),
    "dgc_state_set_iterations": (ctypes.c_int32, [_vp, ctypes.c_int64, _vp]),
    "dgc_timeline_enable": (ctypes.c_int32, [_vp, ctypes.c_int32]),
    "dgc_timeline_read": (ctypes.c_int32, [_vp, _vp, _vp]),
    "dgc_profile_enable": (ctypes.c_int32, [_vp, ctypes.c_int32]),
    "dgc_profile_read": (ctypes.c_int32, [_vp, _vp, ctypes.c_int32,
                                          ctypes.POINTER(ctypes.c_int32)]),
    **{name: (ctypes.c_int32, [ctypes.c_char_p, _vp]) for name in (
        "dgc_gated_scan_forward", "dgc_gated_scan_backward", "dgc_gated_scan_step",
        "dgc_top_logits", "dgc_distill_forward", "dgc_distill_backward", "dgc_distill_loss_grad")},
    "dgc_gated_scan_check": (ctypes.c_int32, [_vp]),
    **{name: (ctypes.c_int32, [ctypes.c_char_p, _vp]) for name in (
        "dgc_decay_attention_forward", "dgc_decay_attention_backward", "dgc_decay_attention_step",
        "dgc_vocab_loss_forward", "dgc_vocab_loss_backward", "dgc_vocab_loss_grad")},
    "dgc_tensor_check": (ctypes.c_int32, [_vp]),
    "dgc_decay_attention_workspace_bytes": (ctypes.c_int64, [ctypes.c_char_p, ctypes.c_int32]),
    "dgc_vocab_loss_workspace_bytes": (ctypes.c_int64, [ctypes.c_char_p, ctypes.c_int32]),
    "dgc_gated_scan_workspace_bytes": (ctypes.c_int64, [ctypes.c_char_p]),
    "dgc_launch_count": (ctypes.c_uint64, []),
    "dgc_error_string": (ctypes.c_char_p, [ctypes.c_int32]),
}
for _name, (_res, _args) in _sigs.items():
    _fn = getattr(_lib, _name)
    _fn.restype = _res
    _fn.argtypes = _args

EXPORTED = tuple(_sigs)


class DgcError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = int(code)
        super().__init__(f"{where}: {_lib.dgc_error_string(int(code)).decode()} ({code})")


def _check(code: int, where: str) -> None:
    if code != OK:
        raise DgcError(code, where)


def _stream(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _dev(t: torch.Tensor, dtype) -> int:
    if not (t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise ValueError(f"expected a contiguous CUDA {dtype} tensor")
    return t.data_ptr()


def warmup_sparsity(stage: int) -> float:
    s = ctypes.c_double()
    _check(_lib.dgc_warmup_sparsity(int(stage), ctypes.byref(s)), "dgc_warmup_sparsity")
    return s.value


def launch_count() -> int:
    return int(_lib.dgc_launch_count())


class State:
    """One worker of Algorithm 4: owns u and v on the device."""

    def __init__(self, tensor_numel: Sequence[int], num_workers: int, momentum: float,
                 clip_threshold: float, sparsity: float, sample_ratio: float = 0.01,
                 seed: int = 0, device: int = 0, debug_sample_rank: int = 0,
                 nesterov: bool = False, select_mode: int = 0, clip_scope: int = 0):
        numel = (ctypes.c_int64 * len(tensor_numel))(*[int(n) for n in tensor_numel])
        cfg = Config(len(tensor_numel), int(num_workers), numel, float(momentum),
                     float(clip_threshold), float(sparsity), float(sample_ratio), int(seed),
                     int(device), int(debug_sample_rank), int(bool(nesterov)), int(select_mode),
                     int(clip_scope))
        self._h = _vp()
        self.num_tensors = len(tensor_numel)
        self.device = int(device)
        _check(_lib.dgc_state_create(ctypes.byref(cfg), ctypes.byref(self._h)), "dgc_state_create")
        self._refresh_layout()

    def _refresh_layout(self) -> None:
        T = self.num_tensors
        off = np.zeros(T, np.int64)
        k = np.zeros(T, np.int64)
        out = np.zeros(T + 1, np.int64)
        alen = ctypes.c_int64()
        _check(_lib.dgc_layout(self._h, off.ctypes.data_as(_i64p), k.ctypes.data_as(_i64p),
                               out.ctypes.data_as(_i64p), ctypes.byref(alen)), "dgc_layout")
        self.arena_offset, self.k, self.out_offset, self.arena_len = off, k, out, int(alen.value)
        self.max_nnz = int(_lib.dgc_max_nnz(self._h))

    def close(self) -> None:
        if self._h:
            _check(_lib.dgc_state_destroy(self._h), "dgc_state_destroy")
            self._h = _vp()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_sparsity(self, sparsity: float) -> None:
        _check(_lib.dgc_set_sparsity(self._h, float(sparsity)), "dgc_set_sparsity")
        self._refresh_layout()

    def compress(self, grad: torch.Tensor, out_idx: torch.Tensor, out_val: torch.Tensor,
                 stream=None) -> None:
        if grad.numel() != self.arena_len:
            raise ValueError("gradient arena has the wrong length")
        cap = min(out_idx.numel(), out_val.numel())
        _check(_lib.dgc_compress(self._h, _dev(grad, torch.float32), _dev(out_idx, torch.int32),
                                 _dev(out_val, torch.float32), cap, _stream(stream)),
               "dgc_compress")

    def compress_host(self, grad: torch.Tensor, out_idx: torch.Tensor, out_val: torch.Tensor,
                      stream=None) -> None:
        for t, dt in ((grad, torch.float32), (out_idx, torch.int32), (out_val, torch.float32)):
            if t.is_cuda or t.dtype != dt or not t.is_contiguous():
                raise ValueError("expected contiguous host tensors")
        if grad.numel() != self.arena_len:
            raise ValueError("gradient arena has the wrong length")
        cap = min(out_idx.numel(), out_val.numel())
        _check(_lib.dgc_compress_host(self._h, grad.data_ptr(), out_idx.data_ptr(),
                                      out_val.data_ptr(), cap, _stream(stream)),
               "dgc_compress_host")

    def status(self, stream=None) -> Status:
        s = Status()
        _check(_lib.dgc_get_status(self._h, _stream(stream), ctypes.byref(s)), "dgc_get_status")
        return s

    def nnz(self, stream=None):
        """(total, per-tensor) entries written by the last compress call."""
        total = ctypes.c_int64()
        per = np.zeros(self.num_tensors, np.int64)
        _check(_lib.dgc_get_nnz(self._h, _stream(stream), ctypes.byref(total),
                                per.ctypes.data_as(_i64p)), "dgc_get_nnz")
        return int(total.value), per

    def thresholds(self, stream=None):
        kth = np.zeros(self.num_tensors, np.uint32)
        cand = np.zeros(self.num_tensors, np.int32)
        _check(_lib.dgc_get_thresholds(self._h, _stream(stream), kth.ctypes.data, cand.ctypes.data),
               "dgc_get_thresholds")
        return kth, cand

    def clip(self, stream=None):
        """(norms float64[T], coefficients float32[T]) of the last compress call's clipping."""
        norms = np.zeros(self.num_tensors, np.float64)
        coefs = np.ones(self.num_tensors, np.float32)
        _check(_lib.dgc_get_clip(self._h, _stream(stream), norms.ctypes.data, coefs.ctypes.data),
               "dgc_get_clip")
        return norms, coefs

    def profile_enable(self, max_calls: int) -> None:
        _check(_lib.dgc_profile_enable(self._h, int(max_calls)), "dgc_profile_enable")

    def profile_read(self, capacity: int) -> np.ndarray:
        """[calls, 5] stage durations in ms: norm, sample, streaming pass, select, emit."""
        ms = np.zeros((max(int(capacity), 1), 5), np.float32)
        n = ctypes.c_int32()
        _check(_lib.dgc_profile_read(self._h, ms.ctypes.data, int(capacity), ctypes.byref(n)),
               "dgc_profile_read")
        return ms[:n.value].copy()

    def read(self, stream=None):
        u = np.empty(self.arena_len, np.float32)
        v = np.empty(self.arena_len, np.float32)
        _check(_lib.dgc_state_read(self._h, u.ctypes.data, v.ctypes.data, _stream(stream)),
               "dgc_state_read")
        return u, v

    def write(self, u: Optional[np.ndarray], v: Optional[np.ndarray], stream=None) -> None:
        for a in (u, v):
            if a is not None and (a.dtype != np.float32 or a.size != self.arena_len
                                  or not a.flags["C_CONTIGUOUS"]):
                raise ValueError("expected contiguous float32 arrays of arena_len")
        _check(_lib.dgc_state_write(self._h, None if u is None else u.ctypes.data,
                                    None if v is None else v.ctypes.data, _stream(stream)),
               "dgc_state_write")

    def timeline_enable(self, on: bool = True) -> None:
        _check(_lib.dgc_timeline_enable(self._h, int(bool(on))), "dgc_timeline_enable")

    def timeline_read(self, stream=None) -> np.ndarray:
        """[4 kernels][first block start, last block start] in ns of the GPU timer."""
        out = np.zeros(8, np.uint64)
        _check(_lib.dgc_timeline_read(self._h, _stream(stream), out.ctypes.data),
               "dgc_timeline_read")
        return out.reshape(4, 2)

    def set_iterations(self, iterations: int, stream=None) -> None:
        _check(_lib.dgc_state_set_iterations(self._h, int(iterations), _stream(stream)),
               "dgc_state_set_iterations")


def compress_batch(states: Sequence["State"], grads: Sequence[torch.Tensor],
                   out_idx: Sequence[torch.Tensor], out_val: Sequence[torch.Tensor],
                   stream=None) -> None:
    """dgc_compress for several workers on one GPU with overlapped kernels (same results)."""
    n = len(states)
    sp = (_vp * n)(*[st._h for st in states])
    gp = (_vp * n)(*[_dev(g, torch.float32) for g in grads])
    ip = (_vp * n)(*[_dev(t, torch.int32) for t in out_idx])
    vp = (_vp * n)(*[_dev(t, torch.float32) for t in out_val])
    cap = (ctypes.c_int64 * n)(*[min(a.numel(), b.numel()) for a, b in zip(out_idx, out_val)])
    for st, g in zip(states, grads):
        if g.numel() != st.arena_len:
            raise ValueError("gradient arena has the wrong length")
    _check(_lib.dgc_compress_batch(n, sp, gp, ip, vp, cap, _stream(stream)), "dgc_compress_batch")


def compress_host_batch(states: Sequence["State"], grads: Sequence[torch.Tensor],
                        out_idx: Sequence[torch.Tensor], out_val: Sequence[torch.Tensor],
                        stream=None) -> None:
    """dgc_compress_host for several workers on one GPU: host gradients in, host lists out,
    the workers' copies and kernels overlapped; the lists are valid on return."""
    n = len(states)
    for st, g, a, b in zip(states, grads, out_idx, out_val):
        for t, dt in ((g, torch.float32), (a, torch.int32), (b, torch.float32)):
            if t.is_cuda or t.dtype != dt or not t.is_contiguous():
                raise ValueError("expected contiguous host tensors")
        if g.numel() != st.arena_len:
            raise ValueError("gradient arena has the wrong length")
    sp = (_vp * n)(*[st._h for st in states])
    gp = (_vp * n)(*[g.data_ptr() for g in grads])
    ip = (_vp * n)(*[t.data_ptr() for t in out_idx])
    vp = (_vp * n)(*[t.data_ptr() for t in out_val])
    cap = (ctypes.c_int64 * n)(*[min(a.numel(), b.numel()) for a, b in zip(out_idx, out_val)])
    _check(_lib.dgc_compress_host_batch(n, sp, gp, ip, vp, cap, _stream(stream)),
           "dgc_compress_host_batch")


def decode_workspace_bytes(num_workers: int, dense_len: int) -> int:
    return int(_lib.dgc_decode_workspace_bytes(int(num_workers), int(dense_len)))


def decode_accumulate(idx_lists: Sequence[torch.Tensor], val_lists: Sequence[torch.Tensor],
                      dense_out: torch.Tensor, workspace: torch.Tensor, stream=None,
                      nnz: Optional[Sequence[int]] = None) -> None:
    n = len(idx_lists)
    ip = (_vp * n)(*[_dev(t, torch.int32) for t in idx_lists])
    vp = (_vp * n)(*[_dev(t, torch.float32) for t in val_lists])
    cnt = (ctypes.c_int64 * n)(*[int(c) for c in (nnz if nnz is not None
                                                  else [t.numel() for t in idx_lists])])
    _check(_lib.dgc_decode_accumulate(n, ip, vp, cnt, _dev(dense_out, torch.float32),
                                      dense_out.numel(), workspace.data_ptr(),
                                      workspace.numel() * workspace.element_size(),
                                      _stream(stream)), "dgc_decode_accumulate")


def decode_rejected(num_workers: int, dense_len: int, workspace: Optional[torch.Tensor] = None,
                    stream=None) -> int:
    """Pairs the last decode call on `workspace` (None: the built-in scratch of the static
    variant) skipped or flagged because their index was out of range or out of order."""
    out = ctypes.c_int64()
    _check(_lib.dgc_decode_rejected(int(num_workers), int(dense_len),
                                    None if workspace is None else workspace.data_ptr(),
                                    _stream(stream), ctypes.byref(out)), "dgc_decode_rejected")
    return int(out.value)


def decode_accumulate_sgd(idx_lists: Sequence[torch.Tensor], val_lists: Sequence[torch.Tensor],
                          dense_out: torch.Tensor, w: torch.Tensor, lr: float,
                          workspace: torch.Tensor, stream=None,
                          nnz: Optional[Sequence[int]] = None) -> None:
    """dense_out <- sum of the workers' lists and w <- w - lr * dense_out in one pass."""
    n = len(idx_lists)
    ip = (_vp * n)(*[_dev(t, torch.int32) for t in idx_lists])
    vp = (_vp * n)(*[_dev(t, torch.float32) for t in val_lists])
    cnt = (ctypes.c_int64 * n)(*[int(c) for c in (nnz if nnz is not None
                                                  else [t.numel() for t in idx_lists])])
    if w.numel() != dense_out.numel():
        raise ValueError("length mismatch")
    _check(_lib.dgc_decode_accumulate_sgd(n, ip, vp, cnt, _dev(dense_out, torch.float32),
                                          _dev(w, torch.float32), w.numel(), float(lr),
                                          workspace.data_ptr(),
                                          workspace.numel() * workspace.element_size(),
                                          _stream(stream)), "dgc_decode_accumulate_sgd")


def decode_apply_sgd(idx_lists: Sequence[torch.Tensor], val_lists: Sequence[torch.Tensor],
                     w: torch.Tensor, lr: float, workspace: torch.Tensor, stream=None,
                     nnz: Optional[Sequence[int]] = None) -> None:
    """w <- w - lr * (sum of the workers' sparse lists), touching only the listed entries."""
    n = len(idx_lists)
    ip = (_vp * n)(*[_dev(t, torch.int32) for t in idx_lists])
    vp = (_vp * n)(*[_dev(t, torch.float32) for t in val_lists])
    cnt = (ctypes.c_int64 * n)(*[int(c) for c in (nnz if nnz is not None
                                                  else [t.numel() for t in idx_lists])])
    _check(_lib.dgc_decode_apply_sgd(n, ip, vp, cnt, _dev(w, torch.float32), w.numel(), float(lr),
                                     workspace.data_ptr(),
                                     workspace.numel() * workspace.element_size(),
                                     _stream(stream)), "dgc_decode_apply_sgd")


def runlength_max_entries(nnz: int, dense_len: int) -> int:
    return int(_lib.dgc_runlength_max_entries(int(nnz), int(dense_len)))


def encode_runlength(idx: torch.Tensor, val: torch.Tensor, dense_len: int, stream=None):
    """Sec. 3.1 encode(): returns (runs uint16, values float32) device tensors trimmed to the
    encoded length (synchronises to read the count)."""
    nnz = idx.numel()
    cap = runlength_max_entries(nnz, dense_len)
    runs = torch.empty(cap, dtype=torch.uint16, device=idx.device)
    values = torch.empty(cap, dtype=torch.float32, device=idx.device)
    count = torch.zeros(1, dtype=torch.int64, device=idx.device)
    ws = torch.empty(max(int(_lib.dgc_runlength_workspace_bytes(nnz)), 8), dtype=torch.uint8,
                     device=idx.device)
    _check(_lib.dgc_encode_runlength(_dev(idx, torch.int32) if nnz else None,
                                     _dev(val, torch.float32) if nnz else None, nnz,
                                     runs.data_ptr(), values.data_ptr(), cap, count.data_ptr(),
                                     ws.data_ptr(), ws.numel(), _stream(stream)),
           "dgc_encode_runlength")
    n = int(count.item())
    return runs[:n], values[:n]


def decode_runlength(runs: torch.Tensor, values: torch.Tensor, stream=None):
    """Inverse of encode_runlength: (idx int32, val float32, dense position after the last entry)."""
    n = runs.numel()
    idx = torch.empty(n, dtype=torch.int32, device=runs.device)
    val = torch.empty(n, dtype=torch.float32, device=runs.device)
    end = torch.zeros(1, dtype=torch.int64, device=runs.device)
    ws = torch.empty(max(int(_lib.dgc_runlength_workspace_bytes(n)), 8), dtype=torch.uint8,
                     device=runs.device)
    if not (runs.is_cuda and runs.dtype == torch.uint16 and runs.is_contiguous()):
        raise ValueError("expected a contiguous CUDA uint16 tensor")
    _check(_lib.dgc_decode_runlength(runs.data_ptr() if n else None,
                                     _dev(values, torch.float32) if n else None, n,
                                     idx.data_ptr(), val.data_ptr(), end.data_ptr(), ws.data_ptr(),
                                     ws.numel(), _stream(stream)), "dgc_decode_runlength")
    return idx, val, int(end.item())


STATIC_DECODE_WORDS = 1 << 18


def decode_accumulate_static(idx_lists: Sequence[torch.Tensor], val_lists: Sequence[torch.Tensor],
                             dense_out: torch.Tensor, stream=None,
                             nnz: Optional[Sequence[int]] = None) -> None:
    """dgc_decode_accumulate without a workspace argument, for callers that may not allocate
    device memory: the scratch is a fixed 1 MiB array inside the library.  Raises DgcError
    (ECAPACITY) when workers x (tiles + 1025) exceeds STATIC_DECODE_WORDS.  Calls on one device
    share that scratch, so do not let two of them overlap on the GPU."""
    n = len(idx_lists)
    ip = (_vp * n)(*[_dev(t, torch.int32) for t in idx_lists])
    vp = (_vp * n)(*[_dev(t, torch.float32) for t in val_lists])
    cnt = (ctypes.c_int64 * n)(*[int(c) for c in (nnz if nnz is not None
                                                  else [t.numel() for t in idx_lists])])
    _check(_lib.dgc_decode_accumulate_static(n, ip, vp, cnt, _dev(dense_out, torch.float32),
                                             dense_out.numel(), _stream(stream)),
           "dgc_decode_accumulate_static")


def apply_sgd(w: torch.Tensor, dense_grad: torch.Tensor, lr: float, stream=None) -> None:
    if w.numel() != dense_grad.numel():
        raise ValueError("length mismatch")
    _check(_lib.dgc_apply_sgd(_dev(w, torch.float32), _dev(dense_grad, torch.float32), w.numel(),
                              float(lr), _stream(stream)), "dgc_apply_sgd")


# ----------------------------------------------------------------- a recurrent model's step
# These calls take a struct; it is packed in one go, a fraction of the time that a ctypes
# structure or as many ctypes arguments take (a step of a serving loop is not much longer).

MAX_TOP = 256
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}   # DGC_F32, DGC_BF16, DGC_F16
SCAN = struct.Struct("@4iqP6P2P6P2PPq")          # dgc_scan (a matrix is a pointer and a 64-bit stride)
SCAN_ONE = struct.Struct("@4i6P2P")              # dgc_scan_one
TOP = struct.Struct("@4iq2P2P")                  # dgc_top
DISTILL = struct.Struct("@4iq2P3P4f3P2P")        # dgc_distill
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else None
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _enqueue(call, name: str, args: bytes, stream, device: int) -> None:
    """Calls on the tensors' device (made current for the call where it is not), with the given
    stream, or the current one of that device."""
    if device != _current_device():
        with torch.cuda.device(device):
            return _enqueue(call, name, args, stream, device)
    if isinstance(stream, torch.cuda.Stream) and stream.device_index != device:
        raise ValueError(f"stream: it is of device {stream.device_index}, the tensors are on device {device}")
    rc = call(args, _raw_stream(device) if stream is None and _raw_stream else _stream(stream))
    if rc:
        _check(rc, name)


def _first(t: torch.Tensor, what: str):
    """A call's first matrix, and what it says of the others: (type code, type, shape, device,
    pointer, row stride)."""
    dt, shape, device = t.dtype, t.shape, t.get_device()
    code = DTYPES.get(dt)
    if code is None or device < 0 or len(shape) != 2:
        raise ValueError(f"{what}: expected a CUDA float32, bfloat16 or float16 matrix")
    ld, one = t.stride()
    if one != 1 and shape[1] > 1:
        raise ValueError(f"{what}: columns must be adjacent in memory")
    return code, dt, shape, device, t.data_ptr(), ld if shape[0] > 1 else max(shape[1], ld)


def _matrix(t: torch.Tensor, dtype, shape, device: int, what: str):
    """(pointer, row stride) of a matrix whose columns are adjacent."""
    if t.dtype is not dtype or t.get_device() != device or t.shape != shape:
        raise ValueError(f"{what}: expected a {dtype} matrix of shape {tuple(shape)} on device {device}")
    ld, one = t.stride()
    if one != 1 and shape[1] > 1:
        raise ValueError(f"{what}: columns must be adjacent in memory")
    return t.data_ptr(), ld if shape[0] > 1 else max(shape[1], ld)


def _vec(t: Optional[torch.Tensor], dtype, numel: int, device: int, what: str) -> int:
    """Pointer of a contiguous tensor of `numel` elements; 0 for None."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.get_device() != device or not t.is_contiguous() or t.numel() != numel:
        raise ValueError(f"{what}: expected a contiguous {dtype} tensor of {numel} elements on device {device}")
    return t.data_ptr()


def _stream_context(stream, device: int):
    """Makes torch allocate from the call's stream.  (An external stream of handle 0 would not be
    the default stream but one of torch's own.)"""
    if stream is None:
        return contextlib.nullcontext()
    if isinstance(stream, torch.cuda.Stream):
        return torch.cuda.stream(stream)
    return torch.cuda.stream(torch.cuda.ExternalStream(int(stream), device=device) if int(stream)
                             else torch.cuda.default_stream(device))


def _scan(call, name: str, args: bytes, tokens: int, num_seqs: int, stream, device: int) -> None:
    """The scan calls, with a workspace where one is of use (asked for long sequences only)."""
    if tokens >= 2048 * num_seqs > 0:
        need = int(_lib.dgc_gated_scan_workspace_bytes(args))
        if need > 0:
            # from the call's own stream: what was freed on another may still be written there
            with _stream_context(stream, device):
                work = torch.empty(need, dtype=torch.uint8, device=f"cuda:{device}")
            args = args[:-16] + struct.pack("@Pq", work.data_ptr(), need)
    _enqueue(call, name, args, stream, device)


def gated_scan_forward(gate: torch.Tensor, x: torch.Tensor, h: torch.Tensor,
                       seq_start: Optional[torch.Tensor] = None, num_seqs: int = 1,
                       h0: Optional[torch.Tensor] = None, h_last: Optional[torch.Tensor] = None,
                       reverse: bool = False, stream=None) -> None:
    """h_t = f_t h_{t-1} + (1 - f_t) x_t, f = sigmoid(gate), over packed sequences: rows
    seq_start[s] .. seq_start[s+1] of the [tokens, channels] matrices (seq_start None: num_seqs
    sequences of equal length).  Writes h, and the last states to h_last."""
    code, dt, shape, dev, zp, zl = _first(gate, "gate")
    n, c = shape
    xp, xl = _matrix(x, dt, shape, dev, "x")
    hp, hl = _matrix(h, dt, shape, dev, "h")
    args = SCAN.pack(code, num_seqs, c, 1 if reverse else 0, n,
                     _vec(seq_start, torch.int32, num_seqs + 1, dev, "seq_start"), zp, zl, xp, xl, hp, hl,
                     _vec(h0, torch.float32, num_seqs * c, dev, "h0"),
                     _vec(h_last, torch.float32, num_seqs * c, dev, "h_last"), 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)
    _scan(_lib.dgc_gated_scan_forward, "dgc_gated_scan_forward", args, n, num_seqs, stream, dev)


def gated_scan_backward(gate: torch.Tensor, x: torch.Tensor, h: torch.Tensor, dh: torch.Tensor,
                        dgate: torch.Tensor, dx: torch.Tensor,
                        seq_start: Optional[torch.Tensor] = None, num_seqs: int = 1,
                        h0: Optional[torch.Tensor] = None, dh_last: Optional[torch.Tensor] = None,
                        dh0: Optional[torch.Tensor] = None, reverse: bool = False,
                        stream=None) -> None:
    """Gradients of gated_scan_forward: writes dgate, dx and dh0 from dh (of h) and dh_last."""
    code, dt, shape, dev, zp, zl = _first(gate, "gate")
    n, c = shape
    xp, xl = _matrix(x, dt, shape, dev, "x")
    hp, hl = _matrix(h, dt, shape, dev, "h")
    dp, dl = _matrix(dh, dt, shape, dev, "dh")
    gp, gl = _matrix(dgate, dt, shape, dev, "dgate")
    yp, yl = _matrix(dx, dt, shape, dev, "dx")
    args = SCAN.pack(code, num_seqs, c, 1 if reverse else 0, n,
                     _vec(seq_start, torch.int32, num_seqs + 1, dev, "seq_start"), zp, zl, xp, xl, hp, hl,
                     _vec(h0, torch.float32, num_seqs * c, dev, "h0"), 0, dp, dl, gp, gl, yp, yl,
                     _vec(dh_last, torch.float32, num_seqs * c, dev, "dh_last"),
                     _vec(dh0, torch.float32, num_seqs * c, dev, "dh0"), 0, 0)
    _scan(_lib.dgc_gated_scan_backward, "dgc_gated_scan_backward", args, n, num_seqs, stream, dev)


def gated_scan_step(gate: torch.Tensor, x: torch.Tensor, state: torch.Tensor, out: torch.Tensor,
                    slots: Optional[torch.Tensor] = None, stream=None) -> None:
    """One token for each row: row slots[r] of `state` (fp32 [slots, channels]) is advanced in
    place and written to out[r]; a slot outside the cache marks an idle row."""
    code, dt, shape, dev, zp, zl = _first(gate, "gate")
    n, c = shape
    xp, xl = _matrix(x, dt, shape, dev, "x")
    op, ol = _matrix(out, dt, shape, dev, "out")
    rows = state.shape[0]
    args = SCAN_ONE.pack(code, n, c, rows, zp, zl, xp, xl, op, ol,
                         _vec(state, torch.float32, rows * c, dev, "state"),
                         _vec(slots, torch.int32, n, dev, "slots"))
    _enqueue(_lib.dgc_gated_scan_step, "dgc_gated_scan_step", args, stream, dev)


def gated_scan_check(stream=None) -> None:
    """Synchronises and raises DgcError if a scan kernel's bounded wait has run out on the current device."""
    _check(_lib.dgc_gated_scan_check(_stream(stream)), "dgc_gated_scan_check")


def top_logits(logits: torch.Tensor, idx: torch.Tensor, val: torch.Tensor, stream=None) -> None:
    """The k largest entries of every row, largest first (idx, val: [rows, k]; the lowest index
    first among equals; -inf is never listed, missing entries are (-1, -inf))."""
    code, dt, shape, dev, lp, ll = _first(logits, "logits")
    n, v = shape
    k = idx.shape[-1]
    args = TOP.pack(code, v, k, 0, n, lp, ll, _vec(idx, torch.int32, n * k, dev, "idx"),
                    _vec(val, torch.float32, n * k, dev, "val"))
    _enqueue(_lib.dgc_top_logits, "dgc_top_logits", args, stream, dev)


def distill_forward(logits: torch.Tensor, idx: torch.Tensor, val: torch.Tensor, loss: torch.Tensor,
                    stats: Optional[torch.Tensor] = None, temperature: float = 1.0,
                    soft_weight: float = 1.0, hard_weight: float = 0.0,
                    labels: Optional[torch.Tensor] = None, stream=None) -> None:
    """loss[r] = soft_weight T^2 KL(teacher's listed distribution || student's) + hard_weight
    cross entropy with labels[r]; stats [rows, 2] is kept for distill_backward."""
    code, dt, shape, dev, lp, ll = _first(logits, "logits")
    n, v = shape
    k = idx.shape[-1]
    args = DISTILL.pack(code, v, k, 0, n, lp, ll, _vec(idx, torch.int32, n * k, dev, "idx"),
                        _vec(val, torch.float32, n * k, dev, "val"),
                        _vec(labels, torch.int32, n, dev, "labels"), temperature, soft_weight,
                        hard_weight, 0.0, _vec(loss, torch.float32, n, dev, "loss"),
                        _vec(stats, torch.float32, 2 * n, dev, "stats"), 0, 0, 0)
    _enqueue(_lib.dgc_distill_forward, "dgc_distill_forward", args, stream, dev)


def distill_backward(logits: torch.Tensor, idx: torch.Tensor, val: torch.Tensor, stats: torch.Tensor,
                     dloss: torch.Tensor, dlogits: torch.Tensor, temperature: float = 1.0,
                     soft_weight: float = 1.0, hard_weight: float = 0.0,
                     labels: Optional[torch.Tensor] = None, stream=None) -> None:
    """The gradient of distill_forward's losses, dloss[r] being that of row r's; dlogits may be
    the logits themselves."""
    code, dt, shape, dev, lp, ll = _first(logits, "logits")
    n, v = shape
    dp, dl = _matrix(dlogits, dt, shape, dev, "dlogits")
    k = idx.shape[-1]
    args = DISTILL.pack(code, v, k, 0, n, lp, ll, _vec(idx, torch.int32, n * k, dev, "idx"),
                        _vec(val, torch.float32, n * k, dev, "val"),
                        _vec(labels, torch.int32, n, dev, "labels"), temperature, soft_weight,
                        hard_weight, 0.0, 0, _vec(stats, torch.float32, 2 * n, dev, "stats"),
                        _vec(dloss, torch.float32, n, dev, "dloss"), dp, dl)
    _enqueue(_lib.dgc_distill_backward, "dgc_distill_backward", args, stream, dev)


def distill_loss_grad(logits: torch.Tensor, idx: torch.Tensor, val: torch.Tensor,
                      dloss: torch.Tensor, loss: torch.Tensor, dlogits: torch.Tensor,
                      temperature: float = 1.0, soft_weight: float = 1.0, hard_weight: float = 0.0,
                      labels: Optional[torch.Tensor] = None, stream=None) -> None:
    """distill_forward and distill_backward in one call, the logits read from memory once."""
    code, dt, shape, dev, lp, ll = _first(logits, "logits")
    n, v = shape
    dp, dl = _matrix(dlogits, dt, shape, dev, "dlogits")
    k = idx.shape[-1]
    args = DISTILL.pack(code, v, k, 0, n, lp, ll, _vec(idx, torch.int32, n * k, dev, "idx"),
                        _vec(val, torch.float32, n * k, dev, "val"),
                        _vec(labels, torch.int32, n, dev, "labels"), temperature, soft_weight,
                        hard_weight, 0.0, _vec(loss, torch.float32, n, dev, "loss"), 0,
                        _vec(dloss, torch.float32, n, dev, "dloss"), dp, dl)
    _enqueue(_lib.dgc_distill_loss_grad, "dgc_distill_loss_grad", args, stream, dev)


# ----------------------------------------------------------------- linear attention, large vocabularies

MAX_HEAD_DIM = 128
ATTENTION = struct.Struct("@5ifq2P" + "P2q" * 4 + "2P" + "P2q" * 4 + "2PPq")   # dgc_attention
ATTENTION_ONE = struct.Struct("@6ifiP" + "P2q" * 4 + "2P")                     # dgc_attention_one
VOCAB_LOSS = struct.Struct("@4iqPqPq5PPqPqPPq")                                # dgc_vocab_loss
_NO_HEADS = (0, 0, 0)


def _heads(t: torch.Tensor, dtype, shape, device: int, what: str):
    """(pointer, strides of tokens and heads) of a [tokens, heads, dim] tensor whose last dimension is adjacent."""
    if t.dtype is not dtype or t.get_device() != device or t.shape != shape:
        raise ValueError(f"{what}: expected a {dtype} tensor of shape {tuple(shape)} on device {device}")
    ld, head, one = t.stride()
    if one != 1 and shape[2] > 1:
        raise ValueError(f"{what}: a head's elements must be adjacent in memory")
    return t.data_ptr(), ld, head


def _first_heads(q: torch.Tensor, v: torch.Tensor):
    """(type code, type, device, shapes of q and k, of v and out)."""
    dt, shape, device = q.dtype, q.shape, q.get_device()
    code = DTYPES.get(dt)
    if code is None or device < 0 or len(shape) != 3:
        raise ValueError("q: expected a CUDA float32, bfloat16 or float16 tensor [tokens, heads, key_dim]")
    if len(v.shape) != 3 or v.shape[:2] != shape[:2]:
        raise ValueError(f"v: expected [{shape[0]}, {shape[1]}, value_dim]")
    return code, dt, device, shape, v.shape


def _work(need: int, stream, device: int):
    """Workspace from the call's own stream: what was freed on another may still be written there."""
    with _stream_context(stream, device):
        return torch.empty(need, dtype=torch.uint8, device=f"cuda:{device}")


def _attend(call, name: str, args: bytes, backward: int, stream, device: int) -> None:
    need = int(_lib.dgc_decay_attention_workspace_bytes(args, backward))
    if need > 0:
        work = _work(need, stream, device)
        args = args[:-16] + struct.pack("@Pq", work.data_ptr(), need)
    _enqueue(call, name, args, stream, device)


def decay_attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, decay: torch.Tensor,
                            seq_start: Optional[torch.Tensor] = None, num_seqs: int = 1,
                            s0: Optional[torch.Tensor] = None, s_last: Optional[torch.Tensor] = None,
                            scale: float = 1.0, stream=None) -> None:
    """S_t = decay S_{t-1} + k_t v_t^T, out_t = scale S_t^T q_t for each head, over packed sequences:
    tokens seq_start[s] .. seq_start[s+1] of the [tokens, heads, dim] tensors (seq_start None: num_seqs
    sequences of equal length).  States are fp32 [num_seqs, heads, key_dim, value_dim]."""
    code, dt, dev, kd, vd = _first_heads(q, v)
    n, h, dk = kd
    dv, states = vd[2], num_seqs * h * dk * vd[2]
    args = ATTENTION.pack(code, num_seqs, h, dk, dv, scale, n, _vec(seq_start, torch.int32, num_seqs + 1, dev, "seq_start"),
                          _vec(decay, torch.float32, h, dev, "decay"), *_heads(q, dt, kd, dev, "q"),
                          *_heads(k, dt, kd, dev, "k"), *_heads(v, dt, vd, dev, "v"), *_heads(out, dt, vd, dev, "out"),
                          _vec(s0, torch.float32, states, dev, "s0"), _vec(s_last, torch.float32, states, dev, "s_last"),
                          *_NO_HEADS, *_NO_HEADS, *_NO_HEADS, *_NO_HEADS, 0, 0, 0, 0)
    _attend(_lib.dgc_decay_attention_forward, "dgc_decay_attention_forward", args, 0, stream, dev)


def decay_attention_backward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, dout: torch.Tensor, dq: torch.Tensor,
                             dk: torch.Tensor, dv: torch.Tensor, decay: torch.Tensor,
                             seq_start: Optional[torch.Tensor] = None, num_seqs: int = 1,
                             s0: Optional[torch.Tensor] = None, ds_last: Optional[torch.Tensor] = None,
                             ds0: Optional[torch.Tensor] = None, scale: float = 1.0, stream=None) -> None:
    """Gradients of decay_attention_forward: writes dq, dk, dv and ds0 from dout and ds_last (each head its
    own: heads that share a tensor add theirs up)."""
    code, dt, dev, kd, vd = _first_heads(q, v)
    n, h, kdim = kd
    states = num_seqs * h * kdim * vd[2]
    args = ATTENTION.pack(code, num_seqs, h, kdim, vd[2], scale, n,
                          _vec(seq_start, torch.int32, num_seqs + 1, dev, "seq_start"),
                          _vec(decay, torch.float32, h, dev, "decay"), *_heads(q, dt, kd, dev, "q"),
                          *_heads(k, dt, kd, dev, "k"), *_heads(v, dt, vd, dev, "v"), *_NO_HEADS,
                          _vec(s0, torch.float32, states, dev, "s0"), 0, *_heads(dout, dt, vd, dev, "dout"),
                          *_heads(dq, dt, kd, dev, "dq"), *_heads(dk, dt, kd, dev, "dk"), *_heads(dv, dt, vd, dev, "dv"),
                          _vec(ds_last, torch.float32, states, dev, "ds_last"),
                          _vec(ds0, torch.float32, states, dev, "ds0"), 0, 0)
    _attend(_lib.dgc_decay_attention_backward, "dgc_decay_attention_backward", args, 1, stream, dev)


def decay_attention_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, state: torch.Tensor, out: torch.Tensor,
                         decay: torch.Tensor, slots: Optional[torch.Tensor] = None, scale: float = 1.0,
                         stream=None) -> None:
    """One token for each row: state number slots[r] of `state` (fp32 [slots, heads, key_dim, value_dim]) is
    advanced in place, out[r] is read from it; a slot outside the cache marks an idle row."""
    code, dt, dev, kd, vd = _first_heads(q, v)
    n, h, dk = kd
    rows = state.shape[0]
    args = ATTENTION_ONE.pack(code, n, h, dk, vd[2], rows, scale, 0, _vec(decay, torch.float32, h, dev, "decay"),
                              *_heads(q, dt, kd, dev, "q"), *_heads(k, dt, kd, dev, "k"), *_heads(v, dt, vd, dev, "v"),
                              *_heads(out, dt, vd, dev, "out"),
                              _vec(state, torch.float32, rows * h * dk * vd[2], dev, "state"),
                              _vec(slots, torch.int32, n, dev, "slots"))
    _enqueue(_lib.dgc_decay_attention_step, "dgc_decay_attention_step", args, stream, dev)


def _vocab_loss(call, name: str, gradient: int, hidden, weight, labels, bias, loss, stats, dloss, dhidden, dweight,
                dbias, stream) -> None:
    code, dt, shape, dev, hp, hl = _first(hidden, "hidden")
    n, d = shape
    v = weight.shape[0]
    wp, wl = _matrix(weight, dt, torch.Size((v, d)), dev, "weight")
    dhp, dhl = _matrix(dhidden, dt, shape, dev, "dhidden") if gradient else (0, 0)
    dwp, dwl = _matrix(dweight, dt, torch.Size((v, d)), dev, "dweight") if gradient else (0, 0)
    args = VOCAB_LOSS.pack(code, v, d, 0, n, hp, hl, wp, wl, _vec(bias, dt, v, dev, "bias"),
                           _vec(labels, torch.int32, n, dev, "labels"), _vec(loss, torch.float32, n, dev, "loss"),
                           _vec(stats, torch.float32, 2 * n, dev, "stats"), _vec(dloss, torch.float32, n, dev, "dloss"),
                           dhp, dhl, dwp, dwl, _vec(dbias, dt, v, dev, "dbias"), 0, 0)
    need = int(_lib.dgc_vocab_loss_workspace_bytes(args, gradient))
    if need > 0:
        work = _work(need, stream, dev)
        args = args[:-16] + struct.pack("@Pq", work.data_ptr(), need)
    _enqueue(call, name, args, stream, dev)


def vocab_loss_forward(hidden: torch.Tensor, weight: torch.Tensor, labels: torch.Tensor, loss: torch.Tensor,
                       stats: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, stream=None) -> None:
    """loss[r] = cross entropy of softmax(hidden[r] weight^T + bias) with labels[r] (0 for a label outside the
    vocabulary: a padding row); the logits are not kept.  stats [rows, 2] is kept for vocab_loss_backward."""
    _vocab_loss(_lib.dgc_vocab_loss_forward, "dgc_vocab_loss_forward", 0, hidden, weight, labels, bias, loss, stats, None,
                None, None, None, stream)


def vocab_loss_backward(hidden: torch.Tensor, weight: torch.Tensor, labels: torch.Tensor, stats: torch.Tensor,
                        dloss: torch.Tensor, dhidden: torch.Tensor, dweight: torch.Tensor,
                        bias: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None, stream=None) -> None:
    """The gradient of vocab_loss_forward's losses, dloss[r] being that of row r's."""
    _vocab_loss(_lib.dgc_vocab_loss_backward, "dgc_vocab_loss_backward", 1, hidden, weight, labels, bias, None, stats, dloss,
                dhidden, dweight, dbias, stream)


def vocab_loss_grad(hidden: torch.Tensor, weight: torch.Tensor, labels: torch.Tensor, dloss: torch.Tensor,
                    loss: torch.Tensor, dhidden: torch.Tensor, dweight: torch.Tensor,
                    bias: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None, stream=None) -> None:
    """vocab_loss_forward and vocab_loss_backward in one call."""
    _vocab_loss(_lib.dgc_vocab_loss_grad, "dgc_vocab_loss_grad", 1, hidden, weight, labels, bias, loss, None, dloss, dhidden,
                dweight, dbias, stream)


def tensor_check(stream=None) -> None:
    """Synchronises and raises DgcError if a bounded wait of a decay_attention or vocab_loss kernel has run out on
    the current device."""
    _check(_lib.dgc_tensor_check(_stream(stream)), "dgc_tensor_check")
