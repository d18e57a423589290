"""ctypes binding of ``libadacomp.so``: argument marshalling only.

Every step of the hot path runs inside the CUDA library; this module checks tensor
dtype / device / contiguity, passes raw pointers and raises :class:`AdacompError`
on a non-zero status.  The function names mirror ``include/adacomp.h``;
:class:`Selector` and :class:`Server` are small conveniences that own the
workspace tensors (PyTorch allocates all device memory).

Importing this module loads the shared library and fails loudly if it has not
been built (``python -m paper_1702_04683_b200.build``).  There is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence, Tuple

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libadacomp.so")

OK, ERR_INVALID, ERR_ALLOC, ERR_CUDA, ERR_WINDOW, ERR_CAPACITY, ERR_UNSORTED, ERR_TIMEOUT, ERR_UNIMPLEMENTED = \
    0, -1, -2, -3, -4, -5, -6, -7, -8


class AdacompError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        text = _lib.adacomp_status_string(status).decode()
        extra = f" (cudaError {_lib.adacomp_last_cuda_error()})" if status == ERR_CUDA else ""
        super().__init__(f"{where}: {text}{extra} [{status}]")


class Segment(ctypes.Structure):
    _fields_ = [("offset", ctypes.c_uint64), ("n", ctypes.c_uint32), ("k", ctypes.c_uint32)]


class GradTensor(ctypes.Structure):
    _fields_ = [("d_grad", ctypes.c_void_p), ("d_out", ctypes.c_void_p), ("n", ctypes.c_uint64),
                ("grad_type", ctypes.c_int32), ("out_type", ctypes.c_int32)]


class Rows(ctypes.Structure):
    _fields_ = [("d_data", ctypes.c_void_p), ("type", ctypes.c_int32), ("group", ctypes.c_uint32),
                ("row_stride", ctypes.c_uint64), ("group_stride", ctypes.c_uint64)]


#: element types of the operators that take more than fp32, and types of token numbers
ELEMENT_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
TOKEN_TYPES = {torch.int32: 0, torch.int64: 1}


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_1702_04683_b200.build` "
            "(nvcc, sm_100a). There is no fallback implementation.")
    L = ctypes.CDLL(LIB_PATH)
    vp, u32, u64, i32, f32 = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_int, ctypes.c_float
    P = ctypes.POINTER
    sig = {
        "adacomp_status_string": (ctypes.c_char_p, [i32]),
        "adacomp_version": (i32, []),
        "adacomp_last_cuda_error": (i32, []),
        "adacomp_kernel_launches": (u64, []),
        "adacomp_keep_count": (i32, [u64, u32, u32, P(u32)]),
        "adacomp_select_workspace_bytes": (i32, [P(Segment), u32, u32, P(ctypes.c_size_t)]),
        "adacomp_select_create": (i32, [P(vp), P(Segment), u32, u32, vp, ctypes.c_size_t, i32]),
        "adacomp_select": (i32, [vp, vp, u64, u32, vp, vp, vp]),
        "adacomp_select_host": (i32, [vp, vp, u64, u32, vp, vp, vp, vp, vp, vp]),
        "adacomp_select_set_route": (i32, [vp, i32]),
        "adacomp_select_route_info": (i32, [vp, P(u32)]),
        "adacomp_select_set_profiling": (i32, [vp, i32]),
        "adacomp_select_profile": (i32, [vp, P(f32), u32, P(u64)]),
        "adacomp_select_stage_name": (ctypes.c_char_p, [u32]),
        "adacomp_select_static": (i32, [vp, u32, u32, vp, vp, i32, vp]),
        "adacomp_select_static_last_error": (i32, [i32, vp]),
        "adacomp_select_pairs_per_worker": (i32, [vp, P(u64)]),
        "adacomp_select_last_error": (i32, [vp, vp, P(u64)]),
        "adacomp_select_destroy": (i32, [vp]),
        "adacomp_server_workspace_bytes": (i32, [u64, u64, P(ctypes.c_size_t)]),
        "adacomp_server_create": (i32, [P(vp), u64, u64, u32, vp, ctypes.c_size_t, i32]),
        "adacomp_server_reset": (i32, [vp, vp, vp]),
        "adacomp_server_pull": (i32, [vp, vp, P(u64), vp]),
        "adacomp_apply": (i32, [vp, vp, vp, P(u64), P(u32), P(u64), u32, f32, vp, vp]),
        "adacomp_apply_host": (i32, [vp, vp, vp, P(u64), P(u32), P(u64), u32, f32, vp, vp, vp, vp, vp]),
        "adacomp_server_timestamp": (i32, [vp, P(u64)]),
        "adacomp_server_set_validation": (i32, [vp, i32]),
        "adacomp_server_set_mode": (i32, [vp, i32]),
        "adacomp_encode_capacity_words": (u64, [u64]),
        "adacomp_encode_indices": (i32, [vp, u64, u32, vp, u64, vp, i32, vp]),
        "adacomp_decode_indices": (i32, [vp, u64, vp, u64, u32, vp, i32, vp]),
        "adacomp_encode_values_capacity_words": (u64, [u64]),
        "adacomp_encode_values": (i32, [vp, u64, u32, vp, u64, vp, i32, vp]),
        "adacomp_decode_values": (i32, [vp, u64, vp, u64, u32, vp, i32, vp]),
        "adacomp_server_set_rule": (i32, [vp, i32]),
        "adacomp_apply_dense": (i32, [vp, vp, u64, f32, vp]),
        "adacomp_select_gather": (i32, [vp, vp, u64, u32, vp, vp, vp]),
        "adacomp_server_debug_skip_positions": (i32, [vp, u64]),
        "adacomp_server_last_error": (i32, [vp, vp]),
        "adacomp_server_destroy": (i32, [vp]),
        "adacomp_clip_workspace_bytes": (i32, [u32, P(ctypes.c_size_t)]),
        "adacomp_clip_create": (i32, [P(vp), u32, vp, ctypes.c_size_t, i32]),
        "adacomp_grad_norm": (i32, [vp, vp, u32, u64, u32, f32, vp, vp]),
        "adacomp_clip": (i32, [vp, vp, u32, u64, u64, u32, f32, f32, vp, vp, vp]),
        "adacomp_clip_destroy": (i32, [vp]),
        "adacomp_embed_workspace_bytes": (i32, [u32, u32, u32, u32, P(ctypes.c_size_t)]),
        "adacomp_embed_create": (i32, [P(vp), u32, u32, u32, u32, u32, vp, ctypes.c_size_t, i32]),
        "adacomp_embed_lookup": (i32, [vp, vp, vp, u32, f32, vp, vp]),
        "adacomp_embed_grad_rows": (i32, [vp, vp, u32, u32, vp, f32, vp, vp, vp, i32, vp, u64, vp]),
        "adacomp_embed_grad_dense": (i32, [vp, vp, u32, u32, vp, f32, vp, i32, vp]),
        "adacomp_embed_set_wait_limit": (i32, [vp, u32]),
        "adacomp_embed_last_error": (i32, [vp, vp]),
        "adacomp_embed_destroy": (i32, [vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    return L, tuple(sig)


_lib, EXPORTS = _load()


def _check(status: int, where: str) -> None:
    if status != OK:
        raise AdacompError(status, where)


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream)


def _dev(t: torch.Tensor, dtype, name: str) -> int:
    if not (t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise TypeError(f"{name}: need a contiguous CUDA tensor of {dtype}")
    return t.data_ptr()


def _host(t: torch.Tensor, dtype, name: str) -> int:
    if t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name}: need a contiguous host tensor of {dtype}")
    return t.data_ptr()


def _u64_array(a) -> np.ndarray:
    return np.ascontiguousarray(a, dtype=np.uint64)


# ----------------------------------------------------------------------------- plain functions

def adacomp_version() -> int:
    return int(_lib.adacomp_version())


def adacomp_kernel_launches() -> int:
    return int(_lib.adacomp_kernel_launches())


def adacomp_status_string(status: int) -> str:
    return _lib.adacomp_status_string(status).decode()


def adacomp_keep_count(n: int, c_num: int, c_den: int) -> int:
    k = ctypes.c_uint32(0)
    _check(_lib.adacomp_keep_count(n, c_num, c_den, ctypes.byref(k)), "adacomp_keep_count")
    return int(k.value)


def make_segments(sizes: Sequence[int], keep: Tuple[int, int], offsets: Optional[Sequence[int]] = None):
    """Segment table for consecutive tensors of the given sizes and a keep fraction (num, den)."""
    segs = (Segment * len(sizes))()
    off = 0
    for l, n in enumerate(sizes):
        segs[l].offset = offsets[l] if offsets is not None else off
        segs[l].n = n
        segs[l].k = adacomp_keep_count(n, keep[0], keep[1])
        off += n
    return segs


def segments_from(offsets: Sequence[int], ns: Sequence[int], ks: Sequence[int]):
    segs = (Segment * len(ns))()
    for l in range(len(ns)):
        segs[l].offset, segs[l].n, segs[l].k = int(offsets[l]), int(ns[l]), int(ks[l])
    return segs


def adacomp_select_static(grad: torch.Tensor, k: int, idx_out: torch.Tensor, val_out: torch.Tensor,
                          stream: Optional[torch.cuda.Stream] = None) -> None:
    """Top-k-by-magnitude of one tensor through the entry point that allocates nothing: the caller
    brings the input and both outputs, the scratch is a fixed array inside the library."""
    if not (grad.is_cuda and grad.dtype == torch.float32 and grad.dim() == 1 and grad.stride(0) == 1):
        raise TypeError("grad: need a 1-D contiguous CUDA fp32 tensor")
    _check(_lib.adacomp_select_static(grad.data_ptr(), grad.numel(), int(k), _dev(idx_out, torch.int32, "idx_out"),
                                      _dev(val_out, torch.float32, "val_out"), grad.device.index,
                                      _stream_ptr(stream)), "adacomp_select_static")


def adacomp_select_static_last_error(device_index: int = 0, stream: Optional[torch.cuda.Stream] = None) -> int:
    """Waits for the stream; first device-side error of adacomp_select_static calls since the last read."""
    return int(_lib.adacomp_select_static_last_error(int(device_index), _stream_ptr(stream)))


# ----------------------------------------------------------------------------- worker side

def adacomp_encode_capacity_words(pairs_per_worker: int) -> int:
    return int(_lib.adacomp_encode_capacity_words(int(pairs_per_worker)))


def adacomp_encode_indices(idx: torch.Tensor, stream: Optional[torch.cuda.Stream] = None):
    """idx [W, K] (int32 holding uint32 bit patterns) -> (words [W, capacity] int32, block_off [W, n_blocks + 1]
    int64): the block-wise gap coding of every worker's index list."""
    if idx.dim() == 1:
        idx = idx.unsqueeze(0)
    W, K = idx.shape
    cap = adacomp_encode_capacity_words(K)
    words = torch.empty((W, max(cap, 1)), dtype=torch.int32, device=idx.device)
    off = torch.empty((W, (K + 255) // 256 + 1), dtype=torch.int64, device=idx.device)
    _check(_lib.adacomp_encode_indices(_dev(idx, torch.int32, "idx") if K else None, K, W, words.data_ptr(), words.shape[1],
                                       off.data_ptr(), idx.device.index or 0, _stream_ptr(stream)), "adacomp_encode_indices")
    return words, off


def adacomp_decode_indices(words: torch.Tensor, block_off: torch.Tensor, pairs_per_worker: int,
                           stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    W = words.shape[0]
    out = torch.empty((W, pairs_per_worker), dtype=torch.int32, device=words.device)
    _check(_lib.adacomp_decode_indices(_dev(words, torch.int32, "words"), words.shape[1], _dev(block_off, torch.int64, "block_off"),
                                       int(pairs_per_worker), W, out.data_ptr(), words.device.index or 0, _stream_ptr(stream)),
           "adacomp_decode_indices")
    return out


def adacomp_encode_values_capacity_words(pairs_per_worker: int) -> int:
    return int(_lib.adacomp_encode_values_capacity_words(int(pairs_per_worker)))


def adacomp_encode_values(val: torch.Tensor, stream: Optional[torch.cuda.Stream] = None):
    """val [W, K] float32 -> (words [W, capacity] int32, block_off [W, n_blocks + 1] int64): the lossless block-wise
    packing of every worker's values."""
    if val.dim() == 1:
        val = val.unsqueeze(0)
    W, K = val.shape
    cap = adacomp_encode_values_capacity_words(K)
    words = torch.empty((W, max(cap, 1)), dtype=torch.int32, device=val.device)
    off = torch.empty((W, (K + 255) // 256 + 1), dtype=torch.int64, device=val.device)
    _check(_lib.adacomp_encode_values(_dev(val, torch.float32, "val") if K else None, K, W, words.data_ptr(), words.shape[1],
                                      off.data_ptr(), val.device.index or 0, _stream_ptr(stream)), "adacomp_encode_values")
    return words, off


def adacomp_decode_values(words: torch.Tensor, block_off: torch.Tensor, pairs_per_worker: int,
                          stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    W = words.shape[0]
    out = torch.empty((W, pairs_per_worker), dtype=torch.float32, device=words.device)
    _check(_lib.adacomp_decode_values(_dev(words, torch.int32, "words"), words.shape[1], _dev(block_off, torch.int64, "block_off"),
                                      int(pairs_per_worker), W, out.data_ptr(), words.device.index or 0, _stream_ptr(stream)),
           "adacomp_decode_values")
    return out


class Selector:
    """SELECT_GRAD (Algorithm 1) for a fixed tensor layout; owns its device workspace."""

    def __init__(self, segments, max_workers: int, device: Optional[torch.device] = None):
        self.device = torch.device(device if device is not None else "cuda")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.segments = segments
        self.n_segs = len(segments)
        self.max_workers = int(max_workers)
        nbytes = ctypes.c_size_t(0)
        _check(_lib.adacomp_select_workspace_bytes(segments, self.n_segs, self.max_workers, ctypes.byref(nbytes)),
               "adacomp_select_workspace_bytes")
        self.workspace = torch.empty(max(int(nbytes.value), 256), dtype=torch.uint8, device=self.device)
        h = ctypes.c_void_p()
        _check(_lib.adacomp_select_create(ctypes.byref(h), segments, self.n_segs, self.max_workers,
                                          self.workspace.data_ptr(), self.workspace.numel(), self.device.index),
               "adacomp_select_create")
        self._h = h
        k = ctypes.c_uint64(0)
        _check(_lib.adacomp_select_pairs_per_worker(self._h, ctypes.byref(k)), "adacomp_select_pairs_per_worker")
        self.pairs_per_worker = int(k.value)

    def select(self, grads: torch.Tensor, idx_out: Optional[torch.Tensor] = None,
               val_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
        """grads: [W, stride] (or [stride]) fp32 on the device -> (idx [W, K] as int32 bit
        pattern of uint32, val [W, K] fp32)."""
        if grads.dim() == 1:
            grads = grads.unsqueeze(0)
        if grads.stride(-1) != 1:
            raise TypeError("grads: innermost dimension must be contiguous")
        W = grads.shape[0]
        stride = grads.stride(0) if W > 1 else grads.shape[1]
        if not (grads.is_cuda and grads.dtype == torch.float32):
            raise TypeError("grads: need a CUDA fp32 tensor")
        K = self.pairs_per_worker
        if idx_out is None:
            idx_out = torch.empty((W, K), dtype=torch.int32, device=grads.device)
        if val_out is None:
            val_out = torch.empty((W, K), dtype=torch.float32, device=grads.device)
        _check(_lib.adacomp_select(self._h, grads.data_ptr(), stride, W, _dev(idx_out, torch.int32, "idx_out"),
                                   _dev(val_out, torch.float32, "val_out"), _stream_ptr(stream)), "adacomp_select")
        return idx_out, val_out

    def select_host(self, h_grads: torch.Tensor, d_grads: torch.Tensor, d_idx: torch.Tensor, d_val: torch.Tensor,
                    h_idx: torch.Tensor, h_val: torch.Tensor, stream: Optional[torch.cuda.Stream] = None):
        W = h_grads.shape[0]
        _check(_lib.adacomp_select_host(self._h, _host(h_grads, torch.float32, "h_grads"), h_grads.shape[1], W,
                                        _dev(d_grads, torch.float32, "d_grads"), _dev(d_idx, torch.int32, "d_idx"),
                                        _dev(d_val, torch.float32, "d_val"), _host(h_idx, torch.int32, "h_idx"),
                                        _host(h_val, torch.float32, "h_val"), _stream_ptr(stream)),
               "adacomp_select_host")

    def gather(self, grads: torch.Tensor, idx: torch.Tensor, val_out: Optional[torch.Tensor] = None,
               stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """val[w][e] = grads[w][idx[w][e]] for idx of shape [W, pairs_per_worker]."""
        g = grads if grads.dim() == 2 else grads.unsqueeze(0)
        W = g.shape[0]
        if idx.numel() != W * self.pairs_per_worker:
            raise ValueError("idx needs pairs_per_worker entries per worker")
        if val_out is None:
            val_out = torch.empty((W, self.pairs_per_worker), dtype=torch.float32, device=g.device)
        if g.stride(1) != 1 or not (g.is_cuda and g.dtype == torch.float32):
            raise TypeError("grads: need a CUDA fp32 tensor whose innermost dimension is contiguous")
        _check(_lib.adacomp_select_gather(self._h, g.data_ptr(), g.stride(0) if W > 1 else g.shape[1],
                                          W, _dev(idx, torch.int32, "idx"), _dev(val_out, torch.float32, "val_out"),
                                          _stream_ptr(stream)), "adacomp_select_gather")
        return val_out

    def set_route(self, route: int):
        """0 = automatic (bracketed single pass where eligible), 1 = general route only."""
        _check(_lib.adacomp_select_set_route(self._h, int(route)), "adacomp_select_set_route")

    def route_info(self) -> dict:
        """Tensors on the cluster route and the cluster shape chosen on this device."""
        info = (ctypes.c_uint32 * 4)()
        _check(_lib.adacomp_select_route_info(self._h, info), "adacomp_select_route_info")
        return {"cluster_tensors": int(info[0]), "blocks_per_cluster": int(info[1]), "ring_slots": int(info[2]) & 255,
                "warps_per_block": int(info[2]) >> 8, "resident_clusters": int(info[3])}

    def set_profiling(self, on):
        """False / 0: off; True / 1: CUDA events around every kernel; 2: around the pass over the gradient only."""
        _check(_lib.adacomp_select_set_profiling(self._h, int(on)), "adacomp_select_set_profiling")

    def profile(self) -> dict:
        """Mean device milliseconds per kernel and call since profiling was switched on."""
        n = 0
        while _lib.adacomp_select_stage_name(n):
            n += 1
        ms = (ctypes.c_float * n)()
        calls = ctypes.c_uint64(0)
        _check(_lib.adacomp_select_profile(self._h, ms, n, ctypes.byref(calls)), "adacomp_select_profile")
        out = {_lib.adacomp_select_stage_name(i).decode(): float(ms[i]) for i in range(n)}
        out["calls"] = int(calls.value)
        return out

    def last_error(self, stream: Optional[torch.cuda.Stream] = None) -> Tuple[int, int]:
        """(status, selections that took the general route in the last call); waits for the stream."""
        stats = (ctypes.c_uint64 * 4)()
        status = _lib.adacomp_select_last_error(self._h, _stream_ptr(stream), stats)
        return int(status), int(stats[0])

    def close(self):
        if getattr(self, "_h", None):
            _lib.adacomp_select_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ----------------------------------------------------------------------------- server side

class Server:
    """Parameter server of Algorithm 2; owns its device workspace, borrows theta."""

    def __init__(self, theta: torch.Tensor, history_pairs: int, max_window_updates: int):
        self.device = theta.device
        self.n_params = theta.numel()
        nbytes = ctypes.c_size_t(0)
        _check(_lib.adacomp_server_workspace_bytes(self.n_params, history_pairs, ctypes.byref(nbytes)),
               "adacomp_server_workspace_bytes")
        self.workspace = torch.empty(max(int(nbytes.value), 256), dtype=torch.uint8, device=self.device)
        h = ctypes.c_void_p()
        _check(_lib.adacomp_server_create(ctypes.byref(h), self.n_params, history_pairs, max_window_updates,
                                          self.workspace.data_ptr(), self.workspace.numel(), self.device.index),
               "adacomp_server_create")
        self._h = h
        self.reset(theta)

    def reset(self, theta: torch.Tensor, stream: Optional[torch.cuda.Stream] = None):
        if theta.numel() != self.n_params:
            raise ValueError("theta has the wrong size")
        self.theta = theta
        _check(_lib.adacomp_server_reset(self._h, _dev(theta, torch.float32, "theta"), _stream_ptr(stream)),
               "adacomp_server_reset")

    def pull(self, theta_copy: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> int:
        ts = ctypes.c_uint64(0)
        ptr = _dev(theta_copy, torch.float32, "theta_copy") if theta_copy is not None else None
        _check(_lib.adacomp_server_pull(self._h, ptr, ctypes.byref(ts), _stream_ptr(stream)), "adacomp_server_pull")
        return int(ts.value)

    def apply(self, idx: torch.Tensor, val: torch.Tensor, pair_begin, pair_count, pull_ts, lr: float,
              sigma_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
        """Applies len(pull_ts) updates in array (= arrival) order; update b is pairs
        [pair_begin[b], pair_begin[b] + pair_count[b]) of idx / val."""
        pb, pj = _u64_array(pair_begin), _u64_array(pull_ts)
        pc = np.ascontiguousarray(pair_count, dtype=np.uint32)
        if not (pb.size == pj.size == pc.size):
            raise ValueError("pair_begin, pair_count and pull_ts need one entry per update")
        sig = _dev(sigma_out, torch.int32, "sigma_out") if sigma_out is not None else None
        _check(_lib.adacomp_apply(self._h, _dev(idx, torch.int32, "idx"), _dev(val, torch.float32, "val"),
                                  pb.ctypes.data_as(ctypes.POINTER(ctypes.c_uint64)),
                                  pc.ctypes.data_as(ctypes.POINTER(ctypes.c_uint32)),
                                  pj.ctypes.data_as(ctypes.POINTER(ctypes.c_uint64)), pj.size, float(lr), sig,
                                  _stream_ptr(stream)), "adacomp_apply")

    def apply_host(self, h_idx: torch.Tensor, h_val: torch.Tensor, pair_begin, pair_count, pull_ts, lr: float,
                   d_idx: torch.Tensor, d_val: torch.Tensor, d_sigma: Optional[torch.Tensor] = None,
                   h_sigma: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
        pb, pj = _u64_array(pair_begin), _u64_array(pull_ts)
        pc = np.ascontiguousarray(pair_count, dtype=np.uint32)
        if not (pb.size == pj.size == pc.size):
            raise ValueError("pair_begin, pair_count and pull_ts need one entry per update")
        _check(_lib.adacomp_apply_host(self._h, _host(h_idx, torch.int32, "h_idx"), _host(h_val, torch.float32, "h_val"),
                                       pb.ctypes.data_as(ctypes.POINTER(ctypes.c_uint64)),
                                       pc.ctypes.data_as(ctypes.POINTER(ctypes.c_uint32)),
                                       pj.ctypes.data_as(ctypes.POINTER(ctypes.c_uint64)), pj.size, float(lr),
                                       _dev(d_idx, torch.int32, "d_idx"), _dev(d_val, torch.float32, "d_val"),
                                       _dev(d_sigma, torch.int32, "d_sigma") if d_sigma is not None else None,
                                       _host(h_sigma, torch.int32, "h_sigma") if h_sigma is not None else None,
                                       _stream_ptr(stream)), "adacomp_apply_host")

    @property
    def timestamp(self) -> int:
        ts = ctypes.c_uint64(0)
        _check(_lib.adacomp_server_timestamp(self._h, ctypes.byref(ts)), "adacomp_server_timestamp")
        return int(ts.value)

    def set_validation(self, on: bool):
        _check(_lib.adacomp_server_set_validation(self._h, int(on)), "adacomp_server_set_validation")

    def set_mode(self, mode: int):
        """0 automatic, 1 one launch per update, 2 batches that touch only the named parameters, 3 batches over a dense sweep,
        4 the paper's sorted lists with one search per update of the window (only switchable at timestamp 0)."""
        _check(_lib.adacomp_server_set_mode(self._h, int(mode)), "adacomp_server_set_mode")

    def set_rule(self, rule: int):
        """0 AdaComp (per-parameter staleness), 1 the competitors' rule (the update's staleness i - j)."""
        _check(_lib.adacomp_server_set_rule(self._h, int(rule)), "adacomp_server_set_rule")

    def apply_dense(self, delta: torch.Tensor, pull_ts: int, lr: float, stream: Optional[torch.cuda.Stream] = None):
        """One dense update under rule 1: Theta <- Theta - lr / (i - pull_ts) * delta."""
        if delta.numel() != self.n_params:
            raise ValueError("a dense update has one entry per parameter")
        _check(_lib.adacomp_apply_dense(self._h, _dev(delta, torch.float32, "delta"), int(pull_ts), float(lr),
                                        _stream_ptr(stream)), "adacomp_apply_dense")

    def debug_skip_positions(self, count: int):
        _check(_lib.adacomp_server_debug_skip_positions(self._h, int(count)), "adacomp_server_debug_skip_positions")

    def last_error(self, stream: Optional[torch.cuda.Stream] = None) -> int:
        return int(_lib.adacomp_server_last_error(self._h, _stream_ptr(stream)))

    def close(self):
        if getattr(self, "_h", None):
            _lib.adacomp_server_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ----------------------------------------------------------------------------- clipping

def _empty(like: torch.Tensor, shape, dtype, stream: Optional[torch.cuda.Stream]) -> torch.Tensor:
    """An output tensor on the device of `like` that belongs to the stream its kernels run on."""
    if stream is None:
        return like.new_empty(shape) if like.dtype == dtype else like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _element_type(t: torch.Tensor, device: int, name: str) -> int:
    kind = ELEMENT_TYPES.get(t.dtype)
    if kind is None or t.get_device() != device:
        raise TypeError(f"{name}: need a float32, bfloat16 or float16 tensor on cuda:{device}")
    return kind


class _Handle:
    """What :class:`Clipper` and :class:`Embedding` share: a device workspace and the streams that work in it."""

    def _take_workspace(self, nbytes: int) -> None:
        """Device memory for the handle.  The allocator hands out memory that earlier work of the current stream may still write to,
        and handles clear theirs on the default stream: that work is waited for."""
        self.workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=self.device)
        home = torch.cuda.current_stream(self.device)
        home.synchronize()
        self._streams = {home.cuda_stream}

    def _stream_on(self, stream: Optional[torch.cuda.Stream]) -> int:
        """The given stream, or the device's current one (asked for without building a stream object, which costs as much as a
        launch).  The allocator is told of streams other than the workspace's own: a handle may be dropped while they run."""
        raw = torch._C._cuda_getCurrentRawStream(self._index) if stream is None else stream.cuda_stream
        if raw not in self._streams:
            self.workspace.record_stream(torch.cuda.current_stream(self.device) if stream is None else stream)
            self._streams.add(raw)
        return raw


def _is_dense(t: torch.Tensor) -> bool:
    """Whether the tensor's entries fill one stretch of memory, in whatever order of its dimensions."""
    if t.is_contiguous():
        return True
    expect = 1
    for stride, size in sorted((st, n) for st, n in zip(t.stride(), t.shape) if n != 1):
        if stride != expect:
            return False
        expect *= size
    return True


class GradList:
    """One worker's gradient tensors, and where their clipped values go (``out``: one tensor for each, of any of the three
    types and with the same shape and strides; None: in place).  Holds on to the tensors and only says where they are: a
    program whose gradients stay in place makes the list once, values are read when a call runs."""

    def __init__(self, grads: Sequence[torch.Tensor], out: Optional[Sequence[torch.Tensor]] = None):
        self.grads = list(grads)
        self.out = self.grads if out is None else list(out)
        if not self.grads:
            raise ValueError("grads: need at least one tensor")
        if len(self.out) != len(self.grads):
            raise ValueError("out: need one tensor for each gradient")
        self.device = self.grads[0].get_device()
        if self.device < 0:
            raise TypeError("grads: need CUDA tensors")
        self.table = (GradTensor * len(self.grads))()
        spans = []                              # (begin, end, written)
        for i, (g, o) in enumerate(zip(self.grads, self.out)):
            kind, out_kind = _element_type(g, self.device, "grads"), _element_type(o, self.device, "out")
            if o is not g and (o.shape != g.shape or (o.stride() != g.stride() and not (o.is_contiguous() and g.is_contiguous()))):
                raise ValueError("out: need the shape and strides of the gradient")
            if not _is_dense(g):
                raise TypeError("grads: need tensors without gaps")
            e, n, at, to = self.table[i], g.numel(), g.data_ptr(), o.data_ptr()
            e.d_grad, e.d_out, e.n, e.grad_type, e.out_type = at, to, n, kind, out_kind
            if n:
                in_place = at == to and g.dtype == o.dtype
                spans.append((at, at + n * g.element_size(), in_place))
                if not in_place:
                    spans.append((to, to + n * o.element_size(), True))
        spans.sort()
        reach = reach_written = 0               # how far the tensors before extend, and those of them that are written
        self.overlapping = False
        for begin, end, written in spans:
            self.overlapping |= begin < reach_written or (written and begin < reach)
            reach = max(reach, end)
            if written:
                reach_written = max(reach_written, end)
        if out is not None:
            self.check_apart()

    def check_apart(self):
        """Tensors that share memory can be measured, not clipped."""
        if self.overlapping:
            raise ValueError("out: overlaps a gradient or another output")


class Clipper(_Handle):
    """Global gradient norm and clipping; owns its device workspace.  Gradients are a :class:`GradList`, a sequence of tensors
    (one worker, any shapes), or a matrix [W, P] whose rows are the flat gradients of W workers."""

    def __init__(self, max_workers: int = 1, device: Optional[torch.device] = None):
        self.device = torch.device(device if device is not None else "cuda")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index
        self.max_workers = int(max_workers)
        nbytes = ctypes.c_size_t(0)
        _check(_lib.adacomp_clip_workspace_bytes(self.max_workers, ctypes.byref(nbytes)), "adacomp_clip_workspace_bytes")
        self._take_workspace(int(nbytes.value))
        h = ctypes.c_void_p()
        _check(_lib.adacomp_clip_create(ctypes.byref(h), self.max_workers, self.workspace.data_ptr(), self.workspace.numel(),
                                        self.device.index), "adacomp_clip_create")
        self._h = h

    def _given(self, grads, out=None, write=False):
        """(table, tensors, workers, gradient stride, output stride, outputs)"""
        if not isinstance(grads, (torch.Tensor, GradList)):
            grads = GradList(grads, out)
        elif out is not None and isinstance(grads, GradList):
            raise ValueError("out: the list already says where its outputs go")
        if isinstance(grads, GradList):
            if grads.device != self._index:
                raise TypeError(f"grads: need tensors on {self.device}")
            if write:
                grads.check_apart()
            return grads.table, len(grads.grads), 1, 0, 0, grads.out
        kind, shape = _element_type(grads, self._index, "grads"), grads.shape
        if out is None:
            out, out_kind = grads, kind
        else:
            out_kind = _element_type(out, self._index, "out")
        if len(shape) != 2 or out.shape != shape:
            raise ValueError("grads: need a matrix [workers, entries], and out of the same shape")
        W, n = shape
        strides, out_strides = grads.stride(), out.stride()
        if n > 1 and (strides[1] != 1 or out_strides[1] != 1):
            raise TypeError("grads, out: need contiguous rows")
        if write and W > 1 and out_strides[0] < n:
            raise TypeError("out: need rows that do not overlap")
        if out is not grads:
            at, size, to, out_size = grads.data_ptr(), grads.element_size(), out.data_ptr(), out.element_size()
            apart, out_apart = strides[0] * size, out_strides[0] * out_size
            same = at == to and grads.dtype == out.dtype and (W == 1 or apart == out_apart)
            if not same and n and at < to + (W - 1) * out_apart + n * out_size and to < at + (W - 1) * apart + n * size:
                # rows of one buffer may hold both, next to each other
                if W == 1 or apart != out_apart or not n * size <= (to - at) % apart <= apart - n * out_size:
                    raise ValueError("out: overlaps the gradients")
        e = GradTensor(grads.data_ptr(), out.data_ptr(), n, kind, out_kind)
        return ctypes.byref(e), 1, W, strides[0] if W > 1 else 0, out_strides[0] if W > 1 else 0, out

    def norm(self, grads, scale: float = 1.0, norm_out: Optional[torch.Tensor] = None,
             stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """|scale| times the norm over all of a worker's entries: float32 [W]."""
        table, count, W, stride, _, _ = self._given(grads)
        if norm_out is None:
            norm_out = _empty(self.workspace, (W,), torch.float32, stream)
        elif norm_out.numel() != W:
            raise ValueError("norm_out: need one entry per worker")
        _check(_lib.adacomp_grad_norm(self._h, table, count, stride, W, float(scale), _dev(norm_out, torch.float32, "norm_out"),
                                      self._stream_on(stream)), "adacomp_grad_norm")
        return norm_out

    def clip(self, grads, max_norm: float, scale: float = 1.0, out=None, norm_out: Optional[torch.Tensor] = None,
             coef_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
        """out = grads * scale * min(1, max_norm / (norm + 1e-6)) -> (out, norm [W]).  ``out`` defaults to the gradients
        themselves; ``coef_out`` [W] receives the factors."""
        table, count, W, stride, out_stride, out = self._given(grads, out, write=True)
        if norm_out is None:
            norm_out = _empty(self.workspace, (W,), torch.float32, stream)
        for t, name in ((norm_out, "norm_out"), (coef_out, "coef_out")):
            if t is not None and t.numel() != W:
                raise ValueError(f"{name}: need one entry per worker")
        _check(_lib.adacomp_clip(self._h, table, count, stride, out_stride, W, float(scale), float(max_norm),
                                 _dev(norm_out, torch.float32, "norm_out"),
                                 _dev(coef_out, torch.float32, "coef_out") if coef_out is not None else None,
                                 self._stream_on(stream)), "adacomp_clip")
        return out, norm_out

    def close(self):
        if getattr(self, "_h", None):
            _lib.adacomp_clip_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ----------------------------------------------------------------------------- embedding tables

def _rows(t: torch.Tensor, dims: int, kind: int, name: str) -> Rows:
    """The first `dims` dimensions of a tensor as the numbering of its rows."""
    shape = t.shape
    if t.is_contiguous():
        row = 1
        for n in shape[dims:]:
            row *= n
        return Rows(t.data_ptr(), kind, 0, row, 0)
    r = Rows(t.data_ptr(), kind)
    strides = t.stride()
    merged = []                                 # [rows, distance], outermost first; neighbours that make one run are joined
    for n, st in zip(shape[:dims], strides[:dims]):
        if n == 1:
            continue
        if merged and merged[-1][1] == n * st:
            merged[-1] = [merged[-1][0] * n, st]
        else:
            merged.append([n, st])
    if len(merged) > 2 or any(st < 0 for _, st in merged):
        raise TypeError(f"{name}: rows need at most two distances between them")
    if merged:
        r.row_stride = merged[-1][1]
    if len(merged) == 2:
        r.group, r.group_stride = merged[1][0], merged[0][1]
    return r


class Embedding(_Handle):
    """Embedding tables of `vocab` rows of `dim` entries: lookup with scaling, and the gradient by sorted tokens; owns its
    device workspace.  ``max_tokens`` bounds the tokens of a gradient call (0: lookups only)."""

    def __init__(self, vocab: int, dim: int, max_tokens: int = 0, max_workers: int = 1, padding_idx: Optional[int] = None,
                 device: Optional[torch.device] = None):
        self.device = torch.device(device if device is not None else "cuda")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index
        self.vocab, self.dim, self.max_tokens, self.max_workers = int(vocab), int(dim), int(max_tokens), int(max_workers)
        if padding_idx is not None and not 0 <= padding_idx < self.vocab:
            raise ValueError("padding_idx: need a token of the vocabulary")
        pad = 0xFFFFFFFF if padding_idx is None else int(padding_idx)
        for n in (self.vocab, self.dim, self.max_tokens, self.max_workers):
            if not 0 <= n < 1 << 32:
                raise AdacompError(ERR_INVALID, "adacomp_embed_workspace_bytes")
        nbytes = ctypes.c_size_t(0)
        _check(_lib.adacomp_embed_workspace_bytes(self.vocab, self.dim, self.max_tokens, self.max_workers, ctypes.byref(nbytes)),
               "adacomp_embed_workspace_bytes")
        self._take_workspace(int(nbytes.value))
        h = ctypes.c_void_p()
        _check(_lib.adacomp_embed_create(ctypes.byref(h), self.vocab, self.dim, self.max_tokens, self.max_workers, pad,
                                         self.workspace.data_ptr(), self.workspace.numel(), self.device.index),
               "adacomp_embed_create")
        self._h = h

    def _tokens(self, tokens: torch.Tensor) -> Rows:
        kind = TOKEN_TYPES.get(tokens.dtype)
        if kind is None or tokens.get_device() != self._index:
            raise TypeError(f"tokens: need an int32 or int64 tensor on {self.device}")
        if tokens.numel() >= 1 << 31:
            raise ValueError("tokens: too many")
        return _rows(tokens, tokens.dim(), kind, "tokens")

    def _wide(self, t: torch.Tensor, name: str) -> Rows:
        kind = _element_type(t, self._index, name)
        shape = t.shape
        if not shape or shape[-1] != self.dim:
            raise TypeError(f"{name}: need rows of {self.dim} entries")
        if t.is_contiguous():
            return Rows(t.data_ptr(), kind, 0, self.dim, 0)
        if self.dim > 1 and t.stride(-1) != 1:
            raise TypeError(f"{name}: need contiguous rows")
        return _rows(t, len(shape) - 1, kind, name)

    def lookup(self, table: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0, out: Optional[torch.Tensor] = None,
               dtype: Optional[torch.dtype] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """table [vocab, dim], tokens of any shape -> [*tokens.shape, dim] = table[tokens] * scale, of ``dtype`` (the
        table's by default)."""
        if table.dim() != 2 or table.shape[0] != self.vocab:
            raise ValueError(f"table: need {self.vocab} rows")
        shape = (*tokens.shape, self.dim)
        ids = self._tokens(tokens)
        if out is None:
            out = _empty(table, shape, dtype or table.dtype, stream)
        elif out.shape != shape or (dtype is not None and out.dtype != dtype):
            raise ValueError("out: need a row for every token, and the type asked for")
        _check(_lib.adacomp_embed_lookup(self._h, ctypes.byref(self._wide(table, "table")), ctypes.byref(ids), tokens.numel(),
                                         float(scale), ctypes.byref(self._wide(out, "out")), self._stream_on(stream)),
               "adacomp_embed_lookup")
        return out

    def _batch(self, tokens: torch.Tensor, grad: torch.Tensor, workers: int):
        """(tokens, tokens of a worker, gradient's rows)"""
        n, shape = tokens.numel(), grad.shape
        if workers < 1 or n % workers:
            raise ValueError("tokens: need the same number for every worker")
        if grad.numel() != n * self.dim:
            raise ValueError("grad: need a row for every token")
        if len(shape) > 2:
            # a list of rows or of tokens is in the order of the other; two shapes have to be the same, but for ones
            given = tokens.shape
            if len(given) > 1 and shape[:-1] != given and [n for n in shape[:-1] if n != 1] != [n for n in given if n != 1]:
                raise ValueError("grad: need the shape of the tokens")
        return self._tokens(tokens), n // workers, self._wide(grad, "grad")

    def _grad_rows(self, tokens, grad, scale, workers, rows_out, values_out, idx_out, offset, stream):
        ids, per_worker, rows = self._batch(tokens, grad, workers)
        n = per_worker * workers
        for t, need, name in ((rows_out, n, "rows_out"), (values_out, n * self.dim, "values_out"), (idx_out, n * self.dim, "idx_out")):
            if t is not None and t.numel() < need:
                raise ValueError(f"{name}: too small")
        begin = _empty(self.workspace, (workers + 1,), torch.int64, stream)
        kind = _element_type(values_out, self._index, "values_out")
        _check(_lib.adacomp_embed_grad_rows(self._h, ctypes.byref(ids), per_worker, workers, ctypes.byref(rows), float(scale),
                                            _dev(rows_out, torch.int32, "rows_out") if rows_out is not None else None,
                                            begin.data_ptr(), _dev(values_out, values_out.dtype, "values_out"), kind,
                                            _dev(idx_out, torch.int32, "idx_out") if idx_out is not None else None, int(offset),
                                            self._stream_on(stream)), "adacomp_embed_grad_rows")
        return begin

    def grad_rows(self, tokens: torch.Tensor, grad: torch.Tensor, scale: float = 1.0, workers: int = 1,
                  dtype: torch.dtype = torch.float32, rows_out: Optional[torch.Tensor] = None,
                  values_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
        """Gradient of the table as its distinct rows -> (rows int32 [N], values [N, dim], row_begin int64 [workers + 1]) with
        N = tokens.numel(): worker w's tokens (its share of the flattened ``tokens``) gave the entries row_begin[w] ..
        row_begin[w + 1] of the two lists; what lies behind the last is left as it was."""
        n = tokens.numel()
        if rows_out is None:
            rows_out = _empty(grad, (n,), torch.int32, stream)
        if values_out is None:
            values_out = _empty(grad, (n, self.dim), dtype, stream)
        begin = self._grad_rows(tokens, grad, scale, workers, rows_out, values_out, None, 0, stream)
        return rows_out, values_out, begin

    def grad_update(self, tokens: torch.Tensor, grad: torch.Tensor, scale: float = 1.0, workers: int = 1, offset: int = 0,
                    idx_out: Optional[torch.Tensor] = None, val_out: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None):
        """The same gradient as updates for :meth:`Server.apply` -> (idx int32 [N, dim] holding uint32, val float32 [N, dim],
        row_begin int64 [workers + 1]); the table is entries offset .. offset + vocab * dim - 1 of the parameters.  Worker w's
        update is pairs row_begin[w] * dim .. row_begin[w + 1] * dim - 1."""
        n = tokens.numel()
        if idx_out is None:
            idx_out = _empty(grad, (n, self.dim), torch.int32, stream)
        if val_out is None:
            val_out = _empty(grad, (n, self.dim), torch.float32, stream)
        elif val_out.dtype != torch.float32:
            raise TypeError("val_out: updates are float32")
        begin = self._grad_rows(tokens, grad, scale, workers, None, val_out, idx_out, offset, stream)
        return idx_out, val_out, begin

    def grad_dense(self, tokens: torch.Tensor, grad: torch.Tensor, out: torch.Tensor, scale: float = 1.0, accumulate: bool = False,
                   workers: int = 1, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """The whole table's gradient into ``out`` [vocab, dim] or [workers, vocab, dim]; ``accumulate``: added to what is
        there instead of replacing it."""
        ids, per_worker, rows = self._batch(tokens, grad, workers)
        want = (self.vocab, self.dim)
        if tuple(out.shape) != (workers, *want) and not (workers == 1 and tuple(out.shape) == want):
            raise ValueError("out: need a table for every worker")
        if out.data_ptr() == grad.data_ptr() and grad.numel():
            raise ValueError("out: overlaps the gradient")
        _check(_lib.adacomp_embed_grad_dense(self._h, ctypes.byref(ids), per_worker, workers, ctypes.byref(rows), float(scale),
                                             ctypes.byref(self._wide(out, "out")), int(accumulate), self._stream_on(stream)),
               "adacomp_embed_grad_dense")
        return out

    def set_wait_limit(self, polls: int) -> None:
        """How often the blocks of a large sort look for each other before they give up (ERR_TIMEOUT); 0: once."""
        _check(_lib.adacomp_embed_set_wait_limit(self._h, int(polls)), "adacomp_embed_set_wait_limit")

    def last_error(self, stream: Optional[torch.cuda.Stream] = None) -> int:
        """Waits for the stream; the first error the device recorded since the last call (a token outside the vocabulary)."""
        return int(_lib.adacomp_embed_last_error(self._h, self._stream_on(stream)))

    def close(self):
        if getattr(self, "_h", None):
            _lib.adacomp_embed_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def raw():
    """The ctypes library object, for tests that call the C ABI directly."""
    return _lib
