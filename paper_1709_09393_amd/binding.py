"""ctypes binding over ``libslimdp.so`` (the C ABI of ``include/slimdp.h``).

Argument marshalling only: every step of the path runs in the library's HIP kernels.
torch is used for device memory and the stream; there is no CPU fallback -- if the shared
library is missing or no GPU is present the calls raise.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import List, Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libslimdp.so")

TILE = 4096
MAX_WORKERS = 32

OK = 0
ERR_INVALID_ARG = -1
ERR_OUT_OF_RANGE = -2
ERR_STALE_CORE = -3
ERR_WORKSPACE = -4
ERR_HIP = -5
ERR_DEVICE_STATUS = -6
SELECT_REUSE_HISTOGRAM = 1
PACK_UPDATES_AS_SCORED = 1
LOCAL_FIRST = 1
QUANT_BUCKET = 512
F32, F16, BF16 = 0, 1, 2
GRAD_ACCUMULATE = 1
MAX_ROWS = 1 << 24
MAX_NORM_COLS = 65536
MAX_FEATURES = 1 << 20
MAX_TILES = 1 << 23
MAX_VOCAB = 1 << 24
MAX_TEACHER = 1024
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
LINEAR_FORWARD, LINEAR_EPILOGUE_BACKWARD, LINEAR_BACKWARD = 0, 1, 2

EXPORTS = [
    "slimdp_create", "slimdp_destroy", "slimdp_workspace_bytes", "slimdp_capture_bytes", "slimdp_num_tiles",
    "slimdp_tile_starts", "slimdp_last_error", "slimdp_synchronize", "slimdp_set_option",
    "slimdp_score", "slimdp_dense_update_score", "slimdp_select_core", "slimdp_sample_explore", "slimdp_explore_hint", "slimdp_tile_offsets",
    "slimdp_pack", "slimdp_merge", "slimdp_pull", "slimdp_core_signature", "slimdp_debug_philox",
    "slimdp_select_core_static", "slimdp_import_core", "slimdp_local_step", "slimdp_local_step_pack", "slimdp_pull_local_step", "slimdp_quantize",
    "slimdp_dequantize", "slimdp_layer_norm", "slimdp_layer_norm_backward", "slimdp_layer_norm_workspace_bytes", "slimdp_linear",
    "slimdp_linear_epilogue_backward", "slimdp_linear_backward", "slimdp_linear_workspace_bytes", "slimdp_distill_loss",
]


class SlimDPError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libslimdp error {code}: {msg}")
        self.code = code


_lib = None
_vp = C.c_void_p
_u64p = C.POINTER(C.c_uint64)
_vpp = C.POINTER(C.c_void_p)


def load() -> C.CDLL:
    """Loads the in-tree shared library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()')")
    L = C.CDLL(LIB_PATH)
    L.slimdp_create.argtypes = [C.POINTER(_vp), C.c_uint64, C.c_uint32, C.c_uint32, _u64p, C.c_uint64, _vp]
    L.slimdp_create.restype = C.c_int
    L.slimdp_destroy.argtypes = [_vp]
    L.slimdp_destroy.restype = C.c_int
    L.slimdp_workspace_bytes.argtypes = [C.c_uint64, C.c_uint32, C.c_uint32, _u64p]
    L.slimdp_workspace_bytes.restype = C.c_uint64
    L.slimdp_capture_bytes.argtypes = [C.c_uint64, C.c_uint32, C.c_uint32, _u64p]
    L.slimdp_capture_bytes.restype = C.c_uint64
    L.slimdp_num_tiles.argtypes = [C.c_uint64, C.c_uint32, _u64p]
    L.slimdp_num_tiles.restype = C.c_uint64
    L.slimdp_tile_starts.argtypes = [_vp, C.POINTER(C.c_uint32)]
    L.slimdp_tile_starts.restype = C.c_int
    L.slimdp_last_error.argtypes = [_vp]
    L.slimdp_last_error.restype = C.c_char_p
    L.slimdp_synchronize.argtypes = [_vp]
    L.slimdp_synchronize.restype = C.c_int
    L.slimdp_set_option.argtypes = [_vp, C.c_char_p, C.c_int64]
    L.slimdp_set_option.restype = C.c_int
    L.slimdp_score.argtypes = [_vp, _vp, _vpp, C.c_uint32, C.c_float, _vp]
    L.slimdp_score.restype = C.c_int
    L.slimdp_dense_update_score.argtypes = [_vp, _vp, _vpp, C.c_uint32, C.c_float, C.c_float, _vp]
    L.slimdp_dense_update_score.restype = C.c_int
    L.slimdp_core_signature.argtypes = [_vp, _vp, C.c_uint64, _vp]
    L.slimdp_core_signature.restype = C.c_int
    L.slimdp_select_core.argtypes = [_vp, _vp, _u64p, C.c_uint32, _vp, _vp, _vp, _u64p]
    L.slimdp_select_core.restype = C.c_int
    L.slimdp_sample_explore.argtypes = [_vp, _vp, _u64p, C.c_uint32, C.c_uint32, C.c_uint64, _u64p, _vpp, _vpp]
    L.slimdp_sample_explore.restype = C.c_int
    L.slimdp_explore_hint.argtypes = [_vp, _u64p, C.c_uint32, C.c_uint32, C.c_uint64, _u64p]
    L.slimdp_explore_hint.restype = C.c_int
    L.slimdp_tile_offsets.argtypes = [_vp, _vp, C.c_uint64, _vp]
    L.slimdp_tile_offsets.restype = C.c_int
    L.slimdp_pack.argtypes = [_vp, C.c_uint32, _vpp, _vp, _vp, C.c_uint64, _vpp, _vpp, _u64p, _vpp, _vpp, C.c_uint64,
                              C.c_uint32]
    L.slimdp_pack.restype = C.c_int
    L.slimdp_merge.argtypes = [_vp, _vp, C.c_float, C.c_uint64, C.c_uint32, _vp, _vp, C.c_uint64, _vpp, _vpp, _vpp,
                               _vpp, _u64p]
    L.slimdp_merge.restype = C.c_int
    L.slimdp_pull.argtypes = [_vp, _vp, C.c_uint64, C.c_uint32, _vp, _vp, C.c_uint64, _vpp, _vpp, _u64p, _vpp, _vpp,
                              _vpp]
    L.slimdp_pull.restype = C.c_int
    L.slimdp_debug_philox.argtypes = [_vp, C.c_uint64, C.c_uint32, C.c_uint32, C.c_uint64, _vp]
    L.slimdp_debug_philox.restype = C.c_int
    L.slimdp_select_core_static.argtypes = [_vp, C.c_uint64, C.c_uint64, _vp, _vp, _vp, _vp]
    L.slimdp_select_core_static.restype = C.c_int
    L.slimdp_import_core.argtypes = [_vp, _vp, _u64p, _vp, _vp, _u64p]
    L.slimdp_import_core.restype = C.c_int
    L.slimdp_local_step.argtypes = [_vp, C.c_uint32, _vpp, _vpp, _vpp, C.c_float, C.c_uint32]
    L.slimdp_local_step.restype = C.c_int
    L.slimdp_local_step_pack.argtypes = [_vp, C.c_uint32, _vpp, _vpp, _vpp, C.c_float, C.c_uint32, _vp, _vp, C.c_uint64, _vpp,
                                         _vpp, _u64p, _vpp, _vpp, C.c_uint64]
    L.slimdp_local_step_pack.restype = C.c_int
    L.slimdp_pull_local_step.argtypes = [_vp, _vp, C.c_uint64, C.c_uint32, _vp, _vp, C.c_uint64, _vpp, _vpp, _u64p, _vpp, _vpp,
                                         _vpp, C.c_float, C.c_uint32]
    L.slimdp_pull_local_step.restype = C.c_int
    L.slimdp_quantize.argtypes = [_vp, C.c_uint32, C.c_uint32, _vpp, _u64p, C.c_uint32, C.c_uint64, _vpp, _vpp]
    L.slimdp_quantize.restype = C.c_int
    L.slimdp_dequantize.argtypes = [_vp, C.c_uint32, _vpp, _vpp, _u64p, _vpp]
    L.slimdp_dequantize.restype = C.c_int
    u32, u64, f32 = C.c_uint32, C.c_uint64, C.c_float
    L.slimdp_layer_norm.argtypes = [_vp, u32, _u64p, u64, u32, _vpp, u64, _vpp, _vpp, f32, _vpp, u64, _vpp, _vpp]
    L.slimdp_layer_norm.restype = C.c_int
    L.slimdp_layer_norm_backward.argtypes = [_vp, u32, _u64p, u64, u32, _vpp, u64, _vpp, u64, _vpp, _vpp, _vpp, _vpp, u64, _vpp, _vpp, u32,
                                             _vp, u64]
    L.slimdp_layer_norm_backward.restype = C.c_int
    L.slimdp_layer_norm_workspace_bytes.argtypes = [u32, _u64p, u64, u32]
    L.slimdp_layer_norm_workspace_bytes.restype = u64
    L.slimdp_linear.argtypes = [_vp, u32, _u64p, u64, u64, u32, _vpp, u64, _vpp, u64, _vpp, u32, _vpp, u64, _vpp, u64, _vpp, u64, _vp, u64]
    L.slimdp_linear.restype = C.c_int
    L.slimdp_linear_epilogue_backward.argtypes = [_vp, u32, _u64p, u64, u32, _vpp, u64, _vpp, u64, u32, _vpp, u64, _vpp, u32, _vp, u64]
    L.slimdp_linear_epilogue_backward.restype = C.c_int
    L.slimdp_linear_backward.argtypes = [_vp, u32, _u64p, u64, u64, u32, _vpp, u64, _vpp, u64, _vpp, u64, _vpp, u64, _vpp, u32, _vp, u64]
    L.slimdp_linear_backward.restype = C.c_int
    L.slimdp_linear_workspace_bytes.argtypes = [u32, _u64p, u64, u64, u32, u32]
    L.slimdp_linear_workspace_bytes.restype = u64
    L.slimdp_distill_loss.argtypes = [_vp, u32, _u64p, u64, u32, _vpp, u64, u64, _vpp, _vpp, u64, f32, _vpp, _vpp, _vpp, _vpp, u64]
    L.slimdp_distill_loss.restype = C.c_int
    _lib = L
    return L


_arrays = {}


def _array(kind, n: int):
    """The ctypes array type (made once: making it takes longer than filling it)."""
    got = _arrays.get((kind, n))
    if got is None:
        got = _arrays[(kind, n)] = kind * n
    return got


def _u64arr(vals) -> "C.Array":
    vals = [int(v) for v in vals]
    return _array(C.c_uint64, max(1, len(vals)))(*vals)


def _types(torch) -> dict:
    """Numbers of the element types: the library's, and 3 for int32 (lists of indices)."""
    global _type_numbers
    if _type_numbers is None:
        _type_numbers = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16, torch.int32: 3}
    return _type_numbers


def _tables():
    """The compiled form of the checks below (None where it is not built: they then run as written)."""
    global _helper
    if _helper is False:
        try:
            from . import _tables as helper
        except ImportError:
            helper = None
        _helper = helper
    return _helper


_type_numbers = None
_helper = False


def _seg_off(n: int, seg_off) -> "C.Array":
    if seg_off is None:
        seg_off = [0, n]
    return _u64arr(seg_off)


def num_tiles(n: int, seg_off=None) -> int:
    so = [0, n] if seg_off is None else [int(x) for x in seg_off]
    return int(load().slimdp_num_tiles(n, len(so) - 1, _u64arr(so)))


def workspace_bytes(n: int, max_workers: int, seg_off=None) -> int:
    so = [0, n] if seg_off is None else [int(x) for x in seg_off]
    return int(load().slimdp_workspace_bytes(n, max_workers, len(so) - 1, _u64arr(so)))


def capture_bytes(n: int, max_workers: int, seg_off=None) -> int:
    so = [0, n] if seg_off is None else [int(x) for x in seg_off]
    return int(load().slimdp_capture_bytes(n, max_workers, len(so) - 1, _u64arr(so)))


def _ptr(t) -> Optional[int]:
    """Device address of a torch tensor (None passes NULL)."""
    if t is None:
        return None
    return t.data_ptr() if t.numel() else (t.data_ptr() or None)


def _table(ts: Optional[Sequence]) -> "C.Array":
    if ts is None:
        return None
    arr = (C.c_void_p * max(1, len(ts)))()
    for j, t in enumerate(ts):
        arr[j] = _ptr(t)
    return arr


STATIC_MAX_N = 1 << 20


def select_core_static(score, k: int, core_idx, core_bits, core_off, stream=None) -> None:
    """slimdp_select_core_static: flat selection without a context; every array is the caller's (nothing is allocated)."""
    import torch
    st = stream if stream is not None else torch.cuda.current_stream()
    rc = load().slimdp_select_core_static(_ptr(score), score.numel(), int(k), _ptr(core_idx), _ptr(core_bits),
                                          _ptr(core_off), C.c_void_p(st.cuda_stream))
    if rc != OK:
        raise SlimDPError(rc, load().slimdp_last_error(None).decode())


class SlimDP:
    """One context: n parameters, up to max_workers logical workers, one GPU, one stream."""

    _index = -1          # the device's number as tensors give it

    def __init__(self, n: int, max_workers: int, seg_off=None, seed: int = 0, stream=None):
        import torch
        self._torch = torch
        self._L = load()
        if not torch.cuda.is_available():
            raise RuntimeError("libslimdp needs a GPU: torch.cuda.is_available() is False")
        self.n = int(n)
        self.max_workers = int(max_workers)
        self.seg_off = [0, self.n] if seg_off is None else [int(x) for x in seg_off]
        self.n_seg = len(self.seg_off) - 1
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        self._h = C.c_void_p()
        rc = self._L.slimdp_create(C.byref(self._h), self.n, self.max_workers, self.n_seg, _u64arr(self.seg_off),
                                   int(seed), C.c_void_p(self.stream.cuda_stream))
        if rc != OK:
            msg = self._L.slimdp_last_error(None).decode()
            self._h = None
            raise SlimDPError(rc, msg)
        self.T = num_tiles(self.n, self.seg_off)
        self.device = torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index
        self._raw_stream = self.stream.cuda_stream

    # -- plumbing ------------------------------------------------------------------------
    def _check(self, rc: int) -> None:
        if rc != OK:
            raise SlimDPError(rc, self._L.slimdp_last_error(self._h).decode())

    def close(self) -> None:
        if getattr(self, "_h", None):
            self._L.slimdp_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def synchronize(self) -> None:
        self._check(self._L.slimdp_synchronize(self._h))

    def set_option(self, name: str, value: int) -> None:
        self._check(self._L.slimdp_set_option(self._h, name.encode(), int(value)))

    def tile_starts(self) -> np.ndarray:
        out = np.zeros(self.T + 1, dtype=np.uint32)
        self._check(self._L.slimdp_tile_starts(self._h, out.ctypes.data_as(C.POINTER(C.c_uint32))))
        return out

    def _empty(self, count: int, dtype):
        return self._torch.empty(int(count), dtype=dtype, device=self.device)

    # -- the path ------------------------------------------------------------------------
    def score(self, w, g: Sequence, c: float, out=None):
        torch = self._torch
        if out is None:
            out = self._empty(self.n, torch.float32)
        self._check(self._L.slimdp_score(self._h, _ptr(w), _table(g), len(g), C.c_float(c), _ptr(out)))
        return out

    def dense_update_score(self, w, g: Sequence, lr: float, c: float, out=None):
        """w <- w - lr * sum of all updates (in place), then the significance of the new model."""
        torch = self._torch
        if out is None:
            out = self._empty(self.n, torch.float32)
        self._check(self._L.slimdp_dense_update_score(self._h, _ptr(w), _table(g), len(g), C.c_float(lr), C.c_float(c),
                                                      _ptr(out)))
        return out

    def select_core(self, score, k_seg, reuse_histogram: bool = False, core_idx=None, core_bits=None, core_off=None):
        torch = self._torch
        ks = [int(k_seg)] if np.isscalar(k_seg) else [int(x) for x in k_seg]
        K = sum(ks)
        if core_idx is None:
            core_idx = self._empty(K, torch.int32)
        if core_bits is None:
            core_bits = self._empty((self.n + 31) // 32, torch.int32)
        if core_off is None:
            core_off = self._empty(self.T + 1, torch.int32)
        epoch = C.c_uint64(0)
        self._check(self._L.slimdp_select_core(self._h, _ptr(score), _u64arr(ks),
                                               SELECT_REUSE_HISTOGRAM if reuse_histogram else 0, _ptr(core_idx),
                                               _ptr(core_bits), _ptr(core_off), C.byref(epoch)))
        return core_idx, core_bits, core_off, int(epoch.value)

    def sample_explore(self, core_bits, k_seg, iteration: int, m_seg, worker0: int = 0, n_workers: int = 1,
                       expl_idx: Optional[List] = None, expl_off: Optional[List] = None):
        torch = self._torch
        ks = [int(k_seg)] if np.isscalar(k_seg) else [int(x) for x in k_seg]
        ms = [int(m_seg)] if np.isscalar(m_seg) else [int(x) for x in m_seg]
        M = sum(ms)
        if expl_idx is None:
            expl_idx = [self._empty(M, torch.int32) for _ in range(n_workers)]
        if expl_off is None:
            expl_off = [self._empty(self.T + 1, torch.int32) for _ in range(n_workers)]
        self._check(self._L.slimdp_sample_explore(self._h, _ptr(core_bits), _u64arr(ks), worker0, n_workers,
                                                  int(iteration), _u64arr(ms), _table(expl_idx), _table(expl_off)))
        return expl_idx, expl_off

    def explore_hint(self, k_seg, iteration: int, m_seg, worker0: int = 0, n_workers: int = 1) -> None:
        ks = [int(k_seg)] if np.isscalar(k_seg) else [int(x) for x in k_seg]
        ms = [int(m_seg)] if np.isscalar(m_seg) else [int(x) for x in m_seg]
        self._check(self._L.slimdp_explore_hint(self._h, _u64arr(ks), worker0, n_workers, int(iteration), _u64arr(ms)))

    def tile_offsets(self, idx, out=None):
        if out is None:
            out = self._empty(self.T + 1, self._torch.int32)
        self._check(self._L.slimdp_tile_offsets(self._h, _ptr(idx), idx.numel(), _ptr(out)))
        return out

    def pack(self, g: Sequence, core_idx, core_off, expl_idx: Sequence, expl_off: Sequence, core_epoch: int,
             core_val: Optional[List] = None, expl_val: Optional[List] = None, updates_as_scored: bool = False):
        """updates_as_scored: g is, unchanged, what the last score() on this context read."""
        torch = self._torch
        nw = len(g)
        k = core_idx.numel()
        if core_val is None:
            core_val = [self._empty(k, torch.float32) for _ in range(nw)]
        if expl_val is None:
            expl_val = [self._empty(expl_idx[q].numel(), torch.float32) for q in range(nw)]
        mw = _u64arr([expl_idx[q].numel() for q in range(nw)])
        self._check(self._L.slimdp_pack(self._h, nw, _table(g), _ptr(core_idx), _ptr(core_off), k, _table(expl_idx),
                                        _table(expl_off), mw, _table(core_val), _table(expl_val), int(core_epoch),
                                        PACK_UPDATES_AS_SCORED if updates_as_scored else 0))
        return core_val, expl_val

    def merge(self, w, lr: float, core_epoch: int, core_idx, core_off, core_val: Sequence, expl_idx: Sequence,
              expl_off: Sequence, expl_val: Sequence) -> None:
        nw = len(core_val)
        mw = _u64arr([expl_idx[q].numel() for q in range(nw)])
        self._check(self._L.slimdp_merge(self._h, _ptr(w), C.c_float(lr), int(core_epoch), nw, _ptr(core_idx),
                                         _ptr(core_off), core_idx.numel(), _table(core_val), _table(expl_idx),
                                         _table(expl_off), _table(expl_val), mw))

    def pull(self, w, core_epoch: int, core_idx, core_off, expl_idx: Sequence, expl_off: Sequence,
             w_local: Optional[Sequence] = None, core_out: Optional[List] = None, expl_out: Optional[List] = None):
        torch = self._torch
        nw = len(expl_idx)
        k = core_idx.numel()
        if core_out is None:
            core_out = [self._empty(k, torch.float32) for _ in range(nw)]
        if expl_out is None:
            expl_out = [self._empty(expl_idx[q].numel(), torch.float32) for q in range(nw)]
        mw = _u64arr([expl_idx[q].numel() for q in range(nw)])
        self._check(self._L.slimdp_pull(self._h, _ptr(w), int(core_epoch), nw, _ptr(core_idx), _ptr(core_off), k,
                                        _table(expl_idx), _table(expl_off), mw, _table(core_out), _table(expl_out),
                                        _table(w_local)))
        return core_out, expl_out

    def core_signature(self, core_idx):
        """Signature of the cached core keys; returns a one-element int64 device tensor (read it after synchronize)."""
        out = self._empty(1, self._torch.int64)
        self._check(self._L.slimdp_core_signature(self._h, _ptr(core_idx), core_idx.numel(), _ptr(out)))
        return out

    def debug_philox(self, iteration: int, worker: int, i0: int, count: int):
        out = self._empty(count, self._torch.int32)
        self._check(self._L.slimdp_debug_philox(self._h, int(iteration), int(worker), int(i0), int(count), _ptr(out)))
        return out

    def import_core(self, core_idx, k_seg, core_bits=None, core_off=None):
        """Adopts core keys saved from another context (resume); returns (core_bits, core_off, epoch)."""
        torch = self._torch
        ks = [int(k_seg)] if np.isscalar(k_seg) else [int(x) for x in k_seg]
        if core_bits is None:
            core_bits = self._empty((self.n + 31) // 32, torch.int32)
        if core_off is None:
            core_off = self._empty(self.T + 1, torch.int32)
        epoch = C.c_uint64(0)
        self._check(self._L.slimdp_import_core(self._h, _ptr(core_idx), _u64arr(ks), _ptr(core_bits), _ptr(core_off),
                                               C.byref(epoch)))
        return core_bits, core_off, int(epoch.value)

    # -- worker side and wire codec ------------------------------------------------------
    def local_step(self, w_local: Sequence, grad: Sequence, delta: Sequence, eta: float, first: bool) -> None:
        """One mini-batch step on every local model; delta accumulates the update (first: starts a new sum)."""
        self._check(self._L.slimdp_local_step(self._h, len(w_local), _table(w_local), _table(grad), _table(delta),
                                              C.c_float(eta), LOCAL_FIRST if first else 0))

    def local_step_pack(self, w_local: Sequence, grad: Sequence, delta: Sequence, eta: float, first: bool, core_idx,
                        core_off, expl_idx: Sequence, expl_off: Sequence, core_epoch: int,
                        core_val: Optional[List] = None, expl_val: Optional[List] = None):
        """local_step() and pack(delta, ...) in one pass over the update vectors."""
        torch = self._torch
        nw = len(w_local)
        k = core_idx.numel()
        if core_val is None:
            core_val = [self._empty(k, torch.float32) for _ in range(nw)]
        if expl_val is None:
            expl_val = [self._empty(expl_idx[q].numel(), torch.float32) for q in range(nw)]
        mw = _u64arr([expl_idx[q].numel() for q in range(nw)])
        self._check(self._L.slimdp_local_step_pack(self._h, nw, _table(w_local), _table(grad), _table(delta), C.c_float(eta),
                                                   LOCAL_FIRST if first else 0, _ptr(core_idx), _ptr(core_off), k,
                                                   _table(expl_idx), _table(expl_off), mw, _table(core_val),
                                                   _table(expl_val), int(core_epoch)))
        return core_val, expl_val

    def pull_local_step(self, w, core_epoch: int, core_idx, core_off, expl_idx: Sequence, expl_off: Sequence,
                        w_local: Sequence, grad: Sequence, delta: Sequence, eta: float, first: bool = True) -> None:
        """pull(..., w_local=w_local) (its value outputs aside) and local_step() in one pass over the local models."""
        nw = len(w_local)
        mw = _u64arr([expl_idx[q].numel() for q in range(nw)])
        self._check(self._L.slimdp_pull_local_step(self._h, _ptr(w), int(core_epoch), nw, _ptr(core_idx), _ptr(core_off),
                                                   core_idx.numel(), _table(expl_idx), _table(expl_off), mw, _table(w_local),
                                                   _table(grad), _table(delta), C.c_float(eta), LOCAL_FIRST if first else 0))

    def quantize(self, val: Sequence, kind: int, iteration: int, worker0: int = 0, code=None, scale=None):
        torch = self._torch
        nw = len(val)
        if code is None:
            code = [self._empty(v.numel(), torch.uint8) for v in val]
        if scale is None:
            scale = [self._empty((v.numel() + QUANT_BUCKET - 1) // QUANT_BUCKET, torch.float32) for v in val]
        cnt = _u64arr([v.numel() for v in val])
        self._check(self._L.slimdp_quantize(self._h, nw, int(worker0), _table(val), cnt, int(kind), int(iteration),
                                            _table(code), _table(scale)))
        return code, scale

    def dequantize(self, code: Sequence, scale: Sequence, out=None):
        torch = self._torch
        nw = len(code)
        if out is None:
            out = [self._empty(c.numel(), torch.float32) for c in code]
        cnt = _u64arr([c.numel() for c in code])
        self._check(self._L.slimdp_dequantize(self._h, nw, _table(code), _table(scale), cnt, _table(out)))
        return out


    # -- operators of LocalTrain ---------------------------------------------------------
    # Lists hold one tensor a worker: matrices [rows of the worker, columns] with consecutive columns, rows any distance apart (the
    # same for all workers); parameters of the local model and their gradients binary32 and contiguous (pieces of flat vectors).
    # With accumulate, gradients of parameters are added to the arrays given for them, and none is made for those that are not given.
    def _layout(self, who: str, x: Sequence):
        """(rows of every worker, columns, dtype number, torch dtype) from a call's first list."""
        if x[0].dim() != 2:
            raise ValueError(f"{who}: expected one two-dimensional tensor a worker")
        dtype = x[0].dtype
        code = _types(self._torch).get(dtype, 3)
        if code > BF16:
            raise ValueError(f"{who}: unsupported dtype {dtype}")
        return [v.shape[0] for v in x], x[0].shape[1], code, dtype

    def _matrix(self, who: str, name: str, ts, rows, cols: int, dtype):
        """Pointer table and row distance of a list of matrices; (None, 0) for none."""
        if ts is None:
            return None, 0
        if len(ts) != len(rows):
            raise ValueError(f"{who}: {name} holds {len(ts)} tensors for {len(rows)} workers")
        fast = _tables()
        if fast is not None:
            table = _array(C.c_void_p, len(ts))()
            ld = fast.matrix(ts if type(ts) is list else list(ts), rows, cols, _types(self._torch)[dtype], self._index, C.addressof(table))
            if ld >= 0:
                return table, ld or cols
        ptrs, ld, device = [], -1, self._index
        for t, r in zip(ts, rows):                     # a handful of attributes a tensor: small calls wait for this loop
            if t.dtype is not dtype or t.shape != (r, cols) or t.get_device() != device:
                raise ValueError(f"{who}: {name}[{len(ptrs)}] is {tuple(t.shape)} {t.dtype} on {t.device}, "
                                 f"expected {(r, cols)} {dtype} on {self.device}")
            if r == 0:
                ptrs.append(None)
                continue
            step, inner = t.stride()
            if inner != 1 and cols > 1:
                raise ValueError(f"{who}: columns of {name}[{len(ptrs)}] are not consecutive")
            if r > 1 and step != ld:
                if ld >= 0 or step < cols:
                    raise ValueError(f"{who}: rows of {name}[{len(ptrs)}] are {step} elements apart, expected {max(ld, cols)}")
                ld = step
            ptrs.append(t.data_ptr())
            if not ptrs[-1] and cols:
                raise ValueError(f"{who}: {name}[{len(ptrs) - 1}] has no memory")
        return _array(C.c_void_p, len(ptrs))(*ptrs), max(ld, cols)

    def _vectors(self, who: str, name: str, ts, sizes, dtype):
        """Pointer table of a list of contiguous tensors of the given numbers of elements; None for none, also for single workers."""
        if ts is None:
            return None
        if len(ts) != len(sizes):
            raise ValueError(f"{who}: {name} holds {len(ts)} tensors for {len(sizes)} workers")
        fast = _tables()
        if fast is not None:
            table = _array(C.c_void_p, len(ts))()
            if fast.vectors(ts if type(ts) is list else list(ts), sizes, _types(self._torch)[dtype], self._index, C.addressof(table)) == 0:
                return table
        ptrs, device = [], self._index
        for t, n in zip(ts, sizes):
            if t is None or (n == 0 and t.numel() == 0):
                ptrs.append(None)
                continue
            if t.dtype is not dtype or t.numel() != n or t.get_device() != device or not t.is_contiguous():
                raise ValueError(f"{who}: {name}[{len(ptrs)}] is {tuple(t.shape)} {t.dtype} on {t.device}, "
                                 f"expected {n} consecutive {dtype} on {self.device}")
            ptrs.append(t.data_ptr())
            if not ptrs[-1] and n:
                raise ValueError(f"{who}: {name}[{len(ptrs) - 1}] has no memory")
        return _array(C.c_void_p, len(ptrs))(*ptrs)

    def _new(self, make):
        """Runs make with the context's stream current: memory goes back to the allocator in the order of that stream's work."""
        torch = self._torch
        if torch._C._cuda_getCurrentRawStream(self._index) == self._raw_stream:      # a torch.cuda.Stream object takes ten times as long
            return make()
        with torch.cuda.device(self.device), torch.cuda.stream(self.stream):
            return make()

    def _workspace(self, nbytes: int):
        """Scratch for one call; the tensor is to live until the call is enqueued."""
        if not nbytes:
            return None
        return self._new(lambda: self._torch.empty(nbytes, dtype=self._torch.uint8, device=self.device))

    def _matrices(self, rows, cols: int, dtype):
        return self._new(lambda: [self._torch.empty((r, cols), dtype=dtype, device=self.device) for r in rows])

    def _flat(self, sizes, dtype=None):
        return self._new(lambda: [self._torch.empty(n, dtype=dtype or self._torch.float32, device=self.device) for n in sizes])

    def layer_norm(self, x: Sequence, weight: Optional[Sequence], bias: Optional[Sequence], eps: float = 1e-5, y: Optional[List] = None,
                   mean: Optional[List] = None, rstd: Optional[List] = None):
        """Layer norm of every worker's rows; returns (y, mean, rstd), the latter two for the backward pass."""
        who, f32 = "layer_norm", self._torch.float32
        rows, cols, code, dtype = self._layout(who, x)
        if y is None:
            y = self._matrices(rows, cols, dtype)
        if mean is None:
            mean = self._flat(rows)
        if rstd is None:
            rstd = self._flat(rows)
        px, ldx = self._matrix(who, "x", x, rows, cols, dtype)
        py, ldy = self._matrix(who, "y", y, rows, cols, dtype)
        per = [cols] * len(rows)
        self._check(self._L.slimdp_layer_norm(self._h, len(rows), _u64arr(rows), cols, code, px, ldx, self._vectors(who, "weight", weight, per, f32),
                                              self._vectors(who, "bias", bias, per, f32), eps, py, ldy,
                                              self._vectors(who, "mean", mean, rows, f32), self._vectors(who, "rstd", rstd, rows, f32)))
        return y, mean, rstd

    def layer_norm_backward(self, dy: Sequence, x: Sequence, weight: Optional[Sequence], mean: Sequence, rstd: Sequence,
                            dx: Optional[List] = None, dweight: Optional[List] = None, dbias: Optional[List] = None,
                            accumulate: bool = False, want_dx: bool = True, want_params: bool = True):
        """Gradients of layer_norm(): returns (dx, dweight, dbias), None for what is neither given nor wanted."""
        who, f32 = "layer_norm_backward", self._torch.float32
        rows, cols, code, dtype = self._layout(who, x)
        per = [cols] * len(rows)
        if dx is None and want_dx:
            dx = self._matrices(rows, cols, dtype)
        if want_params and not accumulate:
            dweight = dweight if dweight is not None else self._flat(per)
            dbias = dbias if dbias is not None else self._flat(per)
        pdy, lddy = self._matrix(who, "dy", dy, rows, cols, dtype)
        px, ldx = self._matrix(who, "x", x, rows, cols, dtype)
        pdx, lddx = self._matrix(who, "dx", dx, rows, cols, dtype)
        n = _u64arr(rows)
        ws = self._workspace(self._L.slimdp_layer_norm_workspace_bytes(len(rows), n, cols, code) if dweight is not None or dbias is not None else 0)
        self._check(self._L.slimdp_layer_norm_backward(
            self._h, len(rows), n, cols, code, pdy, lddy, px, ldx, self._vectors(who, "weight", weight, per, f32),
            self._vectors(who, "mean", mean, rows, f32), self._vectors(who, "rstd", rstd, rows, f32), pdx, lddx,
            self._vectors(who, "dweight", dweight, per, f32), self._vectors(who, "dbias", dbias, per, f32),
            GRAD_ACCUMULATE if accumulate else 0, _ptr(ws), ws.numel() if ws is not None else 0))
        return dx, dweight, dbias

    def linear(self, x: Sequence, weight: Sequence, bias: Optional[Sequence] = None, activation: str = "none",
               residual: Optional[Sequence] = None, y: Optional[List] = None, z: Optional[List] = None, keep: bool = False):
        """activation(x weight^T + bias) + residual; returns (y, z), z (before the activation, for the backward pass) if given or keep."""
        who, f32 = "linear", self._torch.float32
        rows, cols, code, dtype = self._layout(who, x)
        out = weight[0].shape[0]
        if y is None:
            y = self._matrices(rows, out, dtype)
        if z is None and keep:
            z = self._matrices(rows, out, dtype)
        outs = [out] * len(rows)
        px, ldx = self._matrix(who, "x", x, rows, cols, dtype)
        pw, ldw = self._matrix(who, "weight", weight, outs, cols, dtype)
        pr, ldr = self._matrix(who, "residual", residual, rows, out, dtype)
        py, ldy = self._matrix(who, "y", y, rows, out, dtype)
        pz, ldz = self._matrix(who, "z", z, rows, out, dtype)
        n = _u64arr(rows)
        ws = self._workspace(self._L.slimdp_linear_workspace_bytes(len(rows), n, cols, out, code, LINEAR_FORWARD))
        self._check(self._L.slimdp_linear(self._h, len(rows), n, cols, out, code, px, ldx, pw, ldw, self._vectors(who, "bias", bias, outs, f32),
                                          ACTIVATIONS[activation], pr, ldr, py, ldy, pz, ldz, _ptr(ws), ws.numel() if ws is not None else 0))
        return y, z

    def linear_epilogue_backward(self, dy: Sequence, z: Optional[Sequence] = None, activation: str = "none", dz: Optional[List] = None,
                                 dbias: Optional[List] = None, accumulate: bool = False, want_dbias: bool = True):
        """Gradients of linear()'s epilogue: returns (dz, dbias).  Without an activation dz is dy, and none is written unless given."""
        who, f32 = "linear_epilogue_backward", self._torch.float32
        rows, out, code, dtype = self._layout(who, dy)
        per = [out] * len(rows)
        if dz is None and activation != "none":
            dz = self._matrices(rows, out, dtype)
        if dbias is None and want_dbias and not accumulate:
            dbias = self._flat(per)
        pdy, lddy = self._matrix(who, "dy", dy, rows, out, dtype)
        pz, ldz = self._matrix(who, "z", z if activation != "none" else None, rows, out, dtype)
        pdz, lddz = self._matrix(who, "dz", dz, rows, out, dtype)
        n = _u64arr(rows)
        ws = self._workspace(self._L.slimdp_linear_workspace_bytes(len(rows), n, 1, out, code, LINEAR_EPILOGUE_BACKWARD) if dbias is not None else 0)
        self._check(self._L.slimdp_linear_epilogue_backward(self._h, len(rows), n, out, code, pdy, lddy, pz, ldz, ACTIVATIONS[activation],
                                                            pdz, lddz, self._vectors(who, "dbias", dbias, per, f32),
                                                            GRAD_ACCUMULATE if accumulate else 0, _ptr(ws), ws.numel() if ws is not None else 0))
        return (dz if dz is not None else dy), dbias

    def linear_backward(self, dz: Sequence, x: Optional[Sequence], weight: Optional[Sequence], dx: Optional[List] = None,
                        dweight: Optional[List] = None, accumulate: bool = False, want_dx: bool = True, want_dweight: bool = True):
        """Gradients of linear()'s product: returns (dx, dweight), None for what is neither given nor wanted."""
        who, f32 = "linear_backward", self._torch.float32
        rows, out, code, dtype = self._layout(who, dz)
        cols = (x if x is not None else weight)[0].shape[1]
        W = len(rows)
        if dx is None and want_dx:
            dx = self._matrices(rows, cols, dtype)
        if dweight is None and want_dweight and not accumulate:
            dweight = [v.view(out, cols) for v in self._flat([out * cols] * W)]
        pdz, lddz = self._matrix(who, "dz", dz, rows, out, dtype)
        px, ldx = self._matrix(who, "x", x, rows, cols, dtype)
        pw, ldw = self._matrix(who, "weight", weight, [out] * W, cols, dtype)
        pdx, lddx = self._matrix(who, "dx", dx, rows, cols, dtype)
        n = _u64arr(rows)
        ws = self._workspace(self._L.slimdp_linear_workspace_bytes(W, n, cols, out, code, LINEAR_BACKWARD))
        self._check(self._L.slimdp_linear_backward(self._h, W, n, cols, out, code, pdz, lddz, px, ldx, pw, ldw, pdx, lddx,
                                                   self._vectors(who, "dweight", dweight, [out * cols] * W, f32),
                                                   GRAD_ACCUMULATE if accumulate else 0, _ptr(ws), ws.numel() if ws is not None else 0))
        return dx, dweight

    def distill_loss(self, logits: Sequence, index: Sequence, value: Sequence, temperature: float = 1.0,
                     row_weight: Optional[Sequence] = None, loss: Optional[List] = None, lse: Optional[List] = None,
                     dlogits: Optional[List] = None, want_grad: bool = True):
        """Distillation from the teacher's top logits (int32 index, -1 = no entry; binary32 value): returns (loss, lse, dlogits), dlogits
        None if neither given nor wanted."""
        who, torch = "distill_loss", self._torch
        rows, vocab, code, dtype = self._layout(who, logits)
        top = index[0].shape[1]
        if loss is None:
            loss = self._flat(rows)
        if lse is None:
            lse = self._flat(rows)
        if dlogits is None and want_grad:
            dlogits = self._matrices(rows, vocab, dtype)
        pl, ldl = self._matrix(who, "logits", logits, rows, vocab, dtype)
        pi, ldt = self._matrix(who, "index", index, rows, top, torch.int32)
        pv, ldv = self._matrix(who, "value", value, rows, top, torch.float32)
        if ldt != ldv:
            raise ValueError(f"{who}: rows of index and value lie {ldt} and {ldv} elements apart")
        pd, lddl = self._matrix(who, "dlogits", dlogits, rows, vocab, dtype)
        self._check(self._L.slimdp_distill_loss(self._h, len(rows), _u64arr(rows), vocab, code, pl, ldl, top, pi, pv, ldt, temperature,
                                                self._vectors(who, "row_weight", row_weight, rows, torch.float32),
                                                self._vectors(who, "loss", loss, rows, torch.float32),
                                                self._vectors(who, "lse", lse, rows, torch.float32), pd, lddl))
        return loss, lse, dlogits


def wire_bytes(k: int, m: int, quantized: bool) -> int:
    """Bytes one worker pushes (core values + explorer <key, value> pairs), plain or with 8-bit values."""
    if not quantized:
        return 4 * (k + 2 * m)
    nb = lambda c: (c + QUANT_BUCKET - 1) // QUANT_BUCKET
    return k + 4 * nb(k) + 5 * m + 4 * nb(m)
