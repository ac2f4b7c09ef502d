"""ctypes binding of the C-ABI library declared in ``include/rcd.h``.

Argument marshalling only: every step of the computation runs in the CUDA
kernels of ``librcd.so``.  PyTorch supplies device memory and streams.  If the
compiled library is missing, importing this module raises; there is no CPU
fallback of any kind.

The functions keep the names of the C entry points (``rcd_similarity``,
``rcd_partition``, ``rcd_partition_host``, ``rcd_objective``, ``rcd_quotas``,
``rcd_rms_norm``, ``rcd_linear``, ``rcd_linear_cross_entropy`` and their ``_backward``,
``rcd_orthogonalize``, ...);
``Context`` wraps ``rcd_create`` / ``rcd_destroy``.
"""
from __future__ import annotations

import ctypes as C
import math
import os
from typing import Dict, Optional, Sequence, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librcd.so")

RCD_FEAT_I8 = 0
RCD_FEAT_BF16 = 1
RCD_SIM_DOT = 0
RCD_SIM_GAUSSIAN = 1
RCD_OBJ_FACILITY = 0
RCD_OBJ_GRAPH_CUT = 1
RCD_FORM_LAUNCHES, RCD_FORM_BARRIERS, RCD_FORM_ASYNC, RCD_FORM_CLASS_PER_CTA, RCD_FORM_CLUSTER, RCD_FORM_ROUNDS, RCD_FORM_CUT_CHAIN, RCD_FORM_SMALL, RCD_FORM_CUT_STEPS = range(1, 10)

RCD_ELEM_I8, RCD_ELEM_BF16, RCD_ELEM_F16, RCD_ELEM_F32 = range(4)
RCD_ACT_NONE, RCD_ACT_RELU, RCD_ACT_GELU, RCD_ACT_GELU_TANH, RCD_ACT_SILU = range(5)
# int8 features made by `normalize`: rows of root mean square 1 on a scale that cuts them off at four times that
RCD_FEATURE_SCALE = 4.0 / 127.0
# a, b, c of a Newton-Schulz step that brings small singular values up fast and leaves them between 0.65 and 1.25
RCD_QUINTIC = (3.4445, -4.7750, 2.0315)

STATUS_NAMES = {0: "RCD_OK", 1: "RCD_ERR_INVALID_ARG", 2: "RCD_ERR_UNSUPPORTED", 3: "RCD_ERR_WORKSPACE_TOO_SMALL",
                4: "RCD_ERR_CUDA", 5: "RCD_ERR_TIMEOUT", 6: "RCD_ERR_INTERNAL"}

# every symbol include/rcd.h declares
EXPORTS = ["rcd_create", "rcd_destroy", "rcd_last_error", "rcd_version", "rcd_sync_status", "rcd_selftest_bounded_wait", "rcd_get_profile",
           "rcd_quotas", "rcd_similarity", "rcd_similarity_gaussian_workspace_bytes", "rcd_similarity_gaussian",
           "rcd_partition_workspace_bytes", "rcd_partition",
           "rcd_partition_host_workspace_bytes", "rcd_partition_host", "rcd_objective_workspace_bytes",
           "rcd_objective", "rcd_objective_class_static",
           "rcd_worker_lists_workspace_bytes", "rcd_worker_lists", "rcd_batch_sizes", "rcd_batch_sizes_rule",
           "rcd_rms_norm", "rcd_quantize_rows", "rcd_rms_norm_backward_workspace_bytes", "rcd_rms_norm_backward",
           "rcd_linear_workspace_bytes", "rcd_linear", "rcd_linear_backward_workspace_bytes", "rcd_linear_backward",
           "rcd_linear_cross_entropy_workspace_bytes", "rcd_linear_cross_entropy", "rcd_linear_cross_entropy_backward_workspace_bytes",
           "rcd_linear_cross_entropy_backward", "rcd_orthogonalize_workspace_bytes", "rcd_orthogonalize",
           "rcd_yardstick_read", "rcd_yardstick_mma"]


class RcdError(RuntimeError):
    def __init__(self, status: int, message: str = ""):
        self.status = int(status)
        super().__init__("%s%s" % (STATUS_NAMES.get(self.status, str(status)), (": " + message) if message else ""))


class RcdConfig(C.Structure):
    _fields_ = [("sweep_batch_max", C.c_int32), ("similarity_path", C.c_int32), ("profile", C.c_int32),
                ("greedy_path", C.c_int32), ("similarity_kind", C.c_int32), ("objective", C.c_int32), ("sweep_mode", C.c_int32), ("async_group", C.c_int32),
                ("async_help_min", C.c_int32), ("threshold_from", C.c_int32), ("threshold_hit_shift", C.c_int32),
                ("lazy_mode", C.c_int32), ("lazy_from", C.c_int32), ("dense_ring", C.c_int32), ("incremental", C.c_int32), ("incremental_max", C.c_int32)]


class RcdProfile(C.Structure):
    _fields_ = [("total_ms", C.c_double), ("group_ms", C.c_double), ("similarity_ms", C.c_double),
                ("greedy_ms", C.c_double), ("sweep_ms", C.c_double), ("sweep_launches", C.c_int64),
                ("sweep_bytes", C.c_int64), ("sweep_elem_ops", C.c_int64), ("kernel_launches", C.c_int64),
                ("steps", C.c_int64), ("similarity_tc_launches", C.c_int64), ("persistent_sweep_ns", C.c_int64),
                ("persistent_pick_ns", C.c_int64), ("threshold_hits", C.c_int64),
                ("threshold_elems", C.c_int64), ("threshold_max_blocks", C.c_int64),
                ("async_lull_ns", C.c_int64), ("async_visits", C.c_int64), ("async_attempts", C.c_int64),
                ("lazy_sweeps", C.c_int64), ("lazy_misses", C.c_int64), ("lazy_rows", C.c_int64),
                ("lazy_rows_skipped", C.c_int64), ("incremental_updates", C.c_int64), ("incremental_rows", C.c_int64), ("threshold_pass_ns", C.c_int64), ("threshold_pass_bytes", C.c_int64), ("noted_picks", C.c_int64),
                ("greedy_form", C.c_int64), ("round_lists", C.c_int64), ("round_tiles", C.c_int64)]


class RcdNormArgs(C.Structure):
    _fields_ = [("rows", C.c_int64), ("d", C.c_int64), ("x_type", C.c_int), ("x", C.c_void_p), ("ldx", C.c_int64),
                ("residual", C.c_void_p), ("ld_residual", C.c_int64), ("weight", C.c_void_p), ("weight_type", C.c_int),
                ("eps", C.c_float), ("sum", C.c_void_p), ("ld_sum", C.c_int64), ("y_type", C.c_int), ("y", C.c_void_p),
                ("ldy", C.c_int64), ("scale", C.c_float), ("scales", C.c_void_p)]


class RcdNormBackArgs(C.Structure):
    _fields_ = [("rows", C.c_int64), ("d", C.c_int64), ("type", C.c_int), ("dy", C.c_void_p), ("ld_dy", C.c_int64),
                ("h", C.c_void_p), ("ld_h", C.c_int64), ("weight", C.c_void_p), ("weight_type", C.c_int), ("eps", C.c_float),
                ("dsum", C.c_void_p), ("ld_dsum", C.c_int64), ("dx", C.c_void_p), ("ld_dx", C.c_int64), ("dweight", C.c_void_p)]


class RcdLinearArgs(C.Structure):
    _fields_ = [("rows", C.c_int64), ("n", C.c_int64), ("k", C.c_int64), ("type", C.c_int), ("x", C.c_void_p), ("ldx", C.c_int64),
                ("w", C.c_void_p), ("ldw", C.c_int64), ("x_scales", C.c_void_p), ("w_scales", C.c_void_p), ("bias", C.c_void_p),
                ("activation", C.c_int), ("residual", C.c_void_p), ("ld_residual", C.c_int64), ("y_type", C.c_int),
                ("y", C.c_void_p), ("ldy", C.c_int64), ("preact", C.c_void_p), ("ld_preact", C.c_int64)]


class RcdLinearBackArgs(C.Structure):
    _fields_ = [("rows", C.c_int64), ("n", C.c_int64), ("k", C.c_int64), ("type", C.c_int), ("dy", C.c_void_p), ("ld_dy", C.c_int64),
                ("x", C.c_void_p), ("ldx", C.c_int64), ("w", C.c_void_p), ("ldw", C.c_int64), ("activation", C.c_int),
                ("preact", C.c_void_p), ("ld_preact", C.c_int64), ("dx", C.c_void_p), ("ld_dx", C.c_int64), ("dw_type", C.c_int),
                ("dw", C.c_void_p), ("ld_dw", C.c_int64), ("dbias", C.c_void_p)]


class RcdCrossEntropyArgs(C.Structure):
    _fields_ = [("rows", C.c_int64), ("n", C.c_int64), ("k", C.c_int64), ("type", C.c_int), ("x", C.c_void_p), ("ldx", C.c_int64),
                ("w", C.c_void_p), ("ldw", C.c_int64), ("bias", C.c_void_p), ("labels", C.c_void_p), ("loss", C.c_void_p), ("lse", C.c_void_p)]


class RcdCrossEntropyBackArgs(C.Structure):
    _fields_ = [("rows", C.c_int64), ("n", C.c_int64), ("k", C.c_int64), ("type", C.c_int), ("x", C.c_void_p), ("ldx", C.c_int64),
                ("w", C.c_void_p), ("ldw", C.c_int64), ("bias", C.c_void_p), ("labels", C.c_void_p), ("lse", C.c_void_p), ("dloss", C.c_void_p),
                ("dlse", C.c_void_p), ("piece", C.c_int64), ("dx", C.c_void_p), ("ld_dx", C.c_int64), ("dw_type", C.c_int), ("dw", C.c_void_p),
                ("ld_dw", C.c_int64), ("dbias", C.c_void_p)]


class RcdOrthogonalizeArgs(C.Structure):
    _fields_ = [("batch", C.c_int64), ("rows", C.c_int64), ("cols", C.c_int64), ("type", C.c_int), ("g", C.c_void_p), ("ld_g", C.c_int64),
                ("step_g", C.c_int64), ("steps", C.c_int32), ("coefficients_host", C.c_void_p), ("eps", C.c_float), ("o", C.c_void_p),
                ("ld_o", C.c_int64), ("step_o", C.c_int64)]


def _load() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError("%s is missing: build it with `python -m paper_2211_00839_b200.build` "
                          "(there is no CPU fallback)" % LIB_PATH)
    lib = C.CDLL(LIB_PATH)
    vp, i64, i32, sz = C.c_void_p, C.c_int64, C.c_int32, C.c_size_t
    lib.rcd_create.argtypes = [C.POINTER(vp), C.c_int, C.POINTER(RcdConfig)]
    lib.rcd_destroy.argtypes = [vp]
    lib.rcd_destroy.restype = None
    lib.rcd_last_error.argtypes = [vp]
    lib.rcd_last_error.restype = C.c_char_p
    lib.rcd_version.argtypes = []
    lib.rcd_version.restype = C.c_char_p
    lib.rcd_sync_status.argtypes = [vp, vp]
    lib.rcd_selftest_bounded_wait.argtypes = [vp, vp]
    lib.rcd_get_profile.argtypes = [vp, C.POINTER(RcdProfile)]
    lib.rcd_quotas.argtypes = [i64, vp, i32, vp]
    lib.rcd_similarity.argtypes = [vp, vp, C.c_int, i64, i64, i64, vp, i64, vp]
    lib.rcd_similarity_gaussian_workspace_bytes.argtypes = [vp, i64, i64, C.POINTER(sz)]
    lib.rcd_similarity_gaussian.argtypes = [vp, vp, C.c_int, i64, i64, i64, vp, i64, vp, vp, sz, vp]
    for name in ("rcd_partition_workspace_bytes", "rcd_partition_host_workspace_bytes",
                 "rcd_objective_workspace_bytes"):
        getattr(lib, name).argtypes = [vp, C.c_int, i64, i64, i32, i64, i32, C.POINTER(sz)]
    lib.rcd_partition.argtypes = [vp, vp, C.c_int, i64, i64, vp, i32, vp, i32, vp, vp, vp, vp, sz, vp]
    lib.rcd_partition_host.argtypes = [vp, vp, C.c_int, i64, i64, vp, i32, vp, i32, vp, vp, vp, vp, sz, vp]
    lib.rcd_objective.argtypes = [vp, vp, C.c_int, i64, i64, vp, i32, vp, i32, vp, vp, vp, sz, vp]
    lib.rcd_objective_class_static.argtypes = [vp, vp, C.c_int, i64, i64, vp, i32, vp, vp, vp]
    lib.rcd_worker_lists_workspace_bytes.argtypes = [vp, i64, i32, C.POINTER(sz)]
    lib.rcd_worker_lists.argtypes = [vp, vp, i64, i32, vp, vp, vp, sz, vp]
    lib.rcd_batch_sizes.argtypes = [i64, vp, i32, vp]
    lib.rcd_batch_sizes_rule.argtypes = [i64, vp, i32, C.c_int, vp]
    lib.rcd_rms_norm.argtypes = [vp, C.POINTER(RcdNormArgs), vp]
    lib.rcd_quantize_rows.argtypes = [vp, vp, C.c_int, i64, i64, i64, vp, i64, vp, vp]
    lib.rcd_rms_norm_backward_workspace_bytes.argtypes = [vp, C.POINTER(RcdNormBackArgs), C.POINTER(sz)]
    lib.rcd_rms_norm_backward.argtypes = [vp, C.POINTER(RcdNormBackArgs), vp, sz, vp]
    lib.rcd_linear_workspace_bytes.argtypes = [vp, C.POINTER(RcdLinearArgs), C.POINTER(sz)]
    lib.rcd_linear.argtypes = [vp, C.POINTER(RcdLinearArgs), vp, sz, vp]
    lib.rcd_linear_backward_workspace_bytes.argtypes = [vp, C.POINTER(RcdLinearBackArgs), C.POINTER(sz)]
    lib.rcd_linear_backward.argtypes = [vp, C.POINTER(RcdLinearBackArgs), vp, sz, vp]
    lib.rcd_linear_cross_entropy_workspace_bytes.argtypes = [vp, C.POINTER(RcdCrossEntropyArgs), C.POINTER(sz)]
    lib.rcd_linear_cross_entropy.argtypes = [vp, C.POINTER(RcdCrossEntropyArgs), vp, sz, vp]
    lib.rcd_linear_cross_entropy_backward_workspace_bytes.argtypes = [vp, C.POINTER(RcdCrossEntropyBackArgs), C.POINTER(sz)]
    lib.rcd_linear_cross_entropy_backward.argtypes = [vp, C.POINTER(RcdCrossEntropyBackArgs), vp, sz, vp]
    lib.rcd_orthogonalize_workspace_bytes.argtypes = [vp, C.POINTER(RcdOrthogonalizeArgs), C.POINTER(sz)]
    lib.rcd_orthogonalize.argtypes = [vp, C.POINTER(RcdOrthogonalizeArgs), vp, sz, vp]
    lib.rcd_yardstick_read.argtypes = [vp, vp, sz, i32, vp]
    lib.rcd_yardstick_mma.argtypes = [vp, C.c_int, i32, C.POINTER(C.c_double), vp]
    for name in EXPORTS:
        f = getattr(lib, name)
        if name not in ("rcd_destroy", "rcd_last_error", "rcd_version"):
            f.restype = C.c_int
    return lib


lib = _load()


def rcd_version() -> str:
    return lib.rcd_version().decode()


def rcd_quotas(M: int, capacities: Sequence[float]) -> np.ndarray:
    """Integer quotas of one class (host only; no GPU needed)."""
    r = np.ascontiguousarray(capacities, dtype=np.float64)
    out = np.empty(len(r), dtype=np.int32)
    st = lib.rcd_quotas(int(M), r.ctypes.data_as(C.c_void_p), len(r), out.ctypes.data_as(C.c_void_p))
    if st != 0:
        raise RcdError(st, "rcd_quotas")
    return out


RCD_BATCH_PROPORTIONAL = 0
RCD_BATCH_AS_PRINTED = 1


def rcd_batch_sizes(B: int, capacities: Sequence[float], rule: int = RCD_BATCH_PROPORTIONAL) -> np.ndarray:
    """Per-worker batch sizes (host only; no GPU needed): b_j = B r_j / r_1, or with
    ``rule=RCD_BATCH_AS_PRINTED`` the ratio as Algorithm 2 prints it, B r_1 / r_j."""
    r = np.ascontiguousarray(capacities, dtype=np.float64)
    out = np.empty(len(r), dtype=np.int64)
    if rule == RCD_BATCH_PROPORTIONAL:
        st = lib.rcd_batch_sizes(int(B), r.ctypes.data_as(C.c_void_p), len(r), out.ctypes.data_as(C.c_void_p))
    else:
        st = lib.rcd_batch_sizes_rule(int(B), r.ctypes.data_as(C.c_void_p), len(r), int(rule), out.ctypes.data_as(C.c_void_p))
    if st != 0:
        raise RcdError(st, "rcd_batch_sizes")
    return out


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _dtype_code(t) -> int:
    torch = _torch()
    if t.dtype == torch.int8:
        return RCD_FEAT_I8
    if t.dtype == torch.bfloat16:
        return RCD_FEAT_BF16
    raise TypeError("features must be torch.int8 or torch.bfloat16, got %s" % t.dtype)


_ELEM = {}


def _elem(dtype, name: str) -> int:
    if not _ELEM:
        torch = _torch()
        _ELEM.update({torch.int8: RCD_ELEM_I8, torch.bfloat16: RCD_ELEM_BF16, torch.float16: RCD_ELEM_F16, torch.float32: RCD_ELEM_F32})
    code = _ELEM.get(dtype)
    if code is None:
        raise TypeError("%s must be int8, bfloat16, float16 or float32, got %s" % (name, dtype))
    return code


def features_to_torch(features: np.ndarray, device=None, pin: bool = False):
    """numpy int8, or uint16 bf16 bit patterns -> torch int8 / bfloat16 tensor (optionally pinned / on device)."""
    torch = _torch()
    if features.dtype == np.int8:
        t = torch.from_numpy(np.ascontiguousarray(features))
    elif features.dtype == np.uint16:
        t = torch.from_numpy(np.ascontiguousarray(features).view(np.int16)).view(torch.bfloat16)
    else:
        raise TypeError("features must be int8 or uint16 (bf16 bits)")
    if pin:
        t = t.pin_memory()
    if device is not None:
        t = t.to(device)
    return t


class Context:
    """Owns one ``rcd_ctx`` on a CUDA device."""

    def __init__(self, device: int = 0, sweep_batch_max: int = 0, similarity_path: int = 0, profile: int = 0,
                 greedy_path: int = 0, similarity_kind: int = 0, objective: int = 0, sweep_mode: int = 0,
                 async_group: int = 0, async_help_min: int = 0, threshold_from: int = 0, threshold_hit_shift: int = 0,
                 lazy_mode: int = 0, lazy_from: int = 0, dense_ring: int = 0, incremental: int = 0, incremental_max: int = 0):
        torch = _torch()
        if not torch.cuda.is_available():
            raise RcdError(4, "no CUDA device: this library has no CPU path")
        self.device = int(device)
        self.torch_device = torch.device("cuda", self.device)
        cfg = RcdConfig()
        cfg.sweep_batch_max = sweep_batch_max
        cfg.similarity_path = similarity_path
        cfg.profile = profile
        cfg.greedy_path = greedy_path
        cfg.similarity_kind = similarity_kind
        cfg.objective = objective
        cfg.sweep_mode = sweep_mode
        cfg.async_group = async_group
        cfg.async_help_min = async_help_min
        cfg.threshold_from = threshold_from
        cfg.threshold_hit_shift = threshold_hit_shift
        cfg.lazy_mode = lazy_mode
        cfg.lazy_from = lazy_from
        cfg.dense_ring = dense_ring
        cfg.incremental = incremental
        cfg.incremental_max = incremental_max
        self.similarity_kind = similarity_kind
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self._h = C.c_void_p()
        st = lib.rcd_create(C.byref(self._h), self.device, C.byref(cfg))
        if st != 0:
            raise RcdError(st, "rcd_create")
        self._ws = None

    def close(self):
        if getattr(self, "_h", None) is not None and self._h:
            lib.rcd_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    # -- helpers
    def _check(self, st: int):
        if st != 0:
            raise RcdError(st, lib.rcd_last_error(self._h).decode())

    def _stream(self):
        # (the raw handle where this torch gives it: a Stream object is a tenth of a small call's time)
        raw = self._raw_stream
        return C.c_void_p(raw(self.device) if raw is not None else _torch().cuda.current_stream(self.torch_device).cuda_stream)

    def workspace(self, nbytes: int):
        """A cached uint8 device tensor of at least ``nbytes`` (torch's allocator aligns it to 512 bytes)."""
        torch = _torch()
        if self._ws is None or self._ws.numel() < nbytes:
            self._ws = None
            self._ws = torch.empty(int(nbytes), dtype=torch.uint8, device=self.torch_device)
        return self._ws

    def selftest_bounded_wait(self):
        """Enqueue the wait that can never be satisfied; the following sync_status() raises RCD_ERR_TIMEOUT."""
        self._check(lib.rcd_selftest_bounded_wait(self._h, self._stream()))

    def sync_status(self):
        """Waits for the current stream and raises what the last call recorded on the device, or any norm or product since it was last asked."""
        self._check(lib.rcd_sync_status(self._h, self._stream()))

    def profile(self) -> Dict[str, float]:
        p = RcdProfile()
        self._check(lib.rcd_get_profile(self._h, C.byref(p)))
        return {k: getattr(p, k) for k, _ in RcdProfile._fields_ if k != "reserved"}

    # -- entry points
    def rcd_similarity(self, X):
        """X: [batch, M, d] (or [M, d]) int8 / bfloat16 on the device -> S [batch, M, ld] int32 / float32."""
        torch = _torch()
        if X.dim() == 2:
            X = X.unsqueeze(0)
        X = X.contiguous()
        batch, M, d = X.shape
        ld = (M + 3) // 4 * 4
        code = _dtype_code(X)
        S = torch.empty((batch, M, ld), dtype=torch.int32 if code == RCD_FEAT_I8 else torch.float32,
                        device=X.device)
        self._check(lib.rcd_similarity(self._h, C.c_void_p(X.data_ptr()), code, M, d, batch,
                                       C.c_void_p(S.data_ptr()), ld, self._stream()))
        return S

    def _value_dtype(self, code: int):
        torch = _torch()
        return torch.int64 if (code == RCD_FEAT_I8 and self.similarity_kind == RCD_SIM_DOT) else torch.float64

    def rcd_similarity_gaussian(self, X):
        """X: [batch, M, d] (or [M, d]) int8 / bfloat16 on the device -> (S [batch, M, ld] float32, sigma [batch] float32)."""
        torch = _torch()
        if X.dim() == 2:
            X = X.unsqueeze(0)
        X = X.contiguous()
        batch, M, d = X.shape
        ld = (M + 3) // 4 * 4
        code = _dtype_code(X)
        S = torch.empty((batch, M, ld), dtype=torch.float32, device=X.device)
        sigma = torch.empty(batch, dtype=torch.float32, device=X.device)
        need = C.c_size_t()
        self._check(lib.rcd_similarity_gaussian_workspace_bytes(self._h, M, batch, C.byref(need)))
        ws = self.workspace(int(need.value))
        self._check(lib.rcd_similarity_gaussian(self._h, C.c_void_p(X.data_ptr()), code, M, d, batch,
                                                C.c_void_p(S.data_ptr()), ld, C.c_void_p(sigma.data_ptr()),
                                                C.c_void_p(ws.data_ptr()), ws.numel(), self._stream()))
        return S, sigma

    def partition_workspace_bytes(self, code: int, N: int, d: int, L: int, M_max: int, W: int, host: bool = False) -> int:
        out = C.c_size_t()
        fn = lib.rcd_partition_host_workspace_bytes if host else lib.rcd_partition_workspace_bytes
        self._check(fn(self._h, code, N, d, L, M_max, W, C.byref(out)))
        return int(out.value)

    def features(self, hidden, kind: int = RCD_FEAT_BF16, scale: float = RCD_FEATURE_SCALE):
        """Rows as they come (bfloat16, float16 or float32 [N, d]) to what a partition reads, by ``rcd_rms_norm`` without eps:
        ``RCD_FEAT_BF16`` L2-normalised rows (products are cosines), ``RCD_FEAT_I8`` rows of root mean square 1 as int8 on the one
        ``scale`` (cut off at 127 of it).  A row of zeros stays one."""
        torch = _torch()
        if hidden.dim() != 2:
            raise ValueError("features are rows: [N, d], got %s" % (tuple(hidden.shape),))
        if kind == RCD_FEAT_I8:
            return self.rcd_rms_norm(hidden, eps=0.0, out_dtype=torch.int8, scale=scale)[0]
        if kind != RCD_FEAT_BF16:
            raise ValueError("kind must be RCD_FEAT_I8 or RCD_FEAT_BF16")
        unit = torch.full((hidden.shape[1],), float(hidden.shape[1]) ** -0.5, dtype=torch.float32, device=self.torch_device)
        return self.rcd_rms_norm(hidden, weight=unit, eps=0.0, out_dtype=torch.bfloat16)[0]

    def rcd_partition(self, features, labels, capacities: Sequence[float], L: int, M_max: Optional[int] = None,
                      want_order: bool = True, want_values: bool = True, normalize: Optional[int] = None):
        """Device tensors in, device tensors out: (assignment[N] int32, order[N] int32 | None, part_values[L,W] | None).

        ``normalize`` (RCD_FEAT_BF16 or RCD_FEAT_I8): the features are rows as they come, see ``features``.
        Enqueues on the current torch stream; call ``sync_status()`` (or synchronise) before reading."""
        torch = _torch()
        if normalize is not None:
            features = self.features(features, normalize)
        features = features.contiguous()
        labels = labels.contiguous()
        assert labels.dtype == torch.int32 and labels.is_cuda and features.is_cuda
        N, d = features.shape
        code = _dtype_code(features)
        caps = np.ascontiguousarray(capacities, dtype=np.float64)
        W = len(caps)
        if M_max is None:
            M_max = N
        nbytes = self.partition_workspace_bytes(code, N, d, L, M_max, W)
        ws = self.workspace(nbytes)
        assignment = torch.empty(N, dtype=torch.int32, device=features.device)
        order = torch.empty(N, dtype=torch.int32, device=features.device) if want_order else None
        values = None
        if want_values:
            values = torch.empty((L, W), dtype=self._value_dtype(code), device=features.device)
        self._check(lib.rcd_partition(self._h, C.c_void_p(features.data_ptr()), code, N, d,
                                      C.c_void_p(labels.data_ptr()), L, caps.ctypes.data_as(C.c_void_p), W,
                                      C.c_void_p(assignment.data_ptr()),
                                      C.c_void_p(order.data_ptr()) if order is not None else None,
                                      C.c_void_p(values.data_ptr()) if values is not None else None,
                                      C.c_void_p(ws.data_ptr()), ws.numel(), self._stream()))
        return assignment, order, values

    def rcd_partition_host(self, features, labels, capacities: Sequence[float], L: int, M_max: Optional[int] = None,
                           out: Optional[Tuple] = None):
        """Host tensors in (torch CPU tensors, ideally pinned), host tensors out; copies run inside the call.

        Returns (assignment[N] int32, order[N] int32, part_values[L,W]) as torch CPU tensors (pinned)."""
        torch = _torch()
        assert not features.is_cuda and not labels.is_cuda and labels.dtype == torch.int32
        features = features.contiguous()
        labels = labels.contiguous()
        N, d = features.shape
        code = _dtype_code(features)
        caps = np.ascontiguousarray(capacities, dtype=np.float64)
        W = len(caps)
        if M_max is None:
            M_max = N
        nbytes = self.partition_workspace_bytes(code, N, d, L, M_max, W, host=True)
        ws = self.workspace(nbytes)
        if out is None:
            assignment = torch.empty(N, dtype=torch.int32).pin_memory()
            order = torch.empty(N, dtype=torch.int32).pin_memory()
            values = torch.empty((L, W), dtype=self._value_dtype(code)).pin_memory()
        else:
            assignment, order, values = out
        with torch.cuda.device(self.torch_device):
            self._check(lib.rcd_partition_host(self._h, C.c_void_p(features.data_ptr()), code, N, d,
                                               C.c_void_p(labels.data_ptr()), L, caps.ctypes.data_as(C.c_void_p), W,
                                               C.c_void_p(assignment.data_ptr()), C.c_void_p(order.data_ptr()),
                                               C.c_void_p(values.data_ptr()), C.c_void_p(ws.data_ptr()), ws.numel(),
                                               self._stream()))
        return assignment, order, values

    def rcd_objective(self, features, labels, assignment, W: int, L: int, M_max: Optional[int] = None, normalize: Optional[int] = None):
        """f(A_j^l) from the plain definition for a given assignment -> (part_values[L,W], total[1]); ``normalize`` as for rcd_partition."""
        torch = _torch()
        if normalize is not None:
            features = self.features(features, normalize)
        features = features.contiguous()
        labels = labels.contiguous()
        assignment = assignment.contiguous()
        N, d = features.shape
        code = _dtype_code(features)
        if M_max is None:
            M_max = N
        out = C.c_size_t()
        self._check(lib.rcd_objective_workspace_bytes(self._h, code, N, d, L, M_max, W, C.byref(out)))
        ws = self.workspace(int(out.value))
        vdt = self._value_dtype(code)
        values = torch.empty((L, W), dtype=vdt, device=features.device)
        total = torch.empty(1, dtype=vdt, device=features.device)
        self._check(lib.rcd_objective(self._h, C.c_void_p(features.data_ptr()), code, N, d,
                                      C.c_void_p(labels.data_ptr()), L, C.c_void_p(assignment.data_ptr()), W,
                                      C.c_void_p(values.data_ptr()), C.c_void_p(total.data_ptr()),
                                      C.c_void_p(ws.data_ptr()), ws.numel(), self._stream()))
        return values, total

    # -- from hidden states to features.  (None of these calls is recorded by autograd, also where an argument requires a gradient: the
    # gradients are the calls' own _backward, which a torch.autograd.Function of the program's can call.)
    def _rows(self, t, name: str, d: Optional[int] = None, rows: Optional[int] = None, dtype=None):
        """A tensor [..., d] on this context's device as (tensor to keep alive, rows, d, elements between rows)."""
        if t.device != self.torch_device:
            raise ValueError("%s is on %s, the context on %s" % (name, t.device, self.torch_device))
        if dtype is not None and t.dtype != dtype:
            raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
        if t.dim() != 2:
            if t.dim() == 0:
                raise ValueError("%s has no dimension" % name)
            t = t.reshape(math.prod(t.shape[:-1]), t.shape[-1])
        r, n = t.shape
        if (d is not None and n != d) or (rows is not None and r != rows):
            raise ValueError("%s has shape %s, expected %s rows of %s" % (name, tuple(t.shape), r if rows is None else rows, n if d is None else d))
        s0, s1 = t.stride()
        if (n > 1 and s1 != 1) or (r > 1 and s0 < n):
            t = t.contiguous()
            s0 = n
        return t, r, n, (s0 if s0 > n else n)

    def _vector(self, t, name: str, n: int, dtype=None):
        if t.device != self.torch_device:
            raise ValueError("%s is on %s, the context on %s" % (name, t.device, self.torch_device))
        if dtype is not None and t.dtype != dtype:
            raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
        if t.dim() != 1 or t.shape[0] != n:
            raise ValueError("%s has shape %s, expected (%d,)" % (name, tuple(t.shape), n))
        return t if t.stride(0) == 1 or n <= 1 else t.contiguous()

    def _out(self, t, name: str, shape, dtype):
        """A caller's output: it is written in place, so nothing about it is put right."""
        if t.device != self.torch_device or t.dtype != dtype or tuple(t.shape) != tuple(shape):
            raise ValueError("%s must be %s of shape %s on %s" % (name, dtype, tuple(shape), self.torch_device))
        if t.dim() == 1:
            if t.stride(0) != 1 and t.shape[0] > 1:
                raise ValueError("%s must be dense" % name)
            return t.shape[0]
        if t.dim() > 2 and not t.is_contiguous():
            raise ValueError("%s must be dense" % name)
        s0, s1 = t.stride()[-2:]
        if (t.shape[-1] > 1 and s1 != 1) or (t.shape[-2] > 1 and s0 < t.shape[-1]):
            raise ValueError("%s: the elements of a row must lie next to each other" % name)
        return max(s0, t.shape[-1])

    def _scratch(self, nbytes: int):
        """A workspace of this call alone: a captured graph keeps its own, whatever other calls do."""
        return _torch().empty(nbytes, dtype=_torch().uint8, device=self.torch_device) if nbytes else None

    def rcd_rms_norm(self, x, residual=None, weight=None, eps: float = 1e-6, out_dtype=None, scale: Optional[float] = None,
                     want_sum: bool = False, out=None, sum_out=None):
        """y = h * weight / sqrt(mean(h^2) + eps), h = x + residual, for rows [..., d] in bfloat16, float16 or float32.

        ``out_dtype`` (default: x's) may be int8: with a scale per row, or all rows on the one ``scale``.  Returns
        (y, scales [rows] | None, h rounded to x's type | None).  ``out`` and ``sum_out`` take y and h in place of new tensors;
        ``sum_out`` may be ``x`` or ``residual`` itself.  Autograd does not record the call: ``rcd_rms_norm_backward`` is its gradient."""
        torch = _torch()
        a = RcdNormArgs()
        kept, rows, d, a.ldx = self._rows(x, "x")
        a.rows, a.d, a.x_type, a.x = rows, d, _elem(x.dtype, "x"), kept.data_ptr()
        keep = [kept]
        if residual is not None:
            r, _, _, a.ld_residual = self._rows(residual, "residual", d, rows, x.dtype)
            a.residual = r.data_ptr()
            keep.append(r)
        if weight is not None:
            w = self._vector(weight, "weight", d)
            a.weight, a.weight_type = w.data_ptr(), _elem(w.dtype, "weight")
            keep.append(w)
        a.eps = eps
        kind = (x.dtype if out_dtype is None else out_dtype) if out is None else out.dtype
        a.y_type = _elem(kind, "out_dtype")
        y = (x.new_empty(x.shape) if kind == x.dtype else x.new_empty(x.shape, dtype=kind)) if out is None else out
        a.ldy = d if out is None else self._out(out, "out", x.shape, kind if out_dtype is None else out_dtype)
        a.y = y.data_ptr()
        scales = total = None
        if scale is not None:
            if not scale > 0.0:
                raise ValueError("scale must be positive")
            a.scale = scale
        elif a.y_type == RCD_ELEM_I8:
            scales = torch.empty(rows, dtype=torch.float32, device=self.torch_device)
            a.scales = scales.data_ptr()
        if want_sum or sum_out is not None:
            total = x.new_empty(x.shape) if sum_out is None else sum_out
            a.ld_sum = d if sum_out is None else self._out(sum_out, "sum_out", x.shape, x.dtype)
            a.sum = total.data_ptr()
        self._check(lib.rcd_rms_norm(self._h, C.byref(a), self._stream()))
        return y, scales, total

    def rcd_quantize_rows(self, x):
        """Rows [..., d] to (int8 of the same shape, scales [rows] float32): x is about q * scale of its row."""
        torch = _torch()
        kept, rows, d, ld = self._rows(x, "x")
        q = torch.empty(x.shape, dtype=torch.int8, device=self.torch_device)
        scales = torch.empty(rows, dtype=torch.float32, device=self.torch_device)
        self._check(lib.rcd_quantize_rows(self._h, kept.data_ptr(), _elem(x.dtype, "x"), rows, d, ld, q.data_ptr(), d,
                                          scales.data_ptr(), self._stream()))
        return q, scales

    def rcd_rms_norm_backward(self, dy, h, weight=None, eps: float = 1e-6, dsum=None, want_dweight: bool = True):
        """Gradients of ``rcd_rms_norm``'s y from dy: (dx, which is the residual's gradient too, dweight [d] float32 | None).

        ``h``: the sum that ``rcd_rms_norm`` returned, or its x; ``dsum``: the gradient that reaches h from elsewhere."""
        torch = _torch()
        a = RcdNormBackArgs()
        hk, rows, d, a.ld_h = self._rows(h, "h")
        yk, _, _, a.ld_dy = self._rows(dy, "dy", d, rows, h.dtype)
        a.rows, a.d, a.type, a.h, a.dy, a.eps = rows, d, _elem(h.dtype, "h"), hk.data_ptr(), yk.data_ptr(), eps
        keep = [hk, yk]
        if weight is not None:
            w = self._vector(weight, "weight", d)
            a.weight, a.weight_type = w.data_ptr(), _elem(w.dtype, "weight")
            keep.append(w)
        if dsum is not None:
            s, _, _, a.ld_dsum = self._rows(dsum, "dsum", d, rows, h.dtype)
            a.dsum = s.data_ptr()
            keep.append(s)
        dx = torch.empty(h.shape, dtype=h.dtype, device=self.torch_device)
        a.dx, a.ld_dx = dx.data_ptr(), d
        dw = None
        if weight is not None and want_dweight:
            dw = torch.empty(d, dtype=torch.float32, device=self.torch_device)
            a.dweight = dw.data_ptr()
        need = C.c_size_t()
        self._check(lib.rcd_rms_norm_backward_workspace_bytes(self._h, C.byref(a), C.byref(need)))
        ws = self._scratch(need.value)
        self._check(lib.rcd_rms_norm_backward(self._h, C.byref(a), ws.data_ptr() if ws is not None else None, need.value, self._stream()))
        return dx, dw

    def rcd_linear(self, x, w, bias=None, residual=None, activation: int = RCD_ACT_NONE, x_scales=None, w_scales=None,
                   out_dtype=None, want_preact: bool = False, out=None):
        """act(x w^T + bias) + residual for x [..., k] and w [n, k] in bfloat16, float16 or int8 (x_scales [rows], w_scales [n]).

        bias: float32 [n]; residual: [..., n] in the output's type; ``out_dtype``: default x's type, bfloat16 for int8.
        Returns (y [..., n], the values before the activation | None).  Autograd does not record the call: ``rcd_linear_backward`` is its
        gradient (bfloat16 and float16)."""
        torch = _torch()
        a = RcdLinearArgs()
        xk, rows, k, a.ldx = self._rows(x, "x")
        wk, n, _, a.ldw = self._rows(w, "w", k, None, x.dtype)
        if w.dim() != 2:
            raise ValueError("w must be [n, k]")
        a.rows, a.n, a.k, a.type, a.x, a.w, a.activation = rows, n, k, _elem(x.dtype, "x"), xk.data_ptr(), wk.data_ptr(), activation
        keep = [xk, wk]
        if out is not None:
            kind = out.dtype
        else:
            kind = out_dtype if out_dtype is not None else torch.bfloat16 if x.dtype == torch.int8 else x.dtype
        a.y_type = _elem(kind, "out_dtype")
        shape = (*x.shape[:-1], n)
        y = (x.new_empty(shape) if kind == x.dtype else x.new_empty(shape, dtype=kind)) if out is None else out
        a.ldy = n if out is None else self._out(out, "out", shape, kind if out_dtype is None else out_dtype)
        a.y = y.data_ptr()
        if bias is not None:
            b = self._vector(bias, "bias", n, torch.float32)
            a.bias = b.data_ptr()
            keep.append(b)
        if x_scales is not None:
            b = self._vector(x_scales, "x_scales", rows, torch.float32)
            a.x_scales = b.data_ptr()
            keep.append(b)
        if w_scales is not None:
            b = self._vector(w_scales, "w_scales", n, torch.float32)
            a.w_scales = b.data_ptr()
            keep.append(b)
        if residual is not None:
            r, _, _, a.ld_residual = self._rows(residual, "residual", n, rows, kind)
            a.residual = r.data_ptr()
            keep.append(r)
        pre = None
        if want_preact:
            pre = torch.empty(shape, dtype=kind, device=self.torch_device)
            a.preact, a.ld_preact = pre.data_ptr(), n
        need = C.c_size_t()
        self._check(lib.rcd_linear_workspace_bytes(self._h, C.byref(a), C.byref(need)))
        ws = self._scratch(need.value)
        self._check(lib.rcd_linear(self._h, C.byref(a), ws.data_ptr() if ws is not None else None, need.value, self._stream()))
        return y, pre

    def rcd_linear_backward(self, dy, x, w, preact=None, activation: int = RCD_ACT_NONE, dw_dtype=None, want_dx: bool = True,
                            want_dw: bool = True, want_dbias: bool = True):
        """Gradients of ``rcd_linear`` (bfloat16 or float16, no scales) from dy [..., n]: (dx [..., k], dw [n, k], dbias [n] float32),
        None where not wanted.  ``preact``: the values before the activation that ``rcd_linear`` returned; the residual's gradient is dy.
        ``dw_dtype``: default x's type, or float32."""
        torch = _torch()
        a = RcdLinearBackArgs()
        xk, rows, k, a.ldx = self._rows(x, "x")
        wk, n, _, a.ldw = self._rows(w, "w", k, None, x.dtype)
        if w.dim() != 2:
            raise ValueError("w must be [n, k]")
        yk, _, _, a.ld_dy = self._rows(dy, "dy", n, rows, x.dtype)
        a.rows, a.n, a.k, a.type, a.x, a.w, a.dy, a.activation = rows, n, k, _elem(x.dtype, "x"), xk.data_ptr(), wk.data_ptr(), yk.data_ptr(), activation
        keep = [xk, wk, yk]
        if preact is not None:
            z, _, _, a.ld_preact = self._rows(preact, "preact", n, rows, x.dtype)
            a.preact = z.data_ptr()
            keep.append(z)
        dx = dw = db = None
        if want_dx:
            dx = torch.empty(x.shape, dtype=x.dtype, device=self.torch_device)
            a.dx, a.ld_dx = dx.data_ptr(), k
        kind = x.dtype if dw_dtype is None else dw_dtype
        a.dw_type = _elem(kind, "dw_dtype")
        if want_dw:
            dw = torch.empty((n, k), dtype=kind, device=self.torch_device)
            a.dw, a.ld_dw = dw.data_ptr(), k
        if want_dbias:
            db = torch.empty(n, dtype=torch.float32, device=self.torch_device)
            a.dbias = db.data_ptr()
        need = C.c_size_t()
        self._check(lib.rcd_linear_backward_workspace_bytes(self._h, C.byref(a), C.byref(need)))
        ws = self._scratch(need.value)
        self._check(lib.rcd_linear_backward(self._h, C.byref(a), ws.data_ptr() if ws is not None else None, need.value, self._stream()))
        return dx, dw, db


    # -- training a head or a projection.  (Not recorded by autograd either.)
    def _per_row(self, t, name: str, shape, dtype):
        """One value for every row of x: a tensor of x's leading dimensions, dense."""
        if t.device != self.torch_device:
            raise ValueError("%s is on %s, the context on %s" % (name, t.device, self.torch_device))
        if t.dtype != dtype:
            raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
        if t.shape != shape:
            raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
        return t if t.is_contiguous() else t.contiguous()

    def rcd_linear_cross_entropy(self, x, w, labels, bias=None):
        """Softmax cross entropy of the head x w^T + bias on the samples' labels, without its logits in memory: (loss, lse), float32 of the rows' shape.

        x [..., k] and w [n, k] in bfloat16 or float16, labels [...] int32 (a negative one: the row is passed over), bias [n] float32 (-inf closes
        a class).  lse is the log of the sum of exponentials, which ``rcd_linear_cross_entropy_backward`` reads.  Autograd does not record the call."""
        torch = _torch()
        f32 = torch.float32
        xk, rows, k, ldx = self._rows(x, "x")
        if w.dim() != 2:
            raise ValueError("w must be [n, k]")
        wk, n, _, ldw = self._rows(w, "w", k, None, x.dtype)
        shape = x.shape[:-1]
        lk = self._per_row(labels, "labels", shape, torch.int32)
        b = None if bias is None else self._vector(bias, "bias", n, f32)
        loss, lse = torch.empty_like(lk, dtype=f32), torch.empty_like(lk, dtype=f32)
        a = RcdCrossEntropyArgs(rows, n, k, _elem(x.dtype, "x"), xk.data_ptr(), ldx, wk.data_ptr(), ldw, None if b is None else b.data_ptr(), lk.data_ptr(),
                                loss.data_ptr(), lse.data_ptr())
        need = C.c_size_t()
        self._check(lib.rcd_linear_cross_entropy_workspace_bytes(self._h, C.byref(a), C.byref(need)))
        ws = self._scratch(need.value)
        self._check(lib.rcd_linear_cross_entropy(self._h, C.byref(a), ws.data_ptr() if ws is not None else None, need.value, self._stream()))
        return loss, lse

    def rcd_linear_cross_entropy_backward(self, x, w, labels, lse, bias=None, dloss=None, dlse=None, dw_dtype=None, want_dx: bool = True,
                                          want_dw: bool = True, want_dbias: bool = True, piece: int = 0):
        """Gradients of ``rcd_linear_cross_entropy`` from those of loss and lse ([...] float32; None: ones, zeros): (dx [..., k], dw [n, k],
        dbias [n] float32), None where not wanted.  lse: what the forward call returned for the same x, w and bias.

        The logits are made again, ``piece`` classes at a time (0: as many as take 512 MB of workspace), and their gradients rounded to x's type for dx and dw,
        not for dbias; with dbias dx and dw may differ in their last bits.  ``dw_dtype``: default x's type, or float32."""
        torch = _torch()
        f32 = torch.float32
        xk, rows, k, ldx = self._rows(x, "x")
        if w.dim() != 2:
            raise ValueError("w must be [n, k]")
        wk, n, _, ldw = self._rows(w, "w", k, None, x.dtype)
        shape = x.shape[:-1]
        lk, sk = self._per_row(labels, "labels", shape, torch.int32), self._per_row(lse, "lse", shape, f32)
        b = None if bias is None else self._vector(bias, "bias", n, f32)
        gk = None if dloss is None else self._per_row(dloss, "dloss", shape, f32)
        hk = None if dlse is None else self._per_row(dlse, "dlse", shape, f32)
        kind = x.dtype if dw_dtype is None else dw_dtype
        dx = x.new_empty(x.shape) if want_dx else None
        dw = (w.new_empty((n, k)) if kind == w.dtype else w.new_empty((n, k), dtype=kind)) if want_dw else None
        db = x.new_empty(n, dtype=f32) if want_dbias else None

        def at(t):
            return None if t is None else t.data_ptr()
        a = RcdCrossEntropyBackArgs(rows, n, k, _elem(x.dtype, "x"), xk.data_ptr(), ldx, wk.data_ptr(), ldw, at(b), lk.data_ptr(), sk.data_ptr(), at(gk), at(hk), piece,
                                    at(dx), k, _elem(kind, "dw_dtype"), at(dw), k, at(db))
        need = C.c_size_t()
        self._check(lib.rcd_linear_cross_entropy_backward_workspace_bytes(self._h, C.byref(a), C.byref(need)))
        ws = self._scratch(need.value)
        self._check(lib.rcd_linear_cross_entropy_backward(self._h, C.byref(a), ws.data_ptr() if ws is not None else None, need.value, self._stream()))
        return dx, dw, db

    def rcd_orthogonalize(self, g, steps: int = 5, coefficients=RCD_QUINTIC, eps: float = 1e-7, out=None):
        """A weight gradient with its singular values brought near one, bfloat16 of g's shape: g / |g|, then Newton-Schulz steps.

        g [..., rows, cols] in bfloat16, float16 or float32, every matrix by itself (``rcd_linear_backward``'s dw, or several stacked).
        ``coefficients``: (a, b, c) of every step, or a sequence of ``steps`` such.  ``out`` takes the result in place of a new tensor."""
        torch = _torch()
        if g.device != self.torch_device:
            raise ValueError("g is on %s, the context on %s" % (g.device, self.torch_device))
        if g.dim() < 2:
            raise ValueError("g must be [..., rows, cols], got shape %s" % (tuple(g.shape),))
        steps = int(steps)
        each = tuple(coefficients)
        if len(each) == 3 and not hasattr(each[0], "__len__"):
            each = (each,) * max(steps, 0)
        if len(each) != max(steps, 0) or any(len(c) != 3 for c in each):
            raise ValueError("coefficients must be (a, b, c), or %d of them" % steps)
        c = (C.c_float * (3 * len(each)))(*(v for abc in each for v in abc))

        def matrices(t):
            """(tensor, batch, elements from row to row and from matrix to matrix) of [..., rows, cols] as it lies, or None where its rows are not dense or its
            matrices not equally far apart."""
            rows, cols = t.shape[-2:]
            if t.is_contiguous():
                return t, math.prod(t.shape[:-2]), max(cols, 1), rows * cols
            if t.dim() > 3:
                v = t.flatten(0, -3)
                if v.data_ptr() != t.data_ptr():              # (a copy: no view of it has one leading dimension)
                    return None
                t = v
            s1, s2 = t.stride()[-2:]
            batch, s0 = (t.shape[0], t.stride(0)) if t.dim() == 3 else (1, 0)
            ld = max(s1, cols, 1) if rows > 1 else max(cols, 1)
            if (cols > 1 and s2 != 1) or (rows > 1 and s1 < cols) or (batch > 1 and s0 < (rows - 1) * ld + cols):
                return None
            return t, batch, ld, s0 if batch > 1 else rows * ld

        a = RcdOrthogonalizeArgs()
        v, a.batch, a.ld_g, a.step_g = matrices(g) or matrices(g.contiguous())
        a.rows, a.cols = g.shape[-2:]
        a.type, a.g, a.eps, a.steps, a.coefficients_host = _elem(g.dtype, "g"), v.data_ptr(), eps, steps, C.addressof(c)
        if out is None:
            out = g.new_empty(g.shape, dtype=torch.bfloat16)
        elif out.device != self.torch_device or out.dtype != torch.bfloat16 or out.shape != g.shape:
            raise ValueError("out must be bfloat16 of shape %s on %s" % (tuple(g.shape), self.torch_device))
        o = matrices(out)
        if o is None:
            raise ValueError("out: the elements of a row must lie next to each other, and its matrices equally far apart")
        _, _, a.ld_o, a.step_o = o
        a.o = out.data_ptr()
        need = C.c_size_t()
        self._check(lib.rcd_orthogonalize_workspace_bytes(self._h, C.byref(a), C.byref(need)))
        ws = self._scratch(need.value)
        self._check(lib.rcd_orthogonalize(self._h, C.byref(a), ws.data_ptr() if ws is not None else None, need.value, self._stream()))
        return out


def rcd_worker_lists(ctx: Context, assignment, W: int):
    """assignment [N] int32 on the device -> (offsets [W+1] int64, indices [N] int32): worker j's samples are
    indices[offsets[j]:offsets[j+1]], ascending."""
    torch = _torch()
    assignment = assignment.contiguous()
    N = assignment.numel()
    out = C.c_size_t()
    ctx._check(lib.rcd_worker_lists_workspace_bytes(ctx._h, N, W, C.byref(out)))
    ws = ctx.workspace(int(out.value))
    offsets = torch.empty(W + 1, dtype=torch.int64, device=assignment.device)
    indices = torch.empty(N, dtype=torch.int32, device=assignment.device)
    ctx._check(lib.rcd_worker_lists(ctx._h, C.c_void_p(assignment.data_ptr()), N, W, C.c_void_p(offsets.data_ptr()),
                                    C.c_void_p(indices.data_ptr()), C.c_void_p(ws.data_ptr()), ws.numel(), ctx._stream()))
    return offsets, indices


def rcd_objective_class_static(ctx: Context, S, assignment, W: int, part_values, total):
    """Block values of one class from its similarity matrix, for callers that cannot allocate.

    Everything is passed in: ``S`` [M, ld] int32 / float32, ``assignment`` [M] int32, and the
    outputs ``part_values`` [W] and ``total`` [1] (int64 for int32 S, float64 for float32 S), all
    device tensors the caller already owns.  This wrapper allocates nothing either."""
    torch = _torch()
    M, ld = S.shape
    code = RCD_FEAT_I8 if S.dtype == torch.int32 else RCD_FEAT_BF16
    ctx._check(lib.rcd_objective_class_static(ctx._h, C.c_void_p(S.data_ptr()), code, M, ld,
                                              C.c_void_p(assignment.data_ptr()), W,
                                              C.c_void_p(part_values.data_ptr()), C.c_void_p(total.data_ptr()),
                                              ctx._stream()))


def rcd_yardstick_read(ctx: Context, buffer, repeats: int = 1) -> int:
    """Enqueues the read-only sweep over ``buffer`` (any device tensor); returns the bytes one call reads."""
    nbytes = buffer.numel() * buffer.element_size() // 16 * 16
    ctx._check(lib.rcd_yardstick_read(ctx._h, C.c_void_p(buffer.data_ptr()), nbytes, int(repeats), ctx._stream()))
    return nbytes * int(repeats)


def rcd_yardstick_mma(ctx: Context, dtype_code: int, iterations: int) -> float:
    """Enqueues the tensor-core peak loop; returns the arithmetic operations the launch performs."""
    ops = C.c_double()
    ctx._check(lib.rcd_yardstick_mma(ctx._h, int(dtype_code), int(iterations), C.byref(ops), ctx._stream()))
    return float(ops.value)


def rcd_similarity(ctx: Context, X):
    return ctx.rcd_similarity(X)


def rcd_partition(ctx: Context, features, labels, capacities, L, **kw):
    return ctx.rcd_partition(features, labels, capacities, L, **kw)


def rcd_partition_host(ctx: Context, features, labels, capacities, L, **kw):
    return ctx.rcd_partition_host(features, labels, capacities, L, **kw)


def rcd_objective(ctx: Context, features, labels, assignment, W, L, **kw):
    return ctx.rcd_objective(features, labels, assignment, W, L, **kw)


def rcd_rms_norm(ctx: Context, x, **kw):
    return ctx.rcd_rms_norm(x, **kw)


def rcd_rms_norm_backward(ctx: Context, dy, h, **kw):
    return ctx.rcd_rms_norm_backward(dy, h, **kw)


def rcd_quantize_rows(ctx: Context, x):
    return ctx.rcd_quantize_rows(x)


def rcd_linear(ctx: Context, x, w, **kw):
    return ctx.rcd_linear(x, w, **kw)


def rcd_linear_backward(ctx: Context, dy, x, w, **kw):
    return ctx.rcd_linear_backward(dy, x, w, **kw)


def rcd_linear_cross_entropy(ctx: Context, x, w, labels, **kw):
    return ctx.rcd_linear_cross_entropy(x, w, labels, **kw)


def rcd_linear_cross_entropy_backward(ctx: Context, x, w, labels, lse, **kw):
    return ctx.rcd_linear_cross_entropy_backward(x, w, labels, lse, **kw)


def rcd_orthogonalize(ctx: Context, g, **kw):
    return ctx.rcd_orthogonalize(g, **kw)
