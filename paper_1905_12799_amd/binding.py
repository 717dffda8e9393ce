"""Thin ctypes binding over librls.so (the C ABI of include/rls.h).

Argument marshalling only: every step of the path runs in the HIP kernels behind the C calls.
PyTorch supplies device memory (tensors) and the current HIP stream; nothing here computes.
The library must have been built (python -m paper_1905_12799_amd.build, or __graft_entry__.build());
loading fails loudly when it is missing.
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple, Optional, Sequence, Tuple

import torch

from . import build as _build

RLS_OK = 0
RLS_STATUS_NONFINITE = 1
RLS_STATUS_RANGE = 2
MAX_D, MAX_K, MAX_DEPTH = 32, 128, 12
MAX_CHOICES = 1 << 24
MAX_TOP = 128
F32, BF16, F16 = 0, 1, 2
_TYPE_OF = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}


class RlsError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        super().__init__(f"{what}: {error_string(code)} (code {code})")


class _Forest(ctypes.Structure):
    _fields_ = [("n_trees", ctypes.c_int32), ("depth", ctypes.c_int32), ("n_features", ctypes.c_int32),
                ("base", ctypes.c_float), ("feat_dev", ctypes.c_void_p), ("thr_dev", ctypes.c_void_p),
                ("leaf_dev", ctypes.c_void_p)]


class _Domains(ctypes.Structure):
    _fields_ = [("n_knobs", ctypes.c_int32), ("offsets_dev", ctypes.c_void_p), ("values_dev", ctypes.c_void_p)]


class _Sequence(ctypes.Structure):
    _fields_ = [("data_dev", ctypes.c_void_p), ("batch_stride", ctypes.c_int64), ("step_stride", ctypes.c_int64)]


class _ScanShape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("steps", ctypes.c_int64), ("channels", ctypes.c_int64), ("type", ctypes.c_int32),
                ("gate_type", ctypes.c_int32), ("reverse", ctypes.c_int32)]


class _DeltaShape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("steps", ctypes.c_int64), ("heads", ctypes.c_int32), ("key_heads", ctypes.c_int32), ("key_dim", ctypes.c_int32),
                ("value_dim", ctypes.c_int32), ("type", ctypes.c_int32), ("scale", ctypes.c_float)]


class _Heads(ctypes.Structure):
    _fields_ = [("data_dev", ctypes.c_void_p), ("batch_stride", ctypes.c_int64), ("step_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class _AdamwTensor(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("param_type", ctypes.c_int32), ("grad_type", ctypes.c_int32), ("param_dev", ctypes.c_void_p),
                ("grad_dev", ctypes.c_void_p), ("master_dev", ctypes.c_void_p), ("m_dev", ctypes.c_void_p), ("v_dev", ctypes.c_void_p),
                ("m_scale_dev", ctypes.c_void_p), ("v_scale_dev", ctypes.c_void_p)]


class _AdamwOptions(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("step", ctypes.c_int64), ("seed", ctypes.c_uint64), ("state_bits", ctypes.c_int32),
                ("grad_scale_dev", ctypes.c_void_p)]


_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(_build.LIB):
            raise ImportError(f"{_build.LIB} is missing: build it with `python -m paper_1905_12799_amd.build`")
        L = ctypes.CDLL(_build.LIB)
        L.rls_version.restype = ctypes.c_int32
        L.rls_error_string.restype = ctypes.c_char_p
        L.rls_error_string.argtypes = [ctypes.c_int32]
        L.rls_last_hip_error.restype = ctypes.c_int32
        L.rls_kmeans_sweep_workspace_bytes.restype = ctypes.c_int64
        L.rls_kmeans_sweep_workspace_bytes.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                                       ctypes.c_int32]
        L.rls_kmeans_sweep_least_workspace_bytes.restype = ctypes.c_int64
        L.rls_kmeans_sweep_least_workspace_bytes.argtypes = L.rls_kmeans_sweep_workspace_bytes.argtypes
        i32, i64, u64, vp, f64 = ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_double
        L.rls_gbt_score.restype = i32
        L.rls_gbt_score.argtypes = [ctypes.POINTER(_Forest), vp, i64, i32, i64, vp, vp]
        L.rls_gbt_score_batched.restype = i32
        L.rls_gbt_score_batched.argtypes = [ctypes.POINTER(_Forest), i32, vp, i64, i32, i64, i64, vp, vp]
        L.rls_kmeanspp_chain.restype = i32
        L.rls_kmeanspp_chain.argtypes = [vp, i64, i32, i64, i32, u64, vp, vp, i64, vp]
        L.rls_kmeans_sweep.restype = i32
        L.rls_kmeans_sweep.argtypes = [vp, i64, i32, i64, i32, i32, i32, u64, vp, vp, vp, vp, vp, vp, vp, i64, vp]
        L.rls_kmeans_sweep_batched.restype = i32
        L.rls_kmeans_sweep_static.restype = i32
        L.rls_kmeans_sweep_static.argtypes = [vp, i64, i32, i64, i32, i32, i32, u64, vp, vp, vp, vp, vp, vp, vp]
        L.rls_kmeans_sweep_batched.argtypes = [i32, vp, i64, i32, i64, i64, i32, i32, i32, ctypes.POINTER(u64), vp, vp,
                                               vp, vp, vp, vp, vp, i64, vp]
        L.rls_kmeans_sweep_until_knee_workspace_bytes.restype = ctypes.c_int64
        L.rls_kmeans_sweep_until_knee_workspace_bytes.argtypes = [i64, i32, i32, i32, i32]
        L.rls_kmeans_sweep_until_knee.restype = i32
        L.rls_kmeans_sweep_until_knee.argtypes = [vp, i64, i32, i64, i32, i32, i32, i32, u64, vp, f64, vp, vp, vp,
                                                  ctypes.POINTER(f64), ctypes.POINTER(i32), ctypes.POINTER(i32), vp, vp,
                                                  i64, vp]
        L.rls_pick_knee.restype = i32
        L.rls_pick_knee.argtypes = [ctypes.POINTER(f64), i32, i32, f64, ctypes.POINTER(i32)]
        L.rls_snap_to_valid.restype = i32
        L.rls_snap_to_valid.argtypes = [vp, i32, i32, i64, ctypes.POINTER(_Domains), vp, vp]
        L.rls_snap_to_valid_batched.restype = i32
        L.rls_snap_to_valid_batched.argtypes = [i32, vp, i32, i32, i64, i64, ctypes.POINTER(_Domains), vp, vp]
        L.rls_knob_modes.restype = i32
        L.rls_knob_modes.argtypes = [vp, i64, i32, i64, ctypes.POINTER(_Domains), i32, vp, vp, vp]
        L.rls_replace_visited.restype = i32
        L.rls_replace_visited.argtypes = [vp, i32, i32, vp, i64, vp, vp, vp]
        L.rls_apply_actions.restype = i32
        L.rls_apply_actions.argtypes = [vp, vp, i64, ctypes.POINTER(_Domains), vp, vp, i64, vp]
        L.rls_sample_workspace_bytes.restype = i64
        L.rls_sample_workspace_bytes.argtypes = [i64, i64]
        L.rls_sample.restype = i32
        L.rls_sample.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, i64, vp]
        L.rls_token_logprobs_workspace_bytes.restype = i64
        L.rls_token_logprobs_workspace_bytes.argtypes = [i64, i64, i32]
        L.rls_token_logprobs.restype = i32
        L.rls_token_logprobs.argtypes = [vp, i32, i64, i64, i64, vp, vp, i32, vp, vp, vp, vp, vp, vp, i64, vp]
        L.rls_token_logprobs_backward.restype = i32
        L.rls_token_logprobs_backward.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, i64, vp]
        L.rls_distill_loss_workspace_bytes.restype = i64
        L.rls_distill_loss_workspace_bytes.argtypes = [i64, i64]
        L.rls_distill_loss.restype = i32
        L.rls_distill_loss.argtypes = [vp, i32, i64, i64, i64, vp, vp, i32, i32, vp, vp, vp, vp, i64, vp]
        L.rls_distill_loss_backward.restype = i32
        L.rls_distill_loss_backward.argtypes = [vp, i32, i64, i64, i64, vp, vp, i32, i32, vp, vp, vp, vp, i64, vp]
        seq = vp                                         # addresses within one array: see _sequences
        L.rls_linear_scan_workspace_bytes.restype = i64
        L.rls_linear_scan_workspace_bytes.argtypes = [i64, i64, i64]
        L.rls_linear_scan.restype = i32
        L.rls_linear_scan.argtypes = [ctypes.POINTER(_ScanShape), seq, seq, vp, vp, seq, vp, vp, i64, vp]
        L.rls_linear_scan_backward.restype = i32
        L.rls_linear_scan_backward.argtypes = [ctypes.POINTER(_ScanShape), seq, seq, seq, vp, vp, vp, seq, seq, vp, vp, i64, vp]
        L.rls_gated_delta_workspace_bytes.restype = i64
        L.rls_gated_delta_workspace_bytes.argtypes = [ctypes.POINTER(_DeltaShape), i32]
        L.rls_gated_delta.restype = i32
        L.rls_gated_delta.argtypes = [ctypes.POINTER(_DeltaShape), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, vp]
        L.rls_gated_delta_backward.restype = i32
        L.rls_gated_delta_backward.argtypes = [ctypes.POINTER(_DeltaShape), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, vp]
        L.rls_adamw_step.restype = i32
        L.rls_adamw_step.argtypes = [ctypes.POINTER(_AdamwTensor), i32, ctypes.POINTER(_AdamwOptions), vp]
        L.rls_profile_enable.restype = i32
        L.rls_profile_enable.argtypes = [i32]
        L.rls_profile_read.restype = i32
        L.rls_profile_read.argtypes = [ctypes.POINTER(i32), ctypes.POINTER(f64)]
        _lib = L
    return _lib


def version() -> int:
    return int(lib().rls_version())


def error_string(code: int) -> str:
    return lib().rls_error_string(ctypes.c_int32(code)).decode()


def profile_enable(on: bool) -> None:
    _check(lib().rls_profile_enable(1 if on else 0), "rls_profile_enable")


def profile_read():
    """(launches timed, total milliseconds) of the Lloyd step kernel since the last read."""
    n, ms = ctypes.c_int32(0), ctypes.c_double(0.0)
    _check(lib().rls_profile_read(ctypes.byref(n), ctypes.byref(ms)), "rls_profile_read")
    return int(n.value), float(ms.value)


def _stream() -> ctypes.c_void_p:
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _raw_stream(device: int) -> int:
    """The current stream of the device that a call's tensors are on, as a number (making a Stream object of it takes 3 us, a fifth of a short call)."""
    if device != torch._C._cuda_getDevice():
        raise ValueError(f"the tensors are on device {device}, which is not the current one")
    return torch._C._cuda_getCurrentRawStream(device)


def _ptr(t: Optional[torch.Tensor]) -> ctypes.c_void_p:
    return ctypes.c_void_p(None if t is None else t.data_ptr())


def _written(*tensors: torch.Tensor) -> None:
    """Tells autograd that a call has changed a caller's tensors in place, as torch's own operations do."""
    torch._C._increment_version([t for t in tensors if not t.is_inference()])


def _check(rc: int, what: str) -> None:
    if rc != RLS_OK:
        raise RlsError(rc, what)


def _dev(t: torch.Tensor, dtype: torch.dtype, name: str) -> torch.Tensor:
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous device tensor of dtype {dtype}")
    return t


def _mat(t: torch.Tensor, name: str) -> torch.Tensor:
    """fp32 device matrix (optionally with a leading batch dimension) whose rows are contiguous."""
    if not t.is_cuda or t.dtype != torch.float32 or t.stride(-1) != 1:
        raise ValueError(f"{name} must be an fp32 device tensor with unit stride along the features")
    return t


class DeviceForest:
    """Device-resident forest (arrays as in rls_forest): feat int32 [T, 2^D-1], thr fp32, leaf fp32 [T, 2^D]."""

    def __init__(self, n_trees: int, depth: int, n_features: int, base: float, feat, thr, leaf, device="cuda"):
        self.n_trees, self.depth, self.n_features, self.base = int(n_trees), int(depth), int(n_features), float(base)
        self.feat = torch.as_tensor(feat, dtype=torch.int32).contiguous().to(device)
        self.thr = torch.as_tensor(thr, dtype=torch.float32).contiguous().to(device)
        self.leaf = torch.as_tensor(leaf, dtype=torch.float32).contiguous().to(device)

    @classmethod
    def from_host(cls, f, device="cuda") -> "DeviceForest":
        return cls(f.n_trees, f.depth, f.n_features, f.base, f.feat, f.thr, f.leaf, device)

    def struct(self) -> _Forest:
        return _Forest(self.n_trees, self.depth, self.n_features, self.base, self.feat.data_ptr(),
                       self.thr.data_ptr(), self.leaf.data_ptr())


class DeviceDomains:
    """Device-resident knob domains in CSR form (rls_knob_domains)."""

    def __init__(self, offsets, values, device="cuda"):
        self.offsets = torch.as_tensor(offsets, dtype=torch.int32).contiguous().to(device)
        self.values = torch.as_tensor(values, dtype=torch.float32).contiguous().to(device)
        self.n_knobs = int(self.offsets.numel()) - 1
        self.n_values = int(self.values.numel())

    def struct(self) -> _Domains:
        return _Domains(self.n_knobs, self.offsets.data_ptr(), self.values.data_ptr())


def gbt_score(forest: DeviceForest, X: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    _mat(X, "X")
    N, d = X.shape
    out = torch.empty(N, dtype=torch.float32, device=X.device) if out is None else _dev(out, torch.float32, "out")
    st = forest.struct()
    _check(lib().rls_gbt_score(ctypes.byref(st), _ptr(X), N, d, X.stride(0), _ptr(out), _stream()), "rls_gbt_score")
    return out


def gbt_score_batched(forests: Sequence[DeviceForest], X: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    _mat(X, "X")
    B, N, d = X.shape
    out = torch.empty((B, N), dtype=torch.float32, device=X.device) if out is None else _dev(out, torch.float32, "out")
    arr = (_Forest * B)(*[f.struct() for f in forests])
    _check(lib().rls_gbt_score_batched(arr, B, _ptr(X), N, d, X.stride(1), X.stride(0), _ptr(out), _stream()),
           "rls_gbt_score_batched")
    return out


def kmeans_sweep_workspace_bytes(N: int, d: int, k_min: int, k_max: int, batch: int = 1) -> int:
    n = int(lib().rls_kmeans_sweep_workspace_bytes(N, d, k_min, k_max, batch))
    if n < 0:
        raise RlsError(n, "rls_kmeans_sweep_workspace_bytes")
    return n


def kmeans_sweep_least_workspace_bytes(N: int, d: int, k_min: int, k_max: int, batch: int = 1) -> int:
    n = int(lib().rls_kmeans_sweep_least_workspace_bytes(N, d, k_min, k_max, batch))
    if n < 0:
        raise RlsError(n, "rls_kmeans_sweep_least_workspace_bytes")
    return n


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(nbytes + 256, dtype=torch.uint8, device=device)


def _aligned_ptr(ws: torch.Tensor) -> int:
    return (ws.data_ptr() + 255) // 256 * 256


def kmeanspp_chain(X: torch.Tensor, k_max: int, seed: int, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    _mat(X, "X")
    N, d = X.shape
    need = kmeans_sweep_workspace_bytes(N, d, k_max, k_max, 1)
    ws = _workspace(need, X.device) if workspace is None else workspace
    idx = torch.empty(k_max, dtype=torch.int64, device=X.device)
    base = _aligned_ptr(ws)
    avail = ws.numel() - (base - ws.data_ptr())
    _check(lib().rls_kmeanspp_chain(_ptr(X), N, d, X.stride(0), k_max, ctypes.c_uint64(seed), _ptr(idx),
                                    ctypes.c_void_p(base), avail, _stream()), "rls_kmeanspp_chain")
    return idx


class SweepResult:
    """Outputs of a sweep, all device tensors. centroids is packed; use centroids_of(k)."""

    def __init__(self, k_min, k_max, d, labels, centroids, inertia, trace, status):
        self.k_min, self.k_max, self.d = k_min, k_max, d
        self.labels, self.centroids, self.inertia, self.trace, self.status = labels, centroids, inertia, trace, status

    def centroids_of(self, k: int, b: Optional[int] = None) -> torch.Tensor:
        off = sum(range(self.k_min, k)) * self.d
        c = self.centroids if b is None else self.centroids[b]
        return c[off:off + k * self.d].view(k, self.d)


def kmeans_sweep(X: torch.Tensor, k_min: int, k_max: int, iters: int, seed: int = 0,
                 init_idx: Optional[torch.Tensor] = None, want_labels: bool = True, want_trace: bool = False,
                 workspace: Optional[torch.Tensor] = None, check_status: bool = True) -> SweepResult:
    _mat(X, "X")
    N, d = X.shape
    n_k = k_max - k_min + 1
    rows = sum(range(k_min, k_max + 1))
    need = kmeans_sweep_workspace_bytes(N, d, k_min, k_max, 1)
    ws = _workspace(need, X.device) if workspace is None else workspace
    dev = X.device
    labels = torch.empty((n_k, N), dtype=torch.int32, device=dev) if want_labels else None
    centroids = torch.empty(rows * d, dtype=torch.float32, device=dev)
    inertia = torch.empty(n_k, dtype=torch.float64, device=dev)
    trace = torch.empty((n_k, iters + 1), dtype=torch.float64, device=dev) if want_trace else None
    status = torch.empty(1, dtype=torch.int32, device=dev)
    if init_idx is not None:
        _dev(init_idx, torch.int64, "init_idx")
        if init_idx.numel() < k_max:
            raise ValueError("init_idx needs k_max entries")
    base = _aligned_ptr(ws)
    avail = ws.numel() - (base - ws.data_ptr())
    rc = lib().rls_kmeans_sweep(_ptr(X), N, d, X.stride(0), k_min, k_max, iters, ctypes.c_uint64(seed), _ptr(init_idx),
                                _ptr(labels), _ptr(centroids), _ptr(inertia), _ptr(trace), _ptr(status),
                                ctypes.c_void_p(base), avail, _stream())
    _check(rc, "rls_kmeans_sweep")
    if check_status:
        st = int(status.item())
        if st != 0:
            raise RuntimeError(f"rls_kmeans_sweep: data precondition violated, status bits {st}")
    return SweepResult(k_min, k_max, d, labels, centroids, inertia, trace, status)


STATIC_WORKSPACE_BYTES = 64 << 20


def kmeans_sweep_static(X: torch.Tensor, k_min: int, k_max: int, iters: int, seed: int = 0,
                        init_idx: Optional[torch.Tensor] = None, want_trace: bool = False,
                        out: Optional[SweepResult] = None) -> SweepResult:
    """rls_kmeans_sweep_static: the sweep on the library's own fixed workspace (the call allocates nothing).
    `out` supplies the output tensors (labels may be None); without it they are allocated here, before the call."""
    _mat(X, "X")
    N, d = X.shape
    n_k = k_max - k_min + 1
    rows = sum(range(k_min, k_max + 1))
    dev = X.device
    if out is None:
        out = SweepResult(k_min, k_max, d, torch.empty((n_k, N), dtype=torch.int32, device=dev),
                          torch.empty(rows * d, dtype=torch.float32, device=dev),
                          torch.empty(n_k, dtype=torch.float64, device=dev),
                          torch.empty((n_k, iters + 1), dtype=torch.float64, device=dev) if want_trace else None,
                          torch.empty(1, dtype=torch.int32, device=dev))
    if init_idx is not None:
        _dev(init_idx, torch.int64, "init_idx")
        if init_idx.numel() < k_max:
            raise ValueError("init_idx needs k_max entries")
    rc = lib().rls_kmeans_sweep_static(_ptr(X), N, d, X.stride(0), k_min, k_max, iters, ctypes.c_uint64(seed),
                                       _ptr(init_idx), _ptr(out.labels), _ptr(out.centroids), _ptr(out.inertia),
                                       _ptr(out.trace), _ptr(out.status), _stream())
    _check(rc, "rls_kmeans_sweep_static")
    return out


def kmeans_sweep_until_knee(X: torch.Tensor, k_min: int, k_max: int, k_wave: int, iters: int, knee_const: float,
                            seed: int = 0, init_idx: Optional[torch.Tensor] = None, want_labels: bool = True,
                            workspace: Optional[torch.Tensor] = None) -> Tuple[int, int, SweepResult]:
    """Algorithm 1's loop with its early exit: returns (chosen k, number of k computed, results).

    The result arrays are sized for the whole range; only the first `n_done` runs are written. Synchronises the
    current stream after every wave of k_wave values of k."""
    _mat(X, "X")
    N, d = X.shape
    n_k = k_max - k_min + 1
    rows = sum(range(k_min, k_max + 1))
    need = int(lib().rls_kmeans_sweep_until_knee_workspace_bytes(N, d, k_min, k_max, k_wave))
    if need < 0:
        _check(need, "rls_kmeans_sweep_until_knee_workspace_bytes")
    ws = _workspace(need, X.device) if workspace is None else workspace
    dev = X.device
    labels = torch.empty((n_k, N), dtype=torch.int32, device=dev) if want_labels else None
    centroids = torch.empty(rows * d, dtype=torch.float32, device=dev)
    inertia = torch.empty(n_k, dtype=torch.float64, device=dev)
    status = torch.empty(1, dtype=torch.int32, device=dev)
    if init_idx is not None:
        _dev(init_idx, torch.int64, "init_idx")
        if init_idx.numel() < k_max:
            raise ValueError("init_idx needs k_max entries")
    inertia_host = (ctypes.c_double * n_k)()
    k_out, n_done = ctypes.c_int32(0), ctypes.c_int32(0)
    base = _aligned_ptr(ws)
    avail = ws.numel() - (base - ws.data_ptr())
    rc = lib().rls_kmeans_sweep_until_knee(_ptr(X), N, d, X.stride(0), k_min, k_max, k_wave, iters, ctypes.c_uint64(seed),
                                           _ptr(init_idx), float(knee_const), _ptr(labels), _ptr(centroids), _ptr(inertia),
                                           inertia_host, ctypes.byref(k_out), ctypes.byref(n_done), _ptr(status),
                                           ctypes.c_void_p(base), avail, _stream())
    _check(rc, "rls_kmeans_sweep_until_knee")
    st = int(status.item())
    if st != 0:
        raise RuntimeError(f"rls_kmeans_sweep_until_knee: data precondition violated, status bits {st}")
    return int(k_out.value), int(n_done.value), SweepResult(k_min, k_max, d, labels, centroids, inertia, None, status)


def kmeans_sweep_batched(X: torch.Tensor, k_min: int, k_max: int, iters: int, seeds: Optional[Sequence[int]] = None,
                         init_idx: Optional[torch.Tensor] = None, want_labels: bool = True, want_trace: bool = False,
                         workspace: Optional[torch.Tensor] = None, check_status: bool = True) -> SweepResult:
    _mat(X, "X")
    B, N, d = X.shape
    n_k = k_max - k_min + 1
    rows = sum(range(k_min, k_max + 1))
    need = kmeans_sweep_workspace_bytes(N, d, k_min, k_max, B)
    ws = _workspace(need, X.device) if workspace is None else workspace
    dev = X.device
    labels = torch.empty((B, n_k, N), dtype=torch.int32, device=dev) if want_labels else None
    centroids = torch.empty((B, rows * d), dtype=torch.float32, device=dev)
    inertia = torch.empty((B, n_k), dtype=torch.float64, device=dev)
    trace = torch.empty((B, n_k, iters + 1), dtype=torch.float64, device=dev) if want_trace else None
    status = torch.empty(B, dtype=torch.int32, device=dev)
    seeds_arr = None
    if seeds is not None:
        seeds_arr = (ctypes.c_uint64 * B)(*[int(s) for s in seeds])
    if init_idx is not None:
        _dev(init_idx, torch.int64, "init_idx")
    base = _aligned_ptr(ws)
    avail = ws.numel() - (base - ws.data_ptr())
    rc = lib().rls_kmeans_sweep_batched(B, _ptr(X), N, d, X.stride(1), X.stride(0), k_min, k_max, iters, seeds_arr,
                                        _ptr(init_idx), _ptr(labels), _ptr(centroids), _ptr(inertia), _ptr(trace),
                                        _ptr(status), ctypes.c_void_p(base), avail, _stream())
    _check(rc, "rls_kmeans_sweep_batched")
    if check_status and bool((status != 0).any().item()):
        raise RuntimeError(f"rls_kmeans_sweep_batched: data precondition violated, status {status.tolist()}")
    return SweepResult(k_min, k_max, d, labels, centroids, inertia, trace, status)


def pick_knee(inertia_host: Sequence[float], k_min: int, k_max: int, knee_const: float) -> int:
    n = k_max - k_min + 1
    arr = (ctypes.c_double * n)(*[float(v) for v in inertia_host[:n]])
    out = ctypes.c_int32(0)
    _check(lib().rls_pick_knee(arr, k_min, k_max, ctypes.c_double(knee_const), ctypes.byref(out)), "rls_pick_knee")
    return int(out.value)


def snap_to_valid(centroids: torch.Tensor, domains: DeviceDomains, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    _mat(centroids, "centroids")
    k, d = centroids.shape
    out = torch.empty((k, domains.n_knobs), dtype=torch.int32, device=centroids.device) if out is None else out
    st = domains.struct()
    _check(lib().rls_snap_to_valid(_ptr(centroids), k, d, centroids.stride(0), ctypes.byref(st), _ptr(out), _stream()),
           "rls_snap_to_valid")
    return out


def knob_modes(X: torch.Tensor, domains: DeviceDomains, hist: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """mode(s_Theta): per knob the domain index most rows take; returns (mode_cfg [n_knobs], hist [n_values])."""
    _mat(X, "X")
    N, d = X.shape
    mode = torch.empty(domains.n_knobs, dtype=torch.int32, device=X.device)
    hist = torch.empty(domains.n_values, dtype=torch.int32, device=X.device) if hist is None else _dev(hist, torch.int32, "hist")
    st = domains.struct()
    _check(lib().rls_knob_modes(_ptr(X), N, d, X.stride(0), ctypes.byref(st), domains.n_values, _ptr(mode), _ptr(hist),
                                _stream()), "rls_knob_modes")
    return mode, hist


def replace_visited(cfg: torch.Tensor, visited: Optional[torch.Tensor], mode_cfg: torch.Tensor) -> torch.Tensor:
    """Rows of cfg (int32 [k][n_knobs], updated in place) found among the visited rows become mode_cfg; returns flags [k]."""
    _dev(cfg, torch.int32, "cfg")
    k, n_knobs = cfg.shape
    if not cfg.is_contiguous():
        raise ValueError("cfg must be contiguous")
    n_visited = 0 if visited is None else int(visited.shape[0])
    if n_visited:
        _dev(visited, torch.int32, "visited")
        if not visited.is_contiguous() or visited.shape[1] != n_knobs:
            raise ValueError("visited must be contiguous [V][n_knobs]")
    replaced = torch.empty(k, dtype=torch.int32, device=cfg.device)
    _check(lib().rls_replace_visited(_ptr(cfg), k, n_knobs, _ptr(visited) if n_visited else None, n_visited,
                                     _ptr(_dev(mode_cfg, torch.int32, "mode_cfg")), _ptr(replaced), _stream()),
           "rls_replace_visited")
    return replaced


def apply_actions(cfg: torch.Tensor, action: torch.Tensor, domains: DeviceDomains, want_features: bool = True):
    """Configuration updater: cfg int32 [m][n_knobs] + action int8 in {-1, 0, +1} -> (new cfg, features [m][n_knobs] or None)."""
    _dev(cfg, torch.int32, "cfg")
    _dev(action, torch.int8, "action")
    m, n_knobs = cfg.shape
    if not (cfg.is_contiguous() and action.is_contiguous()) or action.shape != cfg.shape or n_knobs != domains.n_knobs:
        raise ValueError("cfg and action must be contiguous [m][n_knobs] with the domains' n_knobs")
    out = torch.empty_like(cfg)
    feats = torch.empty((m, n_knobs), dtype=torch.float32, device=cfg.device) if want_features else None
    st = domains.struct()
    _check(lib().rls_apply_actions(_ptr(cfg), _ptr(action), m, ctypes.byref(st), _ptr(out), _ptr(feats), n_knobs, _stream()),
           "rls_apply_actions")
    return out, feats


def snap_to_valid_batched(centroids: torch.Tensor, domains: Sequence[DeviceDomains],
                          out: Optional[torch.Tensor] = None) -> torch.Tensor:
    _mat(centroids, "centroids")
    B, k, d = centroids.shape
    n_knobs = domains[0].n_knobs
    out = torch.empty((B, k, n_knobs), dtype=torch.int32, device=centroids.device) if out is None else out
    arr = (_Domains * B)(*[dm.struct() for dm in domains])
    _check(lib().rls_snap_to_valid_batched(B, _ptr(centroids), k, d, centroids.stride(1), centroids.stride(0), arr,
                                           _ptr(out), _stream()), "rls_snap_to_valid_batched")
    return out


def sample_workspace_bytes(rows: int, n_choices: int) -> int:
    n = int(lib().rls_sample_workspace_bytes(rows, n_choices))
    if n < 0:
        raise RlsError(n, "rls_sample_workspace_bytes")
    return n


def _space(workspace: Optional[torch.Tensor], need, device) -> Tuple[Optional[torch.Tensor], int, int]:
    """Workspace of a call: the caller's, or one of its own of need() bytes; with its 256-byte aligned start and what is left of it."""
    if workspace is None:
        n = need()
        if n == 0:
            return None, 0, 0
        workspace = _workspace(n, device)
    elif not workspace.is_cuda:
        raise ValueError("workspace must be a device tensor")
    base = _aligned_ptr(workspace)
    return workspace, base, max(0, workspace.numel() * workspace.element_size() - (base - workspace.data_ptr()))


def _per_row(t: Optional[torch.Tensor], dtype: torch.dtype, rows: int, name: str) -> int:
    """Address of an array with an entry per row (0 for None)."""
    if t is None:
        return 0
    if t.numel() != rows:
        raise ValueError(f"{name} needs an entry per row")
    return _dev(t, dtype, name).data_ptr()


def sample(logits: torch.Tensor, uniform: torch.Tensor, temperature: Optional[torch.Tensor] = None, top_k: Optional[torch.Tensor] = None,
           top_p: Optional[torch.Tensor] = None, min_p: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
           want_logprob: bool = True, out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """A draw per row of logits [rows, n_choices] (fp32, bf16 or fp16, rows contiguous) from uniform [rows]: (token int32, logprob fp32 or None).

    temperature, top_p, min_p (fp32) and top_k (int32) have an entry per row; None leaves a rule out.  Nothing is differentiated through a draw."""
    if logits.dim() != 2 or not logits.is_cuda or logits.dtype not in _TYPE_OF or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits must be an fp32, bf16 or fp16 device matrix with unit stride along a row")
    rows, n = logits.shape
    device = logits.device
    settings = (_per_row(uniform, torch.float32, rows, "uniform"), _per_row(temperature, torch.float32, rows, "temperature"),
                _per_row(top_k, torch.int32, rows, "top_k"), _per_row(top_p, torch.float32, rows, "top_p"),
                _per_row(min_p, torch.float32, rows, "min_p"))
    token = torch.empty(rows, dtype=torch.int32, device=device) if out is None else out
    to = _per_row(token, torch.int32, rows, "out")
    logprob = torch.empty(rows, dtype=torch.float32, device=device) if want_logprob else None
    ws, base, avail = _space(workspace, lambda: sample_workspace_bytes(rows, n), device)
    _check(lib().rls_sample(logits.data_ptr(), _TYPE_OF[logits.dtype], rows, n, logits.stride(0) if rows > 1 else n, *settings, to,
                            logprob.data_ptr() if want_logprob else 0, base, avail, _raw_stream(logits.get_device())), "rls_sample")
    if out is not None:
        _written(out)
    return token, logprob


class LogProbs(NamedTuple):
    """What token_logprobs returns, a row each: fp32, the tokens int32; None where it was not asked for."""
    logprob: Optional[torch.Tensor]                      # [rows]
    entropy: torch.Tensor                                # [rows]
    top_logprob: Optional[torch.Tensor]                  # [rows, top]
    top_token: Optional[torch.Tensor]                    # [rows, top]
    norm: torch.Tensor                                   # [rows, 2]: the largest logit, and the logarithm of the sum of exponentials


def token_logprobs_workspace_bytes(rows: int, n_choices: int, top: int = 0) -> int:
    n = int(lib().rls_token_logprobs_workspace_bytes(rows, n_choices, top))
    if n < 0:
        raise RlsError(n, "rls_token_logprobs_workspace_bytes")
    return n


def _logits(t: torch.Tensor, name: str = "logits") -> Tuple[int, int, int, int, int]:
    """(address, type, rows, columns, distance of the rows) of a matrix of logits."""
    if t.dim() != 2 or not t.is_cuda or t.dtype not in _TYPE_OF or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be an fp32, bf16 or fp16 device matrix with unit stride along a row")
    rows, n = t.shape
    return t.data_ptr(), _TYPE_OF[t.dtype], rows, n, t.stride(0) if rows > 1 else n


def _rows_of(t: Optional[torch.Tensor], shape, dtype: torch.dtype, name: str) -> int:
    """Address of a contiguous array of that shape (0 for None)."""
    if t is None:
        return 0
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}")
    return _dev(t, dtype, name).data_ptr()


def _gradient_of(logits: torch.Tensor, out: Optional[torch.Tensor]) -> Tuple[torch.Tensor, int, int]:
    """Where the gradient by logits goes: the tensor, its address and the distance of its rows."""
    if out is None:
        out = torch.empty_like(logits, memory_format=torch.contiguous_format)
    elif out.shape != logits.shape or out.dtype != logits.dtype:
        raise ValueError("out must have the shape and the type of the logits")
    at, _, _, _, ld = _logits(out, "out")
    return out, at, ld


def _differentiated(logits: torch.Tensor, temperature: Optional[torch.Tensor]) -> bool:
    """Whether autograd takes part in a call; by a temperature nothing is differentiated, and a call that asks for it is turned down."""
    if not torch.is_grad_enabled():
        return False
    if temperature is not None and temperature.requires_grad:
        raise ValueError("nothing is differentiated by the temperature: pass temperature.detach()")
    return logits.requires_grad


def token_logprobs(logits: torch.Tensor, tokens: Optional[torch.Tensor], temperature: Optional[torch.Tensor] = None, top: int = 0,
                   workspace: Optional[torch.Tensor] = None) -> LogProbs:
    """Log-probability of tokens [rows] (int32; outside the row: 0, a padded position) under logits [rows, n_choices] (fp32, bf16 or fp16, rows
    contiguous), the entropy of every row, and its `top` best entries with their log-probabilities (at most MAX_TOP; -1 where there are fewer).

    temperature (fp32, a constant) has an entry per row.  tokens may be None.  logprob and entropy are differentiable by the logits."""
    if _differentiated(logits, temperature):
        return LogProbs(*_LogProbs.apply(logits, tokens, temperature, top, workspace))
    at, kind, rows, n, ld = _logits(logits)
    device = logits.device
    token_at, temperature_at = _rows_of(tokens, (rows,), torch.int32, "tokens"), _rows_of(temperature, (rows,), torch.float32, "temperature")
    ws, base, avail = _space(workspace, lambda: token_logprobs_workspace_bytes(rows, n, top), device)
    entropy = torch.empty(rows, dtype=torch.float32, device=device)
    logprob = None if tokens is None else torch.empty_like(entropy)
    norm = torch.empty((rows, 2), dtype=torch.float32, device=device)
    best = best_token = None
    if top > 0:
        best, best_token = torch.empty((rows, top), dtype=torch.float32, device=device), torch.empty((rows, top), dtype=torch.int32, device=device)
    _check(lib().rls_token_logprobs(at, kind, rows, n, ld, token_at, temperature_at, top, 0 if tokens is None else logprob.data_ptr(), entropy.data_ptr(),
                                    best.data_ptr() if top > 0 else 0, best_token.data_ptr() if top > 0 else 0, norm.data_ptr(), base, avail,
                                    _raw_stream(logits.get_device())), "rls_token_logprobs")
    return LogProbs(logprob, entropy, best, best_token, norm)


class _LogProbs(torch.autograd.Function):
    """token_logprobs as autograd sees it: logprob and entropy are differentiable, the alternatives and norm are not."""

    @staticmethod
    def forward(ctx, logits, tokens, temperature, top, workspace):
        r = token_logprobs(logits, tokens, temperature, top, workspace)
        ctx.save_for_backward(logits, tokens, temperature, r.norm, r.entropy)
        ctx.mark_non_differentiable(*(t for t in (r.top_logprob, r.top_token, r.norm) if t is not None))
        ctx.set_materialize_grads(False)
        return tuple(r)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dlogprob, dentropy, *_):
        logits, tokens, temperature, norm, entropy = ctx.saved_tensors
        if dlogprob is None and dentropy is None:
            return None, None, None, None, None
        dlogprob, dentropy = (None if d is None else d.contiguous() for d in (dlogprob, dentropy))
        return token_logprobs_backward(logits, tokens, norm, entropy, dlogprob, dentropy, temperature), None, None, None, None


def token_logprobs_backward(logits: torch.Tensor, tokens: Optional[torch.Tensor], norm: torch.Tensor, entropy: Optional[torch.Tensor],
                            dlogprob: Optional[torch.Tensor], dentropy: Optional[torch.Tensor] = None, temperature: Optional[torch.Tensor] = None,
                            out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient by the logits, in their type, from the norm and entropy that token_logprobs returned and the gradients by logprob and entropy
    (either may be None).  `out` may be logits itself."""
    at, kind, rows, n, ld = _logits(logits)
    row = lambda t, dtype, name: _rows_of(t, (rows,), dtype, name)       # noqa: E731
    dlogits, to, ld_to = _gradient_of(logits, out)
    _check(lib().rls_token_logprobs_backward(at, kind, rows, n, ld, row(tokens, torch.int32, "tokens"), row(temperature, torch.float32, "temperature"),
                                             _rows_of(norm, (rows, 2), torch.float32, "norm"), row(entropy, torch.float32, "entropy"),
                                             row(dlogprob, torch.float32, "dlogprob"), row(dentropy, torch.float32, "dentropy"), to, ld_to,
                                             _raw_stream(logits.get_device())), "rls_token_logprobs_backward")
    if out is not None:
        _written(out)
    return dlogits


def distill_loss_workspace_bytes(rows: int, n_choices: int) -> int:
    n = int(lib().rls_distill_loss_workspace_bytes(rows, n_choices))
    if n < 0:
        raise RlsError(n, "rls_distill_loss_workspace_bytes")
    return n


def _teacher(tokens: torch.Tensor, logits: torch.Tensor, rows: int) -> Tuple[int, int, int, int]:
    if logits.dim() != 2 or logits.shape[0] != rows or logits.dtype not in _TYPE_OF:
        raise ValueError("teacher_logits must be [rows, k] in fp32, bf16 or fp16")
    return (_rows_of(tokens, logits.shape, torch.int32, "teacher_tokens"), _dev(logits, logits.dtype, "teacher_logits").data_ptr(),
            _TYPE_OF[logits.dtype], logits.shape[1])


def distill_loss(logits: torch.Tensor, teacher_tokens: torch.Tensor, teacher_logits: torch.Tensor, temperature: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Divergence of every row of logits [rows, n_choices] from the distribution that the teacher's k best entries have among themselves: (loss fp32
    [rows], norm fp32 [rows, 2] as token_logprobs returns it).

    teacher_tokens int32 and teacher_logits (fp32, bf16 or fp16; logits or log-probabilities, such as token_logprobs' alternatives) are [rows, k],
    k at most MAX_TOP; a token outside the row is no entry.  temperature (fp32) has an entry per row.  The loss is differentiable by the logits; the
    teacher and the temperature are constants."""
    if _differentiated(logits, temperature):
        return _Distill.apply(logits, teacher_tokens, teacher_logits, temperature, workspace)
    at, kind, rows, n, ld = _logits(logits)
    token_at, teacher_at, teacher_kind, k = _teacher(teacher_tokens, teacher_logits, rows)
    ws, base, avail = _space(workspace, lambda: distill_loss_workspace_bytes(rows, n), logits.device)
    loss = torch.empty(rows, dtype=torch.float32, device=logits.device)
    norm = torch.empty((rows, 2), dtype=torch.float32, device=logits.device)
    _check(lib().rls_distill_loss(at, kind, rows, n, ld, token_at, teacher_at, teacher_kind, k, _rows_of(temperature, (rows,), torch.float32, "temperature"),
                                  loss.data_ptr(), norm.data_ptr(), base, avail, _raw_stream(logits.get_device())), "rls_distill_loss")
    return loss, norm


class _Distill(torch.autograd.Function):
    """distill_loss as autograd sees it."""

    @staticmethod
    def forward(ctx, logits, teacher_tokens, teacher_logits, temperature, workspace):
        loss, norm = distill_loss(logits, teacher_tokens, teacher_logits, temperature, workspace)
        ctx.save_for_backward(logits, teacher_tokens, teacher_logits, temperature, norm)
        ctx.mark_non_differentiable(norm)
        return loss, norm

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss, _):
        logits, teacher_tokens, teacher_logits, temperature, norm = ctx.saved_tensors
        return distill_loss_backward(logits, teacher_tokens, teacher_logits, norm, dloss.contiguous(), temperature), None, None, None, None


def distill_loss_backward(logits: torch.Tensor, teacher_tokens: torch.Tensor, teacher_logits: torch.Tensor, norm: torch.Tensor, dloss: torch.Tensor,
                          temperature: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient by the logits, in their type, from the norm that distill_loss returned and the gradient dloss [rows].  `out` may be logits itself."""
    at, kind, rows, n, ld = _logits(logits)
    token_at, teacher_at, teacher_kind, k = _teacher(teacher_tokens, teacher_logits, rows)
    dlogits, to, ld_to = _gradient_of(logits, out)
    _check(lib().rls_distill_loss_backward(at, kind, rows, n, ld, token_at, teacher_at, teacher_kind, k,
                                           _rows_of(temperature, (rows,), torch.float32, "temperature"), _rows_of(norm, (rows, 2), torch.float32, "norm"),
                                           _rows_of(dloss, (rows,), torch.float32, "dloss"), to, ld_to, _raw_stream(logits.get_device())),
           "rls_distill_loss_backward")
    if out is not None:
        _written(out)
    return dlogits


def linear_scan_workspace_bytes(batch: int, steps: int, channels: int) -> int:
    n = int(lib().rls_linear_scan_workspace_bytes(batch, steps, channels))
    if n < 0:
        raise RlsError(n, "rls_linear_scan_workspace_bytes")
    return n


def _sequences(shape, *named):
    """rls_sequence structs of (tensor, type, name) side by side in one array, and their addresses; the array has to outlive the call."""
    numbers = []
    for t, dtype, name in named:
        if t.dtype != dtype or t.shape != shape or not t.is_cuda:
            raise ValueError(f"{name} must be a device tensor of shape {tuple(shape)} and type {dtype}")
        per_batch, per_step, per_channel = t.stride()
        if per_channel != 1 and shape[2] > 1:
            raise ValueError(f"{name} must have unit stride along the channels")
        numbers += (t.data_ptr(), per_batch, per_step)
    held = (ctypes.c_int64 * len(numbers))(*numbers)
    base = ctypes.addressof(held)
    return held, range(base, base + ctypes.sizeof(held), ctypes.sizeof(_Sequence))


def _states(t: Optional[torch.Tensor], shape, name: str) -> int:
    if t is None:
        return 0
    if t.dim() != 2 or t.shape[0] != shape[0] or t.shape[1] != shape[2]:
        raise ValueError(f"{name} must be [batch, channels]")
    return _dev(t, torch.float32, name).data_ptr()


def _resets(t: Optional[torch.Tensor], shape) -> int:
    if t is None:
        return 0
    if t.dtype == torch.bool:
        t = t.view(torch.uint8)
    if t.dim() != 2 or t.shape[0] != shape[0] or t.shape[1] != shape[1]:
        raise ValueError("reset must be [batch, steps]")
    return _dev(t, torch.uint8, "reset").data_ptr()


def _scan_shape(a: torch.Tensor, x: torch.Tensor, reverse: bool) -> _ScanShape:
    if x.dim() != 3 or x.dtype not in _TYPE_OF or a.dtype not in (torch.float32, x.dtype):
        raise ValueError("a sequence is [batch, steps, channels] in fp32, bf16 or fp16, its gate of the same type or fp32")
    return _ScanShape(*x.shape, _TYPE_OF[x.dtype], _TYPE_OF[a.dtype], 1 if reverse else 0)


def linear_scan(a: torch.Tensor, b: torch.Tensor, h0: Optional[torch.Tensor] = None, reset: Optional[torch.Tensor] = None, reverse: bool = False,
                workspace: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                last: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """h_t = a_t h_{t-1} + b_t over [batch, steps, channels]: (every state in b's type, the last one in fp32 [batch, channels]).

    a may be fp32 beside a b of fewer bits, and either may be an expanded view; reset [batch, steps] (bytes or bools) cuts the carry;
    reverse runs from the last step to the first.  `last` may be h0 itself, for a state that is updated in place.  Differentiable by a, b and h0."""
    if torch.is_grad_enabled() and (a.requires_grad or b.requires_grad or (h0 is not None and h0.requires_grad)):
        if out is not None or last is not None:
            raise ValueError("out and last are for calls that nothing is differentiated by (torch.no_grad)")
        return _Scan.apply(a, b, h0, reset, reverse, workspace)
    shape, size = _scan_shape(a, b, reverse), b.shape
    B, T, C = size
    # (empty_like takes 0.9 us, empty with a shape, a type and a device 1.9; the call for a single token takes 10)
    h = torch.empty_like(b, memory_format=torch.contiguous_format) if out is None else out
    kept = last is not None
    if not kept:
        last = torch.empty((B, C), dtype=torch.float32, device=b.device) if h0 is None else torch.empty_like(h0)
    ws, base, avail = _space(workspace, lambda: linear_scan_workspace_bytes(B, T, C), b.device)
    held, at = _sequences(size, (a, a.dtype, "a"), (b, b.dtype, "b"), (h, b.dtype, "out"))
    _check(lib().rls_linear_scan(ctypes.byref(shape), at[0], at[1], _states(h0, size, "h0"), _resets(reset, size), at[2], _states(last, size, "last"),
                                 base, avail, _raw_stream(b.get_device())), "rls_linear_scan")
    if out is not None:
        _written(h)
    if kept:
        _written(last)
    return h, last


class _Scan(torch.autograd.Function):
    """linear_scan as autograd sees it: both its results are differentiable."""

    @staticmethod
    def forward(ctx, a, b, h0, reset, reverse, workspace):
        h, last = linear_scan(a, b, h0, reset, reverse, workspace)
        ctx.save_for_backward(a, h, h0, reset)
        ctx.reverse = reverse
        ctx.set_materialize_grads(False)
        return h, last

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dh, dlast):
        a, h, h0, reset = ctx.saved_tensors
        dh = torch.zeros_like(h) if dh is None else dh.contiguous()
        da, db, dh0 = linear_scan_backward(a, h, dh, h0, reset, None if dlast is None else dlast.contiguous(), ctx.reverse)
        return da, db, None if h0 is None else dh0, None, None, None


def linear_scan_backward(a: torch.Tensor, h: torch.Tensor, dh: torch.Tensor, h0: Optional[torch.Tensor] = None, reset: Optional[torch.Tensor] = None,
                         dh_last: Optional[torch.Tensor] = None, reverse: bool = False,
                         workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Gradients of linear_scan from its gates, the states it returned and the gradients by them: (da in a's type, db in h's, dh0 in fp32).

    Where a or b was an expanded view, da or db is the gradient of every element: its sum along the expanded axes is the input's."""
    shape, size = _scan_shape(a, h, reverse), h.shape
    B, T, C = size
    da, db = torch.empty_like(a, memory_format=torch.contiguous_format), torch.empty_like(h, memory_format=torch.contiguous_format)
    dh0 = torch.empty((B, C), dtype=torch.float32, device=h.device)
    ws, base, avail = _space(workspace, lambda: linear_scan_workspace_bytes(B, T, C), h.device)
    held, at = _sequences(size, (a, a.dtype, "a"), (h, h.dtype, "h"), (dh, h.dtype, "dh"), (da, a.dtype, "da"), (db, h.dtype, "db"))
    _check(lib().rls_linear_scan_backward(ctypes.byref(shape), at[0], at[1], at[2], _states(h0, size, "h0"), _resets(reset, size),
                                          _states(dh_last, size, "dh_last"), at[3], at[4], dh0.data_ptr(), base, avail, _raw_stream(h.get_device())),
           "rls_linear_scan_backward")
    return da, db, dh0


def gated_delta_workspace_bytes(batch: int, steps: int, heads: int, key_heads: int, key_dim: int, value_dim: int, backward: bool = False) -> int:
    shape = _DeltaShape(batch, steps, heads, key_heads, key_dim, value_dim, F32, 1.0)
    n = int(lib().rls_gated_delta_workspace_bytes(ctypes.byref(shape), 1 if backward else 0))
    if n < 0:
        raise RlsError(n, "rls_gated_delta_workspace_bytes")
    return n


def _delta_shape(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: Optional[float]) -> _DeltaShape:
    if q.dim() != 4 or v.dim() != 4 or q.shape != k.shape or q.shape[:2] != v.shape[:2] or q.dtype not in _TYPE_OF:
        raise ValueError("q and k are [batch, steps, key_heads, key_dim], v is [batch, steps, heads, value_dim], all in fp32, bf16 or fp16")
    B, T, key_heads, key_dim = q.shape
    return _DeltaShape(B, T, v.shape[2], key_heads, key_dim, v.shape[3], _TYPE_OF[q.dtype], key_dim ** -0.5 if scale is None else scale)


def _heads(dtype: torch.dtype, *named):
    """rls_heads structs of (tensor, shape, name) side by side in one array, and their addresses; the array has to outlive the call."""
    numbers = []
    for t, shape, name in named:
        if t.dtype != dtype or t.shape != shape or not t.is_cuda:
            raise ValueError(f"{name} must be a device tensor of shape {tuple(shape)} and type {dtype}")
        per_batch, per_step, per_head, one = t.stride()
        if one != 1 and shape[3] > 1:
            raise ValueError(f"{name} must have unit stride along its last dimension")
        numbers += (t.data_ptr(), per_batch, per_step, per_head)
    held = (ctypes.c_int64 * len(numbers))(*numbers)
    base = ctypes.addressof(held)
    return held, range(base, base + ctypes.sizeof(held), ctypes.sizeof(_Heads))


def _delta_gates(v: torch.Tensor, g: torch.Tensor, beta: torch.Tensor) -> Tuple[int, int]:
    shape = v.shape[:3]
    return _rows_of(g, shape, torch.float32, "g"), _rows_of(beta, shape, torch.float32, "beta")


def gated_delta(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, g: torch.Tensor, beta: torch.Tensor, state: Optional[torch.Tensor] = None,
                reset: Optional[torch.Tensor] = None, scale: Optional[float] = None, workspace: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None, last: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The gated delta rule over [batch, steps, heads, dim]: S = exp(g) S + beta k (v - exp(g) S^T k)^T, o = scale S^T q, with a matrix S [key_dim,
    value_dim] per sequence and head: (o like v, the last state in fp32 [batch, heads, key_dim, value_dim]).

    q and k may have fewer heads than v; g (logarithms of the decay) and beta are fp32 [batch, steps, heads]; reset [batch, steps] (bytes or bools) is set
    where a sequence begins; scale is key_dim ** -0.5 unless given.  `last` may be state itself, for a state that is updated in place.  Differentiable
    by q, k, v, g, beta and state.  Numbers that are not finite reach what follows in their head up to the next reset, as in linear_scan, and nothing else."""
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (q, k, v, g, beta, state)):
        if out is not None or last is not None:
            raise ValueError("out and last are for calls that nothing is differentiated by (torch.no_grad)")
        return _Delta.apply(q, k, v, g, beta, state, reset, scale, workspace)
    shape = _delta_shape(q, k, v, scale)
    size, states = v.shape, (v.shape[0], v.shape[2], q.shape[3], v.shape[3])
    o = torch.empty_like(v, memory_format=torch.contiguous_format) if out is None else out
    kept = last is not None
    if not kept:
        last = torch.empty(states, dtype=torch.float32, device=v.device) if state is None else torch.empty_like(state, memory_format=torch.contiguous_format)
    ws, base, avail = _space(workspace, lambda: gated_delta_workspace_bytes(size[0], size[1], size[2], q.shape[2], q.shape[3], size[3]), v.device)
    held, at = _heads(q.dtype, (q, q.shape, "q"), (k, q.shape, "k"), (v, size, "v"), (o, size, "out"))
    g_at, beta_at = _delta_gates(v, g, beta)
    _check(lib().rls_gated_delta(ctypes.byref(shape), at[0], at[1], at[2], g_at, beta_at, _rows_of(state, states, torch.float32, "state"), _resets(reset, size),
                                 at[3], _rows_of(last, states, torch.float32, "last"), base, avail, _raw_stream(v.get_device())), "rls_gated_delta")
    if out is not None:
        _written(o)
    if kept:
        _written(last)
    return o, last


class _Delta(torch.autograd.Function):
    """gated_delta as autograd sees it: both its results are differentiable."""

    @staticmethod
    def forward(ctx, q, k, v, g, beta, state, reset, scale, workspace):
        o, last = gated_delta(q, k, v, g, beta, state, reset, scale, workspace)
        ctx.save_for_backward(q, k, v, g, beta, state, reset)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return o, last

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, do, dlast):
        q, k, v, g, beta, state, reset = ctx.saved_tensors
        do = torch.zeros_like(v, memory_format=torch.contiguous_format) if do is None else do
        if do.stride(-1) != 1:
            do = do.contiguous()
        grads = gated_delta_backward(q, k, v, g, beta, do, state, reset, None if dlast is None else dlast.contiguous(), ctx.scale)
        return (*grads[:5], None if state is None else grads[5], None, None, None)


def gated_delta_backward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, g: torch.Tensor, beta: torch.Tensor, do: torch.Tensor,
                         state: Optional[torch.Tensor] = None, reset: Optional[torch.Tensor] = None, dlast: Optional[torch.Tensor] = None,
                         scale: Optional[float] = None, workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, ...]:
    """Gradients of gated_delta from its inputs and the gradients by its results: (dq, dk, dv in their types, dg, dbeta and dstate in fp32).

    Where an input was an expanded view, its gradient is that of every element: the sum along the expanded axes is the input's."""
    shape = _delta_shape(q, k, v, scale)
    size, states = v.shape, (v.shape[0], v.shape[2], q.shape[3], v.shape[3])
    dq, dk, dv, dg, dbeta = (torch.empty_like(t, memory_format=torch.contiguous_format) for t in (q, k, v, g, beta))
    dstate = torch.empty(states, dtype=torch.float32, device=v.device)
    ws, base, avail = _space(workspace, lambda: gated_delta_workspace_bytes(size[0], size[1], size[2], q.shape[2], q.shape[3], size[3], True), v.device)
    held, at = _heads(q.dtype, (q, q.shape, "q"), (k, q.shape, "k"), (v, size, "v"), (do, size, "do"), (dq, q.shape, "dq"), (dk, q.shape, "dk"), (dv, size, "dv"))
    g_at, beta_at = _delta_gates(v, g, beta)
    _check(lib().rls_gated_delta_backward(ctypes.byref(shape), at[0], at[1], at[2], g_at, beta_at, _rows_of(state, states, torch.float32, "state"),
                                          _resets(reset, size), at[3], _rows_of(dlast, states, torch.float32, "dlast"), at[4], at[5], at[6], dg.data_ptr(),
                                          dbeta.data_ptr(), dstate.data_ptr(), base, avail, _raw_stream(v.get_device())), "rls_gated_delta_backward")
    return dq, dk, dv, dg, dbeta, dstate


class AdamW:
    """An AdamW optimizer over a list of tensors (fp32, bf16 or fp16): one call per step updates them all.

    state_bits 32 keeps m and v in fp32; 8 keeps m and sqrt(v) as torch.float8_e4m3fn codes (stored as uint8) with a power-of-two scale per
    256 elements, rounded at random from `seed`.  master=True keeps fp32 weights beside bf16 or fp16 parameters.  The moments start at zero;
    exp_avg, exp_avg_sq, their scales and master, lists like params, take over existing ones (a resumed run: `step` steps already done).  The lists are
    the optimizer's own: a tensor put into one of them, or another memory given to a tensor (p.data = ...), counts from the next step on."""

    def __init__(self, params: Sequence[torch.Tensor], state_bits: int = 32, master=None, seed: int = 0, step: int = 0, exp_avg=None,
                 exp_avg_sq=None, exp_avg_scale=None, exp_avg_sq_scale=None):
        self.params, self.state_bits, self.seed, self.step_count = list(params), int(state_bits), int(seed), int(step)
        if self.state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        for p in self.params:
            self._check_param(p)
        if self.state_bits == 8 and ((exp_avg is None) != (exp_avg_scale is None) or (exp_avg_sq is None) != (exp_avg_sq_scale is None)):
            raise ValueError("moments in 8 bits need their scales, and scales their moments")
        held = torch.float32 if self.state_bits == 32 else torch.uint8
        shapes = [p.shape for p in self.params]
        self.exp_avg = self._list(exp_avg, held, shapes)
        self.exp_avg_sq = self._list(exp_avg_sq, held, shapes)
        self.exp_avg_scale = self.exp_avg_sq_scale = None
        if self.state_bits == 8:
            blocks = [((p.numel() + 255) // 256,) for p in self.params]
            self.exp_avg_scale = self._list(exp_avg_scale, torch.float32, blocks)
            self.exp_avg_sq_scale = self._list(exp_avg_sq_scale, torch.float32, blocks)
        if master is True:
            master = [p.detach().float() for p in self.params]
        self.master = list(master) if master else None
        self._take()

    def _list(self, given, dtype, shapes):
        return [torch.zeros(k, dtype=dtype, device=p.device) for p, k in zip(self.params, shapes)] if given is None else list(given)

    def _lists(self):
        """Everything that a step reads and writes, gradients aside: lists with a tensor per parameter."""
        return [x for x in (self.params, self.exp_avg, self.exp_avg_sq, self.exp_avg_scale, self.exp_avg_sq_scale, self.master) if x is not None]

    def _where(self):
        at = torch.Tensor.data_ptr
        places = [*map(at, self.params), *map(at, self.exp_avg), *map(at, self.exp_avg_sq)]
        if self.state_bits == 8:
            places += [*map(at, self.exp_avg_scale), *map(at, self.exp_avg_sq_scale)]
        if self.master is not None:
            places += map(at, self.master)
        return places

    @staticmethod
    def _check_param(p):
        if not p.is_cuda or p.dtype not in _TYPE_OF or not p.is_contiguous():
            raise ValueError("params must be contiguous device tensors of fp32, bf16 or fp16")

    def _take(self):
        """Checks all tensors and takes their addresses (again, where a list has got another tensor or a tensor other memory)."""
        self._addresses = None
        held, wide = (torch.float32, 1) if self.state_bits == 32 else (torch.uint8, 256)
        for name, given, dtype, block in (("exp_avg", self.exp_avg, held, 1), ("exp_avg_sq", self.exp_avg_sq, held, 1), ("master", self.master, torch.float32, 1),
                                          ("exp_avg_scale", self.exp_avg_scale, torch.float32, wide), ("exp_avg_sq_scale", self.exp_avg_sq_scale, torch.float32, wide)):
            if given is None:
                continue
            if len(given) != len(self.params):
                raise ValueError(f"{name} needs a tensor per parameter")
            for t, p in zip(given, self.params):
                if _dev(t, dtype, name).numel() != (p.numel() + block - 1) // block:
                    raise ValueError(f"{name} has a tensor of another size than its parameter's")
        every = [t for x in self._lists() for t in x]
        for p in self.params:
            self._check_param(p)
        self._device = self.params[0].get_device() if self.params else -1
        if any(t.get_device() != self._device for t in every):
            raise ValueError("an optimizer's tensors must be on one device")
        # (an fp32 parameter's entry in master is not used, and may be the parameter itself)
        used = [t for x in self._lists() for t, p in zip(x, self.params) if t.numel() > 0 and not (x is self.master and p.dtype == torch.float32)]
        places = sorted((t.data_ptr(), t.numel() * t.element_size()) for t in used)
        if any(at + size > after for (at, size), (after, _) in zip(places, places[1:])):
            raise ValueError("an optimizer's tensors must not overlap")
        self._tensors = (_AdamwTensor * max(1, len(self.params)))()
        self._each, self._forms = list(self._tensors)[:len(self.params)], [(p.shape, p.dtype) for p in self.params]
        for i, p in enumerate(self.params):
            t = self._each[i]
            t.n, t.param_type, t.param_dev = p.numel(), _TYPE_OF[p.dtype], p.data_ptr()
            t.m_dev, t.v_dev = self.exp_avg[i].data_ptr(), self.exp_avg_sq[i].data_ptr()
            t.master_dev = self.master[i].data_ptr() if self.master and p.dtype != torch.float32 else None
            if self.state_bits == 8:
                t.m_scale_dev, t.v_scale_dev = self.exp_avg_scale[i].data_ptr(), self.exp_avg_sq_scale[i].data_ptr()
        # (the memory stays with these while its addresses are here, so that none of it can become another tensor's)
        self._memory = [t.detach() for t in every]
        self._counted = [p for p in self.params if not p.is_inference()]        # (see _written)
        self._addresses, self._options = self._where(), _AdamwOptions()
        self._grad_types = [None] * len(self.params)

    def step(self, grads: Sequence[torch.Tensor], lr: float = 1e-3, betas: Tuple[float, float] = (0.9, 0.999), eps: float = 1e-8,
             weight_decay: float = 0.01, grad_scale: Optional[torch.Tensor] = None) -> None:
        """One step with these gradients (fp32 or the parameter's type), times grad_scale (one fp32 on the device) where given."""
        if self._where() != self._addresses:
            self._take()
        if len(grads) != len(self.params):
            raise ValueError("step needs a gradient per parameter")
        device = self._device
        for i, (t, (shape, dtype), g, known) in enumerate(zip(self._each, self._forms, grads, self._grad_types)):
            kind = g.dtype
            if g.shape != shape or g.get_device() != device or (kind is not dtype and kind is not torch.float32) or not g.is_contiguous():
                raise ValueError("a gradient must be a contiguous tensor on its parameter's device, of its shape, in fp32 or the parameter's type")
            t.grad_dev = g.data_ptr()
            if kind is not known:
                t.grad_type, self._grad_types[i] = _TYPE_OF[kind], kind
        if grad_scale is not None and _dev(grad_scale, torch.float32, "grad_scale").numel() != 1:
            raise ValueError("grad_scale must hold one number")
        o = self._options
        o.lr, (o.beta1, o.beta2), o.eps, o.weight_decay = lr, betas, eps, weight_decay
        o.step, o.seed, o.state_bits = self.step_count + 1, self.seed & 0xFFFFFFFFFFFFFFFF, self.state_bits
        o.grad_scale_dev = None if grad_scale is None else grad_scale.data_ptr()
        stream = _raw_stream(device) if self.params else 0
        _check(lib().rls_adamw_step(self._tensors, len(self.params), ctypes.byref(o), stream), "rls_adamw_step")
        torch._C._increment_version(self._counted)
        self.step_count += 1
