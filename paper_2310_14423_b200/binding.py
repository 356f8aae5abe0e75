"""Thin ctypes binding over libqsr.so: the same names as include/qsr.h, argument marshalling only.

Every step of the path runs in the library's CUDA kernels.  There is no CPU fallback: loading fails loudly if
the library has not been built (`python -m paper_2310_14423_b200.build`), and calls that need a device return
the library's error codes, raised here as QsrError.

torch is used by callers for device memory and streams; this module asks tensors for their address, layout and device.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqsr.so")

OPT = {"sgdm": 0, "adamw": 1}
SCHED = {"cosine": 0, "step_pow2": 1, "linear": 2, "const": 3, "halving": 4, "cosine_held": 5}
RULE = {"qsr": 0, "const_h": 1, "power": 2, "post_local": 3, "swap": 4}
STATE = {"keep": 0, "average": 1, "reset": 2}

QSR_OK, QSR_EINVAL, QSR_EALIGN, QSR_ECUDA, QSR_ERANGE, QSR_ESTATE = 0, -1, -2, -3, -4, -5
QSR_STATIC_SCRATCH_FLOATS = 1 << 20
QSR_MAX_TOP = 32
STATES = {"f32": 0, "e4m3": 1}
DTYPE = {"torch.float32": 0, "torch.bfloat16": 1, "torch.float16": 2}     # QSR_F32, QSR_BF16, QSR_F16
QSR_NONE = -1

EXPORTS = ("qsr_config_check", "qsr_row_stride_hint", "qsr_config_learning_rate", "qsr_config_round_length", "qsr_config_schedule",
           "qsr_workspace_bytes", "qsr_init", "qsr_destroy", "qsr_round_length", "qsr_set_tensor_table", "qsr_clip_workspace_floats", "qsr_set_grad_clip", "qsr_set_params", "qsr_local_step",
           "qsr_local_step_sync", "qsr_parallel_step", "qsr_sync", "qsr_sync_sum_floats", "qsr_sync_partial", "qsr_local_step_partial", "qsr_sync_finish", "qsr_sync_static", "qsr_run", "qsr_launch_count",
           "qsr_set_launch_shape", "qsr_set_graph_replay", "qsr_set_resident_steps", "qsr_train_host", "qsr_list_workspace_bytes", "qsr_list_create", "qsr_list_destroy", "qsr_list_set_grads",
           "qsr_list_step", "qsr_list_sync", "qsr_list_launch_count", "qsr_token_logprobs", "qsr_token_logprobs_grad", "qsr_muon_workspace_bytes",
           "qsr_muon_create", "qsr_muon_destroy", "qsr_muon_set_grads", "qsr_muon_step", "qsr_muon_sync", "qsr_muon_check", "qsr_muon_launch_count", "qsr_layer_norm",
           "qsr_layer_norm_workspace_bytes", "qsr_layer_norm_grad", "qsr_embed", "qsr_embed_workspace_bytes", "qsr_embed_grad", "qsr_debug_box_muller", "qsr_debug_fast_math", "qsr_debug_copy_patience",
           "qsr_strerror")


class QsrConfig(C.Structure):
    """Mirror of `qsr_config` in include/qsr.h (field order and types must match)."""
    _fields_ = [("K", C.c_int32), ("worker_offset", C.c_int32), ("P", C.c_int64), ("row_stride", C.c_int64),
                ("opt", C.c_int32), ("sched", C.c_int32), ("rule", C.c_int32), ("state_sync", C.c_int32),
                ("momentum", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("weight_decay", C.c_double), ("eta_max", C.c_double), ("eta_min", C.c_double),
                ("alpha", C.c_double), ("noise_std", C.c_double),
                ("T", C.c_int64), ("T_warmup", C.c_int64), ("H_base", C.c_int64), ("t_state_origin", C.c_int64),
                ("seed", C.c_uint64), ("gamma", C.c_double), ("t_switch", C.c_int64), ("t_hold", C.c_int64),
                ("t_period", C.c_int64)]


class QsrTensor(C.Structure):
    """Mirror of `qsr_tensor`."""
    _fields_ = [("param", C.c_void_p), ("copy", C.c_void_p), ("grad", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("m_scale", C.c_void_p), ("v_scale", C.c_void_p), ("numel", C.c_int64), ("param_type", C.c_int32),
                ("grad_type", C.c_int32), ("copy_type", C.c_int32), ("wd_scale", C.c_float)]


class QsrListConfig(C.Structure):
    """Mirror of `qsr_list_config`."""
    _fields_ = [("n_tensors", C.c_int32), ("workers", C.c_int32), ("states", C.c_int32), ("reserved", C.c_int32),
                ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("weight_decay", C.c_double),
                ("clip_norm", C.c_double), ("grad_norm", C.c_void_p)]


class QsrLogprobArgs(C.Structure):
    """Mirror of `qsr_logprob_args`."""
    _fields_ = [("logits", C.c_void_p), ("tokens", C.c_void_p), ("rows", C.c_int64), ("vocab", C.c_int64),
                ("row_stride", C.c_int64), ("logits_type", C.c_int32), ("n_top", C.c_int32), ("inv_temperature", C.c_double),
                ("logprob", C.c_void_p), ("entropy", C.c_void_p), ("row_stats", C.c_void_p), ("top_logprob", C.c_void_p),
                ("top_token", C.c_void_p), ("d_logprob", C.c_void_p), ("d_entropy", C.c_void_p), ("d_logits", C.c_void_p),
                ("d_row_stride", C.c_int64)]


class QsrMatrix(C.Structure):
    """Mirror of `qsr_matrix`."""
    _fields_ = [("param", C.c_void_p), ("copy", C.c_void_p), ("grad", C.c_void_p), ("momentum", C.c_void_p), ("rows", C.c_int64),
                ("cols", C.c_int64), ("param_type", C.c_int32), ("grad_type", C.c_int32), ("copy_type", C.c_int32), ("wd_scale", C.c_float),
                ("update_scale", C.c_float), ("reserved", C.c_int32)]


class QsrMuonConfig(C.Structure):
    """Mirror of `qsr_muon_config`."""
    _fields_ = [("n_matrices", C.c_int32), ("workers", C.c_int32), ("products", C.c_int32), ("iterations", C.c_int32), ("nesterov", C.c_int32),
                ("reserved", C.c_int32), ("beta", C.c_double), ("eps", C.c_double), ("weight_decay", C.c_double)]


class QsrLayerNormArgs(C.Structure):
    """Mirror of `qsr_layer_norm_args`."""
    _fields_ = [("x", C.c_void_p), ("weight", C.c_void_p), ("bias", C.c_void_p), ("mean", C.c_void_p), ("rstd", C.c_void_p),
                ("rows", C.c_int64), ("width", C.c_int64), ("x_stride", C.c_int64), ("type", C.c_int32), ("weight_type", C.c_int32),
                ("eps", C.c_double), ("y", C.c_void_p), ("y_stride", C.c_int64), ("d_y", C.c_void_p), ("d_y_stride", C.c_int64),
                ("d_x", C.c_void_p), ("d_x_stride", C.c_int64), ("d_weight", C.c_void_p), ("d_bias", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64)]


class QsrEmbedArgs(C.Structure):
    """Mirror of `qsr_embed_args`."""
    _fields_ = [("table", C.c_void_p), ("tokens", C.c_void_p), ("out", C.c_void_p), ("rows", C.c_int64), ("vocab", C.c_int64),
                ("width", C.c_int64), ("table_stride", C.c_int64), ("out_stride", C.c_int64), ("table_type", C.c_int32),
                ("out_type", C.c_int32), ("scale", C.c_double), ("accumulate", C.c_int32), ("reserved", C.c_int32),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64)]


class QsrError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = int(status)
        super().__init__(f"{where}: {strerror(status)} (status {status})")


_lib = None


def lib():
    """The loaded library.  Raises if it is missing: the product has no other implementation to fall back to."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} not found; build it with `python -m paper_2310_14423_b200.build` "
                              "(needs nvcc; there is no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        cfg, vp, i64, i32 = C.POINTER(QsrConfig), C.c_void_p, C.c_int64, C.c_int32
        sig = {
            "qsr_config_check": (C.c_int, [cfg]),
            "qsr_row_stride_hint": (i64, [i64]),
            "qsr_config_learning_rate": (C.c_double, [cfg, i64]),
            "qsr_config_round_length": (i64, [cfg, i64]),
            "qsr_config_schedule": (i64, [cfg, vp, vp, i64]),
            "qsr_workspace_bytes": (i64, [cfg]),
            "qsr_init": (C.c_int, [C.POINTER(vp), cfg, vp, vp, vp, vp, vp, vp]),
            "qsr_destroy": (C.c_int, [vp]),
            "qsr_round_length": (i64, [vp, i64]),
            "qsr_set_tensor_table": (C.c_int, [vp, i32, vp, vp]),
            "qsr_clip_workspace_floats": (i64, [vp]),
            "qsr_set_grad_clip": (C.c_int, [vp, C.c_double, vp]),
            "qsr_set_params": (C.c_int, [vp, vp]),
            "qsr_local_step": (C.c_int, [vp, i64, vp]),
            "qsr_local_step_sync": (C.c_int, [vp, i64, vp, i64]),
            "qsr_parallel_step": (C.c_int, [vp, i64, vp]),
            "qsr_sync": (C.c_int, [vp, i64]),
            "qsr_sync_sum_floats": (i64, [vp]),
            "qsr_sync_partial": (C.c_int, [vp, vp]),
            "qsr_local_step_partial": (C.c_int, [vp, i64, vp, vp]),
            "qsr_sync_finish": (C.c_int, [vp, vp, i32, i64]),
            "qsr_sync_static": (C.c_int, [vp, i64]),
            "qsr_run": (C.c_int, [vp, i64, i64, vp, vp, i64, C.POINTER(i64)]),
            "qsr_launch_count": (i64, [vp]),
            "qsr_set_launch_shape": (C.c_int, [vp, i32, i32, i32]),
            "qsr_set_graph_replay": (C.c_int, [vp, i32]),
            "qsr_set_resident_steps": (C.c_int, [vp, i32]),
            "qsr_train_host": (C.c_int, [cfg, vp, vp, vp, vp, vp, i64, i64, vp, vp, vp, i64, C.POINTER(i64), C.POINTER(i64)]),
            "qsr_list_workspace_bytes": (i64, [vp, i32, i32]),
            "qsr_list_create": (C.c_int, [C.POINTER(vp), C.POINTER(QsrListConfig), C.POINTER(QsrTensor), vp, i64, vp]),
            "qsr_list_destroy": (C.c_int, [vp]),
            "qsr_list_set_grads": (C.c_int, [vp, vp]),
            "qsr_list_step": (C.c_int, [vp, i64, C.c_double, C.c_double]),
            "qsr_list_sync": (C.c_int, [vp, i32]),
            "qsr_list_launch_count": (i64, [vp]),
            "qsr_token_logprobs": (C.c_int, [C.POINTER(QsrLogprobArgs), vp]),
            "qsr_token_logprobs_grad": (C.c_int, [C.POINTER(QsrLogprobArgs), vp]),
            "qsr_muon_workspace_bytes": (i64, [vp, vp, i32, i32, i32]),
            "qsr_muon_create": (C.c_int, [C.POINTER(vp), C.POINTER(QsrMuonConfig), C.POINTER(QsrMatrix), vp, i64, vp]),
            "qsr_muon_destroy": (C.c_int, [vp]),
            "qsr_muon_set_grads": (C.c_int, [vp, vp]),
            "qsr_muon_step": (C.c_int, [vp, C.c_double, C.c_double]),
            "qsr_muon_sync": (C.c_int, [vp, i32]),
            "qsr_muon_check": (C.c_int, [vp]),
            "qsr_muon_launch_count": (i64, [vp]),
            "qsr_layer_norm": (C.c_int, [C.POINTER(QsrLayerNormArgs), vp]),
            "qsr_layer_norm_workspace_bytes": (i64, [i64, i64]),
            "qsr_layer_norm_grad": (C.c_int, [C.POINTER(QsrLayerNormArgs), vp]),
            "qsr_embed": (C.c_int, [C.POINTER(QsrEmbedArgs), vp]),
            "qsr_embed_workspace_bytes": (i64, [i64, i64, i64]),
            "qsr_embed_grad": (C.c_int, [C.POINTER(QsrEmbedArgs), vp]),
            "qsr_debug_box_muller": (C.c_int, [vp, i64, vp, vp, vp, vp]),
            "qsr_debug_fast_math": (C.c_int, [vp, i64, vp, vp, vp]),
            "qsr_debug_copy_patience": (C.c_int, [i64]),
            "qsr_strerror": (C.c_char_p, [C.c_int]),
        }
        for name in EXPORTS:
            fn = getattr(L, name)
            fn.restype, fn.argtypes = sig[name]
        _lib = L
    return _lib


def strerror(status: int) -> str:
    return lib().qsr_strerror(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != QSR_OK:
        raise QsrError(status, where)


def make_config(w, K: Optional[int] = None, row_stride: Optional[int] = None, worker_offset: Optional[int] = None,
                t_state_origin: int = 0) -> QsrConfig:
    """qsr_config from a workload description (an object with the fields of workloads.Workload)."""
    P = int(w.P)
    return QsrConfig(K=int(w.K if K is None else K),
                     worker_offset=int(w.worker_offset if worker_offset is None else worker_offset),
                     P=P, row_stride=int((P + 3) // 4 * 4 if row_stride is None else row_stride),
                     opt=OPT[w.opt], sched=SCHED[w.sched], rule=RULE[w.rule], state_sync=STATE[w.state_sync],
                     momentum=w.momentum, beta1=w.beta1, beta2=w.beta2, eps=w.eps, weight_decay=w.weight_decay,
                     eta_max=w.eta_max, eta_min=w.eta_min, alpha=w.alpha, noise_std=w.noise_std,
                     T=int(w.T), T_warmup=int(w.T_warmup), H_base=int(w.H_base), t_state_origin=int(t_state_origin),
                     seed=int(w.noise_seed), gamma=float(getattr(w, "gamma", 2.0)),
                     t_switch=int(getattr(w, "t_switch", 0)), t_hold=int(getattr(w, "t_hold", 0)),
                     t_period=max(1, int(getattr(w, "t_period", 1))))


# ---- host-only schedule ---------------------------------------------------------------------------------

def qsr_config_check(cfg: QsrConfig) -> int:
    return int(lib().qsr_config_check(C.byref(cfg)))


def qsr_config_learning_rate(cfg: QsrConfig, t: int) -> float:
    return float(lib().qsr_config_learning_rate(C.byref(cfg), int(t)))


def qsr_config_round_length(cfg: QsrConfig, t: int) -> int:
    H = int(lib().qsr_config_round_length(C.byref(cfg), int(t)))
    if H < 0:
        raise QsrError(H, "qsr_config_round_length")
    return H


def qsr_config_schedule(cfg: QsrConfig) -> Tuple[np.ndarray, np.ndarray]:
    cap = int(cfg.T)
    st, H = np.empty(cap, np.int64), np.empty(cap, np.int64)
    n = int(lib().qsr_config_schedule(C.byref(cfg), st.ctypes.data, H.ctypes.data, cap))
    if n < 0:
        raise QsrError(n, "qsr_config_schedule")
    return st[:n].copy(), H[:n].copy()


def qsr_row_stride_hint(P: int) -> int:
    n = int(lib().qsr_row_stride_hint(int(P)))
    if n < 0:
        raise QsrError(n, "qsr_row_stride_hint")
    return n


def qsr_workspace_bytes(cfg: QsrConfig) -> int:
    n = int(lib().qsr_workspace_bytes(C.byref(cfg)))
    if n < 0:
        raise QsrError(n, "qsr_workspace_bytes")
    return n


# ---- context --------------------------------------------------------------------------------------------

class _Names(dict):
    """Name of a torch dtype; kept, because forming it anew costs more than the rest of an argument's check."""

    def __missing__(self, dtype):
        self[dtype] = name = str(dtype)
        return name


_NAMES = _Names()


def _current_device() -> int:
    """Index of the device that the library's launches go to (torch is initialised: callers hold a CUDA tensor)."""
    global _current_device
    from torch._C import _cuda_getDevice
    _current_device = _cuda_getDevice          # from now on without the way round through Python
    return _current_device()


def _dptr(t) -> Optional[int]:
    """Device address of a torch tensor (or None)."""
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous CUDA tensor")
    return int(t.data_ptr())


class Context:
    """Owner of one `qsr_ctx`.  Keeps references to the tensors whose memory the library borrows."""

    def __init__(self, cfg: QsrConfig, params, state1, state2=None, lam=None, theta_star=None, stream: int = 0):
        self.cfg = cfg
        self._keep = (params, state1, state2, lam, theta_star)
        self._h = C.c_void_p()
        _check(lib().qsr_init(C.byref(self._h), C.byref(cfg), _dptr(params), _dptr(state1), _dptr(state2),
                              _dptr(lam), _dptr(theta_star), C.c_void_p(stream)), "qsr_init")

    def close(self) -> None:
        if self._h:
            lib().qsr_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def qsr_round_length(self, t: int) -> int:
        H = int(lib().qsr_round_length(self._h, int(t)))
        if H < 0:
            raise QsrError(H, "qsr_round_length")
        return H

    def qsr_set_tensor_table(self, tensor_end=None, wd_scale=None) -> None:
        """tensor_end: CUDA int64 tensor [n]; wd_scale: CUDA float32 tensor [n]; None clears the table."""
        n = 0 if tensor_end is None else int(tensor_end.numel())
        self._table = (tensor_end, wd_scale)
        _check(lib().qsr_set_tensor_table(self._h, n, _dptr(tensor_end), _dptr(wd_scale)), "qsr_set_tensor_table")

    def qsr_clip_workspace_floats(self) -> int:
        return int(lib().qsr_clip_workspace_floats(self._h))

    def qsr_set_grad_clip(self, max_norm: float, workspace=None) -> None:
        self._clip_ws = workspace
        _check(lib().qsr_set_grad_clip(self._h, float(max_norm), _dptr(workspace)), "qsr_set_grad_clip")

    def qsr_set_params(self, theta0) -> None:
        _check(lib().qsr_set_params(self._h, _dptr(theta0)), "qsr_set_params")

    def qsr_local_step(self, t: int, grads=None) -> None:
        _check(lib().qsr_local_step(self._h, int(t), _dptr(grads)), "qsr_local_step")

    def qsr_local_step_sync(self, t: int, t_next: int, grads=None) -> None:
        _check(lib().qsr_local_step_sync(self._h, int(t), _dptr(grads), int(t_next)), "qsr_local_step_sync")

    def qsr_parallel_step(self, t: int, grads=None) -> None:
        _check(lib().qsr_parallel_step(self._h, int(t), _dptr(grads)), "qsr_parallel_step")

    def qsr_sync(self, t_next: int) -> None:
        _check(lib().qsr_sync(self._h, int(t_next)), "qsr_sync")

    def qsr_sync_sum_floats(self) -> int:
        return int(lib().qsr_sync_sum_floats(self._h))

    def qsr_sync_partial(self, sums) -> None:
        _check(lib().qsr_sync_partial(self._h, _dptr(sums)), "qsr_sync_partial")

    def qsr_local_step_partial(self, t: int, sums, grads=None) -> None:
        _check(lib().qsr_local_step_partial(self._h, int(t), _dptr(grads), _dptr(sums)), "qsr_local_step_partial")

    def qsr_sync_finish(self, sums, K_total: int, t_next: int) -> None:
        _check(lib().qsr_sync_finish(self._h, _dptr(sums), int(K_total), int(t_next)), "qsr_sync_finish")

    def qsr_sync_static(self, t_next: int) -> None:
        """qsr_sync through the library's built-in scratch array: for callers that cannot allocate the `sum` buffer.
        Raises QsrError(QSR_ERANGE) when the problem exceeds QSR_STATIC_SCRATCH_FLOATS."""
        _check(lib().qsr_sync_static(self._h, int(t_next)), "qsr_sync_static")

    def qsr_run(self, t_begin: int = 0, t_end: Optional[int] = None) -> Tuple[np.ndarray, np.ndarray]:
        t_end = int(self.cfg.T if t_end is None else t_end)
        cap = max(1, t_end - int(t_begin))
        st, H = np.empty(cap, np.int64), np.empty(cap, np.int64)
        n = C.c_int64(0)
        _check(lib().qsr_run(self._h, int(t_begin), t_end, st.ctypes.data, H.ctypes.data, cap, C.byref(n)), "qsr_run")
        return st[:n.value].copy(), H[:n.value].copy()

    def qsr_launch_count(self) -> int:
        return int(lib().qsr_launch_count(self._h))

    def qsr_set_graph_replay(self, max_steps_per_graph: int) -> None:
        _check(lib().qsr_set_graph_replay(self._h, max_steps_per_graph), "qsr_set_graph_replay")

    def qsr_set_resident_steps(self, max_steps_per_launch: int) -> None:
        """Benchmark-only: up to this many consecutive steps per launch, state held in registers (0 = off)."""
        _check(lib().qsr_set_resident_steps(self._h, max_steps_per_launch), "qsr_set_resident_steps")

    def qsr_set_launch_shape(self, step_threads: int = 0, step_rows_in_flight: int = 0, sync_threads: int = 0) -> None:
        _check(lib().qsr_set_launch_shape(self._h, step_threads, step_rows_in_flight, sync_threads), "qsr_set_launch_shape")


def qsr_train_host(cfg: QsrConfig, theta0: np.ndarray, lam: np.ndarray, theta_star: np.ndarray, theta_out: np.ndarray,
                   workspace, t_end: Optional[int] = None, stream: int = 0):
    """Whole run from host arrays (numpy float32 [P], or pinned torch CPU tensors exposing data_ptr()).
    `workspace` is a CUDA tensor of at least qsr_workspace_bytes(cfg) bytes.
    Returns (round starts, round lengths, kernel launches)."""
    def hptr(a):
        return int(a.ctypes.data) if isinstance(a, np.ndarray) else int(a.data_ptr())
    t_end = int(cfg.T if t_end is None else t_end)
    cap = max(1, t_end)
    st, H = np.empty(cap, np.int64), np.empty(cap, np.int64)
    n, launches = C.c_int64(0), C.c_int64(0)
    nbytes = int(workspace.numel() * workspace.element_size())
    _check(lib().qsr_train_host(C.byref(cfg), hptr(theta0), hptr(lam), hptr(theta_star), hptr(theta_out),
                                _dptr(workspace), nbytes, t_end, C.c_void_p(stream),
                                st.ctypes.data, H.ctypes.data, cap, C.byref(n), C.byref(launches)), "qsr_train_host")
    return st[:n.value].copy(), H[:n.value].copy(), int(launches.value)


# ---- lists of tensors -----------------------------------------------------------------------------------

def _dense(t) -> bool:
    """Whether the tensor's elements fill a stretch of memory without gaps, in whatever order of dimensions."""
    if t.is_contiguous():
        return True
    expect = 1
    for stride, size in sorted((st, n) for st, n in zip(t.stride(), t.shape) if n != 1):
        if stride != expect:
            return False
        expect *= size
    return True


def _element(t, like, what: str, i: int, dtypes=DTYPE):
    """Device address of operand `what` of list entry i: a dense CUDA tensor with as many elements as the parameter, in the
    same order in memory."""
    name, device = _NAMES[t.dtype], like.get_device()
    if name not in dtypes:
        raise ValueError(f"{what}[{i}]: {name} is not supported (one of {', '.join(sorted(dtypes))})")
    if device < 0 or t.get_device() != device:
        raise ValueError(f"{what}[{i}]: expected a CUDA tensor on {like.device}")
    numel = t.numel()
    if numel != like.numel():
        raise ValueError(f"{what}[{i}]: {numel} elements for a parameter of {like.numel()}")
    if not (t.is_contiguous() and like.is_contiguous()) and not (t.shape == like.shape and t.stride() == like.stride() and _dense(t)):
        raise ValueError(f"{what}[{i}]: shape {tuple(t.shape)} with strides {t.stride()} does not lie in memory like its parameter")
    return t.data_ptr() if numel else None


def qsr_list_workspace_bytes(numels, workers: int = 1) -> int:
    """Bytes of device workspace for a TensorList over tensors of these sizes (all workers' tensors)."""
    a = np.ascontiguousarray(list(numels), np.int64)
    n = int(lib().qsr_list_workspace_bytes(a.ctypes.data, a.size, int(workers)))
    if n < 0:
        raise QsrError(n, "qsr_list_workspace_bytes")
    return n


def _in_use(tensors, stream: int, device) -> None:
    """Keeps the tensors' memory from being given out again before `stream` has done its work so far."""
    import torch
    on = torch.cuda.ExternalStream(stream, device) if stream else torch.cuda.default_stream(device)
    for t in tensors:
        if t is not None:
            t.record_stream(on)


class TensorList:
    """Owner of one `qsr_list`: AdamW steps and replica means over a model's own tensors.

    params / grads / copies: lists of CUDA tensors in float32, bfloat16 or float16 (grads and copies may be None, or None in
    places); with several workers, worker 0's tensors first, then worker 1's, and so on.  m, v: float32 tensors, or
    float8_e4m3fn with m_scale / v_scale (float32, one per 256 elements, in memory order).  wd_scale: a factor on the
    weight decay per tensor (default 1).  workspace: a CUDA tensor of qsr_list_workspace_bytes bytes.  Keeps references
    to the tensors whose memory the library borrows.

    Work goes to `stream`, and the caller orders it after what fills the tensors.  Gradients that qsr_list_set_grads replaces are
    marked as in use there (Tensor.record_stream), so that their memory is not given out again while an enqueued step reads
    it.  All other tensors, and the last gradients, are let go with the list: with `stream` idle, or recorded by the caller."""

    def __init__(self, params, grads, m, v, m_scale=None, v_scale=None, copies=None, wd_scale=None, workers: int = 1,
                 beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.0,
                 clip_norm: float = 0.0, grad_norm=None, workspace=None, stream: int = 0):
        self._h = C.c_void_p()
        n = len(params)
        columns = {"grads": grads, "m": m, "v": v, "m_scale": m_scale, "v_scale": v_scale, "copies": copies, "wd_scale": wd_scale}
        for what, column in columns.items():
            if column is None and what in ("m", "v"):
                raise ValueError(f"{what} is required")
            if column is not None and len(column) != n:
                raise ValueError(f"{what}: {len(column)} entries for {n} parameters")
        codes = n > 0 and str(m[0].dtype) == "torch.float8_e4m3fn"
        if codes and (m_scale is None or v_scale is None):
            raise ValueError("states in 8 bits need m_scale and v_scale")
        state_types = {"torch.float8_e4m3fn": 0} if codes else {"torch.float32": 0}
        device = params[0].get_device() if n else -1
        for what, t in [("workspace", workspace), ("grad_norm", grad_norm)]:
            if t is not None and n and t.get_device() != device:
                raise ValueError(f"{what}: expected a CUDA tensor on cuda:{device}")
        entries = (QsrTensor * max(1, n))()
        for i, p in enumerate(params):
            e = entries[i]
            e.numel, e.param_type, e.wd_scale = p.numel(), DTYPE.get(str(p.dtype), QSR_NONE), 1.0 if wd_scale is None else wd_scale[i]
            e.param = _element(p, p, "params", i)
            if p.get_device() != device:
                raise ValueError(f"params[{i}]: expected a CUDA tensor on cuda:{device}")
            e.m, e.v = _element(m[i], p, "m", i, state_types), _element(v[i], p, "v", i, state_types)
            e.copy_type = QSR_NONE
            if copies is not None and copies[i] is not None:
                e.copy, e.copy_type = _element(copies[i], p, "copies", i), DTYPE[str(copies[i].dtype)]
            g = None if grads is None else grads[i]
            if g is not None:
                e.grad, e.grad_type = _element(g, p, "grads", i), DTYPE[str(g.dtype)]
            else:
                e.grad_type = e.param_type
            if codes:
                for name, scales in (("m_scale", m_scale), ("v_scale", v_scale)):
                    if str(scales[i].dtype) != "torch.float32" or scales[i].numel() != (p.numel() + 255) // 256 or scales[i].get_device() != device:
                        raise ValueError(f"{name}[{i}]: one float32 per 256 elements is expected, on cuda:{device}")
                    setattr(e, name, _dptr(scales[i]) if p.numel() else None)
        if grad_norm is not None and (str(grad_norm.dtype) != "torch.float32" or grad_norm.numel() != workers):
            raise ValueError("grad_norm: one float32 per worker is expected")
        if n and device != _current_device():
            raise ValueError(f"the tensors are on cuda:{device}, which is not the current device")
        cfg = QsrListConfig(n_tensors=n, workers=int(workers), states=STATES["e4m3" if codes else "f32"], beta1=beta1, beta2=beta2,
                            eps=eps, weight_decay=weight_decay, clip_norm=clip_norm, grad_norm=_dptr(grad_norm))
        nbytes = 0 if workspace is None else int(workspace.numel() * workspace.element_size())
        self._params, self._grad_types = list(params), [entries[i].grad_type for i in range(n)]
        self._keep = [None if x is None else list(x) for x in (m, v, m_scale, v_scale, copies)] + [grad_norm, workspace]
        self._grads, self._stream = None if grads is None else list(grads), int(stream)
        _check(lib().qsr_list_create(C.byref(self._h), C.byref(cfg), entries, _dptr(workspace), nbytes, C.c_void_p(stream)),
               "qsr_list_create")

    def close(self) -> None:
        if self._h:
            lib().qsr_list_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def qsr_list_set_grads(self, grads) -> None:
        """New gradient tensors (one per parameter, of the types the list was made with)."""
        if len(grads) != len(self._params):
            raise ValueError(f"{len(grads)} gradients for {len(self._params)} parameters")
        only = {v: {k: 0} for k, v in DTYPE.items()}
        table = (C.c_void_p * max(1, len(grads)))()
        for i, (g, p) in enumerate(zip(grads, self._params)):
            table[i] = _element(g, p, "grads", i, only[self._grad_types[i]])
        _check(lib().qsr_list_set_grads(self._h, table), "qsr_list_set_grads")
        if self._grads is not None:
            _in_use(self._grads, self._stream, self._params[0].device)
        self._grads = list(grads)

    def qsr_list_step(self, n: int, lr: float, grad_scale: float = 1.0) -> None:
        _check(lib().qsr_list_step(self._h, n, lr, grad_scale), "qsr_list_step")

    def qsr_list_sync(self, state_sync: str = "keep") -> None:
        _check(lib().qsr_list_sync(self._h, STATE[state_sync]), "qsr_list_sync")

    def qsr_list_launch_count(self) -> int:
        return int(lib().qsr_list_launch_count(self._h))


# ---- log probabilities of given tokens ------------------------------------------------------------------

def _vector(t, what: str, n: int, dtype: str, device: int) -> Optional[int]:
    """Device address of a contiguous tensor of n elements of `dtype` on the CUDA device of that index; None for None."""
    if t is None:
        return None
    if _NAMES[t.dtype] != dtype or t.numel() != n or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{what}: a contiguous tensor of {n} x {dtype} on cuda:{device} is expected")
    return t.data_ptr()


def _matrix(t, shape, what: str, device: int):
    """Row stride of a matrix with adjacent columns (that of a single row means nothing) on the CUDA device of that index."""
    if len(shape) != 2 or device < 0 or t.get_device() != device:
        raise ValueError(f"{what}: a CUDA matrix is expected, all tensors on the same device")
    if t.is_contiguous():
        return shape[1]
    stride = t.stride()
    if shape[1] > 1 and stride[1] != 1:
        raise ValueError(f"{what}: a matrix with adjacent columns is expected")
    return max(stride[0], shape[1]) if shape[0] <= 1 else stride[0]


def _logprob_args(logits, tokens, inv_temperature, entropy, row_stats, d_logprob, d_entropy, d_logits) -> Tuple[QsrLogprobArgs, int, int]:
    """Arguments that both calls share, with the number of rows and the index of the device."""
    shape, device = logits.shape, logits.get_device()
    stride, kind = _matrix(logits, shape, "logits", device), DTYPE.get(_NAMES[logits.dtype])
    if kind is None:
        raise ValueError(f"logits: {logits.dtype} is not supported (one of {', '.join(sorted(DTYPE))})")
    R, V = shape
    f32 = "torch.float32"
    if device != _current_device():
        raise ValueError(f"the logits are on cuda:{device}, which is not the current device")
    a = QsrLogprobArgs(logits.data_ptr(), _vector(tokens, "tokens", R, "torch.int64", device), R, V, stride, kind, 0, inv_temperature, None,
                       _vector(entropy, "entropy", R, f32, device), _vector(row_stats, "row_stats", 2 * R, f32, device), None, None,
                       _vector(d_logprob, "d_logprob", R, f32, device), _vector(d_entropy, "d_entropy", R, f32, device))
    if d_logits is not None:
        if d_logits.shape != shape or d_logits.dtype != logits.dtype:
            raise ValueError("d_logits: shape and type of the logits are expected")
        a.d_logits, a.d_row_stride = d_logits.data_ptr(), _matrix(d_logits, shape, "d_logits", device)
    return a, R, device


def qsr_token_logprobs(logits, tokens, logprob, entropy=None, row_stats=None, top_logprob=None, top_token=None,
                       inv_temperature: float = 1.0, d_logprob=None, d_entropy=None, d_logits=None, stream: int = 0) -> None:
    """Log probability of each row's token, with optional entropy, row statistics, top alternatives ([rows, n] tensors, n at
    most QSR_MAX_TOP) and, if d_logits is given, the gradient in the same pass.  All tensors are the caller's."""
    a, R, device = _logprob_args(logits, tokens, inv_temperature, entropy, row_stats, d_logprob, d_entropy, d_logits)
    a.logprob = _vector(logprob, "logprob", R, "torch.float32", device)
    if (top_logprob is None) != (top_token is None):
        raise ValueError("top_logprob and top_token come together")
    if top_token is not None:
        if top_token.dim() != 2:
            raise ValueError("top_token: [rows, n] is expected")
        a.n_top = n = top_token.shape[1]
        a.top_logprob = _vector(top_logprob, "top_logprob", R * n, "torch.float32", device)
        a.top_token = _vector(top_token, "top_token", R * n, "torch.int64", device)
    _check(lib().qsr_token_logprobs(C.byref(a), stream), "qsr_token_logprobs")


def qsr_token_logprobs_grad(logits, tokens, row_stats, d_logits, d_logprob=None, d_entropy=None, entropy=None,
                            inv_temperature: float = 1.0, stream: int = 0) -> None:
    """Gradient of sum(d_logprob * logprob + d_entropy * entropy) with respect to the logits, from the row_stats (and entropy)
    that qsr_token_logprobs wrote for the same logits and temperature."""
    a, _, _ = _logprob_args(logits, tokens, inv_temperature, entropy, row_stats, d_logprob, d_entropy, d_logits)
    _check(lib().qsr_token_logprobs_grad(C.byref(a), stream), "qsr_token_logprobs_grad")


# ---- matrices stepped by their orthogonalised momentum --------------------------------------------------

def qsr_muon_workspace_bytes(shapes, workers: int = 1, products: int = 1) -> int:
    """Bytes of device workspace for a MuonList over matrices of these (rows, columns) (all workers' matrices)."""
    rows, cols = (np.ascontiguousarray([int(s[i]) for s in shapes], np.int64) for i in (0, 1))
    n = int(lib().qsr_muon_workspace_bytes(rows.ctypes.data, cols.ctypes.data, rows.size, int(workers), int(products)))
    if n < 0:
        raise QsrError(n, "qsr_muon_workspace_bytes")
    return n


def _entry(t, like, what: str, i: int, dtypes=DTYPE):
    """Device address of operand `what` of matrix i: contiguous and of the parameter's shape."""
    if t.shape != like.shape or not t.is_contiguous():
        raise ValueError(f"{what}[{i}]: a contiguous matrix of shape {tuple(like.shape)} is expected")
    return _element(t, like, what, i, dtypes)


class MuonList:
    """Owner of one `qsr_muon`: steps of matrices by their orthogonalised momentum, and replica means over them.

    params / grads / copies: lists of contiguous 2-D CUDA tensors in float32, bfloat16 or float16 (grads and copies may be None, or
    None in places); momentum: float32; with several workers, worker 0's matrices first, then worker 1's, and so on.
    wd_scale, update_scale: factors on the weight decay and on the update per matrix (default: 1, and sqrt(max(1, rows / columns))).
    products: 1 (fp16: right for bf16 parameters) or 3 (nearly fp32, at three times the cost; for fp32 and fp16 parameters whose
    steps are compared with fp32 ones); include/qsr.h has the errors.  workspace: a CUDA tensor of qsr_muon_workspace_bytes bytes.  Keeps references to the
    tensors whose memory the library borrows; streams and lifetimes as at TensorList."""

    def __init__(self, params, grads, momentum, copies=None, wd_scale=None, update_scale=None, workers: int = 1, beta: float = 0.95,
                 nesterov: bool = True, weight_decay: float = 0.0, eps: float = 1e-7, iterations: int = 5, products: int = 1,
                 workspace=None, stream: int = 0):
        self._h = C.c_void_p()
        n = len(params)
        for what, column in (("grads", grads), ("momentum", momentum), ("copies", copies), ("wd_scale", wd_scale), ("update_scale", update_scale)):
            if column is None and what == "momentum":
                raise ValueError("momentum is required")
            if column is not None and len(column) != n:
                raise ValueError(f"{what}: {len(column)} entries for {n} matrices")
        device = params[0].get_device() if n else -1
        if workspace is not None and n and workspace.get_device() != device:
            raise ValueError(f"workspace: expected a CUDA tensor on cuda:{device}")
        entries = (QsrMatrix * max(1, n))()
        for i, p in enumerate(params):
            if p.dim() != 2:
                raise ValueError(f"params[{i}]: a matrix is expected")
            e = entries[i]
            e.rows, e.cols = p.shape
            e.param, e.param_type = _entry(p, p, "params", i), DTYPE.get(_NAMES[p.dtype], QSR_NONE)
            if p.get_device() != device:
                raise ValueError(f"params[{i}]: expected a CUDA tensor on cuda:{device}")
            e.momentum = _entry(momentum[i], p, "momentum", i, {"torch.float32": 0})
            e.copy_type = QSR_NONE
            if copies is not None and copies[i] is not None:
                e.copy, e.copy_type = _entry(copies[i], p, "copies", i), DTYPE[_NAMES[copies[i].dtype]]
            g = None if grads is None else grads[i]
            e.grad_type = e.param_type
            if g is not None:
                e.grad, e.grad_type = _entry(g, p, "grads", i), DTYPE[_NAMES[g.dtype]]
            e.wd_scale = 1.0 if wd_scale is None else wd_scale[i]
            e.update_scale = max(1.0, e.rows / max(1, e.cols)) ** 0.5 if update_scale is None else update_scale[i]
        if n:
            _on_current(device, "the matrices are")
        cfg = QsrMuonConfig(n_matrices=n, workers=int(workers), products=int(products), iterations=int(iterations), nesterov=int(bool(nesterov)),
                            beta=beta, eps=eps, weight_decay=weight_decay)
        nbytes = 0 if workspace is None else int(workspace.numel() * workspace.element_size())
        self._params, self._grad_types = list(params), [entries[i].grad_type for i in range(n)]
        self._keep = [None if x is None else list(x) for x in (momentum, copies)] + [workspace]
        self._grads, self._stream = None if grads is None else list(grads), int(stream)
        _check(lib().qsr_muon_create(C.byref(self._h), C.byref(cfg), entries, _dptr(workspace), nbytes, C.c_void_p(stream)), "qsr_muon_create")

    def close(self) -> None:
        if self._h:
            lib().qsr_muon_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def qsr_muon_set_grads(self, grads) -> None:
        """New gradient tensors (one per matrix, of the types the list was made with)."""
        if len(grads) != len(self._params):
            raise ValueError(f"{len(grads)} gradients for {len(self._params)} matrices")
        only = {v: {k: 0} for k, v in DTYPE.items()}
        table = (C.c_void_p * max(1, len(grads)))()
        for i, (g, p) in enumerate(zip(grads, self._params)):
            table[i] = _entry(g, p, "grads", i, only[self._grad_types[i]])
        _check(lib().qsr_muon_set_grads(self._h, table), "qsr_muon_set_grads")
        if self._grads is not None:
            _in_use(self._grads, self._stream, self._params[0].device)
        self._grads = list(grads)

    def qsr_muon_step(self, lr: float, grad_scale: float = 1.0) -> None:
        _check(lib().qsr_muon_step(self._h, lr, grad_scale), "qsr_muon_step")

    def qsr_muon_sync(self, state_sync: str = "keep") -> None:
        _check(lib().qsr_muon_sync(self._h, STATE[state_sync]), "qsr_muon_sync")

    def qsr_muon_check(self) -> None:
        """Waits for the stream; raises if a wait inside an earlier step ran out."""
        _check(lib().qsr_muon_check(self._h), "qsr_muon_check")

    def qsr_muon_launch_count(self) -> int:
        return int(lib().qsr_muon_launch_count(self._h))


# ---- layer norm and embedding ---------------------------------------------------------------------------

def _kind(t, what: str) -> int:
    kind = DTYPE.get(_NAMES[t.dtype])
    if kind is None:
        raise ValueError(f"{what}: {t.dtype} is not supported (one of {', '.join(sorted(DTYPE))})")
    return kind


def _workspace(t, device: int) -> Tuple[Optional[int], int]:
    """Address and bytes of a workspace on the CUDA device of that index."""
    if t is None:
        return None, 0
    if t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"workspace: a contiguous tensor on cuda:{device} is expected")
    return t.data_ptr(), int(t.numel() * t.element_size())


def _on_current(device: int, what: str) -> None:
    if device != _current_device():
        raise ValueError(f"{what} on cuda:{device}, which is not the current device")


def _like(t, x, shape, what: str, device: int) -> Tuple[int, int]:
    """Address and row stride of a matrix of the shape and type of x."""
    if t.shape != shape or t.dtype != x.dtype:
        raise ValueError(f"{what}: shape and type of x are expected")
    return t.data_ptr(), _matrix(t, shape, what, device)


def qsr_layer_norm(x, y, weight=None, bias=None, mean=None, rstd=None, eps: float = 1e-5, stream: int = 0) -> None:
    """Layer norm of each row of x into y (x itself is fine), with optional weight and bias (one type), and the rows' statistics
    (float32) that qsr_layer_norm_grad takes.  Matrices may be columns of wider buffers.  All tensors are the caller's."""
    shape, device = x.shape, x.get_device()
    stride = _matrix(x, shape, "x", device)
    _on_current(device, "x is")
    R, N = shape
    kind = _kind(x, "x")
    given = weight if weight is not None else bias
    weight_kind, name = (kind, "") if given is None else (_kind(given, "weight"), _NAMES[given.dtype])
    to, y_stride = _like(y, x, shape, "y", device)
    a = QsrLayerNormArgs(x.data_ptr(), _vector(weight, "weight", N, name, device), _vector(bias, "bias", N, name, device),
                         _vector(mean, "mean", R, "torch.float32", device), _vector(rstd, "rstd", R, "torch.float32", device), R, N, stride, kind,
                         weight_kind, eps, to, y_stride)
    _check(lib().qsr_layer_norm(C.byref(a), stream), "qsr_layer_norm")


def qsr_layer_norm_workspace_bytes(rows: int, width: int) -> int:
    """Bytes of device workspace for the gradients of weight and bias."""
    n = int(lib().qsr_layer_norm_workspace_bytes(rows, width))
    if n < 0:
        raise QsrError(n, "qsr_layer_norm_workspace_bytes")
    return n


def qsr_layer_norm_grad(x, d_y, mean, rstd, d_x=None, weight=None, d_weight=None, d_bias=None, workspace=None, stream: int = 0) -> None:
    """Gradients of layer norm from the statistics that qsr_layer_norm wrote: of x (x or d_y may be written over), and of weight and
    bias (of the weight's type, with a workspace of qsr_layer_norm_workspace_bytes bytes), each if it is given."""
    shape, device = x.shape, x.get_device()
    stride = _matrix(x, shape, "x", device)
    _on_current(device, "x is")
    R, N = shape
    kind = _kind(x, "x")
    given = weight if weight is not None else d_weight if d_weight is not None else d_bias
    weight_kind, name = (kind, "") if given is None else (_kind(given, "weight"), _NAMES[given.dtype])
    dy, dy_stride = _like(d_y, x, shape, "d_y", device)
    dx, dx_stride = (None, N) if d_x is None else _like(d_x, x, shape, "d_x", device)
    at, nbytes = _workspace(workspace, device)
    a = QsrLayerNormArgs(x.data_ptr(), _vector(weight, "weight", N, name, device), None, _vector(mean, "mean", R, "torch.float32", device),
                         _vector(rstd, "rstd", R, "torch.float32", device), R, N, stride, kind, weight_kind, 0.0, None, N, dy, dy_stride, dx, dx_stride,
                         _vector(d_weight, "d_weight", N, name, device), _vector(d_bias, "d_bias", N, name, device), at, nbytes)
    _check(lib().qsr_layer_norm_grad(C.byref(a), stream), "qsr_layer_norm_grad")


def _embed_args(table, tokens, out, scale, table_name: str, out_name: str) -> Tuple[QsrEmbedArgs, int]:
    device = table.get_device()
    (V, N), (R, columns) = shape, out_shape = table.shape, out.shape
    stride, out_stride = _matrix(table, shape, table_name, device), _matrix(out, out_shape, out_name, device)
    _on_current(device, f"{table_name} is")
    if columns != N:
        raise ValueError(f"{out_name}: {columns} columns for a table of {N}")
    return QsrEmbedArgs(table.data_ptr(), _vector(tokens, "tokens", R, "torch.int64", device), out.data_ptr(), R, V, N, stride, out_stride,
                        _kind(table, table_name), _kind(out, out_name), scale), device


def qsr_embed(table, tokens, out, scale: float = 1.0, stream: int = 0) -> None:
    """out[r] = scale * table[tokens[r]] (zeros where a token is negative).  The matrices may differ in type, and be columns of
    wider buffers."""
    a, _ = _embed_args(table, tokens, out, scale, "table", "out")
    _check(lib().qsr_embed(C.byref(a), stream), "qsr_embed")


def qsr_embed_workspace_bytes(rows: int, vocab: int, width: int) -> int:
    """Bytes of device workspace for qsr_embed_grad."""
    n = int(lib().qsr_embed_workspace_bytes(rows, vocab, width))
    if n < 0:
        raise QsrError(n, "qsr_embed_workspace_bytes")
    return n


def qsr_embed_grad(d_out, tokens, d_table, scale: float = 1.0, accumulate: bool = False, workspace=None, stream: int = 0) -> None:
    """Gradient of qsr_embed's table: written whole, or (accumulate) added to the rows of tokens that occur."""
    a, device = _embed_args(d_table, tokens, d_out, scale, "d_table", "d_out")
    a.accumulate = 1 if accumulate else 0
    a.workspace, a.workspace_bytes = _workspace(workspace, device)
    _check(lib().qsr_embed_grad(C.byref(a), stream), "qsr_embed_grad")


def qsr_debug_box_muller(words, radius, sine, cosine, stream: int = 0) -> None:
    """Test hook: Box-Muller radius / sine / cosine of each uint32 generator word (CUDA tensors; words as int32 bits)."""
    n = int(words.numel())
    _check(lib().qsr_debug_box_muller(_dptr(words), n, _dptr(radius), _dptr(sine), _dptr(cosine), C.c_void_p(stream)),
           "qsr_debug_box_muller")


def qsr_debug_fast_math(x, root, reciprocal, stream: int = 0) -> None:
    """Test hook: the library's single-instruction square root and reciprocal of each float of x (CUDA tensors)."""
    _check(lib().qsr_debug_fast_math(_dptr(x), int(x.numel()), _dptr(root), _dptr(reciprocal), C.c_void_p(stream)),
           "qsr_debug_fast_math")


def qsr_debug_copy_patience(clocks: int = -1) -> None:
    """Test hook: limit of the waits for copies in layer norm's kernels from now on; 0: they run out at once, negative: the usual one."""
    _check(lib().qsr_debug_copy_patience(int(clocks)), "qsr_debug_copy_patience")
