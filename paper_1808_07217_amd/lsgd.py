"""Python binding of liblsgd (ctypes): argument marshalling only.

Every step of the local-SGD path runs in the HIP kernels behind the C ABI
declared in include/lsgd.h. PyTorch supplies device memory and the stream.
If the library has not been built this module raises ImportError; there is
no fallback implementation.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import NamedTuple, Optional, Sequence, Tuple, Union

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblsgd.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m "
        "paper_1808_07217_amd.build` (hipcc, gfx950) before use")

MAX_LAYERS = 8
FP32, BF16 = 0, 1
MODELS = {"mlp": 0, "resnet20": 1}
SCHEMES = {"local": 0, "sign": 1, "ef_sign": 2}
SAMPLERS = {"iid": 0, "epoch": 1}
_c = ctypes


class Config(_c.Structure):
    _fields_ = [
        ("model", _c.c_int32),
        ("n_layers", _c.c_int32),
        ("widths", _c.c_int32 * (MAX_LAYERS + 1)),
        ("K", _c.c_int32),
        ("B_loc", _c.c_int32),
        ("gemm_dtype", _c.c_int32),
        ("nesterov", _c.c_int32),
        ("momentum", _c.c_float),
        ("weight_decay", _c.c_float),
        ("global_momentum", _c.c_float),
        ("scheme", _c.c_int32),
        ("sampler", _c.c_int32),
        ("seed", _c.c_uint64),
        ("N", _c.c_int64),
    ]


_lib = _c.CDLL(LIB_PATH)
_P = _c.c_void_p
_I, _L = _c.c_int32, _c.c_int64
_SIGS = {
    "lsgd_param_count": [_c.POINTER(Config), _c.POINTER(_c.c_int64)],
    "lsgd_workspace_bytes": [_c.POINTER(Config), _c.POINTER(_c.c_size_t)],
    "lsgd_init_replicas": [_c.POINTER(Config), _P, _P, _P, _P, _c.c_size_t, _P,
                           _c.POINTER(_P)],
    "lsgd_local_step": [_P, _c.c_float, _P],
    "lsgd_average": [_P],
    "lsgd_run_round": [_P, _c.c_int32, _c.POINTER(_c.c_float), _P],
    "lsgd_average_blocks": [_P, _c.c_int32],
    "lsgd_synchronise": [_P, _c.c_float],
    "lsgd_read_error_memory": [_P, _c.c_int32, _P],
    "lsgd_write_momentum": [_P, _c.c_int32, _P],
    "lsgd_write_error_memory": [_P, _c.c_int32, _P],
    "lsgd_sign_sync_scratch_bytes": [_c.c_int32, _c.c_int64, _P],
    "lsgd_replica_sign_sync": [_P, _c.c_int32, _c.c_int64, _P, _P, _P,
                               _c.c_size_t, _P],
    "lsgd_replica_sign_sync_static": [_P, _c.c_int32, _c.c_int64, _P, _P, _P],
    "lsgd_read_global_momentum": [_P, _P],
    "lsgd_write_global_momentum": [_P, _P],
    "lsgd_replica_average_global_momentum": [_P, _c.c_int32, _c.c_int64, _P, _P,
                                             _c.c_float, _c.c_float, _P],
    "lsgd_run_hierarchical_round": [_P, _c.c_int32, _c.c_int32, _c.c_int32,
                                    _c.POINTER(_c.c_float), _P],
    "lsgd_read_params": [_P, _c.c_int32, _P],
    "lsgd_read_momentum": [_P, _c.c_int32, _P],
    "lsgd_write_params": [_P, _c.c_int32, _P],
    "lsgd_get_step": [_P, _c.POINTER(_c.c_int64)],
    "lsgd_set_step": [_P, _c.c_int64],
    "lsgd_sample_indices": [_P, _c.c_int64, _P],
    "lsgd_sync": [_P],
    "lsgd_state_bytes": [_c.POINTER(Config), _c.POINTER(_c.c_size_t)],
    "lsgd_set_lazy_average": [_P, _c.c_int32],
    "lsgd_read_state": [_P, _P],
    "lsgd_write_state": [_P, _P],
    "lsgd_destroy": [_P],
    "lsgd_status_string": [_c.c_int],
    "lsgd_last_error": [_P],
    "lsgd_profile_enable": [_P, _c.c_int32],
    "lsgd_profile_select": [_P, _c.c_char_p, _c.c_int32],
    "lsgd_profile_report": [_P, _c.c_char_p, _c.c_size_t],
    "lsgd_grouped_gemm": [_c.c_int32, _c.c_int32, _c.c_int32, _c.c_int32,
                          _c.c_int32, _c.c_int32, _c.c_int32, _P, _c.c_int64,
                          _c.c_int64, _P, _c.c_int64, _c.c_int64, _P,
                          _c.c_int32, _P, _P],
    "lsgd_replica_average": [_P, _c.c_int32, _c.c_int64, _P],
    "lsgd_replica_average_blocks": [_P, _c.c_int32, _c.c_int32, _c.c_int64, _P],
    "lsgd_sgd_update": [_P, _P, _P, _c.c_int64, _c.c_float, _c.c_float,
                        _c.c_float, _c.c_int32, _P],
    "lsgd_quantise_blocks": [_I, _I, _I, _I, _I, _P, _L, _L, _P, _P, _P, _P, _P],
    "lsgd_grouped_gemm_blocks_workspace_bytes": [_I, _I, _I, _I, _I, _c.POINTER(_c.c_size_t)],
    "lsgd_grouped_gemm_blocks_cut": [_I, _I, _I, _I, _I, _P],
    "lsgd_grouped_gemm_blocks": [_I, _I, _I, _I, _I, _I, _I, _P, _L, _P, _L, _P, _L, _P, _L,
                                 _P, _L, _L, _P, _c.c_size_t, _P],
    "lsgd_orthogonalise_workspace_bytes": [_I, _I, _I, _I, _c.POINTER(_c.c_size_t)],
    "lsgd_orthogonalise_cut": [_I, _I, _I, _I, _P],
    "lsgd_orthogonalise": [_I, _I, _I, _I, _P, _L, _L, _P, _L, _L, _I, _c.POINTER(_c.c_float),
                           _c.c_float, _P, _c.c_size_t, _P],
    "lsgd_orthogonal_update": [_I, _I, _I, _I, _P, _L, _L, _P, _L, _L, _P, _L, _L, _c.c_float,
                               _c.c_float, _c.c_float, _I, _c.c_float, _I,
                               _c.POINTER(_c.c_float), _c.c_float, _P, _c.c_size_t, _P],
}
for _name, _args in _SIGS.items():
    _f = getattr(_lib, _name)
    _f.argtypes = _args
    _f.restype = _c.c_int
_lib.lsgd_status_string.restype = _c.c_char_p
_lib.lsgd_last_error.restype = _c.c_char_p

EXPORTED = tuple(_SIGS)


E_NONFINITE = 6
STATE_MAGIC = 0x3154535F4447534C
STATE_SECTIONS = ("W", "U", "RS", "w_sync", "u_global", "E")


class LsgdError(RuntimeError):
    def __init__(self, msg, status):
        super().__init__(msg)
        self.status = status


class NonFiniteLoss(LsgdError):
    """lsgd_sync reported LSGD_E_NONFINITE: a local step's loss was not
    finite."""


def _check(status: int, ctx=None) -> None:
    if status != 0:
        msg = _lib.lsgd_status_string(status).decode()
        if ctx:
            detail = _lib.lsgd_last_error(ctx).decode()
            if detail:
                msg += f" ({detail})"
        cls = NonFiniteLoss if status == E_NONFINITE else LsgdError
        raise cls(f"liblsgd: {msg} [status {status}]", status)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else _c.c_void_p(t.data_ptr())


def _stream_handle(stream) -> _c.c_void_p:
    return _c.c_void_p(stream.cuda_stream)


def make_config(widths: Sequence[int], K: int, B_loc: int, N: int, *,
                dtype: str = "fp32", momentum: float = 0.0,
                weight_decay: float = 0.0, nesterov: bool = False,
                seed: int = 0, model: str = "mlp",
                global_momentum: float = 0.0, scheme: str = "local",
                sampler: str = "iid") -> Config:
    """widths: d_0 .. d_L for the MLP; (3072, classes) for resnet20."""
    if not 2 <= len(widths) <= MAX_LAYERS + 1:
        raise ValueError("widths must list d_0 .. d_L with 1 <= L <= 8")
    cfg = Config()
    cfg.model = MODELS[model]
    cfg.n_layers = len(widths) - 1
    for i, w in enumerate(widths):
        cfg.widths[i] = int(w)
    cfg.K, cfg.B_loc, cfg.N = int(K), int(B_loc), int(N)
    cfg.gemm_dtype = {"fp32": FP32, "bf16": BF16}[dtype]
    cfg.nesterov = int(bool(nesterov))
    cfg.momentum = float(momentum)
    cfg.weight_decay = float(weight_decay)
    cfg.global_momentum = float(global_momentum)
    cfg.scheme = SCHEMES[scheme]
    cfg.sampler = SAMPLERS[sampler]
    cfg.seed = int(seed) & (2**64 - 1)
    return cfg


def param_count(cfg: Config) -> int:
    out = _c.c_int64()
    _check(_lib.lsgd_param_count(_c.byref(cfg), _c.byref(out)))
    return out.value


def workspace_bytes(cfg: Config) -> int:
    out = _c.c_size_t()
    _check(_lib.lsgd_workspace_bytes(_c.byref(cfg), _c.byref(out)))
    return out.value


def state_bytes(cfg: Config) -> int:
    out = _c.c_size_t()
    _check(_lib.lsgd_state_bytes(_c.byref(cfg), _c.byref(out)))
    return out.value


def _aligned_bytes(n: int, device) -> torch.Tensor:
    """A uint8 device tensor of n bytes starting on a 256-byte boundary."""
    raw = torch.empty(n + 256, dtype=torch.uint8, device=device)
    off = (-raw.data_ptr()) % 256
    return raw[off:off + n]


def parse_state(blob: torch.Tensor) -> dict:
    """The header fields and section views (float32 [rows][n] on the blob's
    device) of a state blob, by the layout lsgd.h documents."""
    words = blob[:64].cpu().view(torch.int64).tolist()
    if words[0] & (2**64 - 1) != STATE_MAGIC:
        raise ValueError("not a state blob")
    K, P, R, step, mask, total = words[2], words[3], words[4], words[5], words[6], words[7]
    out = {"K": K, "P": P, "R": R, "step": step, "mask": mask, "bytes": total}
    o = 256
    shapes = {"W": (K, P), "U": (K, P), "RS": (K, R), "w_sync": (1, P),
              "u_global": (1, P), "E": (K, P)}
    for i, name in enumerate(STATE_SECTIONS):
        if not mask >> i & 1:
            continue
        rows, n = shapes[name]
        out[name] = blob[o:o + rows * n * 4].view(torch.float32).view(rows, n)
        o = (o + rows * n * 4 + 255) // 256 * 256
    return out


class Replicas:
    """K model replicas resident on one GPU (the K workers of local SGD)."""

    def __init__(self, cfg: Config, X: torch.Tensor, y: torch.Tensor,
                 w0: torch.Tensor, stream: Optional[torch.cuda.Stream] = None):
        dev = X.device
        if dev.type != "cuda":
            raise ValueError("X must be a CUDA (HIP) tensor")
        if X.dtype != torch.float32 or not X.is_contiguous() or X.dim() != 2:
            raise ValueError("X must be a contiguous float32 [N][d_0] tensor")
        if y.dtype != torch.int32 or y.device != dev or y.numel() != X.shape[0]:
            raise ValueError("y must be int32 [N] on X's device")
        if X.shape[0] != cfg.N or X.shape[1] != cfg.widths[0]:
            raise ValueError("X shape does not match the config")
        self.cfg = cfg
        self.K, self.B = cfg.K, cfg.B_loc
        self.P = param_count(cfg)
        if w0.dtype != torch.float32 or w0.numel() != self.P or w0.device != dev:
            raise ValueError(f"w0 must be float32 [{self.P}] on X's device")
        self.device = dev
        self.stream = stream or torch.cuda.current_stream(dev)
        nbytes = workspace_bytes(cfg)
        self._ws_raw = torch.empty(nbytes + 256, dtype=torch.uint8, device=dev)
        off = (-self._ws_raw.data_ptr()) % 256
        self.ws = self._ws_raw[off:off + nbytes]
        self._keep = (X, y, w0.contiguous())
        ctx = _c.c_void_p()
        _check(_lib.lsgd_init_replicas(
            _c.byref(cfg), _ptr(X), _ptr(y), _ptr(self._keep[2]), _ptr(self.ws),
            nbytes, _stream_handle(self.stream), _c.byref(ctx)))
        self._ctx = ctx

    # -- hot path --------------------------------------------------------
    def local_step(self, lr: float, loss: Optional[torch.Tensor] = None):
        _check(_lib.lsgd_local_step(self._ctx, float(lr), _ptr(loss)), self._ctx)

    def average(self):
        _check(_lib.lsgd_average(self._ctx), self._ctx)

    def set_lazy_average(self, enable: bool = True):
        """The lazy form of the plain average (lsgd_set_lazy_average)."""
        _check(_lib.lsgd_set_lazy_average(self._ctx, int(bool(enable))), self._ctx)

    def run_round(self, lrs: Sequence[float], loss: Optional[torch.Tensor] = None):
        H = len(lrs)
        arr = (_c.c_float * max(H, 1))(*[float(v) for v in lrs])
        _check(_lib.lsgd_run_round(self._ctx, H, arr, _ptr(loss)), self._ctx)

    def synchronise(self, lr: float):
        """End-of-round synchronisation: the average, or with a global
        momentum factor its momentum form at step size ``lr``."""
        _check(_lib.lsgd_synchronise(self._ctx, float(lr)), self._ctx)

    def average_blocks(self, Kb: int):
        """Hierarchical block synchronisation: each block of Kb consecutive
        replicas takes its mean."""
        _check(_lib.lsgd_average_blocks(self._ctx, int(Kb)), self._ctx)

    def run_hierarchical_round(self, H: int, Hb: int, Kb: int,
                               lrs: Sequence[float],
                               loss: Optional[torch.Tensor] = None):
        """Hb x (H local steps, block average over blocks of Kb), then the
        global average; ``lrs`` holds the H * Hb step sizes."""
        if len(lrs) != H * Hb:
            raise ValueError("lrs must hold H * Hb step sizes")
        arr = (_c.c_float * max(1, len(lrs)))(*[float(v) for v in lrs])
        _check(_lib.lsgd_run_hierarchical_round(self._ctx, int(H), int(Hb),
                                                int(Kb), arr, _ptr(loss)),
               self._ctx)

    # -- state -----------------------------------------------------------
    def read_params(self, replica: int = -1, out=None) -> torch.Tensor:
        out = out if out is not None else torch.empty(self.P, device=self.device)
        _check(_lib.lsgd_read_params(self._ctx, int(replica), _ptr(out)), self._ctx)
        return out

    def read_global_momentum(self, out=None) -> torch.Tensor:
        out = out if out is not None else torch.empty(self.P, device=self.device)
        _check(_lib.lsgd_read_global_momentum(self._ctx, _ptr(out)), self._ctx)
        return out

    def write_global_momentum(self, src: torch.Tensor):
        src = src.contiguous()
        if src.dtype != torch.float32 or src.numel() != self.P:
            raise ValueError("src must be float32 with P elements")
        _check(_lib.lsgd_write_global_momentum(self._ctx, _ptr(src)), self._ctx)

    def write_momentum(self, replica: int, src: torch.Tensor):
        src = src.contiguous()
        if src.dtype != torch.float32 or src.numel() != self.P:
            raise ValueError("src must be float32 with P elements")
        _check(_lib.lsgd_write_momentum(self._ctx, int(replica), _ptr(src)), self._ctx)

    def read_error_memory(self, replica: int, out=None) -> torch.Tensor:
        out = out if out is not None else torch.empty(self.P, device=self.device)
        _check(_lib.lsgd_read_error_memory(self._ctx, int(replica), _ptr(out)),
               self._ctx)
        return out

    def write_error_memory(self, replica: int, src: torch.Tensor):
        src = src.contiguous()
        if src.dtype != torch.float32 or src.numel() != self.P:
            raise ValueError("src must be float32 with P elements")
        _check(_lib.lsgd_write_error_memory(self._ctx, int(replica), _ptr(src)),
               self._ctx)

    def read_momentum(self, replica: int, out=None) -> torch.Tensor:
        out = out if out is not None else torch.empty(self.P, device=self.device)
        _check(_lib.lsgd_read_momentum(self._ctx, int(replica), _ptr(out)), self._ctx)
        return out

    def write_params(self, src: torch.Tensor, replica: int = -1):
        if src.dtype != torch.float32 or src.numel() != self.P:
            raise ValueError("src must be float32 [P]")
        _check(_lib.lsgd_write_params(self._ctx, int(replica), _ptr(src)), self._ctx)

    @property
    def step(self) -> int:
        out = _c.c_int64()
        _check(_lib.lsgd_get_step(self._ctx, _c.byref(out)))
        return out.value

    @step.setter
    def step(self, s: int):
        _check(_lib.lsgd_set_step(self._ctx, int(s)), self._ctx)

    def sample_indices(self, step: int) -> torch.Tensor:
        out = torch.empty((self.K, self.B), dtype=torch.int32, device=self.device)
        _check(_lib.lsgd_sample_indices(self._ctx, int(step), _ptr(out)), self._ctx)
        return out

    def profile(self, enable: bool = True):
        """Bracket every launch with HIP events (see lsgd_profile_enable)."""
        _check(_lib.lsgd_profile_enable(self._ctx, int(bool(enable))), self._ctx)

    def profile_select(self, tag: Optional[str] = None, every: int = 1):
        """Bracket only every ``every``-th launch tagged ``tag`` (None: all
        launches)."""
        _check(_lib.lsgd_profile_select(
            self._ctx, None if tag is None else tag.encode(), int(every)),
            self._ctx)

    def profile_report(self) -> dict:
        """{tag: (launches, total_ms)} since profiling was enabled; clears."""
        buf = _c.create_string_buffer(1 << 16)
        _check(_lib.lsgd_profile_report(self._ctx, buf, len(buf)), self._ctx)
        out = {}
        for line in buf.value.decode().splitlines():
            tag, n, ms = line.split()
            out[tag] = (int(n), float(ms))
        return out

    def sync(self):
        """Wait for the stream; raises NonFiniteLoss after a non-finite
        loss (see lsgd_sync)."""
        _check(_lib.lsgd_sync(self._ctx), self._ctx)

    def read_state(self, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The whole training state as one device blob (lsgd_read_state)."""
        n = state_bytes(self.cfg)
        out = out if out is not None else _aligned_bytes(n, self.device)
        if out.dtype != torch.uint8 or out.numel() < n or out.data_ptr() % 256:
            raise ValueError(f"out must be a 256-byte aligned uint8 tensor of {n} bytes")
        _check(_lib.lsgd_read_state(self._ctx, _ptr(out)), self._ctx)
        return out

    def write_state(self, blob: torch.Tensor):
        """Restore a blob written by read_state (lsgd_write_state)."""
        if blob.dtype != torch.uint8 or blob.data_ptr() % 256:
            raise ValueError("blob must be a 256-byte aligned uint8 tensor")
        _check(_lib.lsgd_write_state(self._ctx, _ptr(blob)), self._ctx)

    def close(self):
        if getattr(self, "_ctx", None):
            _lib.lsgd_destroy(self._ctx)
            self._ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def run_schedule(reps: Replicas, schedule, loss: Optional[torch.Tensor] = None):
    """Run rounds [(H_t, lr_t), ...] back to back; ``loss`` (fp32 [sum H_t][K])
    receives the per-step, per-replica losses."""
    row = 0
    for H, lr in schedule:
        reps.run_round([lr] * H, None if loss is None else loss[row:row + H])
        row += H


def post_local_schedule(H: int, rounds: int, lr: float, warm_rounds: int = 0,
                        lr_after_switch: Optional[float] = None):
    """Post-local SGD (section 3 of the paper): H_(t) = 1 for t <= t'
    (= warm_rounds), else H; the step size switches at the same time."""
    lr2 = lr if lr_after_switch is None or warm_rounds == 0 else lr_after_switch
    return [(1, lr)] * warm_rounds + [(H, lr2)] * rounds


# -- building blocks ------------------------------------------------------
def grouped_gemm(A: torch.Tensor, B: torch.Tensor, trans_a=False, trans_b=False,
                 out: Optional[torch.Tensor] = None, splits: int = 1) -> torch.Tensor:
    """C[g] = op(A[g]) @ op(B[g]) on the matrix cores (fp32 or bf16 inputs,
    fp32 accumulation and output). A, B are contiguous 3-D tensors; splits > 1
    runs the split-K path."""
    if A.dtype != B.dtype or A.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("A and B must both be float32 or both bfloat16")
    if A.dim() != 3 or B.dim() != 3 or A.shape[0] != B.shape[0]:
        raise ValueError("A, B must be [G][.][.] with the same G")
    A, B = A.contiguous(), B.contiguous()
    G = A.shape[0]
    M, Kd = (A.shape[2], A.shape[1]) if trans_a else (A.shape[1], A.shape[2])
    Kb, N = (B.shape[2], B.shape[1]) if trans_b else (B.shape[1], B.shape[2])
    if Kb != Kd:
        raise ValueError("inner dimensions differ")
    out = out if out is not None else torch.empty((G, M, N), device=A.device)
    dt = BF16 if A.dtype == torch.bfloat16 else FP32
    part = (torch.empty((splits, G, M, N), device=A.device) if splits > 1
            else None)
    _check(_lib.lsgd_grouped_gemm(
        dt, int(trans_a), int(trans_b), G, M, N, Kd, _ptr(A), A.shape[2],
        A.shape[1] * A.shape[2], _ptr(B), B.shape[2], B.shape[1] * B.shape[2],
        _ptr(out), int(splits), _ptr(part),
        _stream_handle(torch.cuda.current_stream(A.device))))
    return out


def replica_average(W: torch.Tensor) -> None:
    """In-place K-way average of a contiguous float32 [K][P] tensor."""
    if W.dtype != torch.float32 or W.dim() != 2 or not W.is_contiguous():
        raise ValueError("W must be contiguous float32 [K][P]")
    _check(_lib.lsgd_replica_average(
        _ptr(W), W.shape[0], W.shape[1],
        _stream_handle(torch.cuda.current_stream(W.device))))


def replica_average_blocks(W: torch.Tensor, Kb: int) -> None:
    """In-place average within each block of Kb consecutive rows of a
    contiguous float32 [K][P] tensor."""
    if W.dtype != torch.float32 or W.dim() != 2 or not W.is_contiguous():
        raise ValueError("W must be contiguous float32 [K][P]")
    _check(_lib.lsgd_replica_average_blocks(
        _ptr(W), W.shape[0], int(Kb), W.shape[1],
        _stream_handle(torch.cuda.current_stream(W.device))))


def replica_average_global_momentum(W: torch.Tensor, w_sync: torch.Tensor,
                                    u_global: torch.Tensor, m_global: float,
                                    lr: float) -> None:
    """In place: W [K][P] := the global-momentum synchronisation of its rows;
    w_sync and u_global ([P] float32) are updated."""
    for t in (W, w_sync, u_global):
        if t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError("tensors must be contiguous float32")
    if W.dim() != 2 or w_sync.numel() != W.shape[1] or u_global.numel() != W.shape[1]:
        raise ValueError("W must be [K][P], w_sync and u_global [P]")
    _check(_lib.lsgd_replica_average_global_momentum(
        _ptr(W), W.shape[0], W.shape[1], _ptr(w_sync), _ptr(u_global),
        float(m_global), float(lr),
        _stream_handle(torch.cuda.current_stream(W.device))))


def replica_sign_sync(W: torch.Tensor, w_sync: torch.Tensor,
                      E: Optional[torch.Tensor] = None) -> None:
    """In place: the sign-compressed synchronisation of the rows of W [K][P]
    (Algorithm 3; Algorithm 4 with the error memories E [K][P]); w_sync [P]
    is updated. P must be a multiple of 4."""
    ts = (W, w_sync) if E is None else (W, w_sync, E)
    for t in ts:
        if t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError("tensors must be contiguous float32")
    if W.dim() != 2 or w_sync.numel() != W.shape[1] or (
            E is not None and E.shape != W.shape):
        raise ValueError("W, E must be [K][P] and w_sync [P]")
    K, P = W.shape
    nb = _c.c_size_t()
    _check(_lib.lsgd_sign_sync_scratch_bytes(K, P, _c.byref(nb)))
    scratch = torch.empty(max(1, nb.value), dtype=torch.uint8, device=W.device)
    _check(_lib.lsgd_replica_sign_sync(
        _ptr(W), K, P, _ptr(w_sync), _ptr(E), _ptr(scratch), nb.value,
        _stream_handle(torch.cuda.current_stream(W.device))))


def replica_sign_sync_static(W: torch.Tensor, w_sync: torch.Tensor,
                             E: Optional[torch.Tensor] = None) -> None:
    """replica_sign_sync through the entry point that allocates nothing (its
    scratch is the library's static device array)."""
    ts = (W, w_sync) if E is None else (W, w_sync, E)
    for t in ts:
        if t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError("tensors must be contiguous float32")
    if W.dim() != 2 or w_sync.numel() != W.shape[1] or (
            E is not None and E.shape != W.shape):
        raise ValueError("W, E must be [K][P] and w_sync [P]")
    K, P = W.shape
    _check(_lib.lsgd_replica_sign_sync_static(
        _ptr(W), K, P, _ptr(w_sync), _ptr(E),
        _stream_handle(torch.cuda.current_stream(W.device))))


def sgd_update(W, U, G, lr, momentum, weight_decay, nesterov=False,
               sign_step=False) -> None:
    """In-place fused momentum-SGD update of float32 tensors W, U with grad G
    (``sign_step``: move by the sign of the direction, Algorithm 3)."""
    for t in (W, U, G):
        if t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError("W, U, G must be contiguous float32")
    _check(_lib.lsgd_sgd_update(
        _ptr(W), _ptr(U), _ptr(G), W.numel(), float(lr), float(momentum),
        float(weight_decay), int(bool(nesterov)) | (2 if sign_step else 0),
        _stream_handle(torch.cuda.current_stream(W.device))))


# -- large layers: products in 8 bits, orthogonalised updates --------------
FORMATS = {"e4m3": (0, torch.float8_e4m3fn), "e5m2": (1, torch.float8_e5m2)}
# of five Newton-Schulz steps (K. Jordan et al., "Muon: an optimizer for hidden layers in
# neural networks", 2024)
COEFFICIENTS = (3.4445, -4.7750, 2.0315)


class Blocks(NamedTuple):
    """G matrices of M rows and n columns in 8 bits with a scale for each row
    and 128 columns (the layout of lsgd_quantise_blocks): q [G][M][up(n, 128)],
    float8_e4m3fn or float8_e5m2, zeros past column n, and scale
    [G][M][up(ceil(n / 128), 4)], float8_e8m0fnu, 1 past the last block."""
    q: torch.Tensor
    scale: torch.Tensor
    n: int


def _up(n: int, m: int) -> int:
    return (n + m - 1) // m * m


def _enqueue(device: torch.device, call, *args) -> None:
    """``call(*args, stream)`` on the device's current stream, with that device the
    calling thread's. (The stream's raw handle: a torch.cuda.Stream object costs as
    much as the launch.)"""
    i = device.index
    if i == torch.cuda.current_device():
        _check(call(*args, torch._C._cuda_getCurrentRawStream(i)))
    else:
        with torch.cuda.device(i):
            _check(call(*args, torch._C._cuda_getCurrentRawStream(i)))


_FLOATS = (torch.float32, torch.bfloat16)
_FP32 = (torch.float32,)


def _matrices(name: str, X: torch.Tensor, dtypes) -> Tuple[int, int]:
    """Row pitch and group stride of a [G][M][N] device tensor whose columns are
    contiguous."""
    if X.dim() != 3 or X.dtype not in dtypes:
        raise ValueError(f"{name} must be [G][M][N] of "
                         + " or ".join(str(t).replace("torch.", "") for t in dtypes))
    if not X.is_cuda:
        raise ValueError(f"{name} must be a CUDA (HIP) tensor")
    G, M, N = X.shape
    if not (G and M and N):
        raise ValueError(f"{name} is empty")
    sG, sM, sN = X.stride()
    if N > 1 and sN != 1:
        raise ValueError(f"{name}'s columns must be contiguous")
    return (sM if M > 1 else N), (sG if G > 1 else 0)


def _overlap(a: torch.Tensor, b: torch.Tensor) -> bool:
    """Whether two 3-D tensors of contiguous columns share a byte: by their spans where those
    are apart, and else (views into one buffer) by their rows."""
    def span(t):
        (G, M, N), (sG, sM, _), at = t.shape, t.stride(), t.data_ptr()
        return at, at + ((G - 1) * sG + (M - 1) * sM + N) * t.element_size()

    (a0, a1), (b0, b1) = span(a), span(b)
    if a1 <= b0 or b1 <= a0:
        return False

    def rows(t):  # where the runs without a gap start, sorted, and their length
        G, M, N = t.shape
        sG, sM, _ = t.stride()
        if sM == N:
            M, N = 1, M * N
        at = (torch.arange(G) * sG)[:, None] + torch.arange(M) * sM
        return (at.flatten() * t.element_size() + t.data_ptr()).sort()[0], N * t.element_size()

    (ra, na), (rb, nb) = rows(a), rows(b)
    # of a's runs that start before a run of b ends, the last one ends last
    before = torch.searchsorted(ra, rb + nb)
    return bool(((before > 0) & (ra[(before - 1).clamp_min(0)] + na > rb)).any())


def _apart(p: int, n: int, q: int, m: int) -> bool:
    """Whether the n bytes from p and the m bytes from q are apart: what nearly every call
    is told by, in a tenth of _overlap's time."""
    return p + n <= q or q + m <= p


def _same_device(*ts):
    if any(t.device != ts[0].device for t in ts[1:]):
        raise ValueError("all tensors must be on one device")


def _new_blocks(G: int, M: int, n: int, dtype, device) -> Blocks:
    return Blocks(torch.empty((G, M, _up(n, 128)), dtype=dtype, device=device),
                  torch.empty((G, M, _up((n + 127) // 128, 4)), dtype=torch.float8_e8m0fnu,
                              device=device), n)


def quantise_blocks(X: torch.Tensor, fmt: str = "e4m3", both: bool = False
                    ) -> Union[Blocks, Tuple[Blocks, Blocks]]:
    """X [G][M][N] (float32 or bfloat16, columns contiguous) in 8 bits with a
    power-of-two scale for each row and 128 columns (lsgd_quantise_blocks);
    ``both``: (X's blocks, its transpose's) from one read of X."""
    ldx, sX = _matrices("X", X, _FLOATS)
    if fmt not in FORMATS:
        raise ValueError("fmt must be 'e4m3' or 'e5m2'")
    code, dtype = FORMATS[fmt]
    G, M, N = X.shape
    q = _new_blocks(G, M, N, dtype, X.device)
    t = _new_blocks(G, N, M, dtype, X.device) if both else None
    _enqueue(X.device, _lib.lsgd_quantise_blocks,
             BF16 if X.dtype == torch.bfloat16 else FP32, code, G, M, N, X.data_ptr(), ldx, sX,
             q.q.data_ptr(), q.scale.data_ptr(), t.q.data_ptr() if both else None,
             t.scale.data_ptr() if both else None)
    return (q, t) if both else q


_CODES = {d: c for c, d in FORMATS.values()}


def _block_operand(name: str, X: Blocks) -> Tuple[int, int, int, int, int]:
    """Format code, groups, rows and the two group strides of an operand."""
    q, s, n = X
    shape, code = q.shape, _CODES.get(q.dtype)
    if len(shape) != 3 or code is None or s.dtype != torch.float8_e8m0fnu:
        raise ValueError(f"{name} must hold 3-D float8 values and float8_e8m0fnu scales")
    G, M, L = shape
    lds = _up((n + 127) // 128, 4)
    if n < 1 or L != _up(n, 128) or s.shape != (G, M, lds) or not (G and M):
        raise ValueError(f"{name}: shapes do not match the block layout of {n} columns")
    if not (q.is_cuda and s.is_cuda):
        raise ValueError(f"{name} must be on a CUDA (HIP) device")
    if q.is_contiguous() and s.is_contiguous():
        return code, G, M, M * L, M * lds
    for t in (q, s):
        if t.stride(2) != 1 or (M > 1 and t.stride(1) != t.shape[2]):
            raise ValueError(f"{name}: rows must be contiguous and unpadded")
    return code, G, M, (q.stride(0) if G > 1 else 0), (s.stride(0) if G > 1 else 0)


@functools.lru_cache(maxsize=4096)
def _gemm_blocks_workspace(out: int, G: int, M: int, N: int, n: int) -> int:
    nb = _c.c_size_t()
    _check(_lib.lsgd_grouped_gemm_blocks_workspace_bytes(out, G, M, N, n, _c.byref(nb)))
    return nb.value


def grouped_gemm_blocks(A: Blocks, B: Blocks, out: Optional[torch.Tensor] = None,
                        out_dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """C[g] = A[g] @ B[g]^T of two tensors in blocks along the contracted
    dimension (lsgd_grouped_gemm_blocks), C float32 (products in bf16, exact, summed
    in fp32) or bfloat16 (the 8-bit matrix instruction, twice as fast). y = x w takes
    x and w's transpose, dy w^T takes dy and w, and x^T dy the transposes of x and
    dy. A group stride of 0 (``expand``) shares a matrix among the groups. ``out``
    (whose type counts then, not ``out_dtype``) must not overlap A or B."""
    fa, G, M, sA, sSA = _block_operand("A", A)
    fb, Gb, N, sB, sSB = _block_operand("B", B)
    n, dev = A.n, A.q.device
    if n != B.n or G != Gb:
        raise ValueError("A and B must have the same groups and inner dimension")
    if out is None:
        if out_dtype not in _FLOATS:
            raise ValueError("out_dtype must be float32 or bfloat16")
        out = torch.empty((G, M, N), dtype=out_dtype, device=dev)
        ldc, sC = N, M * N
    else:
        ldc, sC = _matrices("out", out, _FLOATS)
        if out.shape != (G, M, N):
            raise ValueError("out must be [G][M][N]")
        p, size = out.data_ptr(), ((G - 1) * sC + (M - 1) * ldc + N) * out.element_size()
        L, lds = A.q.shape[2], A.scale.shape[2]
        if not (_apart(p, size, A.q.data_ptr(), (G - 1) * sA + M * L)
                and _apart(p, size, B.q.data_ptr(), (G - 1) * sB + N * L)
                and _apart(p, size, A.scale.data_ptr(), (G - 1) * sSA + M * lds)
                and _apart(p, size, B.scale.data_ptr(), (G - 1) * sSB + N * lds)) and any(
                    _overlap(out, t) for t in (A.q, A.scale, B.q, B.scale)):
            raise ValueError("out must not overlap A or B")
    if not (A.scale.device == dev and B.q.device == dev and B.scale.device == dev
            and out.device == dev):
        raise ValueError("all tensors must be on one device")
    dt = BF16 if out.dtype == torch.bfloat16 else FP32
    nb = _gemm_blocks_workspace(dt, G, M, N, n)
    ws = torch.empty(nb, dtype=torch.uint8, device=dev) if nb else None
    _enqueue(dev, _lib.lsgd_grouped_gemm_blocks,
             fa, fb, dt, G, M, N, n,
             A.q.data_ptr(), sA, A.scale.data_ptr(), sSA, B.q.data_ptr(), sB,
             B.scale.data_ptr(), sSB, out.data_ptr(), ldc, sC, ws.data_ptr() if nb else None, nb)
    return out


def orthogonalise_workspace(G: int, M: int, N: int, dtype: torch.dtype = torch.float32,
                            device="cuda") -> torch.Tensor:
    """A workspace for ``orthogonalise`` / ``orthogonal_update`` on [G][M][N]
    (``dtype``: the products' precision), for callers that keep one. One
    workspace serves one call at a time: calls on several streams take one each."""
    return _aligned_bytes(_ortho_workspace(_precision(dtype), G, M, N), device)


@functools.lru_cache(maxsize=4096)
def _ortho_workspace(dtype: int, G: int, M: int, N: int) -> int:
    nb = _c.c_size_t()
    _check(_lib.lsgd_orthogonalise_workspace_bytes(dtype, G, M, N, _c.byref(nb)))
    return nb.value


def _precision(dtype: torch.dtype) -> int:
    if dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("the precision must be float32 or bfloat16")
    return BF16 if dtype == torch.bfloat16 else FP32


def _coefficients(c: Sequence[float]):
    if len(c) != 3:
        raise ValueError("coefficients must be (a, b, c)")
    return (_c.c_float * 3)(*[float(v) for v in c])


def _workspace_for(ws, G, M, N, dtype, device) -> torch.Tensor:
    if ws is None:  # (the allocator's blocks start on 512-byte boundaries)
        return torch.empty(_ortho_workspace(_precision(dtype), G, M, N), dtype=torch.uint8,
                           device=device)
    if ws.dtype != torch.uint8 or not ws.is_contiguous() or ws.device != device:
        raise ValueError("workspace must be a contiguous uint8 tensor on the same device")
    return ws


def orthogonalise(X: torch.Tensor, steps: int = 5, coefficients: Sequence[float] = COEFFICIENTS,
                  eps: float = 1e-7, out: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The matrices X [G][M][N] (float32 or bfloat16) taken towards their
    orthogonal factors by Newton-Schulz steps (lsgd_orthogonalise); ``out`` may be
    X itself, and else must not overlap it. X's type is also the products' precision: in
    bfloat16, matrices of 385 rows and columns and more multiply operands of 11 bits and
    are off by 2.0e-3 to 2.3e-3 (rounding to bfloat16 alone by 1.7e-3); ``X.float()``
    keeps fp32 precision throughout."""
    ldx, sX = _matrices("X", X, _FLOATS)
    G, M, N = X.shape
    if out is None:
        out = torch.empty((G, M, N), dtype=X.dtype, device=X.device)
        ldy, sY = N, M * N
    else:
        ldy, sY = _matrices("out", out, (X.dtype,))
        if out.shape != X.shape:
            raise ValueError("out must have X's shape")
        _same_device(X, out)
        if (out.data_ptr(), ldy, sY) != (X.data_ptr(), ldx, sX) and _overlap(out, X):
            raise ValueError("out must be X itself or not overlap it")
    co = _coefficients(coefficients)
    ws = _workspace_for(workspace, G, M, N, X.dtype, X.device)
    _enqueue(X.device, _lib.lsgd_orthogonalise, _precision(X.dtype), G, M, N, X.data_ptr(), ldx,
             sX, out.data_ptr(), ldy, sY, int(steps), co, float(eps), ws.data_ptr(), ws.numel())
    return out


def orthogonal_update(W: torch.Tensor, U: torch.Tensor, G: torch.Tensor, lr: float,
                      momentum: float, weight_decay: float = 0.0, nesterov: bool = False,
                      scale: float = 1.0, steps: int = 5,
                      coefficients: Sequence[float] = COEFFICIENTS, eps: float = 1e-7,
                      gemm_dtype: torch.dtype = torch.float32,
                      workspace: Optional[torch.Tensor] = None) -> None:
    """In-place update of W [K][M][N] and its momentum U with gradient G (all
    float32, columns contiguous; views into the replicas' flat rows are fine):
    u = m u + g, d = g + m u (``nesterov``) or u, w = (1 - lr wd) w - lr scale O(d)
    with O of ``orthogonalise`` (lsgd_orthogonal_update), its products in the precision
    of ``gemm_dtype``. They must not overlap."""
    (ldw, sW), (ldu, sU), (ldg, sG) = (_matrices("W", W, _FP32), _matrices("U", U, _FP32),
                                       _matrices("G", G, _FP32))
    if U.shape != W.shape or G.shape != W.shape:
        raise ValueError("W, U, G must have one shape")
    _same_device(W, U, G)
    K, M, N = W.shape
    w, u, g = W.data_ptr(), U.data_ptr(), G.data_ptr()
    nw, nu, ng = (4 * ((K - 1) * s + (M - 1) * ld + N)
                  for ld, s in ((ldw, sW), (ldu, sU), (ldg, sG)))
    if not (_apart(w, nw, u, nu) and _apart(w, nw, g, ng) and _apart(u, nu, g, ng)) and (
            _overlap(W, U) or _overlap(W, G) or _overlap(U, G)):
        raise ValueError("W, U, G must not overlap")
    co = _coefficients(coefficients)
    ws = _workspace_for(workspace, K, M, N, gemm_dtype, W.device)
    _enqueue(W.device, _lib.lsgd_orthogonal_update, _precision(gemm_dtype), K, M, N,
             w, ldw, sW, u, ldu, sU, g, ldg, sG, float(lr),
             float(momentum), float(weight_decay), int(bool(nesterov)), float(scale), int(steps),
             co, float(eps), ws.data_ptr(), ws.numel())
