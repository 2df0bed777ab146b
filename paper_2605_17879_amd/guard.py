"""ctypes binding of the C ABI in ``include/guard.h`` -- argument marshalling only.

Every function of the header is reachable as ``Detector.<name without gd_>``
taking torch CUDA tensors; PyTorch supplies device memory and streams, nothing
else.  No step of the detector is computed here.
"""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass, field
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libguard_hip.so")
_lib = None

GD_OK = 0
_STATUS = {0: "GD_OK", 1: "GD_ERR_INVALID_ARG", 2: "GD_ERR_BAD_CONFIG",
           3: "GD_ERR_BUFFER_TOO_SMALL", 4: "GD_ERR_UNSUPPORTED", 5: "GD_ERR_HIP"}
NODE_SUM_SCALED = 0
NODE_MAX = 1

EXPORTS = ("gd_default_config", "gd_create", "gd_destroy", "gd_state_bytes", "gd_bind_state",
           "gd_set_streaming_steps", "gd_score_batch", "gd_update_window", "gd_flags",
           "gd_topk_nodes", "gd_severity", "gd_sweep_score", "gd_probe_read", "gd_last_error",
           "gd_default_ledger_config", "gd_ledger_bytes", "gd_bind_ledger", "gd_update_ledger",
           "gd_ledger_flags", "gd_topk_nodes_mean", "gd_set_streaming_hints", "gd_apply_membership",
           "gd_update_ledger_static", "gd_ledger_static_scratch_bytes",
           "gd_embed", "gd_embed_grad", "gd_embed_grad_work_bytes", "gd_vocab_loss", "gd_vocab_loss_grad",
           "gd_vocab_loss_work_bytes", "gd_adamw", "gd_adamw_table_bytes", "gd_adamw_fill_table")

F32, BF16, F16, I32, I64, E4M3 = range(6)      # gd_dtype
STATE_BLOCK = 256                              # GD_STATE_BLOCK


class GuardError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{_STATUS.get(status, status)}: {msg}")
        self.status = status


class _CConfig(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("n_ranks", ctypes.c_uint32),
                ("gpus_per_node", ctypes.c_uint32), ("n_metrics", ctypes.c_uint32),
                ("primary_metric", ctypes.c_uint32), ("min_signals", ctypes.c_uint32),
                ("window", ctypes.c_uint32), ("persist_k", ctypes.c_uint32),
                ("topk", ctypes.c_uint32), ("node_agg", ctypes.c_uint32),
                ("z_threshold", ctypes.c_float), ("node_scale", ctypes.c_float),
                ("rel_floor", ctypes.c_float), ("abs_floor", ctypes.c_float),
                ("direction", ctypes.c_int8 * 8)]


class _CLedgerConfig(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("score_quant", ctypes.c_float),
                ("recur_limit", ctypes.c_uint32), ("reserved", ctypes.c_uint32),
                ("recur_horizon", ctypes.c_uint64)]


class _CMatrix(ctypes.Structure):
    _fields_ = [("d_data", ctypes.c_void_p), ("rows", ctypes.c_uint64), ("cols", ctypes.c_uint64),
                ("stride", ctypes.c_uint64), ("dtype", ctypes.c_uint32), ("reserved", ctypes.c_uint32)]


class _CAdamwTensor(ctypes.Structure):
    _fields_ = [("d_param", ctypes.c_void_p), ("d_grad", ctypes.c_void_p), ("d_m", ctypes.c_void_p),
                ("d_v", ctypes.c_void_p), ("d_m_exp", ctypes.c_void_p), ("d_v_exp", ctypes.c_void_p),
                ("d_copy", ctypes.c_void_p), ("n", ctypes.c_uint64), ("first_index", ctypes.c_uint64),
                ("lr_scale", ctypes.c_double), ("weight_decay", ctypes.c_double),
                ("param_type", ctypes.c_uint32), ("grad_type", ctypes.c_uint32),
                ("copy_type", ctypes.c_uint32), ("state_type", ctypes.c_uint32)]


class _CAdamwConfig(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("seed", ctypes.c_uint32), ("lr", ctypes.c_double),
                ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("step", ctypes.c_uint64)]


def library_path() -> str:
    return _LIB_PATH


def load_library() -> ctypes.CDLL:
    """Load libguard_hip.so; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2605_17879_amd.build` "
            "(or __graft_entry__.build()); there is no CPU fallback")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, u32, u64 = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64
    lib.gd_default_config.argtypes = [ctypes.POINTER(_CConfig), u32, u32, u32, u32]
    lib.gd_default_config.restype = None
    lib.gd_create.argtypes = [ctypes.POINTER(_CConfig), ctypes.POINTER(vp)]
    lib.gd_create.restype = ctypes.c_int
    lib.gd_destroy.argtypes = [vp]
    lib.gd_destroy.restype = ctypes.c_int
    lib.gd_state_bytes.argtypes = [vp]
    lib.gd_state_bytes.restype = ctypes.c_size_t
    lib.gd_bind_state.argtypes = [vp, vp, ctypes.c_size_t]
    lib.gd_bind_state.restype = ctypes.c_int
    lib.gd_set_streaming_steps.argtypes = [vp, u32]
    lib.gd_set_streaming_steps.restype = ctypes.c_int
    lib.gd_set_streaming_hints.argtypes = [vp, vp, vp]
    lib.gd_set_streaming_hints.restype = ctypes.c_int
    lib.gd_score_batch.argtypes = [vp, vp, u32] + [vp] * 9
    lib.gd_score_batch.restype = ctypes.c_int
    lib.gd_update_window.argtypes = [vp, vp, vp, vp, u32, u64, vp]
    lib.gd_update_window.restype = ctypes.c_int
    lib.gd_flags.argtypes = [vp] * 8
    lib.gd_flags.restype = ctypes.c_int
    lib.gd_topk_nodes.argtypes = [vp, u32, vp, vp, vp]
    lib.gd_topk_nodes.restype = ctypes.c_int
    lib.gd_severity.argtypes = [vp, vp, u32, vp, ctypes.c_float, ctypes.c_float, vp, vp, vp]
    lib.gd_severity.restype = ctypes.c_int
    f32 = ctypes.c_float
    lib.gd_sweep_score.argtypes = [vp, vp, vp, u32, f32, f32, f32, vp, vp, vp, vp, vp]
    lib.gd_sweep_score.restype = ctypes.c_int
    lib.gd_probe_read.argtypes = [vp, vp, u64, vp, vp]
    lib.gd_probe_read.restype = ctypes.c_int
    lib.gd_default_ledger_config.argtypes = [ctypes.POINTER(_CLedgerConfig)]
    lib.gd_default_ledger_config.restype = None
    lib.gd_ledger_bytes.argtypes = [vp, u32]
    lib.gd_ledger_bytes.restype = ctypes.c_size_t
    lib.gd_bind_ledger.argtypes = [vp, ctypes.POINTER(_CLedgerConfig), vp, ctypes.c_size_t, u32]
    lib.gd_bind_ledger.restype = ctypes.c_int
    lib.gd_update_ledger.argtypes = [vp, vp, vp, vp, u32, u64, vp]
    lib.gd_update_ledger.restype = ctypes.c_int
    lib.gd_update_ledger_static.argtypes = [vp, vp, vp, vp, u32, u64, vp]
    lib.gd_update_ledger_static.restype = ctypes.c_int
    lib.gd_ledger_static_scratch_bytes.argtypes = []
    lib.gd_ledger_static_scratch_bytes.restype = ctypes.c_size_t
    lib.gd_ledger_flags.argtypes = [vp] * 11
    lib.gd_ledger_flags.restype = ctypes.c_int
    lib.gd_topk_nodes_mean.argtypes = [vp, u32, vp, vp, vp]
    lib.gd_topk_nodes_mean.restype = ctypes.c_int
    lib.gd_apply_membership.argtypes = [vp, vp, u32, vp, vp]
    lib.gd_apply_membership.restype = ctypes.c_int
    mat, sz, i32 = ctypes.POINTER(_CMatrix), ctypes.c_size_t, ctypes.c_int32
    lib.gd_embed.argtypes = [vp, mat, mat, f32, mat, vp]
    lib.gd_embed.restype = ctypes.c_int
    lib.gd_embed_grad_work_bytes.argtypes = [u64, u64, u64]
    lib.gd_embed_grad_work_bytes.restype = sz
    lib.gd_embed_grad.argtypes = [vp, mat, mat, f32, i32, mat, vp, sz, vp]
    lib.gd_embed_grad.restype = ctypes.c_int
    lib.gd_vocab_loss_work_bytes.argtypes = [u64, u64, u64, i32]
    lib.gd_vocab_loss_work_bytes.restype = sz
    lib.gd_vocab_loss.argtypes = [vp, mat, mat, mat, f32, vp, vp, vp, vp, sz, vp]
    lib.gd_vocab_loss.restype = ctypes.c_int
    lib.gd_vocab_loss_grad.argtypes = [vp, mat, mat, mat, f32, vp, vp, vp, vp, mat, mat, vp, sz, vp]
    lib.gd_vocab_loss_grad.restype = ctypes.c_int
    lib.gd_adamw_table_bytes.argtypes = [vp, ctypes.POINTER(_CAdamwTensor), u32]
    lib.gd_adamw_table_bytes.restype = sz
    lib.gd_adamw_fill_table.argtypes = [vp, ctypes.POINTER(_CAdamwTensor), u32, vp, sz]
    lib.gd_adamw_fill_table.restype = ctypes.c_int
    lib.gd_adamw.argtypes = [vp, vp, sz, ctypes.POINTER(_CAdamwConfig), vp, vp]
    lib.gd_adamw.restype = ctypes.c_int
    lib.gd_last_error.argtypes = [vp]
    lib.gd_last_error.restype = ctypes.c_char_p
    _lib = lib
    return lib


@dataclass
class Config:
    """Mirror of ``gd_config``; ``None`` fields take the library's defaults."""

    n_ranks: int
    n_metrics: int
    window: int
    persist_k: int
    gpus_per_node: int = 8
    primary_metric: int = 0
    min_signals: Optional[int] = None
    topk: Optional[int] = None
    node_agg: int = NODE_SUM_SCALED
    z_threshold: Optional[float] = None
    node_scale: Optional[float] = None
    rel_floor: Optional[float] = None
    abs_floor: Optional[float] = None
    direction: Sequence[int] = field(default_factory=tuple)

    def to_c(self) -> _CConfig:
        c = _CConfig()
        load_library().gd_default_config(ctypes.byref(c), self.n_ranks, self.n_metrics,
                                         self.window, self.persist_k)
        c.gpus_per_node = self.gpus_per_node
        c.primary_metric = self.primary_metric
        c.node_agg = self.node_agg
        for name in ("min_signals", "topk", "z_threshold", "node_scale", "rel_floor", "abs_floor"):
            v = getattr(self, name)
            if v is not None:
                setattr(c, name, v)
        for i, d in enumerate(self.direction):
            c.direction[i] = int(d)
        return c


_PACK_MATRIX = struct.Struct("=QQQQII").pack            # gd_matrix
_PACK_ADAMW = struct.Struct("=IIddddQ").pack            # gd_adamw_config
_ADAMW_BYTES = ctypes.sizeof(_CAdamwConfig)


def _p(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


class Detector:
    """One ``gd_handle`` plus its (torch-allocated) window state."""

    def __init__(self, cfg: Config, device="cuda:0"):
        import torch
        self._torch = torch
        self.lib = load_library()
        self.cfg = cfg
        self.ccfg = cfg.to_c()
        h = ctypes.c_void_p()
        st = self.lib.gd_create(ctypes.byref(self.ccfg), ctypes.byref(h))
        if st != GD_OK:
            raise GuardError(st, (self.lib.gd_last_error(None) or b"").decode())
        self.h = h
        self.device = torch.device(device)
        self._raw_stream = torch._C._cuda_getCurrentRawStream
        self._index = self.device.index
        self._f32 = torch.float32
        # the operators' entry points as their methods call them: structures come as packed bytes
        vp, f32, sz = ctypes.c_void_p, ctypes.c_float, ctypes.c_size_t
        self._embed = self._entry("gd_embed", vp, vp, vp, f32, vp, vp)
        self._embed_grad = self._entry("gd_embed_grad", vp, vp, vp, f32, ctypes.c_int32, vp, vp, sz, vp)
        self._vocab_loss = self._entry("gd_vocab_loss", vp, vp, vp, vp, f32, vp, vp, vp, vp, sz, vp)
        self._vocab_loss_grad = self._entry("gd_vocab_loss_grad", vp, vp, vp, vp, f32, *[vp] * 7, sz, vp)
        self._adamw = self._entry("gd_adamw", vp, vp, sz, vp, vp, vp)
        self._types = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16, torch.int32: I32, torch.int64: I64}
        self.R, self.M = cfg.n_ranks, cfg.n_metrics
        self.N = self.R // cfg.gpus_per_node
        self.RW, self.NW = (self.R + 63) // 64, (self.N + 63) // 64
        self.state = torch.zeros(self.state_bytes(), dtype=torch.uint8, device=self.device)
        self.bind_state(self.state)
        self.steps_seen = 0

    def close(self):
        if getattr(self, "h", None):
            self.lib.gd_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _entry(self, name: str, *types):
        f = self.lib[name]                              # (a function object of its own)
        f.argtypes, f.restype = types, ctypes.c_int
        return f

    def _check(self, st: int):
        if st != GD_OK:
            raise GuardError(st, (self.lib.gd_last_error(self.h) or b"").decode())

    def _stream(self, stream) -> int:
        if stream is not None:
            return stream.cuda_stream
        # The current stream's handle alone: building the Stream object around it took longer
        # than the rest of a call's marshalling, and a small job's calls are bound by that.
        index = self.device.index
        return self._raw_stream(self._torch.cuda.current_device() if index is None else index)

    # ---- the C ABI, one method per entry point --------------------------------
    def state_bytes(self) -> int:
        return int(self.lib.gd_state_bytes(self.h))

    def bind_state(self, state):
        self._check(self.lib.gd_bind_state(self.h, state.data_ptr(), state.numel() * state.element_size()))
        self.state = state

    def set_streaming_steps(self, max_steps: int):
        """Batches of at most max_steps steps are scored one workgroup per column (0: never)."""
        self._check(self.lib.gd_set_streaming_steps(self.h, max_steps))

    def set_streaming_hints(self, med=None, mad=None):
        """One-step calls start their selection from these [M] medians and MADs (device
        tensors, typically the previous call's outputs; kept alive here)."""
        self._hints = (med, mad)
        self._check(self.lib.gd_set_streaming_hints(self.h, _p(med), _p(mad)))

    def apply_membership(self, x, active, stream=None):
        """NaN (missing) in place wherever active[T][ceil(R/64)] (int64 bit words) has a clear bit."""
        T = x.shape[0]
        assert x.is_cuda and x.is_contiguous() and tuple(x.shape) == (T, self.M, self.R)
        assert active.is_cuda and active.is_contiguous() and tuple(active.shape) == (T, self.RW)
        self._check(self.lib.gd_apply_membership(self.h, x.data_ptr(), T, active.data_ptr(), self._stream(stream)))

    def alloc_outputs(self, T: int, want_z: bool = False) -> dict:
        """Output tensors of gd_score_batch for T steps (plain allocation)."""
        torch, d = self._torch, self.device
        o = dict(
            med=torch.empty((T, self.M), dtype=torch.float32, device=d),
            mad=torch.empty((T, self.M), dtype=torch.float32, device=d),
            z=torch.empty((T, self.M, self.R), dtype=torch.float32, device=d) if want_z else None,
            exceed_mask=torch.empty((T, self.R), dtype=torch.uint8, device=d),
            rank_anom=torch.empty((T, self.RW), dtype=torch.int64, device=d),
            node_z=torch.empty((T, self.N), dtype=torch.float32, device=d),
            node_mask=torch.empty((T, self.N), dtype=torch.uint8, device=d),
            node_anom=torch.empty((T, self.NW), dtype=torch.int64, device=d))
        return o

    def score_batch(self, x, out: dict, stream=None):
        T = x.shape[0]
        assert x.is_cuda and x.is_contiguous() and x.dtype == self._torch.float32
        assert tuple(x.shape) == (T, self.M, self.R)
        self._check(self.lib.gd_score_batch(
            self.h, x.data_ptr(), T, _p(out["med"]), _p(out["mad"]), _p(out.get("z")),
            _p(out["exceed_mask"]), _p(out["rank_anom"]), _p(out["node_z"]), _p(out["node_mask"]),
            _p(out["node_anom"]), self._stream(stream)))

    def update_window(self, out: dict, T: int, first_step_index: Optional[int] = None, stream=None):
        first = self.steps_seen if first_step_index is None else first_step_index
        self._check(self.lib.gd_update_window(self.h, _p(out["rank_anom"]), _p(out["node_anom"]),
                                              _p(out["node_z"]), T, first, self._stream(stream)))
        self.steps_seen = first + T

    def alloc_flags(self) -> dict:
        torch, d = self._torch, self.device
        return dict(rank_flag=torch.empty(self.R, dtype=torch.uint8, device=d),
                    rank_count=torch.empty(self.R, dtype=torch.int16, device=d),
                    rank_first=torch.empty(self.R, dtype=torch.int32, device=d),
                    node_flag=torch.empty(self.N, dtype=torch.uint8, device=d),
                    node_count=torch.empty(self.N, dtype=torch.int16, device=d),
                    node_first=torch.empty(self.N, dtype=torch.int32, device=d))

    def flags(self, f: dict, stream=None):
        self._check(self.lib.gd_flags(self.h, _p(f.get("rank_flag")), _p(f.get("rank_count")),
                                      _p(f.get("rank_first")), _p(f.get("node_flag")),
                                      _p(f.get("node_count")), _p(f.get("node_first")),
                                      self._stream(stream)))

    def alloc_severity(self) -> dict:
        torch, d = self._torch, self.device
        return dict(slowdown=torch.empty(self.N, dtype=torch.float32, device=d),
                    tier=torch.empty(self.N, dtype=torch.uint8, device=d))

    def severity(self, x, out: dict, sev: dict, moderate: float = 0.10, severe: float = 0.20,
                 stream=None):
        """Tiers of the flagged nodes from the batch x that `out` was scored from."""
        T = x.shape[0]
        assert x.is_cuda and x.is_contiguous() and tuple(x.shape) == (T, self.M, self.R)
        self._check(self.lib.gd_severity(self.h, x.data_ptr(), T, _p(out["med"]), moderate, severe,
                                         _p(sev["slowdown"]), _p(sev["tier"]), self._stream(stream)))

    def sweep_score(self, flops, bw, tol_compute: float = 0.05, tol_sym: float = 0.10,
                    tol_bw: float = 0.15, stream=None) -> dict:
        """Single-node sweep scoring of flops[B][8], bw[B][8][8] (device tensors)."""
        torch, d = self._torch, self.device
        B = flops.shape[0]
        assert flops.is_cuda and flops.is_contiguous() and tuple(flops.shape) == (B, 8)
        assert bw.is_cuda and bw.is_contiguous() and tuple(bw.shape) == (B, 8, 8)
        out = dict(shortfall=torch.empty((B, 8), dtype=torch.float32, device=d),
                   gpu_mask=torch.empty(B, dtype=torch.uint8, device=d),
                   link_mask=torch.empty(B, dtype=torch.int32, device=d),
                   verdict=torch.empty(B, dtype=torch.uint8, device=d))
        self._check(self.lib.gd_sweep_score(self.h, flops.data_ptr(), bw.data_ptr(), B, tol_compute,
                                            tol_sym, tol_bw, _p(out["shortfall"]), _p(out["gpu_mask"]),
                                            _p(out["link_mask"]), _p(out["verdict"]),
                                            self._stream(stream)))
        return out

    def probe_read(self, x, sink, stream=None):
        """Stream x through the chip with the scoring kernel's load pattern (a diagnostic)."""
        self._check(self.lib.gd_probe_read(self.h, x.data_ptr(), x.numel() * x.element_size(),
                                           sink.data_ptr(), self._stream(stream)))

    def alloc_topk(self, k: int) -> dict:
        torch, d = self._torch, self.device
        return dict(idx=torch.empty(k, dtype=torch.int32, device=d),
                    key=torch.empty(k, dtype=torch.int64, device=d))

    def topk_nodes(self, k: int, tk: dict, stream=None):
        self._check(self.lib.gd_topk_nodes(self.h, k, _p(tk["idx"]), _p(tk.get("key")),
                                           self._stream(stream)))

    # ---- the ledger ---------------------------------------------------------------
    def ledger_bytes(self, max_T: int) -> int:
        return int(self.lib.gd_ledger_bytes(self.h, max_T))

    def bind_ledger(self, ledger, max_T: int, score_quant: Optional[float] = None,
                    recur_limit: Optional[int] = None, recur_horizon: Optional[int] = None):
        c = _CLedgerConfig()
        self.lib.gd_default_ledger_config(ctypes.byref(c))
        if score_quant is not None:
            c.score_quant = score_quant
        if recur_limit is not None:
            c.recur_limit = recur_limit
        if recur_horizon is not None:
            c.recur_horizon = recur_horizon
        self._check(self.lib.gd_bind_ledger(self.h, ctypes.byref(c), ledger.data_ptr(),
                                            ledger.numel() * ledger.element_size(), max_T))
        self.ledger = ledger
        self.ledger_steps_seen = 0

    def alloc_ledger(self, max_T: int, **cfg):
        """A fresh (zeroed) ledger for batches of up to max_T steps, bound to the handle."""
        led = self._torch.zeros(self.ledger_bytes(max_T), dtype=self._torch.uint8, device=self.device)
        self.bind_ledger(led, max_T, **cfg)
        return led

    def update_ledger(self, out: dict, T: int, first_step_index: Optional[int] = None, stream=None):
        first = self.ledger_steps_seen if first_step_index is None else first_step_index
        self._check(self.lib.gd_update_ledger(self.h, _p(out["exceed_mask"]), _p(out["node_mask"]),
                                              _p(out["node_z"]), T, first, self._stream(stream)))
        self.ledger_steps_seen = first + T

    def update_ledger_static(self, out: dict, T: int, first_step_index: Optional[int] = None, stream=None):
        """gd_update_ledger with the library's static work area (the call allocates nothing)."""
        first = self.ledger_steps_seen if first_step_index is None else first_step_index
        self._check(self.lib.gd_update_ledger_static(self.h, _p(out["exceed_mask"]), _p(out["node_mask"]),
                                                     _p(out["node_z"]), T, first, self._stream(stream)))
        self.ledger_steps_seen = first + T

    def ledger_static_scratch_bytes(self) -> int:
        return int(self.lib.gd_ledger_static_scratch_bytes())

    def alloc_ledger_flags(self) -> dict:
        torch, d = self._torch, self.device
        e = lambda n, t: torch.empty(n, dtype=t, device=d)
        return dict(rank_pmask=e(self.R, torch.uint8), rank_pflag=e(self.R, torch.uint8),
                    rank_pfirst=e(self.R, torch.int32), node_pmask=e(self.N, torch.uint8),
                    node_pflag=e(self.N, torch.uint8), node_pfirst=e(self.N, torch.int32),
                    node_score_sum=e(self.N, torch.int32), node_episodes=e(self.N, torch.uint8),
                    node_terminal_first=e(self.N, torch.int32))

    def ledger_flags(self, f: dict, stream=None):
        self._check(self.lib.gd_ledger_flags(
            self.h, _p(f.get("rank_pmask")), _p(f.get("rank_pflag")), _p(f.get("rank_pfirst")),
            _p(f.get("node_pmask")), _p(f.get("node_pflag")), _p(f.get("node_pfirst")),
            _p(f.get("node_score_sum")), _p(f.get("node_episodes")),
            _p(f.get("node_terminal_first")), self._stream(stream)))

    def topk_nodes_mean(self, k: int, tk: dict, stream=None):
        self._check(self.lib.gd_topk_nodes_mean(self.h, k, _p(tk["idx"]), _p(tk.get("key")),
                                                self._stream(stream)))

    # ---- the operators of a sweep's own training step ---------------------------------
    def _type(self, t) -> int:
        code = self._types.get(t.dtype)
        if code is None:
            raise GuardError(4, f"tensors of {t.dtype} are not built")
        return code

    def _at(self, t) -> int:
        """The address of a tensor on the detector's device."""
        at = t.get_device()
        if at != self._index and (self._index is not None or at < 0):
            raise AssertionError(f"a tensor is on {t.device}, the detector on {self.device}")
        return t.data_ptr()

    def _matrix(self, t) -> bytes:
        """t[rows][cols], rows any distance apart, as a gd_matrix; a list t[n] is a matrix of one column."""
        # (a short call's time is its marshalling: a packed gd_matrix takes a third of a ctypes structure's time)
        shape, strides = t.shape, t.stride()
        if len(shape) == 2:
            rows, cols = shape
            assert cols <= 1 or strides[1] == 1, "the elements of a row must be next to each other"
        else:
            assert len(shape) == 1, "a matrix or a list"
            rows, cols = shape[0], 1
        code = self._types.get(t.dtype)
        if code is None:
            raise GuardError(4, f"tensors of {t.dtype} are not built")
        # the distance to a row that is not there says nothing
        return _PACK_MATRIX(self._at(t), rows, cols, strides[0] if rows > 1 else cols or 1, code, 0)

    def _vector(self, t, n: int):
        """The address of n f32 values next to each other, or None."""
        if t is None:
            return None
        assert t.dtype is self._f32 and t.numel() == n and t.is_contiguous()
        return self._at(t)

    def _bytes(self, n: int):
        return self._torch.empty(n, dtype=self._torch.uint8, device=self.device)

    def embed(self, weight, tokens, out, scale: float = 1.0, stream=None):
        """out[i] = scale * weight[tokens[i]]; zeros for a negative token."""
        m = self._matrix
        self._check(self._embed(self.h, m(weight), m(tokens), scale, m(out), self._stream(stream)))

    def embed_grad_work_bytes(self, n: int, vocab: int, width: int) -> int:
        return int(self.lib.gd_embed_grad_work_bytes(n, vocab, width))

    def alloc_embed_grad_work(self, n: int, vocab: int, width: int):
        return self._bytes(self.embed_grad_work_bytes(n, vocab, width))

    def embed_grad(self, out_grad, tokens, weight_grad, work, scale: float = 1.0, accumulate: bool = False,
                   stream=None):
        """weight_grad[v] = (its old value, with accumulate) + scale * sum of out_grad[i] over tokens[i] == v."""
        m = self._matrix
        self._check(self._embed_grad(self.h, m(out_grad), m(tokens), scale, accumulate, m(weight_grad),
                                     self._at(work), work.nbytes, self._stream(stream)))

    def alloc_vocab_loss(self, n: int) -> dict:
        """Outputs of vocab_loss: loss[n], lse[n] and mean[2] (the mean and the rows in it)."""
        e = lambda k: self._torch.empty(k, dtype=self._torch.float32, device=self.device)
        return dict(loss=e(n), lse=e(n), mean=e(2))

    def vocab_loss_work_bytes(self, n: int, vocab: int, width: int, grad: bool = False) -> int:
        return int(self.lib.gd_vocab_loss_work_bytes(n, vocab, width, int(grad)))

    def alloc_vocab_loss_work(self, n: int, vocab: int, width: int, grad: bool = False):
        """A work area for vocab_loss and, with grad, for vocab_loss_grad too."""
        return self._bytes(self.vocab_loss_work_bytes(n, vocab, width, grad))

    def vocab_loss(self, hidden, weight, targets, out: dict, work, logit_scale: float = 1.0, stream=None):
        """Cross entropy of softmax(logit_scale * hidden weight^T) against targets (negative: left out)."""
        m, v, n = self._matrix, self._vector, targets.shape[0]
        self._check(self._vocab_loss(
            self.h, m(hidden), m(weight), m(targets), logit_scale, v(out["loss"], n), v(out["lse"], n), v(out["mean"], 2),
            self._at(work), work.nbytes, self._stream(stream)))

    def vocab_loss_grad(self, hidden, weight, targets, out: dict, grad: dict, work, grad_mean=None, grad_rows=None,
                        logit_scale: float = 1.0, stream=None):
        """Gradients grad["hidden"] and grad["weight"] (either may be missing) of
        sum(grad_rows * loss) + grad_mean * mean, behind vocab_loss on the same inputs."""
        m, v, n = self._matrix, self._vector, targets.shape[0]
        gh, gw = grad.get("hidden"), grad.get("weight")
        self._check(self._vocab_loss_grad(
            self.h, m(hidden), m(weight), m(targets), logit_scale, v(out["lse"], n), v(out["mean"], 2), v(grad_mean, 1),
            v(grad_rows, n), None if gh is None else m(gh), None if gw is None else m(gw), self._at(work), work.nbytes,
            self._stream(stream)))

    def alloc_adamw_state(self, params, bits: int = 32) -> dict:
        """Fresh moments for a list of tensors: fp32, or 8-bit codes m, v with their m_exp, v_exp."""
        assert bits in (32, 8)
        z = lambda n, t: self._torch.zeros(n, dtype=t, device=self.device)
        kind = self._torch.float32 if bits == 32 else self._torch.uint8
        state = {k: [z(p.numel(), kind) for p in params] for k in ("m", "v")}
        if bits == 8:
            for k in ("m_exp", "v_exp"):
                state[k] = [z(-(-p.numel() // STATE_BLOCK), self._torch.uint8) for p in params]
        return state

    def adamw_table(self, params, grads, state: dict, copies=None, weight_decay=0.0, lr_scale=1.0, first_index=0):
        """What adamw needs to know about its tensors (lists of the same length; weight_decay,
        lr_scale and first_index are lists too, or one value for all).  It holds addresses, and keeps
        the memory there alive.  A tensor that has moved (gradients that are freed and made anew each
        step, storage that is exchanged) needs a new table: an update by the old one reads and writes
        the old memory, and nothing says so.  Making one takes the host 3 us a tensor and copies it
        to the device (160 tensors: 0.5 ms)."""
        torch, n = self._torch, len(params)
        each = lambda v: list(v) if isinstance(v, (list, tuple)) else [v] * n
        eight = "m_exp" in state
        lists = [params, grads, state["m"], state["v"], copies if copies is not None else [None] * n,
                 each(weight_decay), each(lr_scale), each(first_index),
                 state["m_exp"] if eight else [None] * n, state["v_exp"] if eight else [None] * n]
        assert all(len(l) == n for l in lists)
        rows = (_CAdamwTensor * max(n, 1))()
        for row, p, g, m, v, c, decay, rate, first, me, ve in zip(rows, *lists):
            k = p.numel()
            for x in (p, g, m, v, c, me, ve):
                if x is not None:
                    self._at(x)
            assert all(t is None or (t.is_contiguous() and t.numel() == k) for t in (p, g, m, v, c))
            assert all(t is None or (t.is_contiguous() and t.dtype == torch.uint8 and
                                     t.numel() == -(-k // STATE_BLOCK)) for t in (me, ve))
            assert all(t.dtype == (torch.uint8 if eight else torch.float32) for t in (m, v))
            row.d_param, row.d_grad, row.d_m, row.d_v = _p(p), _p(g), _p(m), _p(v)
            row.d_m_exp, row.d_v_exp, row.d_copy = _p(me), _p(ve), _p(c)
            row.n, row.first_index, row.lr_scale, row.weight_decay = k, first, rate, decay
            row.param_type, row.grad_type = self._type(p), self._type(g)
            row.copy_type = BF16 if c is None else self._type(c)
            row.state_type = E4M3 if eight else F32
        size = int(self.lib.gd_adamw_table_bytes(self.h, rows, n))
        if size == 0:
            raise GuardError(1, (self.lib.gd_last_error(self.h) or b"").decode())
        host = torch.empty(size, dtype=torch.uint8)
        self._check(self.lib.gd_adamw_fill_table(self.h, rows, n, host.data_ptr(), size))
        # (a tensor whose storage is exchanged lets the old one go: the storages themselves are kept)
        kept = [t.untyped_storage() for l in (*lists[:5], *lists[8:]) for t in l if t is not None]
        return dict(bytes=host.to(self.device), tensors=lists, storages=kept)

    def adamw(self, table: dict, lr: float, step: int, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
              grad_scale=None, seed: Optional[int] = None, stream=None):
        """One update (step counts from 1) of every tensor of the table, in place.  grad_scale: a
        device scalar that multiplies the gradients; where it is not finite nothing is written.
        seed: of the 8-bit states' rounding, the step unless it is given."""
        # (a step below 1 is refused as 0)
        c = _PACK_ADAMW(_ADAMW_BYTES, (step if seed is None else seed) & 0xFFFFFFFF, lr, beta1, beta2, eps, max(step, 0))
        b = table["bytes"]
        self._check(self._adamw(self.h, b.data_ptr(), b.nbytes, c, self._vector(grad_scale, 1), self._stream(stream)))
