"""ctypes binding of libgrouter.so (the C ABI in include/grouter.h).

Argument marshalling only: every step of the layer runs in the CUDA library.
torch is used for device memory and streams.  There is no fallback: if the
library cannot be loaded this module raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import threading
from typing import Optional

import torch

from . import build as _build

IDX_U8, IDX_I32 = 0, 1
FLAG_ACCUMULATE_DW = 1
FLAG_FUSED_COMBINE = 2
NORM_SOFTMAX, NORM_SIGMOID = 0, 1
GATE_BF16, GATE_F32 = 0, 1
BF16, F32 = 0, 1
ACT_NONE, ACT_RELU, ACT_SILU, ACT_GELU = 0, 1, 2, 3

EXPORTS = ["grouter_create", "grouter_destroy", "grouter_workspace_bytes", "grouter_host_staging_bytes", "grouter_plan",
           "grouter_moe_fwd", "grouter_moe_bwd", "grouter_moe_step_host", "grouter_status", "grouter_strerror",
           "grouter_dense_gemm", "grouter_timing_enable", "grouter_timing_read", "grouter_plan_noalloc", "grouter_host_wait", "grouter_route", "grouter_route_workspace_bytes", "grouter_routing_stats",
           "grouter_fold_greedy_host", "grouter_timing_gap", "grouter_wgrad_chunk_rows", "grouter_gemm_cycles_enable", "grouter_gemm_cycles_read", "grouter_set_wait_limit", "grouter_wait_selftest", "grouter_set_overlap", "grouter_set_active_tokens",
           "grouter_checked_build",
           "grouter_ep_relabel_host", "grouter_ep_layout_host", "grouter_ep_expand_ids", "grouter_ep_dispatch_rows", "grouter_ep_combine_rows",
           "grouter_layernorm_fwd", "grouter_layernorm_bwd", "grouter_layernorm_bwd_workspace_bytes",
           "grouter_linear_fwd", "grouter_linear_bwd", "grouter_linear_bwd_workspace_bytes",
           "grouter_expert_counts", "grouter_balance_loss", "grouter_balance_loss_workspace_bytes",
           "grouter_adamw_layout_host", "grouter_adamw_step", "grouter_adamw_moments"]
KERNEL_SLOTS = ["plan_hist", "plan_permute", "gather_X", "gemm_up_swiglu", "gemm_down", "combine_Y", "gather_dY", "gemm_dH",
                "wgrad_down", "gemm_dX", "wgrad_gate_up", "reduce_dX", "zero_split_dW", "plan_scan"]


class GrouterDims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("T", "d", "ffn", "E_src", "E_tgt", "k", "idx_dtype", "gate_dtype", "flags")]


class AdamwTensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("n", ctypes.c_int64), ("weight_decay", ctypes.c_double),
                ("param_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32)]


class AdamwLayout(ctypes.Structure):
    _fields_ = [("state_elements", ctypes.c_int64), ("table_bytes", ctypes.c_uint64), ("n_tensors", ctypes.c_int32), ("n_chunks", ctypes.c_int32),
                ("needs_master", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class GrouterError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {strerror(code)} ({code})")
        self.code = code


_lib = None


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Loads (building in-tree first if stale or absent) and types the library."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    if path is None:
        path = _build.LIB
        try:
            _build.build(force=bool(os.environ.get("GROUTER_REBUILD")))     # returns at once when the library is newer than every source
        except (OSError, RuntimeError) as err:
            # no compiler here (or the build failed): an existing library is used, loudly; without one there is nothing to fall back to
            if not os.path.exists(path):
                raise
            import sys
            sys.stderr.write(f"paper_2603_06626_b200: could not rebuild libgrouter.so ({err}); loading the existing, possibly stale, library\n")
    lib = ctypes.CDLL(path)
    vp, i32p, f32p = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p
    lib.grouter_create.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.POINTER(GrouterDims)]
    lib.grouter_create.restype = ctypes.c_int
    lib.grouter_destroy.argtypes = [vp]
    lib.grouter_destroy.restype = None
    lib.grouter_workspace_bytes.argtypes = [ctypes.POINTER(GrouterDims)]
    lib.grouter_workspace_bytes.restype = ctypes.c_size_t
    lib.grouter_host_staging_bytes.argtypes = [ctypes.POINTER(GrouterDims)]
    lib.grouter_host_staging_bytes.restype = ctypes.c_size_t
    lib.grouter_plan.argtypes = [vp, vp, i32p, i32p, i32p, i32p, i32p, vp]
    lib.grouter_plan.restype = ctypes.c_int
    lib.grouter_plan_noalloc.argtypes = [vp, ctypes.c_int32, i32p] + [ctypes.c_int32] * 4 + [i32p] * 5 + [vp]
    lib.grouter_plan_noalloc.restype = ctypes.c_int
    lib.grouter_moe_fwd.argtypes = [vp] * 8
    lib.grouter_moe_fwd.restype = ctypes.c_int
    lib.grouter_moe_bwd.argtypes = [vp] * 12
    lib.grouter_moe_bwd.restype = ctypes.c_int
    lib.grouter_moe_step_host.argtypes = [vp] * 15
    lib.grouter_moe_step_host.restype = ctypes.c_int
    lib.grouter_route_workspace_bytes.argtypes = [ctypes.c_int32] * 3
    lib.grouter_route_workspace_bytes.restype = ctypes.c_size_t
    lib.grouter_route.argtypes = [vp, vp, i32p] + [ctypes.c_int32] * 6 + [vp, vp, f32p, vp, i32p, vp]
    lib.grouter_route.restype = ctypes.c_int
    lib.grouter_routing_stats.argtypes = [vp] + [ctypes.c_int32] * 5 + [i32p, ctypes.c_int32, i32p, i32p, f32p, f32p, i32p, i32p, i32p, vp]
    lib.grouter_routing_stats.restype = ctypes.c_int
    lib.grouter_fold_greedy_host.argtypes = [vp, ctypes.c_int32, ctypes.c_int32, vp]
    lib.grouter_fold_greedy_host.restype = ctypes.c_int
    lib.grouter_host_wait.argtypes = [vp, ctypes.c_int32]
    lib.grouter_host_wait.restype = ctypes.c_int
    lib.grouter_status.argtypes = [vp, vp]
    lib.grouter_status.restype = ctypes.c_int
    lib.grouter_strerror.argtypes = [ctypes.c_int]
    lib.grouter_strerror.restype = ctypes.c_char_p
    lib.grouter_dense_gemm.argtypes = [vp, ctypes.c_int, vp, ctypes.c_int, f32p, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, vp, vp]
    lib.grouter_dense_gemm.restype = ctypes.c_int
    lib.grouter_timing_enable.argtypes = [vp, ctypes.c_int32]
    lib.grouter_timing_enable.restype = ctypes.c_int
    lib.grouter_timing_gap.argtypes = [vp, ctypes.c_int32]
    lib.grouter_timing_gap.restype = ctypes.c_int
    lib.grouter_gemm_cycles_enable.argtypes = [vp, ctypes.c_int32]
    lib.grouter_gemm_cycles_enable.restype = ctypes.c_int
    lib.grouter_gemm_cycles_read.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_uint64)]
    lib.grouter_gemm_cycles_read.restype = ctypes.c_int
    lib.grouter_wgrad_chunk_rows.argtypes = [vp]
    lib.grouter_wgrad_chunk_rows.restype = ctypes.c_int32
    lib.grouter_ep_relabel_host.argtypes = [ctypes.c_int32, ctypes.c_int32, vp, vp, vp]
    lib.grouter_ep_relabel_host.restype = ctypes.c_int
    lib.grouter_ep_layout_host.argtypes = [ctypes.c_int32] * 3 + [vp] * 7
    lib.grouter_ep_layout_host.restype = ctypes.c_int
    lib.grouter_ep_expand_ids.argtypes = [vp] + [ctypes.c_int32] * 4 + [vp, vp]
    lib.grouter_ep_expand_ids.restype = ctypes.c_int
    lib.grouter_ep_dispatch_rows.argtypes = [vp] * 5
    lib.grouter_ep_dispatch_rows.restype = ctypes.c_int
    lib.grouter_ep_combine_rows.argtypes = [vp] * 7
    lib.grouter_ep_combine_rows.restype = ctypes.c_int
    lib.grouter_set_active_tokens.argtypes = [vp, ctypes.c_int32]
    lib.grouter_set_active_tokens.restype = ctypes.c_int
    lib.grouter_set_overlap.argtypes = [vp, ctypes.c_int32]
    lib.grouter_set_overlap.restype = ctypes.c_int
    lib.grouter_set_wait_limit.argtypes = [vp, ctypes.c_int64]
    lib.grouter_set_wait_limit.restype = ctypes.c_int
    lib.grouter_wait_selftest.argtypes = [vp, ctypes.c_int64, ctypes.POINTER(ctypes.c_int64), vp]
    lib.grouter_wait_selftest.restype = ctypes.c_int
    lib.grouter_timing_read.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int32)]
    lib.grouter_timing_read.restype = ctypes.c_int
    lib.grouter_checked_build.argtypes = []
    lib.grouter_checked_build.restype = ctypes.c_int
    i32, i64, f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    lib.grouter_layernorm_fwd.argtypes = [vp, i64, vp, vp, i32, i32, i32, i32, f32, vp, vp, vp, vp]
    lib.grouter_layernorm_fwd.restype = ctypes.c_int
    lib.grouter_layernorm_bwd_workspace_bytes.argtypes = [i32, i32]
    lib.grouter_layernorm_bwd_workspace_bytes.restype = ctypes.c_size_t
    lib.grouter_layernorm_bwd.argtypes = [vp, vp, i64, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, vp]
    lib.grouter_layernorm_bwd.restype = ctypes.c_int
    lib.grouter_linear_fwd.argtypes = [vp] * 4 + [i32] * 4 + [vp] * 4
    lib.grouter_linear_fwd.restype = ctypes.c_int
    lib.grouter_linear_bwd_workspace_bytes.argtypes = [i32] * 4
    lib.grouter_linear_bwd_workspace_bytes.restype = ctypes.c_size_t
    lib.grouter_linear_bwd.argtypes = [vp] * 4 + [i32] * 4 + [vp, vp, i32] + [vp] * 4
    lib.grouter_linear_bwd.restype = ctypes.c_int
    lib.grouter_expert_counts.argtypes = [vp, i32, vp, i32, i32, i32, vp, vp, vp, vp]
    lib.grouter_expert_counts.restype = ctypes.c_int
    lib.grouter_balance_loss_workspace_bytes.argtypes = [i32] * 3
    lib.grouter_balance_loss_workspace_bytes.restype = ctypes.c_size_t
    lib.grouter_balance_loss.argtypes = [vp, i64, i32, vp, i32, vp, vp, vp, vp, i32, i32, i32, i32, f32, f32, vp, vp, vp, vp, vp, vp]
    lib.grouter_balance_loss.restype = ctypes.c_int
    f64 = ctypes.c_double
    lib.grouter_adamw_layout_host.argtypes = [ctypes.POINTER(AdamwTensor), i32, ctypes.POINTER(AdamwLayout), vp]
    lib.grouter_adamw_layout_host.restype = ctypes.c_int
    lib.grouter_adamw_step.argtypes = [ctypes.POINTER(AdamwLayout), vp, i32] + [vp] * 5 + [f64] * 4 + [i64, vp, vp]
    lib.grouter_adamw_step.restype = ctypes.c_int
    lib.grouter_adamw_moments.argtypes = [vp] * 4 + [i64, vp, vp, vp]
    lib.grouter_adamw_moments.restype = ctypes.c_int
    if path == _build.LIB:
        _lib = lib
    return lib


@contextlib.contextmanager
def checked_build():
    """Inside the block every call of this module goes through the checked build of the library (compiled on demand):
    kernels that test data-derived indices before use and report GROUTER_ERR_BOUNDS (-9) through the status word."""
    global _lib
    release = load_library()
    try:
        path = _build.build(debug=True)
    except (OSError, RuntimeError) as err:      # as in load_library: an existing library is used, loudly
        path = _build.LIB_DEBUG
        if not os.path.exists(path):
            raise
        import sys
        sys.stderr.write(f"paper_2603_06626_b200: could not rebuild libgrouter_debug.so ({err}); loading the existing, possibly stale, library\n")
    lib = load_library(path)
    if lib.grouter_checked_build() != 1:
        raise RuntimeError("libgrouter_debug.so was not compiled with the index tests")
    _lib = lib
    try:
        yield lib
    finally:
        _lib = release


def strerror(code: int) -> str:
    return load_library().grouter_strerror(code).decode()


def _check(code: int, what: str) -> None:
    if code != 0:
        raise GrouterError(code, what)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    assert t.is_contiguous()
    return t.data_ptr()


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


class GrouterLayer:
    """One layer shape: owns the context and the workspace; thin calls into the C ABI."""

    def __init__(self, T: int, d: int, ffn: int, E_src: int, k: int, E_tgt: Optional[int] = None, idx_dtype: int = IDX_U8,
                 gate_dtype: int = GATE_BF16, device: str = "cuda:0", host_staging: bool = False, flags: int = 0,
                 plan_only: bool = False):
        self.lib = load_library()
        self.device = torch.device(device)
        self.dims = GrouterDims(T, d, ffn, E_src, E_src if E_tgt is None else E_tgt, k, idx_dtype, gate_dtype, flags)
        self.T, self.d, self.ffn, self.k = T, d, ffn, k
        self.T_active = T
        self.E_src, self.E_tgt = E_src, self.dims.E_tgt
        self.R = T * k
        with torch.cuda.device(self.device):
            h = ctypes.c_void_p()
            _check(self.lib.grouter_create(ctypes.byref(h), ctypes.byref(self.dims)), "grouter_create")
            self.ctx = h
            n = self.lib.grouter_workspace_bytes(ctypes.byref(self.dims))
            if n == 0:
                raise GrouterError(-3, "grouter_workspace_bytes")
            self.workspace_bytes = n
            if host_staging:
                n += self.lib.grouter_host_staging_bytes(ctypes.byref(self.dims))
            # plan_only: the caller only builds plans with this context (no forward/backward), so no workspace is needed
            self.workspace = None if plan_only else torch.empty(n, dtype=torch.uint8, device=self.device)
        i32 = dict(dtype=torch.int32, device=self.device)
        self.counts = torch.empty(self.E_tgt, **i32)
        self.offsets = torch.empty(self.E_tgt + 1, **i32)
        self.row_to_slot = torch.empty(self.R, **i32)
        self.slot_to_row = torch.empty(self.R, **i32)

    def close(self) -> None:
        if getattr(self, "ctx", None):
            self.lib.grouter_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def plan(self, idx: torch.Tensor, fold_map: Optional[torch.Tensor] = None):
        """idx [T,k] uint8/int32 (device); fold_map [E_src] int32 or None.  Results land in
        self.counts / offsets / row_to_slot / slot_to_row."""
        _check(self.lib.grouter_plan(self.ctx, _ptr(idx), _ptr(fold_map), _ptr(self.counts), _ptr(self.offsets),
                                     _ptr(self.row_to_slot), _ptr(self.slot_to_row), _stream()), "grouter_plan")
        n = self.T_active * self.k
        return self.counts, self.offsets, self.row_to_slot[:n], self.slot_to_row[:n]

    def forward(self, X, gates, W_gu, W_d, Y=None):
        if Y is None:
            Y = torch.empty_like(X)
        _check(self.lib.grouter_moe_fwd(self.ctx, _ptr(X), _ptr(gates), _ptr(W_gu), _ptr(W_d), _ptr(Y), _ptr(self.workspace),
                                        _stream()), "grouter_moe_fwd")
        return Y

    def backward(self, dY, X, gates, W_gu, W_d, dX=None, dW_gu=None, dW_d=None, dgates=None):
        f32 = dict(dtype=torch.float32, device=self.device)
        dX = torch.empty_like(X) if dX is None else dX
        dW_gu = torch.empty(W_gu.shape, **f32) if dW_gu is None else dW_gu
        dW_d = torch.empty(W_d.shape, **f32) if dW_d is None else dW_d
        dgates = torch.empty((self.T_active, self.k), **f32) if dgates is None else dgates
        _check(self.lib.grouter_moe_bwd(self.ctx, _ptr(dY), _ptr(X), _ptr(gates), _ptr(W_gu), _ptr(W_d), _ptr(dX), _ptr(dW_gu),
                                        _ptr(dW_d), _ptr(dgates), _ptr(self.workspace), _stream()), "grouter_moe_bwd")
        return dX, dW_gu, dW_d, dgates

    def host_wait(self, steps_in_flight: int = 0) -> None:
        """Blocks until all but the `steps_in_flight` (0 or 1) most recent step_host calls are complete."""
        _check(self.lib.grouter_host_wait(self.ctx, steps_in_flight), "grouter_host_wait")

    def step_host(self, idx_h, gates_h, X_h, dY_h, fold_map, W_gu, W_d, Y_h, dX_h, dgates_h, dW_gu, dW_d):
        """Whole step from pinned host tensors (idx, gates, X, dY in; Y, dX, dgates out).  Asynchronous: read the
        outputs (and reuse the inputs) only after host_wait() reports the step complete."""
        _check(self.lib.grouter_moe_step_host(self.ctx, _ptr(idx_h), _ptr(gates_h), _ptr(X_h), _ptr(dY_h), _ptr(fold_map), _ptr(W_gu),
                                              _ptr(W_d), _ptr(Y_h), _ptr(dX_h), _ptr(dgates_h), _ptr(dW_gu), _ptr(dW_d),
                                              _ptr(self.workspace), _stream()), "grouter_moe_step_host")

    def timing_enable(self, n_records: int) -> None:
        _check(self.lib.grouter_timing_enable(self.ctx, n_records), "grouter_timing_enable")

    def timing_gap(self, microseconds: int) -> None:
        """Idle time after every timed kernel (0 = none): kernels are then measured one at a time on a rested GPU."""
        _check(self.lib.grouter_timing_gap(self.ctx, microseconds), "grouter_timing_gap")

    def wgrad_chunk_rows(self) -> int:
        """Rows of one expert that the weight-gradient products contract in one piece."""
        return int(self.lib.grouter_wgrad_chunk_rows(self.ctx))

    def gemm_cycles_enable(self, on: bool) -> None:
        _check(self.lib.grouter_gemm_cycles_enable(self.ctx, 1 if on else 0), "grouter_gemm_cycles_enable")

    def gemm_cycles_read(self):
        """-> {GEMM name: dict(cycles, wait_operands, wait_accumulator, tiles, k_steps)} summed over CTA pairs and launches
        since the last read; synchronises the current stream."""
        buf = (ctypes.c_uint64 * 30)()
        _check(self.lib.grouter_gemm_cycles_read(self.ctx, _stream(), buf), "grouter_gemm_cycles_read")
        names = ["gemm_up_swiglu", "gemm_down", "gemm_dH", "gemm_dX", "wgrad_down", "wgrad_gate_up"]
        keys = ["cycles", "wait_operands", "wait_accumulator", "tiles", "k_steps"]
        return {n: {k: int(buf[5 * i + j]) for j, k in enumerate(keys)} for i, n in enumerate(names)}

    def ep_dispatch_rows(self, src, gates, rows):
        """rows[slot_to_row[s], :] = gate_s * src[token of s, :] (gates None: copy); rows [T*k, d] bf16."""
        _check(self.lib.grouter_ep_dispatch_rows(self.ctx, _ptr(src), _ptr(gates), _ptr(rows), _stream()), "grouter_ep_dispatch_rows")
        return rows

    def ep_combine_rows(self, rows, gates=None, out=None, dY=None, dgates=None):
        """out[t, :] = sum_j gate * rows[slot_to_row[t*k+j], :] and/or dgates[t, j] = <dY[t, :], rows[slot_to_row[t*k+j], :]>."""
        _check(self.lib.grouter_ep_combine_rows(self.ctx, _ptr(rows), _ptr(gates), _ptr(out), _ptr(dY), _ptr(dgates), _stream()),
               "grouter_ep_combine_rows")

    def set_active_tokens(self, tokens: int) -> None:
        """Later calls work on the first `tokens` tokens (<= the T the layer was created for): pass [tokens, ...] tensors.
        The plan outputs are views of the first entries of self.counts / offsets / row_to_slot / slot_to_row."""
        _check(self.lib.grouter_set_active_tokens(self.ctx, tokens), "grouter_set_active_tokens")
        self.T_active = tokens

    def set_overlap(self, on: bool) -> None:
        """Bandwidth-bound kernels of the backward pass beside the GEMMs (default) or in line."""
        _check(self.lib.grouter_set_overlap(self.ctx, 1 if on else 0), "grouter_set_overlap")

    def set_wait_limit(self, microseconds: int) -> None:
        """Limit of every bounded device-side wait of this context's later launches."""
        _check(self.lib.grouter_set_wait_limit(self.ctx, microseconds), "grouter_set_wait_limit")

    def wait_selftest(self, limit_microseconds: int) -> int:
        """One bounded wait that cannot succeed; returns the microseconds the kernel waited.  Leaves GROUTER_ERR_TIMEOUT in
        the status word (read and cleared by status())."""
        waited = ctypes.c_int64(0)
        _check(self.lib.grouter_wait_selftest(self.ctx, limit_microseconds, ctypes.byref(waited), _stream()), "grouter_wait_selftest")
        return int(waited.value)

    def timing_read(self):
        """-> {kernel name: (total ms, launches)} since the last read; synchronises the current stream."""
        n = len(KERNEL_SLOTS)
        ms = (ctypes.c_float * n)()
        cnt = (ctypes.c_int32 * n)()
        _check(self.lib.grouter_timing_read(self.ctx, _stream(), ms, cnt), "grouter_timing_read")
        return {KERNEL_SLOTS[i]: (float(ms[i]), int(cnt[i])) for i in range(n)}

    def status(self) -> int:
        """Synchronises the current stream; returns 0 or a negative GROUTER_ERR_* device status."""
        return self.lib.grouter_status(self.ctx, _stream())

    def check_status(self) -> None:
        _check(self.status(), "device status")


def route(H: torch.Tensor, W_s: torch.Tensor, fold_map: Optional[torch.Tensor], E_tgt: int, k: int, norm: int = NORM_SOFTMAX,
          want_scores: bool = False):
    """Router head (grouter_route): H [T,d_h] bf16, W_s [E_src,d_h] bf16 -> (idx uint8 [T,k], gates bf16 [T,k],
    folded scores f32 [T,E_tgt] or None).  Raises on a device-side status."""
    lib = load_library()
    T, d_h = H.shape
    E_src = W_s.shape[0]
    dev = H.device
    idx = torch.empty((T, k), dtype=torch.uint8, device=dev)
    gates = torch.empty((T, k), dtype=torch.bfloat16, device=dev)
    scores = torch.empty((T, E_tgt), dtype=torch.float32, device=dev) if want_scores else None
    ws = torch.empty(max(1, lib.grouter_route_workspace_bytes(T, E_src, E_tgt)), dtype=torch.uint8, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    with torch.cuda.device(dev):
        _check(lib.grouter_route(_ptr(H), _ptr(W_s), _ptr(fold_map), T, d_h, E_src, E_tgt, k, norm, _ptr(idx), _ptr(gates), _ptr(scores),
                                 _ptr(ws), _ptr(status), _stream()), "grouter_route")
        torch.cuda.synchronize(dev)
    st = int(status.item())
    if st != 0:
        raise GrouterError(-7 if st & 2 else -6, "grouter_route device status")
    return idx, gates, scores


def routing_stats(idx: torch.Tensor, E: int, seq_len: int, node_of_expert: Optional[torch.Tensor] = None, n_nodes: int = 0):
    """grouter_routing_stats: -> dict(loads, coact, phi, max_vio[, local_tokens, best_node]) of device tensors."""
    lib = load_library()
    T, k = idx.shape
    dev = idx.device
    S = T // max(seq_len, 1)
    i32 = dict(dtype=torch.int32, device=dev)
    out = dict(loads=torch.empty(E, **i32), coact=torch.empty((E, E), **i32), phi=torch.empty((S, E), dtype=torch.float32, device=dev),
               max_vio=torch.empty(1, dtype=torch.float32, device=dev))
    if node_of_expert is not None:
        out["local_tokens"] = torch.empty((S, n_nodes), **i32)
        out["best_node"] = torch.empty(S, **i32)
    status = torch.zeros(1, **i32)
    with torch.cuda.device(dev):
        _check(lib.grouter_routing_stats(_ptr(idx), IDX_U8 if idx.dtype == torch.uint8 else IDX_I32, T, k, E, seq_len, _ptr(node_of_expert),
                                         n_nodes, _ptr(out["loads"]), _ptr(out["coact"]), _ptr(out["phi"]), _ptr(out["max_vio"]),
                                         _ptr(out.get("local_tokens")), _ptr(out.get("best_node")), _ptr(status), _stream()),
               "grouter_routing_stats")
        torch.cuda.synchronize(dev)
    out["status"] = int(status.item())
    return out


def fold_greedy(coact, E_tgt: int):
    """grouter_fold_greedy_host: host int32 co-activation matrix [E_src,E_src] (numpy) -> fold_map int32 [E_src] (numpy)."""
    import numpy as np
    lib = load_library()
    P = np.ascontiguousarray(coact, dtype=np.int32)
    fold = np.empty(P.shape[0], dtype=np.int32)
    _check(lib.grouter_fold_greedy_host(P.ctypes.data, P.shape[0], E_tgt, fold.ctypes.data), "grouter_fold_greedy_host")
    return fold


def plan_noalloc(idx: torch.Tensor, fold_map: Optional[torch.Tensor], E_src: int, E_tgt: int, out=None, status=None,
                 null_status: bool = False):
    """Routing plan without a context and without any device allocation inside the library (grouter_plan_noalloc).

    For hosts that may not allocate: pass `out` = (counts[E_tgt], offsets[E_tgt+1], row_to_slot[R], slot_to_row[R])
    int32 device tensors and an int32[1] `status` tensor you already own, and nothing is allocated anywhere.
    When they are omitted this wrapper creates them with torch for convenience (the library still allocates nothing).
    With `null_status` the library is given no status word at all (it then keeps the bits in its own scratch and the
    caller learns nothing about bad ids); the last element of the result is None.
    Limits: T*k <= 524288, E_tgt <= 256.  Calls share one scratch array per GPU: keep them ordered on one stream.
    Returns (counts, offsets, row_to_slot, slot_to_row, status)."""
    lib = load_library()
    T, k = idx.shape
    dt = IDX_U8 if idx.dtype == torch.uint8 else IDX_I32
    i32 = dict(dtype=torch.int32, device=idx.device)
    if out is None:
        out = (torch.empty(E_tgt, **i32), torch.empty(E_tgt + 1, **i32), torch.empty(T * k, **i32), torch.empty(T * k, **i32))
    if status is None and not null_status:
        status = torch.empty(1, **i32)
    with torch.cuda.device(idx.device):
        _check(lib.grouter_plan_noalloc(_ptr(idx), dt, _ptr(fold_map), T, k, E_src, E_tgt, _ptr(out[0]), _ptr(out[1]), _ptr(out[2]),
                                        _ptr(out[3]), _ptr(status), _stream()), "grouter_plan_noalloc")
    return (*out, status)


def _elt(t: torch.Tensor, what: str) -> int:
    """GROUTER_BF16 / GROUTER_F32 of a tensor; other types raise."""
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise TypeError(f"{what}: bfloat16 or float32 expected, got {t.dtype}")


def _expect(what: str, t: Optional[torch.Tensor], shape, dtype=None, like: Optional[torch.Tensor] = None) -> None:
    """Raises unless t (None passes) is a contiguous tensor of this shape (and type), on the same device as `like`."""
    if t is None:
        return
    if t.shape != shape:
        raise ValueError(f"{what}: shape {tuple(shape)} expected, got {tuple(t.shape)}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{what}: {dtype} expected, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{what}: a contiguous tensor is expected")
    if like is not None and t.device != like.device:
        raise ValueError(f"{what}: on {t.device}, the other arguments are on {like.device}")


def _fits(t: Optional[torch.Tensor], shape, dtype, dev: torch.device) -> bool:
    """What _expect checks, in one expression: the calls below ask this first and look for the reason only when it fails."""
    return t is None or (t.shape == shape and t.dtype == dtype and t.device == dev and t.is_contiguous())


def _device_index(dev: torch.device) -> int:
    """Index of a CUDA device; other devices raise."""
    if dev.type != "cuda":
        raise ValueError(f"a CUDA tensor is expected, got one on {dev}")
    return dev.index if dev.index is not None else torch.cuda.current_device()


def _raw_stream(index: int) -> int:
    """Handle of the device's current torch stream, without building a torch.cuda.Stream around it (3 us of a call of 10)."""
    return torch._C._cuda_getCurrentRawStream(index)


def _call(fn, what: str, index: int, *args) -> None:
    """Calls the library with the arguments and the current stream, on the given device; raises on an error code."""
    if torch._C._cuda_getDevice() == index:
        code = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            code = fn(*args, _raw_stream(index))
    if code != 0:
        raise GrouterError(code, what)


def _row_stride(what: str, x: torch.Tensor) -> int:
    """Elements between the rows of a matrix whose rows are contiguous; other layouts raise."""
    if x.dim() == 2 and x.is_contiguous():
        return x.shape[1]
    if x.dim() != 2 or (x.shape[1] > 1 and x.stride(1) != 1):
        raise ValueError(f"{what}: a matrix with contiguous rows is expected")
    if x.shape[0] <= 1:
        return x.shape[1]
    if x.stride(0) < x.shape[1]:
        raise ValueError(f"{what}: rows that overlap")
    return x.stride(0)


def _dense_like(x: torch.Tensor) -> torch.Tensor:
    """An uninitialised contiguous tensor of x's shape and type."""
    return torch.empty_like(x) if x.is_contiguous() else x.new_empty(x.shape)


def layer_norm(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, eps: float = 1e-5):
    """grouter_layernorm_fwd: x [T,d] bf16/f32 (rows may be strided), weight and bias [d] bf16/f32 -> (y, mean f32 [T], rstd f32 [T])."""
    lib = load_library()
    ldx = _row_stride("x", x)
    T, d = x.shape
    on = x.device
    if not (_fits(weight, (d,), weight.dtype, on) and _fits(bias, (d,), weight.dtype, on)):
        _expect("weight", weight, (d,), like=x)
        _expect("bias", bias, (d,), weight.dtype, like=x)
    dt, wt = _elt(x, "x"), _elt(weight, "weight")
    dev = _device_index(on)
    y = _dense_like(x)
    mean = x.new_empty(T, dtype=torch.float32)
    rstd = x.new_empty(T, dtype=torch.float32)
    _call(lib.grouter_layernorm_fwd, "grouter_layernorm_fwd", dev, x.data_ptr(), ldx, weight.data_ptr(), _ptr(bias), T, d, dt, wt, eps, y.data_ptr(),
          mean.data_ptr(), rstd.data_ptr())
    return y, mean, rstd


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, want_bias: bool = True,
                        dw: Optional[torch.Tensor] = None, db: Optional[torch.Tensor] = None):
    """grouter_layernorm_bwd, from the forward's mean and rstd -> (dx like x, dw f32 [d], db f32 [d] or None).  dw, db: tensors to
    write the gradients into, e.g. those an AdamW object reads."""
    lib = load_library()
    ldx = _row_stride("x", x)
    T, d = x.shape
    on, f32 = x.device, torch.float32
    if not (_fits(dy, x.shape, x.dtype, on) and _fits(weight, (d,), weight.dtype, on) and _fits(mean, (T,), f32, on) and
            _fits(rstd, (T,), f32, on) and _fits(dw, (d,), f32, on) and _fits(db, (d,), f32, on)):
        _expect("dy", dy, (T, d), x.dtype, like=x)
        _expect("weight", weight, (d,), like=x)
        for name, v, n in (("mean", mean, T), ("rstd", rstd, T), ("dw", dw, d), ("db", db, d)):
            _expect(name, v, (n,), f32, like=x)
    dt, wt = _elt(x, "x"), _elt(weight, "weight")
    dev = _device_index(on)
    dx = torch.empty_like(dy)
    if dw is None:
        dw = x.new_empty(d, dtype=torch.float32)
    if db is None and want_bias:
        db = x.new_empty(d, dtype=torch.float32)
    ws = x.new_empty(_bytes(lib.grouter_layernorm_bwd_workspace_bytes, dev, T, d), dtype=torch.uint8)
    _call(lib.grouter_layernorm_bwd, "grouter_layernorm_bwd", dev, dy.data_ptr(), x.data_ptr(), ldx, weight.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
          T, d, dt, wt, dx.data_ptr(), dw.data_ptr(), _ptr(db), ws.data_ptr())
    return dx, dw, db


def _bytes(fn, index: int, *args) -> int:
    """Workspace bytes, which depend on the device they are for."""
    if torch._C._cuda_getDevice() == index:
        return fn(*args)
    with torch.cuda.device(index):
        return fn(*args)


_status_words = {}
_status_lock = threading.Lock()


def _status_word(index: int) -> torch.Tensor:
    """The status word of a device that the calls without one of their own share."""
    word = _status_words.get(index)
    if word is not None:
        return word
    with _status_lock:                     # one word a device: a second one would be freed under the kernels that were given it
        word = _status_words.get(index)
        if word is None:
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("the first call on a device sets up its status word: make it outside a stream capture, or pass status=")
            word = torch.zeros(1, dtype=torch.int32, device=torch.device("cuda", index))
            torch.cuda.synchronize(index)  # zeroed before a kernel on any stream can set a bit in it
            _status_words[index] = word
    return word


def check_status(device="cuda:0", status: Optional[torch.Tensor] = None) -> None:
    """Waits for the device; raises when a linear, linear_backward, expert_counts or balance_loss call without a status word of its own
    met a bounded wait that ran out or an expert id out of range since the last check, and clears the bits that it has seen.  That word
    is one for all streams and threads of the process; calls that passed status= are checked by passing the same one here (the device
    is then its own)."""
    index = _device_index(torch.device(device) if status is None else status.device)
    torch.cuda.synchronize(index)
    word = _status_word(index) if status is None else status
    with _status_lock:
        st = int(word.item())
        if st != 0:
            word.bitwise_and_(~st)      # what other threads' calls have found since stays for the next check
            torch.cuda.synchronize(index)
    if st != 0:
        raise GrouterError(-7 if st & 2 else -6, "device status")


def _status_ptr(status: Optional[torch.Tensor], index: int) -> int:
    return (_status_word(index) if status is None else status).data_ptr()


def linear(x: torch.Tensor, W: torch.Tensor, bias: Optional[torch.Tensor] = None, act: int = ACT_NONE, residual: Optional[torch.Tensor] = None,
           save_pre: bool = False, status: Optional[torch.Tensor] = None):
    """grouter_linear_fwd: act(x W^T + bias) + residual, x [T,K], W [N,K], all bf16 -> (y [T,N], x W^T + bias [T,N] or None)."""
    lib = load_library()
    if x.dim() != 2 or W.dim() != 2:
        raise ValueError("x and W: matrices are expected")
    T, K = x.shape
    N = W.shape[0]
    bf, on = torch.bfloat16, x.device
    if not (_fits(x, (T, K), bf, on) and _fits(W, (N, K), bf, on) and _fits(bias, (N,), bf, on) and _fits(residual, (T, N), bf, on) and
            _fits(status, (1,), torch.int32, on)):
        _expect("x", x, (T, K), bf)
        _expect("W", W, (N, K), bf, like=x)
        _expect("bias", bias, (N,), bf, like=x)
        _expect("residual", residual, (T, N), bf, like=x)
        _expect("status", status, (1,), torch.int32, like=x)
    dev = _device_index(on)
    y = x.new_empty((T, N))
    pre = x.new_empty((T, N)) if save_pre else None
    _call(lib.grouter_linear_fwd, "grouter_linear_fwd", dev, x.data_ptr(), W.data_ptr(), _ptr(bias), _ptr(residual), T, K, N, act, y.data_ptr(),
          _ptr(pre), _status_ptr(status, dev))
    return y, pre


def linear_backward(dy: torch.Tensor, x: torch.Tensor, W: torch.Tensor, pre: Optional[torch.Tensor] = None, act: int = ACT_NONE,
                    want_dx: bool = True, want_dW: bool = True, want_bias: bool = False, dW_dtype: torch.dtype = torch.bfloat16,
                    dW: Optional[torch.Tensor] = None, db: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """grouter_linear_bwd; pre: the forward's x W^T + bias, needed with an activation -> (dx bf16 [T,K], dW [N,K] of dW_dtype,
    db f32 [N]), None for what is not wanted.  The residual's gradient is dy.  dW, db: tensors to write the gradients into (dW bf16
    or f32), e.g. those an AdamW object reads."""
    lib = load_library()
    if x.dim() != 2 or W.dim() != 2:
        raise ValueError("x and W: matrices are expected")
    T, K = x.shape
    N = W.shape[0]
    bf, on = torch.bfloat16, x.device
    if not (_fits(x, (T, K), bf, on) and _fits(W, (N, K), bf, on) and _fits(dy, (T, N), bf, on) and _fits(pre, (T, N), bf, on) and
            _fits(db, (N,), torch.float32, on) and _fits(status, (1,), torch.int32, on)):
        _expect("x", x, (T, K), bf)
        _expect("W", W, (N, K), bf, like=x)
        _expect("dy", dy, (T, N), bf, like=x)
        _expect("pre", pre, (T, N), bf, like=x)
        _expect("db", db, (N,), torch.float32, like=x)
        _expect("status", status, (1,), torch.int32, like=x)
    if act != ACT_NONE and pre is None:
        raise ValueError("pre: needed with an activation")
    if dW is not None:
        dW_dtype = dW.dtype
        _expect("dW", dW, (N, K), like=x)
    if dW_dtype != bf and dW_dtype != torch.float32:
        raise TypeError(f"dW: bfloat16 or float32 expected, got {dW_dtype}")
    dev = _device_index(on)
    dx = torch.empty_like(x) if want_dx else None
    if dW is None and want_dW:
        dW = x.new_empty((N, K), dtype=dW_dtype)
    if db is None and want_bias:
        db = x.new_empty(N, dtype=torch.float32)
    ws = x.new_empty(_bytes(lib.grouter_linear_bwd_workspace_bytes, dev, T, K, N, act), dtype=torch.uint8)
    _call(lib.grouter_linear_bwd, "grouter_linear_bwd", dev, dy.data_ptr(), x.data_ptr(), W.data_ptr(), _ptr(pre), T, K, N, act, _ptr(dx), _ptr(dW),
          F32 if dW_dtype == torch.float32 else BF16, _ptr(db), ws.data_ptr(), _status_ptr(status, dev))
    return dx, dW, db


def _idx_dtype(idx: torch.Tensor) -> int:
    if idx.dtype == torch.uint8:
        return IDX_U8
    if idx.dtype == torch.int32:
        return IDX_I32
    raise TypeError(f"idx: uint8 or int32 expected, got {idx.dtype}")


def _check_mask(mask: Optional[torch.Tensor], T: int, like: torch.Tensor) -> None:
    if mask is None:
        return
    if mask.dtype != torch.uint8 and mask.dtype != torch.bool:
        raise TypeError(f"mask: uint8 or bool expected, got {mask.dtype}")
    if not _fits(mask, (T,), mask.dtype, like.device):
        _expect("mask", mask, (T,), like=like)


def expert_counts(idx: torch.Tensor, E: int, mask: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """grouter_expert_counts: idx [T,k] uint8/int32 (16-byte aligned), mask [T] uint8/bool (zero: the token does not count) -> (counts int32 [E],
    counted tokens int32 [1])."""
    lib = load_library()
    if idx.dim() != 2:
        raise ValueError("idx: a matrix is expected")
    T, k = idx.shape
    on = idx.device
    if not (_fits(idx, idx.shape, idx.dtype, on) and _fits(status, (1,), torch.int32, on)):
        _expect("idx", idx, (T, k))
        _expect("status", status, (1,), torch.int32, like=idx)
    _check_mask(mask, T, idx)
    dt = _idx_dtype(idx)
    dev = _device_index(on)
    counts = idx.new_empty(E, dtype=torch.int32)
    n = idx.new_empty(1, dtype=torch.int32)
    _call(lib.grouter_expert_counts, "grouter_expert_counts", dev, idx.data_ptr(), dt, _ptr(mask), T, k, E, counts.data_ptr(), n.data_ptr(),
          _status_ptr(status, dev))
    return counts, n


def balance_loss(logits: torch.Tensor, idx: Optional[torch.Tensor], counts: torch.Tensor, n_tokens: torch.Tensor,
                 mask: Optional[torch.Tensor] = None, balance_coef: float = 1e-2, z_coef: float = 0.0, dgates: Optional[torch.Tensor] = None,
                 norm: int = NORM_SOFTMAX, want_loss: bool = True, want_grad: bool = True, dloss: Optional[torch.Tensor] = None,
                 status: Optional[torch.Tensor] = None):
    """grouter_balance_loss: logits [T,E] bf16/f32 (rows may be strided), counts and n_tokens of expert_counts -> (loss f32 [3]:
    sum, balance, z; dlogits like logits), None for what is not wanted.  With dgates f32 [T,k] (GrouterLayer.backward) and idx [T,k]
    the gradient that comes back through the gates is added to dlogits."""
    lib = load_library()
    ld = _row_stride("logits", logits)
    T, E = logits.shape
    dt = _elt(logits, "logits")
    if dgates is not None and idx is None:
        raise ValueError("idx: needed with dgates")
    k, it = 1, IDX_U8
    if idx is not None:
        if idx.dim() != 2:
            raise ValueError("idx: a matrix is expected")
        k, it = idx.shape[1], _idx_dtype(idx)
    on, i32 = logits.device, torch.int32
    if not (_fits(counts, (E,), i32, on) and _fits(n_tokens, (1,), i32, on) and _fits(dgates, (T, k), torch.float32, on) and
            _fits(status, (1,), i32, on) and (idx is None or _fits(idx, (T, k), idx.dtype, on))):
        _expect("idx", idx, (T, k), like=logits)
        _expect("counts", counts, (E,), i32, like=logits)
        _expect("n_tokens", n_tokens, (1,), i32, like=logits)
        _expect("dgates", dgates, (T, k), torch.float32, like=logits)
        _expect("status", status, (1,), i32, like=logits)
    if dloss is not None:
        if dloss.numel() != 1:
            raise ValueError("dloss: one number is expected")
        _expect("dloss", dloss.reshape(1), (1,), torch.float32, like=logits)
    _check_mask(mask, T, logits)
    dev = _device_index(on)
    loss = logits.new_empty(3, dtype=torch.float32) if want_loss else None
    d = _dense_like(logits) if want_grad else None
    need = _bytes(lib.grouter_balance_loss_workspace_bytes, dev, T, E, k) if want_loss else 0
    ws = logits.new_empty(need, dtype=torch.uint8) if need else None
    _call(lib.grouter_balance_loss, "grouter_balance_loss", dev, logits.data_ptr(), ld, dt, _ptr(idx), it, _ptr(mask), counts.data_ptr(),
          n_tokens.data_ptr(), _ptr(dgates), norm, T, E, k, balance_coef, z_coef, _ptr(dloss), _ptr(loss), _ptr(d), _ptr(ws),
          _status_ptr(status, dev))
    return loss, d


class AdamW:
    """AdamW over a list of tensors, one launch a step (grouter_adamw_*).

    params: contiguous f32 tensors, updated in place, or bf16 tensors with an f32 master copy that this object keeps; grads: one
    contiguous f32 or bf16 tensor for each, whose memory every step reads (the layer's backward writes its gradients into
    caller-owned tensors: keep writing the same ones).  A parameter shares no memory with another one or with a gradient.
    weight_decay: a number, or one for each tensor.  Moments (and masters) lie in flat tensors m, v (and master), tensor i from element
    offsets[i] on: f32 with state_bits 32; with state_bits 8 one byte an element (m, and the root of v) plus m_exp, v_exp, one byte for
    32 elements.  state: those tensors of a run to be continued, with steps_done; without it the moments start at zero and the masters
    at the parameters' values."""

    GROUP = 32

    def __init__(self, params, grads, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay=0.01, state_bits: int = 32,
                 state: Optional[dict] = None, steps_done: int = 0):
        self.lib = load_library()
        self.params, self.grads = list(params), list(grads)
        if not self.params or len(self.params) != len(self.grads):
            raise ValueError("one gradient for every parameter is expected, and at least one")
        if state_bits not in (8, 32):
            raise ValueError(f"state_bits: 8 or 32 expected, got {state_bits}")
        n = len(self.params)
        wd = [float(weight_decay)] * n if isinstance(weight_decay, (int, float)) else [float(w) for w in weight_decay]
        if len(wd) != n:
            raise ValueError("weight_decay: a number, or one for each tensor")
        self.device = self.params[0].device
        self.state_bits, self.steps_done = state_bits, int(steps_done)
        self.lr, self.betas, self.eps = lr, tuple(betas), eps
        desc = (AdamwTensor * n)()
        self.offsets, at = [], 0
        for i, (p, g) in enumerate(zip(self.params, self.grads)):
            _expect(f"gradient {i}", g, p.shape, like=self.params[0])
            _expect(f"parameter {i}", p, p.shape, like=self.params[0])
            if p.data_ptr() == g.data_ptr() and p.dtype != g.dtype and p.numel():
                raise ValueError(f"gradient {i}: of another type in its parameter's memory")
            desc[i] = AdamwTensor(p.data_ptr(), g.data_ptr(), p.numel(), wd[i], _elt(p, f"parameter {i}"), _elt(g, f"gradient {i}"))
            self.offsets.append(at)
            at += (p.numel() + self.GROUP - 1) // self.GROUP * self.GROUP
        self._layout = AdamwLayout()
        _check(self.lib.grouter_adamw_layout_host(desc, n, ctypes.byref(self._layout), None), "grouter_adamw_layout_host")
        size = self._layout.state_elements
        assert size == at
        dev, u8, f32 = self.device, torch.uint8, torch.float32
        given = dict(state or {})
        kinds = dict(m=f32, v=f32) if state_bits == 32 else dict(m=u8, v=u8, m_exp=u8, v_exp=u8)
        if self._layout.needs_master:
            kinds["master"] = f32
        for name in given:
            if name not in kinds:
                raise ValueError(f"state: no {name} is kept here")
        for name, kind in kinds.items():
            shape = (size // self.GROUP if name.endswith("_exp") else size,)
            t = given.get(name)
            if t is None:
                t = torch.zeros(shape, dtype=kind, device=dev)
                if name == "master":
                    for p, o in zip(self.params, self.offsets):
                        t[o:o + p.numel()] = p.detach().reshape(-1)
            _expect(name, t, shape, kind, like=self.params[0])
            setattr(self, name, t)
        host = torch.zeros(max(16, self._layout.table_bytes), dtype=u8)
        _check(self.lib.grouter_adamw_layout_host(desc, n, ctypes.byref(self._layout), host.data_ptr()), "grouter_adamw_layout_host")
        self._table = host.to(dev)
        self._index = _device_index(dev)
        # the addresses of the state, which this object keeps for good
        self._args = (ctypes.byref(self._layout), self._table.data_ptr(), state_bits, _ptr(getattr(self, "master", None)), self.m.data_ptr(),
                      self.v.data_ptr(), _ptr(getattr(self, "m_exp", None)), _ptr(getattr(self, "v_exp", None)))

    def step(self, grad_scale: Optional[torch.Tensor] = None, lr: Optional[float] = None) -> None:
        """One update from the gradients as they are now.  grad_scale: f32 device scalar every gradient is multiplied by."""
        if grad_scale is not None and (grad_scale.numel() != 1 or grad_scale.dtype != torch.float32 or grad_scale.device != self.device):
            raise ValueError("grad_scale: one f32 number on the parameters' device is expected")
        if lr is not None:
            self.lr = lr
        _call(self.lib.grouter_adamw_step, "grouter_adamw_step", self._index, *self._args, self.lr, self.betas[0], self.betas[1], self.eps,
              self.steps_done + 1, _ptr(grad_scale))
        self.steps_done += 1

    def moments(self):
        """(m, v) as flat f32 tensors: the state itself with 32 bits, the values that the codes stand for with 8."""
        if self.state_bits == 32:
            return self.m, self.v
        m, v = self.m.new_empty(self.m.shape, dtype=torch.float32), self.m.new_empty(self.m.shape, dtype=torch.float32)
        _call(self.lib.grouter_adamw_moments, "grouter_adamw_moments", self._index, self.m.data_ptr(), self.v.data_ptr(), self.m_exp.data_ptr(),
              self.v_exp.data_ptr(), self.m.numel(), m.data_ptr(), v.data_ptr())
        return m, v


def dense_gemm(A: torch.Tensor, a_mn_major: bool, B: torch.Tensor, b_mn_major: bool, M: int, N: int, K: int) -> torch.Tensor:
    """C[M,N] f32 = A*B on the tcgen05 core (component check).  A is [M,K] or, MN-major, [K,M]; B is [N,K] or [K,N]."""
    lib = load_library()
    C = torch.empty((M, N), dtype=torch.float32, device=A.device)
    status = torch.zeros(1, dtype=torch.int32, device=A.device)
    _check(lib.grouter_dense_gemm(_ptr(A), int(a_mn_major), _ptr(B), int(b_mn_major), _ptr(C), M, N, K, _ptr(status), _stream()),
           "grouter_dense_gemm")
    torch.cuda.synchronize(A.device)
    if int(status.item()) != 0:
        raise GrouterError(-7, "grouter_dense_gemm device status")
    return C
