"""Thin ctypes binding of libgvq.so: argument marshalling only.

Every function here has the name and the meaning of the C entry point it calls
(see include/gvq.h); tensors are torch CUDA tensors used purely as device
memory, and the current torch stream is handed to the library.  There is no
fallback: if the shared library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import math
from pathlib import Path
from typing import Optional, Sequence

import torch

_PKG = Path(__file__).resolve().parent
LIB_PATH = _PKG / "libgvq.so"
_lib = None

MAX_NODES = 64

STATUS = {0: "GVQ_OK", 1: "GVQ_ERR_NULL", 2: "GVQ_ERR_SHAPE", 3: "GVQ_ERR_ALIGN", 4: "GVQ_ERR_UNSUPPORTED",
          5: "GVQ_ERR_WORKSPACE", 6: "GVQ_ERR_CUDA", 7: "GVQ_ERR_NOT_CONVERGED", 8: "GVQ_ERR_DEGENERATE",
          9: "GVQ_ERR_TIMEOUT", 10: "GVQ_ERR_CAPTURE"}


class GvqError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        msg = lib().gvq_status_string(status).decode()
        super().__init__(f"{what}: {STATUS.get(status, status)} ({msg})")


class _Layout(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int32), ("k", ctypes.c_int32), ("n_layers", ctypes.c_int32),
                ("layer_off", ctypes.POINTER(ctypes.c_int64)), ("layer_len", ctypes.POINTER(ctypes.c_int64))]


def lib() -> ctypes.CDLL:
    """Loads libgvq.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_1811_03617_b200.build` "
                               "(there is no fallback implementation)")
        L = ctypes.CDLL(str(LIB_PATH))
        vp, i32, i64, u64, u32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_uint64, ctypes.c_uint32
        LP = ctypes.POINTER(_Layout)
        L.gvq_status_string.restype = ctypes.c_char_p
        L.gvq_status_string.argtypes = [i32]
        L.gvq_layout_check.argtypes = [LP]
        L.gvq_total_slices.restype = i64
        L.gvq_total_slices.argtypes = [LP]
        L.gvq_total_entries.restype = i64
        L.gvq_total_entries.argtypes = [LP]
        L.gvq_fit_workspace_bytes.restype = ctypes.c_size_t
        L.gvq_fit_workspace_bytes.argtypes = [LP, i32]
        L.gvq_host_workspace_bytes.restype = ctypes.c_size_t
        L.gvq_host_workspace_bytes.argtypes = [LP, i32]
        L.gvq_select_k.argtypes = [vp, i32, ctypes.c_double, ctypes.POINTER(ctypes.c_int32)]
        L.gvq_create.argtypes = [ctypes.POINTER(vp), LP, i32, vp]
        L.gvq_destroy.argtypes = [vp]
        L.gvq_set_stream.argtypes = [vp, vp]
        L.gvq_set_workspace.argtypes = [vp, vp, ctypes.c_size_t]
        L.gvq_last_cuda_error.argtypes = [vp]
        L.gvq_set_projection_path.argtypes = [vp, i32]
        L.gvq_set_fit_path.argtypes = [vp, i32]
        L.gvq_device_status.argtypes = [vp]
        L.gvq_compress.argtypes = [vp, vp, vp, vp, i32, vp]
        L.gvq_aggregate.argtypes = [vp, vp, i32, vp]
        L.gvq_compress_aggregate.argtypes = [vp, vp, i32, vp, vp, vp, vp]
        L.gvq_compress_quantize_aggregate.argtypes = [vp, vp, i32, vp, vp, i32, u64, vp, vp, vp]
        L.gvq_decompress.argtypes = [vp, vp, vp, vp, vp, i32, vp]
        L.gvq_fit_basis.argtypes = [vp, vp, i64, i32, i32, i32, vp, vp, vp, vp]
        L.gvq_refresh_basis.argtypes = [vp, vp, i64, i32, i32, i32, i32, i32, vp, vp, vp, vp]
        L.gvq_fit_basis_static.argtypes = [vp, vp, i64, i32, i32, i32, vp, vp, vp, vp]
        L.gvq_fit_moments_count.restype = i64
        L.gvq_fit_moments_count.argtypes = [LP]
        L.gvq_fit_centre.argtypes = [vp, vp, i64, i32, vp]
        L.gvq_fit_moments.argtypes = [vp, vp, i64, i32, vp, vp]
        L.gvq_fit_from_moments.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, vp]
        L.gvq_quantize.argtypes = [vp, vp, i32, u64, u32, vp, vp]
        L.gvq_compress_aggregate_monitored.argtypes = [vp, vp, i32, vp, vp, vp, vp, vp]
        L.gvq_quantize_aggregate.argtypes = [vp, vp, i32, i32, u64, vp, vp, vp]
        L.gvq_dequantize_aggregate.argtypes = [vp, vp, vp, i32, i32, vp]
        L.gvq_allreduce_host.argtypes = [vp, vp, i32, vp, vp, vp]
        L.gvq_allreduce_host_quantized.argtypes = [vp, vp, i32, vp, vp, i32, u64, vp]
        L.gvq_host_prepare.argtypes = [vp]
        L.gvq_set_limits.argtypes = [vp, i32, i64]
        L.gvq_test_drop_load.argtypes = [vp, i32]
        L.gvq_work_partition.argtypes = [LP, i32, i32, i32, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(i64)]
        L.gvq_quantize_raw4.argtypes = [vp, vp, i32, u64, u32, vp, vp]
        L.gvq_quantize_raw4_aggregate.argtypes = [vp, vp, i32, i32, u64, vp, vp, vp]
        L.gvq_dequantize_raw4_aggregate.argtypes = [vp, vp, vp, vp, i32, i32, vp]
        L.gvq_flatten_layer.argtypes = [vp, vp, vp, i32, i32, i32]
        L.gvq_unflatten_layer.argtypes = [vp, vp, vp, i32, i32, i32]
        L.gvq_mx4_codes_bytes.restype = i64
        L.gvq_mx4_codes_bytes.argtypes = [i64, i64]
        L.gvq_mx4_scales_bytes.restype = i64
        L.gvq_mx4_scales_bytes.argtypes = [i64, i64]
        L.gvq_mx4_quantize.argtypes = [vp, vp, i32, i64, i64, i64, i32, u64, u32, vp, vp, vp, vp]
        L.gvq_mx4_dequantize.argtypes = [vp, vp, vp, i64, i64, vp, i64]
        L.gvq_mx4_matmul.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, vp, i32, i64]
        L.gvq_mx4_quantize_aggregate.argtypes = [vp, vp, i32, u32, i32, u64, vp, vp, vp]
        L.gvq_mx4_dequantize_aggregate.argtypes = [vp, vp, vp, vp, i32, vp]
        i32p = ctypes.POINTER(ctypes.c_int32)
        L.gvq_ortho_workspace_bytes.restype = i64
        L.gvq_ortho_workspace_bytes.argtypes = [LP, i32p, i32p]
        L.gvq_ortho_create.argtypes = [ctypes.POINTER(vp), vp, i32p, i32p, ctypes.POINTER(ctypes.c_float), vp, ctypes.c_size_t]
        L.gvq_ortho_destroy.argtypes = [vp]
        L.gvq_ortho_step.argtypes = [vp, vp, vp, ctypes.c_float, i32, vp, i32, ctypes.c_float, ctypes.c_float]
        L.gvq_orthogonalize.argtypes = [vp, vp, vp, i32]
        L.gvq_exchange_floats.argtypes = [LP]
        L.gvq_exchange_floats.restype = i64
        L.gvq_segment_layout.argtypes = [LP, i32, i32, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32),
                                         ctypes.POINTER(i64), ctypes.POINTER(i64)]
        L.gvq_compress_aggregate_partial.argtypes = [vp, vp, i32, i32, vp, vp, vp]
        L.gvq_exchange_accumulate.argtypes = [vp, vp, vp]
        L.gvq_decompress_exchanged.argtypes = [vp, vp, vp, vp, vp]
        L.gvq_mask_basis.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_int32)]
        L.gvq_packed_floats.restype = i64
        L.gvq_packed_floats.argtypes = [LP, ctypes.POINTER(ctypes.c_int32)]
        L.gvq_set_layer_k.argtypes = [vp, ctypes.POINTER(ctypes.c_int32)]
        L.gvq_exchange_pack.argtypes = [vp, vp, vp]
        L.gvq_exchange_unpack.argtypes = [vp, vp, vp]
        L.gvq_schedule_create.argtypes = [ctypes.POINTER(vp), i32, i32, i32, ctypes.c_double]
        L.gvq_schedule_destroy.argtypes = [vp]
        L.gvq_schedule_phase.argtypes = [vp]
        L.gvq_schedule_nodes_over.argtypes = [vp]
        L.gvq_schedule_step.argtypes = [vp, vp, i32, ctypes.POINTER(i32)]
        L.gvq_schedule_counters.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(i64), ctypes.POINTER(i64)]
        _lib = L
    return _lib


def _ptr_array(tensors: Sequence[torch.Tensor]):
    return (ctypes.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])


def _check(status: int, what: str) -> None:
    if status != 0:
        raise GvqError(status, what)


class HostLayout:
    """Owns the ctypes image of a gvq_layout (host-only helpers work without a GPU)."""

    def __init__(self, d: int, k: int, layer_off: Sequence[int], layer_len: Sequence[int]):
        n = len(layer_len)
        self.d, self.k = int(d), int(k)
        self.layer_off, self.layer_len = [int(v) for v in layer_off], [int(v) for v in layer_len]
        self._off = (ctypes.c_int64 * n)(*self.layer_off)
        self._len = (ctypes.c_int64 * n)(*self.layer_len)
        self.c = _Layout(self.d, self.k, n, self._off, self._len)

    @classmethod
    def of(cls, w) -> "HostLayout":
        return cls(w.d, w.k, w.layer_off, w.layer_len)

    def check(self) -> int:
        return lib().gvq_layout_check(ctypes.byref(self.c))

    def total_slices(self) -> int:
        return lib().gvq_total_slices(ctypes.byref(self.c))

    def total_entries(self) -> int:
        return lib().gvq_total_entries(ctypes.byref(self.c))

    def fit_workspace_bytes(self, L: int) -> int:
        return lib().gvq_fit_workspace_bytes(ctypes.byref(self.c), L)

    def host_workspace_bytes(self, N: int) -> int:
        return lib().gvq_host_workspace_bytes(ctypes.byref(self.c), N)

    def exchange_floats(self) -> int:
        return lib().gvq_exchange_floats(ctypes.byref(self.c))

    def fit_moments_count(self) -> int:
        return lib().gvq_fit_moments_count(ctypes.byref(self.c))

    def packed_floats(self, k_per_layer) -> int:
        ks = (ctypes.c_int32 * len(self.layer_len))(*[int(x) for x in k_per_layer])
        return lib().gvq_packed_floats(ctypes.byref(self.c), ks)


def segment_layout(layout, n_segments: int, j: int):
    """gvq_segment_layout: (HostLayout of segment j or None when it is empty, parent layer of each piece)."""
    hl = layout if isinstance(layout, HostLayout) else HostLayout.of(layout)
    n = len(hl.layer_len)
    n_pieces = ctypes.c_int32(0)
    layer = (ctypes.c_int32 * n)()
    off, ln = (ctypes.c_int64 * n)(), (ctypes.c_int64 * n)()
    _check(lib().gvq_segment_layout(ctypes.byref(hl.c), n_segments, j, ctypes.byref(n_pieces), layer, off, ln),
           "gvq_segment_layout")
    m = n_pieces.value
    if m == 0:
        return None, []
    return HostLayout(hl.d, hl.k, list(off[:m]), list(ln[:m])), list(layer[:m])


def work_partition(layout, kind: int, n_nodes: int, n_parts: int):
    """gvq_work_partition: (list of n_parts + 1 unit indices, total units)."""
    hl = layout if isinstance(layout, HostLayout) else HostLayout.of(layout)
    start = (ctypes.c_int32 * (n_parts + 1))()
    total = ctypes.c_int64(0)
    _check(lib().gvq_work_partition(ctypes.byref(hl.c), kind, n_nodes, n_parts, start, ctypes.byref(total)),
           "gvq_work_partition")
    return list(start), total.value


def select_k(evals, lambda_loss: float) -> int:
    """gvq_select_k (Eq. 6) on one layer's descending eigenvalues (host tensor / sequence)."""
    ev = torch.as_tensor(evals, dtype=torch.float32).contiguous().cpu()
    out = ctypes.c_int32(0)
    _check(lib().gvq_select_k(ev.data_ptr(), ev.numel(), float(lambda_loss), ctypes.byref(out)), "gvq_select_k")
    return out.value


PHASE_COLLECT, PHASE_COMPRESS = 0, 1
ACT_NONE, ACT_FIT, ACT_RESTART = 0, 1, 2


class Schedule:
    """gvq_schedule: the collect / fit / compress plan with the majority rule on Eq. 7's loss (host only)."""

    def __init__(self, L_t: int, L_c: int, n_nodes: int, loss_threshold: float):
        self._h = ctypes.c_void_p()
        _check(lib().gvq_schedule_create(ctypes.byref(self._h), L_t, L_c, n_nodes, float(loss_threshold)),
               "gvq_schedule_create")

    def close(self):
        if self._h:
            lib().gvq_schedule_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def phase(self) -> int:
        return lib().gvq_schedule_phase(self._h)

    @property
    def nodes_over(self) -> int:
        return lib().gvq_schedule_nodes_over(self._h)

    def step(self, monitor_host: Optional[torch.Tensor] = None) -> int:
        """Call after every iteration; monitor_host: None or a CPU float64 tensor [n_layers][2][n_nodes]."""
        action = ctypes.c_int(0)
        ptr, n_layers = None, 0
        if monitor_host is not None:
            assert monitor_host.dtype == torch.float64 and not monitor_host.is_cuda and monitor_host.is_contiguous()
            ptr, n_layers = monitor_host.data_ptr(), monitor_host.shape[0]
        _check(lib().gvq_schedule_step(self._h, ptr, n_layers, ctypes.byref(action)), "gvq_schedule_step")
        return action.value

    def counters(self):
        a, b, c = ctypes.c_int64(0), ctypes.c_int64(0), ctypes.c_int64(0)
        _check(lib().gvq_schedule_counters(self._h, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)),
               "gvq_schedule_counters")
        return {"iteration": a.value, "refreshes": b.value, "early_stops": c.value}


# the handle alone, without a Stream object around it (a tenth of the time), where this torch has it
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)

_F32 = torch.float32
DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _dtype(t: torch.Tensor) -> int:
    d = DTYPE.get(t.dtype)
    if d is None:
        raise TypeError(f"gvq takes float32, bfloat16 and float16 here, not {t.dtype}")
    return d


def _rows(t: torch.Tensor, device: int, what: str):
    """(rows, cols, leading dimension) of a 2-D tensor on that CUDA device whose rows are contiguous."""
    shape = t.shape
    if len(shape) != 2 or t.get_device() != device:
        raise ValueError(f"{what}: a 2-D tensor on cuda:{device} is wanted")
    rows, cols = shape
    ld, step = t.stride()
    if cols > 1 and step != 1:
        raise ValueError(f"{what}: the entries of a row have to be contiguous")
    return rows, cols, ld if rows > 1 else cols


class Mx4:
    """A matrix [rows][cols] in microscaled 4-bit floating point: device bytes `codes` and `scales` (see gvq.h)."""

    __slots__ = ("rows", "cols", "device", "_codes", "_scales", "_buf", "codes_ptr", "scales_ptr")

    def __init__(self, rows: int, cols: int, codes: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None,
                 device=None):
        rows, cols = int(rows), int(cols)
        nb = (cols + 31) // 32
        tiles = ((rows + 127) // 128) * ((nb + 3) // 4)
        if rows < 1 or cols < 1 or tiles >= 0x7FFFFFFF:
            raise ValueError(f"no 4-bit matrix of {rows} x {cols}")
        self.rows, self.cols = rows, cols
        if codes is None and scales is None:       # one allocation for both
            at = (rows * nb * 16 + 255) & ~255
            self._buf = buf = torch.empty(at + tiles * 512, dtype=torch.uint8, device=device or "cuda")
            self._codes = None
            self.device = buf.get_device()
            self.codes_ptr = p = buf.data_ptr()
            self.scales_ptr = p + at
            return
        if codes is None or scales is None:
            raise ValueError("codes and scales come together")
        nc, ns = self._sizes()
        for t, n in ((codes, nc), (scales, ns)):
            if t.dtype != torch.uint8 or not t.is_cuda or not t.is_contiguous() or t.numel() < n:
                raise ValueError(f"a 4-bit matrix of {rows} x {cols} has {nc} bytes of codes and {ns} of scales, contiguous")
        self.device = codes.get_device()
        if scales.get_device() != self.device:
            raise ValueError("codes and scales are on one device")
        self._codes, self._scales = codes, scales
        self.codes_ptr, self.scales_ptr = codes.data_ptr(), scales.data_ptr()

    def _sizes(self):
        """Bytes of codes and of scales."""
        nb = (self.cols + 31) // 32
        return self.rows * nb * 16, ((self.rows + 127) // 128) * ((nb + 3) // 4) * 512

    def _views(self):
        if self._codes is None:
            nc, ns = self._sizes()
            at = self.scales_ptr - self.codes_ptr
            self._codes, self._scales = self._buf[:nc], self._buf[at:at + ns]
        return self._codes, self._scales

    @property
    def codes(self) -> torch.Tensor:
        return self._views()[0]

    @property
    def scales(self) -> torch.Tensor:
        return self._views()[1]


class Context:
    """gvq_ctx for one layout on one CUDA device."""

    def __init__(self, layout, device: Optional[int] = None):
        self.layout = layout if isinstance(layout, HostLayout) else HostLayout.of(layout)
        if not torch.cuda.is_available():
            raise RuntimeError("gvq needs a CUDA device (there is no CPU fallback)")
        self.device = torch.cuda.current_device() if device is None else int(device)
        self._h = ctypes.c_void_p()
        st = lib().gvq_create(ctypes.byref(self._h), ctypes.byref(self.layout.c), self.device, self._stream())
        _check(st, "gvq_create")
        self.d, self.k = self.layout.d, self.layout.k
        self.S = self.layout.total_slices()
        self.M = self.layout.total_entries()
        self.n_layers = len(self.layout.layer_len)
        self._ws = None

    def _stream(self):
        return ctypes.c_void_p(torch.cuda.current_stream(self.device).cuda_stream)

    def _raw_stream(self) -> int:
        if _current_raw_stream is not None:
            return _current_raw_stream(self.device)
        return torch.cuda.current_stream(self.device).cuda_stream

    def _sync_stream(self):
        """Hands the current stream over.  The library knows which one it has; a copy of that kept here would go stale when
        somebody else sets it."""
        status = lib().gvq_set_stream(self._h, self._raw_stream())
        if status:
            raise GvqError(status, "gvq_set_stream")

    def close(self):
        if self._h:
            lib().gvq_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_projection_path(self, path: int):
        _check(lib().gvq_set_projection_path(self._h, path), "gvq_set_projection_path")

    def set_fit_path(self, path: int):
        _check(lib().gvq_set_fit_path(self._h, path), "gvq_set_fit_path")

    def set_limits(self, max_sweeps: int = 0, wait_cycles: int = 0):
        """gvq_set_limits (testing hook): 0 restores a default."""
        _check(lib().gvq_set_limits(self._h, int(max_sweeps), int(wait_cycles)), "gvq_set_limits")

    def test_drop_load(self, on: bool):
        _check(lib().gvq_test_drop_load(self._h, 1 if on else 0), "gvq_test_drop_load")

    def device_status(self):
        self._sync_stream()
        _check(lib().gvq_device_status(self._h), "gvq_device_status")

    def set_workspace(self, ws: Optional[torch.Tensor]):
        self._ws = ws
        if ws is None:
            _check(lib().gvq_set_workspace(self._h, None, 0), "gvq_set_workspace")
        else:
            _check(lib().gvq_set_workspace(self._h, ws.data_ptr(), ws.numel() * ws.element_size()),
                   "gvq_set_workspace")

    def ensure_workspace(self, nbytes: int):
        if self._ws is None or self._ws.numel() < nbytes:
            self.set_workspace(torch.empty(max(nbytes, 256), dtype=torch.uint8, device=f"cuda:{self.device}"))

    # ---- hot path -------------------------------------------------------------------------
    def compress(self, g_node, Ut, mu, N, s_node):
        self._sync_stream()
        _check(lib().gvq_compress(self._h, g_node.data_ptr(), Ut.data_ptr(), mu.data_ptr(), N, s_node.data_ptr()),
               "gvq_compress")

    def aggregate(self, s_nodes, s_sum):
        self._sync_stream()
        _check(lib().gvq_aggregate(self._h, _ptr_array(s_nodes), len(s_nodes), s_sum.data_ptr()), "gvq_aggregate")

    def compress_aggregate(self, g_nodes, Ut, mu, s_sum, s_nodes=None):
        self._sync_stream()
        sn = _ptr_array(s_nodes) if s_nodes is not None else None
        _check(lib().gvq_compress_aggregate(self._h, _ptr_array(g_nodes), len(g_nodes), Ut.data_ptr(),
                                            mu.data_ptr(), s_sum.data_ptr(), sn), "gvq_compress_aggregate")

    def compress_aggregate_partial(self, g_nodes, N, Ut, mu, x):
        self._sync_stream()
        _check(lib().gvq_compress_aggregate_partial(self._h, _ptr_array(g_nodes), len(g_nodes), N, Ut.data_ptr(),
                                                    mu.data_ptr(), x.data_ptr()), "gvq_compress_aggregate_partial")

    def exchange_accumulate(self, x_acc, x_in):
        self._sync_stream()
        _check(lib().gvq_exchange_accumulate(self._h, x_acc.data_ptr(), x_in.data_ptr()), "gvq_exchange_accumulate")

    def decompress_exchanged(self, x, Ut, mu, g_hat):
        self._sync_stream()
        _check(lib().gvq_decompress_exchanged(self._h, x.data_ptr(), Ut.data_ptr(), mu.data_ptr(), g_hat.data_ptr()),
               "gvq_decompress_exchanged")

    def quantize_raw4(self, g_node, levels, seed, node, q4, norms):
        self._sync_stream()
        _check(lib().gvq_quantize_raw4(self._h, g_node.data_ptr(), levels, seed, node, q4.data_ptr(), norms.data_ptr()),
               "gvq_quantize_raw4")

    def quantize_raw4_aggregate(self, g_nodes, levels, seed, g_sum, q4_nodes=None, norms_nodes=None):
        self._sync_stream()
        qp = _ptr_array(q4_nodes) if q4_nodes is not None else None
        npp = _ptr_array(norms_nodes) if norms_nodes is not None else None
        _check(lib().gvq_quantize_raw4_aggregate(self._h, _ptr_array(g_nodes), len(g_nodes), levels, seed,
                                                 g_sum.data_ptr(), qp, npp), "gvq_quantize_raw4_aggregate")

    def dequantize_raw4_aggregate(self, q4_nodes, norms_nodes, g_nodes_for_tails, levels, g_sum):
        self._sync_stream()
        gp = _ptr_array(g_nodes_for_tails) if g_nodes_for_tails is not None else None
        _check(lib().gvq_dequantize_raw4_aggregate(self._h, _ptr_array(q4_nodes), _ptr_array(norms_nodes), gp, levels,
                                                   len(q4_nodes), g_sum.data_ptr()), "gvq_dequantize_raw4_aggregate")

    # ---- microscaled 4-bit floating point ---------------------------------------------------
    def _mx4(self, x, by_rows, by_cols, stochastic, seed, node, out=None, out_t=None):
        rows, cols, ld = _rows(x, self.device, "mx4_quantize")
        dtype = _dtype(x)
        c = s = ct = st = None
        if by_rows:
            if out is None:
                out = Mx4(rows, cols, device=x.device)
            elif out.rows != rows or out.cols != cols or out.device != self.device:
                raise ValueError("mx4_quantize: the output is of another size or on another device")
            c, s = out.codes_ptr, out.scales_ptr
        if by_cols:
            if out_t is None:
                out_t = Mx4(cols, rows, device=x.device)
            elif out_t.rows != cols or out_t.cols != rows or out_t.device != self.device:
                raise ValueError("mx4_quantize: the output is of another size or on another device")
            ct, st = out_t.codes_ptr, out_t.scales_ptr
        self._sync_stream()
        status = lib().gvq_mx4_quantize(self._h, x.data_ptr(), dtype, rows, cols, ld, 1 if stochastic else 0, seed, node, c, s,
                                        ct, st)
        if status:
            raise GvqError(status, "gvq_mx4_quantize")
        return out, out_t

    def mx4_quantize(self, x, stochastic=False, seed=0, node=0, out: Optional[Mx4] = None) -> Mx4:
        """gvq_mx4_quantize along the rows of x [rows, cols]."""
        return self._mx4(x, True, False, stochastic, seed, node, out=out)[0]

    def mx4_quantize_transposed(self, x, stochastic=False, seed=0, node=0, out: Optional[Mx4] = None) -> Mx4:
        """gvq_mx4_quantize along the columns of x: the quantized [cols, rows] matrix."""
        return self._mx4(x, False, True, stochastic, seed, node, out_t=out)[1]

    def mx4_quantize_both(self, x, stochastic=False, seed=0, node=0, out: Optional[Mx4] = None,
                          out_t: Optional[Mx4] = None):
        """gvq_mx4_quantize along the rows and along the columns, reading x once: (by rows, by columns)."""
        return self._mx4(x, True, True, stochastic, seed, node, out, out_t)

    def mx4_dequantize(self, q: Mx4, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """gvq_mx4_dequantize: what q stands for, float32 [rows, cols]."""
        if out is None:
            out = torch.empty((q.rows, q.cols), device=f"cuda:{self.device}")
        rows, cols, ld = _rows(out, self.device, "mx4_dequantize")
        if (rows, cols) != (q.rows, q.cols) or out.dtype != torch.float32 or q.device != self.device:
            raise ValueError("mx4_dequantize: a float32 output of the matrix's size, on its device, is wanted")
        self._sync_stream()
        _check(lib().gvq_mx4_dequantize(self._h, q.codes_ptr, q.scales_ptr, rows, cols, out.data_ptr(), ld),
               "gvq_mx4_dequantize")
        return out

    def mx4_matmul(self, a: Mx4, b: Mx4, out: torch.Tensor) -> torch.Tensor:
        """gvq_mx4_matmul: out [a.rows, b.rows] = a b^T; out is float32, bfloat16 or float16."""
        rows, cols, ld = _rows(out, self.device, "mx4_matmul")
        if a.cols != b.cols or (rows, cols) != (a.rows, b.rows):
            raise ValueError(f"mx4_matmul: [{a.rows}, {a.cols}] x [{b.rows}, {b.cols}]^T does not give [{rows}, {cols}]")
        if a.device != self.device or b.device != self.device:
            raise ValueError(f"mx4_matmul: operands on cuda:{a.device} and cuda:{b.device}, the context on cuda:{self.device}")
        self._sync_stream()
        status = lib().gvq_mx4_matmul(self._h, a.codes_ptr, a.scales_ptr, b.codes_ptr, b.scales_ptr, rows, cols, a.cols,
                                      out.data_ptr(), _dtype(out), ld)
        if status:
            raise GvqError(status, "gvq_mx4_matmul")
        return out

    def _flat(self, t: torch.Tensor, what: str):
        if t.get_device() != self.device or not t.is_contiguous() or t.numel() < self.M:
            raise ValueError(f"{what}: a contiguous tensor of {self.M} entries on cuda:{self.device} is wanted")
        return t.data_ptr()

    def _flat_fp32(self, t: torch.Tensor, what: str):
        if t.dtype is not _F32:
            raise TypeError(f"{what}: float32 is wanted, not {t.dtype}")
        return self._flat(t, what)

    def _flats(self, tensors, what: str):
        M, device = self.M, self.device
        for t in tensors:
            if t.dtype is not _F32 or t.get_device() != device or t.numel() < M or not t.is_contiguous():
                self._flat_fp32(t, what)
        return _ptr_array(tensors)

    def _slices(self, q_nodes: Sequence[Mx4], n: int, what: str):
        """(codes, scales) of one [S][d] matrix per node, as host arrays."""
        if len(q_nodes) != n:
            raise ValueError(f"{what}: one 4-bit matrix per node is wanted ({n}), not {len(q_nodes)}")
        for q in q_nodes:
            if q.rows != self.S or q.cols != self.d or q.device != self.device:
                raise ValueError(f"{what}: a node's slices are {self.S} x {self.d} on cuda:{self.device}, "
                                 f"not {q.rows} x {q.cols} on cuda:{q.device}")
        vpn = ctypes.c_void_p * n
        return vpn(*[q.codes_ptr for q in q_nodes]), vpn(*[q.scales_ptr for q in q_nodes])

    def mx4_slices(self) -> Mx4:
        """Room for one node's quantized slices, a matrix [S][d]."""
        return Mx4(self.S, self.d, device=f"cuda:{self.device}")

    def mx4_quantize_aggregate(self, g_nodes, g_sum, stochastic=True, seed=0, node0=0,
                               out: Optional[Sequence[Mx4]] = None):
        """gvq_mx4_quantize_aggregate; out: one mx4_slices() per node that receives what it would send."""
        what = "gvq_mx4_quantize_aggregate"
        n = len(g_nodes)
        cp, sp = self._slices(out, n, what) if out is not None else (None, None)
        gp, total = self._flats(g_nodes, what), self._flat_fp32(g_sum, what) if g_sum is not None else None
        self._sync_stream()
        _check(lib().gvq_mx4_quantize_aggregate(self._h, gp, n, node0, 1 if stochastic else 0, seed, total, cp, sp), what)

    def mx4_dequantize_aggregate(self, q_nodes: Sequence[Mx4], g_nodes_for_tails, g_sum):
        """gvq_mx4_dequantize_aggregate; g_nodes_for_tails: the same nodes' gradients, or None for a layout without tails."""
        what = "gvq_mx4_dequantize_aggregate"
        n = len(q_nodes)
        cp, sp = self._slices(q_nodes, n, what)
        if g_nodes_for_tails is not None and len(g_nodes_for_tails) != n:
            raise ValueError(f"{what}: one gradient per node is wanted ({n}), not {len(g_nodes_for_tails)}")
        gp = self._flats(g_nodes_for_tails, what) if g_nodes_for_tails is not None else None
        total = self._flat_fp32(g_sum, what)
        self._sync_stream()
        _check(lib().gvq_mx4_dequantize_aggregate(self._h, cp, sp, gp, n, total), what)

    def flatten_layer(self, framework, flat, F, D, X):
        self._sync_stream()
        _check(lib().gvq_flatten_layer(self._h, framework.data_ptr(), flat.data_ptr(), F, D, X), "gvq_flatten_layer")

    def unflatten_layer(self, flat, framework, F, D, X):
        self._sync_stream()
        _check(lib().gvq_unflatten_layer(self._h, flat.data_ptr(), framework.data_ptr(), F, D, X), "gvq_unflatten_layer")

    def mask_basis(self, Ut, k_per_layer):
        ks = (ctypes.c_int32 * self.n_layers)(*[int(x) for x in k_per_layer])
        self._sync_stream()
        _check(lib().gvq_mask_basis(self._h, Ut.data_ptr(), ks), "gvq_mask_basis")

    def set_layer_k(self, k_per_layer):
        """gvq_set_layer_k: per-layer compressed lengths for exchange_pack / exchange_unpack (None = all k)."""
        self._sync_stream()
        ks = None if k_per_layer is None else (ctypes.c_int32 * self.n_layers)(*[int(x) for x in k_per_layer])
        _check(lib().gvq_set_layer_k(self._h, ks), "gvq_set_layer_k")

    def exchange_pack(self, x, x_packed):
        self._sync_stream()
        _check(lib().gvq_exchange_pack(self._h, x.data_ptr(), x_packed.data_ptr()), "gvq_exchange_pack")

    def exchange_unpack(self, x_packed, x):
        self._sync_stream()
        _check(lib().gvq_exchange_unpack(self._h, x_packed.data_ptr(), x.data_ptr()), "gvq_exchange_unpack")

    def compress_aggregate_monitored(self, g_nodes, Ut, mu, s_sum, monitor, s_nodes=None):
        self._sync_stream()
        sn = _ptr_array(s_nodes) if s_nodes is not None else None
        _check(lib().gvq_compress_aggregate_monitored(self._h, _ptr_array(g_nodes), len(g_nodes), Ut.data_ptr(),
                                                      mu.data_ptr(), s_sum.data_ptr(), sn, monitor.data_ptr()),
               "gvq_compress_aggregate_monitored")

    def compress_quantize_aggregate(self, g_nodes, Ut, mu, levels, seed, s_sum, q_nodes=None, norms_nodes=None):
        self._sync_stream()
        qp = _ptr_array(q_nodes) if q_nodes is not None else None
        npp = _ptr_array(norms_nodes) if norms_nodes is not None else None
        _check(lib().gvq_compress_quantize_aggregate(self._h, _ptr_array(g_nodes), len(g_nodes), Ut.data_ptr(),
                                                     mu.data_ptr(), levels, seed, s_sum.data_ptr(), qp, npp),
               "gvq_compress_quantize_aggregate")

    def decompress(self, s_sum, Ut, mu, g_nodes_for_tails, N, g_hat):
        self._sync_stream()
        gp = _ptr_array(g_nodes_for_tails) if g_nodes_for_tails is not None else None
        _check(lib().gvq_decompress(self._h, s_sum.data_ptr(), Ut.data_ptr(), mu.data_ptr(), gp, N,
                                    g_hat.data_ptr()), "gvq_decompress")

    def fit_basis(self, hist, N, samples_are_sums_of, Ut, mu, evals):
        """Returns the per-layer sweep counts (host list)."""
        self._sync_stream()
        L = hist.shape[0]
        self.ensure_workspace(self.layout.fit_workspace_bytes(L))
        info = (ctypes.c_int32 * self.n_layers)()
        st = lib().gvq_fit_basis(self._h, hist.data_ptr(), hist.stride(0) if L > 1 else hist.shape[1], L, N,
                                 samples_are_sums_of, Ut.data_ptr(), mu.data_ptr(), evals.data_ptr(), info)
        _check(st, "gvq_fit_basis")
        return list(info)

    def fit_centre(self, hist, centre):
        """gvq_fit_centre: the point per layer that a fit spread over participants centres by."""
        self._sync_stream()
        L = hist.shape[0]
        _check(lib().gvq_fit_centre(self._h, hist.data_ptr(), hist.stride(0) if L > 1 else hist.shape[1], L,
                                    centre.data_ptr()), "gvq_fit_centre")

    def fit_moments(self, hist, centre, moments):
        """gvq_fit_moments: this participant's additive moments (fp64 [fit_moments_count]) about `centre`."""
        self._sync_stream()
        L = hist.shape[0]
        self.ensure_workspace(self.layout.fit_workspace_bytes(L))
        _check(lib().gvq_fit_moments(self._h, hist.data_ptr(), hist.stride(0) if L > 1 else hist.shape[1], L,
                                     centre.data_ptr(), moments.data_ptr()), "gvq_fit_moments")

    def fit_from_moments(self, moments, centre, N, samples_are_sums_of, Ut, mu, evals):
        """gvq_fit_from_moments: the fit from the summed moments.  Returns the per-layer sweep counts."""
        self._sync_stream()
        self.ensure_workspace(self.layout.fit_workspace_bytes(1))
        info = (ctypes.c_int32 * self.n_layers)()
        _check(lib().gvq_fit_from_moments(self._h, moments.data_ptr(), centre.data_ptr(), N, samples_are_sums_of,
                                          Ut.data_ptr(), mu.data_ptr(), evals.data_ptr(), info), "gvq_fit_from_moments")
        return list(info)

    def refresh_basis(self, hist, N, samples_are_sums_of, Ut, mu, evals_k, trace, iters=6, warm_start=True):
        """gvq_refresh_basis: the k leading eigenpairs by subspace iteration (Ut is read when warm_start)."""
        self._sync_stream()
        L = hist.shape[0]
        self.ensure_workspace(self.layout.fit_workspace_bytes(L))
        st = lib().gvq_refresh_basis(self._h, hist.data_ptr(), hist.stride(0) if L > 1 else hist.shape[1], L, N,
                                     samples_are_sums_of, 1 if warm_start else 0, iters, Ut.data_ptr(), mu.data_ptr(),
                                     evals_k.data_ptr(), trace.data_ptr())
        _check(st, "gvq_refresh_basis")

    def fit_basis_static(self, hist, N, samples_are_sums_of, Ut, mu, evals):
        """gvq_fit_basis_static: the same fit, with the library's built-in scratch array instead of a
        workspace -- for callers that cannot allocate device memory.  Returns the sweep counts."""
        self._sync_stream()
        L = hist.shape[0]
        info = (ctypes.c_int32 * self.n_layers)()
        st = lib().gvq_fit_basis_static(self._h, hist.data_ptr(), hist.stride(0) if L > 1 else hist.shape[1], L, N,
                                        samples_are_sums_of, Ut.data_ptr(), mu.data_ptr(), evals.data_ptr(), info)
        _check(st, "gvq_fit_basis_static")
        return list(info)

    def quantize(self, s_node, levels, seed, node, q, norms):
        self._sync_stream()
        _check(lib().gvq_quantize(self._h, s_node.data_ptr(), levels, seed, node, q.data_ptr(), norms.data_ptr()),
               "gvq_quantize")

    def quantize_aggregate(self, s_nodes, levels, seed, s_sum, q_nodes=None, norms_nodes=None):
        self._sync_stream()
        qp = _ptr_array(q_nodes) if q_nodes is not None else None
        npp = _ptr_array(norms_nodes) if norms_nodes is not None else None
        _check(lib().gvq_quantize_aggregate(self._h, _ptr_array(s_nodes), len(s_nodes), levels, seed, s_sum.data_ptr(),
                                            qp, npp), "gvq_quantize_aggregate")

    def dequantize_aggregate(self, q_nodes, norms_nodes, levels, s_sum):
        self._sync_stream()
        _check(lib().gvq_dequantize_aggregate(self._h, _ptr_array(q_nodes), _ptr_array(norms_nodes), levels,
                                              len(q_nodes), s_sum.data_ptr()), "gvq_dequantize_aggregate")

    def host_prepare(self):
        """gvq_host_prepare: builds the chunk pipeline of allreduce_host once (outside the training loop)."""
        _check(lib().gvq_host_prepare(self._h), "gvq_host_prepare")

    def allreduce_host(self, g_nodes_host, Ut, mu, g_hat_host, levels: int = 0, seed: int = 0):
        """g_nodes_host: CPU tensors (pinned for speed); Ut, mu: device; g_hat_host: CPU tensor.
        levels > 0: gvq_allreduce_host_quantized."""
        self._sync_stream()
        self.ensure_workspace(self.layout.host_workspace_bytes(len(g_nodes_host)))
        if levels > 0:
            _check(lib().gvq_allreduce_host_quantized(self._h, _ptr_array(g_nodes_host), len(g_nodes_host), Ut.data_ptr(),
                                                      mu.data_ptr(), levels, seed, g_hat_host.data_ptr()),
                   "gvq_allreduce_host_quantized")
        else:
            _check(lib().gvq_allreduce_host(self._h, _ptr_array(g_nodes_host), len(g_nodes_host), Ut.data_ptr(),
                                            mu.data_ptr(), g_hat_host.data_ptr()), "gvq_allreduce_host")


class OrthoPlan:
    """gvq_ortho: the orthogonalised update of a context's layers that are matrices, rows[l] x cols[l] (0, 0: not one).

    scales: the update's factor of each layer.  None: sqrt(max(1, outputs / inputs)), a layer's outputs being its rows
    (W[out][in]), or its columns where `flattened` says that layers are in gvq_flatten_layer's order, [inputs][filters]
    (one truth value for all layers or one for each)."""

    def __init__(self, ctx: Context, rows: Sequence[int], cols: Sequence[int], scales: Optional[Sequence[float]] = None,
                 flattened=False):
        self._h = ctypes.c_void_p()
        n = ctx.n_layers
        if len(rows) != n or len(cols) != n or (scales is not None and len(scales) != n):
            raise ValueError(f"OrthoPlan: one entry per layer is wanted ({n})")
        if scales is None and flattened is not False:
            order = [bool(flattened)] * n if isinstance(flattened, (bool, int)) else list(flattened)
            if len(order) != n:
                raise ValueError(f"OrthoPlan: one entry per layer is wanted ({n})")
            scales = [math.sqrt(max(1.0, (v / u if f else u / v) if u and v else 1.0)) for u, v, f in zip(rows, cols, order)]
        elif flattened is not False:
            raise ValueError("OrthoPlan: scales are given, so the layers' order has no use")
        self.ctx = ctx                       # the plan uses its stream and must not outlive it
        r, c = (ctypes.c_int32 * n)(*[int(v) for v in rows]), (ctypes.c_int32 * n)(*[int(v) for v in cols])
        nbytes = lib().gvq_ortho_workspace_bytes(ctypes.byref(ctx.layout.c), r, c)
        if nbytes < 0:
            raise GvqError(2, "gvq_ortho_workspace_bytes")
        self._ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=f"cuda:{ctx.device}")
        s = None if scales is None else (ctypes.c_float * n)(*[float(v) for v in scales])
        _check(lib().gvq_ortho_create(ctypes.byref(self._h), ctx._h, r, c, s, self._ws.data_ptr(), self._ws.numel()),
               "gvq_ortho_create")

    def close(self):
        if self._h:
            lib().gvq_ortho_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _ready(self, what: str):
        """The plan's calls use its context, which may have been closed before it: the library cannot tell."""
        if not self._h or not self.ctx._h:
            raise GvqError(1, what)
        self.ctx._sync_stream()

    def step(self, g, momentum, w, lr: float, weight_decay: float = 0.0, beta: float = 0.95, nesterov: bool = True):
        """gvq_ortho_step on flat buffers: momentum and w are updated in place."""
        self._ready("gvq_ortho_step")
        _check(lib().gvq_ortho_step(self._h, self.ctx._flat_fp32(g, "g"), self.ctx._flat_fp32(momentum, "momentum"), beta,
                                    1 if nesterov else 0, self.ctx._flat(w, "w"), _dtype(w), lr, weight_decay), "gvq_ortho_step")

    def orthogonalize(self, g, out):
        """gvq_orthogonalize: the plan's matrices of the flat buffer g, orthogonalised, into `out`."""
        self._ready("gvq_orthogonalize")
        _check(lib().gvq_orthogonalize(self._h, self.ctx._flat_fp32(g, "g"), self.ctx._flat(out, "out"), _dtype(out)),
               "gvq_orthogonalize")
