"""Thin ctypes binding of libqg.so (declared in include/qg.h).

Argument marshalling only: every step of the path runs in the HIP kernels of the library.
PyTorch supplies device memory and the current stream, nothing else.  There is no fallback:
if the library cannot be loaded or a call returns an error, a RuntimeError is raised.
"""
import ctypes
import os
import struct
from typing import List, Optional, Sequence, Tuple

import torch

from . import build as _build

QG_LAYOUT_CANONICAL = 0
QG_LAYOUT_DEVICE = 1
QG_LAYOUT_DEVICE_NARROW = 2
QG_MAX_GROUPED = 16
QG_F32, QG_BF16, QG_F16, QG_E4M3 = range(4)
QG_MAX_PLANES = 8

_LIB = None


class _Desc(ctypes.Structure):
    _fields_ = [("packed", ctypes.c_void_p), ("N", ctypes.c_int64), ("K", ctypes.c_int64),
                ("bits", ctypes.c_int), ("group", ctypes.c_int),
                ("x", ctypes.c_void_p), ("y", ctypes.c_void_p)]


def lib():
    """Load libqg.so, building it first only if no built library is present; a library that
    was built from other sources than the ones in csrc/ is refused (RuntimeError)."""
    global _LIB
    if _LIB is None:
        override = os.environ.get("QG_LIBRARY")             # a library built elsewhere: used as it is
        path = override or _build.OUT
        if not os.path.exists(path):
            path = _build.build(force=True)
        L = ctypes.CDLL(path)
        if not override:
            # a library built from other sources than the ones beside it is not used silently
            L.qg_build_id.restype = ctypes.c_char_p
            built_from = L.qg_build_id().decode() if hasattr(L, "qg_build_id") else "none"
            if built_from != _build.source_id():
                raise RuntimeError(f"{path} is stale (built from {built_from}, sources are "
                                   f"{_build.source_id()}): run `python -m paper_2307_03738_amd.build`")
        i64, i32, vp, sz = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
        L.qg_cell.restype = i32
        L.qg_cell.argtypes = [i32]
        L.qg_build_id.restype = ctypes.c_char_p
        L.qg_build_id.argtypes = []
        L.qg_status_string.restype = ctypes.c_char_p
        L.qg_status_string.argtypes = [i32]
        L.qg_packed_bytes.restype = sz
        L.qg_packed_bytes.argtypes = [i64, i64, i32, i32, i32]
        L.qg_workspace_bytes.restype = sz
        L.qg_workspace_bytes.argtypes = [i64, i64, i32, i32, i32]
        L.qg_workspace_init.restype = i32
        L.qg_workspace_init.argtypes = [vp, sz, vp]
        L.qg_quantize.restype = i32
        L.qg_quantize.argtypes = [vp, i64, i64, i32, i32, vp, vp, vp, vp]
        L.qg_pack.restype = i32
        L.qg_pack.argtypes = [vp, vp, vp, i64, i64, i32, i32, i32, vp, vp]
        L.qg_unpack.restype = i32
        L.qg_unpack.argtypes = [vp, i64, i64, i32, i32, i32, vp, vp, vp, vp]
        L.qg_gemv.restype = i32
        L.qg_gemv.argtypes = [vp, i64, i64, i32, i32, vp, vp, vp, sz, vp]
        L.qg_gemv_noalloc.restype = i32
        L.qg_gemv_noalloc.argtypes = [vp, i64, i64, i32, i32, vp, vp, vp]
        L.qg_last_gemv_kernel.restype = ctypes.c_char_p
        L.qg_last_gemv_kernel.argtypes = []
        L.qg_gemv_grouped.restype = i32
        L.qg_gemv_grouped.argtypes = [ctypes.POINTER(_Desc), i32, vp, sz, vp]
        L.qg_gemv_swiglu.restype = i32
        L.qg_gemv_swiglu.argtypes = [vp, i64, i64, i32, i32, vp, vp, vp, sz, vp]
        L.qg_gemm_small.restype = i32
        L.qg_gemm_small.argtypes = [vp, i64, i64, i32, i32, vp, i32, vp, vp, sz, vp]
        L.qg_set_gemv_tuning.restype = i32
        L.qg_set_gemv_tuning.argtypes = [i32, i32, i32]
        L.qg_gemv_autotune.restype = i32
        L.qg_gemv_autotune.argtypes = [ctypes.POINTER(_Desc), i32, i32, vp, sz, vp, i32,
                                       ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i32),
                                       ctypes.POINTER(ctypes.c_float)]
        L.qg_gemv_autotune_report.restype = i32
        L.qg_gemv_autotune_report.argtypes = [ctypes.POINTER(ctypes.c_float), i32, ctypes.POINTER(i32), ctypes.POINTER(i32)]
        L.qg_set_gemm_tuning.restype = i32
        L.qg_set_gemm_tuning.argtypes = [i32, i32]
        L.qg_to_narrow.restype = i32
        L.qg_to_narrow.argtypes = [vp, i64, i64, i32, i32, vp, vp]
        L.qg_from_narrow.restype = i32
        L.qg_from_narrow.argtypes = [vp, i64, i64, i32, i32, vp, vp]
        L.qg_gemv_narrow.restype = i32
        L.qg_gemv_narrow.argtypes = [vp, i64, i64, i32, i32, vp, vp, vp]
        L.qg_gemv_grouped_narrow.restype = i32
        L.qg_gemv_grouped_narrow.argtypes = [ctypes.POINTER(_Desc), i32, vp]
        L.qg_set_narrow_tuning.restype = i32
        L.qg_set_narrow_tuning.argtypes = [i32]
        L.qg_last_narrow_kernel.restype = ctypes.c_char_p
        L.qg_last_narrow_kernel.argtypes = []
        L.qg_gemv_record_tuning.restype = i32
        L.qg_gemv_record_tuning.argtypes = [ctypes.POINTER(_Desc), i32, i32, i32, i32]
        L.qg_clear_tuning.restype = None
        L.qg_clear_tuning.argtypes = []
        L.qg_gemm_autotune.restype = i32
        L.qg_gemm_autotune.argtypes = [ctypes.POINTER(vp), i32, i64, i64, i32, i32, vp, i32, vp, vp, sz, vp, i32,
                                       ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(ctypes.c_float)]
        L.qg_gemm_autotune_report.restype = i32
        L.qg_gemm_autotune_report.argtypes = [ctypes.POINTER(ctypes.c_float), i32, ctypes.POINTER(i32), ctypes.POINTER(i32)]
        cp = ctypes.c_char_p                                # a description packed by value
        L.qg_rms_norm.restype = i32
        L.qg_rms_norm.argtypes = [cp, vp]
        L.qg_kv_append.restype = i32
        L.qg_kv_append.argtypes = [cp, vp]
        L.qg_paged_attention.restype = i32
        L.qg_paged_attention.argtypes = [cp, vp]
        L.qg_paged_attention_workspace_bytes.restype = sz
        L.qg_paged_attention_workspace_bytes.argtypes = [i32, i32, i32, i32]
        L.qg_pages_resize.restype = i32
        L.qg_pages_resize.argtypes = [cp, vp, cp, i32, vp, vp, sz, vp]
        L.qg_pages_fork.restype = i32
        L.qg_pages_fork.argtypes = [cp, vp, vp]
        L.qg_pages_compact.restype = i32
        L.qg_pages_compact.argtypes = [cp, cp, i32, vp, vp, sz, vp]
        L.qg_pages_copy.restype = i32
        L.qg_pages_copy.argtypes = [cp, i32, i64, vp, i32, vp]
        L.qg_pages_workspace_bytes.restype = sz
        L.qg_pages_workspace_bytes.argtypes = [i32, i32, i64]
        L.qg_route.restype = i32
        L.qg_route.argtypes = [cp, vp]
        L.qg_expert_plan.restype = i32
        L.qg_expert_plan.argtypes = [vp, i64, i32, i32, vp, vp, vp, vp]
        L.qg_experts_product.restype = i32
        L.qg_experts_product.argtypes = [cp, vp]
        L.qg_experts_workspace_bytes.restype = sz
        L.qg_experts_workspace_bytes.argtypes = [i64, i64, i32]
        L.qg_experts_combine.restype = i32
        L.qg_experts_combine.argtypes = [cp, vp]
        _LIB = L
    return _LIB


def _check(rc: int, what: str):
    if rc != 0:
        raise RuntimeError(f"{what}: {lib().qg_status_string(rc).decode()} (status {rc})")


# A small product takes 3 us on the GPU; its call took 8.4 us of host time, of which building a Stream
# object to read its handle and asking the library for a blob's size again were about a third
# (512 x 512 4-bit g64: 8.2 -> 5.6 us per call).
def _stream() -> int:
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _dev(t: torch.Tensor, dtype, name: str) -> torch.Tensor:
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor on the GPU")
    return t


# A new contiguous tensor (torch.empty takes 0.4 us more of the caller's time each; a conversion makes five).
def _rows(n: int, k: int, dtype, device) -> torch.Tensor:
    return torch.empty_strided((n, k), (k, 1), dtype=dtype, device=device)


def _bytes(n: int, device) -> torch.Tensor:
    return torch.empty_strided((n,), (1,), dtype=torch.uint8, device=device)


def qg_cell(bits: int) -> int:
    return int(lib().qg_cell(bits))


_SIZES = {}        # blob sizes, at most 1024 of them
_values = struct.Struct("5q").pack


def qg_packed_bytes(N: int, K: int, bits: int, group: int, layout: int = QG_LAYOUT_DEVICE) -> int:
    # remembered by the values the arguments have now (512.0, which is equal to 512, is refused; a tensor or
    # array of one number may change); what has none of 64 bits goes to the library as it is
    try:
        key = _values(N, K, bits, group, layout)
    except Exception:
        return int(lib().qg_packed_bytes(N, K, bits, group, layout))
    nbytes = _SIZES.get(key)
    if nbytes is None:
        if len(_SIZES) >= 1024:
            _SIZES.clear()
        nbytes = _SIZES[key] = int(lib().qg_packed_bytes(N, K, bits, group, layout))
    return nbytes


def qg_workspace_bytes(N: int, K: int, bits: int, group: int, M: int = 1) -> int:
    return int(lib().qg_workspace_bytes(N, K, bits, group, M))


def qg_workspace_init(workspace: torch.Tensor):
    _check(lib().qg_workspace_init(workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                   _stream()), "qg_workspace_init")


def new_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    """Allocate a workspace of at least nbytes and zero it with the library's own fill."""
    ws = torch.empty(max(256, (nbytes + 255) // 256 * 256), dtype=torch.uint8, device=device)
    qg_workspace_init(ws)
    return ws


def qg_quantize(W: torch.Tensor, bits: int, group: int) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    _dev(W, torch.float32, "W")
    N, K = W.shape
    if group <= 0 or K % group:
        _check(2, "qg_quantize")
    device = W.device
    q = _rows(N, K, torch.uint8, device)
    s = _rows(N, K // group, torch.float32, device)
    z = _rows(N, K // group, torch.uint8, device)
    _check(lib().qg_quantize(W.data_ptr(), N, K, bits, group, q.data_ptr(), s.data_ptr(), z.data_ptr(),
                             _stream()), "qg_quantize")
    return q, s, z


def qg_pack(q: torch.Tensor, s: torch.Tensor, z: torch.Tensor, bits: int, group: int,
            layout: int = QG_LAYOUT_DEVICE) -> torch.Tensor:
    _dev(q, torch.uint8, "q"); _dev(s, torch.float32, "s"); _dev(z, torch.uint8, "z")
    N, K = q.shape
    nbytes = qg_packed_bytes(N, K, bits, group, layout)
    if nbytes == 0:
        _check(2, "qg_pack")
    packed = _bytes(nbytes, q.device)
    _check(lib().qg_pack(q.data_ptr(), s.data_ptr(), z.data_ptr(), N, K, bits, group, layout,
                         packed.data_ptr(), _stream()), "qg_pack")
    return packed


def qg_unpack(packed: torch.Tensor, N: int, K: int, bits: int, group: int,
              layout: int = QG_LAYOUT_DEVICE) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    _dev(packed, torch.uint8, "packed")
    if packed.numel() < qg_packed_bytes(N, K, bits, group, layout) or group <= 0 or K % group:
        _check(2, "qg_unpack")
    device = packed.device
    q = _rows(N, K, torch.uint8, device)
    s = _rows(N, K // group, torch.float32, device)
    z = _rows(N, K // group, torch.uint8, device)
    _check(lib().qg_unpack(packed.data_ptr(), N, K, bits, group, layout, q.data_ptr(), s.data_ptr(),
                           z.data_ptr(), _stream()), "qg_unpack")
    return q, s, z


def qg_gemv(packed: torch.Tensor, N: int, K: int, bits: int, group: int, x: torch.Tensor,
            y: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    _dev(packed, torch.uint8, "packed"); _dev(x, torch.float32, "x")
    if x.numel() != K or packed.numel() < qg_packed_bytes(N, K, bits, group, QG_LAYOUT_DEVICE):
        _check(2, "qg_gemv")
    if y is None:
        y = torch.empty(N, dtype=torch.float32, device=x.device)
    if workspace is None:
        workspace = new_workspace(qg_workspace_bytes(N, K, bits, group, 1), x.device)
    rc = (_LIB or lib()).qg_gemv(packed.data_ptr(), N, K, bits, group, x.data_ptr(), y.data_ptr(),
                                 workspace.data_ptr(), workspace.numel(), _stream())
    if rc != 0:
        _check(rc, "qg_gemv")
    return y


def qg_gemv_noalloc(packed: torch.Tensor, N: int, K: int, bits: int, group: int, x: torch.Tensor,
                    y: torch.Tensor) -> torch.Tensor:
    """qg_gemv with the library's own scratch array: no workspace argument, nothing allocated
    by the call (y is the caller's)."""
    _dev(packed, torch.uint8, "packed"); _dev(x, torch.float32, "x"); _dev(y, torch.float32, "y")
    if x.numel() != K or y.numel() != N or packed.numel() < qg_packed_bytes(N, K, bits, group, QG_LAYOUT_DEVICE):
        _check(2, "qg_gemv_noalloc")
    _check(lib().qg_gemv_noalloc(packed.data_ptr(), N, K, bits, group, x.data_ptr(), y.data_ptr(), _stream()),
           "qg_gemv_noalloc")
    return y


def qg_to_narrow(packed: torch.Tensor, N: int, K: int, bits: int, group: int) -> torch.Tensor:
    """The narrow-layout copy of a QG_LAYOUT_DEVICE blob."""
    _dev(packed, torch.uint8, "packed")
    nbytes = qg_packed_bytes(N, K, bits, group, QG_LAYOUT_DEVICE_NARROW)
    if nbytes == 0:
        _check(3, "qg_to_narrow")
    if packed.numel() < qg_packed_bytes(N, K, bits, group, QG_LAYOUT_DEVICE):
        _check(2, "qg_to_narrow")
    out = _bytes(nbytes, packed.device)
    _check(lib().qg_to_narrow(packed.data_ptr(), N, K, bits, group, out.data_ptr(), _stream()), "qg_to_narrow")
    return out


def qg_from_narrow(narrow: torch.Tensor, N: int, K: int, bits: int, group: int) -> torch.Tensor:
    _dev(narrow, torch.uint8, "narrow")
    if narrow.numel() < qg_packed_bytes(N, K, bits, group, QG_LAYOUT_DEVICE_NARROW) or \
            qg_packed_bytes(N, K, bits, group, QG_LAYOUT_DEVICE_NARROW) == 0:
        _check(2, "qg_from_narrow")
    out = torch.empty(qg_packed_bytes(N, K, bits, group, QG_LAYOUT_DEVICE), dtype=torch.uint8, device=narrow.device)
    _check(lib().qg_from_narrow(narrow.data_ptr(), N, K, bits, group, out.data_ptr(), _stream()), "qg_from_narrow")
    return out


def qg_gemv_narrow(narrow: torch.Tensor, N: int, K: int, bits: int, group: int, x: torch.Tensor,
                   y: Optional[torch.Tensor] = None) -> torch.Tensor:
    _dev(narrow, torch.uint8, "narrow"); _dev(x, torch.float32, "x")
    nbytes = qg_packed_bytes(N, K, bits, group, QG_LAYOUT_DEVICE_NARROW)
    if nbytes == 0:
        _check(3, "qg_gemv_narrow")
    if x.numel() != K or narrow.numel() < nbytes:
        _check(2, "qg_gemv_narrow")
    if y is None:
        y = torch.empty(N, dtype=torch.float32, device=x.device)
    _dev(y, torch.float32, "y")
    if y.numel() != N:
        _check(2, "qg_gemv_narrow")
    _check(lib().qg_gemv_narrow(narrow.data_ptr(), N, K, bits, group, x.data_ptr(), y.data_ptr(), _stream()),
           "qg_gemv_narrow")
    return y


class GroupedGemvNarrow:
    """A prepared grouped launch on narrow-layout blobs (dicts with packed, N, K, bits, group, x, y)."""

    def __init__(self, problems: Sequence[dict]):
        self.count = len(problems)
        self.descs = (_Desc * self.count)()
        self._keep = list(problems)
        for i, p in enumerate(problems):
            _dev(p["packed"], torch.uint8, "packed"); _dev(p["x"], torch.float32, "x"); _dev(p["y"], torch.float32, "y")
            nbytes = qg_packed_bytes(p["N"], p["K"], p["bits"], p["group"], QG_LAYOUT_DEVICE_NARROW)
            if nbytes == 0:
                _check(3, "qg_gemv_grouped_narrow")
            if p["x"].numel() != p["K"] or p["y"].numel() != p["N"] or p["packed"].numel() < nbytes:
                _check(2, "qg_gemv_grouped_narrow")
            self.descs[i] = _Desc(p["packed"].data_ptr(), p["N"], p["K"], p["bits"], p["group"],
                                  p["x"].data_ptr(), p["y"].data_ptr())
        self._fn = lib().qg_gemv_grouped_narrow

    def launch(self, stream: Optional[int] = None):
        rc = self._fn(self.descs, self.count, _stream() if stream is None else stream)
        if rc != 0:
            _check(rc, "qg_gemv_grouped_narrow")


def qg_set_narrow_tuning(tiles_per_wave: int = 0):
    _check(lib().qg_set_narrow_tuning(tiles_per_wave), "qg_set_narrow_tuning")


def qg_last_narrow_kernel() -> str:
    return lib().qg_last_narrow_kernel().decode()


def qg_last_gemv_kernel() -> str:
    return lib().qg_last_gemv_kernel().decode()


class GroupedGemv:
    """A prepared grouped launch: the descriptor array is built once, launch() enqueues it."""

    def __init__(self, problems: Sequence[dict], workspace: Optional[torch.Tensor] = None):
        # problems: dicts with packed, N, K, bits, group, x, y
        self.count = len(problems)
        self.descs = (_Desc * self.count)()
        self._keep = list(problems)
        need = 0
        for i, p in enumerate(problems):
            _dev(p["packed"], torch.uint8, "packed"); _dev(p["x"], torch.float32, "x"); _dev(p["y"], torch.float32, "y")
            if p["x"].numel() != p["K"] or p["y"].numel() != p["N"] or \
                    p["packed"].numel() < qg_packed_bytes(p["N"], p["K"], p["bits"], p["group"]):
                _check(2, "qg_gemv_grouped")
            self.descs[i] = _Desc(p["packed"].data_ptr(), p["N"], p["K"], p["bits"], p["group"],
                                  p["x"].data_ptr(), p["y"].data_ptr())
            need += qg_workspace_bytes(p["N"], p["K"], p["bits"], p["group"], 1)
        self.workspace = workspace if workspace is not None else new_workspace(need, problems[0]["x"].device)
        self._fn = lib().qg_gemv_grouped

    def launch(self, stream: Optional[int] = None):
        rc = self._fn(self.descs, self.count, self.workspace.data_ptr(), self.workspace.numel(),
                      _stream() if stream is None else stream)
        if rc != 0:
            _check(rc, "qg_gemv_grouped")


def qg_gemv_grouped(problems: Sequence[dict], workspace: Optional[torch.Tensor] = None):
    GroupedGemv(problems, workspace).launch()
    return [p["y"] for p in problems]


def qg_gemv_swiglu(packed: torch.Tensor, I: int, K: int, bits: int, group: int, x: torch.Tensor,
                   h: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    _dev(packed, torch.uint8, "packed"); _dev(x, torch.float32, "x")
    if x.numel() != K or packed.numel() < qg_packed_bytes(2 * I, K, bits, group, QG_LAYOUT_DEVICE):
        _check(2, "qg_gemv_swiglu")
    if h is None:
        h = torch.empty(I, dtype=torch.float32, device=x.device)
    if workspace is None:
        workspace = new_workspace(qg_workspace_bytes(2 * I, K, bits, group, 1), x.device)
    _check(lib().qg_gemv_swiglu(packed.data_ptr(), I, K, bits, group, x.data_ptr(), h.data_ptr(),
                                workspace.data_ptr(), workspace.numel(), _stream()), "qg_gemv_swiglu")
    return h


def qg_gemm_small(packed: torch.Tensor, N: int, K: int, bits: int, group: int, X: torch.Tensor,
                  Y: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    _dev(packed, torch.uint8, "packed"); _dev(X, torch.float32, "X")
    M = X.shape[0]
    if X.dim() != 2 or X.shape[1] != K or packed.numel() < qg_packed_bytes(N, K, bits, group, QG_LAYOUT_DEVICE):
        _check(2, "qg_gemm_small")
    if Y is None:
        Y = torch.empty((M, N), dtype=torch.float32, device=X.device)
    if workspace is None:
        workspace = new_workspace(qg_workspace_bytes(N, K, bits, group, M), X.device)
    rc = (_LIB or lib()).qg_gemm_small(packed.data_ptr(), N, K, bits, group, X.data_ptr(), M, Y.data_ptr(),
                                       workspace.data_ptr(), workspace.numel(), _stream())
    if rc != 0:
        _check(rc, "qg_gemm_small")
    return Y


def qg_set_gemv_tuning(waves_per_block: int = 0, bytes_per_wave: int = 0, kernel: int = 0):
    _check(lib().qg_set_gemv_tuning(waves_per_block, bytes_per_wave, kernel), "qg_set_gemv_tuning")


def qg_gemv_autotune(launches, repeats: int = 20):
    """Times the candidates on the prepared launch(es) -- a GroupedGemv or a list of them with the
    same shapes, rotated -- and leaves the fastest installed; returns (waves_per_block,
    bytes_per_wave, kernel, microseconds per launch)."""
    if isinstance(launches, GroupedGemv):
        launches = [launches]
    count = launches[0].count
    if any(l.count != count for l in launches):
        _check(2, "qg_gemv_autotune")
    descs = (_Desc * (count * len(launches)))()
    for s, l in enumerate(launches):
        for i in range(count):
            descs[s * count + i] = l.descs[i]
    ws = launches[0].workspace
    w, b, k = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    us = ctypes.c_float()
    _check(lib().qg_gemv_autotune(descs, count, len(launches), ws.data_ptr(), ws.numel(), _stream(), repeats,
                                  ctypes.byref(w), ctypes.byref(b), ctypes.byref(k), ctypes.byref(us)),
           "qg_gemv_autotune")
    return w.value, b.value, k.value, us.value


AUTOTUNE_TEAMS = (0, 2, 4, 8, 12, 16)
AUTOTUNE_SIZES = (0, 4096, 8192, 16384, 32768, 49152, 65536)


def qg_gemv_autotune_report():
    """(microseconds per candidate, -1 where the budget dropped it; number timed; number dropped)
    of the last qg_gemv_autotune.  Candidate ((kernel - 1) * 6 + team index) * 7 + size index."""
    us = (ctypes.c_float * 168)()
    timed, dropped = ctypes.c_int(), ctypes.c_int()
    _check(lib().qg_gemv_autotune_report(us, 168, ctypes.byref(timed), ctypes.byref(dropped)), "qg_gemv_autotune_report")
    return list(us), timed.value, dropped.value


def qg_gemv_record_tuning(problems: Sequence[dict], waves_per_block: int, bytes_per_wave: int, kernel: int):
    """Records a launch shape for every later launch whose list of (N, K, bits, group) equals that of
    `problems` (dicts with N, K, bits, group)."""
    descs = (_Desc * len(problems))()
    for i, p in enumerate(problems):
        descs[i] = _Desc(0, p["N"], p["K"], p["bits"], p["group"], 0, 0)
    _check(lib().qg_gemv_record_tuning(descs, len(problems), waves_per_block, bytes_per_wave, kernel),
           "qg_gemv_record_tuning")


def qg_clear_tuning():
    lib().qg_clear_tuning()


def qg_gemm_autotune(packed_sets: Sequence[torch.Tensor], N: int, K: int, bits: int, group: int, X: torch.Tensor,
                     Y: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, repeats: int = 20):
    """Searches the launch shape of qg_gemm_small for this problem, records the fastest and returns
    (K ranges, shape, microseconds per call)."""
    _dev(X, torch.float32, "X")
    M = X.shape[0]
    for b in packed_sets:
        _dev(b, torch.uint8, "packed")
        if b.numel() < qg_packed_bytes(N, K, bits, group, QG_LAYOUT_DEVICE):
            _check(2, "qg_gemm_autotune")
    if X.dim() != 2 or X.shape[1] != K:
        _check(2, "qg_gemm_autotune")
    if Y is None:
        Y = torch.empty((M, N), dtype=torch.float32, device=X.device)
    if workspace is None:
        workspace = new_workspace(qg_workspace_bytes(N, K, bits, group, M), X.device)
    ptrs = (ctypes.c_void_p * len(packed_sets))(*[b.data_ptr() for b in packed_sets])
    sp, sh, us = ctypes.c_int(), ctypes.c_int(), ctypes.c_float()
    _check(lib().qg_gemm_autotune(ptrs, len(packed_sets), N, K, bits, group, X.data_ptr(), M, Y.data_ptr(),
                                  workspace.data_ptr(), workspace.numel(), _stream(), repeats,
                                  ctypes.byref(sp), ctypes.byref(sh), ctypes.byref(us)), "qg_gemm_autotune")
    return sp.value, sh.value, us.value


GEMM_AUTOTUNE_SHAPES = (0, -1) + tuple(range(1, 14))


def qg_gemm_autotune_report():
    """(microseconds per candidate: -1 dropped by the price, -2 not a plan of its own; number timed;
    number dropped) of the last qg_gemm_autotune.  Candidate = GEMM_AUTOTUNE_SHAPES.index(shape) * 8 +
    K ranges - 1."""
    us = (ctypes.c_float * 120)()
    timed, dropped = ctypes.c_int(), ctypes.c_int()
    _check(lib().qg_gemm_autotune_report(us, 120, ctypes.byref(timed), ctypes.byref(dropped)), "qg_gemm_autotune_report")
    return list(us), timed.value, dropped.value


def qg_set_gemm_tuning(splits: int = 0, shape: int = 0):
    _check(lib().qg_set_gemm_tuning(splits, shape), "qg_set_gemm_tuning")


# --- between the products of a token's step --------------------------------------------------------------------

_TYPES = {torch.float32: QG_F32, torch.bfloat16: QG_BF16, torch.float16: QG_F16, torch.float8_e4m3fn: QG_E4M3}
_E4M3 = torch.float8_e4m3fn
# descriptions as include/qg.h lays them out (8-byte members first, so that nothing is padded in between)
_NORM = struct.Struct("6Q4q4if4x").pack
_CACHE = "5Q2q6i"
_APPEND = struct.Struct(_CACHE + "7Q5q4i").pack
_ATTENTION = struct.Struct(_CACHE + "5Qq4if4x2Q").pack
_BOOK = struct.Struct("6Qq3i4x").pack
_PLANE = struct.Struct("Qqq").pack


# A call of a few microseconds on the GPU must not take longer to describe: outputs that are made here are not looked at again, and
# what every call asks of its tensors is asked once (norm of one row: 9.9 -> 8.3 us a call, 2.4 of them the launch).
_FLOATS = {t: k for t, k in _TYPES.items() if k != QG_E4M3}
_CELLS = {t: k for t, k in _TYPES.items() if k != QG_F32}


def _type(t: torch.Tensor, name: str, types=_FLOATS) -> int:
    kind = types.get(t.dtype)
    if kind is None:
        raise ValueError(f"{name}: expected one of {', '.join(map(str, types))}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name}: expected a tensor on the GPU")
    return kind


def _whole(t: torch.Tensor, dtype, name: str, shape) -> int:
    if t.dtype is not dtype or t.shape != shape or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on the GPU")
    return t.data_ptr()


def _heads(t: torch.Tensor, dtype, name: str, shape):
    """Address and stride of a [tokens][heads][head_dim] tensor whose tokens may lie apart (a part of a stacked product's output)."""
    if t.dtype is not dtype or t.shape != shape or not t.is_cuda:
        raise ValueError(f"{name}: expected a {dtype} tensor of shape {tuple(shape)} on the GPU")
    token, head, element = t.stride()
    if element != 1 or (head != shape[2] and shape[1] != 1):
        raise ValueError(f"{name}: the heads of a token have to lie together")
    return t.data_ptr(), token


def qg_rms_norm(x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-5, residual: Optional[torch.Tensor] = None,
                dtype: Optional[torch.dtype] = None, group: int = 0, y: Optional[torch.Tensor] = None,
                h: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None):
    """(y, h, scales) of rows x [rows][K]: h = x + residual in x's type (None without a residual), y its norm times the
    weight in `dtype` (x's own if not given); torch.float8_e4m3fn comes with scales [rows][K / group] (group 0: one for a
    row), other types with None.  x and residual may have rows that lie apart; h may be either."""
    shape = x.shape
    if len(shape) != 2:
        raise ValueError("x: expected [rows][K]")
    rows, K = shape
    kind, device = _type(x, "x"), x.device
    xstride, element = x.stride()
    if element != 1 and K > 1:
        raise ValueError("x: expected contiguous rows")
    wkind = _type(weight, "weight")
    if weight.shape != (K,) or group < 0 or (group and K % group):
        _check(2, "qg_rms_norm")
    if not weight.is_contiguous():
        raise ValueError("weight: expected a contiguous tensor")
    if dtype is None:
        dtype = x.dtype if y is None else y.dtype
    ykind = _TYPES.get(dtype)
    if ykind is None:
        raise ValueError(f"dtype: {dtype} is not supported")
    if y is None:
        y = _rows(rows, K, dtype, device)
    else:
        _whole(y, dtype, "y", shape)
    hp = rp = rstride = sp = 0
    if residual is not None:
        if residual.dtype is not x.dtype or residual.shape != shape or not residual.is_cuda:
            raise ValueError(f"residual: expected a {x.dtype} tensor of shape {tuple(shape)} on the GPU")
        rstride, element = residual.stride()
        if element != 1 and K > 1:
            raise ValueError("residual: expected contiguous rows")
        if h is None:
            h = _rows(rows, K, x.dtype, device)
        else:
            _whole(h, x.dtype, "h", shape)
        hp, rp = h.data_ptr(), residual.data_ptr()
    elif h is not None:
        raise ValueError("h: there is none without a residual")
    if ykind == QG_E4M3:
        groups = K // group if group else 1
        if scales is None:
            scales = _rows(rows, groups, torch.float32, device)
        else:
            _whole(scales, torch.float32, "scales", (rows, groups))
        sp = scales.data_ptr()
    elif scales is not None:
        raise ValueError("scales: float8_e4m3fn only")
    rc = (_LIB or lib()).qg_rms_norm(_NORM(x.data_ptr(), rp, weight.data_ptr(), hp, y.data_ptr(), sp, rows, K, xstride, rstride,
                                           kind, wkind, ykind, group, eps), _stream())
    if rc != 0:
        _check(rc, "qg_rms_norm")
    return y, h, scales


def _cache(k, v, tables, k_scale, v_scale):
    """The packed members of a qg_kv_cache, checked."""
    shape = k.shape
    kind = _type(k, "k", _CELLS)
    if len(shape) != 4 or not k.is_contiguous():
        raise ValueError("k: expected a contiguous tensor [pages][kv_heads][page][head_dim]")
    ksp = vsp = 0
    if kind == QG_E4M3:
        if k_scale is None or v_scale is None:
            raise ValueError("k_scale, v_scale: a cache in float8_e4m3fn has them")
        ksp, vsp = _whole(k_scale, torch.float32, "k_scale", shape[:3]), _whole(v_scale, torch.float32, "v_scale", shape[:3])
    tshape = tables.shape
    if tables.dtype is not torch.int32 or not tables.is_cuda or len(tshape) != 2:
        raise ValueError("tables: expected an int32 tensor [rows][max_pages] on the GPU")
    tstride, element = tables.stride()
    if element != 1 and tshape[1] > 1:
        raise ValueError("tables: expected contiguous rows")
    pages, kv_heads, page, head_dim = shape
    return (k.data_ptr(), _whole(v, k.dtype, "v", shape), ksp, vsp, tables.data_ptr(), tstride, pages, tshape[0], tshape[1], kv_heads, page,
            head_dim, kind)


def qg_kv_append(k_cache: torch.Tensor, v_cache: torch.Tensor, tables: torch.Tensor, rows: torch.Tensor, positions: torch.Tensor,
                 k: torch.Tensor, v: torch.Tensor, q: Optional[torch.Tensor] = None, cos_sin: Optional[torch.Tensor] = None,
                 interleaved: bool = False, k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None,
                 q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """Stores k and v [tokens][kv_heads][head_dim] in the cache's pages at each token's row and position, k and q rotated by
    cos_sin [positions][rope_dim] (cosines, then sines; None: not at all), and returns the rotated q.  A token of a row
    or position without a page (row -1, say) is padding."""
    cache = _cache(k_cache, v_cache, tables, k_scale, v_scale)
    kv_heads, D = cache[9], cache[11]
    tokens, dtype = k.shape[0], k.dtype
    kind = _type(k, "k")
    heads = qp = qs = qop = 0
    kp, ks = _heads(k, dtype, "k", (tokens, kv_heads, D))
    vp, vs = _heads(v, dtype, "v", (tokens, kv_heads, D))
    if q is not None:
        if q.dim() != 3:
            raise ValueError("q: expected [tokens][heads][head_dim]")
        heads = q.shape[1]
        qp, qs = _heads(q, dtype, "q", (tokens, heads, D))
        if q_out is None:
            q_out = torch.empty_strided((tokens, heads, D), (heads * D, D, 1), dtype=dtype, device=q.device)
        else:
            _whole(q_out, dtype, "q_out", (tokens, heads, D))
        qop = q_out.data_ptr()
    rp, pp = _whole(rows, torch.int32, "rows", (tokens,)), _whole(positions, torch.int32, "positions", (tokens,))
    cp = rope = angles = 0
    if cos_sin is not None:
        if cos_sin.dim() != 2:
            raise ValueError("cos_sin: expected [positions][rope_dim]")
        angles, rope = cos_sin.shape
        cp = _whole(cos_sin, torch.float32, "cos_sin", (angles, rope))
    rc = (_LIB or lib()).qg_kv_append(_APPEND(*cache, rp, pp, qp, kp, vp, qop, cp, tokens, qs, ks, vs, angles,
                                              kind, heads, rope, 1 if interleaved else 0), _stream())
    if rc != 0:
        _check(rc, "qg_kv_append")
    return q_out


def qg_paged_attention_workspace_bytes(batch: int, heads: int, kv_heads: int, head_dim: int) -> int:
    return int(lib().qg_paged_attention_workspace_bytes(batch, heads, kv_heads, head_dim))


def qg_paged_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, tables: torch.Tensor, lens: torch.Tensor,
                       scale: float, first: Optional[torch.Tensor] = None, window: int = 0, k_scale: Optional[torch.Tensor] = None,
                       v_scale: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, lse=False,
                       workspace: Optional[torch.Tensor] = None):
    """(out, lse) of one new token q [batch][heads][head_dim] of each sequence over its cells [max(first, lens - window), lens)
    of the cache.  lse [batch][heads] is written if asked for by True or handed in, otherwise None."""
    cache = _cache(k_cache, v_cache, tables, k_scale, v_scale)
    shape = q.shape
    if len(shape) != 3:
        raise ValueError("q: expected [batch][heads][head_dim]")
    batch, heads, D = shape
    dtype, device = q.dtype, q.device
    kind = _type(q, "q")
    qp, qs = _heads(q, dtype, "q", (batch, heads, cache[11]))
    if out is None:
        out = torch.empty_strided((batch, heads, D), (heads * D, D, 1), dtype=dtype, device=device)
    else:
        _whole(out, dtype, "out", shape)
    lp = _whole(lens, torch.int32, "lens", (batch,))
    fp = 0 if first is None else _whole(first, torch.int32, "first", (batch,))
    if lse is True:
        lse = _rows(batch, heads, torch.float32, device)
        ep = lse.data_ptr()
    elif lse is False or lse is None:
        lse, ep = None, 0
    else:
        ep = _whole(lse, torch.float32, "lse", (batch, heads))
    L = _LIB or lib()
    if workspace is None:
        workspace = new_workspace(L.qg_paged_attention_workspace_bytes(batch, heads, cache[9], D), device)
    rc = L.qg_paged_attention(_ATTENTION(*cache, lp, fp, qp, out.data_ptr(), ep, qs, batch, heads, kind, window, scale,
                                         workspace.data_ptr(), workspace.numel() * workspace.element_size()), _stream())
    if rc != 0:
        _check(rc, "qg_paged_attention")
    return out, lse


def qg_pages_workspace_bytes(rows: int, max_pages: int, pages: int) -> int:
    return int(lib().qg_pages_workspace_bytes(rows, max_pages, pages))


def _planes(planes, pages: int) -> bytes:
    """Tensors [layers][pages][...] whose pages move with the book, packed as qg_page_plane."""
    packed = b""
    for t in planes:
        shape = t.shape
        if len(shape) < 3 or shape[1] != pages or not t.is_cuda or not t.is_contiguous():
            raise ValueError("planes: expected contiguous tensors [layers][pages][...] on the GPU")
        packed += _PLANE(t.data_ptr(), shape[0], t.stride(1) * t.element_size())
    return packed


def _ints(n: int, device) -> torch.Tensor:
    return torch.empty_strided((n,), (1,), dtype=torch.int32, device=device)


def _book(tables, lens, refs, page, out):
    """(packed qg_page_book, rows, max_pages, pages, tables_out, lens_out, refs_out)"""
    i32 = torch.int32
    shape = tables.shape
    if len(shape) != 2 or refs.dim() != 1:
        raise ValueError("tables, refs: expected [rows][max_pages] and [pages]")
    rows, columns = shape
    pages = refs.shape[0]
    tp, rp = _whole(tables, i32, "tables", shape), _whole(refs, i32, "refs", (pages,))
    lp = 0 if lens is None else _whole(lens, i32, "lens", (rows,))
    if out is None:
        device = tables.device
        t, n, r = _rows(rows, columns, i32, device), None if lens is None else _ints(rows, device), _ints(pages, device)
    else:
        t, n, r = out
        _whole(t, i32, "tables out", shape)
        _whole(r, i32, "refs out", (pages,))
        if lens is not None:
            _whole(n, i32, "lens out", (rows,))
    return _BOOK(tp, lp, rp, t.data_ptr(), 0 if n is None else n.data_ptr(), r.data_ptr(), pages, rows, columns, page), rows, columns, pages, t, n, r


def qg_pages_resize(tables: torch.Tensor, lens: torch.Tensor, refs: torch.Tensor, page: int, new_lens: torch.Tensor,
                    planes: Sequence[torch.Tensor] = (), out=None, lacking: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None):
    """(tables, lens, refs, lacking) after every row got its new length: pages let go of and taken, shared last pages of rows
    that grow copied in all planes ([layers][pages][...]).  lacking [1]: 0, or how many free pages were missing
    (then nothing changed).  out: (tables, lens, refs) to write into, the old ones for instance."""
    book, rows, columns, pages, t, n, r = _book(tables, lens, refs, page, out)
    np_ = _whole(new_lens, torch.int32, "new_lens", (rows,))
    if lacking is None:
        lacking = _ints(1, tables.device)
    else:
        _whole(lacking, torch.int32, "lacking", (1,))
    L = _LIB or lib()
    if workspace is None:
        workspace = _bytes(max(256, L.qg_pages_workspace_bytes(rows, columns, pages)), tables.device)
    rc = L.qg_pages_resize(book, np_, _planes(planes, pages), len(planes), lacking.data_ptr(),
                           workspace.data_ptr(), workspace.numel(), _stream())
    if rc != 0:
        _check(rc, "qg_pages_resize")
    return t, n, r, lacking


def qg_pages_fork(tables: torch.Tensor, lens: torch.Tensor, refs: torch.Tensor, parents: torch.Tensor, out=None):
    """(tables, lens, refs) with row b the former row parents[b] (-1: empty), pages shared.  out must not be the old ones."""
    book, rows, _, _, t, n, r = _book(tables, lens, refs, 1, out)
    rc = (_LIB or lib()).qg_pages_fork(book, _whole(parents, torch.int32, "parents", (rows,)), _stream())
    if rc != 0:
        _check(rc, "qg_pages_fork")
    return t, n, r


def qg_pages_compact(tables: torch.Tensor, refs: torch.Tensor, planes: Sequence[torch.Tensor] = (), out=None,
                     live: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """(tables, refs, live) with the pages in use moved to the lower end of the pool in all planes; live [1]: how many
    there are.  out: (tables, refs) to write into, the old ones for instance."""
    book, rows, columns, pages, t, _, r = _book(tables, None, refs, 1, None if out is None else (out[0], None, out[1]))
    if live is None:
        live = _ints(1, tables.device)
    else:
        _whole(live, torch.int32, "live", (1,))
    L = _LIB or lib()
    if workspace is None:
        workspace = _bytes(max(256, L.qg_pages_workspace_bytes(rows, columns, pages)), tables.device)
    rc = L.qg_pages_compact(book, _planes(planes, pages), len(planes), live.data_ptr(),
                            workspace.data_ptr(), workspace.numel(), _stream())
    if rc != 0:
        _check(rc, "qg_pages_compact")
    return t, r, live


def qg_pages_copy(planes: Sequence[torch.Tensor], pairs: torch.Tensor):
    """Copies page pairs[i][0] onto page pairs[i][1] in all planes [layers][pages][...]."""
    pages = planes[0].shape[1] if len(planes) and planes[0].dim() > 1 else 0
    if pairs.dim() != 2 or pairs.shape[1] != 2:
        raise ValueError("pairs: expected [count][2]")
    _check((_LIB or lib()).qg_pages_copy(_planes(planes, pages), len(planes), pages, _dev(pairs, torch.int32, "pairs").data_ptr(),
                                         pairs.shape[0], _stream()), "qg_pages_copy")


# --- a layer of experts -----------------------------------------------------------------------------------------

_ROUTE = struct.Struct("4Q2q8if4x").pack
_EXPERTS = struct.Struct("5Q6q6i2Q").pack
_COMBINE = struct.Struct("5Q4q3i4x").pack
_SCORES = {"softmax": 0, "sigmoid": 1}


def _matrix_rows(t: torch.Tensor, name: str, shape=None, types=_FLOATS):
    """(address, stride of rows, type) of a matrix whose rows may lie apart."""
    kind = _type(t, name, types)
    if t.dim() != 2 or (shape is not None and t.shape != shape):
        raise ValueError(f"{name}: expected a matrix" + (f" of shape {tuple(shape)}" if shape is not None else ""))
    stride, element = t.stride()
    if element != 1 and t.shape[1] > 1:
        raise ValueError(f"{name}: expected contiguous rows")
    return t.data_ptr(), stride, kind


def _stream_of(*tensors) -> int:
    """The current stream of the current device, which all of a call's tensors have to lie on (those that the call makes lie where its first does)."""
    device = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError(f"expected tensors on the current device ({device}), got one on {t.device}")
    return torch._C._cuda_getCurrentRawStream(device)


def qg_route(logits: torch.Tensor, top_k: int, bias: Optional[torch.Tensor] = None, score: str = "softmax", groups: int = 1,
             top_groups: Optional[int] = None, group_best: int = 1, renormalise: bool = True, scale: float = 1.0,
             ids: Optional[torch.Tensor] = None, weights: Optional[torch.Tensor] = None):
    """(ids, weights) [tokens][top_k] of the experts that logits [tokens][experts] choose, the best first: scores are softmax or sigmoid of the
    logits, `bias` [experts] counts for the choice alone, and of `groups` of neighbouring experts the top_groups best take part.
    An id -1 has weight 0: no expert was left (a logit of -inf is an expert that is switched off)."""
    lp, stride, kind = _matrix_rows(logits, "logits")
    tokens, experts = logits.shape
    if score not in _SCORES:
        raise ValueError("score: softmax or sigmoid")
    bp = 0 if bias is None else _whole(bias, torch.float32, "bias", (experts,))
    shape, device, stream = (tokens, top_k), logits.device, _stream_of(logits, bias, ids, weights)
    if top_k <= 0:
        _check(2, "qg_route")
    if ids is None:
        ids = _rows(tokens, top_k, torch.int32, device)
    else:
        _whole(ids, torch.int32, "ids", shape)
    if weights is None:
        weights = _rows(tokens, top_k, torch.float32, device)
    else:
        _whole(weights, torch.float32, "weights", shape)
    rc = (_LIB or lib()).qg_route(_ROUTE(lp, bp, ids.data_ptr(), weights.data_ptr(), tokens, stride, kind, experts, top_k, _SCORES[score],
                                         groups, groups if top_groups is None else top_groups, group_best, 1 if renormalise else 0, scale), stream)
    if rc != 0:
        _check(rc, "qg_route")
    return ids, weights


def qg_expert_plan(ids: torch.Tensor, experts: int, out=None):
    """(offsets [experts + 1], slot_tokens [tokens * top_k], slots [tokens][top_k]): the choices ids [tokens][top_k] ordered by expert.
    Expert e has the slots offsets[e] ... offsets[e + 1] - 1; an id outside 0 ... experts - 1 gets none (-1).  out: the three to write into."""
    shape = ids.shape
    if len(shape) != 2:
        raise ValueError("ids: expected [tokens][top_k]")
    tokens, top_k = shape
    ip, device = _whole(ids, torch.int32, "ids", shape), ids.device
    if experts <= 0 or top_k <= 0:
        _check(2, "qg_expert_plan")
    stream = _stream_of(ids, *(() if out is None else out))
    if out is None:
        offsets, slot_tokens, slots = _ints(experts + 1, device), _ints(tokens * top_k, device), _rows(tokens, top_k, torch.int32, device)
    else:
        offsets, slot_tokens, slots = out
        _whole(offsets, torch.int32, "offsets", (experts + 1,))
        _whole(slot_tokens, torch.int32, "slot_tokens", (tokens * top_k,))
        _whole(slots, torch.int32, "slots", shape)
    rc = (_LIB or lib()).qg_expert_plan(ip, tokens, top_k, experts, offsets.data_ptr(), slot_tokens.data_ptr(), slots.data_ptr(), stream)
    if rc != 0:
        _check(rc, "qg_expert_plan")
    return offsets, slot_tokens, slots


def qg_experts_workspace_bytes(x_rows: int, K: int, dtype: torch.dtype = torch.float32) -> int:
    return int(lib().qg_experts_workspace_bytes(x_rows, K, _FLOATS[dtype]))


def qg_experts_product(packed: torch.Tensor, N: int, K: int, bits: int, group: int, x: torch.Tensor, offsets: torch.Tensor,
                       rows: Optional[torch.Tensor] = None, gated: bool = False, dtype: Optional[torch.dtype] = None,
                       y: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y[p] = What_e x[rows[p]] (x[p], if rows is None) for each slot p of each expert e (offsets of qg_expert_plan) in `dtype` (x's own if not given);
    gated: silu(gate) * up of N / 2 columns, What_e's first N / 2 rows being gate.  packed: [experts][bytes], an expert's qg_pack blob a row.
    Slots past the last expert's are not written."""
    xp, xs, kind = _matrix_rows(x, "x")
    if packed.dtype is not torch.uint8 or packed.dim() != 2 or not packed.is_cuda or (packed.stride(1) != 1 and packed.shape[1] > 1):
        raise ValueError("packed: expected a uint8 tensor [experts][bytes] on the GPU")
    experts, nbytes = packed.shape
    x_rows, width = x.shape
    if width != K or nbytes < qg_packed_bytes(N, K, bits, group, QG_LAYOUT_DEVICE):
        _check(2, "qg_experts_product")
    op = _whole(offsets, torch.int32, "offsets", (experts + 1,))
    if rows is None:
        rp, slots = 0, x_rows if y is None else y.shape[0]
    else:
        slots = rows.shape[0]
        rp = _whole(rows, torch.int32, "rows", (slots,))
    columns, stream = N // 2 if gated else N, _stream_of(packed, x, offsets, rows, y, workspace)
    if y is None:
        y = _rows(slots, columns, x.dtype if dtype is None else dtype, x.device)
    else:
        _whole(y, y.dtype if dtype is None else dtype, "y", (slots, columns))
    ykind = _type(y, "y")
    L = _LIB or lib()
    if workspace is None:
        workspace = _bytes(max(256, L.qg_experts_workspace_bytes(x_rows, K, kind)), x.device)
    elif not workspace.is_contiguous():
        raise ValueError("workspace: expected a contiguous tensor")
    rc = L.qg_experts_product(_EXPERTS(packed.data_ptr(), xp, op, rp, y.data_ptr(), N, K, packed.stride(0), x_rows, xs, slots,
                                       bits, group, experts, kind, ykind, 1 if gated else 0,
                                       workspace.data_ptr(), workspace.numel() * workspace.element_size()), stream)
    if rc != 0:
        _check(rc, "qg_experts_product")
    return y


def qg_experts_combine(y: torch.Tensor, slots: torch.Tensor, weights: torch.Tensor, residual: Optional[torch.Tensor] = None,
                       dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """out[t] = residual[t] + sum over j of weights[t][j] y[slots[t][j]] in `dtype` (the residual's, or y's own, if not given); a slot
    outside y's rows adds nothing.  out may be the residual."""
    kind = _type(y, "y")
    if y.dim() != 2 or not y.is_contiguous():
        raise ValueError("y: expected a contiguous matrix [slots][N]")
    y_rows, N = y.shape
    shape = slots.shape
    if len(shape) != 2:
        raise ValueError("slots: expected [tokens][top_k]")
    tokens, top_k = shape
    sp, wp = _whole(slots, torch.int32, "slots", shape), _whole(weights, torch.float32, "weights", shape)
    if dtype is None:
        dtype = out.dtype if out is not None else residual.dtype if residual is not None else y.dtype
    stream = _stream_of(y, slots, weights, residual, out)
    if out is None:
        out = _rows(tokens, N, dtype, y.device)
    else:
        _whole(out, dtype, "out", (tokens, N))
    okind = _type(out, "out")
    rp = rs = 0
    if residual is not None:
        if residual.dtype is not dtype:
            raise ValueError(f"residual: expected a {dtype} tensor")
        rp, rs, _ = _matrix_rows(residual, "residual", (tokens, N))
    rc = (_LIB or lib()).qg_experts_combine(_COMBINE(y.data_ptr(), sp, wp, rp, out.data_ptr(), y_rows, tokens, N, rs, kind, okind, top_k), stream)
    if rc != 0:
        _check(rc, "qg_experts_combine")
    return out
