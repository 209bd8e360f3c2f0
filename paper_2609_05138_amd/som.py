"""Thin ctypes binding of libsom (include/som.h) for torch device tensors.

Argument marshalling only: every step of the search runs in the HIP
library.  There is no CPU path: if the library is not built, or a tensor is
not on a ROCm device, calls raise.  Function names match the C entry points.
"""

from __future__ import annotations

import ctypes
import os
from typing import Optional, Tuple

import torch  # imported before the library so both share one HIP runtime

_PKG = os.path.dirname(os.path.abspath(__file__))
# SOM_LIBRARY names another build of the same library (the host-sanitized
# one, for CPU-side checks); it must exist like the default one
LIB_PATH = os.environ.get("SOM_LIBRARY") or os.path.join(_PKG, "libsom.so")

SOM_OK = 0
SOM_ERR_INVALID_ARG = 1
SOM_ERR_INVALID_CSR = 2
SOM_ERR_WORKSPACE = 3
SOM_ERR_HIP = 4

EXPORTS = (
    "som_abi_version",
    "som_last_error",
    "som_codebook_norms",
    "som_codebook_ldw",
    "som_bmu_workspace_bytes",
    "som_bmu_search",
    "som_bmu_search_top2",
    "som_bmu_search_noalloc",
    "som_plan_bytes",
    "som_plan",
    "som_bmu_search_planned_workspace_bytes",
    "som_bmu_search_planned",
    "som_bmu_search_top2_planned",
    "som_tile_plan",
    "som_group_plan",
    "som_cluster_workspace_bytes",
    "som_cluster_order",
    "som_codebook_norms_f16",
    "som_bmu_search_f16",
    "som_bmu_search_top2_f16",
    "som_bmu_search_planned_f16",
    "som_bmu_search_top2_planned_f16",
    "som_bmu_search_unfused_workspace_bytes",
    "som_bmu_search_unfused",
    "som_update_accumulate",
    "som_update_workspace_bytes",
    "som_update_finish",
    "som_update_finish_f16",
    "som_probe_read",
    "som_probe_lds",
    "som_rms_norm",
    "som_rms_norm_backward_workspace_bytes",
    "som_rms_norm_backward",
    "som_product_workspace_bytes",
    "som_product",
    "som_product_backward_workspace_bytes",
    "som_product_backward",
    "som_dropout",
)

# som_dtype and som_act
DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2, torch.float8_e4m3fn: 3}
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}


class SomError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"libsom status {status}: {msg}")
        self.status = status


class som_bmu_opts(ctypes.Structure):
    _fields_ = [
        ("kernel", ctypes.c_int32),
        ("tile_docs", ctypes.c_int32),
        ("lane_neurons", ctypes.c_int32),
        ("group_tiles", ctypes.c_int32),
        ("mask_mode", ctypes.c_int32),
        ("slice_neurons", ctypes.c_int32),
        ("validate", ctypes.c_int32),
        ("storage", ctypes.c_int32),
        ("schedule", ctypes.c_int32),
        ("neuron_chunk", ctypes.c_int32),
        ("sweep", ctypes.c_int32),
    ]


class som_epilogue(ctypes.Structure):
    _fields_ = [
        ("act", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("alpha", ctypes.c_float),
        ("x_scale", ctypes.c_void_p),
        ("w_scale", ctypes.c_void_p),
        ("bias", ctypes.c_void_p),
        ("residual", ctypes.c_void_p),
        ("ldr", ctypes.c_int64),
        ("pre", ctypes.c_void_p),
        ("ldp", ctypes.c_int64),
    ]


_lib = None

_i64 = ctypes.c_int64
_i32 = ctypes.c_int32
_vp = ctypes.c_void_p
_sz = ctypes.c_size_t


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libsom.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError(
            f"{path} is missing: build it with `python -m paper_2609_05138_amd.build` "
            "(there is no CPU fallback)")
    lib = ctypes.CDLL(path)
    lib.som_abi_version.restype = _i32
    lib.som_abi_version.argtypes = []
    lib.som_last_error.restype = ctypes.c_char_p
    lib.som_last_error.argtypes = []
    lib.som_codebook_norms.restype = _i32
    lib.som_codebook_norms.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp]
    lib.som_codebook_ldw.restype = _i64
    lib.som_codebook_ldw.argtypes = [_i64]
    lib.som_bmu_workspace_bytes.restype = _sz
    lib.som_bmu_workspace_bytes.argtypes = [_i64, _i64, _i64, _i64, ctypes.POINTER(som_bmu_opts)]
    lib.som_bmu_search.restype = _i32
    lib.som_bmu_search.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _vp, _i64, _i64, _vp, _vp, _vp,
                                   ctypes.POINTER(som_bmu_opts), _vp, _sz, _vp]
    lib.som_bmu_search_noalloc.restype = _i32
    lib.som_bmu_search_noalloc.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _vp, _i64, _i64, _vp, _vp, _vp,
                                           ctypes.POINTER(som_bmu_opts), _vp]
    lib.som_plan_bytes.restype = _sz
    lib.som_plan_bytes.argtypes = [_i64, _i64, ctypes.POINTER(som_bmu_opts)]
    lib.som_plan.restype = _i32
    lib.som_plan.argtypes = [_vp, _vp, _i64, _i64, _i64, _vp, ctypes.POINTER(som_bmu_opts), _vp, _sz, _vp]
    lib.som_bmu_search_planned_workspace_bytes.restype = _sz
    lib.som_bmu_search_planned_workspace_bytes.argtypes = [_i64, _i64, ctypes.POINTER(som_bmu_opts)]
    lib.som_bmu_search_top2.restype = _i32
    lib.som_bmu_search_top2.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _vp, _i64, _i64, _vp, _vp, _vp, _vp, _vp,
                                        ctypes.POINTER(som_bmu_opts), _vp, _sz, _vp]
    lib.som_bmu_search_top2_planned.restype = _i32
    lib.som_bmu_search_top2_planned.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _i64, _vp, _vp, _sz,
                                                _vp, _vp, _vp, _vp, ctypes.POINTER(som_bmu_opts), _vp, _sz, _vp]
    lib.som_bmu_search_planned.restype = _i32
    lib.som_bmu_search_planned.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _i64, _vp, _vp, _sz,
                                           _vp, _vp, ctypes.POINTER(som_bmu_opts), _vp, _sz, _vp]
    lib.som_tile_plan.restype = _i32
    lib.som_tile_plan.argtypes = [_vp, _vp, _i64, _i64, _i64, _vp, _i32, _vp, _vp, _vp, _vp, _vp]
    lib.som_group_plan.restype = _i32
    lib.som_group_plan.argtypes = [_vp, _vp, _i64, _i64, _i64, _vp, _i32, _vp, _vp, _vp, _vp, _vp]
    lib.som_cluster_workspace_bytes.restype = _sz
    lib.som_cluster_workspace_bytes.argtypes = [_i64, _i64, _i64]
    # the fp16 functions take the same arguments (W as binary16 bit patterns)
    for base in ("som_codebook_norms", "som_bmu_search", "som_bmu_search_top2", "som_bmu_search_planned",
                 "som_bmu_search_top2_planned"):
        fn = getattr(lib, base + "_f16")
        fn.restype = _i32
        fn.argtypes = getattr(lib, base).argtypes
    lib.som_bmu_search_unfused_workspace_bytes.restype = _sz
    lib.som_bmu_search_unfused_workspace_bytes.argtypes = [_i64, _i64, _i64, _i64, ctypes.POINTER(som_bmu_opts), _i64]
    lib.som_bmu_search_unfused.restype = _i32
    lib.som_bmu_search_unfused.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _vp, _i64, _i64, _vp, _vp, _vp,
                                           ctypes.POINTER(som_bmu_opts), _i64, _vp, _sz, _vp]
    lib.som_update_accumulate.restype = _i32
    lib.som_update_accumulate.argtypes = [_vp, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _vp, _vp]
    lib.som_update_workspace_bytes.restype = _sz
    lib.som_update_workspace_bytes.argtypes = [_i64, _i64]
    for fn in (lib.som_update_finish, lib.som_update_finish_f16):
        fn.restype = _i32
        fn.argtypes = [_vp, _i64, _i64, _i32, _i32, ctypes.c_double, _vp, _i64, _vp, _vp, _sz, _vp]
    lib.som_probe_read.restype = _i32
    lib.som_probe_read.argtypes = [_vp, _i64, _i32, _vp, _vp]
    lib.som_probe_lds.restype = _i32
    lib.som_probe_lds.argtypes = [_i32, _vp, ctypes.POINTER(ctypes.c_int64), _vp]
    lib.som_cluster_order.restype = _i32
    lib.som_cluster_order.argtypes = [_vp, _vp, _i64, _i64, _i64, _vp, _vp, _sz, _vp]
    lib.som_rms_norm.restype = _i32
    lib.som_rms_norm.argtypes = [_vp, _i64, _vp, _i64, _vp, _i32, _i64, _i64, ctypes.c_float, _i32, _vp, _i64, _vp,
                                 _i64, _vp, _vp]
    lib.som_rms_norm_backward_workspace_bytes.restype = _sz
    lib.som_rms_norm_backward_workspace_bytes.argtypes = [_i64, _i64]
    lib.som_rms_norm_backward.restype = _i32
    lib.som_rms_norm_backward.argtypes = [_vp, _i64, _vp, _i64, _vp, _vp, _i64, _i32, _i64, _i64, ctypes.c_float, _vp,
                                          _i64, _vp, _vp, _sz, _vp]
    for name in ("som_product_workspace_bytes", "som_product_backward_workspace_bytes"):
        fn = getattr(lib, name)
        fn.restype = _sz
        fn.argtypes = [_i64, _i64, _i64, _i32]
    lib.som_product.restype = _i32
    lib.som_product.argtypes = [_vp, _i64, _vp, _i64, _i32, _i32, _i64, _i64, _i64, _vp, _i64, _i32,
                                ctypes.POINTER(som_epilogue), _vp, _sz, _vp]
    lib.som_product_backward.restype = _i32
    lib.som_product_backward.argtypes = [_vp, _i64, _vp, _i64, _vp, _i64, _i32, _i32, _i64, _i64, _i64, _i32, _vp,
                                         _i64, ctypes.c_float, _vp, _i64, _vp, _i64, _vp, _vp, _sz, _vp]
    lib.som_dropout.restype = _i32
    lib.som_dropout.argtypes = [_vp, _i64, _vp, _i64, _i32, _i64, _i64, ctypes.c_double, ctypes.c_uint64,
                                ctypes.c_uint64, _vp, _i64, _vp]
    _lib = lib
    return lib


def _check(status: int) -> None:
    if status != SOM_OK:
        raise SomError(status, load().som_last_error().decode(errors="replace"))


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _dev(t: torch.Tensor, dtype, name: str) -> torch.Tensor:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be on a ROCm device (got {t.device})")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _codebook(W: torch.Tensor) -> str:
    """Check the codebook tensor; return the C function suffix for its dtype."""
    if isinstance(W, torch.Tensor) and W.dtype == torch.float16:
        _dev(W, torch.float16, "W")
        return "_f16"
    _dev(W, torch.float32, "W")
    return ""


def _stream(stream) -> ctypes.c_void_p:
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _opts(kernel=0, tile_docs=0, lane_neurons=0, group_tiles=0, mask_mode=0, slice_neurons=0,
          validate=False, storage=0, schedule=0, neuron_chunk=0, sweep=0) -> som_bmu_opts:
    return som_bmu_opts(int(kernel), int(tile_docs), int(lane_neurons), int(group_tiles), int(mask_mode),
                        int(slice_neurons), int(bool(validate)), int(storage), int(schedule), int(neuron_chunk),
                        int(sweep))


def _n_neurons(N, norms, W) -> int:
    """N of a search: explicit, else the length of the norms vector.

    The codebook's second dimension is its row stride, which may exceed N
    (padding to the recommended stride); its padding columns are not
    neurons, so they are never the default."""
    if N is not None:
        return int(N)
    return int(norms.numel())


def _workspace(nbytes: int, device) -> torch.Tensor:
    # torch's caching allocator returns 256-byte (or better) aligned blocks
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)


def som_abi_version() -> int:
    return int(load().som_abi_version())


def som_last_error() -> str:
    return load().som_last_error().decode(errors="replace")


def som_codebook_ldw(N: int) -> int:
    """Recommended row stride (floats) of a feature-major codebook of N neurons."""
    return int(load().som_codebook_ldw(int(N)))


def som_codebook_norms(W: torch.Tensor, N: Optional[int] = None, norms: Optional[torch.Tensor] = None,
                       stream=None) -> torch.Tensor:
    """||w_j||^2 for j < N of the feature-major codebook W [F, ldw] (fp32 or fp16).

    N defaults to the length of ``norms`` when it is given, else to ldw (a
    codebook padded beyond N needs N)."""
    lib = load()
    sfx = _codebook(W)
    F, ldw = W.shape
    n = int(N) if N is not None else (int(norms.numel()) if norms is not None else ldw)
    if norms is None:
        norms = torch.empty(n, dtype=torch.float32, device=W.device)
    _dev(norms, torch.float32, "norms")
    if norms.numel() < n:
        raise ValueError("norms is too small")
    _check(getattr(lib, "som_codebook_norms" + sfx)(_ptr(W), F, n, ldw, _ptr(norms), _stream(stream)))
    return norms


def som_bmu_workspace_bytes(F: int, N: int, B: int, nnz: int, validate=False, **knobs) -> int:
    o = _opts(validate=validate, **knobs)
    return int(load().som_bmu_workspace_bytes(F, N, B, nnz, ctypes.byref(o)))


def _outputs(B, device, pairs):
    out = []
    for t, dtype, name in pairs:
        if t is None:
            t = torch.empty(B, dtype=dtype, device=device)
        _dev(t, dtype, name)
        if t.numel() < B:
            raise ValueError(f"{name} is too small")
        out.append(t)
    return out


def _search(top2, W, norms, indptr, indices, N, perm, validate, outs, ws, stream, knobs):
    lib = load()
    sfx = _codebook(W)
    _dev(norms, torch.float32, "norms")
    _dev(indptr, torch.int32, "indptr")
    _dev(indices, torch.int32, "indices")
    F, ldw = W.shape
    n = _n_neurons(N, norms, W)
    if norms.numel() < n:
        raise ValueError("norms must hold at least N values")
    B = indptr.numel() - 1
    nnz = indices.numel()
    if perm is not None:
        _dev(perm, torch.int32, "perm")
        if perm.numel() != B:
            raise ValueError("perm must have B entries")
    names = (("bmu", torch.int32), ("dist", torch.float32), ("bmu2", torch.int32), ("dist2", torch.float32))
    outs = _outputs(B, W.device, [(t, dt, nm) for t, (nm, dt) in zip(outs, names)])
    o = _opts(validate=validate, **knobs)
    need = int(lib.som_bmu_workspace_bytes(F, n, B, nnz, ctypes.byref(o)))
    if ws is None:
        ws = _workspace(need, W.device)
    _dev(ws, torch.uint8, "ws")
    common = (_ptr(W), F, n, ldw, _ptr(norms), _ptr(indptr), _ptr(indices), B, nnz, _ptr(perm))
    tail = (ctypes.byref(o), _ptr(ws), ws.numel(), _stream(stream))
    if top2:
        _check(getattr(lib, "som_bmu_search_top2" + sfx)(*common, *(_ptr(t) for t in outs), *tail))
    else:
        _check(getattr(lib, "som_bmu_search" + sfx)(*common, *(_ptr(t) for t in outs), *tail))
    return tuple(outs)


def som_bmu_search(W: torch.Tensor, norms: torch.Tensor, indptr: torch.Tensor, indices: torch.Tensor,
                   N: Optional[int] = None, perm: Optional[torch.Tensor] = None, validate: bool = False,
                   bmu: Optional[torch.Tensor] = None, dist: Optional[torch.Tensor] = None,
                   ws: Optional[torch.Tensor] = None, stream=None, **knobs) -> Tuple[torch.Tensor, torch.Tensor]:
    """BMU index (int32) and squared distance (fp32) of every CSR document.

    ``N`` defaults to the length of ``norms``.  ``knobs``: kernel, tile_docs,
    lane_neurons, group_tiles, mask_mode, slice_neurons, schedule,
    neuron_chunk, sweep (fields of som_bmu_opts; only sweep changes a
    result, in rounding: 1 = ascending feature order, 2 = rotated, the
    default wherever it is available)."""
    return _search(False, W, norms, indptr, indices, N, perm, validate, (bmu, dist), ws, stream, knobs)


def som_bmu_search_top2(W: torch.Tensor, norms: torch.Tensor, indptr: torch.Tensor, indices: torch.Tensor,
                        N: Optional[int] = None, perm: Optional[torch.Tensor] = None, validate: bool = False,
                        bmu: Optional[torch.Tensor] = None, dist: Optional[torch.Tensor] = None,
                        bmu2: Optional[torch.Tensor] = None, dist2: Optional[torch.Tensor] = None,
                        ws: Optional[torch.Tensor] = None, stream=None, **knobs):
    """(bmu, dist, bmu2, dist2): best and second-best unit of every document
    (bmu2 = -1 and dist2 = +inf when N == 1)."""
    return _search(True, W, norms, indptr, indices, N, perm, validate, (bmu, dist, bmu2, dist2), ws, stream,
                   knobs)


NOALLOC_SCRATCH_BYTES = 64 << 20


def som_bmu_search_noalloc(W: torch.Tensor, norms: torch.Tensor, indptr: torch.Tensor, indices: torch.Tensor,
                           N: Optional[int] = None, perm: Optional[torch.Tensor] = None,
                           bmu: Optional[torch.Tensor] = None, dist: Optional[torch.Tensor] = None, stream=None,
                           **knobs) -> Tuple[torch.Tensor, torch.Tensor]:
    """som_bmu_search whose workspace is the library's static device array
    (no allocation by the library; fp32 codebook; bmu and dist are allocated
    here only when not given)."""
    lib = load()
    _dev(W, torch.float32, "W")
    _dev(norms, torch.float32, "norms")
    _dev(indptr, torch.int32, "indptr")
    _dev(indices, torch.int32, "indices")
    F, ldw = W.shape
    n = _n_neurons(N, norms, W)
    if norms.numel() < n:
        raise ValueError("norms must hold at least N values")
    B = indptr.numel() - 1
    if perm is not None:
        _dev(perm, torch.int32, "perm")
        if perm.numel() != B:
            raise ValueError("perm must have B entries")
    bmu, dist = _outputs(B, W.device, [(bmu, torch.int32, "bmu"), (dist, torch.float32, "dist")])
    o = _opts(**knobs)
    _check(lib.som_bmu_search_noalloc(_ptr(W), F, n, ldw, _ptr(norms), _ptr(indptr), _ptr(indices), B,
                                      indices.numel(), _ptr(perm), _ptr(bmu), _ptr(dist), ctypes.byref(o),
                                      _stream(stream)))
    return bmu, dist


class Plan:
    """An opaque search plan (device buffer) and how it was built."""

    def __init__(self, buf, knobs, B, nnz, perm):
        self.buf = buf
        self.knobs = dict(knobs)
        self.B = B
        self.nnz = nnz
        self.perm = perm


def som_plan(indptr: torch.Tensor, indices: torch.Tensor, F: int, perm: Optional[torch.Tensor] = None,
             plan: Optional[torch.Tensor] = None, stream=None, **knobs) -> Plan:
    """Plan of a batch for som_bmu_search_planned (codebook-independent).

    ``knobs`` as for som_bmu_search, plus ``storage`` (0 = fp32, 1 = fp16):
    the storage type whose automatic tile size the plan takes; the planned
    search resolves the same geometry from the plan's knobs, whatever the
    codebook it is given."""
    lib = load()
    _dev(indptr, torch.int32, "indptr")
    _dev(indices, torch.int32, "indices")
    B = indptr.numel() - 1
    nnz = indices.numel()
    if perm is not None:
        _dev(perm, torch.int32, "perm")
    o = _opts(**knobs)
    need = int(lib.som_plan_bytes(B, nnz, ctypes.byref(o)))
    if plan is None:
        plan = _workspace(need, indptr.device)
    _dev(plan, torch.uint8, "plan")
    _check(lib.som_plan(_ptr(indptr), _ptr(indices), B, F, nnz, _ptr(perm), ctypes.byref(o), _ptr(plan),
                        plan.numel(), _stream(stream)))
    return Plan(plan, knobs, B, nnz, perm)


def som_bmu_search_planned_workspace_bytes(N: int, B: int, **knobs) -> int:
    o = _opts(**knobs)
    return int(load().som_bmu_search_planned_workspace_bytes(N, B, ctypes.byref(o)))


def _planned(top2, W, norms, indptr, plan, N, outs, ws, stream):
    lib = load()
    sfx = _codebook(W)
    _dev(norms, torch.float32, "norms")
    _dev(indptr, torch.int32, "indptr")
    F, ldw = W.shape
    n = _n_neurons(N, norms, W)
    if norms.numel() < n:
        raise ValueError("norms must hold at least N values")
    B = indptr.numel() - 1
    if B != plan.B:
        raise ValueError("plan was built for another batch")
    names = (("bmu", torch.int32), ("dist", torch.float32), ("bmu2", torch.int32), ("dist2", torch.float32))
    outs = _outputs(B, W.device, [(t, dt, nm) for t, (nm, dt) in zip(outs, names)])
    o = _opts(**plan.knobs)
    if ws is None:
        ws = _workspace(lib.som_bmu_search_planned_workspace_bytes(n, B, ctypes.byref(o)), W.device)
    _dev(ws, torch.uint8, "ws")
    common = (_ptr(W), F, n, ldw, _ptr(norms), _ptr(indptr), B, plan.nnz, _ptr(plan.perm), _ptr(plan.buf),
              plan.buf.numel())
    tail = (ctypes.byref(o), _ptr(ws), ws.numel(), _stream(stream))
    if top2:
        _check(getattr(lib, "som_bmu_search_top2_planned" + sfx)(*common, *(_ptr(t) for t in outs), *tail))
    else:
        _check(getattr(lib, "som_bmu_search_planned" + sfx)(*common, *(_ptr(t) for t in outs), *tail))
    return tuple(outs)


def som_bmu_search_planned(W: torch.Tensor, norms: torch.Tensor, indptr: torch.Tensor, plan: Plan,
                           N: Optional[int] = None, bmu: Optional[torch.Tensor] = None,
                           dist: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                           stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The search stage on a prebuilt plan (same indptr, perm and knobs)."""
    return _planned(False, W, norms, indptr, plan, N, (bmu, dist), ws, stream)


def som_bmu_search_top2_planned(W: torch.Tensor, norms: torch.Tensor, indptr: torch.Tensor, plan: Plan,
                                N: Optional[int] = None, bmu: Optional[torch.Tensor] = None,
                                dist: Optional[torch.Tensor] = None, bmu2: Optional[torch.Tensor] = None,
                                dist2: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                                stream=None):
    """Top-2 search stage on a prebuilt plan: (bmu, dist, bmu2, dist2)."""
    return _planned(True, W, norms, indptr, plan, N, (bmu, dist, bmu2, dist2), ws, stream)


def som_tile_plan(indptr: torch.Tensor, indices: torch.Tensor, F: int, tile_docs: int = 8,
                  perm: Optional[torch.Tensor] = None, stream=None):
    """Tile plan as explicit arrays: (tile_offset, tile_count, union_feat, union_mask).

    union_mask is int32 [nnz] for tile_docs <= 32, else [nnz, tile_docs // 32]
    (bit s of the entry's mask in word s // 32)."""
    lib = load()
    _dev(indptr, torch.int32, "indptr")
    _dev(indices, torch.int32, "indices")
    B = indptr.numel() - 1
    nnz = indices.numel()
    T = int(tile_docs)
    ntiles = (B + T - 1) // T if T > 0 else 0
    dev = indptr.device
    if perm is not None:
        _dev(perm, torch.int32, "perm")
    tile_offset = torch.empty(ntiles + 1, dtype=torch.int32, device=dev)
    tile_count = torch.empty(max(ntiles, 1), dtype=torch.int32, device=dev)
    union_feat = torch.empty(max(nnz, 1), dtype=torch.int32, device=dev)
    mw = (T + 31) // 32 if T > 0 else 1
    union_mask = torch.empty((max(nnz, 1), mw) if mw > 1 else max(nnz, 1), dtype=torch.int32, device=dev)
    _check(lib.som_tile_plan(_ptr(indptr), _ptr(indices), B, F, nnz, _ptr(perm), T, _ptr(tile_offset),
                             _ptr(tile_count), _ptr(union_feat), _ptr(union_mask), _stream(stream)))
    return tile_offset, tile_count[:ntiles], union_feat, union_mask


def som_group_plan(indptr: torch.Tensor, indices: torch.Tensor, F: int, group_docs: int = 1024,
                   perm: Optional[torch.Tensor] = None, stream=None):
    """Kernel-2 group plan as explicit arrays: (group_offset, group_count, group_feat, entry_pos)."""
    lib = load()
    _dev(indptr, torch.int32, "indptr")
    _dev(indices, torch.int32, "indices")
    B = indptr.numel() - 1
    nnz = indices.numel()
    D = int(group_docs)
    ng = (B + D - 1) // D if D > 0 else 0
    dev = indptr.device
    if perm is not None:
        _dev(perm, torch.int32, "perm")
    offset = torch.empty(ng + 1, dtype=torch.int32, device=dev)
    count = torch.empty(max(ng, 1), dtype=torch.int32, device=dev)
    feat = torch.empty(max(nnz, 1), dtype=torch.int32, device=dev)
    pos = torch.empty(max(nnz, 1), dtype=torch.int32, device=dev)
    _check(lib.som_group_plan(_ptr(indptr), _ptr(indices), B, F, nnz, _ptr(perm), D, _ptr(offset),
                              _ptr(count), _ptr(feat), _ptr(pos), _stream(stream)))
    return offset, count[:ng], feat, pos


def som_cluster_workspace_bytes(B: int, F: int, nnz: int) -> int:
    return int(load().som_cluster_workspace_bytes(B, F, nnz))


def som_cluster_order(indptr: torch.Tensor, indices: torch.Tensor, F: int,
                      perm: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                      stream=None) -> torch.Tensor:
    """Tile order grouping documents by their two highest-df features."""
    lib = load()
    _dev(indptr, torch.int32, "indptr")
    _dev(indices, torch.int32, "indices")
    B = indptr.numel() - 1
    nnz = indices.numel()
    if perm is None:
        perm = torch.empty(max(B, 1), dtype=torch.int32, device=indptr.device)
    _dev(perm, torch.int32, "perm")
    if ws is None:
        ws = _workspace(lib.som_cluster_workspace_bytes(B, F, nnz), indptr.device)
    _dev(ws, torch.uint8, "ws")
    _check(lib.som_cluster_order(_ptr(indptr), _ptr(indices), B, F, nnz, _ptr(perm), _ptr(ws), ws.numel(),
                                 _stream(stream)))
    return perm[:B]


def som_update_accumulate(indptr: torch.Tensor, indices: torch.Tensor, bmu: torch.Tensor, F: int, N: int,
                          acc: torch.Tensor, count: torch.Tensor, stream=None) -> None:
    """acc [F, ld_acc] and count [N] (int32 tensors holding uint32 counts) += one searched batch."""
    lib = load()
    for t, name in ((indptr, "indptr"), (indices, "indices"), (bmu, "bmu"), (acc, "acc"), (count, "count")):
        _dev(t, torch.int32, name)
    B = indptr.numel() - 1
    if acc.dim() != 2 or acc.shape[0] != F or acc.shape[1] < N or count.numel() < N or bmu.numel() < B:
        raise ValueError("acc must be [F, >= N], count [>= N], bmu [>= B]")
    _check(lib.som_update_accumulate(_ptr(indptr), _ptr(indices), B, indices.numel(), _ptr(bmu), F, N, _ptr(acc),
                                     acc.shape[1], _ptr(count), _stream(stream)))


def som_update_workspace_bytes(F: int, N: int) -> int:
    return int(load().som_update_workspace_bytes(F, N))


def som_update_finish(W: torch.Tensor, rows: int, cols: int, sigma: float, acc: torch.Tensor, count: torch.Tensor,
                      ws: Optional[torch.Tensor] = None, stream=None) -> None:
    """Blur the accumulators over the neighbourhood and write the new weights into W (fp32 or fp16)."""
    lib = load()
    sfx = _codebook(W)
    _dev(acc, torch.int32, "acc")
    _dev(count, torch.int32, "count")
    F, ldw = W.shape
    if acc.dim() != 2 or acc.shape[0] != F:
        raise ValueError("acc must be [F, ld_acc]")
    if ws is None:
        ws = _workspace(lib.som_update_workspace_bytes(F, rows * cols), W.device)
    _dev(ws, torch.uint8, "ws")
    _check(getattr(lib, "som_update_finish" + sfx)(_ptr(W), F, ldw, rows, cols, float(sigma), _ptr(acc),
                                                   acc.shape[1], _ptr(count), _ptr(ws), ws.numel(),
                                                   _stream(stream)))


def som_bmu_search_unfused_workspace_bytes(F: int, N: int, B: int, nnz: int, block_docs: int, **knobs) -> int:
    o = _opts(**knobs)
    return int(load().som_bmu_search_unfused_workspace_bytes(F, N, B, nnz, ctypes.byref(o), int(block_docs)))


def som_bmu_search_unfused(W: torch.Tensor, norms: torch.Tensor, indptr: torch.Tensor, indices: torch.Tensor,
                           N: Optional[int] = None, perm: Optional[torch.Tensor] = None, block_docs: int = 8192,
                           bmu: Optional[torch.Tensor] = None, dist: Optional[torch.Tensor] = None,
                           ws: Optional[torch.Tensor] = None, stream=None, **knobs) -> Tuple[torch.Tensor, torch.Tensor]:
    """The search with a materialised score block (the unfused comparator):
    same (bmu, dist) as som_bmu_search, bit for bit."""
    lib = load()
    _dev(W, torch.float32, "W")
    _dev(norms, torch.float32, "norms")
    _dev(indptr, torch.int32, "indptr")
    _dev(indices, torch.int32, "indices")
    F, ldw = W.shape
    n = _n_neurons(N, norms, W)
    if norms.numel() < n:
        raise ValueError("norms must hold at least N values")
    B = indptr.numel() - 1
    nnz = indices.numel()
    if perm is not None:
        _dev(perm, torch.int32, "perm")
    bmu, dist = _outputs(B, W.device, [(bmu, torch.int32, "bmu"), (dist, torch.float32, "dist")])
    o = _opts(**knobs)
    if ws is None:
        ws = _workspace(lib.som_bmu_search_unfused_workspace_bytes(F, n, B, nnz, ctypes.byref(o), int(block_docs)),
                        W.device)
    _dev(ws, torch.uint8, "ws")
    _check(lib.som_bmu_search_unfused(_ptr(W), F, n, ldw, _ptr(norms), _ptr(indptr), _ptr(indices), B, nnz,
                                      _ptr(perm), _ptr(bmu), _ptr(dist), ctypes.byref(o), int(block_docs), _ptr(ws),
                                      ws.numel(), _stream(stream)))
    return bmu, dist


def som_probe_read(buf: torch.Tensor, nbytes: int, passes: int = 1, sink: Optional[torch.Tensor] = None,
                   stream=None) -> None:
    """Read-bandwidth probe over the first nbytes of a device tensor (see som.h)."""
    lib = load()
    if not buf.is_cuda or not buf.is_contiguous():
        raise ValueError("buf must be a contiguous ROCm device tensor")
    if nbytes > buf.numel() * buf.element_size():
        raise ValueError("nbytes exceeds the tensor")
    if sink is None:
        sink = torch.empty(1, dtype=torch.int32, device=buf.device)
    _check(lib.som_probe_read(_ptr(buf), int(nbytes), int(passes), _ptr(sink), _stream(stream)))


def som_probe_lds(iters: int, sink: torch.Tensor, stream=None) -> int:
    """LDS read probe (see som.h); returns the bytes the launch reads from LDS."""
    lib = load()
    _dev(sink, torch.int32, "sink")
    nbytes = ctypes.c_int64(0)
    _check(lib.som_probe_lds(int(iters), _ptr(sink), ctypes.byref(nbytes), _stream(stream)))
    return int(nbytes.value)



# ---------------------------------------------------------------------------
# Dense documents.  All tensors of a call are on one device, and it runs there, whichever
# device is the current one.
# ---------------------------------------------------------------------------

def _rows(t: torch.Tensor, name: str, dtype=None, shape=None, device=None):
    """Check a matrix of contiguous rows (device: the index of the first tensor's; None: this is
    it); return its pointer and row stride."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if device is None:
        if not t.is_cuda:
            raise ValueError(f"{name} must be on a ROCm device (got {t.device})")
    elif t.get_device() != device:
        raise ValueError(f"{name} must be on cuda:{device} like the first tensor (got {t.device})")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    size = t.shape
    if len(size) != 2:
        raise ValueError(f"{name} must have two dimensions")
    if shape is not None and size != shape:
        raise ValueError(f"{name} must be {shape[0]} x {shape[1]} (got {size[0]} x {size[1]})")
    rows, cols = size
    ld, one = t.stride()
    if one != 1 and cols > 1:
        raise ValueError(f"{name}: the elements of a row must be contiguous")
    if ld < cols:
        if rows > 1:
            raise ValueError(f"{name}: rows must not overlap")
        ld = cols
    return t.data_ptr(), ld


def _raw_stream(device: int, stream) -> int:
    """The given stream, which has to be the device's, or its current one (asked for by
    itself: torch.cuda.current_stream() takes longer than a launch)."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device)
    if getattr(stream, "device_index", device) != device:
        raise ValueError(f"stream must be one of cuda:{device}, like the tensors (got cuda:{stream.device_index})")
    return stream.cuda_stream


def _vector(t: Optional[torch.Tensor], name: str, n: int, device: int, dtype=torch.float32):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.get_device() != device:
        raise ValueError(f"{name} must be on cuda:{device} like the first tensor (got {t.device})")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    if t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must have {n} contiguous entries")
    return t.data_ptr()


def _float_type(t: torch.Tensor, name: str, types) -> int:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.dtype not in types:
        raise TypeError(f"{name} must be one of {', '.join(str(x) for x in types)} (got {t.dtype})")
    return DTYPES[t.dtype]


_FLOATS = (torch.float32, torch.float16, torch.bfloat16)
_HALVES = (torch.float16, torch.bfloat16)


def _weights(W: torch.Tensor, name: str, dtype, device: int):
    """A K x N weight matrix: (pointer, row stride, 1 if unit-major).

    Feature-major rows (W[k, :] contiguous, like a codebook) or, as the
    transposed view of an N x K matrix, unit-major ones."""
    if not isinstance(W, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if W.dim() != 2:
        raise ValueError(f"{name} must have two dimensions")
    units = W.stride(0) == 1 and (W.stride(1) != 1 or dtype == torch.float8_e4m3fn)
    p, ld = _rows(W.t() if units else W, name, dtype, None, device)
    return p, ld, int(units)


def _new(shape, dtype, device, stream):
    """An output.  On a stream that is not the current one it is that stream's memory
    (nothing earlier on the current one can still use it), which is not handed out
    again before the current stream, whose caller has it, is done with it either."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    t.record_stream(torch.cuda.current_stream(device))
    return t


def _scratch(ws, need: int, device, stream):
    """(tensor, pointer, bytes) of the workspace: the caller's, or one for this call, of
    the memory of the stream that uses it: it is free for that stream's next call only."""
    if ws is None:
        if need == 0:
            return None, None, 0
        if stream is None:
            ws = torch.empty(need, dtype=torch.uint8, device=device)
        else:
            with torch.cuda.stream(stream):
                ws = torch.empty(need, dtype=torch.uint8, device=device)
    else:
        _dev(ws, torch.uint8, "ws")
        if ws.device != device:
            raise ValueError(f"ws must be on {device} like the first tensor (got {ws.device})")
    return ws, ws.data_ptr(), ws.numel()


def _unwanted(need: bool, given: Optional[torch.Tensor], name: str) -> None:
    if not need and given is not None:
        raise ValueError(f"{name} goes with need_{name}")


def som_rms_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                 residual: Optional[torch.Tensor] = None, q8: bool = False, y: Optional[torch.Tensor] = None,
                 h: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None, stream=None):
    """(y, h, scale) of the root-mean-square norm of the rows of x + residual.

    h = x + residual (None without a residual, unless given), y = h /
    sqrt(mean h^2 + eps) * weight in x's type (fp32, fp16, bf16).  With ``q8`` y
    is float8_e4m3fn and scale (fp32, else None) holds each row's factor:
    y * scale[:, None] is the norm.  ``h`` may be x or the residual, which
    updates a residual stream in place."""
    lib = load()
    dt = _float_type(x, "x", _FLOATS)
    xp, ldx = _rows(x, "x")
    device = x.get_device()
    if torch._C._cuda_getDevice() != device:       # a launch goes to the current one
        with torch.cuda.device(device):
            return som_rms_norm(x, weight, eps, residual, q8, y, h, scale, stream)
    rows, cols = x.shape
    shape = x.shape
    rp, ldr = (None, 0) if residual is None else _rows(residual, "residual", x.dtype, shape, device)
    wp = _vector(weight, "weight", cols, device, x.dtype)
    yt = torch.float8_e4m3fn if q8 else x.dtype
    if y is None:
        y = _new(shape, yt, x.device, stream)
    yp, ldy = _rows(y, "y", yt, shape, device)
    if h is None and residual is not None:
        h = _new(shape, x.dtype, x.device, stream)
    hp, ldh = (None, 0) if h is None else _rows(h, "h", x.dtype, shape, device)
    if q8 and scale is None:
        scale = _new(rows, torch.float32, x.device, stream)
    if scale is not None and not q8:
        raise ValueError("scale goes with q8")
    sp = _vector(scale, "scale", rows, device)
    _check(lib.som_rms_norm(xp, ldx, rp, ldr, wp, dt, rows, cols, eps, 1 if q8 else 0, yp, ldy, hp, ldh, sp,
                            _raw_stream(device, stream)))
    return y, h, scale


def som_rms_norm_backward(dy: torch.Tensor, h: torch.Tensor, weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                          dh: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None,
                          dweight: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None,
                          need_dweight: bool = True):
    """(dx, dweight) of som_rms_norm: from the gradient of y, the h it returned (x
    without a residual) and the gradient ``dh`` that reaches h itself.  dx is the
    gradient of x and of the residual; dweight is fp32, or None (and not calculated)
    without ``need_dweight``."""
    lib = load()
    dt = _float_type(h, "h", _FLOATS)
    hp, ldh = _rows(h, "h")
    device = h.get_device()
    if torch._C._cuda_getDevice() != device:       # a launch goes to the current one
        with torch.cuda.device(device):
            return som_rms_norm_backward(dy, h, weight, eps, dh, dx, dweight, ws, stream, need_dweight)
    rows, cols = h.shape
    shape = (rows, cols)
    gp, ldg = _rows(dy, "dy", h.dtype, shape, device)
    wp = _vector(weight, "weight", cols, device, h.dtype)
    ep, lde = (None, 0) if dh is None else _rows(dh, "dh", h.dtype, shape, device)
    if dx is None:
        dx = _new(shape, h.dtype, h.device, stream)
    xp, ldx = _rows(dx, "dx", h.dtype, shape, device)
    if need_dweight and dweight is None:
        dweight = _new(cols, torch.float32, h.device, stream)
    _unwanted(need_dweight, dweight, "dweight")
    dwp = _vector(dweight, "dweight", cols, device)
    ws, wsp, n = _scratch(ws, lib.som_rms_norm_backward_workspace_bytes(rows, cols), h.device, stream)
    _check(lib.som_rms_norm_backward(gp, ldg, hp, ldh, wp, ep, lde, dt, rows, cols, eps, xp, ldx, dwp, wsp, n,
                                     _raw_stream(device, stream)))
    return dx, dweight


def som_product_workspace_bytes(M: int, N: int, K: int, dtype=torch.bfloat16) -> int:
    return int(load().som_product_workspace_bytes(M, N, K, DTYPES[dtype]))


def som_product(x: torch.Tensor, W: torch.Tensor, bias: Optional[torch.Tensor] = None, act: str = "none",
                residual: Optional[torch.Tensor] = None, alpha: float = 1.0,
                x_scale: Optional[torch.Tensor] = None, w_scale: Optional[torch.Tensor] = None,
                y: Optional[torch.Tensor] = None, dtype=None, pre: Optional[torch.Tensor] = None,
                ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """act(alpha x_scale w_scale (x @ W) + bias) + residual.

    x [M, K] and W [K, N] in fp16, bf16 or float8_e4m3fn; W with contiguous rows
    (feature-major, like a codebook) or as the transposed view of an N x K matrix
    (unit-major; the only layout of 8-bit weights).  y has type ``dtype`` (x's, or
    fp32; 8-bit x: bf16 unless given).  bias [N], x_scale [M] and w_scale [N] are fp32.
    act: none, relu, gelu, gelu_tanh or silu.  ``pre`` (like y), if given, receives
    the activation's argument for som_product_backward.  A dense document's scores
    against a codebook: alpha=-2, bias=its norms, dtype=torch.float32."""
    lib = load()
    xt = _float_type(x, "x", (*_HALVES, torch.float8_e4m3fn))
    xp, ldx = _rows(x, "x")
    device = x.get_device()
    if torch._C._cuda_getDevice() != device:       # a launch goes to the current one
        with torch.cuda.device(device):
            return som_product(x, W, bias, act, residual, alpha, x_scale, w_scale, y, dtype, pre, ws, stream)
    M, K = x.shape
    Wp, ldw, units = _weights(W, "W", x.dtype, device)
    if W.shape[0] != K:
        raise ValueError(f"x has {K} columns and W {W.shape[0]} rows")
    N = W.shape[1]
    if act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {', '.join(ACTIVATIONS)}")
    shape = (M, N)
    if y is None:
        y = _new(shape, dtype or (torch.bfloat16 if xt == 3 else x.dtype), x.device, stream)
    elif dtype is not None and y.dtype != dtype:
        raise TypeError(f"y must be {dtype} (got {y.dtype})")
    yt = _float_type(y, "y", _FLOATS)
    yp, ldy = _rows(y, "y", None, shape, device)
    rp, ldr = (None, 0) if residual is None else _rows(residual, "residual", y.dtype, shape, device)
    pp, ldp = (None, 0) if pre is None else _rows(pre, "pre", y.dtype, shape, device)
    e = som_epilogue(ACTIVATIONS[act], 0, alpha, _vector(x_scale, "x_scale", M, device),
                     _vector(w_scale, "w_scale", N, device), _vector(bias, "bias", N, device), rp, ldr, pp, ldp)
    ws, wsp, n = _scratch(ws, lib.som_product_workspace_bytes(M, N, K, xt), x.device, stream)
    _check(lib.som_product(xp, ldx, Wp, ldw, units, xt, M, N, K, yp, ldy, yt, ctypes.byref(e), wsp, n,
                           _raw_stream(device, stream)))
    return y


def som_product_backward_workspace_bytes(M: int, N: int, K: int, dtype=torch.bfloat16) -> int:
    return int(load().som_product_backward_workspace_bytes(M, N, K, DTYPES[dtype]))


def som_product_backward(dy: torch.Tensor, x: torch.Tensor, W: torch.Tensor, act: str = "none",
                         pre: Optional[torch.Tensor] = None, alpha: float = 1.0, dx: Optional[torch.Tensor] = None,
                         dW: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None,
                         ws: Optional[torch.Tensor] = None, stream=None, need_dx: bool = True, need_dW: bool = True,
                         need_dbias: bool = True):
    """(dx, dW, dbias) of som_product, in x's type (fp16 or bf16), dW laid out as W
    is; dbias is fp32.  ``pre`` is what som_product stored (not needed without an
    activation).  The residual's gradient is dy.  One that is not needed is None, and its
    product or sum is left out."""
    lib = load()
    dt = _float_type(x, "x", _HALVES)
    xp, ldx = _rows(x, "x")
    device = x.get_device()
    if torch._C._cuda_getDevice() != device:       # a launch goes to the current one
        with torch.cuda.device(device):
            return som_product_backward(dy, x, W, act, pre, alpha, dx, dW, dbias, ws, stream, need_dx, need_dW,
                                        need_dbias)
    M, K = x.shape
    Wp, ldw, units = _weights(W, "W", x.dtype, device)
    if W.shape[0] != K:
        raise ValueError(f"x has {K} columns and W {W.shape[0]} rows")
    N = W.shape[1]
    gp, ldg = _rows(dy, "dy", x.dtype, (M, N), device)
    if act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {', '.join(ACTIVATIONS)}")
    if pre is None and act != "none":
        raise ValueError("pre is needed for an activation's gradient")
    pp, ldp = (None, 0) if pre is None else _rows(pre, "pre", x.dtype, (M, N), device)
    for need, given, name in ((need_dx, dx, "dx"), (need_dW, dW, "dW"), (need_dbias, dbias, "dbias")):
        _unwanted(need, given, name)
    if need_dx and dx is None:
        dx = _new((M, K), x.dtype, x.device, stream)
    dxp, lddx = (None, 0) if dx is None else _rows(dx, "dx", x.dtype, (M, K), device)
    if need_dW and dW is None:
        dW = _new((N, K), x.dtype, x.device, stream).t() if units else _new((K, N), x.dtype, x.device, stream)
    dWp, lddw = (None, 0) if dW is None else _rows(dW.t() if units else dW, "dW", x.dtype,
                                                   (N, K) if units else (K, N), device)
    if need_dbias and dbias is None:
        dbias = _new(N, torch.float32, x.device, stream)
    dbp = _vector(dbias, "dbias", N, device)
    ws, wsp, n = _scratch(ws, lib.som_product_backward_workspace_bytes(M, N, K, dt), x.device, stream)
    _check(lib.som_product_backward(gp, ldg, xp, ldx, Wp, ldw, units, dt, M, N, K, ACTIVATIONS[act], pp, ldp, alpha,
                                    dxp, lddx, dWp, lddw, dbp, wsp, n, _raw_stream(device, stream)))
    return dx, dW, dbias


def som_dropout(x: torch.Tensor, p: float, seed: int, offset: int = 0, residual: Optional[torch.Tensor] = None,
                y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """x with each element dropped at rate p (a multiple of 2^-16, rounded to), the kept
    ones divided by the share kept, plus the residual.  The mask is a function of
    (seed, offset, row, column): the same call on the gradient is the backward pass."""
    lib = load()
    dt = _float_type(x, "x", _FLOATS)
    xp, ldx = _rows(x, "x")
    device = x.get_device()
    if torch._C._cuda_getDevice() != device:       # a launch goes to the current one
        with torch.cuda.device(device):
            return som_dropout(x, p, seed, offset, residual, y, stream)
    rows, cols = x.shape
    shape = (rows, cols)
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        raise ValueError("seed and offset must be in [0, 2^64)")
    rp, ldr = (None, 0) if residual is None else _rows(residual, "residual", x.dtype, shape, device)
    if y is None:
        y = _new(shape, x.dtype, x.device, stream)
    yp, ldy = _rows(y, "y", x.dtype, shape, device)
    _check(lib.som_dropout(xp, ldx, rp, ldr, dt, rows, cols, p, seed, offset, yp, ldy, _raw_stream(device, stream)))
    return y
