"""ctypes binding with the names of include/kimad.h.  Argument marshalling only."""
from __future__ import annotations

import ctypes as C
import os
from typing import List, Optional, Sequence

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libkimad.so")

KIMAD_REUSE_PROFILE = 1
KIMAD_CFG_CLASSIC_PROFILE = 1
KIMAD_CFG_FULL_DP = 2
KIMAD_CFG_BAND_DP = 4
KIMAD_CFG_DENSE_FALLBACK = 8
KIMAD_CFG_SAMPLE_ALWAYS = 16
KIMAD_VALUES_F32 = 0
KIMAD_VALUES_F16 = 1
KIMAD_VALUES_BF16 = 2
KIMAD_MAX_J = 64
KIMAD_ERR_WORKSPACE_TOO_SMALL = -2
KIMAD_ACT_NONE = 0
KIMAD_ACT_RELU = 1
KIMAD_ACT_GELU = 2
KIMAD_ACT_SILU = 3
KIMAD_WANT_DX = 1
KIMAD_WANT_DW = 2
KIMAD_WANT_DB = 4
FEW_ROWS = 96                                                    # products of so many rows may go by a kernel that needs no workspace

EXPORTED_SYMBOLS = [
    "kimad_workspace_bytes", "kimad_plan_create", "kimad_plan_destroy", "kimad_plan_grid_sizes",
    "kimad_profile", "kimad_allocate", "kimad_allocate_static", "kimad_compress_ef", "kimad_step",
    "kimad_error_at", "kimad_uniform_sizes", "kimad_payload_layer_counts",
    "kimad_profile_diagnostics", "kimad_allocate_diagnostics", "kimad_allocate_route", "kimad_plan_layer_states",
    "kimad_plan_set_timing", "kimad_plan_get_timings",
    "kimad_server_apply", "kimad_selftest_wave_primitives", "kimad_selftest_allocate_withheld",
    "kimad_budget_bytes", "kimad_strerror", "kimad_version",
    "kimad_mx4_quantise", "kimad_mx4_dequantise", "kimad_mx4_matmul", "kimad_mx4_matmul_workspace_bytes",
    "kimad_mx4_update_words", "kimad_mx4_compress_ef", "kimad_mx4_server_apply",
    "kimad_distill", "kimad_distill_grad", "kimad_distill_workspace_bytes",
    "kimad_linear", "kimad_linear_workspace_bytes", "kimad_linear_grad", "kimad_linear_grad_workspace_bytes",
    "kimad_linear_xent", "kimad_linear_xent_workspace_bytes", "kimad_dropout",
]


class KimadError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {kimad_strerror(code)} ({code})")


class _Layer(C.Structure):
    _fields_ = [("g", C.c_void_p), ("h", C.c_void_p), ("n", C.c_uint64)]


class _Payload(C.Structure):
    _fields_ = [("idx", C.c_void_p), ("val", C.c_void_p), ("offsets", C.c_void_p), ("capacity_pairs", C.c_uint64),
                ("value_format", C.c_uint32), ("pad", C.c_uint32)]


class _Mx4Update(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p)]


class _Config(C.Structure):
    _fields_ = [("pair_bytes", C.c_uint32), ("cost_units_D", C.c_uint32),
                ("max_budget_bytes", C.c_uint64), ("flags", C.c_uint64),
                ("max_workgroups", C.c_uint32), ("value_format", C.c_uint32)]


_lib = None


def lib() -> C.CDLL:
    """Load libkimad.so (built by paper_2312_08053_amd.build).  Fails loudly when it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: run `python -m paper_2312_08053_amd.build` (there is no CPU fallback)")
    L = C.CDLL(LIB_PATH)
    vp, u32, u64, i32p = C.c_void_p, C.c_uint32, C.c_uint64, C.c_void_p
    L.kimad_workspace_bytes.argtypes = [C.POINTER(C.c_uint64), u32, u32, C.POINTER(_Config), C.POINTER(C.c_uint64)]
    L.kimad_plan_create.argtypes = [C.POINTER(_Layer), u32, C.POINTER(C.c_double), u32, C.POINTER(_Config),
                                    vp, u64, vp, C.POINTER(vp)]
    L.kimad_plan_destroy.argtypes = [vp]
    L.kimad_plan_grid_sizes.argtypes = [vp, C.POINTER(C.c_uint64)]
    L.kimad_profile.argtypes = [vp, vp, u64, vp]
    L.kimad_allocate.argtypes = [vp, vp, u64, vp, vp, vp, i32p, vp]
    L.kimad_allocate_static.argtypes = [vp, vp, u64, vp, vp, vp, i32p, vp]
    L.kimad_compress_ef.argtypes = [vp, vp, vp, vp, vp, u64, u32, i32p, vp]
    L.kimad_step.argtypes = [vp, u64, vp, vp, vp, vp, vp, vp, u64, i32p, vp]
    L.kimad_error_at.argtypes = [vp, vp, vp, vp]
    L.kimad_uniform_sizes.argtypes = [C.POINTER(C.c_uint64), u32, u64, u32, C.POINTER(C.c_uint64), C.POINTER(C.c_uint64)]
    L.kimad_payload_layer_counts.argtypes = [vp, u64, vp, u32, vp, vp]
    L.kimad_profile_diagnostics.argtypes = [vp, C.POINTER(C.c_uint32), vp]
    L.kimad_allocate_diagnostics.argtypes = [vp, C.POINTER(C.c_uint32), vp]
    L.kimad_allocate_route.argtypes = [vp, C.POINTER(C.c_uint32), vp]
    L.kimad_plan_layer_states.argtypes = [vp, C.POINTER(C.c_uint32), u32, C.POINTER(C.c_uint32), vp]
    L.kimad_plan_set_timing.argtypes = [vp, C.c_int]
    L.kimad_plan_get_timings.argtypes = [vp, C.c_char_p, u32, C.POINTER(C.c_float), u32, C.POINTER(C.c_uint32)]
    L.kimad_server_apply.argtypes = [C.POINTER(_Payload), C.POINTER(C.c_void_p), C.POINTER(C.c_double), u32, vp, u32, u64,
                                     vp, C.c_double, vp, vp]
    L.kimad_selftest_wave_primitives.argtypes = [vp, vp, vp, vp, vp]
    L.kimad_selftest_allocate_withheld.argtypes = [vp, vp, u64, vp, vp, vp, i32p, u32, vp, vp]
    f32 = C.c_float
    L.kimad_mx4_quantise.argtypes = [vp, u32, u64, u64, u64, vp, vp, vp, vp, vp]
    L.kimad_mx4_dequantise.argtypes = [vp, vp, u64, u64, vp, u32, u64, vp]
    L.kimad_mx4_matmul_workspace_bytes.argtypes = [u64, u64, u64]
    L.kimad_mx4_matmul.argtypes = [vp, vp, u64, vp, vp, u64, u64, vp, u32, u64, vp, u64, vp]
    L.kimad_mx4_update_words.argtypes = [u32, u64]
    L.kimad_mx4_compress_ef.argtypes = [vp, vp, vp, u32, u64, vp, vp, vp, vp]
    L.kimad_mx4_server_apply.argtypes = [C.POINTER(_Mx4Update), C.POINTER(C.c_void_p), C.POINTER(C.c_double), u32, vp, u32, u64,
                                         vp, C.c_double, vp, vp]
    L.kimad_distill_workspace_bytes.argtypes = [u64, u64, u32]
    L.kimad_distill.argtypes = [vp, u32, u64, u64, u64, vp, vp, u32, f32, vp, vp, vp, vp, u64, vp, u64, vp]
    L.kimad_distill_grad.argtypes = [vp, u32, u64, u64, u64, vp, vp, u32, f32, vp, vp, vp, u64, vp]
    L.kimad_linear_workspace_bytes.argtypes = [vp, u64, vp, u64, u64, u64, u64]
    L.kimad_linear.argtypes = [vp, u64, vp, u64, u32, u64, u64, u64, vp, vp, u64, u32, vp, u64, vp, u32, u64, vp, u64, vp]
    L.kimad_linear_grad_workspace_bytes.argtypes = [vp, u64, vp, u64, vp, u64, u64, u64, u64, u32, u32]
    L.kimad_linear_grad.argtypes = [vp, u64, vp, u64, vp, u64, vp, u64, u32, u64, u64, u64, u32, vp, u64, vp, u32, u64, vp, vp, u64, vp]
    L.kimad_linear_xent_workspace_bytes.argtypes = [vp, u64, vp, u64, u32, u64, u64, u64, u32, u32]
    L.kimad_linear_xent.argtypes = [vp, u64, vp, u64, u32, u64, u64, u64, vp, vp, vp, vp, vp, u64, vp, u32, u64, vp, u64, vp]
    L.kimad_dropout.argtypes = [vp, u32, u64, u64, u64, vp, u64, C.c_double, u64, u64, vp, u64, vp]
    L.kimad_strerror.argtypes = [C.c_int]
    L.kimad_strerror.restype = C.c_char_p
    L.kimad_version.restype = C.c_char_p
    for name in EXPORTED_SYMBOLS:
        if name not in ("kimad_strerror", "kimad_version", "kimad_budget_bytes"):
            getattr(L, name).restype = C.c_int
    L.kimad_budget_bytes.argtypes = [C.c_double, C.c_double, C.c_double, C.c_double, C.c_uint64]
    for name in ("kimad_budget_bytes", "kimad_mx4_matmul_workspace_bytes", "kimad_mx4_update_words", "kimad_distill_workspace_bytes",
                 "kimad_linear_workspace_bytes", "kimad_linear_grad_workspace_bytes", "kimad_linear_xent_workspace_bytes"):
        getattr(L, name).restype = C.c_uint64
    _lib = L
    return L


def kimad_strerror(code: int) -> str:
    return lib().kimad_strerror(int(code)).decode()


def kimad_budget_bytes(bandwidth_bits_per_s: float, t_seconds: float, t_comp_seconds: float, alpha: float = 1.0,
                       cap_bytes: int = 0) -> int:
    return int(lib().kimad_budget_bytes(float(bandwidth_bits_per_s), float(t_seconds), float(t_comp_seconds),
                                        float(alpha), int(cap_bytes)))


def kimad_version() -> str:
    return lib().kimad_version().decode()


def _cfg(pair_bytes=8, D=0, max_budget_bytes=0, cfg_flags=0, max_workgroups=0, value_format=0) -> _Config:
    return _Config(int(pair_bytes), int(D), int(max_budget_bytes), int(cfg_flags), int(max_workgroups), int(value_format))


def _check(code: int, where: str) -> None:
    if code != 0:
        raise KimadError(code, where)


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


_cuda = _current_stream = None                                  # torch.cuda, and the handle of a device's current stream


def _with_torch() -> None:
    global _cuda, _current_stream
    import torch
    _cuda = torch.cuda
    # (the same number without an object around it)
    _current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: int(torch.cuda.current_stream(device).cuda_stream))


def _stream(stream) -> int:
    if stream is not None:
        return int(getattr(stream, "cuda_stream", stream))
    if _cuda is None:
        _with_torch()
    return _current_stream(_cuda.current_device())


def _scratch(nbytes: int, device, stream):
    """Device memory for one call on `stream`.  It comes from that stream's own pool: memory of another stream's would go
    to that stream's next allocation as soon as the call returns, with the kernels still to run."""
    import torch
    handle = _stream(stream)
    if handle == _stream(None):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    with torch.cuda.stream(torch.cuda.ExternalStream(handle, device=device) if handle else torch.cuda.default_stream(device)):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


def kimad_workspace_bytes(sizes: Sequence[int], J: int, pair_bytes=8, D=0, max_budget_bytes=0,
                          cfg_flags=0, max_workgroups=0, value_format=0) -> int:
    n = (C.c_uint64 * len(sizes))(*[int(s) for s in sizes])
    out = C.c_uint64(0)
    cfg = _cfg(pair_bytes, D, max_budget_bytes, cfg_flags, max_workgroups, value_format)
    _check(lib().kimad_workspace_bytes(n, len(sizes), int(J), C.byref(cfg), C.byref(out)), "kimad_workspace_bytes")
    return int(out.value)


def kimad_plan_create(g_ptrs: Sequence[int], h_ptrs: Sequence[int], sizes: Sequence[int], ratios: Sequence[float],
                      workspace_ptr: int, workspace_bytes: int, stream=None, pair_bytes=8, D=0,
                      max_budget_bytes=0, cfg_flags=0, max_workgroups=0, value_format=0) -> int:
    L = len(sizes)
    layers = (_Layer * L)()
    for i in range(L):
        layers[i].g, layers[i].h, layers[i].n = int(g_ptrs[i]), int(h_ptrs[i]), int(sizes[i])
    r = (C.c_double * len(ratios))(*[float(x) for x in ratios])
    cfg = _cfg(pair_bytes, D, max_budget_bytes, cfg_flags, max_workgroups, value_format)
    plan = C.c_void_p(0)
    _check(lib().kimad_plan_create(layers, L, r, len(ratios), C.byref(cfg), C.c_void_p(int(workspace_ptr)),
                                   int(workspace_bytes), C.c_void_p(_stream(stream)), C.byref(plan)),
           "kimad_plan_create")
    return int(plan.value)


def kimad_plan_destroy(plan: int) -> None:
    _check(lib().kimad_plan_destroy(C.c_void_p(plan)), "kimad_plan_destroy")


def kimad_profile(plan: int, err_table, budget_hint_bytes: int = 0, stream=None) -> None:
    _check(lib().kimad_profile(C.c_void_p(plan), C.c_void_p(_ptr(err_table)), int(budget_hint_bytes),
                               C.c_void_p(_stream(stream))), "kimad_profile")


def kimad_allocate(plan: int, err_table, budget_bytes: int, j_out, K_out, offsets_out, status_out,
                   stream=None) -> None:
    _check(lib().kimad_allocate(C.c_void_p(plan), C.c_void_p(_ptr(err_table)), int(budget_bytes),
                                C.c_void_p(_ptr(j_out)), C.c_void_p(_ptr(K_out)), C.c_void_p(_ptr(offsets_out)),
                                C.c_void_p(_ptr(status_out)), C.c_void_p(_stream(stream))), "kimad_allocate")


def kimad_allocate_static(plan: int, err_table, budget_bytes: int, j_out, K_out, offsets_out, status_out,
                          stream=None) -> None:
    _check(lib().kimad_allocate_static(C.c_void_p(plan), C.c_void_p(_ptr(err_table)), int(budget_bytes),
                                       C.c_void_p(_ptr(j_out)), C.c_void_p(_ptr(K_out)), C.c_void_p(_ptr(offsets_out)),
                                       C.c_void_p(_ptr(status_out)), C.c_void_p(_stream(stream))), "kimad_allocate_static")


def kimad_compress_ef(plan: int, K, offsets, idx_out, val_out, capacity_pairs: int, flags: int, status_out,
                      stream=None) -> None:
    _check(lib().kimad_compress_ef(C.c_void_p(plan), C.c_void_p(_ptr(K)), C.c_void_p(_ptr(offsets)),
                                   C.c_void_p(_ptr(idx_out)), C.c_void_p(_ptr(val_out)), int(capacity_pairs),
                                   int(flags), C.c_void_p(_ptr(status_out)), C.c_void_p(_stream(stream))),
           "kimad_compress_ef")


def kimad_step(plan: int, budget_bytes: int, err_table, j_out, K_out, offsets_out, idx_out, val_out,
               capacity_pairs: int, status_out, stream=None) -> None:
    _check(lib().kimad_step(C.c_void_p(plan), int(budget_bytes), C.c_void_p(_ptr(err_table)),
                            C.c_void_p(_ptr(j_out)), C.c_void_p(_ptr(K_out)), C.c_void_p(_ptr(offsets_out)),
                            C.c_void_p(_ptr(idx_out)), C.c_void_p(_ptr(val_out)), int(capacity_pairs),
                            C.c_void_p(_ptr(status_out)), C.c_void_p(_stream(stream))), "kimad_step")


def kimad_error_at(plan: int, K, err_out, stream=None) -> None:
    _check(lib().kimad_error_at(C.c_void_p(plan), C.c_void_p(_ptr(K)), C.c_void_p(_ptr(err_out)),
                                C.c_void_p(_stream(stream))), "kimad_error_at")


def kimad_uniform_sizes(sizes: Sequence[int], budget_bytes: int, pair_bytes: int = 8):
    """([K_i], pairs of the whole-model TopK of the same budget): host arithmetic of the library."""
    L = len(sizes)
    n = (C.c_uint64 * L)(*[int(s) for s in sizes])
    out = (C.c_uint64 * L)()
    pairs = C.c_uint64(0)
    _check(lib().kimad_uniform_sizes(n, L, int(budget_bytes), int(pair_bytes), out, C.byref(pairs)), "kimad_uniform_sizes")
    return [int(v) for v in out], int(pairs.value)


def kimad_payload_layer_counts(idx, pairs: int, layer_start, counts_out, stream=None) -> None:
    _check(lib().kimad_payload_layer_counts(C.c_void_p(_ptr(idx)), int(pairs), C.c_void_p(_ptr(layer_start)),
                                            int(layer_start.numel()) - 1, C.c_void_p(_ptr(counts_out)),
                                            C.c_void_p(_stream(stream))), "kimad_payload_layer_counts")


def kimad_server_apply(payloads, u_hats, weights, layer_start, d: int, x=None, gamma: float = 0.0, stream=None,
                       status_out=None):
    """payloads: list of (idx, val, offsets) device tensors, one per worker; u_hats: list of flat fp32
    device tensors (updated in place); layer_start: device uint64/int64 tensor [L+1]; x: flat fp32 model
    or None; status_out: device int32[M] (allocated here if None).  Returns status_out."""
    M = len(u_hats)
    def cap(i, v):
        return 0 if i is None or v is None else min(int(i.numel()), int(v.numel()))

    def fmt(v):                                           # half-precision payloads are torch.float16 tensors
        return KIMAD_VALUES_F16 if v is not None and v.element_size() == 2 else KIMAD_VALUES_F32
    pl = (_Payload * M)(*[_Payload(_ptr(i), _ptr(v), _ptr(o), cap(i, v), fmt(v), 0) for (i, v, o) in payloads])
    uh = (C.c_void_p * M)(*[_ptr(u) for u in u_hats])
    w = (C.c_double * M)(*[float(t) for t in weights])
    if status_out is None:
        import torch
        status_out = torch.empty(M, dtype=torch.int32, device=u_hats[0].device)
    _check(lib().kimad_server_apply(pl, uh, w, M, C.c_void_p(_ptr(layer_start)), int(layer_start.numel()) - 1, int(d),
                                    C.c_void_p(_ptr(x) if x is not None else 0), float(gamma),
                                    C.c_void_p(_ptr(status_out)), C.c_void_p(_stream(stream))), "kimad_server_apply")
    return status_out


def kimad_selftest_wave_primitives(in_u32, in_f64, out_u32, out_f64, stream=None) -> None:
    _check(lib().kimad_selftest_wave_primitives(C.c_void_p(_ptr(in_u32)), C.c_void_p(_ptr(in_f64)), C.c_void_p(_ptr(out_u32)),
                                                C.c_void_p(_ptr(out_f64)), C.c_void_p(_stream(stream))),
           "kimad_selftest_wave_primitives")


def kimad_selftest_allocate_withheld(plan: int, err_table, budget_bytes: int, j_out, K_out, offsets_out, status_out,
                                     polls: int, given_up_out, stream=None) -> None:
    _check(lib().kimad_selftest_allocate_withheld(C.c_void_p(plan), C.c_void_p(_ptr(err_table)), int(budget_bytes),
                                                  C.c_void_p(_ptr(j_out)), C.c_void_p(_ptr(K_out)), C.c_void_p(_ptr(offsets_out)),
                                                  C.c_void_p(_ptr(status_out)), int(polls), C.c_void_p(_ptr(given_up_out)),
                                                  C.c_void_p(_stream(stream))), "kimad_selftest_allocate_withheld")


# Small calls take less time on the device than in here: what follows asks each tensor for little, and for most of it once.
_TYPES = {}


def _type(t) -> int:
    """KIMAD_VALUES_* of a tensor's type."""
    if not _TYPES:
        import torch
        _TYPES.update({torch.float32: KIMAD_VALUES_F32, torch.float16: KIMAD_VALUES_F16, torch.bfloat16: KIMAD_VALUES_BF16})
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise TypeError(f"float32, float16 or bfloat16 is wanted, got {t.dtype}")
    return kind


def _rows(t, what: str):
    """(rows, columns, elements from row to row) of a matrix whose rows are contiguous."""
    shape, strides = t.shape, t.stride()
    if len(shape) == 2:
        rows, cols = shape
        ld, one = strides
        if (one == 1 or cols <= 1) and (ld >= cols or rows <= 1):
            return rows, cols, ld if rows > 1 else cols
    raise ValueError(f"{what}: a matrix with contiguous rows is wanted, got shape {tuple(shape)}, strides {strides}")


class _Kinds(dict):
    def __missing__(self, dtype):
        import torch
        self.update({torch.float32: "float32", torch.int32: "int32", torch.uint32: "int32", torch.int64: "int64", torch.uint64: "int64",
                     torch.uint8: "uint8"})
        return self.setdefault(dtype, None)


_KINDS = _Kinds()                                                # torch is not imported before a tensor is there


def _holds(t, count: int, kind: str, what: str) -> int:
    """The address of a contiguous tensor of at least `count` elements of a kind: "float32", or "int32", "int64", "uint8", the whole numbers
    of so many bits (of the two larger ones, unsigned ones too)."""
    if _KINDS[t.dtype] != kind or t.numel() < count or not t.is_contiguous():
        raise ValueError(f"{what}: {count} contiguous elements of {kind} are wanted, got {t.numel()} of {t.dtype}, strides {t.stride()}")
    return t.data_ptr()


def _room(workspace):
    """Address and bytes of a workspace, a tensor of any type whose elements lie side by side; zeros without one."""
    if workspace is None:
        return 0, 0
    if not workspace.is_contiguous():
        raise ValueError(f"workspace: a contiguous tensor is wanted, got shape {tuple(workspace.shape)}, strides {workspace.stride()}")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _on_device(stream, *tensors) -> int:
    """The handle of the stream that a call on these tensors (or None) goes to.  Host memory is refused, and memory of another device than the one that the
    kernels run on: a kernel that reads it faults.  A given stream runs on its own device, the null stream and torch's current one on the
    current device."""
    where = None
    for t in tensors:
        if t is not None:
            device = t.get_device()
            if device != where:
                if device < 0:
                    raise ValueError(f"device tensors are wanted, got one of shape {tuple(t.shape)} on {t.device}")
                if where is not None:
                    raise ValueError(f"tensors of one device are wanted, got devices {where} and {device}")
                where = device
    if stream is not None:
        handle = _stream(stream)
        if handle:
            return handle
    if _cuda is None:
        _with_torch()
    if where != _cuda.current_device():
        raise ValueError(f"tensors of the current device are wanted, {_cuda.current_device()}, got device {where}")
    return _current_stream(where) if stream is None else handle


def _holds_mx4(codes, scales, rows: int, cols: int, what: str):
    """The addresses of a quantised matrix.  Its codes and scales have its own shape: both are laid out by it, so that a part of a
    larger matrix's is no smaller matrix.  One-dimensional ones are buffers with room for it, as through the C call."""
    words = (cols + 127) // 128
    if codes.shape == (rows, 64 * words) and scales.shape == (words, rows):
        if _KINDS[codes.dtype] == "uint8" and _KINDS[scales.dtype] == "int32" and codes.is_contiguous() and scales.is_contiguous():
            return codes.data_ptr(), scales.data_ptr()
    elif (codes.shape != (rows, 64 * words) and codes.dim() != 1) or (scales.shape != (words, rows) and scales.dim() != 1):
        raise ValueError(f"{what}: shapes {(rows, 64 * words)} and {(words, rows)} are wanted, got {tuple(codes.shape)} and {tuple(scales.shape)}")
    return _holds(codes, rows * words * 64, "uint8", what), _holds(scales, rows * words, "int32", what)


def mx4_empty(rows: int, cols: int, device="cuda"):
    """(codes uint8 [rows, 64 W], scales int32 [W, rows]) for a matrix in 4 bits, W = ceil(cols / 128); not filled."""
    import torch
    words = -(-int(cols) // 128)
    return (torch.empty(int(rows), 64 * words, dtype=torch.uint8, device=device),
            torch.empty(words, int(rows), dtype=torch.int32, device=device))


def kimad_mx4_quantise(x, codes=None, scales=None, codes_t=None, scales_t=None, stream=None) -> None:
    """x [rows, cols] along rows into codes, scales, along columns into codes_t, scales_t (each pair from mx4_empty for
    that shape, or flat buffers with room for it, or None)."""
    rows, cols, ld = _rows(x, "x")
    if (codes is None) != (scales is None) or (codes_t is None) != (scales_t is None):
        raise ValueError("codes and scales are wanted together")
    c, s = (0, 0) if codes is None else _holds_mx4(codes, scales, rows, cols, "codes and scales")
    ct, st = (0, 0) if codes_t is None else _holds_mx4(codes_t, scales_t, cols, rows, "codes_t and scales_t")
    kind = _type(x)
    handle = _on_device(stream, x, codes, scales, codes_t, scales_t)
    rc = lib().kimad_mx4_quantise(x.data_ptr(), kind, rows, cols, ld, c, s, ct, st, handle)
    if rc:
        _check(rc, "kimad_mx4_quantise")


def kimad_mx4_dequantise(codes, scales, out, stream=None) -> None:
    """The values of a quantised matrix into out [rows, cols]."""
    rows, cols, ld = _rows(out, "out")
    c, s = _holds_mx4(codes, scales, rows, cols, "codes and scales")
    kind = _type(out)
    handle = _on_device(stream, codes, scales, out)
    rc = lib().kimad_mx4_dequantise(c, s, rows, cols, out.data_ptr(), kind, ld, handle)
    if rc:
        _check(rc, "kimad_mx4_dequantise")


def kimad_mx4_matmul_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(lib().kimad_mx4_matmul_workspace_bytes(int(M), int(N), int(K)))


def kimad_mx4_matmul(a_codes, a_scales, b_codes, b_scales, K: int, out, workspace=None, stream=None) -> None:
    """out [M, N] = A B^T of quantised matrices A [M, K] and B [N, K].  workspace: a device tensor (allocated here if None and
    one is of use)."""
    M, N, ld = _rows(out, "out")
    a, sa = _holds_mx4(a_codes, a_scales, M, K, "A's codes and scales")
    b, sb = _holds_mx4(b_codes, b_scales, N, K, "B's codes and scales")
    kind = _type(out)
    ws, nbytes = _room(workspace)
    handle = _on_device(stream, a_codes, a_scales, b_codes, b_scales, out, workspace)
    L = lib()
    if workspace is None:
        nbytes = L.kimad_mx4_matmul_workspace_bytes(M, N, K)
        if nbytes:
            workspace = _scratch(nbytes, out.device, stream)
            ws = workspace.data_ptr()
    rc = L.kimad_mx4_matmul(a, sa, M, b, sb, N, K, out.data_ptr(), kind, ld, ws, nbytes, handle)
    if rc:
        _check(rc, "kimad_mx4_matmul")


def kimad_mx4_update_words(L: int, d: int) -> int:
    return int(lib().kimad_mx4_update_words(int(L), int(d)))


def kimad_mx4_compress_ef(g, h, layer_start, codes, scales, status_out=None, stream=None) -> None:
    """One worker's update in 4 bits: g, h flat fp32 tensors (h is updated in place), layer_start device int64[L+1], codes uint8
    [words, 64] and scales int32 [words] with words = kimad_mx4_update_words(L, d); status_out: device int32[1] or None."""
    d, L = g.numel(), layer_start.numel() - 1
    words = d // 128 + L
    args = (_holds(g, d, "float32", "g"), _holds(h, d, "float32", "h"), _holds(layer_start, 2, "int64", "layer_start"), L, d,
            _holds(codes, words * 64, "uint8", "codes"), _holds(scales, words, "int32", "scales"),
            0 if status_out is None else _holds(status_out, 1, "int32", "status_out"))
    handle = _on_device(stream, g, h, layer_start, codes, scales, status_out)
    rc = lib().kimad_mx4_compress_ef(*args, handle)
    if rc:
        _check(rc, "kimad_mx4_compress_ef")


def kimad_mx4_server_apply(updates, u_hats, weights, layer_start, d: int, x=None, gamma: float = 0.0, status_out=None,
                           stream=None) -> None:
    """updates: list of (codes, scales) as kimad_mx4_compress_ef writes them, one per worker; u_hats: list of flat fp32 tensors
    (updated in place); x: flat fp32 model or None; status_out: device int32[1] or None."""
    M, L, d = len(u_hats), layer_start.numel() - 1, int(d)
    words = d // 128 + L
    if len(updates) != M or len(weights) != M:
        raise ValueError(f"{M} estimators, {len(updates)} updates and {len(weights)} weights")
    up, uh, w = (_Mx4Update * M)(), (C.c_void_p * M)(), (C.c_double * M)(*weights)
    tensors = [layer_start, x, status_out, *u_hats]
    for m, (codes, scales) in enumerate(updates):
        tensors += (codes, scales)
        up[m].codes, up[m].scales = _holds(codes, words * 64, "uint8", "codes"), _holds(scales, words, "int32", "scales")
        uh[m] = _holds(u_hats[m], d, "float32", "u_hats")
    args = (up, uh, w, M, _holds(layer_start, 2, "int64", "layer_start"), L, d, 0 if x is None else _holds(x, d, "float32", "x"), gamma,
            0 if status_out is None else _holds(status_out, 1, "int32", "status_out"))
    handle = _on_device(stream, *tensors)
    rc = lib().kimad_mx4_server_apply(*args, handle)
    if rc:
        _check(rc, "kimad_mx4_server_apply")


def kimad_distill_workspace_bytes(rows: int, vocab: int, k: int) -> int:
    return int(lib().kimad_distill_workspace_bytes(int(rows), int(vocab), int(k)))


def _distill_inputs(logits, t_idx, t_val, row_weight, grad):
    """The leading arguments of both calls, and the trailing ones for row_weight and grad."""
    rows, vocab, ld = _rows(logits, "logits")
    kind = _type(logits)
    shape = t_idx.shape
    if len(shape) != 2 or shape[0] != rows or t_val.shape != shape:
        raise ValueError(f"entries: [rows, k] is wanted twice, got {tuple(shape)} and {tuple(t_val.shape)} for {rows} rows")
    k = shape[1]
    lead = (logits.data_ptr(), kind, rows, vocab, ld, _holds(t_idx, rows * k, "int32", "t_idx"), _holds(t_val, rows * k, "float32", "t_val"), k)
    weight = 0 if row_weight is None else _holds(row_weight, rows, "float32", "row_weight")
    if grad is None:
        return lead, weight, 0, 0
    g_rows, g_vocab, ld_grad = _rows(grad, "grad")
    if (g_rows, g_vocab) != (rows, vocab) or _type(grad) != kind:
        raise ValueError(f"grad: the logits' shape and type are wanted, got {tuple(grad.shape)} of {grad.dtype}")
    return lead, weight, grad.data_ptr(), ld_grad


def kimad_distill(logits, t_idx, t_val, temperature: float, loss=None, stats=None, grad=None, row_weight=None, workspace=None,
                  stream=None) -> None:
    """Distillation loss (float32 [rows]), statistics (float32 [rows, 2]) and gradient (like logits) of logits [rows, vocab]
    against a teacher's top entries t_idx int32, t_val float32 [rows, k]; an output that is None is left out."""
    lead, weight, g, ld_grad = _distill_inputs(logits, t_idx, t_val, row_weight, grad)
    _, _, rows, vocab, _, _, _, k = lead
    at_loss = 0 if loss is None else _holds(loss, rows, "float32", "loss")
    at_stats = 0 if stats is None else _holds(stats, 2 * rows, "float32", "stats")
    ws, nbytes = _room(workspace)
    handle = _on_device(stream, logits, t_idx, t_val, loss, stats, grad, row_weight, workspace)
    L = lib()
    if workspace is None:
        nbytes = L.kimad_distill_workspace_bytes(rows, vocab, k)
        if nbytes:
            workspace = _scratch(nbytes, logits.device, stream)
            ws = workspace.data_ptr()
    rc = L.kimad_distill(*lead, temperature, weight, at_loss, at_stats, g, ld_grad, ws, nbytes, handle)
    if rc:
        _check(rc, "kimad_distill")


def kimad_distill_grad(logits, t_idx, t_val, temperature: float, stats, grad, row_weight=None, stream=None) -> None:
    """The gradient alone, from the statistics of an earlier kimad_distill."""
    lead, weight, g, ld_grad = _distill_inputs(logits, t_idx, t_val, row_weight, grad)
    at = _holds(stats, 2 * lead[2], "float32", "stats")
    handle = _on_device(stream, logits, t_idx, t_val, stats, grad, row_weight)
    rc = lib().kimad_distill_grad(*lead, temperature, weight, at, g, ld_grad, handle)
    if rc:
        _check(rc, "kimad_distill_grad")


def _half(t, what: str) -> int:
    """KIMAD_VALUES_* of an operand of a product in 16 bits."""
    kind = _type(t)
    if kind == KIMAD_VALUES_F32:
        raise TypeError(f"{what}: float16 or bfloat16 is wanted, got {t.dtype}")
    return kind


def _matrix(t, shape, dtypes, what: str):
    """(address, elements from row to row) of a matrix of this shape and one of these types; zeros for None."""
    if t is None:
        return 0, 0
    rows, cols, ld = _rows(t, what)
    if (rows, cols) != shape or t.dtype not in dtypes:
        raise ValueError(f"{what}: shape {tuple(shape)} of {' or '.join(str(d) for d in dtypes)} is wanted, got {tuple(t.shape)} of {t.dtype}")
    return t.data_ptr(), ld


def _for_call(workspace, nbytes: int, device, stream):
    """(address, bytes, the tensor) of a call's workspace: the given one, or one from the stream's pool."""
    if workspace is not None:
        return *_room(workspace), workspace
    if not nbytes:
        return 0, 0, None
    workspace = _scratch(nbytes, device, stream)
    return workspace.data_ptr(), nbytes, workspace


def kimad_linear_workspace_bytes(x, w) -> int:
    """Bytes that kimad_linear of these operands needs."""
    (M, K, ld_x), (N, K2, ld_w) = _rows(x, "x"), _rows(w, "w")
    return int(lib().kimad_linear_workspace_bytes(x.data_ptr(), ld_x, w.data_ptr(), ld_w, M, N, K))


def kimad_linear(x, w, out, bias=None, residual=None, act: int = KIMAD_ACT_NONE, z=None, workspace=None, stream=None) -> None:
    """out [M, N] = act(x w^T + bias) + residual of x [M, K], w [N, K], bias [N], residual [M, N], all of one type, float16 or bfloat16; out
    may be float32 too, and may be residual itself.  act: KIMAD_ACT_*.  z [M, N] or None: what the activation is of, kept for
    kimad_linear_grad.  workspace: a device tensor (allocated here if None and one is needed)."""
    (M, K, ld_x), (N, K2, ld_w) = _rows(x, "x"), _rows(w, "w")
    kind, dtype = _half(x, "x"), x.dtype
    if K2 != K or w.dtype != dtype:
        raise ValueError(f"w: rows of {K} elements of {dtype} are wanted, got {K2} of {w.dtype}")
    out_kind = _type(out)
    at_out, ld_out = _matrix(out, (M, N), (dtype, out.dtype if out_kind == KIMAD_VALUES_F32 else dtype), "out")
    at_res, ld_res = _matrix(residual, (M, N), (dtype,), "residual")
    at_z, ld_z = _matrix(z, (M, N), (dtype,), "z")
    if bias is not None and (bias.shape != (N,) or bias.dtype != dtype or not bias.is_contiguous()):
        raise ValueError(f"bias: {N} contiguous elements of {dtype} are wanted, got {tuple(bias.shape)} of {bias.dtype}")
    handle = _on_device(stream, x, w, out, bias, residual, z, workspace)
    L = lib()
    args = (x.data_ptr(), ld_x, w.data_ptr(), ld_w, kind, M, N, K, _ptr(bias), at_res, ld_res, act, at_z, ld_z, at_out, out_kind, ld_out)
    if workspace is None and M <= FEW_ROWS:                      # (these seldom need one: asked for only then)
        rc = L.kimad_linear(*args, 0, 0, handle)
    else:
        rc = KIMAD_ERR_WORKSPACE_TOO_SMALL
    if rc == KIMAD_ERR_WORKSPACE_TOO_SMALL:
        need = 0 if workspace is not None else L.kimad_linear_workspace_bytes(*args[:4], M, N, K)
        ws, nbytes, kept = _for_call(workspace, need, x.device, stream)
        rc = L.kimad_linear(*args, ws, nbytes, handle)
    if rc:
        _check(rc, "kimad_linear")


def _linear_grad_inputs(dy, x, w, dx, dw, db):
    """(M, N, K, the six leading arguments, wants): x may be None where dw is, w where dx is."""
    M, N, ld_dy = _rows(dy, "dy")
    if (dx is not None and w is None) or (dw is not None and x is None):
        raise ValueError("w is wanted with dx, x with dw")
    K = w.shape[-1] if w is not None else x.shape[-1] if x is not None else 0
    at_x, ld_x = _matrix(x, (M, K), (dy.dtype,), "x")
    at_w, ld_w = _matrix(w, (N, K), (dy.dtype,), "w")
    wants = (KIMAD_WANT_DX if dx is not None else 0) | (KIMAD_WANT_DW if dw is not None else 0) | (KIMAD_WANT_DB if db is not None else 0)
    return M, N, K, (dy.data_ptr(), ld_dy, at_x, max(ld_x, K), at_w, max(ld_w, K)), wants


def kimad_linear_grad_workspace_bytes(dy, x, w, act: int = KIMAD_ACT_NONE, dx=None, dw=None, db=None) -> int:
    """Bytes that kimad_linear_grad with these arguments needs."""
    M, N, K, lead, wants = _linear_grad_inputs(dy, x, w, dx, dw, db)
    return int(lib().kimad_linear_grad_workspace_bytes(*lead, M, N, K, act, wants))


def kimad_linear_grad(dy, x, w, z=None, act: int = KIMAD_ACT_NONE, dx=None, dw=None, db=None, workspace=None, stream=None) -> None:
    """The gradient of kimad_linear: dx [M, K], dw [N, K] (float32 too), db float32 [N] from dy [M, N]; an output that is None is left out.  x may be
    None without dw, w without dx, z (as kimad_linear left it) without an activation.  The residual's gradient is dy."""
    M, N, K, lead, wants = _linear_grad_inputs(dy, x, w, dx, dw, db)
    kind, dtype = _half(dy, "dy"), dy.dtype
    if act and z is None:
        raise ValueError("z is wanted with an activation")
    at_z, ld_z = _matrix(z, (M, N), (dtype,), "z")
    at_dx, ld_dx = _matrix(dx, (M, K), (dtype,), "dx")
    dw_kind = kind if dw is None else _type(dw)
    at_dw, ld_dw = _matrix(dw, (N, K), (dtype, dw.dtype if dw_kind == KIMAD_VALUES_F32 else dtype) if dw is not None else (), "dw")
    at_db = 0 if db is None else _holds(db, N, "float32", "db")
    handle = _on_device(stream, dy, x, w, z, dx, dw, db, workspace)
    L = lib()
    need = 0 if workspace is not None else L.kimad_linear_grad_workspace_bytes(*lead, M, N, K, act, wants)
    ws, nbytes, kept = _for_call(workspace, need, dy.device, stream)
    rc = L.kimad_linear_grad(*lead, at_z, ld_z, kind, M, N, K, act, at_dx, ld_dx, at_dw, dw_kind, ld_dw, at_db, ws, nbytes, handle)
    if rc:
        _check(rc, "kimad_linear_grad")


def _xent_inputs(x, w, dx, dw):
    (rows, dim, ld_x), (vocab, dim2, ld_w) = _rows(x, "x"), _rows(w, "w")
    kind = _half(x, "x")
    if dim2 != dim or w.dtype != x.dtype:
        raise ValueError(f"w: rows of {dim} elements of {x.dtype} are wanted, got {dim2} of {w.dtype}")
    wants = (KIMAD_WANT_DX if dx is not None else 0) | (KIMAD_WANT_DW if dw is not None else 0)
    return rows, vocab, dim, (x.data_ptr(), ld_x, w.data_ptr(), ld_w, kind, rows, vocab, dim), wants, kind if dw is None else _type(dw)


def kimad_linear_xent_workspace_bytes(x, w, dx=None, dw=None) -> int:
    """Bytes that kimad_linear_xent with these arguments needs."""
    _, _, _, lead, wants, dw_kind = _xent_inputs(x, w, dx, dw)
    return int(lib().kimad_linear_xent_workspace_bytes(*lead, wants, dw_kind))


def kimad_linear_xent(x, w, target, loss=None, lse=None, dx=None, dw=None, row_weight=None, workspace=None, stream=None) -> None:
    """Cross entropy of the head w [vocab, dim] on x [rows, dim] (one type, float16 or bfloat16) against target int32 [rows] (none: below 0, or vocab and
    more), each row's times row_weight float32 [rows]: loss and lse float32 [rows], dx [rows, dim], dw [vocab, dim] (float32 too);
    an output that is None is left out.  workspace: a device tensor (allocated here if None)."""
    rows, vocab, dim, lead, wants, dw_kind = _xent_inputs(x, w, dx, dw)
    at_target = _holds(target, rows, "int32", "target")
    at_weight = 0 if row_weight is None else _holds(row_weight, rows, "float32", "row_weight")
    at_loss = 0 if loss is None else _holds(loss, rows, "float32", "loss")
    at_lse = 0 if lse is None else _holds(lse, rows, "float32", "lse")
    at_dx, ld_dx = _matrix(dx, (rows, dim), (x.dtype,), "dx")
    at_dw, ld_dw = _matrix(dw, (vocab, dim), (x.dtype, dw.dtype if dw_kind == KIMAD_VALUES_F32 else x.dtype) if dw is not None else (), "dw")
    handle = _on_device(stream, x, w, target, loss, lse, dx, dw, row_weight, workspace)
    L = lib()
    need = 0 if workspace is not None else L.kimad_linear_xent_workspace_bytes(*lead, wants, dw_kind)
    ws, nbytes, kept = _for_call(workspace, need, x.device, stream)
    rc = L.kimad_linear_xent(*lead, at_target, at_weight, at_loss, at_lse, at_dx, ld_dx, at_dw, dw_kind, ld_dw, ws, nbytes, handle)
    if rc:
        _check(rc, "kimad_linear_xent")


def kimad_dropout(x, out, p: float, seed: int, offset: int = 0, residual=None, stream=None) -> None:
    """out = residual + (x where it is kept, else 0) / (1 - p) of matrices of one type (float32 too), elements counted along the rows; the same seed and offset (whole
    numbers of 64 bits) keep the same elements, so that the gradient is the same call on dy without residual.  out may be x or
    residual."""
    rows, cols, ld = _rows(x, "x")
    kind = _type(x)
    at_out, ld_out = _matrix(out, (rows, cols), (x.dtype,), "out")
    at_res, ld_res = _matrix(residual, (rows, cols), (x.dtype,), "residual")
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        raise ValueError(f"seed and offset: whole numbers of 64 bits are wanted, got {seed} and {offset}")
    handle = _on_device(stream, x, out, residual)
    rc = lib().kimad_dropout(x.data_ptr(), kind, rows, cols, ld, at_res, ld_res, p, int(seed), int(offset), at_out, ld_out, handle)
    if rc:
        _check(rc, "kimad_dropout")


class Plan:
    """Owns the torch tensors a plan needs (workspace, outputs) and forwards to the C calls.

    ``g`` and ``h`` are flat fp32 CUDA tensors holding the layers back to back in the order of
    ``sizes`` (or lists of per-layer tensors).
    """

    def __init__(self, g, h, sizes: Sequence[int], ratios: Sequence[float], pair_bytes: int = 0, D: int = 0,
                 max_budget_bytes: int = 0, cfg_flags: int = 0, capacity_pairs: Optional[int] = None,
                 max_workgroups: int = 0, value_format: int = 0):
        import torch
        self.torch = torch
        self.sizes = [int(s) for s in sizes]
        self.L, self.J = len(self.sizes), len(ratios)
        self.ratios = [float(r) for r in ratios]
        if isinstance(g, (list, tuple)):
            g_ptrs = [int(t.data_ptr()) for t in g]
            h_ptrs = [int(t.data_ptr()) for t in h]
            dev = g[0].device
        else:
            starts = np.concatenate([[0], np.cumsum(self.sizes)])
            g_ptrs = [int(g.data_ptr()) + 4 * int(s) for s in starts[:-1]]
            h_ptrs = [int(h.data_ptr()) + 4 * int(s) for s in starts[:-1]]
            dev = g.device
        self._keep = (g, h)
        self.device = dev
        self.value_format = int(value_format)
        self.pair_bytes = int(pair_bytes) if pair_bytes else (6 if value_format == KIMAD_VALUES_F16 else 8)
        nbytes = kimad_workspace_bytes(self.sizes, self.J, pair_bytes, D, max_budget_bytes, cfg_flags, max_workgroups,
                                       value_format)
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=dev)
        base = int(self.workspace.data_ptr())
        self._ws_ptr = (base + 255) // 256 * 256
        self.workspace_bytes = nbytes
        self.handle = kimad_plan_create(g_ptrs, h_ptrs, self.sizes, self.ratios, self._ws_ptr, nbytes,
                                        None, pair_bytes, D, max_budget_bytes, cfg_flags, max_workgroups, value_format)
        d = int(sum(self.sizes))
        self.capacity_pairs = int(capacity_pairs) if capacity_pairs is not None else d
        self.err_table = torch.empty(self.L * self.J, dtype=torch.float64, device=dev)
        self.j = torch.empty(self.L, dtype=torch.int32, device=dev)
        self.K = torch.empty(self.L, dtype=torch.int64, device=dev)
        self.offsets = torch.empty(self.L + 1, dtype=torch.int64, device=dev)
        self.status = torch.zeros(2, dtype=torch.int32, device=dev)
        self.idx = torch.empty(self.capacity_pairs, dtype=torch.int32, device=dev)
        self.val = torch.empty(self.capacity_pairs, device=dev,
                               dtype=torch.float16 if value_format == KIMAD_VALUES_F16 else torch.float32)

    def grid_sizes(self) -> np.ndarray:
        out = (C.c_uint64 * (self.L * self.J))()
        _check(lib().kimad_plan_grid_sizes(C.c_void_p(self.handle), out), "kimad_plan_grid_sizes")
        return np.array(out[:], dtype=np.int64).reshape(self.L, self.J)

    def profile(self, err_table=None, budget_hint_bytes: int = 0):
        t = self.err_table if err_table is None else err_table
        kimad_profile(self.handle, t, budget_hint_bytes)
        return t

    def allocate(self, budget_bytes: int, err_table=None):
        t = self.err_table if err_table is None else err_table
        kimad_allocate(self.handle, t, budget_bytes, self.j, self.K, self.offsets, self.status[0:1])
        return self.j, self.K, self.offsets, self.status[0:1]

    def compress_ef(self, K=None, offsets=None, reuse_profile: bool = False):
        K = self.K if K is None else K
        offsets = self.offsets if offsets is None else offsets
        kimad_compress_ef(self.handle, K, offsets, self.idx, self.val, self.capacity_pairs,
                          KIMAD_REUSE_PROFILE if reuse_profile else 0, self.status[1:2])
        return self.idx, self.val, self.status[1:2]

    def step(self, budget_bytes: int):
        kimad_step(self.handle, budget_bytes, self.err_table, self.j, self.K, self.offsets, self.idx, self.val,
                   self.capacity_pairs, self.status)
        return self.status

    def error_at(self, K, err_out=None):
        """Per-layer TopK error at the sizes K (device int64[L]); returns a device float64[L]."""
        if err_out is None:
            err_out = self.torch.empty(self.L, dtype=self.torch.float64, device=self.device)
        kimad_error_at(self.handle, K, err_out)
        return err_out

    def diagnostics(self):
        out = (C.c_uint32 * 4)()
        _check(lib().kimad_profile_diagnostics(C.c_void_p(self.handle), out, C.c_void_p(_stream(None))),
               "kimad_profile_diagnostics")
        return dict(uncertified=int(out[0]), recomputed=int(out[1]), pool_entries=int(out[2]),
                    redo_layers=int(out[3]))

    def allocate_diagnostics(self):
        out = (C.c_uint32 * 4)()
        _check(lib().kimad_allocate_diagnostics(C.c_void_p(self.handle), out, C.c_void_p(_stream(None))),
               "kimad_allocate_diagnostics")
        return dict(max_band=int(out[0]), sum_bands=int(out[1]), whole_rows=int(out[2]), upgrades=int(out[3]))

    def allocate_route(self):
        """How the last allocation went: dict(route, rows_decided, from_left, at_once)."""
        out = (C.c_uint32 * 2)()
        _check(lib().kimad_allocate_route(C.c_void_p(self.handle), out, C.c_void_p(_stream(None))), "kimad_allocate_route")
        return dict(route=("none", "rows", "band", "tree", "halves")[out[0]], rows_decided=bool(out[1] & 1), from_left=bool(out[1] & 2),
                    at_once=bool(out[1] & 4))

    def layer_states(self):
        """Per tiled layer: dict(layer, spill_bin, slots_pre, slots_cand, redo, spill_cnt, spill_valid, mode)."""
        out = (C.c_uint32 * (8 * self.L))()
        cnt = C.c_uint32(0)
        _check(lib().kimad_plan_layer_states(C.c_void_p(self.handle), out, self.L, C.byref(cnt),
                                             C.c_void_p(_stream(None))), "kimad_plan_layer_states")
        names = ("layer", "spill_bin", "slots_pre", "slots_cand", "redo", "spill_cnt", "spill_valid", "mode")
        return [dict(zip(names, out[8 * b:8 * b + 8])) for b in range(cnt.value)]

    def set_timing(self, enable: bool) -> None:
        _check(lib().kimad_plan_set_timing(C.c_void_p(self.handle), int(bool(enable))), "kimad_plan_set_timing")

    def get_timings(self):
        """[(kernel name, milliseconds)] for every launch since the last call (timing must be on)."""
        names = C.create_string_buffer(65536)
        ms = (C.c_float * 1024)()
        cnt = C.c_uint32(0)
        _check(lib().kimad_plan_get_timings(C.c_void_p(self.handle), names, 65536, ms, 1024, C.byref(cnt)),
               "kimad_plan_get_timings")
        nm = names.value.decode().split("\n")[:cnt.value]
        return [(nm[k], float(ms[k])) for k in range(cnt.value)]

    def close(self):
        if getattr(self, "handle", 0):
            kimad_plan_destroy(self.handle)
            self.handle = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
