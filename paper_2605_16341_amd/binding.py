"""ctypes binding of liborthdion.so: the same entry points as include/orthdion.h, plus a thin
convenience class.  Argument marshalling only - every step of the method runs in the HIP
kernels.  There is no CPU fallback: a missing library is an error."""
from __future__ import annotations

import array
import contextlib
import ctypes
import operator
import os
from typing import List, Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liborthdion.so")

ORTHDION_OK = 0
ORTHDION_E_INVALID_ARG = -1
ORTHDION_E_NULL_PTR = -2
ORTHDION_E_BAD_SHAPE = -3
ORTHDION_E_WORKSPACE_TOO_SMALL = -4
ORTHDION_E_MISALIGNED = -5
ORTHDION_E_HIP = -6
ORTHDION_E_NO_STEP = -7
ORTHDION_E_NO_MEMORY = -8

ORTHDION_F32, ORTHDION_BF16 = 0, 1
ORTHDION_QR, ORTHDION_COLNORM = 0, 1
ORTHDION_EF_DION, ORTHDION_EF_PAPER, ORTHDION_EF_POLYAK = 0, 1, 2
ORTHDION_PREC_AUTO, ORTHDION_PREC_FAST, ORTHDION_PREC_EXACT = 0, 1, 2

EXPORTS = ["orthdion_create", "orthdion_workspace_bytes", "orthdion_set_lr", "orthdion_set_mu",
           "orthdion_set_variant", "orthdion_step", "orthdion_get_info", "orthdion_workspace_layout",
           "orthdion_profile_begin", "orthdion_profile_end", "orthdion_set_diagnostics",
           "orthdion_get_diagnostics", "orthdion_rank_policy", "orthdion_resize_q", "orthdion_strerror",
           "orthdion_destroy", "orthdion_step_static", "orthdion_static_scratch_bytes", "orthdion_get_warnings",
           "orthdion_get_groups", "orthdion_muon_create", "orthdion_muon_workspace_bytes", "orthdion_muon_get_tiles", "orthdion_muon_set_lr",
           "orthdion_muon_set_mu", "orthdion_muon_set_weight_decay", "orthdion_muon_step", "orthdion_muon_orthogonalise",
           "orthdion_muon_get_info", "orthdion_muon_destroy", "orthdion_adamw_create", "orthdion_adamw_set_lr",
           "orthdion_adamw_step", "orthdion_adamw_destroy"]

DIAG = ["b_norm", "r_norm", "tracking_error", "residual_ratio", "inner", "nu", "erank", "g_norm"]
ORTHDION_NDIAG = len(DIAG)

PHASES = ["stats", "proj", "proj_reduce", "gram_left", "chol_left", "orth_left", "guard_left", "finish_left", "back",
          "back_reduce", "gram_right", "chol_right", "orth_right", "guard_right", "finish_right", "efx"]
ORTHDION_NPHASE = len(PHASES)


class orthdion_matdesc(ctypes.Structure):
    _fields_ = [("m", ctypes.c_int64), ("n", ctypes.c_int64), ("r", ctypes.c_int32),
                ("ldx", ctypes.c_int64), ("ldg", ctypes.c_int64), ("ldm", ctypes.c_int64)]


class orthdion_config(ctypes.Structure):
    _fields_ = [("x_dtype", ctypes.c_int), ("g_dtype", ctypes.c_int), ("variant", ctypes.c_int),
                ("ef", ctypes.c_int), ("precision", ctypes.c_int), ("mu", ctypes.c_float),
                ("lr", ctypes.c_float), ("groups", ctypes.c_int32)]


ORTHDION_MUON_MAX_STEPS = 32
# the published quintic of the Muon optimizer, five steps
MUON_COEFFS = ((3.4445, -4.7750, 2.0315),) * 5


class orthdion_muon_matdesc(ctypes.Structure):
    _fields_ = [("m", ctypes.c_int64), ("n", ctypes.c_int64), ("ldx", ctypes.c_int64), ("ldg", ctypes.c_int64),
                ("ldm", ctypes.c_int64), ("scale", ctypes.c_float)]


class orthdion_muon_config(ctypes.Structure):
    _fields_ = [("x_dtype", ctypes.c_int), ("g_dtype", ctypes.c_int), ("precision", ctypes.c_int),
                ("nesterov", ctypes.c_int32), ("steps", ctypes.c_int32),
                ("coeffs", ctypes.c_float * (3 * ORTHDION_MUON_MAX_STEPS)), ("mu", ctypes.c_float), ("lr", ctypes.c_float),
                ("weight_decay", ctypes.c_float), ("eps", ctypes.c_float)]


class orthdion_adamw_desc(ctypes.Structure):
    _fields_ = [("length", ctypes.c_int64), ("lr_scale", ctypes.c_float), ("weight_decay", ctypes.c_float)]


class orthdion_adamw_config(ctypes.Structure):
    _fields_ = [("x_dtype", ctypes.c_int), ("g_dtype", ctypes.c_int), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("lr", ctypes.c_float), ("eps", ctypes.c_float)]


_lib: Optional[ctypes.CDLL] = None


def _share_torch_hip_runtime() -> None:
    """PyTorch wheels ship their own copy of the HIP runtime (same SONAME as ROCm's).  Device
    pointers and streams are only meaningful inside one runtime instance, so when this
    library is loaded before torch it must bind to torch's copy, not to /opt/rocm's: map
    torch's copy first and the loader resolves our dependency to it by SONAME."""
    import importlib.util
    try:
        spec = importlib.util.find_spec("torch")
    except (ImportError, ValueError):
        spec = None
    if spec is None or not spec.submodule_search_locations:
        return
    cand = os.path.join(list(spec.submodule_search_locations)[0], "lib", "libamdhip64.so")
    if os.path.exists(cand):
        ctypes.CDLL(cand, mode=ctypes.RTLD_GLOBAL)


def load() -> ctypes.CDLL:
    """Loads the in-tree library (built by build.py); raises if it is not there."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2605_16341_amd.build` "
                           "(there is no fallback path)")
    _share_torch_hip_runtime()
    lib = ctypes.CDLL(LIB_PATH)
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    lib.orthdion_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(orthdion_matdesc), ctypes.c_int32,
                                    ctypes.POINTER(orthdion_config)]
    lib.orthdion_create.restype = ctypes.c_int
    lib.orthdion_workspace_bytes.argtypes = [vp]
    lib.orthdion_workspace_bytes.restype = sz
    lib.orthdion_get_groups.argtypes = [vp]
    lib.orthdion_get_groups.restype = ctypes.c_int32
    lib.orthdion_set_lr.argtypes = [vp, ctypes.c_float]
    lib.orthdion_set_lr.restype = ctypes.c_int
    lib.orthdion_set_mu.argtypes = [vp, ctypes.c_float]
    lib.orthdion_set_mu.restype = ctypes.c_int
    lib.orthdion_set_variant.argtypes = [vp, ctypes.c_int]
    lib.orthdion_set_variant.restype = ctypes.c_int
    lib.orthdion_step.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp),
                                  ctypes.POINTER(vp), vp, sz, vp]
    lib.orthdion_step.restype = ctypes.c_int
    lib.orthdion_step_static.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp),
                                         ctypes.POINTER(vp), vp]
    lib.orthdion_step_static.restype = ctypes.c_int
    lib.orthdion_static_scratch_bytes.argtypes = []
    lib.orthdion_static_scratch_bytes.restype = sz
    lib.orthdion_get_info.argtypes = [vp, ctypes.POINTER(ctypes.c_int32), vp]
    lib.orthdion_get_info.restype = ctypes.c_int
    lib.orthdion_get_warnings.argtypes = [vp, ctypes.POINTER(ctypes.c_uint32), vp]
    lib.orthdion_get_warnings.restype = ctypes.c_int
    lib.orthdion_workspace_layout.argtypes = [vp, ctypes.c_int32] + [ctypes.POINTER(sz)] * 6
    lib.orthdion_workspace_layout.restype = ctypes.c_int
    lib.orthdion_profile_begin.argtypes = [vp, ctypes.c_uint32, ctypes.c_int32]
    lib.orthdion_profile_begin.restype = ctypes.c_int
    lib.orthdion_profile_end.argtypes = [vp, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int32)]
    lib.orthdion_profile_end.restype = ctypes.c_int
    lib.orthdion_set_diagnostics.argtypes = [vp, ctypes.c_int32]
    lib.orthdion_set_diagnostics.restype = ctypes.c_int
    lib.orthdion_get_diagnostics.argtypes = [vp, ctypes.POINTER(ctypes.c_float), vp]
    lib.orthdion_get_diagnostics.restype = ctypes.c_int
    lib.orthdion_rank_policy.argtypes = [ctypes.c_float, ctypes.c_float, ctypes.c_int32, ctypes.c_int32,
                                         ctypes.c_float, ctypes.c_float, ctypes.POINTER(ctypes.c_float),
                                         ctypes.POINTER(ctypes.c_int32)]
    lib.orthdion_rank_policy.restype = ctypes.c_int
    lib.orthdion_resize_q.argtypes = [vp, ctypes.c_int64, ctypes.c_int32, vp, ctypes.c_int32, vp, vp]
    lib.orthdion_resize_q.restype = ctypes.c_int
    lib.orthdion_strerror.argtypes = [ctypes.c_int]
    lib.orthdion_strerror.restype = ctypes.c_char_p
    lib.orthdion_destroy.argtypes = [vp]
    lib.orthdion_destroy.restype = ctypes.c_int
    pp, f32 = ctypes.POINTER(vp), ctypes.c_float
    for name, args, res in (
            ("orthdion_muon_create", [pp, ctypes.POINTER(orthdion_muon_matdesc), ctypes.c_int32, ctypes.POINTER(orthdion_muon_config)], ctypes.c_int),
            ("orthdion_muon_workspace_bytes", [vp], sz),
            ("orthdion_muon_get_tiles", [vp, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32)], ctypes.c_int), ("orthdion_muon_set_lr", [vp, f32], ctypes.c_int),
            ("orthdion_muon_set_mu", [vp, f32], ctypes.c_int), ("orthdion_muon_set_weight_decay", [vp, f32], ctypes.c_int),
            ("orthdion_muon_step", [vp, pp, pp, pp, vp, sz, vp], ctypes.c_int),
            ("orthdion_muon_orthogonalise", [vp, pp, pp, vp, sz, vp], ctypes.c_int),
            ("orthdion_muon_get_info", [vp, ctypes.POINTER(ctypes.c_int32), vp], ctypes.c_int),
            ("orthdion_muon_destroy", [vp], ctypes.c_int),
            ("orthdion_adamw_create", [pp, ctypes.POINTER(orthdion_adamw_desc), ctypes.c_int32, ctypes.POINTER(orthdion_adamw_config)], ctypes.c_int),
            ("orthdion_adamw_set_lr", [vp, f32], ctypes.c_int),
            ("orthdion_adamw_step", [vp, pp, pp, pp, pp, vp, vp], ctypes.c_int), ("orthdion_adamw_destroy", [vp], ctypes.c_int)):
        getattr(lib, name).argtypes = args
        getattr(lib, name).restype = res
    _lib = lib
    return lib


class OrthDionError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        super().__init__(f"orthdion status {status}: {orthdion_strerror(status)}")


def orthdion_strerror(status: int) -> str:
    return load().orthdion_strerror(int(status)).decode()


def _check(status: int) -> None:
    if status != ORTHDION_OK:
        raise OrthDionError(status)


def orthdion_create(shapes: Sequence[Sequence[int]], r, x_dtype: int, g_dtype: int, variant: int = ORTHDION_QR,
                    ef: int = ORTHDION_EF_DION, precision: int = ORTHDION_PREC_AUTO, mu: float = 0.95,
                    lr: float = 0.01, lds: Optional[Sequence[Sequence[int]]] = None, groups: int = 0) -> int:
    """`shapes` is a list of (m, n); `r` one rank or one per matrix; `lds` optional
    (ldx, ldg, ldm) per matrix (default n); `groups` 0 (the library chooses), 1 or 2.  Returns
    the opaque handle as an int."""
    lib = load()
    nmat = len(shapes)
    ranks = [int(r)] * nmat if isinstance(r, int) else [int(v) for v in r]
    descs = (orthdion_matdesc * max(nmat, 1))()
    for i, (m, n) in enumerate(shapes):
        ld = lds[i] if lds is not None else (n, n, n)
        descs[i] = orthdion_matdesc(int(m), int(n), ranks[i], int(ld[0]), int(ld[1]), int(ld[2]))
    cfg = orthdion_config(int(x_dtype), int(g_dtype), int(variant), int(ef), int(precision), float(mu), float(lr), int(groups))
    handle = ctypes.c_void_p()
    _check(lib.orthdion_create(ctypes.byref(handle), descs, nmat, ctypes.byref(cfg)))
    return handle.value


def orthdion_workspace_bytes(handle: int) -> int:
    return int(load().orthdion_workspace_bytes(handle))


def orthdion_get_groups(handle: int) -> int:
    return int(load().orthdion_get_groups(handle))


def orthdion_set_lr(handle: int, lr: float) -> None:
    _check(load().orthdion_set_lr(handle, float(lr)))


def orthdion_set_mu(handle: int, mu: float) -> None:
    _check(load().orthdion_set_mu(handle, float(mu)))


def orthdion_set_variant(handle: int, variant: int) -> None:
    _check(load().orthdion_set_variant(handle, int(variant)))


def _ptr_array(ptrs: Sequence[Optional[int]]):
    """Host array of device addresses; None is a null pointer."""
    try:
        return (ctypes.c_void_p * len(ptrs)).from_buffer(array.array("Q", ptrs)) if len(ptrs) else (ctypes.c_void_p * 0)()
    except (TypeError, OverflowError):         # what else ctypes takes for an address: None, c_void_p, an address as a signed number
        return (ctypes.c_void_p * len(ptrs))(*ptrs)


def orthdion_step(handle: int, X: Sequence[int], G: Sequence[int], M: Sequence[int], Q: Sequence[int],
                  workspace: int, workspace_bytes: int, stream: int = 0) -> None:
    """X, G, M, Q: device addresses (ints), one per matrix; `stream` a hipStream_t as int."""
    _check(load().orthdion_step(handle, _ptr_array(X), _ptr_array(G), _ptr_array(M), _ptr_array(Q),
                                ctypes.c_void_p(workspace), workspace_bytes, ctypes.c_void_p(stream)))


def orthdion_step_static(handle: int, X: Sequence[int], G: Sequence[int], M: Sequence[int], Q: Sequence[int],
                         stream: int = 0) -> None:
    """orthdion_step on the library's own device scratch (no workspace argument)."""
    _check(load().orthdion_step_static(handle, _ptr_array(X), _ptr_array(G), _ptr_array(M), _ptr_array(Q),
                                       ctypes.c_void_p(stream)))


def orthdion_static_scratch_bytes() -> int:
    return int(load().orthdion_static_scratch_bytes())


def orthdion_get_info(handle: int, nmat: int, stream: int = 0) -> List[int]:
    out = (ctypes.c_int32 * nmat)()
    _check(load().orthdion_get_info(handle, out, ctypes.c_void_p(stream)))
    return list(out)


WARN_B_CLIPPED, WARN_R_CLIPPED, WARN_B_SCALE_BLIND, WARN_WAIT_EXPIRED = 1, 2, 4, 8


def orthdion_get_warnings(handle: int, nmat: int, stream: int = 0) -> List[int]:
    out = (ctypes.c_uint32 * nmat)()
    _check(load().orthdion_get_warnings(handle, out, ctypes.c_void_p(stream)))
    return list(out)


def orthdion_workspace_layout(handle: int, index: int) -> dict:
    vals = [ctypes.c_size_t() for _ in range(6)]
    _check(load().orthdion_workspace_layout(handle, int(index), *[ctypes.byref(v) for v in vals]))
    keys = ["P", "R", "T_P1", "T_P2", "T_Q1", "T_Q2"]
    return {k: int(v.value) for k, v in zip(keys, vals)}


def orthdion_profile_begin(handle: int, phase_mask: int, max_steps: int) -> None:
    _check(load().orthdion_profile_begin(handle, int(phase_mask), int(max_steps)))


def orthdion_profile_end(handle: int) -> dict:
    """{phase name: (total milliseconds, intervals)} for the phases that were bracketed."""
    ms = (ctypes.c_float * ORTHDION_NPHASE)()
    cnt = (ctypes.c_int32 * ORTHDION_NPHASE)()
    _check(load().orthdion_profile_end(handle, ms, cnt))
    return {PHASES[i]: (float(ms[i]), int(cnt[i])) for i in range(ORTHDION_NPHASE) if cnt[i] > 0}


def orthdion_set_diagnostics(handle: int, enable: bool) -> None:
    _check(load().orthdion_set_diagnostics(handle, 1 if enable else 0))


def orthdion_get_diagnostics(handle: int, nmat: int, stream: int = 0) -> List[dict]:
    """One {name: value} dict per matrix for the most recent step (names in DIAG)."""
    out = (ctypes.c_float * (nmat * ORTHDION_NDIAG))()
    _check(load().orthdion_get_diagnostics(handle, out, ctypes.c_void_p(stream)))
    return [{DIAG[k]: float(out[i * ORTHDION_NDIAG + k]) for k in range(ORTHDION_NDIAG)} for i in range(nmat)]


def orthdion_rank_policy(e_t: float, ema_prev: float, r_min: int, r_max: int, alpha: float, gamma: float):
    """(new EMA, next rank) of the adaptive-rank rule."""
    ema, nxt = ctypes.c_float(), ctypes.c_int32()
    _check(load().orthdion_rank_policy(float(e_t), float(ema_prev), int(r_min), int(r_max), float(alpha),
                                       float(gamma), ctypes.byref(ema), ctypes.byref(nxt)))
    return float(ema.value), int(nxt.value)


def orthdion_resize_q(q_old: int, n: int, r_old: int, q_new: int, r_new: int, pad: int = 0, stream: int = 0) -> None:
    """Device addresses as ints; `pad` may be 0 only when the rank does not grow."""
    _check(load().orthdion_resize_q(ctypes.c_void_p(q_old), int(n), int(r_old), ctypes.c_void_p(q_new), int(r_new),
                                    ctypes.c_void_p(pad or None), ctypes.c_void_p(stream)))


def orthdion_destroy(handle: int) -> None:
    _check(load().orthdion_destroy(handle))


def orthdion_muon_create(shapes: Sequence[Sequence[int]], x_dtype: int, g_dtype: int, precision: int = ORTHDION_PREC_AUTO,
                         nesterov: bool = True, coeffs: Sequence[Sequence[float]] = MUON_COEFFS, mu: float = 0.95, lr: float = 0.02,
                         weight_decay: float = 0.0, eps: float = 1e-7, scales: Optional[Sequence[float]] = None,
                         lds: Optional[Sequence[Sequence[int]]] = None) -> int:
    """`shapes` is a list of (m, n); `coeffs` one (a, b, c) per Newton-Schulz step; `scales` one factor of the update per
    matrix (default 1); `lds` optional (ldx, ldg, ldm) per matrix (default n).  Returns the opaque handle as an int."""
    nmat = len(shapes)
    descs = (orthdion_muon_matdesc * max(nmat, 1))()
    for i, (m, n) in enumerate(shapes):
        ld = lds[i] if lds is not None else (n, n, n)
        descs[i] = orthdion_muon_matdesc(int(m), int(n), int(ld[0]), int(ld[1]), int(ld[2]), 1.0 if scales is None else float(scales[i]))
    if any(len(step) != 3 for step in coeffs) or len(coeffs) > ORTHDION_MUON_MAX_STEPS:
        raise ValueError(f"coeffs: at most {ORTHDION_MUON_MAX_STEPS} triples (a, b, c)")
    flat = [float(v) for step in coeffs for v in step]
    cfg = orthdion_muon_config(int(x_dtype), int(g_dtype), int(precision), int(nesterov), len(coeffs),
                               (ctypes.c_float * (3 * ORTHDION_MUON_MAX_STEPS))(*flat), float(mu), float(lr), float(weight_decay), float(eps))
    handle = ctypes.c_void_p()
    _check(load().orthdion_muon_create(ctypes.byref(handle), descs, nmat, ctypes.byref(cfg)))
    return handle.value


def orthdion_muon_workspace_bytes(handle: int) -> int:
    return int(load().orthdion_muon_workspace_bytes(handle))


# kinds of products as orthdion_muon_get_tiles counts them
MUON_PRODUCTS = ("gram", "symmetric", "apply", "full", "last_wide", "last_tall")


def orthdion_muon_get_tiles(handle: int, step: bool) -> dict:
    """Widths of the tiles that each kind of product is computed on, as a set; kinds that a call has none of are left out."""
    out = (ctypes.c_int32 * len(MUON_PRODUCTS))()
    _check(load().orthdion_muon_get_tiles(handle, int(step), out))
    return {name: {64 * (k + 1) for k in range(4) if bits >> k & 1} for name, bits in zip(MUON_PRODUCTS, out) if bits}


def orthdion_muon_set_lr(handle: int, lr: float) -> None:
    _check(load().orthdion_muon_set_lr(handle, float(lr)))


def orthdion_muon_set_mu(handle: int, mu: float) -> None:
    _check(load().orthdion_muon_set_mu(handle, float(mu)))


def orthdion_muon_set_weight_decay(handle: int, weight_decay: float) -> None:
    _check(load().orthdion_muon_set_weight_decay(handle, float(weight_decay)))


def orthdion_muon_step(handle: int, X: Sequence[int], G: Sequence[int], M: Sequence[int], workspace: int, workspace_bytes: int,
                       stream: int = 0) -> None:
    """X, G, M: device addresses (ints), one per matrix."""
    _check(load().orthdion_muon_step(handle, _ptr_array(X), _ptr_array(G), _ptr_array(M), ctypes.c_void_p(workspace),
                                     workspace_bytes, ctypes.c_void_p(stream)))


def orthdion_muon_orthogonalise(handle: int, A: Sequence[int], O: Sequence[int], workspace: int, workspace_bytes: int,
                                stream: int = 0) -> None:
    _check(load().orthdion_muon_orthogonalise(handle, _ptr_array(A), _ptr_array(O), ctypes.c_void_p(workspace), workspace_bytes,
                                              ctypes.c_void_p(stream)))


def orthdion_muon_get_info(handle: int, nmat: int, stream: int = 0) -> List[int]:
    out = (ctypes.c_int32 * nmat)()
    _check(load().orthdion_muon_get_info(handle, out, ctypes.c_void_p(stream)))
    return list(out)


def orthdion_muon_destroy(handle: int) -> None:
    _check(load().orthdion_muon_destroy(handle))


def orthdion_adamw_create(lengths: Sequence[int], x_dtype: int, g_dtype: int, lr: float = 1e-3, beta1: float = 0.9, beta2: float = 0.999,
                          eps: float = 1e-8, weight_decays: Optional[Sequence[float]] = None,
                          lr_scales: Optional[Sequence[float]] = None) -> int:
    """`lengths`: elements of every tensor; one weight decay (default 0) and factor of lr (default 1) each."""
    count = len(lengths)
    descs = (orthdion_adamw_desc * max(count, 1))()
    for i, n in enumerate(lengths):
        descs[i] = orthdion_adamw_desc(int(n), 1.0 if lr_scales is None else float(lr_scales[i]),
                                       0.0 if weight_decays is None else float(weight_decays[i]))
    cfg = orthdion_adamw_config(int(x_dtype), int(g_dtype), float(beta1), float(beta2), float(lr), float(eps))
    handle = ctypes.c_void_p()
    _check(load().orthdion_adamw_create(ctypes.byref(handle), descs, count, ctypes.byref(cfg)))
    return handle.value


def orthdion_adamw_set_lr(handle: int, lr: float) -> None:
    _check(load().orthdion_adamw_set_lr(handle, float(lr)))


def orthdion_adamw_step(handle: int, X: Sequence[int], G: Sequence[int], M: Sequence[int], V: Sequence[int], counter: int,
                        stream: int = 0) -> None:
    """Device addresses as ints; `counter` that of two int32, [steps taken, 0]."""
    _check(load().orthdion_adamw_step(handle, _ptr_array(X), _ptr_array(G), _ptr_array(M), _ptr_array(V), ctypes.c_void_p(counter),
                                      ctypes.c_void_p(stream)))


def orthdion_adamw_destroy(handle: int) -> None:
    _check(load().orthdion_adamw_destroy(handle))


class OrthDion:
    """Owns a handle and a torch-allocated workspace; `step` takes lists of torch tensors
    (device memory and the current stream come from torch; nothing else does)."""

    def __init__(self, shapes, r, x_dtype="bf16", g_dtype=None, variant="qr", ef="dion", precision="auto",
                 mu=0.95, lr=0.01, device="cuda:0", groups=0):
        import torch
        g_dtype = g_dtype or x_dtype
        dt = {"f32": ORTHDION_F32, "bf16": ORTHDION_BF16}
        self.shapes = [tuple(s) for s in shapes]
        self.nmat = len(self.shapes)
        self.r = r
        self._x_dtype = {"f32": torch.float32, "bf16": torch.bfloat16}[x_dtype]
        self._g_dtype = {"f32": torch.float32, "bf16": torch.bfloat16}[g_dtype]
        self.handle = orthdion_create(self.shapes, r, dt[x_dtype], dt[g_dtype],
                                      {"qr": ORTHDION_QR, "colnorm": ORTHDION_COLNORM}[variant],
                                      {"dion": ORTHDION_EF_DION, "paper": ORTHDION_EF_PAPER, "polyak": ORTHDION_EF_POLYAK}[ef],
                                      {"auto": ORTHDION_PREC_AUTO, "fast": ORTHDION_PREC_FAST,
                                       "exact": ORTHDION_PREC_EXACT}[precision], mu, lr, groups=groups)
        self.workspace_bytes = orthdion_workspace_bytes(self.handle)
        self.groups = orthdion_get_groups(self.handle)
        self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=device)
        self._torch = torch

    def _check_buffers(self, X, G, M, Q) -> None:
        """The library sees raw addresses only: a tensor of the wrong type, shape or layout
        would be read and written out of bounds, so it is refused here."""
        torch = self._torch
        for name, seq in (("X", X), ("G", G), ("M", M), ("Q", Q)):
            if len(seq) != self.nmat:
                raise ValueError(f"{name}: expected {self.nmat} tensors, got {len(seq)}")
        for i, (m, n) in enumerate(self.shapes):
            r = self.r if isinstance(self.r, int) else self.r[i]
            want = {"X": ((m, n), self._x_dtype), "G": ((m, n), self._g_dtype), "M": ((m, n), torch.float32),
                    "Q": ((n, r), torch.float32)}
            for name, t in (("X", X[i]), ("G", G[i]), ("M", M[i]), ("Q", Q[i])):
                shape, dtype = want[name]
                if not t.is_cuda or tuple(t.shape) != shape or t.dtype != dtype or not t.is_contiguous():
                    raise ValueError(f"{name}[{i}]: need a contiguous {dtype} device tensor of shape {shape}, got "
                                     f"{t.dtype} {tuple(t.shape)} on {t.device}, contiguous={t.is_contiguous()}")

    def step(self, X, G, M, Q, stream=None) -> None:
        torch = self._torch
        self._check_buffers(X, G, M, Q)
        st = stream if stream is not None else torch.cuda.current_stream().cuda_stream
        orthdion_step(self.handle, [t.data_ptr() for t in X], [t.data_ptr() for t in G],
                      [t.data_ptr() for t in M], [t.data_ptr() for t in Q],
                      self.workspace.data_ptr(), self.workspace_bytes, st)

    def info(self, stream=None) -> List[int]:
        st = stream if stream is not None else self._torch.cuda.current_stream().cuda_stream
        return orthdion_get_info(self.handle, self.nmat, st)

    def warnings(self, stream=None) -> List[int]:
        st = stream if stream is not None else self._torch.cuda.current_stream().cuda_stream
        return orthdion_get_warnings(self.handle, self.nmat, st)

    def set_diagnostics(self, enable: bool) -> None:
        orthdion_set_diagnostics(self.handle, enable)

    def diagnostics(self, stream=None) -> List[dict]:
        st = stream if stream is not None else self._torch.cuda.current_stream().cuda_stream
        return orthdion_get_diagnostics(self.handle, self.nmat, st)

    def debug_factors(self, index: int) -> dict:
        """P, R and the triangular factors the last step left in the workspace (copies)."""
        torch = self._torch
        lay = orthdion_workspace_layout(self.handle, index)
        m, n = self.shapes[index]
        r = self.r if isinstance(self.r, int) else self.r[index]
        out = {}
        for key, (rows, cols) in {"P": (m, r), "R": (n, r), "T_P1": (r, r), "T_P2": (r, r), "T_Q1": (r, r),
                                  "T_Q2": (r, r)}.items():
            nbytes = rows * cols * 4
            out[key] = self.workspace[lay[key]:lay[key] + nbytes].view(torch.float32).reshape(rows, cols).clone()
        return out

    def set_lr(self, lr: float) -> None:
        orthdion_set_lr(self.handle, lr)

    def set_mu(self, mu: float) -> None:
        orthdion_set_mu(self.handle, mu)

    def set_variant(self, variant: str) -> None:
        orthdion_set_variant(self.handle, {"qr": ORTHDION_QR, "colnorm": ORTHDION_COLNORM}[variant])

    def close(self) -> None:
        if self.handle:
            orthdion_destroy(self.handle)
            self.handle = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _dtypes(torch, x_dtype: str, g_dtype: Optional[str]):
    """(code, torch type) of x and g; g has x's type unless given."""
    known = {"f32": (ORTHDION_F32, torch.float32), "bf16": (ORTHDION_BF16, torch.bfloat16)}
    for t in (x_dtype, g_dtype or x_dtype):
        if t not in known:
            raise ValueError(f"dtype {t!r}: need one of {sorted(known)}")
    return known[x_dtype], known[g_dtype or x_dtype]


_dtype_of = operator.attrgetter("dtype")


def _on_device(torch, index: int):
    """A context in which device `index` is the current one."""
    return contextlib.nullcontext() if torch.cuda.current_device() == index else torch.cuda.device(index)


def _per_item(name: str, value, count: int) -> List[float]:
    """One float per item from one for all or a sequence."""
    got = [float(value)] * count if isinstance(value, (int, float)) else [float(v) for v in value]
    if len(got) != count:
        raise ValueError(f"{name}: expected one value or {count}, got {len(got)}")
    return got


def _separate(name: str, written: List[int], read=()) -> None:
    """Refuses a call that names one buffer twice among those that it writes, or reads one of them as another operand: workgroups would
    race on it."""
    once = set(written)
    if len(once) != len(written) or not once.isdisjoint(read):
        raise ValueError(f"{name}: one buffer is given twice, or for two operands (a tied parameter steps once; results need memory of their own)")


class Muon:
    """Owns a handle and a torch-allocated workspace of the Muon step; tensors are the caller's.

    shapes   list of (m, n)
    coeffs   one (a, b, c) per Newton-Schulz step
    scale    factor of every matrix's update: "none" (1), "spectral" (sqrt(max(1, m / n))), "rms" (0.2 sqrt(max(m, n)), the
             root mean square of an AdamW update), or a list of numbers
    lds      (ldx, ldg, ldm) per matrix where rows are further apart than n elements, e.g. parts of a fused projection

    A captured step is replayed with the lr, mu and weight decay of its capture, and on this object's workspace: the object has to
    live as long as the graph.
    """

    def __init__(self, shapes, x_dtype="bf16", g_dtype=None, precision="auto", mu=0.95, lr=0.02, weight_decay=0.0, nesterov=True,
                 coeffs=MUON_COEFFS, eps=1e-7, scale="spectral", lds=None, device="cuda:0"):
        import torch
        self.handle = 0
        self._torch = torch
        self.device = torch.device(device)
        self.shapes = [(int(m), int(n)) for m, n in shapes]
        self.nmat = len(self.shapes)
        self.lds = [tuple(int(v) for v in ld) for ld in lds] if lds is not None else [(n, n, n) for _, n in self.shapes]
        if len(self.lds) != self.nmat:
            raise ValueError(f"lds: expected {self.nmat} triples, got {len(self.lds)}")
        self._strides = [[(ld[k], 1) for ld in self.lds] for k in range(3)]
        (xc, self._x_dtype), (gc, self._g_dtype) = _dtypes(torch, x_dtype, g_dtype)
        rules = {"none": lambda m, n: 1.0, "spectral": lambda m, n: max(1.0, m / n) ** 0.5, "rms": lambda m, n: 0.2 * max(m, n) ** 0.5}
        if isinstance(scale, str):
            if scale not in rules:
                raise ValueError(f"scale {scale!r}: need one of {sorted(rules)} or a list of numbers")
            scale = [rules[scale](m, n) if m > 0 and n > 0 else 1.0 for m, n in self.shapes]
        self.handle = orthdion_muon_create(
            self.shapes, xc, gc, {"auto": ORTHDION_PREC_AUTO, "fast": ORTHDION_PREC_FAST, "exact": ORTHDION_PREC_EXACT}[precision],
            nesterov, coeffs, mu, lr, weight_decay, eps, _per_item("scale", scale, self.nmat), self.lds)
        self.workspace_bytes = orthdion_muon_workspace_bytes(self.handle)
        self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=self.device)
        self._home = torch.cuda.current_stream(self.workspace.device).cuda_stream if self.workspace.is_cuda else 0

    def _pointers(self, name: str, seq, dtype, which: int) -> List[int]:
        """Addresses of a list of tensors, after the checks that raw addresses cannot have: one wrong type, shape, stride or
        device would be an access out of bounds."""
        tensor = self._torch.Tensor
        # a handful of C calls a tensor; only what does not pass is looked at one by one
        if (self.workspace.is_cuda and set(map(tensor.get_device, seq)) == {self.workspace.get_device()}
                and set(map(_dtype_of, seq)) == {dtype} and list(map(tensor.size, seq)) == self.shapes
                and list(map(tensor.stride, seq)) == self._strides[which]):
            return list(map(tensor.data_ptr, seq))
        if len(seq) != self.nmat:
            raise ValueError(f"{name}: expected {self.nmat} tensors, got {len(seq)}")
        for i, t in enumerate(seq):
            m, n = self.shapes[i]
            ld = self.lds[i][which]
            rows = t.dim() == 2 and (n == 1 or t.stride(1) == 1) and (m == 1 or t.stride(0) == ld)
            if t.device.type != "cuda" or tuple(t.shape) != (m, n) or t.dtype != dtype or not rows:
                raise ValueError(f"{name}[{i}]: need a {dtype} device tensor of shape {(m, n)} with rows {ld} elements apart, got "
                                 f"{t.dtype} {tuple(t.shape)} with strides {tuple(t.stride())} on {t.device}")
            if t.device != self.workspace.device:
                raise ValueError(f"{name}[{i}]: on {t.device}, the workspace on {self.workspace.device}")
        return [t.data_ptr() for t in seq]

    def _stream(self, stream) -> int:
        """The stream of a call.  The workspace belongs to the stream it was made on: another one is noted, so that its memory is
        not given away while that stream still works on it."""
        torch = self._torch
        if stream is None:
            used = torch.cuda.current_stream(self.workspace.device)
            stream = used.cuda_stream
        elif stream != self._home:
            used = torch.cuda.ExternalStream(stream, device=self.workspace.device)
        if stream != self._home and not torch.cuda.is_current_stream_capturing():
            self.workspace.record_stream(used)
        return stream

    def step(self, X, G, M, stream=None) -> None:
        """One optimizer step: X and M are updated in place."""
        x, g = self._pointers("X", X, self._x_dtype, 0), self._pointers("G", G, self._g_dtype, 1)
        m = self._pointers("M", M, self._torch.float32, 2)
        _separate("X, M", x + m, g)
        with _on_device(self._torch, self.workspace.get_device()):
            orthdion_muon_step(self.handle, x, g, m, self.workspace.data_ptr(), self.workspace_bytes, self._stream(stream))

    def orthogonalise(self, A, out, stream=None) -> None:
        """The orthogonalised A (laid out as G) into `out` (laid out as X)."""
        a, o = self._pointers("A", A, self._g_dtype, 1), self._pointers("out", out, self._x_dtype, 0)
        _separate("out", o, a)
        with _on_device(self._torch, self.workspace.get_device()):
            orthdion_muon_orthogonalise(self.handle, a, o, self.workspace.data_ptr(), self.workspace_bytes, self._stream(stream))

    def info(self, stream=None) -> List[int]:
        """Per matrix of the last call 0, or 1 where B (A) held a NaN or an infinity; from the workspace, so before anything else uses
        that, where it is shared.  Waits for the stream."""
        with _on_device(self._torch, self.workspace.get_device()):
            return orthdion_muon_get_info(self.handle, self.nmat, self._stream(stream))

    def set_lr(self, lr: float) -> None:
        orthdion_muon_set_lr(self.handle, lr)

    def set_mu(self, mu: float) -> None:
        orthdion_muon_set_mu(self.handle, mu)

    def set_weight_decay(self, weight_decay: float) -> None:
        orthdion_muon_set_weight_decay(self.handle, weight_decay)

    def close(self) -> None:
        if self.handle:
            orthdion_muon_destroy(self.handle)
            self.handle = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class AdamW:
    """Owns a handle of the AdamW step over a list of tensors; `lengths` are their numbers of elements.  `weight_decay` and
    `lr_scale` are one number or one per tensor.  A captured step is replayed with the lr of its capture."""

    def __init__(self, lengths, x_dtype="bf16", g_dtype=None, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, lr_scale=1.0):
        import torch
        self.handle = 0
        self._torch = torch
        self.lengths = [int(n) for n in lengths]
        count = len(self.lengths)
        (xc, self._x_dtype), (gc, self._g_dtype) = _dtypes(torch, x_dtype, g_dtype)
        self.handle = orthdion_adamw_create(self.lengths, xc, gc, lr, betas[0], betas[1], eps,
                                            _per_item("weight_decay", weight_decay, count), _per_item("lr_scale", lr_scale, count))

    def _separate_tensors(self, x, g, m, v) -> None:
        """Refuses one buffer for two of the tensors that the step writes, or for one of them and a gradient."""
        written = x + m + v
        once = set(written)
        if len(once) != len(written) or not once.isdisjoint(g):
            held = [[a for a, n in zip(seq, self.lengths) if n > 0] for seq in (x, m, v, g)]       # empty tensors have no memory
            _separate("X, M, V", held[0] + held[1] + held[2], held[3])

    def step(self, X, G, M, V, counter, stream=None) -> None:
        """One step: X, M and V are updated in place.  `counter` is an int32 tensor of two on the tensors' device, [steps taken
        so far, 0]; the step advances it there."""
        torch = self._torch
        if counter.device.type != "cuda" or counter.dtype != torch.int32 or tuple(counter.shape) != (2,) or not counter.is_contiguous():
            raise ValueError(f"counter: need an int32 device tensor of two, got {counter.dtype} {tuple(counter.shape)} on {counter.device}")
        tensor, device, addresses = torch.Tensor, {counter.get_device()}, []
        for name, seq, dtype in (("X", X, self._x_dtype), ("G", G, self._g_dtype), ("M", M, torch.float32), ("V", V, torch.float32)):
            # a handful of C calls a tensor; only what does not pass is looked at one by one
            if not (list(map(tensor.numel, seq)) == self.lengths and set(map(_dtype_of, seq)) == {dtype}
                    and set(map(tensor.get_device, seq)) == device and all(map(tensor.is_contiguous, seq))):
                if len(seq) != len(self.lengths):
                    raise ValueError(f"{name}: expected {len(self.lengths)} tensors, got {len(seq)}")
                for i, t in enumerate(seq):
                    if t.device != counter.device or t.dtype != dtype or t.numel() != self.lengths[i] or not t.is_contiguous():
                        raise ValueError(f"{name}[{i}]: need a contiguous {dtype} tensor of {self.lengths[i]} elements on {counter.device}, "
                                         f"got {t.dtype} {tuple(t.shape)} on {t.device}, contiguous={t.is_contiguous()}")
            addresses.append(list(map(tensor.data_ptr, seq)))
        self._separate_tensors(*addresses)
        with _on_device(torch, counter.get_device()):
            orthdion_adamw_step(self.handle, *addresses, counter.data_ptr(),
                                stream if stream is not None else torch.cuda.current_stream(counter.device).cuda_stream)

    def set_lr(self, lr: float) -> None:
        orthdion_adamw_set_lr(self.handle, lr)

    def close(self) -> None:
        if self.handle:
            orthdion_adamw_destroy(self.handle)
            self.handle = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
