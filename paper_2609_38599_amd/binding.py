"""ctypes binding of libjarq (include/jarq.h).

Argument marshalling only: every step of the refinement runs in the HIP
library.  torch provides device memory and the current stream.  Loading
fails loudly when the library has not been built.
"""

from __future__ import annotations

import contextlib
import ctypes
import os
import warnings
from typing import NamedTuple, Optional

import torch
from torch.autograd import forward_ad

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libjarq.so")

MAX_RECORDED_SWEEPS = 64
NUM_STAGES = 6           # Gram, scale solve, residual product, objective, Babai, panel update
STAGE_NAMES = ("gram", "solve", "residual", "objective", "babai", "panel")
ABI_VERSION = 9
(JARQ_OK, JARQ_EINVAL, JARQ_ENOT_SPD, JARQ_ESCALE_SOLVE, JARQ_EHIP, JARQ_EWORKSPACE,
 JARQ_ESTATIC_LIMIT) = range(7)
STATIC_WORKSPACE_BYTES = 512 << 20
DEC_REJECT, DEC_ACCEPT, DEC_SKIP, DEC_STOPPED = 0, 1, 2, 3


class JarqError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {status_string(status)} (status {status})")
        self.status = status


class Params(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("cols", ctypes.c_int32),
                ("group_size", ctypes.c_int32), ("bits", ctypes.c_int32),
                ("sweeps", ctypes.c_int32), ("tau", ctypes.c_float),
                ("ridge_lambda", ctypes.c_float), ("ridge_rcond", ctypes.c_float),
                ("ridge_accept", ctypes.c_int32)]


class Stats(ctypes.Structure):
    _fields_ = [("stage_mask", ctypes.c_uint32),
                ("sweeps_run", ctypes.c_int32), ("rows_active_end", ctypes.c_int32),
                ("objective_after_scales", ctypes.c_double * MAX_RECORDED_SWEEPS),
                ("accepted_groups", ctypes.c_int64 * MAX_RECORDED_SWEEPS),
                ("codes_changed", ctypes.c_int64 * MAX_RECORDED_SWEEPS),
                ("skipped_groups", ctypes.c_int64 * MAX_RECORDED_SWEEPS),
                ("ridge_rows", ctypes.c_int32 * MAX_RECORDED_SWEEPS),
                ("rows_active", ctypes.c_int32 * MAX_RECORDED_SWEEPS),
                ("correction_blocks", ctypes.c_int64 * MAX_RECORDED_SWEEPS),
                ("gram_listed", ctypes.c_int32 * MAX_RECORDED_SWEEPS),
                ("stage_ms", (ctypes.c_float * NUM_STAGES) * MAX_RECORDED_SWEEPS),
                ("prep_ms", ctypes.c_float)]

    def to_dict(self):
        n = min(self.sweeps_run, MAX_RECORDED_SWEEPS)
        return {
            "stage_mask": self.stage_mask,
            "sweeps_run": self.sweeps_run,
            "rows_active_end": self.rows_active_end,
            "objective_after_scales": [self.objective_after_scales[k] for k in range(n)],
            "accepted_groups": [self.accepted_groups[k] for k in range(n)],
            "codes_changed": [self.codes_changed[k] for k in range(n)],
            "skipped_groups": [self.skipped_groups[k] for k in range(n)],
            "ridge_rows": [self.ridge_rows[k] for k in range(n)],
            "rows_active": [self.rows_active[k] for k in range(n)],
            "correction_blocks": [self.correction_blocks[k] for k in range(n)],
            "gram_listed": [self.gram_listed[k] for k in range(n)],
            "stage_ms": [list(self.stage_ms[k]) for k in range(n)],
            "prep_ms": self.prep_ms,
        }


_vp, _i32, _i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
_f32 = ctypes.c_float


class _AdamWArrays(ctypes.Structure):
    _fields_ = [(n, _vp) for n in ("master", "m", "v", "m_exp", "v_exp")]


class _AdamWOptions(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay")] + [
        ("step", _i64), ("seed", ctypes.c_uint64), ("lr_at", _vp), ("step_at", _vp),
        ("grad_mul", _vp)]


_SIGNATURES = {
    "jarq_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(Params)]),
    "jarq_prepare": (ctypes.c_int, [ctypes.POINTER(Params), _vp, _vp, _vp, ctypes.c_size_t, _vp]),
    "jarq_scale_step": (ctypes.c_int, [ctypes.POINTER(Params), _vp, _vp, _vp, _vp, _vp,
                                       ctypes.c_size_t, _vp]),
    "jarq_code_step": (ctypes.c_int, [ctypes.POINTER(Params), _vp, _vp, _vp, _vp, _vp, _vp,
                                      ctypes.c_size_t, _vp, _vp, _vp]),
    "jarq_sweeps": (ctypes.c_int, [ctypes.POINTER(Params), _vp, _vp, _vp, _vp, _vp, _vp,
                                   ctypes.c_size_t, _vp, ctypes.POINTER(Stats)]),
    "jarq_refine": (ctypes.c_int, [ctypes.POINTER(Params), _vp, _vp, _vp, _vp, _vp, _vp,
                                   ctypes.c_size_t, _vp, ctypes.POINTER(Stats)]),
    "jarq_refine_static": (ctypes.c_int, [ctypes.POINTER(Params), _vp, _vp, _vp, _vp, _vp, _vp,
                                          ctypes.POINTER(Stats)]),
    "jarq_objective": (ctypes.c_int, [ctypes.POINTER(Params), _vp, _vp, _vp, _vp, _vp, _vp,
                                      ctypes.c_size_t, _vp, _vp]),
    "jarq_stop_sweeps": (ctypes.c_int, [ctypes.POINTER(Params), _vp, ctypes.c_size_t, _vp, _vp]),
    "jarq_hessian_accumulate": (ctypes.c_int, [_vp, ctypes.c_int64, ctypes.c_int32, ctypes.c_double,
                                               _vp, _vp]),
    "jarq_hessian_accumulate_bf16": (ctypes.c_int, [_vp, ctypes.c_int64, ctypes.c_int32,
                                                    ctypes.c_double, _vp, _vp]),
    "jarq_hessian_finalize": (ctypes.c_int, [_vp, ctypes.c_int32, ctypes.c_double, ctypes.c_double,
                                             _vp, _vp]),
    "jarq_rtn": (ctypes.c_int, [ctypes.POINTER(Params), _vp, _vp, _vp, _vp, _vp]),
    "jarq_cross_accumulate": (ctypes.c_int, [_vp, _vp, ctypes.c_int64, ctypes.c_int32,
                                             ctypes.c_double, _vp, _vp]),
    "jarq_qep_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(Params)]),
    "jarq_qep_correct": (ctypes.c_int, [ctypes.POINTER(Params), _vp, _vp, _vp, ctypes.c_double,
                                        _vp, _vp, ctypes.c_size_t, _vp]),
    "jarq_canonicalize": (ctypes.c_int, [ctypes.POINTER(Params), _vp, _vp, _vp, _vp]),
    "jarq_dequantize": (ctypes.c_int, [ctypes.POINTER(Params), _vp, _vp, _vp, _vp, ctypes.c_int32,
                                       _vp, _vp]),
    "jarq_pack_codes": (ctypes.c_int, [ctypes.POINTER(Params), _vp, _vp, _vp]),
    "jarq_unpack_codes": (ctypes.c_int, [ctypes.POINTER(Params), _vp, _vp, _vp]),
    "jarq_act_order": (ctypes.c_int, [_vp, ctypes.c_int32, _vp, _vp]),
    "jarq_permute": (ctypes.c_int, [ctypes.POINTER(Params), _vp, _vp, _vp, _vp, _vp, _vp]),
    "jarq_gptq_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(Params)]),
    "jarq_gptq": (ctypes.c_int, [ctypes.POINTER(Params), _vp, _vp, _vp, _vp, _vp, _vp,
                                 ctypes.c_size_t, _vp]),
    "jarq_gated_forward": (ctypes.c_int, [_i32, _i32, _i64, _i32, _i32, _vp, _vp, _vp, _vp, _vp,
                                          _vp]),
    "jarq_gated_workspace_bytes": (ctypes.c_size_t, [_i64, _i32, _i32]),
    "jarq_gated_backward": (ctypes.c_int, [_i32, _i32, _i64, _i32, _i32, _vp, _vp, _vp, _vp, _vp,
                                           _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]),
    "jarq_quant_rows_i8": (ctypes.c_int, [_i32, _vp, _i64, _i32, _vp, _vp, _vp]),
    "jarq_codes_i8": (ctypes.c_int, [ctypes.POINTER(Params), _vp, _vp, _vp, _vp, _vp]),
    "jarq_matmul_i8": (ctypes.c_int, [_i32, _i64, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp]),
    "jarq_linear_i8_workspace_bytes": (ctypes.c_size_t, [_i64, _i32]),
    "jarq_linear_i8": (ctypes.c_int, [_i32, _i64, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp,
                                      ctypes.c_size_t, _vp]),
    "jarq_token_logprobs_workspace_bytes": (ctypes.c_size_t, [_i64, _i32, _i32]),
    "jarq_token_logprobs": (ctypes.c_int, [_i32, _vp, _i64, _i64, _i32, _vp, _i32, _vp, _vp, _vp,
                                           _vp, _vp, _vp, ctypes.c_size_t, _vp]),
    "jarq_token_logprobs_backward": (ctypes.c_int, [_i32, _vp, _i64, _i64, _i32, _vp, _vp, _vp,
                                                    _vp, _vp, _vp, _i64, _vp]),
    "jarq_token_logprobs_keep": (ctypes.c_int, [_i32, _vp, _i64, _i64, _i32, _vp, _i32, _vp, _vp,
                                                _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]),
    "jarq_token_logprobs_keep_backward": (ctypes.c_int, [_i32, _vp, _i64, _i64, _i32, _vp, _vp,
                                                         _vp, _vp, _vp, _vp, _vp, _i64, _vp]),
    "jarq_rms_norm": (ctypes.c_int, [_i32, _i32, _i64, _i32, _vp, _vp, _vp, _f32, _vp, _vp, _vp]),
    "jarq_rms_norm_i8": (ctypes.c_int, [_i32, _i32, _i64, _i32, _vp, _vp, _vp, _f32, _vp, _vp, _vp,
                                        _vp]),
    "jarq_rms_norm_workspace_bytes": (ctypes.c_size_t, [_i64, _i32]),
    "jarq_rms_norm_backward": (ctypes.c_int, [_i32, _i32, _i64, _i32, _vp, _vp, _vp, _vp, _f32,
                                              _vp, _vp, _vp, ctypes.c_size_t, _vp]),
    "jarq_linear_logprobs_workspace_bytes": (ctypes.c_size_t, [_i64, _i32, _i32]),
    "jarq_linear_logprobs": (ctypes.c_int, [_i32, _i64, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp,
                                            _vp, ctypes.c_size_t, _vp]),
    "jarq_linear_logprobs_backward_workspace_bytes": (ctypes.c_size_t, [_i64, _i32, _i32]),
    "jarq_linear_logprobs_backward": (ctypes.c_int, [_i32, _i64, _i32, _i32, _vp, _vp, _vp, _vp,
                                                     _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                                     ctypes.c_size_t, _vp]),
    "jarq_adamw_state_length": (_i64, [_i32, _vp]),
    "jarq_adamw_step": (ctypes.c_int, [_i32, _i32, _i32, _vp, ctypes.POINTER(_AdamWArrays),
                                       ctypes.POINTER(_AdamWArrays),
                                       ctypes.POINTER(_AdamWOptions), _vp]),
    "jarq_lds_probe": (ctypes.c_int64, [ctypes.c_int32, ctypes.c_int32, _vp, _vp]),
    "jarq_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "jarq_abi_version": (ctypes.c_int32, []),
}
EXPORTED = tuple(_SIGNATURES)

_lib = None


def load_library(path: str = LIB_PATH):
    """Load libjarq.so; raises ImportError if it is missing (no fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError(f"libjarq.so not built at {path}; run paper_2609_38599_amd/build.py")
    lib = ctypes.CDLL(path)
    for name, (res, args) in _SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    if lib.jarq_abi_version() != ABI_VERSION:
        raise ImportError(f"{path} has ABI version {lib.jarq_abi_version()}, this binding expects "
                          f"{ABI_VERSION}; rebuild with paper_2609_38599_amd/build.py")
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().jarq_status_string(int(status)).decode()


def make_params(rows, cols, group_size, bits, sweeps=1, tau=-1.0, ridge_lambda=1e-4,
                ridge_rcond=1e-10, ridge_accept=False) -> Params:
    return Params(int(rows), int(cols), int(group_size), int(bits), int(sweeps), float(tau),
                  float(ridge_lambda), float(ridge_rcond), int(bool(ridge_accept)))


def workspace_bytes(p: Params) -> int:
    return int(load_library().jarq_workspace_bytes(ctypes.byref(p)))


def alloc_workspace(p: Params, device=None) -> torch.Tensor:
    n = workspace_bytes(p)
    if n == 0:
        raise JarqError(JARQ_EINVAL, "workspace_bytes")
    ws = torch.empty(n + 256, dtype=torch.uint8, device=device or "cuda")
    off = (-ws.data_ptr()) % 256
    return ws[off:off + n]


def _ptr(t, dtype, name):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _check(status, what):
    if status != JARQ_OK:
        raise JarqError(status, what)


def prepare(p: Params, W, H, ws, stream=None):
    lib = load_library()
    _check(lib.jarq_prepare(ctypes.byref(p), _ptr(W, torch.float32, "W"),
                            _ptr(H, torch.float32, "H"), _ptr(ws, torch.uint8, "workspace"),
                            ws.numel(), _stream(stream)), "jarq_prepare")


def scale_step(p: Params, H, codes, scales, zeros, ws, stream=None):
    lib = load_library()
    _check(lib.jarq_scale_step(ctypes.byref(p), _ptr(H, torch.float32, "H"),
                               _ptr(codes, torch.uint8, "codes"),
                               _ptr(scales, torch.float32, "scales"),
                               _ptr(zeros, torch.int32, "zeros"),
                               _ptr(ws, torch.uint8, "workspace"), ws.numel(), _stream(stream)),
           "jarq_scale_step")


def code_step(p: Params, W, H, codes, scales, zeros, ws, cand=None, decision=None, stream=None):
    lib = load_library()
    _check(lib.jarq_code_step(ctypes.byref(p), _ptr(W, torch.float32, "W"),
                              _ptr(H, torch.float32, "H"), _ptr(codes, torch.uint8, "codes"),
                              _ptr(scales, torch.float32, "scales"),
                              _ptr(zeros, torch.int32, "zeros"),
                              _ptr(ws, torch.uint8, "workspace"), ws.numel(), _stream(stream),
                              _ptr(cand, torch.uint8, "cand"),
                              _ptr(decision, torch.uint8, "decision")), "jarq_code_step")


def sweeps(p: Params, W, H, codes, scales, zeros, ws, stream=None, want_stats=True, check=True,
           stage_mask=0):
    """jarq_sweeps; stage_mask selects the stages timed with HIP events (0 = all)."""
    lib = load_library()
    st = Stats() if want_stats else None
    if st is not None:
        st.stage_mask = stage_mask
    status = lib.jarq_sweeps(ctypes.byref(p), _ptr(W, torch.float32, "W"),
                             _ptr(H, torch.float32, "H"), _ptr(codes, torch.uint8, "codes"),
                             _ptr(scales, torch.float32, "scales"),
                             _ptr(zeros, torch.int32, "zeros"),
                             _ptr(ws, torch.uint8, "workspace"), ws.numel(), _stream(stream),
                             ctypes.byref(st) if st is not None else None)
    if check:
        _check(status, "jarq_sweeps")
    return (st.to_dict() if st is not None else None) if check else (status, st)


def refine(p: Params, W, H, codes, scales, zeros, ws, stream=None, want_stats=True, check=True,
           stage_mask=0):
    lib = load_library()
    st = Stats() if want_stats else None
    if st is not None:
        st.stage_mask = stage_mask
    status = lib.jarq_refine(ctypes.byref(p), _ptr(W, torch.float32, "W"),
                             _ptr(H, torch.float32, "H"), _ptr(codes, torch.uint8, "codes"),
                             _ptr(scales, torch.float32, "scales"),
                             _ptr(zeros, torch.int32, "zeros"),
                             _ptr(ws, torch.uint8, "workspace"), ws.numel(), _stream(stream),
                             ctypes.byref(st) if st is not None else None)
    if check:
        _check(status, "jarq_refine")
    return (st.to_dict() if st is not None else None) if check else (status, st)


def refine_static(p: Params, W, H, codes, scales, zeros, stream=None, want_stats=True,
                  check=True):
    """jarq_refine_static: jarq_refine on the library's static workspace (no allocation)."""
    lib = load_library()
    st = Stats() if want_stats else None
    status = lib.jarq_refine_static(ctypes.byref(p), _ptr(W, torch.float32, "W"),
                                    _ptr(H, torch.float32, "H"), _ptr(codes, torch.uint8, "codes"),
                                    _ptr(scales, torch.float32, "scales"),
                                    _ptr(zeros, torch.int32, "zeros"), _stream(stream),
                                    ctypes.byref(st) if st is not None else None)
    if check:
        _check(status, "jarq_refine_static")
    return (st.to_dict() if st is not None else None) if check else (status, st)


def objective(p: Params, W, H, codes, scales, zeros, ws, out=None, stream=None):
    lib = load_library()
    if out is None:
        out = torch.empty(p.rows, dtype=torch.float64, device=W.device)
    _check(lib.jarq_objective(ctypes.byref(p), _ptr(W, torch.float32, "W"),
                              _ptr(H, torch.float32, "H"), _ptr(codes, torch.uint8, "codes"),
                              _ptr(scales, torch.float32, "scales"),
                              _ptr(zeros, torch.int32, "zeros"),
                              _ptr(ws, torch.uint8, "workspace"), ws.numel(), _stream(stream),
                              _ptr(out, torch.float64, "row_objective")), "jarq_objective")
    return out


def stop_sweeps(p: Params, ws, out=None, stream=None):
    """Per row, the iteration at which the last sweeps call stopped it (0 = never)."""
    lib = load_library()
    if out is None:
        out = torch.empty(p.rows, dtype=torch.int32, device=ws.device)
    _check(lib.jarq_stop_sweeps(ctypes.byref(p), _ptr(ws, torch.uint8, "workspace"), ws.numel(),
                                _ptr(out, torch.int32, "stop_sweep"), _stream(stream)),
           "jarq_stop_sweeps")
    return out


def hessian_accumulate(X, Hacc, alpha=1.0, stream=None):
    """Hacc += alpha X^T X for one chunk X [m, d] fp32 or bf16 (Hacc [d, d] fp64)."""
    lib = load_library()
    if X.dim() != 2 or Hacc.shape != (X.shape[1], X.shape[1]):
        raise ValueError("X must be [m, d] and Hacc [d, d]")
    if X.dtype == torch.bfloat16:
        _check(lib.jarq_hessian_accumulate_bf16(_ptr(X, torch.bfloat16, "X"), X.shape[0],
                                                X.shape[1], float(alpha),
                                                _ptr(Hacc, torch.float64, "Hacc"), _stream(stream)),
               "jarq_hessian_accumulate_bf16")
        return
    _check(lib.jarq_hessian_accumulate(_ptr(X, torch.float32, "X"), X.shape[0], X.shape[1],
                                       float(alpha), _ptr(Hacc, torch.float64, "Hacc"),
                                       _stream(stream)), "jarq_hessian_accumulate")


def hessian_finalize(Hacc, damp=0.0, nu2=0.0, out=None, stream=None):
    """H = Hacc + (damp mean(diag Hacc) + nu2) I as fp32."""
    lib = load_library()
    d = Hacc.shape[0]
    if Hacc.dim() != 2 or Hacc.shape[1] != d:
        raise ValueError("Hacc must be square")
    if out is None:
        out = torch.empty(d, d, dtype=torch.float32, device=Hacc.device)
    _check(lib.jarq_hessian_finalize(_ptr(Hacc, torch.float64, "Hacc"), d, float(damp),
                                     float(nu2), _ptr(out, torch.float32, "H"), _stream(stream)),
           "jarq_hessian_finalize")
    return out


def hessian(chunks, d, alpha=1.0, damp=0.0, nu2=0.0, device=None, stream=None):
    """The fp32 Hessian of a stream of fp32 device chunks [m_c, d]."""
    Hacc = torch.zeros(d, d, dtype=torch.float64, device=device or "cuda")
    for X in chunks:
        hessian_accumulate(X, Hacc, alpha, stream)
    return hessian_finalize(Hacc, damp, nu2, stream=stream)


def rtn(p: Params, W, codes=None, scales=None, zeros=None, stream=None):
    """Round-to-nearest host state (codes, scales, zeros) of W."""
    lib = load_library()
    G = p.cols // p.group_size
    dev = W.device
    if codes is None:
        codes = torch.empty(p.rows, p.cols, dtype=torch.uint8, device=dev)
    if scales is None:
        scales = torch.empty(p.rows, G, dtype=torch.float32, device=dev)
    if zeros is None:
        zeros = torch.empty(p.rows, G, dtype=torch.int32, device=dev)
    _check(lib.jarq_rtn(ctypes.byref(p), _ptr(W, torch.float32, "W"),
                        _ptr(codes, torch.uint8, "codes"), _ptr(scales, torch.float32, "scales"),
                        _ptr(zeros, torch.int32, "zeros"), _stream(stream)), "jarq_rtn")
    return codes, scales, zeros


DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


def canonicalize(p: Params, codes, scales, zeros, stream=None):
    """In place: groups with a negative scale get s' = -s, q' = qmax - q, z' = qmax - z."""
    lib = load_library()
    _check(lib.jarq_canonicalize(ctypes.byref(p), _ptr(codes, torch.uint8, "codes"),
                                 _ptr(scales, torch.float32, "scales"),
                                 _ptr(zeros, torch.int32, "zeros"), _stream(stream)),
           "jarq_canonicalize")


def dequantize(p: Params, codes, scales, zeros, dtype=torch.float32, perm=None, out=None,
               stream=None):
    """s (q - z) as `dtype`; with perm, written back in the original column order."""
    lib = load_library()
    if out is None:
        out = torch.empty(p.rows, p.cols, dtype=dtype, device=codes.device)
    _check(lib.jarq_dequantize(ctypes.byref(p), _ptr(codes, torch.uint8, "codes"),
                               _ptr(scales, torch.float32, "scales"),
                               _ptr(zeros, torch.int32, "zeros"), _ptr(perm, torch.int32, "perm"),
                               DTYPES[out.dtype], _ptr(out, out.dtype, "out"), _stream(stream)),
           "jarq_dequantize")
    return out


def packed_words_per_row(p: Params) -> int:
    return (p.cols * p.bits + 31) // 32


def pack_codes(p: Params, codes, out=None, stream=None):
    lib = load_library()
    if out is None:
        out = torch.empty(p.rows, packed_words_per_row(p), dtype=torch.int32, device=codes.device)
    _check(lib.jarq_pack_codes(ctypes.byref(p), _ptr(codes, torch.uint8, "codes"),
                               _ptr(out, torch.int32, "packed"), _stream(stream)),
           "jarq_pack_codes")
    return out


def unpack_codes(p: Params, packed, out=None, stream=None):
    lib = load_library()
    if out is None:
        out = torch.empty(p.rows, p.cols, dtype=torch.uint8, device=packed.device)
    _check(lib.jarq_unpack_codes(ctypes.byref(p), _ptr(packed, torch.int32, "packed"),
                                 _ptr(out, torch.uint8, "codes"), _stream(stream)),
           "jarq_unpack_codes")
    return out


def act_order(H, out=None, stream=None):
    lib = load_library()
    d = H.shape[0]
    if out is None:
        out = torch.empty(d, dtype=torch.int32, device=H.device)
    _check(lib.jarq_act_order(_ptr(H, torch.float32, "H"), d, _ptr(out, torch.int32, "perm"),
                              _stream(stream)), "jarq_act_order")
    return out


def permute(p: Params, perm, W, H, stream=None):
    lib = load_library()
    Wp, Hp = torch.empty_like(W), torch.empty_like(H)
    _check(lib.jarq_permute(ctypes.byref(p), _ptr(perm, torch.int32, "perm"),
                            _ptr(W, torch.float32, "W"), _ptr(H, torch.float32, "H"),
                            _ptr(Wp, torch.float32, "Wp"), _ptr(Hp, torch.float32, "Hp"),
                            _stream(stream)), "jarq_permute")
    return Wp, Hp


def _scratch(n, dev):
    raw = torch.empty(n + 256, dtype=torch.uint8, device=dev)
    off = (-raw.data_ptr()) % 256
    return raw[off:off + n]


def cross_accumulate(Xq, X, Dacc, alpha=1.0, stream=None):
    """Dacc += alpha Xq^T (X - Xq) for one chunk of tokens (Dacc [d, d] fp64)."""
    lib = load_library()
    if Xq.shape != X.shape or Xq.dim() != 2 or Dacc.shape != (X.shape[1], X.shape[1]):
        raise ValueError("Xq and X must be [m, d] and Dacc [d, d]")
    _check(lib.jarq_cross_accumulate(_ptr(Xq, torch.float32, "Xq"), _ptr(X, torch.float32, "X"),
                                     X.shape[0], X.shape[1], float(alpha),
                                     _ptr(Dacc, torch.float64, "Dacc"), _stream(stream)),
           "jarq_cross_accumulate")


def qep_correct(p: Params, W, H, D, mu, out=None, ws=None, stream=None):
    """W_corr = W + (1 - mu) (W D^T) H^{-1} (fp32)."""
    lib = load_library()
    if out is None:
        out = torch.empty_like(W)
    n = int(lib.jarq_qep_workspace_bytes(ctypes.byref(p)))
    if n == 0:
        raise JarqError(JARQ_EINVAL, "jarq_qep_workspace_bytes")
    if ws is None:
        ws = _scratch(n, W.device)
    _check(lib.jarq_qep_correct(ctypes.byref(p), _ptr(W, torch.float32, "W"),
                                _ptr(H, torch.float32, "H"), _ptr(D, torch.float64, "D"),
                                float(mu), _ptr(out, torch.float32, "Wcorr"),
                                _ptr(ws, torch.uint8, "workspace"), ws.numel(), _stream(stream)),
           "jarq_qep_correct")
    return out


def gptq(p: Params, W, H, codes=None, scales=None, zeros=None, ws=None, stream=None):
    """GPTQ-style host state (codes, scales, zeros) of W under H."""
    lib = load_library()
    G = p.cols // p.group_size
    dev = W.device
    if codes is None:
        codes = torch.empty(p.rows, p.cols, dtype=torch.uint8, device=dev)
    if scales is None:
        scales = torch.empty(p.rows, G, dtype=torch.float32, device=dev)
    if zeros is None:
        zeros = torch.empty(p.rows, G, dtype=torch.int32, device=dev)
    n = int(lib.jarq_gptq_workspace_bytes(ctypes.byref(p)))
    if n == 0:
        raise JarqError(JARQ_EINVAL, "jarq_gptq_workspace_bytes")
    if ws is None:
        raw = torch.empty(n + 256, dtype=torch.uint8, device=dev)
        off = (-raw.data_ptr()) % 256
        ws = raw[off:off + n]
    _check(lib.jarq_gptq(ctypes.byref(p), _ptr(W, torch.float32, "W"), _ptr(H, torch.float32, "H"),
                         _ptr(codes, torch.uint8, "codes"), _ptr(scales, torch.float32, "scales"),
                         _ptr(zeros, torch.int32, "zeros"), _ptr(ws, torch.uint8, "workspace"),
                         ws.numel(), _stream(stream)), "jarq_gptq")
    return codes, scales, zeros


# ---- running, training and evaluating refined layers ----

ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2}


_INLINE = contextlib.nullcontext()


def _on(stream):
    """Where a call's own allocations belong: the stream that it runs on."""
    return _INLINE if stream is None else torch.cuda.stream(stream)


def _device(t, name):
    """The device of a call, t's.  It has to be the current one, where kernels are launched."""
    at = t.get_device()
    if at < 0:
        raise ValueError(f"{name} must be a device tensor")
    if at != torch._C._cuda_getDevice():
        raise ValueError(f"{name} is on cuda:{at}, but cuda:{torch._C._cuda_getDevice()} is the "
                         "current device (torch.cuda.set_device or torch.cuda.device changes it)")
    return at


def _at(t, dtype, name, device):
    """The address of a dense tensor on the call's device, None without one."""
    if t is None:
        return None
    try:
        if t.dtype == dtype and t.get_device() == device and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        raise TypeError(f"{name} must be a torch.Tensor") from None
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.get_device() != device:
        raise ValueError(f"{name} must be on cuda:{device}, got {t.device}")
    raise ValueError(f"{name} must be contiguous")


def _own(t):
    """The address of a tensor that the call made itself, None without one."""
    return None if t is None else t.data_ptr()


def _queue(stream, device):
    """The handle of `stream`, by default the current one of the call's device.

    (The raw handle: a Stream object of the current stream takes 2.7 us to make.)
    """
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device)
    if stream.device_index != device:
        raise ValueError(f"stream must be of cuda:{device}, got cuda:{stream.device_index}")
    return stream.cuda_stream


def _work(n, like):
    """n bytes of workspace on like's device, aligned to 256 bytes."""
    ws = torch.empty(n, dtype=torch.uint8, device=like.device)
    return ws if ws.data_ptr() % 256 == 0 else _scratch(n, like.device)


_written = torch.autograd.graph.increment_version


def _wrote(*tensors):
    """Tells autograd that a call has written into these tensors (or None).

    A backward pass that kept one of them then says that it is no longer what it was.
    """
    _written([t for t in tensors if t is not None])


def _dual(*tensors):
    """Whether one of them (or None) carries a tangent of forward-mode differentiation."""
    return forward_ad._current_level >= 0 and any(
        t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors)


def _outside(call, gradient):
    """Says that the result of an input that requires a gradient or has a tangent is none of autograd's."""
    if torch.is_grad_enabled():
        warnings.warn(f"{call}: the result is outside autograd's graph; {gradient} "
                      "(this is not said under torch.no_grad())", stacklevel=3)


def _rows(t, name, cols=None):
    if not isinstance(t, torch.Tensor) or t.dim() != 2 or (cols is not None and t.shape[1] != cols):
        raise ValueError(f"{name} must be [rows, {'cols' if cols is None else cols}]")
    return t.shape


def _act(act):
    if act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}, got {act!r}")
    return ACTIVATIONS[act]


def _dtype(t, name):
    if t.dtype not in DTYPES:
        raise TypeError(f"{name} must be float32, float16 or bfloat16, got {t.dtype}")
    return DTYPES[t.dtype]


def gated_forward(X, Wg, Wu, act="silu", out=None, save=False, stream=None):
    """act(X Wg^T) * (X Wu^T) for X [tokens, d], Wg and Wu [f, d] in 16 bits.

    With save, returns (Y, pre): pre [2, tokens, f] fp32 is for gated_backward, which gives the
    gradients; autograd records none.
    """
    lib = load_library()
    T, d = _rows(X, "X")
    f, _ = _rows(Wg, "Wg", d)
    at = _device(X, "X")
    if _rows(Wu, "Wu", d)[0] != f:
        raise ValueError("Wg and Wu must have the same shape")
    pre, given = None, out is not None
    if (not save and (X.requires_grad or Wg.requires_grad or Wu.requires_grad)
            or _dual(X, Wg, Wu)):
        _outside("gated_forward", "gated_backward gives its gradients, from save=True")
    with _on(stream):
        if out is None:
            out = torch.empty(T, f, dtype=X.dtype, device=X.device)
        elif out.shape != (T, f):
            raise ValueError("out must be [tokens, f]")
        if save:
            pre = torch.empty(2, T, f, dtype=torch.float32, device=X.device)
    dt = X.dtype
    _check(lib.jarq_gated_forward(_dtype(X, "X"), _act(act), T, d, f, _at(X, dt, "X", at),
                                  _at(Wg, dt, "Wg", at), _at(Wu, dt, "Wu", at),
                                  _at(out, dt, "out", at), _own(pre),
                                  _queue(stream, at)),
           "jarq_gated_forward")
    if given:
        _wrote(out)
    return (out, pre) if save else out


def gated_workspace_bytes(tokens, d, f) -> int:
    return int(load_library().jarq_gated_workspace_bytes(tokens, d, f))


def gated_backward(X, Wg, Wu, dY, pre, act="silu", need=(True, True, True), ws=None, stream=None):
    """(dX, dWg, dWu) of gated_forward for dY [tokens, f]; None where not needed."""
    lib = load_library()
    T, d = _rows(X, "X")
    f, _ = _rows(Wg, "Wg", d)
    at = _device(X, "X")
    if _rows(Wu, "Wu", d)[0] != f or _rows(dY, "dY", f)[0] != T or pre.shape != (2, T, f):
        raise ValueError("Wg and Wu must be [f, d], dY [tokens, f] and pre [2, tokens, f]")
    n = int(lib.jarq_gated_workspace_bytes(T, d, f))
    if n == 0:
        raise JarqError(JARQ_EINVAL, "jarq_gated_workspace_bytes")
    dt = X.dtype
    with _on(stream):
        dX, dWg, dWu = (torch.empty_like(t) if wanted else None
                        for t, wanted in zip((X, Wg, Wu), need))
        if ws is None:
            ws = _work(n, X)
    _check(lib.jarq_gated_backward(_dtype(X, "X"), _act(act), T, d, f, _at(X, dt, "X", at),
                                   _at(Wg, dt, "Wg", at), _at(Wu, dt, "Wu", at),
                                   _at(dY, dt, "dY", at), _at(pre, torch.float32, "pre", at),
                                   _own(dX), _own(dWg), _own(dWu),
                                   _at(ws, torch.uint8, "workspace", at), ws.numel(),
                                   _queue(stream, at)), "jarq_gated_backward")
    return dX, dWg, dWu


def quant_rows_i8(X, out=None, scale=None, stream=None):
    """(Q int8, scale fp32 [rows, 1]): the rows of X on 8 bits with a scale each."""
    lib = load_library()
    rows, cols = _rows(X, "X")
    at = _device(X, "X")
    given = out is not None or scale is not None
    with _on(stream):
        if out is None:
            out = torch.empty(rows, cols, dtype=torch.int8, device=X.device)
        if scale is None:
            scale = torch.empty(rows, 1, dtype=torch.float32, device=X.device)
    if out.shape != (rows, cols) or scale.numel() != rows:
        raise ValueError("out must be [rows, cols] and scale hold one value a row")
    _check(lib.jarq_quant_rows_i8(_dtype(X, "X"), _at(X, X.dtype, "X", at), rows, cols,
                                  _at(out, torch.int8, "out", at),
                                  _at(scale, torch.float32, "scale", at), _queue(stream, at)),
           "jarq_quant_rows_i8")
    if given:
        _wrote(out, scale)
    return out, scale


def codes_i8(p: Params, codes, zeros, out=None, stream=None):
    """q - z as int8: a quantized layer's weights for matmul_i8 and linear_i8."""
    lib = load_library()
    at = _device(codes, "codes")
    given = out is not None
    with _on(stream):
        if out is None:
            out = torch.empty(p.rows, p.cols, dtype=torch.int8, device=codes.device)
        flag = torch.empty(1, dtype=torch.int32, device=codes.device)
    n = p.rows * p.cols
    if codes.numel() != n or out.numel() != n or zeros.numel() * p.group_size != n:
        raise ValueError("codes and out must be [rows, cols], zeros [rows, cols / group_size]")
    _check(lib.jarq_codes_i8(ctypes.byref(p), _at(codes, torch.uint8, "codes", at),
                             _at(zeros, torch.int32, "zeros", at), _at(out, torch.int8, "out", at),
                             _own(flag), _queue(stream, at)),
           "jarq_codes_i8")
    if given:
        _wrote(out)
    return out


def _i8_layer(Wq, sw, k):
    """(n, group) of a layer's integers [n, k] with scales [n, 1] or [n, k / group]."""
    n, _ = _rows(Wq, "Wq", k)
    rows, groups = _rows(sw, "sw")
    if rows != n or groups < 1 or k % groups != 0:
        raise ValueError("sw must be [n, 1] or [n, k / group]")
    return n, 0 if groups == 1 else k // groups


def matmul_i8(Xq, sx, Wq, sw, dtype=torch.bfloat16, out=None, stream=None):
    """sx (Xq Wq^T under the scales sw [n, 1] or [n, k / group]) as `dtype`.  Has no gradient."""
    lib = load_library()
    T, k = _rows(Xq, "Xq")
    n, group = _i8_layer(Wq, sw, k)
    at = _device(Xq, "Xq")
    if sx.numel() != T:
        raise ValueError("sx must hold one scale a token")
    if sx.requires_grad or sw.requires_grad or _dual(sx, sw):
        _outside("matmul_i8", "it has no gradient")
    given = out is not None
    with _on(stream):
        if out is None:
            out = torch.empty(T, n, dtype=dtype, device=Xq.device)
        elif out.shape != (T, n):
            raise ValueError("out must be [tokens, n]")
    _check(lib.jarq_matmul_i8(_dtype(out, "out"), T, n, k, group, _at(Xq, torch.int8, "Xq", at),
                              _at(sx, torch.float32, "sx", at), _at(Wq, torch.int8, "Wq", at),
                              _at(sw, torch.float32, "sw", at), _at(out, out.dtype, "out", at),
                              _queue(stream, at)), "jarq_matmul_i8")
    if given:
        _wrote(out)
    return out


def linear_i8(X, Wq, sw, out=None, ws=None, stream=None):
    """X [tokens, k] through the 8-bit layer (Wq [n, k], sw [n, 1] or [n, k / group]).

    Has no gradient.
    """
    lib = load_library()
    T, k = _rows(X, "X")
    n, group = _i8_layer(Wq, sw, k)
    at = _device(X, "X")
    need = int(lib.jarq_linear_i8_workspace_bytes(T, k))
    if need == 0:
        raise JarqError(JARQ_EINVAL, "jarq_linear_i8_workspace_bytes")
    if X.requires_grad or sw.requires_grad or _dual(X, sw):
        _outside("linear_i8", "it has no gradient")
    dt, given = X.dtype, out is not None
    with _on(stream):
        if out is None:
            out = torch.empty(T, n, dtype=dt, device=X.device)
        elif out.shape != (T, n):
            raise ValueError("out must be [tokens, n]")
        if ws is None:
            ws = _work(need, X)
    _check(lib.jarq_linear_i8(_dtype(X, "X"), T, n, k, group, _at(X, dt, "X", at),
                              _at(Wq, torch.int8, "Wq", at), _at(sw, torch.float32, "sw", at),
                              _at(out, dt, "out", at), _at(ws, torch.uint8, "workspace", at),
                              ws.numel(), _queue(stream, at)), "jarq_linear_i8")
    if given:
        _wrote(out)
    return out


class _TokenLogprobs(NamedTuple):
    logprob: torch.Tensor                  # [tokens] fp32
    entropy: torch.Tensor                  # [tokens] fp32
    lse: torch.Tensor                      # [tokens] fp32: log sum exp of the row
    top_index: Optional[torch.Tensor]      # [tokens, top] int32
    top_logprob: Optional[torch.Tensor]    # [tokens, top] fp32


class TokenLogprobs(_TokenLogprobs):
    """What token_logprobs returns; lse_rest [tokens] fp32 is what rounding left of lse.

    A tuple made otherwise has no lse_rest: the backward pass then reads the logits twice.
    """

    lse_rest: Optional[torch.Tensor] = None


def _logits(t, name):
    """(tokens, vocab, row stride) of logits whose rows are dense."""
    T, V = _rows(t, name)
    if V > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must have dense rows")
    ld = t.stride(0) if T > 1 else V
    if ld < V:
        raise ValueError(f"{name} must not have overlapping rows")
    return T, V, ld


def token_logprobs(logits, targets, top=0, ws=None, stream=None) -> TokenLogprobs:
    """Log probabilities of targets [tokens] int64 (< 0: none), entropies, top alternatives.

    token_logprobs_backward gives the logits' gradient; autograd records none.
    """
    lib = load_library()
    T, V, ld = _logits(logits, "logits")
    at = _device(logits, "logits")
    if targets.shape != (T,):
        raise ValueError("targets must be [tokens]")
    n = int(lib.jarq_token_logprobs_workspace_bytes(T, V, top))
    if n == 0:
        raise JarqError(JARQ_EINVAL, "jarq_token_logprobs_workspace_bytes")
    if logits.requires_grad or _dual(logits):
        _outside("token_logprobs", "token_logprobs_backward gives the logits' gradient")
    dev = logits.device
    with _on(stream):
        logprob, entropy, lse, rest = torch.empty(4, T, dtype=torch.float32, device=dev).unbind(0)
        index = torch.empty(T, top, dtype=torch.int32, device=dev) if top else None
        value = torch.empty(T, top, dtype=torch.float32, device=dev) if top else None
        if ws is None:
            ws = _work(n, logits)
    _check(lib.jarq_token_logprobs_keep(
        _dtype(logits, "logits"), logits.data_ptr(), ld, T, V,
        _at(targets, torch.int64, "targets", at), top, logprob.data_ptr(), entropy.data_ptr(),
        lse.data_ptr(), rest.data_ptr(), _own(index), _own(value),
        _at(ws, torch.uint8, "workspace", at), ws.numel(), _queue(stream, at)),
        "jarq_token_logprobs_keep")
    result = TokenLogprobs(logprob, entropy, lse, index, value)
    result.lse_rest = rest
    return result


def token_logprobs_backward(logits, targets, forward: TokenLogprobs, d_logprob, d_entropy=None,
                            out=None, stream=None):
    """Gradient of the logits from those of the log probabilities and entropies [tokens]."""
    lib = load_library()
    T, V, ld = _logits(logits, "logits")
    at = _device(logits, "logits")
    rest = forward.lse_rest
    for t, name in ((targets, "targets"), (forward.lse, "lse"), (rest, "lse_rest"),
                    (forward.entropy, "entropy"), (d_logprob, "d_logprob"),
                    (d_entropy, "d_entropy")):
        if t is not None and t.shape != (T,):
            raise ValueError(f"{name} must be [tokens]")
    given = out is not None
    if out is None:
        with _on(stream):
            out = torch.empty(T, V, dtype=logits.dtype, device=logits.device)
        ld_d = V
    else:
        if out.shape != (T, V) or out.dtype != logits.dtype:
            raise ValueError("out must have the logits' shape and type")
        if out.get_device() != at:
            raise ValueError(f"out must be on cuda:{at}, got {out.device}")
        _, _, ld_d = _logits(out, "out")
    head = (_dtype(logits, "logits"), logits.data_ptr(), ld, T, V,
            _at(targets, torch.int64, "targets", at), _at(forward.lse, torch.float32, "lse", at))
    tail = (_at(forward.entropy, torch.float32, "entropy", at),
            _at(d_logprob, torch.float32, "d_logprob", at),
            _at(d_entropy, torch.float32, "d_entropy", at), out.data_ptr(), ld_d,
            _queue(stream, at))
    if rest is None:
        _check(lib.jarq_token_logprobs_backward(*head, *tail), "jarq_token_logprobs_backward")
    else:
        _check(lib.jarq_token_logprobs_keep_backward(
            *head, _at(rest, torch.float32, "lse_rest", at), *tail),
            "jarq_token_logprobs_keep_backward")
    if given:
        _wrote(out)
    return out


# ---- around a block in a training or serving step ----

def _norm_args(X, gain, residual, at):
    """(type, gain's type, addresses) of a norm's inputs, checked."""
    T, cols = _rows(X, "X")
    dt, gt = X.dtype, gain.dtype
    code = _dtype(X, "X")
    if gt != dt and gt != torch.float32:
        raise TypeError(f"gain must be {dt} or float32, got {gt}")
    if gain.shape != (cols,):
        raise ValueError("gain must be [cols]")
    if residual is not None and residual.shape != X.shape:
        raise ValueError("residual must have the shape of X")
    return code, DTYPES[gt], T, cols, _at(X, dt, "X", at), _at(residual, dt, "residual", at), \
        _at(gain, gt, "gain", at)


def _no_norm_graph(call, X, gain, residual, says):
    if (X.requires_grad or gain.requires_grad or (residual is not None and residual.requires_grad)
            or _dual(X, gain, residual)):
        _outside(call, says)


def _sum_out(sum_out, X, residual):
    """Where X + residual goes, None without a residual."""
    if residual is None:
        if sum_out is not None:
            raise ValueError("sum_out needs a residual")
        return None
    if sum_out is None:
        return torch.empty_like(X)
    if sum_out.shape != X.shape:
        raise ValueError("sum_out must have the shape of X")
    return sum_out


def rms_norm(X, gain, residual=None, eps=1e-6, out=None, sum_out=None, stream=None):
    """The root-mean-square norm of X [tokens, cols] times gain [cols] (X's type or float32).

    With a residual the norm is of H = X + residual, rounded to X's type, and (Y, H) is returned;
    out and sum_out may each be X or the residual.  rms_norm_backward gives the gradients; autograd
    records none.
    """
    lib = load_library()
    at = _device(X, "X")
    code, gcode, T, cols, x, res, g = _norm_args(X, gain, residual, at)
    _no_norm_graph("rms_norm", X, gain, residual, "rms_norm_backward gives its gradients")
    given = out is not None or sum_out is not None
    with _on(stream):
        if out is None:
            out = torch.empty_like(X)
        elif out.shape != X.shape:
            raise ValueError("out must have the shape of X")
        H = _sum_out(sum_out, X, residual)
    _check(lib.jarq_rms_norm(code, gcode, T, cols, x, res, g, eps, _at(H, X.dtype, "sum_out", at),
                             _at(out, X.dtype, "out", at), _queue(stream, at)), "jarq_rms_norm")
    if given:
        _wrote(out, H)
    return out if residual is None else (out, H)


def rms_norm_i8(X, gain, residual=None, eps=1e-6, out=None, scale=None, sum_out=None, stream=None):
    """(Q int8, scale fp32 [rows, 1]) of that norm on 8 bits, for matmul_i8.  Has no gradient.

    With a residual (Q, scale, H).
    """
    lib = load_library()
    at = _device(X, "X")
    code, gcode, T, cols, x, res, g = _norm_args(X, gain, residual, at)
    _no_norm_graph("rms_norm_i8", X, gain, residual, "it has no gradient")
    given = out is not None or scale is not None or sum_out is not None
    with _on(stream):
        if out is None:
            out = torch.empty(T, cols, dtype=torch.int8, device=X.device)
        if scale is None:
            scale = torch.empty(T, 1, dtype=torch.float32, device=X.device)
        H = _sum_out(sum_out, X, residual)
    if out.shape != X.shape or scale.numel() != T:
        raise ValueError("out must have the shape of X and scale hold one value a row")
    _check(lib.jarq_rms_norm_i8(code, gcode, T, cols, x, res, g, eps,
                                _at(H, X.dtype, "sum_out", at), _at(out, torch.int8, "out", at),
                                _at(scale, torch.float32, "scale", at), _queue(stream, at)),
           "jarq_rms_norm_i8")
    if given:
        _wrote(out, scale, H)
    return (out, scale) if residual is None else (out, scale, H)


def rms_norm_backward(H, gain, dY, dH=None, eps=1e-6, need=(True, True), ws=None, stream=None):
    """(dX, dgain) of rms_norm, None where not needed, from H (X where there was no residual).

    dX is the gradient of X and of the residual alike; dH is what reaches H on other ways.
    """
    lib = load_library()
    at = _device(H, "H")
    T, cols = _rows(H, "H")
    if dY.shape != H.shape or (dH is not None and dH.shape != H.shape):
        raise ValueError("dY and dH must have the shape of H")
    code, gcode, T, cols, h, _, g = _norm_args(H, gain, None, at)
    n = int(lib.jarq_rms_norm_workspace_bytes(T, cols))
    if n == 0:
        raise JarqError(JARQ_EINVAL, "jarq_rms_norm_workspace_bytes")
    dt = H.dtype
    with _on(stream):
        dX = torch.empty_like(H) if need[0] else None
        dgain = torch.empty_like(gain) if need[1] else None
        if ws is None:
            ws = _work(n, H)
    _check(lib.jarq_rms_norm_backward(code, gcode, T, cols, h, g, _at(dY, dt, "dY", at),
                                      _at(dH, dt, "dH", at), eps, _own(dX), _own(dgain),
                                      _at(ws, torch.uint8, "workspace", at), ws.numel(),
                                      _queue(stream, at)), "jarq_rms_norm_backward")
    return dX, dgain


class LinearLogprobs(NamedTuple):
    """What linear_logprobs returns: all [tokens] fp32."""

    logprob: torch.Tensor
    lse: torch.Tensor         # log sum exp of the logits
    lse_rest: torch.Tensor    # what rounding left of it


def linear_logprobs(X, W, targets, ws=None, stream=None) -> LinearLogprobs:
    """Log probabilities of targets [tokens] int64 (< 0: none) under the logits X W^T.

    X [tokens, d] and W [vocab, d] in 16 bits; the logits are not formed in memory.
    linear_logprobs_backward gives the gradients; autograd records none.
    """
    lib = load_library()
    T, d = _rows(X, "X")
    V, _ = _rows(W, "W", d)
    at = _device(X, "X")
    if targets.shape != (T,):
        raise ValueError("targets must be [tokens]")
    n = int(lib.jarq_linear_logprobs_workspace_bytes(T, d, V))
    if n == 0:
        raise JarqError(JARQ_EINVAL, "jarq_linear_logprobs_workspace_bytes")
    if X.requires_grad or W.requires_grad or _dual(X, W):
        _outside("linear_logprobs", "linear_logprobs_backward gives its gradients")
    dt = X.dtype
    with _on(stream):
        r = LinearLogprobs(*torch.empty(3, T, dtype=torch.float32, device=X.device).unbind(0))
        if ws is None:
            ws = _work(n, X)
    _check(lib.jarq_linear_logprobs(_dtype(X, "X"), T, d, V, _at(X, dt, "X", at),
                                    _at(W, dt, "W", at), _at(targets, torch.int64, "targets", at),
                                    r.logprob.data_ptr(), r.lse.data_ptr(), r.lse_rest.data_ptr(),
                                    _at(ws, torch.uint8, "workspace", at), ws.numel(),
                                    _queue(stream, at)), "jarq_linear_logprobs")
    return r


def linear_logprobs_backward(X, W, targets, forward: LinearLogprobs, d_logprob, d_lse=None,
                             need=(True, True), ws=None, stream=None):
    """(dX, dW) from the gradients of the log probabilities and of lse [tokens].

    None where not needed.
    """
    lib = load_library()
    T, d = _rows(X, "X")
    V, _ = _rows(W, "W", d)
    at = _device(X, "X")
    for t, name in ((targets, "targets"), (forward.logprob, "logprob"), (forward.lse, "lse"),
                    (forward.lse_rest, "lse_rest"), (d_logprob, "d_logprob"), (d_lse, "d_lse")):
        if t is not None and t.shape != (T,):
            raise ValueError(f"{name} must be [tokens]")
    n = int(lib.jarq_linear_logprobs_backward_workspace_bytes(T, d, V))
    if n == 0:
        raise JarqError(JARQ_EINVAL, "jarq_linear_logprobs_backward_workspace_bytes")
    dt, f32 = X.dtype, torch.float32
    with _on(stream):
        dX, dW = (torch.empty_like(t) if wanted else None for t, wanted in zip((X, W), need))
        if ws is None:
            ws = _work(n, X)
    _check(lib.jarq_linear_logprobs_backward(
        _dtype(X, "X"), T, d, V, _at(X, dt, "X", at), _at(W, dt, "W", at),
        _at(targets, torch.int64, "targets", at), _at(forward.logprob, f32, "logprob", at),
        _at(forward.lse, f32, "lse", at), _at(forward.lse_rest, f32, "lse_rest", at),
        _at(d_logprob, f32, "d_logprob", at), _at(d_lse, f32, "d_lse", at), _own(dX), _own(dW),
        _at(ws, torch.uint8, "workspace", at), ws.numel(), _queue(stream, at)),
        "jarq_linear_logprobs_backward")
    return dX, dW


class AdamWState(NamedTuple):
    """The state of adamw_step for a list of tensors, flat: see adamw_state.

    A tensor's values begin at the sum of the lengths before it, each rounded up to a multiple of
    128.  On 8 bits m and sqrt(v) are held as value * 2^(exp - 134), an exponent a 128.
    """

    master: Optional[torch.Tensor]   # [n] fp32: the parameters of 16 bits; None for fp32 ones
    m: torch.Tensor                  # [n] fp32, or float8_e4m3fn
    v: torch.Tensor                  # [n] fp32: v; or float8_e4m3fn: sqrt(v)
    m_exp: Optional[torch.Tensor]    # [n / 128] uint8 on 8 bits
    v_exp: Optional[torch.Tensor]


def _state_length(numels):
    n = int(load_library().jarq_adamw_state_length(len(numels), (_i64 * len(numels))(*numels)))
    if n < 0:
        raise JarqError(JARQ_EINVAL, "jarq_adamw_state_length")
    return n


def adamw_state(params, bits=32) -> AdamWState:
    """A new state (no moments) for parameters of one type on one device.

    Parameters of 16 bits get a copy in 32, which the steps advance.
    """
    params = list(params)
    if bits not in (8, 32):
        raise ValueError(f"bits must be 8 or 32, got {bits!r}")
    if not params:
        raise ValueError("params must hold a tensor")
    dt = params[0].dtype
    _dtype(params[0], "params[0]")
    at = _device(params[0], "params[0]")
    for k, t in enumerate(params):
        _at(t, dt, f"params[{k}]", at)
    n = _state_length([t.numel() for t in params])
    dev = params[0].device
    master = None
    if dt != torch.float32:
        master = torch.zeros(n, dtype=torch.float32, device=dev)
        first = 0
        for t in params:
            master[first:first + t.numel()] = t.detach().view(-1)
            first += (t.numel() + 127) // 128 * 128
    if bits == 32:
        return AdamWState(master, *(torch.zeros(n, dtype=torch.float32, device=dev)
                                    for _ in range(2)), None, None)
    m, v = (torch.zeros(n, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)
            for _ in range(2))
    return AdamWState(master, m, v, *(torch.zeros(n // 128, dtype=torch.uint8, device=dev)
                                      for _ in range(2)))


def adamw_moments(state: AdamWState):
    """(m, v) of a state as flat fp32 tensors."""
    if state.m_exp is None:
        return state.m, state.v
    m, root = (torch.where(e == 255, torch.nan, torch.ldexp(x.float().view(-1, 128),
                                                            e.int() - 134)).view(-1)
               for x, e in ((state.m, state.m_exp[:, None]), (state.v, state.v_exp[:, None])))
    return m, root * root


_numel, _address, _place, _dense = (torch.Tensor.numel, torch.Tensor.data_ptr,
                                    torch.Tensor.get_device, torch.Tensor.is_contiguous)


def _addresses(tensors, dtype, name, device, numels):
    """The addresses of dense tensors of one type on the call's device, 0 where one is None.

    (Checked all together: 0.2 us a tensor, 0.6 one after the other.)
    """
    try:
        if (list(map(_numel, tensors)) == numels and {t.dtype for t in tensors} == {dtype}
                and set(map(_place, tensors)) == {device} and all(map(_dense, tensors))):
            return list(map(_address, tensors))
    except TypeError:   # one is None, or no tensor
        pass
    found = []
    for k, (t, n) in enumerate(zip(tensors, numels)):
        found.append(_at(t, dtype, f"{name}[{k}]", device) or 0)
        if t is not None and t.numel() != n:
            raise ValueError(f"{name}[{k}] must have {n} values, got {t.numel()}")
    return found


_E4M3, _U8, _F32 = torch.float8_e4m3fn, torch.uint8, torch.float32
_STATE_TYPES = {(32, True): (None, _F32, _F32, None, None), (32, False): (_F32, _F32, _F32, None, None),
                (8, True): (None, _E4M3, _E4M3, _U8, _U8), (8, False): (_F32, _E4M3, _E4M3, _U8, _U8)}


def _state_arrays(s: AdamWState, bits, wide, n, name, device):
    """The addresses of a state's arrays; wide: fp32 parameters, which have no master."""
    found = []
    for part, t, dt, length in zip(AdamWState._fields, s, _STATE_TYPES[bits, wide],
                                   (n, n, n, n // 128, n // 128)):
        if dt is None or t is None:
            if t is not dt:
                raise ValueError(f"{name}.{part} must be {'None' if dt is None else 'a tensor'}")
            found.append(None)
        elif (t.dtype == dt and t.numel() == length and t.get_device() == device
              and t.is_contiguous()):
            found.append(t.data_ptr())
        else:
            if t.numel() != length:
                raise ValueError(f"{name}.{part} must be [{length}]")
            found.append(_at(t, dt, f"{name}.{part}", device))
    return _AdamWArrays(*found)


def _one_value(t, dtype, name, device):
    if t is not None and t.numel() != 1:
        raise ValueError(f"{name} must hold one value")
    return _at(t, dtype, name, device)


def adamw_step(params, grads, state: AdamWState, step, lr, beta1=0.9, beta2=0.999, eps=1e-8,
               weight_decay=0.01, grad_mul=None, seed=0, out=None, stream=None):
    """A step of AdamW on params with the gradients grads, both lists of tensors of one type.

    Updates params and state in place and returns them; with out, a pair (params, state) of other
    tensors, those get the result and the old ones stay.  step counts from 1.  step and lr are
    numbers, or device tensors of one value (int64, float32) that are read when the step runs, as
    in a captured graph; grad_mul, a float32 one, multiplies the gradients (an infinite or NaN
    one: the step changes nothing).  A gradient may be None (its tensor stays; not with out).  On
    8 bits the rounding's noise comes from seed and step.
    """
    lib = load_library()
    params, grads = list(params), list(grads)
    if len(grads) != len(params) or not params:
        raise ValueError("params and grads must hold as many tensors, one at least")
    if not all([isinstance(t, torch.Tensor) for t in params]):
        raise TypeError("params must be tensors")
    dt = params[0].dtype
    code = _dtype(params[0], "params[0]")
    at = _device(params[0], "params[0]")
    bits = 32 if state.m_exp is None else 8
    numels = list(map(_numel, params))
    n = sum([k + 127 & -128 for k in numels])
    old = _addresses(params, dt, "params", at, numels)
    new_params, new_state = (params, state) if out is None else (list(out[0]), out[1])
    if out is not None and (len(new_params) != len(params)
                            or not all([isinstance(t, torch.Tensor) for t in new_params])):
        raise ValueError("out must hold as many parameters")
    new = old if out is None else _addresses(new_params, dt, "out", at, numels)
    table = (_i64 * (4 * len(params)))()
    table[0::4] = _addresses(grads, dt, "grads", at, numels)
    table[1::4], table[2::4], table[3::4] = old, new, numels
    held = _state_arrays(state, bits, dt == torch.float32, n, "state", at)
    to = held if out is None else _state_arrays(new_state, bits, dt == torch.float32, n, "out", at)
    step_at = lr_at = None
    if isinstance(step, torch.Tensor):
        step, step_at = 1, _one_value(step, torch.int64, "step", at)
    if isinstance(lr, torch.Tensor):
        lr, lr_at = 0.0, _one_value(lr, torch.float32, "lr", at)
    options = _AdamWOptions(lr, beta1, beta2, eps, weight_decay, step, seed & (2 ** 64 - 1), lr_at,
                            step_at, _one_value(grad_mul, torch.float32, "grad_mul", at))
    _check(lib.jarq_adamw_step(code, bits, len(params), ctypes.addressof(table), held, to, options,
                               _queue(stream, at)), "jarq_adamw_step")
    _written(new_params + [t for t in new_state if t is not None])
    return new_params, new_state


def lds_probe(workgroups, passes, out=None, stream=None):
    """Run the LDS calibration kernel; returns (LDS bytes moved, out)."""
    lib = load_library()
    if out is None:
        out = torch.empty(workgroups * 256, dtype=torch.float32, device="cuda")
    n = int(lib.jarq_lds_probe(int(workgroups), int(passes), _ptr(out, torch.float32, "out"),
                               _stream(stream)))
    if n < 0:
        raise JarqError(JARQ_EINVAL, "jarq_lds_probe")
    return n, out


def abi_version() -> int:
    return int(load_library().jarq_abi_version())
