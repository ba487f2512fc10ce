"""Thin ctypes binding of libsidco.so: argument marshalling only.

Function names and argument order follow include/sidco.h.  Tensors are torch tensors on the GPU
(torch is used for device memory and streams, nothing else); every step of the sparsifier runs in
the library's HIP kernels.  There is no fallback: a missing library raises.
"""
from __future__ import annotations

import ctypes as C
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsidco.so")

MAX_STAGES = 8
DIST_EXP, DIST_GAMMA_GPD, DIST_GPD = 0, 1, 2
ST_NONFINITE, ST_VAR_ZERO, ST_GAMMA_S, ST_GAMMA_CLAMP, ST_STOPPED, ST_OVERFLOW, ST_FALLBACK = 1, 2, 4, 8, 16, 32, 64

EXPORTS = [
    "sidco_compress", "sidco_compress_static", "sidco_static_max_elements", "sidco_static_init", "sidco_compress_typed", "sidco_workspace_bytes_typed",
    "sidco_compress_batched_typed", "sidco_workspace_bytes_batched_typed", "sidco_controller_compress_typed", "sidco_topk_typed",
    "sidco_dgc_typed", "sidco_compress_ex", "sidco_compress_batched", "sidco_batched_out_offsets",
    "sidco_workspace_bytes_batched", "sidco_read_diag_batched", "sidco_topk", "sidco_dgc", "sidco_dgc_sizes", "sidco_dgc_result", "sidco_adapt_stages", "sidco_controller_create",
    "sidco_controller_destroy", "sidco_controller_stages", "sidco_controller_iteration",
    "sidco_controller_last_average", "sidco_controller_compress", "sidco_scatter_add", "sidco_scatter_check",
    "sidco_fit", "sidco_fit_typed", "sidco_fit_result", "sidco_stage_ratios", "sidco_out_capacity",
    "sidco_workspace_bytes", "sidco_set_workspace", "sidco_reserve", "sidco_release", "sidco_set_status_word",
    "sidco_set_delta1", "sidco_get_diag", "sidco_controller_disturbed",
    "sidco_set_speculation", "sidco_read_diag", "sidco_set_profiling",
    "sidco_get_profile", "sidco_strerror", "sidco_last_hip_error", "sidco_version", "sidco_shutdown",
    "sidco_mx4_code_bytes", "sidco_mx4_scale_bytes", "sidco_mx4_compress", "sidco_mx4_aggregate", "sidco_mx4_quantize",
    "sidco_mx4_dequantize", "sidco_mx4_matmul", "sidco_mx4_linear", "sidco_workspace_bytes_mx4_linear",
    "sidco_newton_schulz_default", "sidco_workspace_bytes_orthogonalize", "sidco_orthogonalize", "sidco_muon_step",
    "sidco_embedding", "sidco_embedding_grad", "sidco_workspace_bytes_embedding_grad", "sidco_dropout", "sidco_dropout_blocks",
    "sidco_cross_entropy", "sidco_workspace_bytes_cross_entropy", "sidco_cross_entropy_grad", "sidco_workspace_bytes_cross_entropy_grad",
    "sidco_cross_entropy_grad_of_loss",
]


class Diag(C.Structure):
    """Mirror of struct sidco_diag."""
    _fields_ = [
        ("eta", C.c_float * MAX_STAGES),
        ("n", C.c_int64 * MAX_STAGES),
        ("stats", (C.c_double * 3) * MAX_STAGES),
        ("selected", C.c_int64),
        ("count", C.c_int32),
        ("stages", C.c_int32),
        ("status", C.c_uint32),
        ("reserved", C.c_uint32),
    ]


class NewtonSchulz(C.Structure):
    """Mirror of struct sidco_newton_schulz."""
    _fields_ = [
        ("steps", C.c_int),
        ("a", C.c_float),
        ("b", C.c_float),
        ("c", C.c_float),
        ("eps", C.c_float),
        ("precision", C.c_int),
    ]


class SidcoError(RuntimeError):
    def __init__(self, code: int, where: str):
        lib = load()
        msg = lib.sidco_strerror(code).decode()
        detail = lib.sidco_last_hip_error().decode()
        if code == -7 or (code == -2 and detail.startswith("sidco_compress_static")):
            msg += " (" + detail + ")"
        super().__init__(f"{where}: error {code}: {msg}")
        self.code = code


_lib = None


def load() -> C.CDLL:
    """Loads libsidco.so; raises if it has not been built (python -m paper_2101_10761_amd.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2101_10761_amd.build` "
            "(there is no CPU or PyTorch fallback for the sparsifier)")
    # One HIP runtime per process: libsidco.so needs libamdhip64.so.7, and so does torch, which ships
    # its own copy.  Loading torch's first makes the dynamic linker resolve ours to the same object;
    # two runtimes in one process cannot both open the device.
    import torch
    bundled = os.path.join(os.path.dirname(torch.__file__), "lib", "libamdhip64.so")
    if os.path.exists(bundled):
        C.CDLL(bundled, mode=C.RTLD_GLOBAL)
    lib = C.CDLL(LIB_PATH)
    vp, f32p, i32p, f64p = C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(C.c_double)
    lib.sidco_compress.argtypes = [vp, f32p, f32p, C.c_int64, C.c_double, C.c_int, C.c_int, i32p, f32p, i32p, f32p]
    lib.sidco_compress.restype = C.c_int
    lib.sidco_compress_static.argtypes = [vp, f32p, f32p, C.c_int64, C.c_double, C.c_int, C.c_int, i32p, f32p, i32p, f32p]
    lib.sidco_compress_static.restype = C.c_int
    lib.sidco_static_init.argtypes = []
    lib.sidco_static_init.restype = C.c_int
    lib.sidco_static_max_elements.argtypes = []
    lib.sidco_static_max_elements.restype = C.c_int64
    lib.sidco_compress_ex.argtypes = [vp, f32p, f32p, C.c_int64, C.c_int, f64p, C.c_int, i32p, f32p, C.c_int64,
                                      i32p, f32p]
    lib.sidco_compress_ex.restype = C.c_int
    lib.sidco_compress_typed.argtypes = [vp, vp, C.c_int, f32p, C.c_int64, C.c_double, C.c_int, C.c_int, i32p, f32p,
                                         i32p, f32p]
    lib.sidco_compress_typed.restype = C.c_int
    lib.sidco_workspace_bytes_typed.argtypes = [C.c_int64, C.c_int, C.c_int]
    lib.sidco_workspace_bytes_typed.restype = C.c_size_t
    lib.sidco_topk.argtypes = [vp, f32p, f32p, C.c_int64, C.c_int64, i32p, f32p, i32p, f32p]
    lib.sidco_topk.restype = C.c_int
    lib.sidco_topk_typed.argtypes = [vp, vp, C.c_int, f32p, C.c_int64, C.c_int64, i32p, f32p, i32p, f32p]
    lib.sidco_topk_typed.restype = C.c_int
    i64p = C.POINTER(C.c_int64)
    lib.sidco_dgc.argtypes = [vp, f32p, f32p, C.c_int64, C.c_double, C.c_double, C.c_uint64, i32p, f32p, i32p, f32p]
    lib.sidco_dgc.restype = C.c_int
    lib.sidco_dgc_typed.argtypes = [vp, vp, C.c_int, f32p, C.c_int64, C.c_double, C.c_double, C.c_uint64, i32p, f32p, i32p,
                                    f32p]
    lib.sidco_dgc_typed.restype = C.c_int
    lib.sidco_compress_batched_typed.argtypes = [vp, vp, C.c_int, f32p, i64p, C.c_int, C.c_double, C.c_int, C.c_int, i32p,
                                                 f32p, i64p, i32p, f32p]
    lib.sidco_compress_batched_typed.restype = C.c_int
    lib.sidco_workspace_bytes_batched_typed.argtypes = [i64p, C.c_int, C.c_int, C.c_int]
    lib.sidco_workspace_bytes_batched_typed.restype = C.c_size_t
    lib.sidco_controller_compress_typed.argtypes = [C.c_void_p, vp, vp, C.c_int, f32p, C.c_int64, i32p, f32p, i32p, f32p]
    lib.sidco_controller_compress_typed.restype = C.c_int
    lib.sidco_dgc_sizes.argtypes = [C.c_int64, C.c_double, C.c_double, i64p]
    lib.sidco_dgc_sizes.restype = C.c_int
    lib.sidco_dgc_result.argtypes = [vp, i64p]
    lib.sidco_dgc_result.restype = C.c_int
    lib.sidco_compress_batched.argtypes = [vp, f32p, f32p, i64p, C.c_int, C.c_double, C.c_int, C.c_int, i32p, f32p,
                                           i64p, i32p, f32p]
    lib.sidco_compress_batched.restype = C.c_int
    lib.sidco_batched_out_offsets.argtypes = [i64p, C.c_int, C.c_double, i64p]
    lib.sidco_batched_out_offsets.restype = C.c_int
    lib.sidco_workspace_bytes_batched.argtypes = [i64p, C.c_int]
    lib.sidco_workspace_bytes_batched.restype = C.c_size_t
    lib.sidco_read_diag_batched.argtypes = [vp, C.c_int, C.POINTER(Diag)]
    lib.sidco_read_diag_batched.restype = C.c_int
    lib.sidco_adapt_stages.argtypes = [C.c_int, C.c_double, C.c_double, C.c_double, C.c_double, C.c_int]
    lib.sidco_adapt_stages.restype = C.c_int
    lib.sidco_controller_create.argtypes = [C.POINTER(C.c_void_p), C.c_double, C.c_int, C.c_int, C.c_int, C.c_int,
                                            C.c_double, C.c_double, C.c_double]
    lib.sidco_controller_create.restype = C.c_int
    lib.sidco_controller_destroy.argtypes = [C.c_void_p]
    lib.sidco_controller_destroy.restype = None
    lib.sidco_controller_stages.argtypes = [C.c_void_p]
    lib.sidco_controller_stages.restype = C.c_int
    lib.sidco_controller_iteration.argtypes = [C.c_void_p]
    lib.sidco_controller_iteration.restype = C.c_int64
    lib.sidco_controller_last_average.argtypes = [C.c_void_p]
    lib.sidco_controller_last_average.restype = C.c_double
    lib.sidco_controller_compress.argtypes = [C.c_void_p, vp, f32p, f32p, C.c_int64, i32p, f32p, i32p, f32p]
    lib.sidco_controller_compress.restype = C.c_int
    lib.sidco_scatter_add.argtypes = [vp, f32p, C.c_int64, i32p, f32p, i32p, C.c_int64, C.c_float]
    lib.sidco_scatter_add.restype = C.c_int
    lib.sidco_scatter_check.argtypes = [vp]
    lib.sidco_scatter_check.restype = C.c_int
    lib.sidco_fit.argtypes = [vp, f32p, f32p, C.c_int64, C.c_int]
    lib.sidco_fit.restype = C.c_int
    lib.sidco_fit_typed.argtypes = [vp, vp, C.c_int, f32p, C.c_int64, C.c_int]
    lib.sidco_fit_typed.restype = C.c_int
    lib.sidco_fit_result.argtypes = [vp, f64p]
    lib.sidco_fit_result.restype = C.c_int
    lib.sidco_stage_ratios.argtypes = [C.c_double, C.c_int, C.c_double, f64p]
    lib.sidco_stage_ratios.restype = C.c_int
    lib.sidco_out_capacity.argtypes = [C.c_int64, C.c_double]
    lib.sidco_out_capacity.restype = C.c_int64
    lib.sidco_workspace_bytes.argtypes = [C.c_int64]
    lib.sidco_workspace_bytes.restype = C.c_size_t
    lib.sidco_set_workspace.argtypes = [vp, C.c_size_t]
    lib.sidco_set_workspace.restype = C.c_int
    lib.sidco_reserve.argtypes = [vp, C.c_size_t]
    lib.sidco_reserve.restype = C.c_int
    lib.sidco_release.argtypes = [vp]
    lib.sidco_release.restype = C.c_int
    lib.sidco_set_status_word.argtypes = [vp, vp]
    lib.sidco_set_status_word.restype = C.c_int
    lib.sidco_set_delta1.argtypes = [C.c_double]
    lib.sidco_set_delta1.restype = C.c_int
    lib.sidco_get_diag.argtypes = [vp, C.POINTER(Diag)]
    lib.sidco_get_diag.restype = C.c_int
    lib.sidco_controller_disturbed.argtypes = [C.c_void_p]
    lib.sidco_controller_disturbed.restype = C.c_int64
    lib.sidco_set_speculation.argtypes = [C.c_double]
    lib.sidco_set_speculation.restype = C.c_int
    lib.sidco_read_diag.argtypes = [vp, C.POINTER(Diag)]
    lib.sidco_read_diag.restype = C.c_int
    lib.sidco_set_profiling.argtypes = [C.c_int]
    lib.sidco_set_profiling.restype = C.c_int
    lib.sidco_get_profile.argtypes = [C.POINTER(C.c_float), C.POINTER(C.c_char_p), C.c_int]
    lib.sidco_get_profile.restype = C.c_int
    i64, u8p = C.c_int64, C.c_void_p
    lib.sidco_mx4_code_bytes.argtypes = [i64, i64]
    lib.sidco_mx4_code_bytes.restype = i64
    lib.sidco_mx4_scale_bytes.argtypes = [i64, i64]
    lib.sidco_mx4_scale_bytes.restype = i64
    lib.sidco_mx4_compress.argtypes = [vp, vp, C.c_int, f32p, i64, u8p, u8p]
    lib.sidco_mx4_compress.restype = C.c_int
    lib.sidco_mx4_aggregate.argtypes = [vp, u8p, i64, u8p, i64, C.c_int, i64, C.c_float, C.c_int, f32p]
    lib.sidco_mx4_aggregate.restype = C.c_int
    lib.sidco_mx4_quantize.argtypes = [vp, vp, C.c_int, i64, i64, i64, u8p, u8p, u8p, u8p]
    lib.sidco_mx4_quantize.restype = C.c_int
    lib.sidco_mx4_dequantize.argtypes = [vp, u8p, u8p, i64, i64, vp, C.c_int, i64]
    lib.sidco_mx4_dequantize.restype = C.c_int
    lib.sidco_mx4_matmul.argtypes = [vp, u8p, u8p, u8p, u8p, i64, i64, i64, C.c_float, C.c_int, vp, C.c_int, i64]
    lib.sidco_mx4_matmul.restype = C.c_int
    lib.sidco_mx4_linear.argtypes = [vp, vp, C.c_int, i64, i64, i64, u8p, u8p, i64, C.c_float, C.c_int, vp, C.c_int, i64]
    lib.sidco_mx4_linear.restype = C.c_int
    lib.sidco_workspace_bytes_mx4_linear.argtypes = [i64, i64]
    lib.sidco_workspace_bytes_mx4_linear.restype = C.c_size_t
    nsp = C.POINTER(NewtonSchulz)
    lib.sidco_newton_schulz_default.argtypes = [nsp]
    lib.sidco_newton_schulz_default.restype = None
    lib.sidco_workspace_bytes_orthogonalize.argtypes = [C.c_int, i64, i64, C.c_int, nsp]
    lib.sidco_workspace_bytes_orthogonalize.restype = C.c_size_t
    lib.sidco_orthogonalize.argtypes = [vp, vp, C.c_int, i64, i64, C.c_int, i64, i64, nsp, vp, C.c_int, i64, i64]
    lib.sidco_orthogonalize.restype = C.c_int
    lib.sidco_muon_step.argtypes = [vp, vp, C.c_int, f32p, vp, C.c_int, C.c_int, i64, i64, C.c_float, C.c_float, C.c_int, C.c_float,
                                    C.c_float, nsp]
    lib.sidco_muon_step.restype = C.c_int
    lib.sidco_embedding.argtypes = [vp, vp, C.c_int, i64, i64, i64, vp, C.c_int, i64, C.c_float, vp, C.c_int, i64]
    lib.sidco_embedding.restype = C.c_int
    lib.sidco_embedding_grad.argtypes = [vp, vp, C.c_int, i64, i64, i64, vp, C.c_int, i64, C.c_float, C.c_int, vp, C.c_int, i64]
    lib.sidco_embedding_grad.restype = C.c_int
    lib.sidco_workspace_bytes_embedding_grad.argtypes = [i64, i64]
    lib.sidco_workspace_bytes_embedding_grad.restype = C.c_size_t
    lib.sidco_dropout.argtypes = [vp, vp, C.c_int, i64, i64, i64, C.c_double, C.c_uint64, C.c_uint64, vp, vp, i64, vp, C.c_int, i64]
    lib.sidco_dropout.restype = C.c_int
    lib.sidco_dropout_blocks.argtypes = [i64, i64]
    lib.sidco_dropout_blocks.restype = i64
    lib.sidco_cross_entropy.argtypes = [vp, vp, vp, C.c_int, i64, i64, i64, i64, i64, vp, C.c_int, f32p, f32p]
    lib.sidco_cross_entropy.restype = C.c_int
    lib.sidco_workspace_bytes_cross_entropy.argtypes = [i64, i64, i64, C.c_int]
    lib.sidco_workspace_bytes_cross_entropy.restype = C.c_size_t
    lib.sidco_cross_entropy_grad.argtypes = [vp, vp, vp, C.c_int, i64, i64, i64, i64, i64, vp, C.c_int, f32p, f32p, vp, i64, vp, C.c_int, i64,
                                             C.c_int]
    lib.sidco_cross_entropy_grad.restype = C.c_int
    lib.sidco_cross_entropy_grad_of_loss.argtypes = [vp, vp, vp, C.c_int, i64, i64, i64, i64, i64, vp, C.c_int, f32p, f32p, f32p, vp, i64, vp,
                                                     C.c_int, i64, C.c_int]
    lib.sidco_cross_entropy_grad_of_loss.restype = C.c_int
    lib.sidco_workspace_bytes_cross_entropy_grad.argtypes = [i64, i64, i64, C.c_int, C.c_int]
    lib.sidco_workspace_bytes_cross_entropy_grad.restype = C.c_size_t
    lib.sidco_strerror.argtypes = [C.c_int]
    lib.sidco_strerror.restype = C.c_char_p
    lib.sidco_last_hip_error.argtypes = []
    lib.sidco_last_hip_error.restype = C.c_char_p
    lib.sidco_version.argtypes = []
    lib.sidco_version.restype = C.c_int
    lib.sidco_shutdown.argtypes = []
    lib.sidco_shutdown.restype = None
    _lib = lib
    return lib


def _check(rc: int, where: str) -> None:
    if rc != 0:
        raise SidcoError(rc, where)


_torch = None


def _import_torch():
    """torch, imported with the first call that needs it and kept: an import statement in every function and check of a
    call costs as much as the check."""
    global _torch
    import torch
    _torch = torch
    return torch


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream_handle(stream):
    torch = _torch or _import_torch()
    if stream is None:
        # the current device's current stream; building torch's Stream object around it takes 2.9 us against 0.3.
        # Builds of torch that lack either of these two internal functions go that way.
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        device = getattr(torch._C, "_cuda_getDevice", None)
        if raw and device and torch.cuda.is_initialized():
            return raw(device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _check_tensor(t, dtype, name, n=None):
    torch = _torch or _import_torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous CUDA tensor of dtype {dtype}")
    if n is not None and t.numel() < n:
        raise ValueError(f"{name} has {t.numel()} elements, needs {n}")


def sidco_stage_ratios(delta: float, stages: int, delta1: float = 0.25) -> list[float]:
    out = (C.c_double * MAX_STAGES)()
    m = load().sidco_stage_ratios(delta, stages, delta1, out)
    if m < 1:
        raise SidcoError(m, "sidco_stage_ratios")
    return [out[i] for i in range(m)]


def sidco_out_capacity(d: int, delta: float) -> int:
    cap = load().sidco_out_capacity(d, delta)
    if cap < 0:
        raise SidcoError(int(cap), "sidco_out_capacity")
    return int(cap)


def sidco_workspace_bytes(d: int) -> int:
    return int(load().sidco_workspace_bytes(d))


def sidco_workspace_bytes_typed(d: int, grad_dtype: int, has_residual: bool) -> int:
    return int(load().sidco_workspace_bytes_typed(d, grad_dtype, 1 if has_residual else 0))


def sidco_set_workspace(buf) -> None:
    """buf: a CUDA uint8 tensor the caller keeps alive, or None to return to library allocation."""
    if buf is None:
        _check(load().sidco_set_workspace(None, 0), "sidco_set_workspace")
    else:
        _check(load().sidco_set_workspace(C.c_void_p(buf.data_ptr()), buf.numel() * buf.element_size()),
               "sidco_set_workspace")


def sidco_reserve(nbytes: int, stream=None) -> None:
    """Grows the library's own workspace of `stream` to at least nbytes (see sidco_workspace_bytes)."""
    _check(load().sidco_reserve(_stream_handle(stream), int(nbytes)), "sidco_reserve")


def sidco_release(stream=None) -> None:
    _check(load().sidco_release(_stream_handle(stream)), "sidco_release")


def sidco_set_status_word(word, stream=None) -> None:
    """word: a CUDA uint32/int32 tensor of one element that receives the status bits of every call on
    `stream`, or None to switch that off."""
    _check(load().sidco_set_status_word(_stream_handle(stream), _ptr(word)), "sidco_set_status_word")


def sidco_set_delta1(delta1: float) -> None:
    _check(load().sidco_set_delta1(float(delta1)), "sidco_set_delta1")


def sidco_compress(grad, residual, delta: float, dist: int, stages: int, out_idx, out_val, out_count, out_eta,
                   stream=None) -> None:
    """Enqueues one sparsifier call; see include/sidco.h.  `residual` may be None."""
    torch = _torch or _import_torch()
    d = grad.numel()
    _check_tensor(grad, torch.float32, "grad")
    if residual is not None:
        _check_tensor(residual, torch.float32, "residual", d)
    cap = sidco_out_capacity(d, delta)
    _check_tensor(out_idx, torch.int32, "out_idx", cap)
    _check_tensor(out_val, torch.float32, "out_val", cap)
    _check_tensor(out_count, torch.int32, "out_count", 1)
    _check_tensor(out_eta, torch.float32, "out_eta", 1)
    _check(load().sidco_compress(_stream_handle(stream), _ptr(grad), _ptr(residual), d, delta, dist, stages,
                                 _ptr(out_idx), _ptr(out_val), _ptr(out_count), _ptr(out_eta)), "sidco_compress")


def sidco_compress_static(grad, residual, delta: float, dist: int, stages: int, out_idx, out_val, out_count, out_eta,
                          stream=None) -> None:
    """sidco_compress in the library's static scratch: no device allocation; d <= sidco_static_max_elements()."""
    torch = _torch or _import_torch()
    d = grad.numel()
    _check_tensor(grad, torch.float32, "grad")
    if residual is not None:
        _check_tensor(residual, torch.float32, "residual", d)
    cap = sidco_out_capacity(d, delta)
    _check_tensor(out_idx, torch.int32, "out_idx", cap)
    _check_tensor(out_val, torch.float32, "out_val", cap)
    _check_tensor(out_count, torch.int32, "out_count", 1)
    _check_tensor(out_eta, torch.float32, "out_eta", 1)
    _check(load().sidco_compress_static(_stream_handle(stream), _ptr(grad), _ptr(residual), d, delta, dist, stages,
                                        _ptr(out_idx), _ptr(out_val), _ptr(out_count), _ptr(out_eta)),
           "sidco_compress_static")


def sidco_static_init() -> None:
    _check(load().sidco_static_init(), "sidco_static_init")


def sidco_static_max_elements() -> int:
    return int(load().sidco_static_max_elements())


GRAD_F32, GRAD_F16, GRAD_BF16 = 0, 1, 2


def sidco_compress_typed(grad, residual, delta: float, dist: int, stages: int, out_idx, out_val, out_count, out_eta,
                         stream=None) -> None:
    """sidco_compress on a gradient tensor of dtype float32, float16 or bfloat16 (the residual stays float32)."""
    torch = _torch or _import_torch()
    codes = {torch.float32: GRAD_F32, torch.float16: GRAD_F16, torch.bfloat16: GRAD_BF16}
    if not isinstance(grad, torch.Tensor) or grad.dtype not in codes:
        raise TypeError("grad must be a CUDA tensor of dtype float32, float16 or bfloat16")
    d = grad.numel()
    _check_tensor(grad, grad.dtype, "grad")
    if residual is not None:
        _check_tensor(residual, torch.float32, "residual", d)
    cap = sidco_out_capacity(d, delta)
    _check_tensor(out_idx, torch.int32, "out_idx", cap)
    _check_tensor(out_val, torch.float32, "out_val", cap)
    _check_tensor(out_count, torch.int32, "out_count", 1)
    _check_tensor(out_eta, torch.float32, "out_eta", 1)
    _check(load().sidco_compress_typed(_stream_handle(stream), _ptr(grad), codes[grad.dtype], _ptr(residual), d, delta,
                                       dist, stages, _ptr(out_idx), _ptr(out_val), _ptr(out_count), _ptr(out_eta)),
           "sidco_compress_typed")


def sidco_compress_ex(grad, residual, dist: int, ratios, out_idx, out_val, out_count, out_eta, stream=None) -> None:
    """Explicit stage ratios; the output capacity is min(len(out_idx), len(out_val))."""
    torch = _torch or _import_torch()
    d = grad.numel()
    _check_tensor(grad, torch.float32, "grad")
    if residual is not None:
        _check_tensor(residual, torch.float32, "residual", d)
    _check_tensor(out_idx, torch.int32, "out_idx", 1)
    _check_tensor(out_val, torch.float32, "out_val", 1)
    _check_tensor(out_count, torch.int32, "out_count", 1)
    _check_tensor(out_eta, torch.float32, "out_eta", 1)
    cap = min(out_idx.numel(), out_val.numel())
    r = (C.c_double * len(ratios))(*ratios)
    _check(load().sidco_compress_ex(_stream_handle(stream), _ptr(grad), _ptr(residual), d, dist, r, len(ratios),
                                    _ptr(out_idx), _ptr(out_val), cap, _ptr(out_count), _ptr(out_eta)),
           "sidco_compress_ex")


def _i64_array(values):
    try:
        return (C.c_int64 * len(values))(*values)
    except TypeError:  # integers of other types than int
        return (C.c_int64 * len(values))(*[int(v) for v in values])


def sidco_batched_out_offsets(offsets, delta: float) -> list[int]:
    """Default placement of the tensors' outputs: sidco_out_capacity pairs each, back to back."""
    n = len(offsets) - 1
    out = (C.c_int64 * (n + 1))()
    _check(load().sidco_batched_out_offsets(_i64_array(offsets), n, delta, out), "sidco_batched_out_offsets")
    return [out[i] for i in range(n + 1)]


def sidco_workspace_bytes_batched(offsets) -> int:
    return int(load().sidco_workspace_bytes_batched(_i64_array(offsets), len(offsets) - 1))


def sidco_compress_batched(grad, residual, offsets, delta: float, dist: int, stages: int, out_idx, out_val, out_offsets,
                           out_counts, out_etas, stream=None) -> None:
    """Enqueues one sparsifier call per tensor of the flat buffer, all in one launch sequence; see include/sidco.h."""
    torch = _torch or _import_torch()
    n = len(offsets) - 1
    _check_tensor(grad, torch.float32, "grad", offsets[-1])
    if residual is not None:
        _check_tensor(residual, torch.float32, "residual", offsets[-1])
    _check_tensor(out_idx, torch.int32, "out_idx", out_offsets[-1])
    _check_tensor(out_val, torch.float32, "out_val", out_offsets[-1])
    _check_tensor(out_counts, torch.int32, "out_counts", n)
    _check_tensor(out_etas, torch.float32, "out_etas", n)
    _check(load().sidco_compress_batched(_stream_handle(stream), _ptr(grad), _ptr(residual), _i64_array(offsets), n, delta,
                                         dist, stages, _ptr(out_idx), _ptr(out_val), _i64_array(out_offsets),
                                         _ptr(out_counts), _ptr(out_etas)), "sidco_compress_batched")


def sidco_read_diag_batched(t: int, stream=None) -> Diag:
    diag = Diag()
    _check(load().sidco_read_diag_batched(_stream_handle(stream), t, C.byref(diag)), "sidco_read_diag_batched")
    return diag


def sidco_topk(grad, residual, k: int, out_idx, out_val, out_count, out_kth, stream=None) -> None:
    """Enqueues the exact Top-k comparator; see include/sidco.h.  `residual` may be None."""
    torch = _torch or _import_torch()
    d = grad.numel()
    _check_tensor(grad, torch.float32, "grad")
    if residual is not None:
        _check_tensor(residual, torch.float32, "residual", d)
    _check_tensor(out_idx, torch.int32, "out_idx", k)
    _check_tensor(out_val, torch.float32, "out_val", k)
    _check_tensor(out_count, torch.int32, "out_count", 1)
    _check_tensor(out_kth, torch.float32, "out_kth", 1)
    _check(load().sidco_topk(_stream_handle(stream), _ptr(grad), _ptr(residual), d, k, _ptr(out_idx), _ptr(out_val),
                             _ptr(out_count), _ptr(out_kth)), "sidco_topk")


def sidco_dgc_sizes(d: int, delta: float, sample_ratio: float = 0.01):
    """(n_s, k_s, k) of the DGC comparator for a vector of d elements."""
    sizes = (C.c_int64 * 3)()
    _check(load().sidco_dgc_sizes(d, delta, sample_ratio, sizes), "sidco_dgc_sizes")
    return int(sizes[0]), int(sizes[1]), int(sizes[2])


def sidco_dgc(grad, residual, delta: float, sample_ratio: float, seed: int, out_idx, out_val, out_count, out_eta,
              stream=None) -> None:
    """Enqueues the DGC comparator; see include/sidco.h.  `residual` may be None."""
    torch = _torch or _import_torch()
    d = grad.numel()
    _check_tensor(grad, torch.float32, "grad")
    if residual is not None:
        _check_tensor(residual, torch.float32, "residual", d)
    k = sidco_dgc_sizes(d, delta, sample_ratio)[2]
    _check_tensor(out_idx, torch.int32, "out_idx", k)
    _check_tensor(out_val, torch.float32, "out_val", k)
    _check_tensor(out_count, torch.int32, "out_count", 1)
    _check_tensor(out_eta, torch.float32, "out_eta", 1)
    _check(load().sidco_dgc(_stream_handle(stream), _ptr(grad), _ptr(residual), d, delta, sample_ratio, seed,
                            _ptr(out_idx), _ptr(out_val), _ptr(out_count), _ptr(out_eta)), "sidco_dgc")


def _grad_code(grad):
    """SIDCO_GRAD_* of a gradient tensor (float32, float16 or bfloat16)."""
    torch = _torch or _import_torch()
    codes = {torch.float32: GRAD_F32, torch.float16: GRAD_F16, torch.bfloat16: GRAD_BF16}
    if not isinstance(grad, torch.Tensor) or grad.dtype not in codes:
        raise TypeError("grad must be a CUDA tensor of dtype float32, float16 or bfloat16")
    _check_tensor(grad, grad.dtype, "grad")
    return codes[grad.dtype]


def sidco_topk_typed(grad, residual, k: int, out_idx, out_val, out_count, out_kth, stream=None) -> None:
    """sidco_topk on a gradient tensor of dtype float32, float16 or bfloat16 (the residual stays float32)."""
    torch = _torch or _import_torch()
    code = _grad_code(grad)
    d = grad.numel()
    if residual is not None:
        _check_tensor(residual, torch.float32, "residual", d)
    _check_tensor(out_idx, torch.int32, "out_idx", k)
    _check_tensor(out_val, torch.float32, "out_val", k)
    _check_tensor(out_count, torch.int32, "out_count", 1)
    _check_tensor(out_kth, torch.float32, "out_kth", 1)
    _check(load().sidco_topk_typed(_stream_handle(stream), _ptr(grad), code, _ptr(residual), d, k, _ptr(out_idx),
                                   _ptr(out_val), _ptr(out_count), _ptr(out_kth)), "sidco_topk_typed")


def sidco_dgc_typed(grad, residual, delta: float, sample_ratio: float, seed: int, out_idx, out_val, out_count, out_eta,
                    stream=None) -> None:
    """sidco_dgc on a gradient tensor of dtype float32, float16 or bfloat16 (the residual stays float32)."""
    torch = _torch or _import_torch()
    code = _grad_code(grad)
    d = grad.numel()
    if residual is not None:
        _check_tensor(residual, torch.float32, "residual", d)
    k = sidco_dgc_sizes(d, delta, sample_ratio)[2]
    _check_tensor(out_idx, torch.int32, "out_idx", k)
    _check_tensor(out_val, torch.float32, "out_val", k)
    _check_tensor(out_count, torch.int32, "out_count", 1)
    _check_tensor(out_eta, torch.float32, "out_eta", 1)
    _check(load().sidco_dgc_typed(_stream_handle(stream), _ptr(grad), code, _ptr(residual), d, delta, sample_ratio, seed,
                                  _ptr(out_idx), _ptr(out_val), _ptr(out_count), _ptr(out_eta)), "sidco_dgc_typed")


def sidco_compress_batched_typed(grad, residual, offsets, delta: float, dist: int, stages: int, out_idx, out_val,
                                 out_offsets, out_counts, out_etas, stream=None) -> None:
    """sidco_compress_batched on a gradient buffer of dtype float32, float16 or bfloat16."""
    torch = _torch or _import_torch()
    code = _grad_code(grad)
    n = len(offsets) - 1
    if grad.numel() < offsets[-1]:
        raise ValueError(f"grad has {grad.numel()} elements, needs {offsets[-1]}")
    if residual is not None:
        _check_tensor(residual, torch.float32, "residual", offsets[-1])
    _check_tensor(out_idx, torch.int32, "out_idx", out_offsets[-1])
    _check_tensor(out_val, torch.float32, "out_val", out_offsets[-1])
    _check_tensor(out_counts, torch.int32, "out_counts", n)
    _check_tensor(out_etas, torch.float32, "out_etas", n)
    _check(load().sidco_compress_batched_typed(_stream_handle(stream), _ptr(grad), code, _ptr(residual),
                                               _i64_array(offsets), n, delta, dist, stages, _ptr(out_idx), _ptr(out_val),
                                               _i64_array(out_offsets), _ptr(out_counts), _ptr(out_etas)),
           "sidco_compress_batched_typed")


def sidco_workspace_bytes_batched_typed(offsets, grad_dtype: int, has_residual: bool) -> int:
    return int(load().sidco_workspace_bytes_batched_typed(_i64_array(offsets), len(offsets) - 1, grad_dtype,
                                                          1 if has_residual else 0))


def sidco_dgc_result(stream=None):
    """(n_s, k_s, first-pass count, entries written) of the last sidco_dgc; synchronises the stream."""
    out = (C.c_int64 * 4)()
    _check(load().sidco_dgc_result(_stream_handle(stream), out), "sidco_dgc_result")
    return tuple(int(v) for v in out)


def sidco_adapt_stages(stages: int, khat_avg: float, k: float, eps_high: float = 0.2, eps_low: float = 0.2,
                       max_stages: int = MAX_STAGES) -> int:
    m = load().sidco_adapt_stages(stages, khat_avg, k, eps_high, eps_low, max_stages)
    if m < 1:
        raise SidcoError(m, "sidco_adapt_stages")
    return m


class Controller:
    """Handle of a sidco_controller (the sparsifier with its stage controller); see include/sidco.h."""

    def __init__(self, delta: float, dist: int, stages: int = 1, max_stages: int = MAX_STAGES, Q: int = 5,
                 eps_high: float = 0.2, eps_low: float = 0.2, delta1: float = 0.25):
        self._h = C.c_void_p()
        _check(load().sidco_controller_create(C.byref(self._h), delta, dist, stages, max_stages, Q, eps_high, eps_low,
                                              delta1), "sidco_controller_create")
        self.delta = delta

    def close(self):
        if self._h:
            load().sidco_controller_destroy(self._h)
            self._h = C.c_void_p()

    __del__ = close

    @property
    def stages(self) -> int:
        return load().sidco_controller_stages(self._h)

    @property
    def iteration(self) -> int:
        return load().sidco_controller_iteration(self._h)

    @property
    def last_average(self) -> float:
        return load().sidco_controller_last_average(self._h)

    @property
    def disturbed(self) -> int:
        """Windows whose count another caller of the same workspace broke (the stages were left as they were)."""
        return int(load().sidco_controller_disturbed(self._h))

    def compress(self, grad, residual, out_idx, out_val, out_count, out_eta, stream=None) -> None:
        """One iteration; `grad` may be float32 (sidco_controller_compress) or float16 / bfloat16
        (sidco_controller_compress_typed)."""
        torch = _torch or _import_torch()
        d = grad.numel()
        code = _grad_code(grad)
        if residual is not None:
            _check_tensor(residual, torch.float32, "residual", d)
        cap = sidco_out_capacity(d, self.delta)
        _check_tensor(out_idx, torch.int32, "out_idx", cap)
        _check_tensor(out_val, torch.float32, "out_val", cap)
        _check_tensor(out_count, torch.int32, "out_count", 1)
        _check_tensor(out_eta, torch.float32, "out_eta", 1)
        if code == GRAD_F32:
            _check(load().sidco_controller_compress(self._h, _stream_handle(stream), _ptr(grad), _ptr(residual), d,
                                                    _ptr(out_idx), _ptr(out_val), _ptr(out_count), _ptr(out_eta)),
                   "sidco_controller_compress")
        else:
            _check(load().sidco_controller_compress_typed(self._h, _stream_handle(stream), _ptr(grad), code,
                                                          _ptr(residual), d, _ptr(out_idx), _ptr(out_val),
                                                          _ptr(out_count), _ptr(out_eta)),
                   "sidco_controller_compress_typed")


def sidco_scatter_add(dense, idx, val, count, scale: float = 1.0, stream=None) -> None:
    """dense[idx[i]] += scale * val[i] for i < count (a device scalar); see include/sidco.h."""
    torch = _torch or _import_torch()
    _check_tensor(dense, torch.float32, "dense")
    _check_tensor(idx, torch.int32, "idx", 1)
    _check_tensor(val, torch.float32, "val", 1)
    _check_tensor(count, torch.int32, "count", 1)
    cap = min(idx.numel(), val.numel())
    _check(load().sidco_scatter_add(_stream_handle(stream), _ptr(dense), dense.numel(), _ptr(idx), _ptr(val), _ptr(count),
                                    cap, scale), "sidco_scatter_add")


def sidco_scatter_check(stream=None) -> bool:
    rc = load().sidco_scatter_check(_stream_handle(stream))
    if rc < 0:
        raise SidcoError(rc, "sidco_scatter_check")
    return bool(rc)


def sidco_fit(grad, residual, dist: int, stream=None) -> None:
    """Enqueues steps 1-2 alone (error-compensation add fused with the stage-1 sums); the gradient may be
    float32, float16 or bfloat16."""
    torch = _torch or _import_torch()
    codes = {torch.float32: GRAD_F32, torch.float16: GRAD_F16, torch.bfloat16: GRAD_BF16}
    if not isinstance(grad, torch.Tensor) or grad.dtype not in codes:
        raise TypeError("grad must be a CUDA tensor of dtype float32, float16 or bfloat16")
    _check_tensor(grad, grad.dtype, "grad")
    if residual is not None:
        _check_tensor(residual, torch.float32, "residual", grad.numel())
    _check(load().sidco_fit_typed(_stream_handle(stream), _ptr(grad), codes[grad.dtype], _ptr(residual), grad.numel(),
                                  dist), "sidco_fit")


def sidco_fit_result(stream=None) -> tuple[float, float, float, float]:
    """(sum|acc|, sum acc^2, sum log|acc|, d) of the last sidco_fit; synchronises."""
    out = (C.c_double * 4)()
    _check(load().sidco_fit_result(_stream_handle(stream), out), "sidco_fit_result")
    return out[0], out[1], out[2], out[3]


def sidco_set_speculation(theta: float) -> None:
    """Position of a dense stage's candidate threshold (0 = lists of all exceedances); see include/sidco.h."""
    _check(load().sidco_set_speculation(float(theta)), "sidco_set_speculation")


def sidco_read_diag(stream=None) -> Diag:
    diag = Diag()
    _check(load().sidco_read_diag(_stream_handle(stream), C.byref(diag)), "sidco_read_diag")
    return diag


def sidco_get_diag(stream=None) -> Diag:
    """The same call under its other exported name."""
    diag = Diag()
    _check(load().sidco_get_diag(_stream_handle(stream), C.byref(diag)), "sidco_get_diag")
    return diag


def sidco_set_profiling(enable: bool) -> None:
    _check(load().sidco_set_profiling(int(bool(enable))), "sidco_set_profiling")


def sidco_get_profile() -> list[tuple[str, float]]:
    """Per-kernel (name, milliseconds) of the last profiled call on the current device."""
    ms = (C.c_float * 16)()
    names = (C.c_char_p * 16)()
    n = load().sidco_get_profile(ms, names, 16)
    if n < 0:
        raise SidcoError(n, "sidco_get_profile")
    return [(names[i].decode(), float(ms[i])) for i in range(n)]


# ---- 4-bit microscaled numbers ----


def sidco_mx4_code_bytes(rows: int, cols: int) -> int:
    n = load().sidco_mx4_code_bytes(rows, cols)
    if n < 0:
        raise SidcoError(int(n), "sidco_mx4_code_bytes")
    return int(n)


def sidco_mx4_scale_bytes(rows: int, cols: int) -> int:
    n = load().sidco_mx4_scale_bytes(rows, cols)
    if n < 0:
        raise SidcoError(int(n), "sidco_mx4_scale_bytes")
    return int(n)


def sidco_workspace_bytes_mx4_linear(rows: int, k: int) -> int:
    return int(load().sidco_workspace_bytes_mx4_linear(rows, k))


_types = None  # torch's element types as the C ABI numbers them


def _element_types():
    global _types
    torch = _torch or _import_torch()
    _types = {torch.float32: GRAD_F32, torch.float16: GRAD_F16, torch.bfloat16: GRAD_BF16}
    return _types


def _check_packed(codes, scales, rows, cols, name):
    """The addresses of packed buffers that hold rows x cols numbers."""
    torch = _torch or _import_torch()
    lines = rows * ((cols + 255) // 256)
    for t, least in ((codes, 128 * lines), (scales, 8 * lines)):
        if not isinstance(t, torch.Tensor) or t.dtype is not torch.uint8 or not t.is_cuda or not t.is_contiguous():
            raise TypeError(f"{name} codes and scales must be contiguous CUDA tensors of dtype torch.uint8")
        if t.numel() < least:
            raise ValueError(f"{name} codes or scales have {t.numel()} bytes, need {least}")
    return codes.data_ptr(), scales.data_ptr()


def _matrix(x, name, dims=2):
    """Element code and row stride of a CUDA matrix (or batch of them) whose rows are contiguous."""
    torch = _torch or _import_torch()
    code = (_types or _element_types()).get(x.dtype) if isinstance(x, torch.Tensor) else None
    if code is None or not x.is_cuda or x.dim() != dims:
        raise TypeError(f"{name} must be a CUDA tensor of {dims} dimensions and dtype float32, float16 or bfloat16")
    rows, cols = x.shape[-2:]
    *_, ld, step = x.stride()
    if step != 1 and cols > 1:
        raise TypeError(f"{name} must have contiguous rows")
    if rows <= 1:
        ld = cols
    elif ld < cols:
        raise ValueError(f"{name}'s rows overlap")
    return code, ld


def sidco_mx4_compress(grad, residual, codes, scales, stream=None) -> None:
    """Error feedback and 4-bit blocks of one flat gradient (float32, float16 or bfloat16); `residual` (float32) may be
    None.  codes, scales: uint8 of sidco_mx4_code_bytes(1, d) and sidco_mx4_scale_bytes(1, d)."""
    torch = _torch or _import_torch()
    code, d = _grad_code(grad), grad.numel()
    _check_tensor(grad, grad.dtype, "grad")
    if residual is not None:
        _check_tensor(residual, torch.float32, "residual", d)
    c, e = _check_packed(codes, scales, 1, d, "the gradient's")
    rc = load().sidco_mx4_compress(_stream_handle(stream), grad.data_ptr(), code, _ptr(residual), d, c, e)
    if rc:
        raise SidcoError(rc, "sidco_mx4_compress")


def sidco_mx4_aggregate(codes, scales, dense, scale: float = 1.0, accumulate: bool = False, stream=None) -> None:
    """dense (+)= scale * the sum of what the workers' blocks stand for; row w of codes and scales is worker w's."""
    torch = _torch or _import_torch()
    _check_tensor(dense, torch.float32, "dense", 1)
    d = dense.numel()
    if not isinstance(codes, torch.Tensor) or not isinstance(scales, torch.Tensor):
        raise TypeError("the workers' codes and scales must be contiguous CUDA tensors of dtype torch.uint8")
    if codes.dim() != 2 or scales.dim() != 2 or codes.shape[0] != scales.shape[0]:
        raise ValueError("codes and scales must have a row for each worker")
    workers, code_stride = codes.shape
    scale_stride = scales.shape[1]
    c, e = _check_packed(codes, scales, 1, 1, "the workers'")
    lines = (d + 255) // 256
    if code_stride < lines * 128 or scale_stride < lines * 8:
        raise ValueError("codes or scales are shorter than dense")
    rc = load().sidco_mx4_aggregate(_stream_handle(stream), c, code_stride, e, scale_stride, workers, d, scale, 1 if accumulate else 0,
                                    dense.data_ptr())
    if rc:
        raise SidcoError(rc, "sidco_mx4_aggregate")


def sidco_mx4_quantize(x, codes, scales, codes_t=None, scales_t=None, stream=None) -> None:
    """4-bit blocks of a matrix along its rows (codes, scales) and, transposed, along its columns (codes_t, scales_t);
    either pair may be None."""
    code, ld = _matrix(x, "x")
    rows, cols = x.shape
    if codes is not None or scales is not None:
        _check_packed(codes, scales, rows, cols, "the rows'")
    if codes_t is not None or scales_t is not None:
        _check_packed(codes_t, scales_t, cols, rows, "the columns'")
    _check(load().sidco_mx4_quantize(_stream_handle(stream), _ptr(x), code, rows, cols, ld, _ptr(codes), _ptr(scales),
                                     _ptr(codes_t), _ptr(scales_t)), "sidco_mx4_quantize")


def sidco_mx4_dequantize(codes, scales, out, stream=None) -> None:
    """What the blocks of out's rows stand for, in out's type."""
    code, ld = _matrix(out, "out")
    rows, cols = out.shape
    _check_packed(codes, scales, rows, cols, "the matrix's")
    _check(load().sidco_mx4_dequantize(_stream_handle(stream), _ptr(codes), _ptr(scales), rows, cols, _ptr(out), code, ld),
           "sidco_mx4_dequantize")


def sidco_mx4_matmul(a_codes, a_scales, b_codes, b_scales, k: int, out, alpha: float = 1.0, accumulate: bool = False,
                     stream=None) -> None:
    """out (+)= alpha A B^T; A has out's rows, B its columns, both of k numbers blocked along k."""
    code, ld = _matrix(out, "out")
    m, n = out.shape
    _check_packed(a_codes, a_scales, m, k, "A's")
    _check_packed(b_codes, b_scales, n, k, "B's")
    _check(load().sidco_mx4_matmul(_stream_handle(stream), _ptr(a_codes), _ptr(a_scales), _ptr(b_codes), _ptr(b_scales), m, n, k,
                                   alpha, int(accumulate), _ptr(out), code, ld), "sidco_mx4_matmul")


def sidco_mx4_linear(x, w_codes, w_scales, out, alpha: float = 1.0, accumulate: bool = False, stream=None) -> None:
    """out (+)= alpha x^ W^T: x's rows are quantised on the way, W has out's columns as its rows."""
    x_code, ldx = _matrix(x, "x")
    code, ld = _matrix(out, "out")
    rows, k = x.shape
    out_rows, n = out.shape
    if out_rows != rows:
        raise ValueError("out must have a row for each of x's")
    w, e = _check_packed(w_codes, w_scales, n, k, "the weight's")
    rc = load().sidco_mx4_linear(_stream_handle(stream), x.data_ptr(), x_code, rows, k, ldx, w, e, n, alpha, 1 if accumulate else 0,
                                 out.data_ptr(), code, ld)
    if rc:
        raise SidcoError(rc, "sidco_mx4_linear")


# ---- the orthogonalised update ----

NS_BY_TYPE, NS_HALF, NS_FULL = 0, 1, 2


def sidco_newton_schulz_default() -> NewtonSchulz:
    opt = NewtonSchulz()
    load().sidco_newton_schulz_default(C.byref(opt))
    return opt


def _newton_schulz(steps, coef, eps, precision):
    a, b, c = coef
    return NewtonSchulz(steps, a, b, c, eps, precision)


def sidco_workspace_bytes_orthogonalize(batch: int, rows: int, cols: int, out_dtype: int, precision: int = NS_BY_TYPE, steps: int = 5,
                                        coef=(3.4445, -4.7750, 2.0315)) -> int:
    """Of a call with these steps and coefficients, which decide the precision of a step and how many go together."""
    opt = _newton_schulz(steps, coef, 1e-7, precision)
    return int(load().sidco_workspace_bytes_orthogonalize(batch, rows, cols, out_dtype, C.byref(opt)))


def _batch(x, name):
    """(element code, row stride, matrix stride, batch, rows, cols) of a matrix or a batch of them."""
    torch = _torch or _import_torch()
    if not isinstance(x, torch.Tensor) or x.dim() not in (2, 3):
        raise TypeError(f"{name} must be a CUDA tensor of 2 or 3 dimensions and dtype float32, float16 or bfloat16")
    if x.dim() == 2:
        x = x[None]
    code, ld = _matrix(x, name, 3)
    batch, rows, cols = x.shape
    stride = x.stride(0) if batch > 1 else rows * ld
    return code, ld, stride, batch, rows, cols


def sidco_orthogonalize(x, out, steps: int = 5, coef=(3.4445, -4.7750, 2.0315), eps: float = 1e-7, precision: int = NS_BY_TYPE,
                        stream=None) -> None:
    """out = the matrix x, or each of a batch, near the closest one with orthonormal rows or columns."""
    code, ld, stride, batch, rows, cols = _batch(x, "x")
    out_code, ldo, out_stride, *shape = _batch(out, "out")
    if shape != [batch, rows, cols]:
        raise ValueError("out must have x's shape")
    opt = _newton_schulz(steps, coef, eps, precision)
    _check(load().sidco_orthogonalize(_stream_handle(stream), _ptr(x), code, ld, stride, batch, rows, cols, C.byref(opt), _ptr(out),
                                      out_code, ldo, out_stride), "sidco_orthogonalize")


def sidco_muon_step(grad, momentum, weight, lr: float, mu: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0,
                    scale: float = 1.0, steps: int = 5, coef=(3.4445, -4.7750, 2.0315), eps: float = 1e-7,
                    precision: int = NS_BY_TYPE, stream=None) -> None:
    """Momentum (float32), its orthogonalisation and the weights' update, in place, for a matrix or a batch of them; all
    three contiguous."""
    torch = _torch or _import_torch()
    code, _, _, batch, rows, cols = _batch(grad, "grad")
    w_code, *_ = _batch(weight, "weight")
    _check_tensor(momentum, torch.float32, "momentum")
    if weight.shape != grad.shape or momentum.shape != grad.shape:
        raise ValueError("grad, momentum and weight must have the same shape")
    _check_tensor(grad, grad.dtype, "grad")
    _check_tensor(weight, weight.dtype, "weight")
    opt = _newton_schulz(steps, coef, eps, precision)
    _check(load().sidco_muon_step(_stream_handle(stream), _ptr(grad), code, _ptr(momentum), _ptr(weight), w_code, batch, rows, cols, lr,
                                  mu, int(nesterov), weight_decay, scale, C.byref(opt)), "sidco_muon_step")


# ---- a language model's ends ----

WORD_I32, WORD_I64 = 0, 1

_word_types = None  # torch's integer types as the C ABI numbers them


# Small calls take the GPU about as long as the host, so these do in fewer steps what _matrix and _stream_handle do, and leave to them
# whatever is out of the ordinary.  A call's tensors are all on the current device: what another one's memory looks like from here
# is not known.


def _words(words, name, device):
    """Address, type and number of a contiguous tensor of words on that device, of any shape."""
    global _word_types
    if _word_types is None:
        torch = _torch or _import_torch()
        _word_types = {torch.int32: WORD_I32, torch.int64: WORD_I64}
    code = _word_types.get(words.dtype) if isinstance(words, _torch.Tensor) else None
    if code is None or not words.is_cuda or not words.is_contiguous():
        raise TypeError(f"{name} must be a contiguous CUDA tensor of dtype int32 or int64")
    if words.get_device() != device:
        raise ValueError(f"{name} must be on the other tensors' device")
    return words.data_ptr(), code, words.numel()


def _rows(x, name, device=None):
    """Address, element code, rows, columns, row stride and device of a CUDA matrix whose rows are contiguous."""
    ordinary = False
    if _types is not None and isinstance(x, _torch.Tensor) and x.dim() == 2:
        code, own = _types.get(x.dtype), x.get_device()
        rows, cols = x.shape
        ld, step = x.stride()
        ordinary = code is not None and own >= 0 and step == 1 and ld >= cols and rows > 1
    if not ordinary:
        code, ld = _matrix(x, name)
        rows, cols = x.shape
        own = x.get_device()
    if device is not None and own != device:
        raise ValueError(f"{name} must be on the other tensors' device")
    return x.data_ptr(), code, rows, cols, ld, own


def _vector(t, name, n, device):
    """Address of a contiguous float32 tensor of at least n elements on that device."""
    torch = _torch or _import_torch()
    _check_tensor(t, torch.float32, name, n)
    if t.get_device() != device:
        raise ValueError(f"{name} must be on the other tensors' device")
    return t.data_ptr()


_raw_stream = _current_device = None


def _stream_on(stream, device):
    """The handle of a stream, or of the current one, of the tensors' device, which has to be the current one."""
    global _raw_stream, _current_device
    if _current_device is None:
        raw, current = getattr(_torch._C, "_cuda_getCurrentRawStream", None), getattr(_torch._C, "_cuda_getDevice", None)
        _current_device = current or _torch.cuda.current_device
        _raw_stream = raw or (lambda device: _torch.cuda.current_stream(device).cuda_stream)
    if device != _current_device():
        raise ValueError("the tensors must be on the current device")
    return _raw_stream(device) if stream is None else stream.cuda_stream


def sidco_embedding(table, words, out, scale: float = 1.0, stream=None) -> None:
    """out[i] = scale * table[words[i]], zeros where words[i] is no row of the table; out has a row for each word."""
    t, code, vocab, dim, ldt, device = _rows(table, "table")
    o, out_code, rows, cols, ldo, _ = _rows(out, "out", device)
    w, word_type, n = _words(words, "words", device)
    if rows != n or cols != dim:
        raise ValueError("out must have a row of the table's length for each word")
    rc = load().sidco_embedding(_stream_on(stream, device), t, code, vocab, dim, ldt, w, word_type, n, scale, o, out_code, ldo)
    if rc:
        raise SidcoError(rc, "sidco_embedding")


def sidco_workspace_bytes_embedding_grad(n: int, dim: int) -> int:
    return int(load().sidco_workspace_bytes_embedding_grad(n, dim))


def sidco_embedding_grad(grad, words, table_grad, scale: float = 1.0, accumulate: bool = False, stream=None) -> None:
    """table_grad[v] (+)= scale * the sum of grad's rows whose word is v."""
    g, code, rows, cols, ldg, device = _rows(grad, "grad")
    t, table_code, vocab, dim, ldt, _ = _rows(table_grad, "table_grad", device)
    w, word_type, n = _words(words, "words", device)
    if rows != n or cols != dim:
        raise ValueError("grad must have a row of the table's length for each word")
    rc = load().sidco_embedding_grad(_stream_on(stream, device), g, code, n, dim, ldg, w, word_type, vocab, scale, 1 if accumulate else 0, t,
                                     table_code, ldt)
    if rc:
        raise SidcoError(rc, "sidco_embedding_grad")


def sidco_dropout_blocks(rows: int, cols: int) -> int:
    n = load().sidco_dropout_blocks(rows, cols)
    if n < 0:
        raise SidcoError(int(n), "sidco_dropout_blocks")
    return int(n)


def sidco_dropout(x, out, p: float, seed: int, offset: int = 0, residual=None, device_offset=None, stream=None) -> None:
    """out = x with elements dropped with probability p and the others scaled, plus residual (of out's type) if given.  seed and
    offset (in blocks of the sequence) are taken modulo 2^64; device_offset, a CUDA tensor of one int64, is added to the
    offset when the call runs."""
    a, code, rows, cols, ldx, device = _rows(x, "x")
    o, out_code, out_rows, out_cols, ldo, _ = _rows(out, "out", device)
    if out_rows != rows or out_cols != cols:
        raise ValueError("out must have x's shape")
    r, ldr = None, 0
    if residual is not None:
        r, res_code, res_rows, res_cols, ldr, _ = _rows(residual, "residual", device)
        if res_code != out_code:
            raise TypeError("residual must have out's dtype")
        if res_rows != rows or res_cols != cols:
            raise ValueError("residual must have x's shape")
    if device_offset is not None:
        _check_tensor(device_offset, _torch.int64, "device_offset", 1)
        if device_offset.get_device() != device:
            raise ValueError("device_offset must be on the other tensors' device")
    rc = load().sidco_dropout(_stream_on(stream, device), a, code, rows, cols, ldx, p, seed & 0xFFFFFFFFFFFFFFFF, offset & 0xFFFFFFFFFFFFFFFF,
                              _ptr(device_offset), r, ldr, o, out_code, ldo)
    if rc:
        raise SidcoError(rc, "sidco_dropout")


def _logits(x, weight, targets):
    """Arguments that both cross entropy calls begin with, and their sizes."""
    a, code, rows, dim, ldx, device = _rows(x, "x")
    b, w_code, vocab, cols, ldw, _ = _rows(weight, "weight", device)
    if w_code != code:
        raise TypeError("weight must have x's dtype")
    w, word_type, n = _words(targets, "targets", device)
    if cols != dim or rows != n:
        raise ValueError("weight must have x's columns, and targets a word for each of its rows")
    return (a, b, code, n, dim, vocab, ldx, ldw, w, word_type), n, code, device


def sidco_workspace_bytes_cross_entropy(n: int, dim: int, vocab: int, dtype: int) -> int:
    return int(load().sidco_workspace_bytes_cross_entropy(n, dim, vocab, dtype))


def sidco_cross_entropy(x, weight, targets, loss, lse, stream=None) -> None:
    """loss[i] = lse[i] - (x weight^T)[i, targets[i]], lse[i] the logarithm of the row's sum of exponentials; either may be None."""
    args, n, _, device = _logits(x, weight, targets)
    a = None if loss is None else _vector(loss, "loss", n, device)
    b = None if lse is None else _vector(lse, "lse", n, device)
    rc = load().sidco_cross_entropy(_stream_on(stream, device), *args, a, b)
    if rc:
        raise SidcoError(rc, "sidco_cross_entropy")


def sidco_workspace_bytes_cross_entropy_grad(n: int, dim: int, vocab: int, dtype: int, weight_grad_dtype: int) -> int:
    return int(load().sidco_workspace_bytes_cross_entropy_grad(n, dim, vocab, dtype, weight_grad_dtype))


def sidco_cross_entropy_grad(x, weight, targets, lse, loss_grad, x_grad=None, weight_grad=None, accumulate: bool = False,
                             stream=None, loss=None) -> None:
    """The gradients of the sum of loss_grad[i] * loss[i] (None: of the losses' sum) with respect to x, in its dtype, and weight, in its
    dtype or float32, or with `accumulate` added to what weight_grad holds; either may be None.  lse is what sidco_cross_entropy
    wrote, and so is loss, which need not be given: with it a call is some microseconds shorter, and in a large batch over a large
    vocabulary the gradients of rows whose loss is tiny, 2^-23 of |lse|, are kept too."""
    args, n, code, device = _logits(x, weight, targets)
    sums = _vector(lse, "lse", n, device)
    known = None if loss is None else _vector(loss, "loss", n, device)
    g = None if loss_grad is None else _vector(loss_grad, "loss_grad", n, device)
    gx = gw = None
    ldgx = ldgw = w_code = 0
    if x_grad is not None:
        gx, x_code, rows, cols, ldgx, _ = _rows(x_grad, "x_grad", device)
        if x_code != code:
            raise TypeError("x_grad must have x's dtype")
        if x_grad.shape != x.shape:
            raise ValueError("x_grad must have x's shape")
    if weight_grad is not None:
        gw, w_code, rows, cols, ldgw, _ = _rows(weight_grad, "weight_grad", device)
        if weight_grad.shape != weight.shape:
            raise ValueError("weight_grad must have weight's shape")
    rc = load().sidco_cross_entropy_grad_of_loss(_stream_on(stream, device), *args, known, sums, g, gx, ldgx, gw, w_code, ldgw,
                                                 1 if accumulate else 0)
    if rc:
        raise SidcoError(rc, "sidco_cross_entropy_grad")


def sidco_version() -> int:
    return load().sidco_version()


def sidco_shutdown() -> None:
    load().sidco_shutdown()
