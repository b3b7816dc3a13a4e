"""Python binding of ``libatb.so`` - the asymmetric-tile-buffered BFP16 x BF16 GEMM for B200.

Argument marshalling only: every step of the hot path (quantisation, dequantisation, the
GEMM, the epilogue) runs in the CUDA kernels behind the C ABI declared in ``include/atb.h``.
The functions carry the C names.  PyTorch is used for device memory and streams.

There is no CPU path: importing works anywhere (the input generators in
``paper_2511_16041_b200.inputs`` need only numpy), but the first call of a device function
raises if the library cannot be loaded.
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("ATB_LIBRARY_PATH") or os.path.join(_HERE, "libatb.so")
_lib = None

ATB_OK = 0
STATUS_NAMES = {
    0: "ATB_OK", 1: "ATB_ERR_NULL_POINTER", 2: "ATB_ERR_BAD_SHAPE", 3: "ATB_ERR_BAD_TILING",
    4: "ATB_ERR_MISALIGNED", 5: "ATB_ERR_UNSUPPORTED_DEVICE", 6: "ATB_ERR_CUDA",
    7: "ATB_ERR_BUFFER_TOO_SMALL", 8: "ATB_ERR_DEVICE_TIMEOUT", 9: "ATB_ERR_BAD_ARGUMENT",
}


class AtbError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


class atb_tiling_t(ctypes.Structure):
    _fields_ = [("T_MA", ctypes.c_int), ("T_MC", ctypes.c_int), ("T_K", ctypes.c_int), ("T_N", ctypes.c_int)]


class atb_hw_params_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("peak_flops_per_cycle", "clock_hz")] + [("n_units", ctypes.c_int)] + \
               [(n, ctypes.c_double) for n in ("bw_bytes_per_s", "a_bytes", "b_bytes", "c_bytes", "a_buf_bytes",
                                               "b_buf_bytes", "c_buf_bytes", "a_scratch_bytes",
                                               "buf_capacity_bytes", "acc_capacity_bytes")] + \
               [("share_rows", ctypes.c_int), ("share_cols", ctypes.c_int)] + \
               [(n, ctypes.c_double) for n in ("eta", "eps_cycles", "ii", "delta_cycles")] + \
               [("mma_rows", ctypes.c_int)] + \
               [(n, ctypes.c_double) for n in ("load_latency_cycles", "pair_efficiency", "launch_seconds", "tile_fixed_cycles",
                                               "drain_cycles_per_column", "pair_tile_cycles", "thin_slab_cost",
                                               "coarse_slab_factor", "deep_kstep_factor", "convert_cycles",
                                               "convert_exposed_cycles", "convert_latency_cycles")] + \
               [("a_unit_cols", ctypes.c_int)]


class atb_tiling_score_t(ctypes.Structure):
    _fields_ = [("t", atb_tiling_t), ("feasible", ctypes.c_int)] + \
               [(n, ctypes.c_double) for n in ("buf_bytes_used", "acc_bytes_used", "ai", "eff_micro", "eff_core",
                                               "mem_bound_flops", "compute_bound_flops", "predicted_flops")]


class atb_plan_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("n_b_stages", "n_raw_stages", "n_a_groups", "dequant_groups",
                                            "acc_buffers", "tmem_columns", "smem_bytes")]


class Tiling(NamedTuple):
    T_MA: int
    T_MC: int
    T_K: int
    T_N: int


EXPORTED_SYMBOLS = [
    "atb_status_string", "atb_last_error_message", "atb_bfp16_mant_bytes", "atb_bfp16_exp_bytes",
    "atb_quantize_bfp16", "atb_gemm", "atb_gemm_bfp16_out", "atb_gemm_config", "atb_gemm_config_tiled", "atb_gemm_splitk", "atb_gemm_splitk_workspace_bytes", "atb_select_splits",
    "atb_gemm_splitk_noalloc",
    "atb_tiling_supported", "atb_tiling_plan", "atb_device_status",
    "atb_hw_params_b200", "atb_hw_params_xdna2", "atb_score_tiling", "atb_select_tiling",
    "atb_layer_norm", "atb_layer_norm_bfp16", "atb_layer_norm_backward", "atb_layer_norm_backward_workspace_bytes",
    "atb_gated_ffn", "atb_gated_ffn_workspace_bytes", "atb_gated_ffn_backward", "atb_gated_ffn_backward_workspace_bytes",
    "atb_linear_cross_entropy", "atb_linear_cross_entropy_workspace_bytes",
    "atb_linear_cross_entropy_backward", "atb_linear_cross_entropy_backward_workspace_bytes",
]


def load_library():
    """Loads ``libatb.so`` (built in-tree by ``_build.build_library``).  Raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                           "`python -m paper_2511_16041_b200._build` (there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    i64, vp, ci = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
    lib.atb_status_string.restype = ctypes.c_char_p
    lib.atb_status_string.argtypes = [ci]
    lib.atb_last_error_message.restype = ctypes.c_char_p
    lib.atb_bfp16_mant_bytes.restype = ctypes.c_size_t
    lib.atb_bfp16_mant_bytes.argtypes = [i64, i64]
    lib.atb_bfp16_exp_bytes.restype = ctypes.c_size_t
    lib.atb_bfp16_exp_bytes.argtypes = [i64, i64]
    lib.atb_quantize_bfp16.restype = ci
    lib.atb_quantize_bfp16.argtypes = [vp, i64, i64, i64, vp, vp, vp]
    lib.atb_gemm.restype = ci
    lib.atb_gemm.argtypes = [i64, i64, i64, ci, ci, ci, ci, vp, vp, vp, i64, vp, i64, vp]
    lib.atb_gemm_bfp16_out.restype = ci
    lib.atb_gemm_bfp16_out.argtypes = [i64, i64, i64, ci, ci, ci, ci, vp, vp, vp, i64, vp, vp, vp]
    lib.atb_gemm_config.restype = ci
    lib.atb_gemm_config.argtypes = [ci, i64, i64, i64, vp, vp, i64, vp, vp, vp, vp, i64, vp]
    lib.atb_gemm_config_tiled.restype = ci
    lib.atb_gemm_config_tiled.argtypes = [ci, i64, i64, i64, ci, ci, ci, ci, vp, vp, i64, vp, vp, vp, vp, i64, vp]
    lib.atb_gemm_splitk.restype = ci
    lib.atb_gemm_splitk.argtypes = [i64, i64, i64, ci, ci, ci, ci, vp, vp, vp, i64, vp, i64, ci, vp, ctypes.c_size_t, vp]
    lib.atb_gemm_splitk_noalloc.restype = ci
    lib.atb_gemm_splitk_noalloc.argtypes = [i64, i64, i64, ci, ci, ci, ci, vp, vp, vp, i64, vp, i64, ci, vp]
    lib.atb_gemm_splitk_workspace_bytes.restype = ctypes.c_size_t
    lib.atb_gemm_splitk_workspace_bytes.argtypes = [i64, i64, ci, ci]
    lib.atb_select_splits.restype = ci
    lib.atb_select_splits.argtypes = [i64, i64, i64, ci, ci, ci]
    lib.atb_tiling_supported.restype = ci
    lib.atb_tiling_supported.argtypes = [ci, ci, ci, ci]
    lib.atb_tiling_plan.restype = ci
    lib.atb_tiling_plan.argtypes = [ci, ci, ci, ci, ctypes.POINTER(atb_plan_t)]
    lib.atb_device_status.restype = ci
    lib.atb_device_status.argtypes = [vp]
    lib.atb_hw_params_b200.restype = None
    lib.atb_hw_params_b200.argtypes = [ctypes.POINTER(atb_hw_params_t)]
    lib.atb_hw_params_xdna2.restype = None
    lib.atb_hw_params_xdna2.argtypes = [ctypes.POINTER(atb_hw_params_t), ci]
    lib.atb_score_tiling.restype = ci
    lib.atb_score_tiling.argtypes = [ctypes.POINTER(atb_hw_params_t), i64, atb_tiling_t,
                                     ctypes.POINTER(atb_tiling_score_t)]
    lib.atb_select_tiling.restype = ci
    lib.atb_select_tiling.argtypes = [i64, i64, i64, ctypes.POINTER(atb_hw_params_t),
                                      ctypes.POINTER(atb_tiling_t), ctypes.POINTER(atb_tiling_score_t),
                                      ctypes.POINTER(ci)]
    cf, sz = ctypes.c_float, ctypes.c_size_t
    for name, restype, argtypes in (
            ("atb_layer_norm", ci, [i64, i64, ci, vp, i64, ci, vp, vp, cf, vp, i64, vp, vp, vp]),
            ("atb_layer_norm_bfp16", ci, [i64, i64, ci, vp, i64, ci, vp, vp, cf, vp, vp, vp, vp, vp]),
            ("atb_layer_norm_backward_workspace_bytes", sz, [i64, i64]),
            ("atb_layer_norm_backward", ci, [i64, i64, ci, vp, i64, vp, i64, ci, vp, vp, vp, vp, i64, vp, vp, vp, sz, vp]),
            ("atb_gated_ffn_workspace_bytes", sz, [i64, i64, i64]),
            ("atb_gated_ffn", ci, [i64, i64, i64, ci, vp, i64, vp, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, sz, vp]),
            ("atb_gated_ffn_backward_workspace_bytes", sz, [i64, i64, i64]),
            ("atb_gated_ffn_backward", ci, [i64, i64, i64, ci, vp, i64, vp, i64, vp, vp, i64, vp, i64, vp, vp, vp, vp, i64, vp, vp, i64,
                                            vp, i64, vp, sz, vp]),
            ("atb_linear_cross_entropy_workspace_bytes", sz, [i64, i64, i64]),
            ("atb_linear_cross_entropy", ci, [i64, i64, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, sz, vp]),
            ("atb_linear_cross_entropy_backward_workspace_bytes", sz, [i64, i64, i64, i64]),
            ("atb_linear_cross_entropy_backward", ci, [i64, i64, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, i64, vp, sz, vp])):
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = restype, argtypes
    _lib = lib
    return lib


def _check(status: int):
    if status != ATB_OK:
        raise AtbError(status, load_library().atb_last_error_message().decode())


def _stream_ptr(stream):
    if stream is None:
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # 3 us less per call than the Stream object
        return ctypes.c_void_p(raw(torch.cuda.current_device()) if raw else torch.cuda.current_stream().cuda_stream)
    if isinstance(stream, int):
        return ctypes.c_void_p(stream)
    return ctypes.c_void_p(stream.cuda_stream)


def _dev_ptr(t):
    return ctypes.c_void_p(t if isinstance(t, int) else t.data_ptr())


# ------------------------------------------------------------------ plain helpers
def atb_status_string(status: int) -> str:
    return load_library().atb_status_string(status).decode()


def atb_last_error_message() -> str:
    return load_library().atb_last_error_message().decode()


def atb_bfp16_mant_bytes(M: int, K: int) -> int:
    return int(load_library().atb_bfp16_mant_bytes(M, K))


def atb_bfp16_exp_bytes(M: int, K: int) -> int:
    return int(load_library().atb_bfp16_exp_bytes(M, K))


def atb_tiling_supported(T_MA: int, T_MC: int, T_K: int, T_N: int) -> bool:
    return bool(load_library().atb_tiling_supported(T_MA, T_MC, T_K, T_N))


def atb_tiling_plan(T_MA: int, T_MC: int, T_K: int, T_N: int) -> atb_plan_t:
    plan = atb_plan_t()
    _check(load_library().atb_tiling_plan(T_MA, T_MC, T_K, T_N, ctypes.byref(plan)))
    return plan


# ------------------------------------------------------------------ device calls
def atb_quantize_bfp16(A, mant=None, exp=None, stream=None):
    """fp32 CUDA tensor ``A[M][K]`` (row stride = lda) -> (mant int8 [M][K], exponent plane uint8).

    The exponent plane is the flat device layout ``[ceil(K/64)][roundup(M,32)][8]``."""
    import torch
    assert A.is_cuda and A.dtype == torch.float32 and A.dim() == 2 and A.stride(1) == 1
    M, K = A.shape
    if mant is None:
        mant = torch.empty((M, K), dtype=torch.int8, device=A.device)
    if exp is None:
        exp = torch.empty(atb_bfp16_exp_bytes(M, K), dtype=torch.uint8, device=A.device)
    _check(load_library().atb_quantize_bfp16(_dev_ptr(A), M, K, A.stride(0) if M > 1 else max(K, A.stride(0)),
                                              _dev_ptr(mant), _dev_ptr(exp), _stream_ptr(stream)))
    return mant, exp


def atb_gemm(M, N, K, T_MA, T_MC, T_K, T_N, A_mant, A_exp, B, C=None, ldb=None, ldc=None, stream=None):
    """``C[M][N] = dequant(A) @ B``; B, C are bf16 CUDA tensors (row-major).  Returns C."""
    import torch
    if C is None:
        C = torch.empty((M, N), dtype=torch.bfloat16, device=B.device)
    if ldb is None:
        ldb = B.stride(0) if not isinstance(B, int) else N
    if ldc is None:
        ldc = C.stride(0) if not isinstance(C, int) else N
    _check(load_library().atb_gemm(M, N, K, T_MA, T_MC, T_K, T_N, _dev_ptr(A_mant), _dev_ptr(A_exp),
                                   _dev_ptr(B), ldb, _dev_ptr(C), ldc, _stream_ptr(stream)))
    return C


def atb_gemm_splitk_workspace_bytes(M: int, N: int, T_MC: int, splits: int) -> int:
    return int(load_library().atb_gemm_splitk_workspace_bytes(M, N, T_MC, splits))


def atb_select_splits(M: int, N: int, K: int, T_MC: int, T_K: int, T_N: int) -> int:
    return int(load_library().atb_select_splits(M, N, K, T_MC, T_K, T_N))


def atb_gemm_splitk(M, N, K, T_MA, T_MC, T_K, T_N, A_mant, A_exp, B, splits, workspace=None, C=None, ldb=None,
                    ldc=None, stream=None):
    """Split-K ``C[M][N] = dequant(A) @ B``; ``workspace`` is a float32 CUDA tensor (allocated if None)."""
    import torch
    if C is None:
        C = torch.empty((M, N), dtype=torch.bfloat16, device=B.device)
    if workspace is None:
        workspace = torch.empty(atb_gemm_splitk_workspace_bytes(M, N, T_MC, splits) // 4, dtype=torch.float32,
                                device=B.device)
    if ldb is None:
        ldb = B.stride(0)
    if ldc is None:
        ldc = C.stride(0)
    _check(load_library().atb_gemm_splitk(M, N, K, T_MA, T_MC, T_K, T_N, _dev_ptr(A_mant), _dev_ptr(A_exp), _dev_ptr(B),
                                          ldb, _dev_ptr(C), ldc, splits, _dev_ptr(workspace),
                                          workspace.numel() * workspace.element_size(), _stream_ptr(stream)))
    return C


def atb_gemm_bfp16_out(M, N, K, T_MA, T_MC, T_K, T_N, A_mant, A_exp, B, C_mant=None, C_exp=None, ldb=None, stream=None):
    """``C = dequant(A) @ B`` written as BFP16 planes (quantising epilogue).  Returns ``(C_mant, C_exp)``:
    an int8 ``[M, N]`` tensor and the exponent plane, both usable as the A operand of the next GEMM."""
    import torch
    if C_mant is None:
        C_mant = torch.empty((M, N), dtype=torch.int8, device=B.device)
    if C_exp is None:
        C_exp = torch.empty(atb_bfp16_exp_bytes(M, N), dtype=torch.uint8, device=B.device)
    if ldb is None:
        ldb = B.stride(0)
    _check(load_library().atb_gemm_bfp16_out(M, N, K, T_MA, T_MC, T_K, T_N, _dev_ptr(A_mant), _dev_ptr(A_exp), _dev_ptr(B),
                                             ldb, _dev_ptr(C_mant), _dev_ptr(C_exp), _stream_ptr(stream)))
    return C_mant, C_exp


def atb_gemm_config_tiled(config, M, N, K, T_MA, T_MC, T_K, T_N, A, A_exp, Bt_mant, Bt_exp, C=None, C_exp=None, stream=None):
    """The paper's precision configurations with the BFP16 operand on the B side (planes of B transposed),
    A streamed in slabs of ``T_MA`` rows; ``T_K, T_N`` = 64, 256 and ``T_MC`` = 256 (one SM) or 512 (a CTA pair
    that shares the converted B tile).

    ``config=1``: ``A`` is a bf16 ``[M, K]`` tensor (``A_exp=None``); returns bf16 ``C``.
    ``config=2``: ``A`` / ``A_exp`` are BFP16 planes; returns ``(C_mant, C_exp)``."""
    import torch
    dev = Bt_mant.device
    if config == 1:
        if C is None:
            C = torch.empty((M, N), dtype=torch.bfloat16, device=dev)
        _check(load_library().atb_gemm_config_tiled(1, M, N, K, T_MA, T_MC, T_K, T_N, _dev_ptr(A), None, A.stride(0),
                                                    _dev_ptr(Bt_mant), _dev_ptr(Bt_exp), _dev_ptr(C), None, C.stride(0),
                                                    _stream_ptr(stream)))
        return C
    if C is None:
        C = torch.empty((M, N), dtype=torch.int8, device=dev)
    if C_exp is None:
        C_exp = torch.empty(atb_bfp16_exp_bytes(M, N), dtype=torch.uint8, device=dev)
    _check(load_library().atb_gemm_config_tiled(config, M, N, K, T_MA, T_MC, T_K, T_N, _dev_ptr(A),
                                                _dev_ptr(A_exp) if A_exp is not None else None, K, _dev_ptr(Bt_mant),
                                                _dev_ptr(Bt_exp), _dev_ptr(C), _dev_ptr(C_exp), N, _stream_ptr(stream)))
    return C, C_exp


def atb_gemm_config(config, M, N, K, A, A_exp, Bt_mant, Bt_exp, C=None, C_exp=None, stream=None):
    """``atb_gemm_config_tiled`` with 128-row slabs, on a CTA pair where M > 256; goes through the C entry of the
    same name."""
    import torch
    dev = Bt_mant.device
    if config == 1:
        if C is None:
            C = torch.empty((M, N), dtype=torch.bfloat16, device=dev)
        _check(load_library().atb_gemm_config(1, M, N, K, _dev_ptr(A), None, A.stride(0), _dev_ptr(Bt_mant), _dev_ptr(Bt_exp),
                                              _dev_ptr(C), None, C.stride(0), _stream_ptr(stream)))
        return C
    if C is None:
        C = torch.empty((M, N), dtype=torch.int8, device=dev)
    if C_exp is None:
        C_exp = torch.empty(atb_bfp16_exp_bytes(M, N), dtype=torch.uint8, device=dev)
    _check(load_library().atb_gemm_config(config, M, N, K, _dev_ptr(A), _dev_ptr(A_exp) if A_exp is not None else None, K,
                                          _dev_ptr(Bt_mant), _dev_ptr(Bt_exp), _dev_ptr(C), _dev_ptr(C_exp), N,
                                          _stream_ptr(stream)))
    return C, C_exp


NOALLOC_SCRATCH_BYTES = 64 * 1024 * 1024


def atb_gemm_splitk_noalloc(M, N, K, T_MA, T_MC, T_K, T_N, A_mant, A_exp, B, splits, C, ldb=None, ldc=None, stream=None):
    """Split-K GEMM whose partial sums live in the library's built-in 64 MiB device array.

    For callers that may not allocate: the binding allocates nothing either, so ``C`` (bf16 CUDA tensor)
    has to be passed in.  Raises ``AtbError`` (ATB_ERR_BUFFER_TOO_SMALL) when
    ``atb_gemm_splitk_workspace_bytes(M, N, T_MC, splits)`` exceeds ``NOALLOC_SCRATCH_BYTES``.
    Calls that may overlap on the GPU must be ordered by the caller: they share the array."""
    if ldb is None:
        ldb = B.stride(0)
    if ldc is None:
        ldc = C.stride(0)
    _check(load_library().atb_gemm_splitk_noalloc(M, N, K, T_MA, T_MC, T_K, T_N, _dev_ptr(A_mant), _dev_ptr(A_exp),
                                                  _dev_ptr(B), ldb, _dev_ptr(C), ldc, splits, _stream_ptr(stream)))
    return C


def atb_device_status(stream=None):
    """Synchronises ``stream`` and raises ``AtbError`` if a kernel gave up a bounded wait."""
    _check(load_library().atb_device_status(_stream_ptr(stream)))


# ------------------------------------------------------------------ host model
def atb_hw_params_b200() -> atb_hw_params_t:
    hw = atb_hw_params_t()
    load_library().atb_hw_params_b200(ctypes.byref(hw))
    return hw


def atb_hw_params_xdna2(precision_config: int) -> atb_hw_params_t:
    hw = atb_hw_params_t()
    load_library().atb_hw_params_xdna2(ctypes.byref(hw), precision_config)
    return hw


def atb_score_tiling(hw: atb_hw_params_t, K: int, tiling) -> atb_tiling_score_t:
    out = atb_tiling_score_t()
    _check(load_library().atb_score_tiling(ctypes.byref(hw), K, atb_tiling_t(*tiling), ctypes.byref(out)))
    return out


def atb_select_tiling(M: int, N: int, K: int, hw: atb_hw_params_t | None = None, max_scores: int = 128):
    """Returns ``(best: Tiling, scores: list[atb_tiling_score_t])`` - scores best first."""
    best = atb_tiling_t()
    scores = (atb_tiling_score_t * max_scores)()
    n = ctypes.c_int(max_scores)
    _check(load_library().atb_select_tiling(M, N, K, ctypes.byref(hw) if hw is not None else None,
                                            ctypes.byref(best), scores, ctypes.byref(n)))
    return Tiling(best.T_MA, best.T_MC, best.T_K, best.T_N), [scores[i] for i in range(n.value)]


# ------------------------------------------------------------------ between the products: norm, feed-forward, loss
ATB_F32, ATB_BF16 = 0, 1
ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2}


def _dtype(t):
    import torch
    if t.dtype == torch.float32:
        return ATB_F32
    if t.dtype == torch.bfloat16:
        return ATB_BF16
    raise TypeError(f"{t.dtype}: float32 or bfloat16")


def _matrix(t, rows, cols, dtype, device, name):
    """Checks a row-major matrix on CUDA device number ``device`` and returns its leading dimension."""
    if t.dtype is dtype and t.shape == (rows, cols) and t.get_device() == device:
        ld, one = t.stride()
        if one == 1 or cols <= 1:
            return ld if rows > 1 or ld > cols else cols
    raise ValueError(f"{name}: a row-major matrix {(rows, cols)} of {dtype} on cuda:{device}, got {tuple(t.shape)} of {t.dtype} on {t.device}, "
                     f"strides {t.stride()}")


def _vector(t, n, dtype, device, name):
    if t.dtype is not dtype or t.shape != (n,) or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous vector of {n} {dtype} on cuda:{device}, got {tuple(t.shape)} of {t.dtype} on {t.device}")


def _opt_ptr(t):
    return None if t is None else t.data_ptr()


def _workspace(workspace, need, like):
    """Address and size of the caller's workspace, or of a new one of ``need`` bytes (kept alive by the third value)."""
    import torch
    if workspace is None:
        if need == 0:
            return None, 0, None
        workspace = like.new_empty((need,), dtype=torch.uint8)
    elif workspace.get_device() != like.get_device() or not workspace.is_contiguous():
        raise ValueError(f"workspace: contiguous, on {like.device}")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


def _device_of(t, name):
    """Number of the CUDA device of the matrix ``t``, which has to be the current one (the kernels are launched there)."""
    import torch
    device = t.get_device()
    if device < 0 or t.dim() != 2:
        raise ValueError(f"{name}: a CUDA matrix, got {tuple(t.shape)} on {t.device}")
    if device != torch.cuda.current_device():
        raise ValueError(f"{name} is on cuda:{device}, the current device is cuda:{torch.cuda.current_device()}")
    return device


def _norm_weights(W, B, N, x_dtype, device):
    """The type code of the weights (any where there are none)."""
    given = W if W is not None else B
    if given is None:
        return ATB_F32
    for t, name in ((W, "W"), (B, "B")):
        if t is not None:
            _vector(t, N, given.dtype, device, name)
    return _dtype(given)


def _out_matrix(t, like, rows, cols, dtype, device, name):
    """An output of the caller's, checked, or a new one; and its leading dimension.  ``like``: a tensor on the device, best one
    of the output's shape and type (a copy of its description costs the host least)."""
    if t is not None:
        return t, _matrix(t, rows, cols, dtype, device, name)
    if like.dtype is dtype and like.shape == (rows, cols) and like.is_contiguous():
        import torch
        return torch.empty_like(like), cols
    return like.new_empty((rows, cols), dtype=dtype), cols


def _out_vector(t, like, n, dtype, device, name):
    if t is not None:
        _vector(t, n, dtype, device, name)
        return t
    if like.dtype is dtype and like.shape == (n,) and like.is_contiguous():
        import torch
        return torch.empty_like(like)
    return like.new_empty((n,), dtype=dtype)


def atb_layer_norm(X, W=None, B=None, eps=1e-5, Y=None, mean=None, rstd=None, stream=None):
    """Layer norm of the rows of ``X`` (float32 or bfloat16 ``[M, N]``); ``W``, ``B``: ``[N]`` of one type, or None.

    Returns ``(Y, mean, rstd)``: the result in X's type and the float32 statistics that the backward pass takes."""
    import torch
    device = _device_of(X, "X")
    (M, N), dtype = X.shape, X.dtype
    ldx = _matrix(X, M, N, dtype, device, "X")
    w_type = _norm_weights(W, B, N, dtype, device)
    Y, ldy = _out_matrix(Y, X, M, N, dtype, device, "Y")
    mean = _out_vector(mean, X, M, torch.float32, device, "mean")
    rstd = _out_vector(rstd, mean, M, torch.float32, device, "rstd")
    _check(load_library().atb_layer_norm(M, N, _dtype(X), X.data_ptr(), ldx, w_type, _opt_ptr(W), _opt_ptr(B), eps, Y.data_ptr(), ldy,
                                         mean.data_ptr(), rstd.data_ptr(), _stream_ptr(stream)))
    return Y, mean, rstd


def atb_layer_norm_bfp16(X, W=None, B=None, eps=1e-5, mant=None, exp=None, mean=None, rstd=None, stream=None):
    """Layer norm that leaves as BFP16 planes, the A operand of ``atb_gemm``.  Returns ``(mant, exp, mean, rstd)``."""
    import torch
    device = _device_of(X, "X")
    (M, N), dtype = X.shape, X.dtype
    ldx = _matrix(X, M, N, dtype, device, "X")
    w_type = _norm_weights(W, B, N, dtype, device)
    mant, ldm = _out_matrix(mant, X, M, N, torch.int8, device, "mant")
    if ldm != N:
        raise ValueError("mant: contiguous")
    exp = _out_vector(exp, X, atb_bfp16_exp_bytes(M, N), torch.uint8, device, "exp")
    mean = _out_vector(mean, X, M, torch.float32, device, "mean")
    rstd = _out_vector(rstd, mean, M, torch.float32, device, "rstd")
    _check(load_library().atb_layer_norm_bfp16(M, N, _dtype(X), X.data_ptr(), ldx, w_type, _opt_ptr(W), _opt_ptr(B), eps,
                                               mant.data_ptr(), exp.data_ptr(), mean.data_ptr(), rstd.data_ptr(), _stream_ptr(stream)))
    return mant, exp, mean, rstd


def atb_layer_norm_backward_workspace_bytes(M: int, N: int) -> int:
    return int(load_library().atb_layer_norm_backward_workspace_bytes(M, N))


def atb_layer_norm_backward(dY, X, W, mean, rstd, dX=None, dW=None, dB=None, workspace=None, stream=None):
    """Gradients ``(dX, dW, dB)`` of ``atb_layer_norm``; dW and dB in W's type (float32 where W is None)."""
    import torch
    device = _device_of(X, "X")
    (M, N), dtype = X.shape, X.dtype
    ldx = _matrix(X, M, N, dtype, device, "X")
    lddy = _matrix(dY, M, N, dtype, device, "dY")
    w_dtype = torch.float32
    if W is not None:
        w_dtype = W.dtype
        _vector(W, N, w_dtype, device, "W")
    _vector(mean, M, torch.float32, device, "mean")
    _vector(rstd, M, torch.float32, device, "rstd")
    dX, lddx = _out_matrix(dX, X, M, N, dtype, device, "dX")
    dW = _out_vector(dW, X if W is None else W, N, w_dtype, device, "dW")
    dB = _out_vector(dB, dW, N, w_dtype, device, "dB")
    lib = load_library()
    ws, ws_bytes, workspace = _workspace(workspace, lib.atb_layer_norm_backward_workspace_bytes(M, N), X)
    _check(lib.atb_layer_norm_backward(M, N, _dtype(X), dY.data_ptr(), lddy, X.data_ptr(), ldx, _dtype(dW), _opt_ptr(W), mean.data_ptr(),
                                       rstd.data_ptr(), dX.data_ptr(), lddx, dW.data_ptr(), dB.data_ptr(), ws, ws_bytes, _stream_ptr(stream)))
    return dX, dW, dB


def _ffn_shapes(X, Wg, Wu, Wd):
    import torch
    device, bf16 = _device_of(X, "X"), torch.bfloat16
    (M, D), F = X.shape, Wd.shape[0]
    ldx, ldw, ldwd = _matrix(X, M, D, bf16, device, "X"), _matrix(Wg, D, F, bf16, device, "Wg"), _matrix(Wd, F, D, bf16, device, "Wd")
    if _matrix(Wu, D, F, bf16, device, "Wu") != ldw:
        raise ValueError("Wg and Wu need the same row stride")
    return M, D, F, ldx, ldw, ldwd, device


def _hidden(t, like, M, F, device, name):
    """H, G or U: the caller's, contiguous, or a new one."""
    import torch
    t, ld = _out_matrix(t, like, M, F, torch.bfloat16, device, name)
    if ld != F:
        raise ValueError(f"{name}: contiguous")
    return t


def _act(act):
    return ACTIVATIONS[act] if act in ACTIVATIONS else int(act)


def atb_gated_ffn_workspace_bytes(M: int, D: int, F: int) -> int:
    return int(load_library().atb_gated_ffn_workspace_bytes(M, D, F))


def atb_gated_ffn(X, Wg, Wu, Wd, act="silu", save=False, Y=None, H=None, G=None, U=None, workspace=None, stream=None):
    """``Y = (act(X Wg) * (X Wu)) Wd`` on bfloat16 matrices ``X [M, D]``, ``Wg``, ``Wu`` ``[D, F]``, ``Wd [F, D]``.

    ``act``: "silu", "gelu" or "gelu_tanh".  Returns Y, or with ``save`` ``(Y, H, G, U)``: what the backward pass takes."""
    import torch
    M, D, F, ldx, ldw, ldwd, device = _ffn_shapes(X, Wg, Wu, Wd)
    Y, ldy = _out_matrix(Y, X, M, D, torch.bfloat16, device, "Y")
    H = _hidden(H, X, M, F, device, "H")
    if save or G is not None or U is not None:
        G, U = _hidden(G, H, M, F, device, "G"), _hidden(U, H, M, F, device, "U")
    lib = load_library()
    ws, ws_bytes, workspace = _workspace(workspace, lib.atb_gated_ffn_workspace_bytes(M, D, F), X)
    _check(lib.atb_gated_ffn(M, D, F, _act(act), X.data_ptr(), ldx, Wg.data_ptr(), Wu.data_ptr(), ldw, Wd.data_ptr(), ldwd, Y.data_ptr(), ldy,
                             H.data_ptr(), _opt_ptr(G), _opt_ptr(U), ws, ws_bytes, _stream_ptr(stream)))
    return (Y, H, G, U) if save else Y


def atb_gated_ffn_backward_workspace_bytes(M: int, D: int, F: int) -> int:
    return int(load_library().atb_gated_ffn_backward_workspace_bytes(M, D, F))


def atb_gated_ffn_backward(dY, X, Wg, Wu, Wd, H, G, U, act="silu", dX=None, dWg=None, dWu=None, dWd=None, workspace=None, stream=None):
    """Gradients ``(dX, dWg, dWu, dWd)`` of ``atb_gated_ffn`` from ``dY`` and the ``H``, ``G``, ``U`` that it saved."""
    import torch
    M, D, F, ldx, ldw, ldwd, device = _ffn_shapes(X, Wg, Wu, Wd)
    bf16 = torch.bfloat16
    lddy = _matrix(dY, M, D, bf16, device, "dY")
    for t, name in ((H, "H"), (G, "G"), (U, "U")):
        if _matrix(t, M, F, bf16, device, name) != F:
            raise ValueError(f"{name}: contiguous")
    dX, lddx = _out_matrix(dX, X, M, D, bf16, device, "dX")
    dWg, lddw = _out_matrix(dWg, Wg, D, F, bf16, device, "dWg")
    dWu, lddu = _out_matrix(dWu, Wu, D, F, bf16, device, "dWu")
    dWd, lddwd = _out_matrix(dWd, Wd, F, D, bf16, device, "dWd")
    if lddu != lddw:
        raise ValueError("dWg and dWu need the same row stride")
    lib = load_library()
    ws, ws_bytes, workspace = _workspace(workspace, lib.atb_gated_ffn_backward_workspace_bytes(M, D, F), X)
    _check(lib.atb_gated_ffn_backward(M, D, F, _act(act), dY.data_ptr(), lddy, X.data_ptr(), ldx, Wg.data_ptr(), Wu.data_ptr(), ldw,
                                      Wd.data_ptr(), ldwd, H.data_ptr(), G.data_ptr(), U.data_ptr(), dX.data_ptr(), lddx, dWg.data_ptr(),
                                      dWu.data_ptr(), lddw, dWd.data_ptr(), lddwd, ws, ws_bytes, _stream_ptr(stream)))
    return dX, dWg, dWu, dWd


def _head_shapes(X, W, labels):
    import torch
    device = _device_of(X, "X")
    (M, D), V = X.shape, W.shape[0]
    ldx, ldw = _matrix(X, M, D, torch.bfloat16, device, "X"), _matrix(W, V, D, torch.bfloat16, device, "W")
    _vector(labels, M, torch.int64, device, "labels")
    return M, V, D, ldx, ldw, device


def atb_linear_cross_entropy_workspace_bytes(M: int, V: int, D: int) -> int:
    return int(load_library().atb_linear_cross_entropy_workspace_bytes(M, V, D))


def atb_linear_cross_entropy(X, W, labels, ignore_index=-100, loss=None, lse=None, workspace=None, stream=None):
    """Cross entropy of the logits ``X W^T`` (bfloat16 ``X [M, D]``, ``W [V, D]``, int64 ``labels [M]``), which are not kept.

    Returns float32 ``(loss, lse)``, ``[M]`` each; rows whose label is ``ignore_index`` have loss 0."""
    import torch
    M, V, D, ldx, ldw, device = _head_shapes(X, W, labels)
    loss = _out_vector(loss, X, M, torch.float32, device, "loss")
    lse = _out_vector(lse, loss, M, torch.float32, device, "lse")
    lib = load_library()
    ws, ws_bytes, workspace = _workspace(workspace, lib.atb_linear_cross_entropy_workspace_bytes(M, V, D), X)
    _check(lib.atb_linear_cross_entropy(M, V, D, X.data_ptr(), ldx, W.data_ptr(), ldw, labels.data_ptr(), ignore_index, loss.data_ptr(),
                                        lse.data_ptr(), ws, ws_bytes, _stream_ptr(stream)))
    return loss, lse


def atb_linear_cross_entropy_backward_workspace_bytes(M: int, V: int, D: int, piece: int = 0) -> int:
    return int(load_library().atb_linear_cross_entropy_backward_workspace_bytes(M, V, D, piece))


def atb_linear_cross_entropy_backward(dloss, X, W, labels, lse, ignore_index=-100, dX=None, dW=None, piece=0, workspace=None, stream=None):
    """Gradients ``(dX, dW)`` (bfloat16) of ``sum(dloss * loss)``; ``piece``: words of the vocabulary per pass (0: chosen)."""
    import torch
    M, V, D, ldx, ldw, device = _head_shapes(X, W, labels)
    _vector(dloss, M, torch.float32, device, "dloss")
    _vector(lse, M, torch.float32, device, "lse")
    dX, lddx = _out_matrix(dX, X, M, D, torch.bfloat16, device, "dX")
    dW, lddw = _out_matrix(dW, W, V, D, torch.bfloat16, device, "dW")
    lib = load_library()
    ws, ws_bytes, workspace = _workspace(workspace, lib.atb_linear_cross_entropy_backward_workspace_bytes(M, V, D, piece), X)
    _check(lib.atb_linear_cross_entropy_backward(M, V, D, X.data_ptr(), ldx, W.data_ptr(), ldw, labels.data_ptr(), ignore_index,
                                                 lse.data_ptr(), dloss.data_ptr(), dX.data_ptr(), lddx, dW.data_ptr(), lddw, piece, ws, ws_bytes,
                                                 _stream_ptr(stream)))
    return dX, dW


# ------------------------------------------------------------------ layout helpers (no arithmetic)
def exp_plane_to_logical(exp_plane, M: int, K: int):
    """Device exponent plane ``[ceil(K/64)][roundup(M,32)][8]`` -> logical ``[M][K/8]`` (numpy)."""
    import numpy as np
    e = np.asarray(exp_plane, dtype=np.uint8).reshape(-1)
    panels, m_pad = -(-K // 64), -(-M // 32) * 32
    e = e.reshape(panels, m_pad, 8).transpose(1, 0, 2).reshape(m_pad, panels * 8)
    return np.ascontiguousarray(e[:M, :K // 8])


def logical_to_exp_plane(exp_logical, M: int, K: int):
    """Logical ``[M][K/8]`` exponents -> flat device plane (numpy uint8, padding zero)."""
    import numpy as np
    panels, m_pad = -(-K // 64), -(-M // 32) * 32
    full = np.zeros((m_pad, panels * 8), np.uint8)
    full[:M, :K // 8] = np.asarray(exp_logical, dtype=np.uint8)
    return np.ascontiguousarray(full.reshape(m_pad, panels, 8).transpose(1, 0, 2)).reshape(-1)
