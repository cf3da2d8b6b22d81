"""Python binding of libkashin (include/kashin.h).

Argument marshalling only: device memory comes from PyTorch tensors, streams
from ``torch.cuda``; every step of the decomposition, coding, transform and
reconstruction runs in the library's CUDA kernels.  Importing this module loads
``libkashin.so`` from this package directory and raises ``ImportError`` if it is
missing -- there is no fallback implementation.

Two layers:

* ``kd_*`` functions mirror the C entry points one to one (raw device pointers
  as Python ints, a status code back);
* tensor-level wrappers take and return torch tensors: ``decompose`` (and
  ``decompose_batch``, ``decompose_batch_host``), ``apply_p`` (``apply_p_batch``,
  ``prepare_p`` + ``apply_p_prepared``), ``reconstruct`` (``reconstruct_batch``),
  ``dequantise`` (``dequantise_batch``), ``rht``, and the products from the 2-bit
  planes ``matmul_2bit`` (fp32) and ``matmul_2bit_f16`` (fp16 or bf16 activations,
  tensor cores), each with a ``_batch`` form; and the serving operators around them,
  ``rmsnorm`` (residual addition, 8-bit output), ``quantise_4bit`` / ``dequantise_4bit`` /
  ``matmul_4bit`` (4-bit weights with group scales) and ``token_logprobs``.

A wrapper's ``stream`` (the current one without it) is where its work goes and whose memory its
own outputs and scratch are.  As with any work on a second stream the caller has the inputs
ready there, and keeps them, and tensors given as ``out``, until that work is done.
"""

from __future__ import annotations

import ctypes
import dataclasses
import functools
import os
from typing import Optional

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libkashin.so")

KD_OK, KD_ERR_INVALID_ARG, KD_ERR_UNSUPPORTED_N, KD_ERR_CUDA, KD_ERR_NONFINITE, KD_ERR_WORKSPACE, KD_ERR_TIMEOUT = range(7)
KD_F32, KD_F16, KD_BF16, KD_E4M3 = 0, 1, 2, 3
KD_VEC_ROWS, KD_VEC_COLUMNS = 0, 1

EXPORTS = ("kd_status_string", "kd_version", "kd_supported", "kd_tuned", "kd_workspace_size", "kd_signs",
           "kd_decompose", "kd_apply_p", "kd_reconstruct", "kd_read_status", "kd_decompose_static",
           "kd_read_status_static", "kd_staging_size_host", "kd_decompose_batch_host",
           "kd_matmul_2bit", "kd_matmul_2bit_batch", "kd_matmul_2bit_f16", "kd_matmul_2bit_f16_batch",
           "kd_matmul_2bit_bf16", "kd_matmul_2bit_bf16_batch",
           "kd_apply_p_batch", "kd_prepare_p", "kd_apply_p_prepared",
           "kd_rht_block", "kd_rht", "kd_dequantise", "kd_dequantise_batch", "kd_measure_fp32_peak",
           "kd_workspace_size_batch", "kd_decompose_batch", "kd_reconstruct_batch",
           "kd_rmsnorm", "kd_quantise_4bit", "kd_dequantise_4bit", "kd_matmul_4bit", "kd_token_logprobs")
KD_MAX_BATCH = 32
KD_MAX_TOP = 32


class KdPlane(ctypes.Structure):
    """kd_plane: one 2-bit code plane to expand (kd_dequantise_batch)."""
    _fields_ = [("codes", ctypes.c_void_p), ("centres", ctypes.c_void_p), ("out", ctypes.c_void_p),
                ("m", ctypes.c_int64), ("ld", ctypes.c_int64)]


class KdRecMat(ctypes.Structure):
    """kd_recmat: one matrix to re-materialise (kd_reconstruct_batch)."""
    _fields_ = [("codes_u", ctypes.c_void_p), ("codes_v", ctypes.c_void_p), ("centres_u", ctypes.c_void_p),
                ("centres_v", ctypes.c_void_p), ("sign_seed", ctypes.c_uint64), ("w_hat", ctypes.c_void_p),
                ("m", ctypes.c_int64), ("ld", ctypes.c_int64)]


class KdPMat(ctypes.Structure):
    """Mirror of kd_pmat (include/kashin.h): rows x -> y = P x with one sign seed."""
    _fields_ = [("x", ctypes.c_void_p), ("y", ctypes.c_void_p), ("m", ctypes.c_int64), ("sign_seed", ctypes.c_uint64)]


class KdFoldMat(ctypes.Structure):
    """Mirror of kd_fold_mat (include/kashin.h): one matrix of kd_matmul_2bit_batch."""
    _fields_ = [("codes_u", ctypes.c_void_p), ("codes_v", ctypes.c_void_p), ("centres_u", ctypes.c_void_p),
                ("centres_v", ctypes.c_void_p), ("x", ctypes.c_void_p), ("xp", ctypes.c_void_p),
                ("y", ctypes.c_void_p), ("n", ctypes.c_int64), ("m", ctypes.c_int64), ("ldx", ctypes.c_int64),
                ("ldy", ctypes.c_int64)]


class KdFoldMatF16(ctypes.Structure):
    """Mirror of kd_fold_mat_f16 (include/kashin.h): one matrix of kd_matmul_2bit_f16_batch."""
    _fields_ = KdFoldMat._fields_


class KdMatrixHost(ctypes.Structure):
    """Mirror of kd_matrix_host (include/kashin.h): every pointer is host memory."""
    _fields_ = [("w", ctypes.c_void_p), ("m", ctypes.c_int64), ("ld", ctypes.c_int64),
                ("sign_seed", ctypes.c_uint64), ("codes_u", ctypes.c_void_p), ("codes_v", ctypes.c_void_p),
                ("centres_u", ctypes.c_void_p), ("centres_v", ctypes.c_void_p), ("coeffs", ctypes.c_void_p)]


class KdMatrix(ctypes.Structure):
    """Mirror of kd_matrix (include/kashin.h)."""
    _fields_ = [("w", ctypes.c_void_p), ("m", ctypes.c_int64), ("ld", ctypes.c_int64),
                ("sign_seed", ctypes.c_uint64), ("codes_u", ctypes.c_void_p), ("codes_v", ctypes.c_void_p),
                ("centres_u", ctypes.c_void_p), ("centres_v", ctypes.c_void_p), ("coeffs", ctypes.c_void_p)]


class KdWeight4(ctypes.Structure):
    """Mirror of kd_weight4 (include/kashin.h)."""
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("zeros", ctypes.c_void_p),
                ("n", ctypes.c_int64), ("m", ctypes.c_int64), ("group", ctypes.c_int32),
                ("scale_dtype", ctypes.c_int32)]


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run paper_2609_11687_gb300.build.build() "
                          "(the CUDA library is required, there is no CPU fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    c_i64, c_u64, c_int, c_vp, c_sz = ctypes.c_int64, ctypes.c_uint64, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
    lib.kd_status_string.argtypes = [c_int]
    lib.kd_status_string.restype = ctypes.c_char_p
    lib.kd_version.argtypes = []
    lib.kd_version.restype = ctypes.c_char_p
    lib.kd_supported.argtypes = [c_i64]
    lib.kd_supported.restype = c_int
    lib.kd_tuned.argtypes = [c_i64]
    lib.kd_tuned.restype = c_int
    lib.kd_workspace_size.argtypes = [c_i64]
    lib.kd_workspace_size.restype = c_sz
    lib.kd_signs.argtypes = [c_u64, c_i64, c_vp]
    lib.kd_signs.restype = c_int
    lib.kd_decompose.argtypes = [c_vp, c_int, c_int, c_i64, c_i64, c_i64, c_u64, c_int, c_int,
                                 c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_sz, c_vp]
    lib.kd_decompose.restype = c_int
    lib.kd_apply_p.argtypes = [c_vp, c_vp, c_i64, c_i64, c_u64, c_vp, c_sz, c_vp]
    lib.kd_apply_p.restype = c_int
    lib.kd_reconstruct.argtypes = [c_vp, c_vp, c_vp, c_vp, c_i64, c_i64, c_u64, c_int, c_int, c_vp,
                                   c_i64, c_vp, c_sz, c_vp]
    lib.kd_reconstruct.restype = c_int
    lib.kd_read_status.argtypes = [c_vp, c_vp]
    lib.kd_read_status.restype = c_int
    lib.kd_decompose_static.argtypes = [c_vp, c_int, c_int, c_i64, c_i64, c_i64, c_u64, c_int, c_int,
                                        c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp]
    lib.kd_decompose_static.restype = c_int
    lib.kd_read_status_static.argtypes = [c_vp]
    lib.kd_read_status_static.restype = c_int
    lib.kd_staging_size_host.argtypes = [c_vp, c_int, c_int, c_int, c_i64]
    lib.kd_staging_size_host.restype = c_sz
    lib.kd_decompose_batch_host.argtypes = [c_vp, c_int, c_int, c_int, c_i64, c_int, c_int, c_vp, c_sz, c_vp,
                                            c_sz, c_vp]
    lib.kd_decompose_batch_host.restype = c_int
    lib.kd_matmul_2bit.argtypes = [c_vp, c_vp, c_vp, c_vp, c_i64, c_i64, c_vp, c_vp, c_i64, c_i64, c_vp, c_i64, c_vp]
    lib.kd_matmul_2bit.restype = c_int
    lib.kd_matmul_2bit_batch.argtypes = [c_vp, c_int, c_i64, c_vp]
    lib.kd_matmul_2bit_batch.restype = c_int
    lib.kd_prepare_p.argtypes = [c_vp, c_int, c_i64, c_vp, ctypes.c_size_t, c_vp]
    lib.kd_prepare_p.restype = c_int
    lib.kd_apply_p_prepared.argtypes = [c_vp, c_int, c_i64, c_vp, ctypes.c_size_t, c_vp]
    lib.kd_apply_p_prepared.restype = c_int
    lib.kd_matmul_2bit_f16.argtypes = [c_vp, c_vp, c_vp, c_vp, c_i64, c_i64, c_vp, c_vp, c_i64, c_i64, c_vp, c_i64,
                                       c_vp]
    lib.kd_matmul_2bit_f16.restype = c_int
    lib.kd_matmul_2bit_f16_batch.argtypes = [c_vp, c_int, c_i64, c_vp]
    lib.kd_matmul_2bit_f16_batch.restype = c_int
    lib.kd_matmul_2bit_bf16.argtypes = lib.kd_matmul_2bit_f16.argtypes
    lib.kd_matmul_2bit_bf16.restype = c_int
    lib.kd_matmul_2bit_bf16_batch.argtypes = [c_vp, c_int, c_i64, c_vp]
    lib.kd_matmul_2bit_bf16_batch.restype = c_int
    lib.kd_apply_p_batch.argtypes = [c_vp, c_int, c_i64, c_vp, c_sz, c_vp]
    lib.kd_apply_p_batch.restype = c_int
    lib.kd_workspace_size_batch.argtypes = [c_i64, c_int]
    lib.kd_workspace_size_batch.restype = c_sz
    lib.kd_decompose_batch.argtypes = [c_vp, c_int, c_int, c_int, c_i64, c_int, c_int, c_vp, c_sz, c_vp]
    lib.kd_decompose_batch.restype = c_int
    lib.kd_reconstruct_batch.argtypes = [c_vp, c_int, c_i64, c_int, c_int, c_vp, c_sz, c_vp]
    lib.kd_reconstruct_batch.restype = c_int
    lib.kd_measure_fp32_peak.argtypes = [c_vp, c_vp]
    lib.kd_measure_fp32_peak.restype = c_int
    lib.kd_dequantise.argtypes = [c_vp, c_vp, c_i64, c_i64, c_int, c_int, c_vp, c_i64, c_vp]
    lib.kd_dequantise.restype = c_int
    lib.kd_dequantise_batch.argtypes = [c_vp, c_int, c_i64, c_int, c_int, c_vp]
    lib.kd_dequantise_batch.restype = c_int
    lib.kd_rht_block.argtypes = [c_i64]
    lib.kd_rht_block.restype = c_i64
    lib.kd_rht.argtypes = [c_vp, c_int, c_i64, c_i64, c_i64, c_u64, c_int, c_vp, c_i64, c_vp, c_vp]
    lib.kd_rht.restype = c_int
    lib.kd_rmsnorm.argtypes = [c_vp, c_int, c_i64, c_i64, c_i64, c_vp, c_int, ctypes.c_float, c_vp, c_i64, c_vp, c_i64,
                               c_vp, c_i64, c_vp, c_vp, c_int, c_i64, c_vp]
    lib.kd_rmsnorm.restype = c_int
    lib.kd_quantise_4bit.argtypes = [c_vp, c_int, c_i64, c_vp, c_vp]
    lib.kd_quantise_4bit.restype = c_int
    lib.kd_dequantise_4bit.argtypes = [c_vp, c_int, c_vp, c_i64, c_vp]
    lib.kd_dequantise_4bit.restype = c_int
    lib.kd_matmul_4bit.argtypes = [c_vp, c_vp, c_int, c_vp, c_i64, c_i64, c_vp, c_int, c_i64, c_vp]
    lib.kd_matmul_4bit.restype = c_int
    lib.kd_token_logprobs.argtypes = [c_vp, c_int, c_i64, c_i64, c_i64, c_vp, c_i64, c_int, c_vp, c_vp, c_vp, c_vp,
                                      c_vp, c_vp]
    lib.kd_token_logprobs.restype = c_int
    return lib


lib = _load()


class KashinError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_string(status)}")


def status_string(s: int) -> str:
    return lib.kd_status_string(int(s)).decode()


def version() -> str:
    return lib.kd_version().decode()


# ---------------------------------------------------------------------------
# one-to-one mirrors of the C entry points
# ---------------------------------------------------------------------------

def kd_supported(n: int) -> int:
    return lib.kd_supported(int(n))


def kd_tuned(n: int) -> bool:
    return bool(lib.kd_tuned(int(n)))


def kd_workspace_size(n: int) -> int:
    return int(lib.kd_workspace_size(int(n)))


def kd_signs(sign_seed: int, n: int) -> np.ndarray:
    out = np.empty(int(n), dtype=np.int8)
    st = lib.kd_signs(ctypes.c_uint64(int(sign_seed) & ((1 << 64) - 1)), int(n), out.ctypes.data)
    if st != KD_OK:
        raise KashinError(st, "kd_signs")
    return out


def kd_decompose(w, dtype, layout, n, m, ld, sign_seed, iters, kmeans_iters, codes_u, codes_v, centres_u,
                 centres_v, coeffs, u, vhat, resid, trace, workspace, ws_bytes, stream) -> int:
    return lib.kd_decompose(w, dtype, layout, n, m, ld, ctypes.c_uint64(int(sign_seed) & ((1 << 64) - 1)),
                            iters, kmeans_iters, codes_u, codes_v, centres_u, centres_v, coeffs, u, vhat, resid,
                            trace, workspace, ws_bytes, stream)


def kd_apply_p(x, y, n, m, sign_seed, workspace, ws_bytes, stream) -> int:
    return lib.kd_apply_p(x, y, n, m, ctypes.c_uint64(int(sign_seed) & ((1 << 64) - 1)), workspace, ws_bytes,
                          stream)


def kd_reconstruct(codes_u, codes_v, centres_u, centres_v, n, m, sign_seed, out_dtype, layout, w_hat, ld,
                   workspace, ws_bytes, stream) -> int:
    return lib.kd_reconstruct(codes_u, codes_v, centres_u, centres_v, n, m,
                              ctypes.c_uint64(int(sign_seed) & ((1 << 64) - 1)), out_dtype, layout, w_hat, ld,
                              workspace, ws_bytes, stream)


def kd_batchable(n: int) -> bool:
    """True when kd_decompose_batch runs all matrices of length n in one launch
    (tuned lengths n <= 8192, as include/kashin.h states); longer vectors and the
    run-time-length path run one launch each."""
    return kd_tuned(n) and int(n) <= 8192


def kd_workspace_size_batch(n: int, count: int) -> int:
    return int(lib.kd_workspace_size_batch(int(n), int(count)))


def kd_decompose_batch(mats, count, dtype, layout, n, iters, kmeans_iters, workspace, ws_bytes, stream) -> int:
    return lib.kd_decompose_batch(mats, count, dtype, layout, n, iters, kmeans_iters, workspace, ws_bytes, stream)


def kd_reconstruct_batch(mats, count, n, out_dtype, layout, workspace, ws_bytes, stream) -> int:
    return lib.kd_reconstruct_batch(mats, count, n, out_dtype, layout, workspace, ws_bytes, stream)


def kd_read_status(workspace, stream) -> int:
    return lib.kd_read_status(workspace, stream)


def kd_decompose_static(w, dtype, layout, n, m, ld, sign_seed, iters, kmeans_iters, codes_u, codes_v, centres_u,
                        centres_v, coeffs, u, vhat, resid, trace, stream) -> int:
    return lib.kd_decompose_static(w, dtype, layout, n, m, ld, ctypes.c_uint64(int(sign_seed) & ((1 << 64) - 1)),
                                   iters, kmeans_iters, codes_u, codes_v, centres_u, centres_v, coeffs, u, vhat,
                                   resid, trace, stream)


def kd_read_status_static(stream) -> int:
    return lib.kd_read_status_static(stream)


def kd_staging_size_host(mats, count, dtype, layout, n) -> int:
    return int(lib.kd_staging_size_host(mats, count, dtype, layout, n))


def kd_decompose_batch_host(mats, count, dtype, layout, n, iters, kmeans_iters, staging, staging_bytes, workspace,
                            ws_bytes, stream) -> int:
    return lib.kd_decompose_batch_host(mats, count, dtype, layout, n, iters, kmeans_iters, staging, staging_bytes,
                                       workspace, ws_bytes, stream)


def kd_dequantise(codes, centres, n, m, out_dtype, layout, out, ld, stream) -> int:
    return lib.kd_dequantise(codes, centres, n, m, out_dtype, layout, out, ld, stream)


def kd_dequantise_batch(planes, count, n, out_dtype, layout, stream) -> int:
    return lib.kd_dequantise_batch(planes, count, n, out_dtype, layout, stream)


def measure_fp32_peak(stream=None) -> float:
    """Measured FP32 TFLOP/s of the current device (packed FFMA chains)."""
    out = ctypes.c_double(0.0)
    st = lib.kd_measure_fp32_peak(ctypes.byref(out), _stream(stream))
    if st != KD_OK:
        raise KashinError(st, "kd_measure_fp32_peak")
    return out.value


def kd_rht_block(n) -> int:
    return int(lib.kd_rht_block(int(n)))


def kd_rht(x, dtype, n, m, ldx, seed, inverse, y, ldy, status, stream) -> int:
    return lib.kd_rht(x, dtype, n, m, ldx, ctypes.c_uint64(int(seed) & ((1 << 64) - 1)), inverse, y, ldy, status,
                      stream)


def kd_rmsnorm(x, dtype, n, rows, ldx, weight, weight_dtype, eps, residual, ld_residual, new_residual,
               ld_new_residual, q, ldq, scale, y, y_dtype, ldy, stream) -> int:
    return lib.kd_rmsnorm(x, dtype, n, rows, ldx, weight, weight_dtype, eps, residual, ld_residual, new_residual,
                          ld_new_residual, q, ldq, scale, y, y_dtype, ldy, stream)


def kd_quantise_4bit(w, dtype, ld, out, stream) -> int:
    return lib.kd_quantise_4bit(w, dtype, ld, out, stream)


def kd_dequantise_4bit(w, out_dtype, out, ld, stream) -> int:
    return lib.kd_dequantise_4bit(w, out_dtype, out, ld, stream)


def kd_matmul_4bit(w, x, x_dtype, x_scale, rows, ldx, y, y_dtype, ldy, stream) -> int:
    return lib.kd_matmul_4bit(w, x, x_dtype, x_scale, rows, ldx, y, y_dtype, ldy, stream)


def kd_token_logprobs(logits, dtype, rows, vocab, ld, ids, tokens, top, logprobs, lse, entropy, top_ids, top_logprobs,
                      stream) -> int:
    return lib.kd_token_logprobs(logits, dtype, rows, vocab, ld, ids, tokens, top, logprobs, lse, entropy, top_ids,
                                 top_logprobs, stream)


# ---------------------------------------------------------------------------
# torch-tensor wrappers
# ---------------------------------------------------------------------------

def _torch():
    import torch
    return torch


def _dtype_code(t) -> int:
    torch = _torch()
    m = {torch.float32: KD_F32, torch.float16: KD_F16, torch.bfloat16: KD_BF16}
    if t not in m:
        raise TypeError(f"unsupported dtype {t}")
    return m[t]


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _ld(t) -> int:
    """Row stride of a 2-D tensor for the C ABI: a single row's stride is never used, so
    report its length (torch and numpy may give a one-row tensor any row stride)."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _stream(stream) -> int:
    torch = _torch()
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def _new(stream, shape, dtype, device):
    """An output allocated here for work on ``stream`` (None: the current one).  The block comes
    from that stream's own pool: one of the current stream's may have been freed with work
    still pending there, which ``stream`` does not wait for.  The caller's stream is noted, so
    that a result dropped there is not given out again before it has been read."""
    torch = _torch()
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if hasattr(stream, "cuda_stream") and not hasattr(stream, "device"):  # a holder of a bare handle
        stream = torch.cuda.ExternalStream(stream.cuda_stream, device=device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    current = torch.cuda.current_stream(device)
    if current != stream:
        t.record_stream(current)
    return t


class Workspace:
    """Device scratch for one vector length (reusable across calls on one stream, ``stream`` or
    the current one)."""

    def __init__(self, n: int, device="cuda", count: int = 1, stream=None):
        torch = _torch()
        self.n = int(n)
        self.count = int(count)
        size = kd_workspace_size(self.n) if self.count == 1 else kd_workspace_size_batch(self.n, self.count)
        if size == 0:
            raise KashinError(KD_ERR_UNSUPPORTED_N if kd_supported(self.n) else KD_ERR_CUDA,
                              f"kd_workspace_size({self.n})")
        self.nbytes = size
        self.buf = _new(stream, (size,), torch.uint8, device)

    @property
    def ptr(self) -> int:
        return self.buf.data_ptr()


@dataclasses.dataclass
class Decomposed:
    codes_u: "object"     # int32 view of uint32 words, (m, ceil(n/16))
    codes_v: "object"
    centres_u: "object"   # float32 (m, 4)
    centres_v: "object"
    coeffs: "object"      # float32 (m, 4) or None
    u: "object"           # float32 (m, n) or None
    vhat: "object"
    resid: "object"
    trace: "object"       # int8 (m, 4*iters + 2*kmeans_iters, n) or None


def decompose(w, iters: int, sign_seed: int, layout: str = "rows", factors: bool = False,
              coeffs: bool = True, trace: bool = False, workspace: Optional[Workspace] = None,
              out: Optional[Decomposed] = None, stream=None, kmeans_iters: int = 0) -> Decomposed:
    """Decompose every vector of ``w`` (Alg. 1) and 2-bit code both factors
    (closed-form centres, then ``kmeans_iters`` Lloyd refinement iterations).

    ``layout='rows'``: ``w`` is (m, n), vector j = ``w[j]`` (nn.Linear weight).
    ``layout='columns'``: ``w`` is (n, m), vector j = ``w[:, j]`` (the paper's W).
    """
    torch = _torch()
    if not w.is_cuda:
        raise ValueError("w must be a CUDA tensor")
    if w.dim() != 2 or w.stride(1) != 1:
        raise ValueError("w must be 2-D with unit inner stride")
    lay = KD_VEC_ROWS if layout == "rows" else KD_VEC_COLUMNS
    if lay == KD_VEC_ROWS:
        m, n = w.shape
    else:
        n, m = w.shape
    ld = _ld(w)
    dev = w.device
    words = (n + 15) // 16
    if out is None:
        def empty(shape, dtype=torch.float32):
            return _new(stream, shape, dtype, dev)
        out = Decomposed(
            codes_u=empty((m, words), torch.int32), codes_v=empty((m, words), torch.int32),
            centres_u=empty((m, 4)), centres_v=empty((m, 4)),
            coeffs=empty((m, 4)) if coeffs else None,
            u=empty((m, n)) if factors else None,
            vhat=empty((m, n)) if factors else None,
            resid=empty((m, n)) if factors else None,
            trace=empty((m, 4 * iters + 2 * kmeans_iters, n), torch.int8) if trace else None)
    ws = workspace if workspace is not None else Workspace(n, dev, stream=stream)
    st = kd_decompose(w.data_ptr(), _dtype_code(w.dtype), lay, n, m, ld, sign_seed, int(iters), int(kmeans_iters),
                      _ptr(out.codes_u), _ptr(out.codes_v), _ptr(out.centres_u), _ptr(out.centres_v),
                      _ptr(out.coeffs), _ptr(out.u), _ptr(out.vhat), _ptr(out.resid), _ptr(out.trace),
                      ws.ptr, ws.nbytes, _stream(stream))
    if st != KD_OK:
        raise KashinError(st, "kd_decompose")
    return out


def decompose_batch(ws, iters: int, sign_seeds, layout: str = "rows", coeffs: bool = False,
                    workspace: Optional[Workspace] = None, outs=None, stream=None, kmeans_iters: int = 0):
    """Decompose and code several matrices of one vector length in one launch
    (kd_decompose_batch): ``ws`` is a list of up to KD_MAX_BATCH CUDA tensors of one
    dtype and layout, ``sign_seeds`` their seeds.  Returns one Decomposed per matrix
    (no factor or trace outputs)."""
    torch = _torch()
    if not 1 <= len(ws) <= KD_MAX_BATCH or len(sign_seeds) != len(ws):
        raise ValueError(f"1..{KD_MAX_BATCH} matrices with one seed each")
    lay = KD_VEC_ROWS if layout == "rows" else KD_VEC_COLUMNS
    n = ws[0].shape[1] if lay == KD_VEC_ROWS else ws[0].shape[0]
    dt = ws[0].dtype
    arr = (KdMatrix * len(ws))()
    res = []
    for i, w in enumerate(ws):
        if not w.is_cuda or w.dim() != 2 or w.stride(1) != 1 or w.dtype != dt:
            raise ValueError("matrices must be 2-D CUDA tensors of one dtype with unit inner stride")
        m = w.shape[0] if lay == KD_VEC_ROWS else w.shape[1]
        if (w.shape[1] if lay == KD_VEC_ROWS else w.shape[0]) != n:
            raise ValueError("matrices must share the vector length")
        if outs is not None:
            o = outs[i]
        else:
            def empty(shape, dtype=torch.float32):
                return _new(stream, shape, dtype, w.device)
            o = Decomposed(codes_u=empty((m, (n + 15) // 16), torch.int32),
                           codes_v=empty((m, (n + 15) // 16), torch.int32),
                           centres_u=empty((m, 4)), centres_v=empty((m, 4)),
                           coeffs=empty((m, 4)) if coeffs else None,
                           u=None, vhat=None, resid=None, trace=None)
        arr[i] = KdMatrix(w.data_ptr(), m, _ld(w), int(sign_seeds[i]) & ((1 << 64) - 1),
                          _ptr(o.codes_u), _ptr(o.codes_v), _ptr(o.centres_u), _ptr(o.centres_v), _ptr(o.coeffs))
        res.append(o)
    wsp = workspace if workspace is not None else Workspace(n, ws[0].device, count=len(ws), stream=stream)
    st = kd_decompose_batch(ctypes.cast(arr, ctypes.c_void_p), len(ws), _dtype_code(dt), lay, n, int(iters),
                            int(kmeans_iters), wsp.ptr, wsp.nbytes, _stream(stream))
    if st != KD_OK:
        raise KashinError(st, "kd_decompose_batch")
    return res


def kd_matmul_2bit(codes_u, codes_v, centres_u, centres_v, n, m, x, xp, batch, ldx, y, ldy, stream) -> int:
    return lib.kd_matmul_2bit(codes_u, codes_v, centres_u, centres_v, n, m, x, xp, batch, ldx, y, ldy, stream)


def matmul_2bit(dec: "Decomposed", x, xp, out=None, stream=None):
    """``Y = X W_hat^T`` from the code planes (App. C): ``x`` and ``xp`` (= apply_p of the
    rows of x with the matrix's sign seed) are fp32 CUDA tensors (batch, n); returns
    (batch, m) fp32."""
    torch = _torch()
    m, words = dec.codes_u.shape
    if x.dim() != 2 or x.dtype != torch.float32 or xp.shape != x.shape or xp.dtype != x.dtype:
        raise ValueError("x and xp must be fp32 (batch, n) tensors of one shape")
    if x.stride(1) != 1 or xp.stride(1) != 1 or _ld(x) != _ld(xp):
        raise ValueError("x and xp need unit inner stride and equal row strides")
    b, n = x.shape
    if (n + 15) // 16 != words:
        raise ValueError("x does not match the code planes' vector length")
    y = out if out is not None else _new(stream, (b, m), torch.float32, x.device)
    st = kd_matmul_2bit(dec.codes_u.data_ptr(), dec.codes_v.data_ptr(), dec.centres_u.data_ptr(),
                        dec.centres_v.data_ptr(), n, m, x.data_ptr(), xp.data_ptr(), b, _ld(x), y.data_ptr(),
                        _ld(y), _stream(stream))
    if st != KD_OK:
        raise KashinError(st, "kd_matmul_2bit")
    return y


def kd_matmul_2bit_batch(mats, count, batch, stream) -> int:
    return lib.kd_matmul_2bit_batch(mats, count, batch, stream)


def kd_matmul_2bit_f16(codes_u, codes_v, centres_u, centres_v, n, m, x, xp, batch, ldx, y, ldy, stream) -> int:
    return lib.kd_matmul_2bit_f16(codes_u, codes_v, centres_u, centres_v, n, m, x, xp, batch, ldx, y, ldy, stream)


def kd_matmul_2bit_f16_batch(mats, count, batch, stream) -> int:
    return lib.kd_matmul_2bit_f16_batch(mats, count, batch, stream)


def kd_matmul_2bit_bf16(codes_u, codes_v, centres_u, centres_v, n, m, x, xp, batch, ldx, y, ldy, stream) -> int:
    return lib.kd_matmul_2bit_bf16(codes_u, codes_v, centres_u, centres_v, n, m, x, xp, batch, ldx, y, ldy, stream)


def kd_matmul_2bit_bf16_batch(mats, count, batch, stream) -> int:
    return lib.kd_matmul_2bit_bf16_batch(mats, count, batch, stream)


def matmul_2bit_f16(dec: "Decomposed", x, xp, out=None, stream=None):
    """kd_matmul_2bit_f16 (or _bf16): ``Y = X W_hat^T`` from the code planes on the tensor
    cores, for fp16 (or bf16) ``x`` and ``xp`` (batch, n) CUDA tensors; returns (batch, m) fp32."""
    return matmul_2bit_f16_batch([dec], [x], [xp], outs=None if out is None else [out], stream=stream)[0]


def matmul_2bit_f16_batch(decs, xs, xps, outs=None, stream=None):
    """kd_matmul_2bit_f16_batch (or _bf16_batch, for bf16 inputs): ``Y_i = X_i W_hat_i^T``
    for several matrices, 16-bit inputs of one type and batch size, one launch per 16 rows."""
    torch = _torch()
    dt = xs[0].dtype
    if dt not in (torch.float16, torch.bfloat16):
        raise ValueError("x must be fp16 or bf16")
    if not 1 <= len(decs) <= KD_MAX_BATCH or len(xs) != len(decs) or len(xps) != len(decs):
        raise ValueError(f"1..{KD_MAX_BATCH} matrices with one x and one xp each")
    b = xs[0].shape[0]
    arr = (KdFoldMatF16 * len(decs))()
    res = []
    for i, (d, x, xp) in enumerate(zip(decs, xs, xps)):
        m, words = d.codes_u.shape
        if x.dim() != 2 or x.shape[0] != b or x.dtype != dt or xp.shape != x.shape \
                or xp.dtype != x.dtype or x.stride(1) != 1 or xp.stride(1) != 1 or _ld(x) != _ld(xp):
            raise ValueError("x and xp must be 16-bit (batch, n) tensors of one type and shape, unit inner stride")
        n = x.shape[1]
        if (n + 15) // 16 != words:
            raise ValueError("x does not match the code planes' vector length")
        y = outs[i] if outs is not None else _new(stream, (b, m), torch.float32, x.device)
        arr[i] = KdFoldMatF16(d.codes_u.data_ptr(), d.codes_v.data_ptr(), d.centres_u.data_ptr(),
                              d.centres_v.data_ptr(), x.data_ptr(), xp.data_ptr(), y.data_ptr(), n, m, _ld(x),
                              _ld(y))
        res.append(y)
    call = kd_matmul_2bit_bf16_batch if dt == torch.bfloat16 else kd_matmul_2bit_f16_batch
    st = call(ctypes.cast(arr, ctypes.c_void_p), len(decs), b, _stream(stream))
    if st != KD_OK:
        raise KashinError(st, "kd_matmul_2bit_bf16_batch" if dt == torch.bfloat16 else "kd_matmul_2bit_f16_batch")
    return res


def kd_apply_p_batch(mats, count, n, workspace, ws_bytes, stream) -> int:
    return lib.kd_apply_p_batch(mats, count, n, workspace, ws_bytes, stream)


def matmul_2bit_batch(decs, xs, xps, outs=None, stream=None):
    """kd_matmul_2bit_batch: ``Y_i = X_i W_hat_i^T`` for several matrices in one launch
    (``decs`` Decomposed, ``xs``/``xps`` fp32 (batch, n_i) CUDA tensors, one batch size)."""
    torch = _torch()
    if not 1 <= len(decs) <= KD_MAX_BATCH or len(xs) != len(decs) or len(xps) != len(decs):
        raise ValueError(f"1..{KD_MAX_BATCH} matrices with one x and one xp each")
    b = xs[0].shape[0]
    arr = (KdFoldMat * len(decs))()
    res = []
    for i, (d, x, xp) in enumerate(zip(decs, xs, xps)):
        m, words = d.codes_u.shape
        if x.dim() != 2 or x.shape[0] != b or x.dtype != torch.float32 or xp.shape != x.shape \
                or xp.dtype != x.dtype or x.stride(1) != 1 or xp.stride(1) != 1 or _ld(x) != _ld(xp):
            raise ValueError("x and xp must be fp32 (batch, n) tensors of one shape, unit inner stride")
        n = x.shape[1]
        if (n + 15) // 16 != words:
            raise ValueError("x does not match the code planes' vector length")
        y = outs[i] if outs is not None else _new(stream, (b, m), torch.float32, x.device)
        arr[i] = KdFoldMat(d.codes_u.data_ptr(), d.codes_v.data_ptr(), d.centres_u.data_ptr(), d.centres_v.data_ptr(),
                           x.data_ptr(), xp.data_ptr(), y.data_ptr(), n, m, _ld(x), _ld(y))
        res.append(y)
    st = kd_matmul_2bit_batch(ctypes.cast(arr, ctypes.c_void_p), len(decs), b, _stream(stream))
    if st != KD_OK:
        raise KashinError(st, "kd_matmul_2bit_batch")
    return res


def apply_p_batch(xs, sign_seeds, outs=None, workspace: Optional[Workspace] = None, stream=None):
    """kd_apply_p_batch: ``y = P x`` for the rows of several fp32 (m_i, n) tensors, each
    with its own sign seed, in one launch."""
    torch = _torch()
    if not 1 <= len(xs) <= KD_MAX_BATCH or len(sign_seeds) != len(xs):
        raise ValueError(f"1..{KD_MAX_BATCH} matrices with one seed each")
    n = xs[0].shape[1]
    arr = (KdPMat * len(xs))()
    res = []
    for i, x in enumerate(xs):
        if x.dtype != torch.float32 or not x.is_contiguous() or x.dim() != 2 or x.shape[1] != n:
            raise ValueError("inputs must be contiguous fp32 (m, n) CUDA tensors of one n")
        y = outs[i] if outs is not None else _new(stream, x.shape, x.dtype, x.device)
        arr[i] = KdPMat(x.data_ptr(), y.data_ptr(), x.shape[0], int(sign_seeds[i]) & ((1 << 64) - 1))
        res.append(y)
    ws = workspace if workspace is not None else Workspace(n, xs[0].device, count=len(xs), stream=stream)
    st = kd_apply_p_batch(ctypes.cast(arr, ctypes.c_void_p), len(xs), n, ws.ptr, ws.nbytes, _stream(stream))
    if st != KD_OK:
        raise KashinError(st, "kd_apply_p_batch")
    return res


def kd_prepare_p(seeds, count, n, workspace, ws_bytes, stream) -> int:
    return lib.kd_prepare_p(seeds, count, n, workspace, ws_bytes, stream)


def kd_apply_p_prepared(mats, count, n, workspace, ws_bytes, stream) -> int:
    return lib.kd_apply_p_prepared(mats, count, n, workspace, ws_bytes, stream)


def prepare_p(n: int, sign_seeds, workspace: Optional[Workspace] = None, device="cuda", stream=None) -> Workspace:
    """kd_prepare_p: P's twiddle table and the sign sets of ``sign_seeds`` written once
    into a workspace (returned) for apply_p_prepared."""
    if not 1 <= len(sign_seeds) <= KD_MAX_BATCH:
        raise ValueError(f"1..{KD_MAX_BATCH} sign seeds")
    ws = workspace if workspace is not None else Workspace(n, device, count=len(sign_seeds), stream=stream)
    seeds = (ctypes.c_uint64 * len(sign_seeds))(*[int(s) & ((1 << 64) - 1) for s in sign_seeds])
    st = kd_prepare_p(ctypes.cast(seeds, ctypes.c_void_p), len(sign_seeds), n, ws.ptr, ws.nbytes, _stream(stream))
    if st != KD_OK:
        raise KashinError(st, "kd_prepare_p")
    return ws


def apply_p_prepared(xs, workspace: Workspace, outs=None, stream=None):
    """kd_apply_p_prepared: ``y_i = P_i x_i`` with the tables prepare_p left in
    ``workspace`` (matrix i takes sign set i)."""
    torch = _torch()
    if not 1 <= len(xs) <= KD_MAX_BATCH:
        raise ValueError(f"1..{KD_MAX_BATCH} matrices")
    n = xs[0].shape[1]
    arr = (KdPMat * len(xs))()
    res = []
    for i, x in enumerate(xs):
        if x.dtype != torch.float32 or not x.is_contiguous() or x.dim() != 2 or x.shape[1] != n:
            raise ValueError("inputs must be contiguous fp32 (m, n) CUDA tensors of one n")
        y = outs[i] if outs is not None else _new(stream, x.shape, x.dtype, x.device)
        arr[i] = KdPMat(x.data_ptr(), y.data_ptr(), x.shape[0], 0)
        res.append(y)
    st = kd_apply_p_prepared(ctypes.cast(arr, ctypes.c_void_p), len(xs), n, workspace.ptr, workspace.nbytes,
                             _stream(stream))
    if st != KD_OK:
        raise KashinError(st, "kd_apply_p_prepared")
    return res


def _host_descriptors(ws, sign_seeds, layout, outs):
    """kd_matrix_host array for host tensors ``ws`` and host outputs ``outs`` (one
    Decomposed of CPU tensors per matrix)."""
    if not 1 <= len(ws) <= KD_MAX_BATCH or len(sign_seeds) != len(ws) or len(outs) != len(ws):
        raise ValueError(f"1..{KD_MAX_BATCH} matrices with one seed and one output set each")
    lay = KD_VEC_ROWS if layout == "rows" else KD_VEC_COLUMNS
    n = ws[0].shape[1] if lay == KD_VEC_ROWS else ws[0].shape[0]
    arr = (KdMatrixHost * len(ws))()
    for i, (w, o) in enumerate(zip(ws, outs)):
        if w.is_cuda or w.dim() != 2 or w.stride(1) != 1 or w.dtype != ws[0].dtype:
            raise ValueError("matrices must be 2-D host tensors of one dtype with unit inner stride")
        m = w.shape[0] if lay == KD_VEC_ROWS else w.shape[1]
        for t in (o.codes_u, o.codes_v, o.centres_u, o.centres_v, o.coeffs):
            if t is not None and t.is_cuda:
                raise ValueError("outputs must be host tensors")
        arr[i] = KdMatrixHost(w.data_ptr(), m, _ld(w), int(sign_seeds[i]) & ((1 << 64) - 1),
                              _ptr(o.codes_u), _ptr(o.codes_v), _ptr(o.centres_u), _ptr(o.centres_v),
                              _ptr(o.coeffs))
    return arr, lay, n


def host_outputs(m: int, n: int, coeffs: bool = False, pin: bool = True) -> Decomposed:
    """Host (pinned) output tensors for one matrix of decompose_batch_host."""
    torch = _torch()
    def mk(shape, dt):
        t = torch.empty(shape, dtype=dt)
        return t.pin_memory() if pin else t
    return Decomposed(codes_u=mk((m, (n + 15) // 16), torch.int32), codes_v=mk((m, (n + 15) // 16), torch.int32),
                      centres_u=mk((m, 4), torch.float32), centres_v=mk((m, 4), torch.float32),
                      coeffs=mk((m, 4), torch.float32) if coeffs else None, u=None, vhat=None, resid=None,
                      trace=None)


def staging_size_host(ws, layout: str = "rows", coeffs: bool = False) -> int:
    """Device staging bytes decompose_batch_host needs for host matrices ``ws``."""
    lay = KD_VEC_ROWS if layout == "rows" else KD_VEC_COLUMNS
    n = ws[0].shape[1] if lay == KD_VEC_ROWS else ws[0].shape[0]
    outs = [host_outputs(w.shape[0] if lay == KD_VEC_ROWS else w.shape[1], n, coeffs, pin=False) for w in ws]
    arr, lay, n = _host_descriptors(ws, [0] * len(ws), layout, outs)
    return kd_staging_size_host(ctypes.cast(arr, ctypes.c_void_p), len(ws), _dtype_code(ws[0].dtype), lay, n)


def decompose_batch_host(ws, iters: int, sign_seeds, outs, staging, workspace: Workspace, layout: str = "rows",
                         stream=None, kmeans_iters: int = 0):
    """kd_decompose_batch_host: host matrices ``ws`` (pinned CPU tensors) in, host
    outputs ``outs`` (from host_outputs) written once ``stream`` completes.  ``staging``
    is a device uint8 tensor of at least staging_size_host(ws) bytes."""
    arr, lay, n = _host_descriptors(ws, sign_seeds, layout, outs)
    st = kd_decompose_batch_host(ctypes.cast(arr, ctypes.c_void_p), len(ws), _dtype_code(ws[0].dtype), lay, n,
                                 int(iters), int(kmeans_iters), staging.data_ptr(),
                                 staging.numel() * staging.element_size(), workspace.ptr, workspace.nbytes,
                                 _stream(stream))
    if st != KD_OK:
        raise KashinError(st, "kd_decompose_batch_host")
    return outs


def read_status(workspace: Workspace, stream=None) -> int:
    return kd_read_status(workspace.ptr, _stream(stream))


def apply_p(x, sign_seed: int, out=None, workspace: Optional[Workspace] = None, stream=None):
    """``y_j = P x_j`` for the rows of the fp32 (m, n) tensor ``x``."""
    torch = _torch()
    if x.dtype != torch.float32 or not x.is_contiguous() or x.dim() != 2:
        raise ValueError("x must be a contiguous fp32 (m, n) CUDA tensor")
    m, n = x.shape
    y = out if out is not None else _new(stream, x.shape, x.dtype, x.device)
    ws = workspace if workspace is not None else Workspace(n, x.device, stream=stream)
    st = kd_apply_p(x.data_ptr(), y.data_ptr(), n, m, sign_seed, ws.ptr, ws.nbytes, _stream(stream))
    if st != KD_OK:
        raise KashinError(st, "kd_apply_p")
    return y


def dequantise(codes, centres, n: int, dtype=None, layout: str = "rows", out=None, stream=None):
    """Dense factor matrix from one 2-bit code plane and its centres (App. C):
    (m, n) for layout "rows", (n, m) for "columns"."""
    torch = _torch()
    dtype = dtype or torch.float32
    m = codes.shape[0]
    lay = KD_VEC_ROWS if layout == "rows" else KD_VEC_COLUMNS
    if out is None:
        out = _new(stream, (m, n) if lay == KD_VEC_ROWS else (n, m), dtype, codes.device)
    st = kd_dequantise(codes.data_ptr(), centres.data_ptr(), n, m, _dtype_code(out.dtype), lay, out.data_ptr(),
                       _ld(out), _stream(stream))
    if st != KD_OK:
        raise KashinError(st, "kd_dequantise")
    return out


def dequantise_batch(planes, n: int, dtype=None, layout: str = "rows", outs=None, stream=None):
    """``dequantise`` for several (codes, centres) planes of one vector length in one
    launch (kd_dequantise_batch); returns one dense matrix per plane."""
    torch = _torch()
    if not 1 <= len(planes) <= KD_MAX_BATCH:
        raise ValueError(f"1..{KD_MAX_BATCH} planes")
    dtype = dtype or torch.float32
    lay = KD_VEC_ROWS if layout == "rows" else KD_VEC_COLUMNS
    arr = (KdPlane * len(planes))()
    res = []
    for i, (codes, centres) in enumerate(planes):
        m = codes.shape[0]
        if outs is not None:
            o = outs[i]
        else:
            o = _new(stream, (m, n) if lay == KD_VEC_ROWS else (n, m), dtype, codes.device)
        if o.dtype != dtype:
            raise ValueError("outputs must share one dtype")
        arr[i] = KdPlane(codes.data_ptr(), centres.data_ptr(), o.data_ptr(), m, _ld(o))
        res.append(o)
    st = kd_dequantise_batch(ctypes.cast(arr, ctypes.c_void_p), len(planes), n, _dtype_code(dtype), lay,
                             _stream(stream))
    if st != KD_OK:
        raise KashinError(st, "kd_dequantise_batch")
    return res


def rht(x, seed: int, inverse: bool = False, out=None, status=None, stream=None):
    """Randomized-Hadamard rotation of the rows of the (m, n) tensor ``x`` (fp32,
    fp16 or bf16, unit inner stride) into an fp32 (m, n) tensor; ``out=x`` rotates
    an fp32 tensor in place (Sec. 4, Kashin-DCT+H).  ``status``: optional int32
    device tensor of one element that collects KD_RHT_ERR_* bits."""
    torch = _torch()
    if x.dim() != 2 or x.stride(1) != 1:
        raise ValueError("x must be a 2-D CUDA tensor with unit inner stride")
    m, n = x.shape
    y = out if out is not None else _new(stream, (m, n), torch.float32, x.device)
    if y.dtype != torch.float32 or y.shape != x.shape or y.stride(1) != 1:
        raise ValueError("out must be an fp32 tensor of x's shape with unit inner stride")
    st = kd_rht(x.data_ptr(), _dtype_code(x.dtype), n, m, _ld(x), seed, 1 if inverse else 0, y.data_ptr(),
                _ld(y), status.data_ptr() if status is not None else None, _stream(stream))
    if st != KD_OK:
        raise KashinError(st, "kd_rht")
    return y


def reconstruct(dec: Decomposed, n: int, sign_seed: int, dtype=None, layout: str = "rows", out=None,
                workspace: Optional[Workspace] = None, stream=None):
    """Dense ``W_hat = U_q + P V_q`` from codes and centres (App. C)."""
    torch = _torch()
    dtype = dtype or torch.float32
    m = dec.codes_u.shape[0]
    lay = KD_VEC_ROWS if layout == "rows" else KD_VEC_COLUMNS
    dev = dec.codes_u.device
    if out is None:
        out = _new(stream, (m, n) if lay == KD_VEC_ROWS else (n, m), dtype, dev)
    ws = workspace if workspace is not None else Workspace(n, dev, stream=stream)
    st = kd_reconstruct(dec.codes_u.data_ptr(), dec.codes_v.data_ptr(), dec.centres_u.data_ptr(),
                        dec.centres_v.data_ptr(), n, m, sign_seed, _dtype_code(out.dtype), lay, out.data_ptr(),
                        _ld(out), ws.ptr, ws.nbytes, _stream(stream))
    if st != KD_OK:
        raise KashinError(st, "kd_reconstruct")
    return out


def reconstruct_batch(decs, n: int, sign_seeds, dtype=None, layout: str = "rows", outs=None,
                      workspace: Optional[Workspace] = None, stream=None):
    """``reconstruct`` for several decomposed matrices of one vector length in one
    launch (kd_reconstruct_batch); returns one dense W_hat per matrix."""
    torch = _torch()
    if not 1 <= len(decs) <= KD_MAX_BATCH or len(sign_seeds) != len(decs):
        raise ValueError(f"1..{KD_MAX_BATCH} matrices with one seed each")
    dtype = dtype or torch.float32
    lay = KD_VEC_ROWS if layout == "rows" else KD_VEC_COLUMNS
    dev = decs[0].codes_u.device
    arr = (KdRecMat * len(decs))()
    res = []
    for i, d in enumerate(decs):
        m = d.codes_u.shape[0]
        o = outs[i] if outs is not None else _new(stream, (m, n) if lay == KD_VEC_ROWS else (n, m), dtype, dev)
        if o.dtype != dtype:
            raise ValueError("outputs must share one dtype")
        arr[i] = KdRecMat(d.codes_u.data_ptr(), d.codes_v.data_ptr(), d.centres_u.data_ptr(), d.centres_v.data_ptr(),
                          int(sign_seeds[i]) & ((1 << 64) - 1), o.data_ptr(), m, _ld(o))
        res.append(o)
    ws = workspace if workspace is not None else Workspace(n, dev, count=len(decs), stream=stream)
    st = kd_reconstruct_batch(ctypes.cast(arr, ctypes.c_void_p), len(decs), n, _dtype_code(dtype), lay, ws.ptr,
                              ws.nbytes, _stream(stream))
    if st != KD_OK:
        raise KashinError(st, "kd_reconstruct_batch")
    return res


def unpack_codes(words, n: int):
    """(m, ceil(n/16)) int32 words -> (m, n) int64 codes (host numpy)."""
    w = np.asarray(words.cpu().numpy() if hasattr(words, "cpu") else words).astype(np.uint32).astype(np.uint64)
    m = w.shape[0]
    idx = np.arange(n)
    return ((w[:, idx // 16] >> (2 * (idx % 16)).astype(np.uint64)) & np.uint64(3)).astype(np.int64).reshape(m, n)


# ---------------------------------------------------------------------------
# serving operators around the coded layers
# ---------------------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def _serve():
    """What every call of a serving operator asks torch for, looked up once: the C codes of
    the element types, and the function that gives a device's current stream handle."""
    torch = _torch()
    floats = {torch.float32: KD_F32, torch.float16: KD_F16, torch.bfloat16: KD_BF16}
    rows4 = {torch.float16: KD_F16, torch.bfloat16: KD_BF16, torch.float8_e4m3fn: KD_E4M3}
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        def raw(index):
            return torch.cuda.current_stream(index).cuda_stream
    return floats, rows4, torch.float32, torch.float8_e4m3fn, raw, torch.cuda.current_device


def _refuse(t, name, types, index, shape):
    """Says what is wrong with one operand of a serving operator."""
    if len(t.shape) != 2 and (shape is None or len(shape) == 2):
        raise ValueError(f"{name} must be 2-D")
    if t.dtype not in types:
        raise ValueError(f"{name} has dtype {t.dtype}: one of {', '.join(map(str, types))} is wanted")
    if not t.is_cuda or t.get_device() != index:
        raise ValueError(f"{name} must be a CUDA tensor on " + ("one device with the others" if index < 0 else f"cuda:{index}"))
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}: {tuple(shape)} is wanted")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} needs unit inner stride")
    raise ValueError(f"{name}'s rows must not overlap")


def _ld2(t, name, types, index, shape=None):
    """Row stride of a 2-D operand after its checks: a CUDA tensor of one of ``types`` on
    device ``index``, of ``shape``, with unit inner stride and rows that do not overlap."""
    size, stride = t.shape, t.stride()
    if len(size) != 2 or t.dtype not in types or t.get_device() != index or index < 0 \
            or (shape is not None and size != shape):
        _refuse(t, name, types, index, shape)
    rows, cols = size
    if cols > 1 and stride[1] != 1:
        _refuse(t, name, types, index, shape)
    if rows <= 1:
        return cols
    if stride[0] < cols:
        _refuse(t, name, types, index, shape)
    return stride[0]


def _vec(t, name, types, index, length):
    """Checks a contiguous vector operand."""
    if t.dtype not in types or t.get_device() != index or index < 0 or t.shape != (length,):
        _refuse(t, name, types, index, (length,))
    if length > 1 and t.stride(0) != 1:
        raise ValueError(f"{name} must be contiguous")


def _call(what, fn, index, stream, *args):
    """fn(*args, stream handle) on device ``index``; KashinError for any status but KD_OK."""
    raw, current = _serve()[4:]
    if current() == index:
        st = fn(*args, raw(index) if stream is None else stream.cuda_stream)
    else:
        with _torch().cuda.device(index):
            st = fn(*args, raw(index) if stream is None else stream.cuda_stream)
    if st:
        raise KashinError(st, what)


@dataclasses.dataclass
class Normed:
    """rmsnorm's outputs; a field that is None is not computed."""
    q: "object" = None         # float8_e4m3fn (rows, n)
    scale: "object" = None     # float32 (rows,): q * scale is the normed row
    y: "object" = None         # fp16, bf16 or fp32 (rows, n)
    residual: "object" = None  # x + residual, x's dtype (rows, n)


def rmsnorm(x, weight, eps: float = 1e-5, residual=None, out: Optional[Normed] = None, stream=None) -> Normed:
    """Root-mean-square norm of the rows of ``x`` (plus ``residual``), in 8 bits with one
    scale a row and/or in a float type (kd_rmsnorm).

    ``x``, ``residual``: (rows, n) CUDA tensors of one dtype (fp16, bf16, fp32), n <= 16384;
    ``weight``: (n,) of that dtype or fp32.  ``out``: the tensors to write (``Normed``; set
    ``y`` for the 16- or 32-bit rows that the 2-bit products and apply_p read, and
    ``residual`` -- it may be the ``residual`` argument itself -- for the sum); without it
    ``q``, ``scale`` and, given a residual, ``residual`` are allocated."""
    floats, _, f32, e4m3, _, _ = _serve()
    dt, shape, index = x.dtype, x.shape, x.get_device()
    ldx = _ld2(x, "x", floats, index)
    rows, n = shape
    wdt = weight.dtype
    _vec(weight, "weight", (dt, f32), index, n)
    if out is None:
        dev = x.device
        out = Normed(q=_new(stream, shape, e4m3, dev), scale=_new(stream, (rows,), f32, dev),
                     residual=None if residual is None else _new(stream, shape, dt, dev))
    q, scale, y, new = out.q, out.scale, out.y, out.residual
    ldr = ldn = ldq = ldy = ydt = 0
    residual_ptr = new_ptr = q_ptr = scale_ptr = y_ptr = None
    if residual is not None:
        ldr, residual_ptr = _ld2(residual, "residual", (dt,), index, shape), residual.data_ptr()
    if new is not None:
        if residual is None:
            raise ValueError("out.residual is written only where a residual is given")
        ldn, new_ptr = _ld2(new, "out.residual", (dt,), index, shape), new.data_ptr()
    if q is not None and scale is not None:
        ldq, q_ptr = _ld2(q, "out.q", (e4m3,), index, shape), q.data_ptr()
        _vec(scale, "out.scale", (f32,), index, rows)
        scale_ptr = scale.data_ptr()
    elif q is not None or scale is not None:
        raise ValueError("out.q and out.scale come together")
    elif y is None:
        raise ValueError("out wants q and scale, or y, or all three")
    if y is not None:
        ldy, y_ptr, ydt = _ld2(y, "out.y", floats, index, shape), y.data_ptr(), floats[y.dtype]
    _call("kd_rmsnorm", lib.kd_rmsnorm, index, stream, x.data_ptr(), floats[dt], n, rows, ldx, weight.data_ptr(),
          floats[wdt], eps, residual_ptr, ldr, new_ptr, ldn, q_ptr, ldq, scale_ptr, y_ptr, ydt, ldy)
    return out


def _by_group(t):
    """A (channels, groups) tensor whose memory holds one group's channels together."""
    return t if t.t().is_contiguous() else t.t().contiguous().t()


class Weight4:
    """A matrix of 4-bit weights (kd_weight4): ``codes`` int32 (m, 4 ceil(n/32)), code i of a
    row at bits 4 (i % 8) of word i // 8; ``scales`` fp16 or bf16 (m, ceil(n/group));
    ``zeros`` uint8 of that shape with values 0..15, or None for 8 everywhere.  The weight is
    ``scale * (code - zero)``.  ``codes`` is contiguous; scales and zeros are kept group by
    group (a tensor in another order is laid out anew here, once, on the current stream: the
    one given is not needed any more)."""

    __slots__ = ("codes", "scales", "zeros", "n", "m", "group", "device", "index", "desc", "ref")

    def __init__(self, codes, scales, zeros=None, *, n: int, group: int = 128):
        torch = _torch()
        if group not in (32, 64, 128):
            raise ValueError("group must be 32, 64 or 128")
        if n < 1 or codes.dim() != 2 or codes.shape[1] != (n + 31) // 32 * 4 or codes.dtype != torch.int32:
            raise ValueError("codes must be int32 (m, 4 ceil(n/32))")
        m = codes.shape[0]
        shape = (m, (n + group - 1) // group)
        if tuple(scales.shape) != shape or scales.dtype not in (torch.float16, torch.bfloat16):
            raise ValueError(f"scales must be fp16 or bf16 {shape}")
        if zeros is not None and (tuple(zeros.shape) != shape or zeros.dtype != torch.uint8):
            raise ValueError(f"zeros must be uint8 {shape}")
        for t in (codes, scales, zeros):
            if t is not None and (not t.is_cuda or t.device != codes.device):
                raise ValueError("codes, scales and zeros must be CUDA tensors on one device")
        if not codes.is_contiguous():
            raise ValueError("codes must be contiguous")
        scales, zeros = _by_group(scales), None if zeros is None else _by_group(zeros)
        self.codes, self.scales, self.zeros = codes, scales, zeros
        self.n, self.m, self.group, self.device = int(n), m, int(group), codes.device
        self.index = codes.get_device()
        self.desc = KdWeight4(codes.data_ptr(), scales.data_ptr(), _ptr(zeros), n, m, group,
                              _dtype_code(scales.dtype))
        self.ref = ctypes.addressof(self.desc)


def quantise_4bit(w, group: int = 128, zeros: bool = False, scale_dtype=None, stream=None) -> Weight4:
    """4-bit weights with a scale for each ``group`` inputs from the (m, n) matrix ``w``
    (nn.Linear layout, fp16, bf16 or fp32; kd_quantise_4bit).  ``zeros``: a zero point per
    group too; ``scale_dtype``: fp16 (the default for fp16 weights) or bf16."""
    torch = _torch()
    floats, index, dev = _serve()[0], w.get_device(), w.device
    ld = _ld2(w, "w", floats, index)
    m, n = w.shape
    if group not in (32, 64, 128):
        raise ValueError("group must be 32, 64 or 128")
    if n < 1:
        raise ValueError("w has no inputs")
    sdt = scale_dtype or (torch.float16 if w.dtype == torch.float16 else torch.bfloat16)
    groups = (n + group - 1) // group
    out = Weight4(_new(stream, (m, (n + 31) // 32 * 4), torch.int32, dev), _new(stream, (groups, m), sdt, dev).t(),
                  _new(stream, (groups, m), torch.uint8, dev).t() if zeros else None, n=n, group=group)
    _call("kd_quantise_4bit", lib.kd_quantise_4bit, index, stream, w.data_ptr(), floats[w.dtype], ld, out.ref)
    return out


def dequantise_4bit(w: Weight4, dtype=None, out=None, stream=None):
    """The dense (m, n) matrix of 4-bit weights (kd_dequantise_4bit), fp32 unless ``dtype``
    or ``out`` says otherwise."""
    floats, _, f32, _, _, _ = _serve()
    y = out if out is not None else _new(stream, (w.m, w.n), dtype or f32, w.device)
    ld = _ld2(y, "out", floats, w.index, (w.m, w.n))
    _call("kd_dequantise_4bit", lib.kd_dequantise_4bit, w.index, stream, w.ref, floats[y.dtype], y.data_ptr(), ld)
    return y


def matmul_4bit(w: Weight4, x, scale=None, out=None, out_dtype=None, stream=None):
    """``Y = X W^T`` for few rows ``x`` (rows, n) in fp16, bf16 or float8_e4m3fn (then with
    ``scale``, fp32 (rows,), as rmsnorm leaves them) and 4-bit weights (kd_matmul_4bit);
    returns (rows, m), fp32 unless ``out`` or ``out_dtype`` says otherwise."""
    floats, types, f32, _, _, _ = _serve()
    index, shape = w.index, x.shape
    ldx = _ld2(x, "x", types, index)
    rows = shape[0]
    if shape[1] != w.n:
        raise ValueError(f"x must be (rows, {w.n})")
    scale_ptr = None
    if scale is not None:
        _vec(scale, "scale", (f32,), index, rows)
        scale_ptr = scale.data_ptr()
    if out is None:
        out = _new(stream, (rows, w.m), out_dtype or f32, w.device)
    ldy = _ld2(out, "out", floats, index, (rows, w.m))
    _call("kd_matmul_4bit", lib.kd_matmul_4bit, index, stream, w.ref, x.data_ptr(), types[x.dtype], scale_ptr, rows,
          ldx, out.data_ptr(), floats[out.dtype], ldy)
    return out


@dataclasses.dataclass
class TokenLogprobs:
    logprobs: "object"      # float32 (rows, tokens)
    lse: "object"           # float32 (rows,) or None
    entropy: "object"       # float32 (rows,) or None
    top_ids: "object"       # int64 (rows, top)
    top_logprobs: "object"  # float32 (rows, top)


def token_logprobs(logits, ids, top: int = 0, out: Optional[TokenLogprobs] = None, stream=None) -> TokenLogprobs:
    """Log probabilities of the tokens ``ids`` (int64 (rows,) or (rows, tokens); negative:
    padding, 0) under softmax of the rows of ``logits`` (rows, vocab), the entropy and the
    ``top`` (0..32) likeliest alternatives (kd_token_logprobs)."""
    floats, _, f32, _, _, _ = _serve()
    index = logits.get_device()
    ld = _ld2(logits, "logits", floats, index)
    rows, vocab = logits.shape
    if ids.dim() == 1:
        ids = ids[:, None]
    i64 = _torch().int64
    if ids.dim() != 2 or ids.shape[0] != rows or ids.dtype != i64 or ids.get_device() != index \
            or not ids.is_contiguous():
        raise ValueError("ids must be a contiguous int64 (rows,) or (rows, tokens) tensor on the logits' device")
    tokens = ids.shape[1]
    if not 0 <= top <= min(vocab, KD_MAX_TOP):
        raise ValueError(f"top must be 0..{min(vocab, KD_MAX_TOP)}")
    if out is None:
        dev = logits.device
        out = TokenLogprobs(_new(stream, (rows, tokens), f32, dev), _new(stream, (rows,), f32, dev),
                            _new(stream, (rows,), f32, dev), _new(stream, (rows, top), i64, dev),
                            _new(stream, (rows, top), f32, dev))
    else:
        for name, dt, size in (("logprobs", f32, (rows, tokens)), ("lse", f32, (rows,)), ("entropy", f32, (rows,)),
                               ("top_ids", i64, (rows, top)), ("top_logprobs", f32, (rows, top))):
            t = getattr(out, name)
            if t is None and (name == "lse" or name == "entropy"):
                continue
            if t is None or t.dtype != dt or t.shape != size or t.get_device() != index or not t.is_contiguous():
                raise ValueError(f"out.{name} must be a contiguous {dt} {size} tensor on the logits' device")
    lse, entropy = out.lse, out.entropy
    _call("kd_token_logprobs", lib.kd_token_logprobs, index, stream, logits.data_ptr(), floats[logits.dtype], rows,
          vocab, ld, ids.data_ptr(), tokens, top, out.logprobs.data_ptr(), None if lse is None else lse.data_ptr(),
          None if entropy is None else entropy.data_ptr(), out.top_ids.data_ptr(), out.top_logprobs.data_ptr())
    return out
