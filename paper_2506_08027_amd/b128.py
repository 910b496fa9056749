"""Binding of ``include/mxfp8_b128.h``: same names as the C ABI, argument checks and marshalling only (see binding.py).

FP8 (E4M3) operands with an FP32 scale for each block of 128. An operand [rows x cols] is a uint8 tensor whose rows lie a multiple of
16 bytes apart; where cols is not a multiple of 16, the bytes up to the next one belong to it and are zero (as the quantizer leaves
them). Scales of VECTORS (blocks along a row) are [ceil(cols / 128) x rows], those of TILES [ceil(rows / 128) x ceil(cols / 128)].
"""
from __future__ import annotations

import torch

from . import binding as _b
from .binding import COLWISE, ROWWISE, WGRAD
from .experts import _activations, _check_status, _fast, _matrix, _ready

B128_VECTORS, B128_TILES = 0, 1
BLOCK = 128


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _up16(n):
    return (n + 15) // 16 * 16


def _operand(q, what, rows=None, cols=None):
    """Leading dimension of an operand, padding bytes included."""
    if q is None or q.dtype != torch.uint8 or q.dim() != 2 or (rows is not None and q.shape[0] != rows) or (cols is not None and q.shape[1] != cols) or \
            (q.numel() and q.stride(1) != 1):
        raise ValueError(f"{what} must be uint8 [{'rows' if rows is None else rows} x {'columns' if cols is None else cols}] with contiguous rows")
    ld = q.stride(0) if q.shape[0] > 1 and q.shape[1] else _up16(q.shape[1])
    if q.numel() and q.storage_offset() + (q.shape[0] - 1) * ld + _up16(q.shape[1]) > q.untyped_storage().nbytes():
        raise ValueError(f"the rows of {what} must be followed by their padding up to a multiple of 16 bytes, the last one too")
    return ld


def _check_scales(s, shape, what):
    if s is None or s.dtype != torch.float32 or not s.is_contiguous() or tuple(s.shape) != shape:
        raise ValueError(f"{what} must be dense float32 [{shape[0]} x {shape[1]}]")


def _scale_shape(shape, rows, cols):
    return (_blocks(rows), _blocks(cols)) if shape == B128_TILES else (_blocks(cols), rows)


# ---- raw entry points: same names and argument order as include/mxfp8_b128.h ---------------------------------------------

def mxfp8_b128_quantize(src, axis, shape=B128_VECTORS, q_row=None, s_row=None, q_colT=None, s_colT=None, stream=None) -> None:
    """src [rows x cols] float32/bfloat16 -> the selected copies: q_row [rows x cols], q_colT [cols x rows], scales of their blocks."""
    if _fast("b128_quantize", "mxfp8_b128_quantize", src, axis, shape, q_row, s_row, q_colT, s_colT, stream):
        return
    _ready(src, q_row, s_row, q_colT, s_colT)
    ld = _matrix(src, "src")
    rows, cols = src.shape
    ax = _b._AXIS[axis]
    if shape not in (B128_VECTORS, B128_TILES):
        raise ValueError(f"shape must be B128_VECTORS or B128_TILES, got {shape!r}")
    lds = [0, 0]
    for i, (wanted, q, s, r, c, name) in enumerate(((ax & ROWWISE, q_row, s_row, rows, cols, "row"), (ax & COLWISE, q_colT, s_colT, cols, rows, "colT"))):
        if wanted:
            lds[i] = _operand(q, f"q_{name}", r, c)
            _check_scales(s, _scale_shape(shape, r, c), f"s_{name}")
    _check_status(_b.load().mxfp8_b128_quantize(_b._ptr(src), _b._dtype_code(src.dtype), rows, cols, ld, ax, shape, _b._ptr(q_row), lds[0], _b._ptr(s_row),
                                                _b._ptr(q_colT), lds[1], _b._ptr(s_colT), _b._stream(stream)), "mxfp8_b128_quantize")


def mxfp8_b128_gemm_workspace(pass_, M: int, N: int, K: int) -> int:
    """Bytes of workspace that mxfp8_b128_gemm needs (host arithmetic in the library)."""
    n = _b.load().mxfp8_b128_gemm_workspace(_b._PASS[pass_], M, N, K)
    if n < 0:
        raise ValueError("bad sizes of a product")
    return n


def mxfp8_b128_gemm(pass_, a_q, a_s, b_q, b_s, c, workspace=None, stream=None) -> None:
    """c [M x N] (float32/bfloat16) = A [M x K] B [N x K]^T; A in vectors, B in tiles ("wgrad": in vectors). A float32 c is made of exact
    products at half the rate, a bfloat16 one by the FP8 instructions. workspace: uint8 of mxfp8_b128_gemm_workspace(pass_, M, N, K) bytes,
    None where that is 0."""
    if _fast("b128_gemm", "mxfp8_b128_gemm", pass_, a_q, a_s, b_q, b_s, c, workspace, stream):
        return
    _ready(a_q, a_s, b_q, b_s, c, workspace)
    lda = _operand(a_q, "a_q")
    M, K = a_q.shape
    ldb = _operand(b_q, "b_q", None, K)
    N, which = b_q.shape[0], _b._PASS[pass_]
    _check_scales(a_s, _scale_shape(B128_VECTORS, M, K), "a_s")
    _check_scales(b_s, _scale_shape(B128_VECTORS if which == WGRAD else B128_TILES, N, K), "b_s")
    ldc = _matrix(c, "c", M, N)
    need = mxfp8_b128_gemm_workspace(which, M, N, K)
    if need and (workspace is None or not workspace.is_contiguous() or workspace.numel() * workspace.element_size() < need):
        raise ValueError(f"this product needs a contiguous workspace of {need} bytes")
    _check_status(_b.load().mxfp8_b128_gemm(which, _b._ptr(a_q), lda, _b._ptr(a_s), _b._ptr(b_q), ldb, _b._ptr(b_s), M, N, K, _b._ptr(c),
                                            _b._dtype_code(c.dtype), ldc, _b._ptr(workspace), _b._stream(stream)), "mxfp8_b128_gemm")


def mxfp8_b128_gemv(x, w_q, w_s, c, stream=None) -> None:
    """c [M x N] (float32/bfloat16) = x [M x K] bfloat16 times the weights w_q [N x K] in tiles, transposed: for a few rows."""
    if _fast("b128_gemv", "mxfp8_b128_gemv", x, w_q, w_s, c, stream):
        return
    _ready(x, w_q, w_s, c)
    ldx = _activations(x)
    M, K = x.shape
    ldw = _operand(w_q, "w_q", None, K)
    N = w_q.shape[0]
    _check_scales(w_s, _scale_shape(B128_TILES, N, K), "w_s")
    ldc = _matrix(c, "c", M, N)
    _check_status(_b.load().mxfp8_b128_gemv(_b._ptr(x), ldx, _b._ptr(w_q), ldw, _b._ptr(w_s), M, N, K, _b._ptr(c), _b._dtype_code(c.dtype), ldc,
                                            _b._stream(stream)), "mxfp8_b128_gemv")


# ---- conveniences that only allocate the outputs -------------------------------------------------------------------------

def b128_quantize(src, axis="both", shape=B128_VECTORS):
    """Allocate outputs and call mxfp8_b128_quantize; keys as for quantize()."""
    ax, out = _b._AXIS[axis], {}
    rows, cols = src.shape
    for wanted, r, c, name in ((ax & ROWWISE, rows, cols, "row"), (ax & COLWISE, cols, rows, "colT")):
        if wanted:
            out[f"q_{name}"] = torch.empty((r, _up16(c)), dtype=torch.uint8, device=src.device)[:, :c]
            out[f"s_{name}"] = torch.empty(_scale_shape(shape, r, c), dtype=torch.float32, device=src.device)
    mxfp8_b128_quantize(src, ax, shape, **out)
    return out


def b128_gemm(pass_, a_q, a_s, b_q, b_s, out_dtype=torch.float32):
    c = torch.empty((a_q.shape[0], b_q.shape[0]), dtype=out_dtype, device=a_q.device)
    need = mxfp8_b128_gemm_workspace(pass_, a_q.shape[0], b_q.shape[0], a_q.shape[1])
    mxfp8_b128_gemm(pass_, a_q, a_s, b_q, b_s, c, torch.empty((need,), dtype=torch.uint8, device=a_q.device) if need else None)
    return c


def b128_gemv(x, w_q, w_s, out_dtype=torch.bfloat16):
    c = torch.empty((x.shape[0], w_q.shape[0]), dtype=out_dtype, device=x.device)
    mxfp8_b128_gemv(x, w_q, w_s, c)
    return c
