"""Binding of ``include/mxfp8_experts.h``: same names as the C ABI, argument checks and marshalling only (see binding.py).

Rows of a mixture-of-experts layer on their way to the grouped products and back, and products of a few rows with MXFP4 weights.
Entry ``t * slots + j`` stands for slot j of token t.
"""
from __future__ import annotations

import torch

from . import binding as _b
from .binding import BOTH, COLWISE, K_BLOCK, OK, ROWWISE, SCALES_ROWMAJOR, MXFP8Error, mxfp8_scale_bytes  # noqa: F401

I32, I64 = 0, 1


def _ready(*tensors):
    """All tensors in GPU memory, on the current device: that is where the call's kernels run."""
    _b._need_cuda(*tensors)
    devices = {t.device for t in tensors if t is not None}
    if len(devices) > 1:
        raise ValueError(f"all tensors must live on one device, got {sorted(map(str, devices))}")
    device = devices.pop()
    if device.type == "cuda" and device.index != torch.cuda.current_device():
        raise ValueError(f"the tensors live on {device}, the current device is cuda:{torch.cuda.current_device()}")


def _int32(value, what):
    """A number that ctypes would cut down to 32 bits without a word."""
    if not -2 ** 31 <= value < 2 ** 31:
        raise ValueError(f"{what} is {value}")
    return value


def _check_index(t, numel, what):
    if t.dtype != torch.int32 or not t.is_contiguous() or (numel is not None and t.numel() != numel):
        raise ValueError(f"{what} must be contiguous int32" + ("" if numel is None else f" of {numel} elements"))


def _check_weights(t, numel):
    if t is not None and (t.dtype != torch.float32 or not t.is_contiguous() or t.numel() != numel):
        raise ValueError(f"weights must be contiguous float32 of {numel} elements")


def _matrix(t, what, rows=None, cols=None):
    """Leading dimension of a matrix with contiguous rows."""
    if t.dim() != 2 or (t.numel() and t.stride(1) != 1) or (rows is not None and t.shape[0] != rows) or (cols is not None and t.shape[1] != cols):
        raise ValueError(f"{what} must be [{'rows' if rows is None else rows} x {'columns' if cols is None else cols}] with contiguous rows")
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1)


def _check_status(rc, what):
    if rc != OK:
        raise MXFP8Error(rc, what)


def _fast(name, what, *args) -> bool:
    """Whether the call of that name in C++ (csrc/fastcall.cpp) did it all."""
    return _b._fast is not None and _b._done(getattr(_b._fast, name)(*args), what)


# ---- raw entry points: same names and argument order as include/mxfp8_experts.h ------------------------------------------

def mxfp8_expert_rows(entries: int, groups: int, align: int) -> int:
    """Rows that sorted entries take at most (host arithmetic in the library)."""
    n = _b.load().mxfp8_expert_rows(entries, _int32(groups, "groups"), _int32(align, "align"))
    if n < 0:
        raise ValueError("bad number of entries, groups or alignment")
    return n


def mxfp8_expert_sort_workspace(entries: int, groups: int) -> int:
    """Bytes of workspace that mxfp8_expert_sort needs (host arithmetic in the library)."""
    n = _b.load().mxfp8_expert_sort_workspace(entries, _int32(groups, "groups"))
    if n < 0:
        raise ValueError("bad number of entries or groups")
    return n


def mxfp8_expert_sort(experts, align, positions, sources, group_ends, workspace=None, stream=None) -> None:
    """experts int32/int64 [tokens x slots] -> positions (int32, as many), sources (int32 [rows]), group_ends (int32 [groups]).
    workspace: uint8 of mxfp8_expert_sort_workspace(entries, groups) bytes, None where that is 0."""
    if _fast("expert_sort", "mxfp8_expert_sort", experts, align, positions, sources, group_ends, workspace, stream):
        return
    _ready(experts, positions, sources, group_ends, workspace)
    if experts.dtype not in (torch.int32, torch.int64) or not experts.is_contiguous():
        raise ValueError("experts must be contiguous int32 or int64")
    entries, groups, align = experts.numel(), group_ends.numel(), _int32(align, "align")
    _check_index(positions, entries, "positions")
    _check_index(sources, None, "sources")
    _check_index(group_ends, None, "group_ends")
    need = mxfp8_expert_sort_workspace(entries, groups)
    if need and (workspace is None or not workspace.is_contiguous() or workspace.numel() * workspace.element_size() < need):
        raise ValueError(f"the sort of {entries} entries to {groups} experts needs a contiguous workspace of {need} bytes")
    _check_status(_b.load().mxfp8_expert_sort(_b._ptr(experts), I64 if experts.dtype == torch.int64 else I32, entries, groups, align, sources.numel(),
                                      _b._ptr(positions), _b._ptr(sources), _b._ptr(group_ends), _b._ptr(workspace), _b._stream(stream)),
          "mxfp8_expert_sort")


def mxfp8_expert_quantize_ex(src, sources, group_ends, slots, weights, axis, q_row=None, s_row=None, q_colT=None, s_colT=None,
                             scale_layout=SCALES_ROWMAJOR, stream=None) -> None:
    """MXFP8 copies of the sorted rows weights[i] * src[i // slots] with i = sources[r], zeros for -1. src [tokens x cols]
    float32/bfloat16; weights float32 [tokens x slots] or None; group_ends int32, or None to convert all rows."""
    if _fast("expert_quantize", "mxfp8_expert_quantize_ex", src, sources, group_ends, slots, weights, axis, q_row, s_row, q_colT, s_colT, scale_layout, stream):
        return
    _ready(src, sources, group_ends, weights, q_row, s_row, q_colT, s_colT)
    ld = _matrix(src, "src")
    tokens, cols = src.shape
    _check_index(sources, None, "sources")
    rows, slots = sources.numel(), _int32(slots, "slots")
    if group_ends is not None:
        _check_index(group_ends, None, "group_ends")
        if not group_ends.numel():
            raise ValueError("group_ends is empty: pass None to convert all rows")
    _check_weights(weights, tokens * slots)
    ax = _b._AXIS[axis]
    if cols % K_BLOCK or rows % K_BLOCK:
        raise ValueError("the rows of the plan and the columns must be multiples of 32")
    for wanted, q, s, shape, name in ((ax & ROWWISE, q_row, s_row, (rows, cols), "row"), (ax & COLWISE, q_colT, s_colT, (cols, rows), "colT")):
        if wanted:
            if q is None or s is None or q.dtype != torch.uint8 or not q.is_contiguous() or tuple(q.shape) != shape:
                raise ValueError(f"q_{name} must be dense uint8 [{shape[0]} x {shape[1]}], s_{name} its scales")
            _b._check_scales(s, *shape, scale_layout, f"s_{name}")
    _check_status(_b.load().mxfp8_expert_quantize_ex(_b._ptr(src), _b._dtype_code(src.dtype), tokens, cols, ld, _b._ptr(sources), slots, _b._ptr(weights),
                                             _b._ptr(group_ends), 0 if group_ends is None else group_ends.numel(), rows, ax, _b._ptr(q_row),
                                             _b._ptr(s_row), _b._ptr(q_colT), _b._ptr(s_colT), scale_layout, _b._stream(stream)),
          "mxfp8_expert_quantize_ex")


def mxfp8_expert_combine(c, positions, weights, out, stream=None) -> None:
    """out [tokens x cols] = sum over slots of weights * c[positions] (None: plain sum). c [rows x cols], positions int32
    [tokens x slots], -1 adds nothing; weights float32 of the same shape."""
    if _fast("expert_combine", "mxfp8_expert_combine", c, positions, weights, out, stream):
        return
    _ready(c, positions, weights, out)
    ldc = _matrix(c, "c")
    rows, cols = c.shape
    if positions.dim() != 2:
        raise ValueError("positions must be [tokens x slots]")
    tokens, slots = positions.shape
    _check_index(positions, None, "positions")
    _check_weights(weights, tokens * slots)
    ld_out = _matrix(out, "out", tokens, cols)
    _check_status(_b.load().mxfp8_expert_combine(_b._ptr(c), _b._dtype_code(c.dtype), rows, cols, ldc, _b._ptr(positions), _b._ptr(weights), tokens, slots,
                                         _b._ptr(out), _b._dtype_code(out.dtype), ld_out, _b._stream(stream)), "mxfp8_expert_combine")


def mxfp8_expert_weight_grad(dy, c, positions, dweights, stream=None) -> None:
    """dweights float32 [tokens x slots] = dot products of dy [tokens x cols] with the rows c[positions], 0 for -1."""
    if _fast("expert_weight_grad", "mxfp8_expert_weight_grad", dy, c, positions, dweights, stream):
        return
    _ready(dy, c, positions, dweights)
    ldc = _matrix(c, "c")
    rows, cols = c.shape
    if positions.dim() != 2:
        raise ValueError("positions must be [tokens x slots]")
    tokens, slots = positions.shape
    _check_index(positions, None, "positions")
    ld_dy = _matrix(dy, "dy", tokens, cols)
    if dweights.dtype != torch.float32 or not dweights.is_contiguous() or dweights.numel() != tokens * slots:
        raise ValueError(f"dweights must be contiguous float32 of {tokens * slots} elements")
    _check_status(_b.load().mxfp8_expert_weight_grad(_b._ptr(dy), _b._dtype_code(dy.dtype), ld_dy, _b._ptr(c), _b._dtype_code(c.dtype), rows, cols, ldc,
                                             _b._ptr(positions), tokens, slots, _b._ptr(dweights), _b._stream(stream)), "mxfp8_expert_weight_grad")


def _activations(x):
    if x.dtype != torch.bfloat16:
        raise TypeError(f"x must be bfloat16, got {x.dtype}")
    return _matrix(x, "x")


def mxfp8_fp4_gemv_ex(x, w_q, w_s, c, scale_layout=SCALES_ROWMAJOR, stream=None) -> None:
    """c [M x N] (float32/bfloat16) = x [M x K] bfloat16 times MXFP4 weights w_q [N x K/2], w_s transposed: for a few rows."""
    if _fast("fp4_gemv", "mxfp8_fp4_gemv_ex", x, w_q, w_s, c, scale_layout, stream):
        return
    _ready(x, w_q, w_s, c)
    ldx = _activations(x)
    (M, K), N = x.shape, c.shape[1] if c.dim() == 2 else -1
    if w_q.dtype != torch.uint8 or not w_q.is_contiguous() or tuple(w_q.shape) != (N, K // 2) or K % K_BLOCK:
        raise ValueError(f"w_q must be dense uint8 [{N} x {K // 2}], K a multiple of 32")
    _b._check_scales(w_s, N, K, scale_layout, "w_s")
    ldc = _matrix(c, "c", M, N)
    _check_status(_b.load().mxfp8_fp4_gemv_ex(_b._ptr(x), ldx, _b._ptr(w_q), _b._ptr(w_s), M, N, K, _b._ptr(c), _b._dtype_code(c.dtype), ldc, scale_layout,
                                      _b._stream(stream)), "mxfp8_fp4_gemv_ex")


def mxfp8_fp4_gemv_grouped_ex(x, sources, slots, w_q, w_s, group_ends, c, scale_layout=SCALES_ROWMAJOR, stream=None) -> None:
    """Row r of c [M x N] = x[sources[r] // slots] (x[r] with sources None) times the weights of the expert that owns row r: w_q
    [groups x N x K/2], w_s (groups scale operands). Rows from the last end on are left as they were."""
    if _fast("fp4_gemv_grouped", "mxfp8_fp4_gemv_grouped_ex", x, sources, slots, w_q, w_s, group_ends, c, scale_layout, stream):
        return
    _ready(x, sources, w_q, w_s, group_ends, c)
    ldx = _activations(x)
    tokens, K = x.shape
    if c.dim() != 2:
        raise ValueError("c must be [rows x N]")
    M, N = c.shape
    _check_index(group_ends, None, "group_ends")
    groups, slots = group_ends.numel(), _int32(slots, "slots")
    if sources is not None:
        _check_index(sources, M, "sources")
    elif tokens < M:
        raise ValueError(f"x has {tokens} rows for {M} of c")
    if w_q.dtype != torch.uint8 or not w_q.is_contiguous() or tuple(w_q.shape) != (groups, N, K // 2) or K % K_BLOCK:
        raise ValueError(f"w_q must be dense uint8 [{groups} x {N} x {K // 2}], K a multiple of 32")
    if w_s.dtype != torch.uint8 or not w_s.is_contiguous() or w_s.numel() != groups * mxfp8_scale_bytes(N, K, scale_layout):
        raise ValueError("w_s must be dense uint8 with one scale operand per expert")
    ldc = _matrix(c, "c")
    _check_status(_b.load().mxfp8_fp4_gemv_grouped_ex(_b._ptr(x), tokens, ldx, _b._ptr(sources), slots, _b._ptr(w_q), _b._ptr(w_s), _b._ptr(group_ends), groups,
                                              M, N, K, _b._ptr(c), _b._dtype_code(c.dtype), ldc, scale_layout, _b._stream(stream)),
          "mxfp8_fp4_gemv_grouped_ex")


# ---- conveniences that only allocate the outputs -------------------------------------------------------------------------

def expert_sort(experts, groups, align=128):
    """Allocate outputs and workspace and call mxfp8_expert_sort. Returns a dict: 'positions' (shape of experts), 'sources'
    [mxfp8_expert_rows(entries, groups, align)], 'group_ends' [groups], all int32."""
    i32 = dict(dtype=torch.int32, device=experts.device)
    out = {"positions": torch.empty(tuple(experts.shape), **i32), "sources": torch.empty((mxfp8_expert_rows(experts.numel(), groups, align),), **i32),
           "group_ends": torch.empty((groups,), **i32)}
    need = mxfp8_expert_sort_workspace(experts.numel(), groups)
    workspace = torch.empty((need,), dtype=torch.uint8, device=experts.device) if need else None
    mxfp8_expert_sort(experts, align, out["positions"], out["sources"], out["group_ends"], workspace)
    return out


def expert_quantize(src, sources, group_ends, slots, weights=None, axis="both", scale_layout=SCALES_ROWMAJOR):
    """Allocate outputs and call mxfp8_expert_quantize_ex; keys as for quantize(). Rows behind the last 128-row tile that holds a row of
    an expert are not written: they hold whatever the allocation held."""
    rows, cols = sources.numel(), src.shape[1]
    ax = _b._AXIS[axis]
    out = {}
    u8 = dict(dtype=torch.uint8, device=src.device)
    tiled = scale_layout != SCALES_ROWMAJOR
    if ax & ROWWISE:
        out["q_row"] = torch.empty((rows, cols), **u8)
        out["s_row"] = torch.empty((mxfp8_scale_bytes(rows, cols, scale_layout),) if tiled else (rows, cols // K_BLOCK), **u8)
    if ax & COLWISE:
        out["q_colT"] = torch.empty((cols, rows), **u8)
        out["s_colT"] = torch.empty((mxfp8_scale_bytes(cols, rows, scale_layout),) if tiled else (cols, rows // K_BLOCK), **u8)
    mxfp8_expert_quantize_ex(src, sources, group_ends, slots, weights, ax, out.get("q_row"), out.get("s_row"), out.get("q_colT"), out.get("s_colT"),
                             scale_layout)
    return out


def expert_combine(c, positions, weights=None, out_dtype=torch.bfloat16):
    out = torch.empty((positions.shape[0], c.shape[1]), dtype=out_dtype, device=c.device)
    mxfp8_expert_combine(c, positions, weights, out)
    return out


def expert_weight_grad(dy, c, positions):
    dweights = torch.empty(tuple(positions.shape), dtype=torch.float32, device=c.device)
    mxfp8_expert_weight_grad(dy, c, positions, dweights)
    return dweights


def fp4_gemv(x, w_q, w_s, out_dtype=torch.bfloat16, scale_layout=SCALES_ROWMAJOR):
    c = torch.empty((x.shape[0], w_q.shape[0]), dtype=out_dtype, device=x.device)
    mxfp8_fp4_gemv_ex(x, w_q, w_s, c, scale_layout)
    return c


def fp4_gemv_grouped(x, sources, slots, w_q, w_s, group_ends, out_dtype=torch.bfloat16, scale_layout=SCALES_ROWMAJOR):
    """Rows from group_ends[-1] on are not written: they hold whatever the allocation held."""
    c = torch.empty((x.shape[0] if sources is None else sources.numel(), w_q.shape[1]), dtype=out_dtype, device=x.device)
    mxfp8_fp4_gemv_grouped_ex(x, sources, slots, w_q, w_s, group_ends, c, scale_layout)
    return c
