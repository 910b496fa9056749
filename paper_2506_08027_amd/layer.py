"""Binding of ``include/mxfp8_layer.h``: same names as the C ABI, argument checks and marshalling only (see binding.py).

A whole mixture-of-experts layer for a few tokens: up-projections with their gate, down-projections, the weighted sum over a token's
experts.
"""
from __future__ import annotations

import torch

from . import binding as _b
from .b128 import _blocks
from .binding import K_BLOCK, SCALES_ROWMAJOR, mxfp8_scale_bytes
from .experts import I32, I64, _activations, _check_status, _check_weights, _fast, _int32, _matrix, _ready

WEIGHTS_MXFP4, WEIGHTS_MXFP8, WEIGHTS_B128 = 0, 1, 2


def mxfp8_expert_layer_workspace(tokens: int, slots: int, inter: int) -> int:
    """Bytes of workspace that mxfp8_expert_layer needs (host arithmetic in the library)."""
    n = _b.load().mxfp8_expert_layer_workspace(tokens, _int32(slots, "slots"), inter)
    if n < 0:
        raise ValueError("bad number of tokens, slots or values between the products")
    return n


def _expert_matrices(q, s, format, groups, rows, cols, scale_layout, what):
    if q.dtype != torch.uint8 or not q.is_contiguous() or tuple(q.shape) != (groups, rows, cols // 2 if format == WEIGHTS_MXFP4 else cols):
        raise ValueError(f"{what}_q must be dense uint8 of {groups} matrices [{rows} x {cols}]" + (", two elements a byte" if format == WEIGHTS_MXFP4 else ""))
    if format == WEIGHTS_B128:
        if s.dtype != torch.float32 or not s.is_contiguous() or tuple(s.shape) != (groups, _blocks(rows), _blocks(cols)):
            raise ValueError(f"{what}_s must be dense float32 [{groups} x {_blocks(rows)} x {_blocks(cols)}]")
    elif cols % K_BLOCK or s.dtype != torch.uint8 or not s.is_contiguous() or s.numel() != groups * mxfp8_scale_bytes(rows, cols, scale_layout):
        raise ValueError(f"{what}_s must be dense uint8 with one scale operand per expert")


def mxfp8_expert_layer(x, experts, weights, format, up_q, up_s, down_q, down_s, out, workspace, scale_layout=SCALES_ROWMAJOR, stream=None) -> None:
    """out [tokens x hidden] (float32/bfloat16) of x [tokens x hidden] bfloat16: sum over slots of weights (float32 [tokens x slots]) times
    the expert's down-projection of silu(gate) * up; experts int32/int64 [tokens x slots]. up_q [groups x 2 inter x hidden] (gates first),
    down_q [groups x hidden x inter], two elements a byte with WEIGHTS_MXFP4. workspace: mxfp8_expert_layer_workspace bytes."""
    if _fast("expert_layer", "mxfp8_expert_layer", x, experts, weights, format, up_q, up_s, down_q, down_s, out, workspace, scale_layout, stream):
        return
    _ready(x, experts, weights, up_q, up_s, down_q, down_s, out, workspace)
    if format not in (WEIGHTS_MXFP4, WEIGHTS_MXFP8, WEIGHTS_B128):
        raise ValueError(f"format must be WEIGHTS_MXFP4, WEIGHTS_MXFP8 or WEIGHTS_B128, got {format!r}")
    ldx = _activations(x)
    tokens, hidden = x.shape
    if experts.dtype not in (torch.int32, torch.int64) or not experts.is_contiguous() or experts.dim() != 2 or experts.shape[0] != tokens:
        raise ValueError(f"experts must be contiguous int32 or int64 [{tokens} x slots]")
    slots = experts.shape[1]
    if weights is None or tuple(weights.shape) != (tokens, slots):
        raise ValueError(f"the layer needs the router's weights, contiguous float32 [{tokens} x {slots}]")
    _check_weights(weights, tokens * slots)
    if down_q.dim() != 3:
        raise ValueError("down_q must be [groups x hidden x inter]")
    groups, inter = down_q.shape[0], down_q.shape[2] * (2 if format == WEIGHTS_MXFP4 else 1)
    _expert_matrices(up_q, up_s, format, groups, 2 * inter, hidden, scale_layout, "up")
    _expert_matrices(down_q, down_s, format, groups, hidden, inter, scale_layout, "down")
    ld_out = _matrix(out, "out", tokens, hidden)
    need = mxfp8_expert_layer_workspace(tokens, slots, inter)
    if need and (workspace is None or not workspace.is_contiguous() or workspace.numel() * workspace.element_size() < need):
        raise ValueError(f"a layer of {tokens} tokens needs a contiguous workspace of {need} bytes")
    _check_status(_b.load().mxfp8_expert_layer(_b._ptr(x), tokens, hidden, ldx, _b._ptr(experts), I64 if experts.dtype == torch.int64 else I32, slots,
                                               _b._ptr(weights), format, _b._ptr(up_q), _b._ptr(up_s), _b._ptr(down_q), _b._ptr(down_s), groups, inter,
                                               _b._ptr(out), _b._dtype_code(out.dtype), ld_out, _b._ptr(workspace), scale_layout, _b._stream(stream)),
                  "mxfp8_expert_layer")


def expert_layer(x, experts, weights, format, up_q, up_s, down_q, down_s, out_dtype=torch.bfloat16, scale_layout=SCALES_ROWMAJOR):
    """Allocate output and workspace and call mxfp8_expert_layer."""
    tokens, hidden = x.shape
    inter = down_q.shape[-1] * (2 if format == WEIGHTS_MXFP4 else 1)
    out = torch.empty((tokens, hidden), dtype=out_dtype, device=x.device)
    workspace = torch.empty((mxfp8_expert_layer_workspace(tokens, experts.shape[1], inter),), dtype=torch.uint8, device=x.device)
    mxfp8_expert_layer(x, experts, weights, format, up_q, up_s, down_q, down_s, out, workspace, scale_layout)
    return out
