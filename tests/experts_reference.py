"""The operators of include/mxfp8_experts.h from their definitions, in numpy: whole numbers exactly, sums in float64."""
import numpy as np

import oracle
from oracle import mxfp4


def plan(experts, groups, align, rows):
    """positions, sources, group_ends, entry by entry."""
    ids = np.asarray(experts).ravel()
    buckets = [[] for _ in range(groups)]
    positions = np.full(ids.size, -1, np.int32)
    sources = np.full(rows, -1, np.int32)
    for i, e in enumerate(ids):
        if 0 <= e < groups:
            buckets[e].append(i)
    ends, at = np.zeros(groups, np.int32), 0
    for e, bucket in enumerate(buckets):
        sources[at:at + len(bucket)] = bucket
        positions[bucket] = np.arange(at, at + len(bucket))
        at += -(-len(bucket) // align) * align
        ends[e] = at
    return positions.reshape(np.shape(experts)), sources, ends


def rows_needed(entries, groups, align):
    return (entries + min(entries, groups) * (align - 1)) // align * align


def product(w, x):
    """w * x of float32 values as FP32 that stands for the exact product in a later rounding: where it is inexact, the neighbour with an
    odd last bit (the product of two float32 is exact in float64). What the nearest value leaves is itself taken in FP32."""
    with np.errstate(over="ignore", invalid="ignore", under="ignore"):
        whole = w.astype(np.float64) * x.astype(np.float64)
        p = (w * x).astype(np.float32)
        rest = (whole - p.astype(np.float64)).astype(np.float32)
    bits = p.view(np.int32)
    move = np.isfinite(p) & (rest != 0) & (bits & 1 == 0)
    return np.where(move, bits + np.where(np.signbit(rest) == np.signbit(p), 1, -1), bits).astype(np.int32).view(np.float32)


def sorted_rows(src, sources, slots, weights=None):
    """FP32 rows as they are quantized; src float32."""
    v = np.zeros((sources.size, src.shape[1]), np.float32)
    given = (sources >= 0) & (sources < src.shape[0] * slots)
    at = sources[given]
    v[given] = src[at // slots]
    if weights is not None:
        v[given] = product(np.broadcast_to(weights.ravel()[at][:, None], v[given].shape), v[given])
    return v


def quantized(v, axis):
    return oracle.quantize_rowwise(v) if axis == "row" else oracle.quantize_colwise(v)


def combine(c, positions, weights=None):
    """(sum, sum of magnitudes) in float64; c float32 or float64."""
    tokens, slots = positions.shape
    out, mag = np.zeros((tokens, c.shape[1])), np.zeros((tokens, c.shape[1]))
    for t in range(tokens):
        for j in range(slots):
            r = positions[t, j]
            if 0 <= r < c.shape[0]:
                x = c[r].astype(np.float64) * (1.0 if weights is None else np.float64(weights[t, j]))
                out[t] += x
                mag[t] += np.abs(x)
    return out, mag


def weight_grad(dy, c, positions):
    tokens, slots = positions.shape
    out, mag = np.zeros((tokens, slots)), np.zeros((tokens, slots))
    for t in range(tokens):
        for j in range(slots):
            r = positions[t, j]
            if 0 <= r < c.shape[0]:
                x = dy[t].astype(np.float64) * c[r].astype(np.float64)
                out[t, j], mag[t, j] = x.sum(), np.abs(x).sum()
    return out, mag


def gemv(x, w_q, w_s):
    """(product, sum of magnitudes) of float32 x with decoded MXFP4 weights."""
    w = mxfp4.dequantize(w_q, w_s)
    x = x.astype(np.float64)
    with np.errstate(invalid="ignore"):
        return x @ w.T, np.abs(x) @ np.abs(w).T


def gemv_grouped(x, sources, slots, w_q, w_s, ends, rows):
    """Rows that belong to no expert are NaN in both."""
    n = w_q.shape[1]
    out, mag = np.full((rows, n), np.nan), np.full((rows, n), np.nan)
    begin = 0
    for e, end in enumerate(ends):
        for r in range(begin, end):
            i = r if sources is None else sources[r]
            if sources is not None and not 0 <= i < x.shape[0] * slots:
                out[r], mag[r] = 0.0, 0.0
                continue
            out[r], mag[r] = (a[0] for a in gemv(x[(i if sources is None else i // slots)][None], w_q[e], w_s[e]))
        begin = max(begin, end)
    return out, mag
