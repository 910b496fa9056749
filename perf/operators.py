"""What a mixture-of-experts layer needs around its grouped products, as cases that can be timed and compared: the sort of
tokens by expert, the sorted and quantized operands, the weighted sum back to tokens, the gradient of its weights, and products
of a few rows with MXFP4 weights (one matrix, or each row with its expert's).

`tokens` rows of activations, each for `slots` experts out of `e`; `align`: what an expert's rows are padded to; `cols`, `n`,
`k`: widths. A token of the padding of a batch belongs to expert -1. `layout` is the layout of the scale bytes.
"""
import math

import torch

own = False

BLOCK = 32
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32, "i32": torch.int32, "i64": torch.int64}
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


def listed():
    return [
        # A few tokens of a running generation: sort without padding, a launch and nothing else.
        {"name": "sort_decode", "op": "sort", "tokens": 6, "slots": 8, "e": 64, "align": 1, "index": "i32"},
        # A training micro-batch of a layer of many small experts, indices as torch.topk gives them.
        {"name": "sort_train", "op": "sort", "tokens": 16384, "slots": 8, "e": 128, "align": 128, "index": "i64"},
        # Operands of the benchmark's mixture-of-experts layer (hidden 2048, 8 experts): forward and weight gradient.
        {"name": "quantize_x", "op": "quantize", "tokens": 8192, "slots": 2, "e": 8, "cols": 2048, "src": "bf16", "weighted": False,
         "axis": "both", "layout": "tiled"},
        # Its FP32 output gradient, times the router's weights, on an unpadded batch of odd length.
        {"name": "quantize_dy_ragged", "op": "quantize", "tokens": 1999, "slots": 2, "e": 8, "cols": 5632, "src": "f32", "weighted": True,
         "axis": "both", "layout": "rowmajor"},
        # Experts' rows back to three tokens of a running generation.
        {"name": "combine_decode", "op": "combine", "tokens": 3, "slots": 8, "e": 64, "cols": 2048, "src": "bf16", "out": "bf16", "weighted": True},
        # The same in training at the benchmark's width.
        {"name": "combine_train", "op": "combine", "tokens": 16384, "slots": 4, "e": 32, "cols": 4096, "src": "bf16", "out": "bf16", "weighted": True},
        # Gradient of the router's weights, an unpadded batch, FP32 output gradient.
        {"name": "weight_grad_ragged", "op": "weight_grad", "tokens": 1003, "slots": 6, "e": 64, "cols": 2880, "dy": "f32", "src": "bf16"},
        # The same for the benchmark's layer.
        {"name": "weight_grad_train", "op": "weight_grad", "tokens": 8192, "slots": 2, "e": 8, "cols": 5632, "dy": "bf16", "src": "bf16"},
        # One token through the QKV layer of an 8B-class model whose weights are kept as MXFP4.
        {"name": "gemv_qkv_one", "op": "gemv", "m": 1, "n": 6144, "k": 4096, "out": "bf16", "layout": "rowmajor"},
        # A dozen tokens through its down-projection: the longest reduction.
        {"name": "gemv_down_12", "op": "gemv", "m": 12, "n": 4096, "k": 14336, "out": "bf16", "layout": "tiled"},
        # One token through the up-projections of its 8 experts out of 64.
        {"name": "experts_one", "op": "experts", "tokens": 1, "slots": 8, "e": 64, "n": 2816, "k": 2048, "out": "bf16", "layout": "rowmajor"},
        # A batch of 48 tokens: nearly every expert has a few rows.
        {"name": "experts_48", "op": "experts", "tokens": 48, "slots": 4, "e": 64, "n": 5632, "k": 2048, "out": "f32", "layout": "tiled"},
    ]


def _size(rng, lo, hi, of=1):
    """A multiple of `of` in [lo, hi], spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / of)) * of))


def draw(rng):
    op = rng.choice(["sort", "quantize", "combine", "weight_grad", "gemv", "experts"])
    layout, out = rng.choice(["rowmajor", "tiled"]), rng.choice(["bf16", "f32"])
    slots = rng.randint(1, 8)
    e = _size(rng, slots, 256)
    if op == "sort":
        return {"op": op, "tokens": _size(rng, 1, 16384), "slots": slots, "e": e, "align": rng.choice([1, 32, 64, 128]), "index": rng.choice(["i32", "i64"])}
    if op == "quantize":
        slots = rng.randint(1, 4)
        return {"op": op, "tokens": _size(rng, 16, 4096), "slots": slots, "e": _size(rng, 4, 32), "cols": _size(rng, 256, 5632, 32),
                "src": rng.choice(["bf16", "f32"]), "weighted": rng.choice([True, False]), "axis": rng.choice(["rowwise", "colwise", "both"]), "layout": layout}
    if op == "combine":
        return {"op": op, "tokens": _size(rng, 1, 8192), "slots": slots, "e": e, "cols": _size(rng, 256, 4096, 32), "src": rng.choice(["bf16", "f32"]),
                "out": out, "weighted": rng.choice([True, False])}
    if op == "weight_grad":
        return {"op": op, "tokens": _size(rng, 1, 8192), "slots": slots, "e": e, "cols": _size(rng, 256, 4096, 32), "dy": rng.choice(["bf16", "f32"]),
                "src": rng.choice(["bf16", "f32"])}
    if op == "gemv":
        return {"op": op, "m": _size(rng, 1, 64), "n": _size(rng, 512, 8192), "k": _size(rng, 512, 14336, 32), "out": out, "layout": layout}
    e = _size(rng, 8, 64)
    return {"op": op, "tokens": _size(rng, 1, 128), "slots": min(slots, e), "e": e, "n": _size(rng, 512, 2816, 32), "k": _size(rng, 512, 2048, 32), "out": out,
            "layout": layout}


# ---- inputs --------------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _activations(g, rows, cols, dtype):
    """N(0, 1) times a lognormal gain per channel, a few outlier channels 50 times larger."""
    gain = torch.exp(torch.randn(cols, generator=g, device="cuda"))
    gain[torch.randperm(cols, generator=g, device="cuda")[: max(1, cols // 1000)]] *= 50.0
    return (torch.randn((rows, cols), generator=g, device="cuda") * gain).to(dtype)


def _gradients(g, rows, cols, dtype):
    """N(0, 1e-3), 0.5 % of the entries 100 times larger."""
    x = 1e-3 * torch.randn((rows, cols), generator=g, device="cuda")
    x[torch.rand((rows, cols), generator=g, device="cuda") < 0.005] *= 100.0
    return x.to(dtype)


def _routing(g, tokens, slots, e):
    """Experts [tokens x slots] of a router with favourites, and its weights (softmax over the chosen). From 64 tokens on one
    in fifty is padding."""
    logits = torch.randn((tokens, e), generator=g, device="cuda") + 0.5 * torch.randn(e, generator=g, device="cuda")
    top = torch.topk(logits, slots, dim=1)
    experts = top.indices
    if tokens >= 64:
        experts = torch.where(torch.rand((tokens, 1), generator=g, device="cuda") < 0.02, torch.full_like(experts, -1), experts)
    return experts, torch.softmax(top.values, dim=1)


def _mxfp4_weights(g, *shape):
    """Codes and scale bytes of weights N(0, 0.02): [.. x n x k/2] and [.. x n x k/32]. Scales of such blocks are 2^-6 or 2^-7."""
    q = torch.randint(0, 256, (*shape[:-1], shape[-1] // 2), dtype=torch.uint8, generator=g, device="cuda")
    s = 120 + torch.randint(0, 2, (*shape[:-1], shape[-1] // BLOCK), dtype=torch.uint8, generator=g, device="cuda")
    return q, s


def _rows(entries, e, align):
    """Rows that the sorted entries take at most."""
    return (entries + min(entries, e) * (align - 1)) // align * align


def _plan(experts, e, align, rows):
    """positions [entries], sources [rows] and ends [e] of the entries sorted by expert, each expert's padded to `align` rows."""
    ids = experts.reshape(-1).long()
    n = ids.numel()
    key = torch.where((ids >= 0) & (ids < e), ids, e)
    order = torch.argsort(key, stable=True)
    counts = torch.zeros(e + 1, dtype=torch.int64, device=ids.device).index_add_(0, key, torch.ones_like(key))
    padded = (counts + align - 1) // align * align
    ends = torch.cumsum(padded, 0)
    sorted_key = key[order]
    rank = torch.arange(n, device=ids.device) - (torch.cumsum(counts, 0) - counts)[sorted_key]
    at = (ends - padded)[sorted_key] + rank
    here = sorted_key < e
    positions = torch.empty_like(ids).index_copy_(0, order, torch.where(here, at, -1))
    sources = torch.full((rows + 1,), -1, dtype=torch.int64, device=ids.device)
    sources.index_copy_(0, torch.where(here, at, rows), order)
    return positions.int(), sources[:rows].int(), ends[:e].int()


def _tile(s):
    """Scale bytes [rows x blocks] in the tiled layout: dwords of four blocks, 64 rows of them together."""
    rows, nb = s.shape[-2:]
    s = torch.nn.functional.pad(s, (0, -nb % 4, 0, -rows % 64))
    return s.reshape(*s.shape[:-2], s.shape[-2] // 64, 64, s.shape[-1] // 4, 4).transpose(-3, -2).reshape(-1)


def _untile(s, groups, rows, nb):
    s = s.reshape(groups, (rows + 63) // 64, (nb + 3) // 4, 64, 4).transpose(2, 3)
    return s.reshape(groups, (rows + 63) // 64 * 64, -1)[:, :rows, :nb]


def prepare(case, seed):
    g, op = _generator(seed), case["op"]
    s = {k: v for k, v in case.items() if k != "name"}
    if op in ("gemv", "experts"):
        e, n, k = case.get("e", 1), case["n"], case["k"]
        s["w_q"], scales = _mxfp4_weights(g, e, n, k)
        s["w_s"] = _tile(scales) if case["layout"] == "tiled" else scales
        rows = case["m"] if op == "gemv" else case["tokens"]
        s["x"] = _activations(g, rows, k, torch.bfloat16)
        if op == "gemv":
            s["w_q"] = s["w_q"][0]
            s["w_s"] = s["w_s"] if case["layout"] == "tiled" else s["w_s"][0]
        else:
            rows *= case["slots"]
            s["experts"], _ = _routing(g, case["tokens"], case["slots"], e)
            s["positions"], s["sources"], s["ends"] = _plan(s["experts"], e, 1, rows)
        s["c"] = torch.zeros((rows, n), dtype=DTYPE[case["out"]], device="cuda")
        return s
    tokens, slots, e = case["tokens"], case["slots"], case["e"]
    experts, weights = _routing(g, tokens, slots, e)
    align = case.get("align", 128)
    rows = _rows(tokens * slots, e, align)
    if op == "sort":
        s["experts"] = experts.to(DTYPE[case["index"]])
        s.update(positions=torch.empty((tokens, slots), dtype=torch.int32, device="cuda"), sources=torch.empty(rows, dtype=torch.int32, device="cuda"),
                 ends=torch.empty(e, dtype=torch.int32, device="cuda"), rows=rows)
        s["workspace"] = torch.empty(4 * e * (tokens * slots // 1024 + 1), dtype=torch.uint8, device="cuda")  # a count per 1024 entries and expert
        return s
    positions, s["sources"], s["ends"] = _plan(experts, e, align, rows)
    s["positions"] = positions.reshape(tokens, slots)
    if op == "quantize":
        cols = case["cols"]
        s["x"] = _activations(g, tokens, cols, torch.bfloat16) if case["src"] == "bf16" else _gradients(g, tokens, cols, torch.float32)
        s["weights"] = weights if case["weighted"] else None
        u8 = dict(dtype=torch.uint8, device="cuda")
        if case["axis"] != "colwise":
            s["q_row"] = torch.zeros((rows, cols), **u8)
            s["s_row"] = torch.zeros((rows, cols // BLOCK), **u8)
        if case["axis"] != "rowwise":
            s["q_colT"] = torch.zeros((cols, rows), **u8)
            s["s_colT"] = torch.zeros((cols, rows // BLOCK), **u8)
        if case["layout"] == "tiled":
            s.update({name: _tile(s[name]) for name in ("s_row", "s_colT") if name in s})
        return s
    s["y"] = _activations(g, rows, case["cols"], DTYPE[case["src"]])
    if op == "combine":
        s["weights"] = weights if case["weighted"] else None
        s["out_rows"] = torch.empty((tokens, case["cols"]), dtype=DTYPE[case["out"]], device="cuda")
    else:
        s["dy_rows"] = _gradients(g, tokens, case["cols"], DTYPE[case["dy"]])
        s["dw"] = torch.empty((tokens, slots), dtype=torch.float32, device="cuda")
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------

def _own(s):
    import paper_2506_08027_amd as mx
    op = s["op"]
    layout = mx.SCALES_TILED if s.get("layout") == "tiled" else mx.SCALES_ROWMAJOR
    if op == "sort":
        mx.mxfp8_expert_sort(s["experts"], s["align"], s["positions"], s["sources"], s["ends"], s["workspace"])
        return [s["positions"], s["sources"], s["ends"]]
    if op == "quantize":
        copies = {name: s[name] for name in ("q_row", "s_row", "q_colT", "s_colT") if name in s}
        mx.mxfp8_expert_quantize_ex(s["x"], s["sources"], s["ends"], s["slots"], s["weights"], s["axis"], **copies, scale_layout=layout)
        return {name: v.view(torch.float8_e4m3fn if name[0] == "q" else torch.float8_e8m0fnu) for name, v in copies.items()}
    if op == "combine":
        mx.mxfp8_expert_combine(s["y"], s["positions"], s["weights"], s["out_rows"])
        return s["out_rows"]
    if op == "weight_grad":
        mx.mxfp8_expert_weight_grad(s["dy_rows"], s["y"], s["positions"], s["dw"])
        return s["dw"]
    if op == "gemv":
        mx.mxfp8_fp4_gemv_ex(s["x"], s["w_q"], s["w_s"], s["c"], layout)
        return s["c"]
    mx.mxfp8_fp4_gemv_grouped_ex(s["x"], s["sources"], s["slots"], s["w_q"], s["w_s"], s["ends"], s["c"], layout)
    return s["c"]


def _quantize_rows(v):
    """E4M3 values and scale exponents + 127 of FP32 v along its rows: the scale is the smallest power of two that keeps a block's
    largest magnitude within 448 (0.875 times 2^9)."""
    blocks = v.reshape(v.shape[0], -1, BLOCK)
    fraction, exponent = torch.frexp(blocks.abs().amax(-1))
    exponent = torch.where(fraction == 0, -127, exponent - 9 + (fraction > 0.875).int()).clamp(-127, 127)
    q = torch.ldexp(blocks, -exponent[..., None]).to(torch.float8_e4m3fn)
    return q.reshape(v.shape), (exponent + 127).to(torch.uint8)


def _dequantized_mxfp4(q, s):
    """FP32 values of codes [e x n x k/2] with scale bytes [e x n x k/32]."""
    value = torch.tensor(E2M1, device=q.device)
    pairs = torch.stack([value[(q & 15).int()], value[(q >> 4).int()]], -1)
    return (pairs.reshape(*s.shape, BLOCK) * torch.exp2(s.float() - 127)[..., None]).reshape(*q.shape[:-1], -1)


def run(s):
    if own:
        return _own(s)
    op = s["op"]
    if op == "sort":
        positions, sources, ends = _plan(s["experts"], s["e"], s["align"], s["rows"])
        return [positions.reshape(s["experts"].shape), sources, ends]
    if op == "quantize":
        src = s["sources"].long()
        v = s["x"].float()[src.clamp(min=0) // s["slots"]]
        if s["weights"] is not None:
            v = v * s["weights"].reshape(-1, 1)[src.clamp(min=0)]
        v = torch.where(src[:, None] >= 0, v, 0.0)
        out = {}
        if s["axis"] != "colwise":
            out["q_row"], out["s_row"] = _quantize_rows(v)
        if s["axis"] != "rowwise":
            out["q_colT"], out["s_colT"] = _quantize_rows(v.t().contiguous())
        for name in ("s_row", "s_colT"):
            if name in out:
                out[name] = (_tile(out[name]) if s["layout"] == "tiled" else out[name]).view(torch.float8_e8m0fnu)
        return out
    if op in ("combine", "weight_grad"):
        at = s["positions"].long()
        rows = torch.where(at[..., None] >= 0, s["y"].float()[at.clamp(min=0)], 0.0)
        if op == "combine":
            return (rows if s["weights"] is None else rows * s["weights"][..., None]).sum(1).to(DTYPE[s["out"]])
        return (rows * s["dy_rows"].float()[:, None, :]).sum(-1)
    e, n, k, x = s.get("e", 1), s["n"], s["k"], s["x"].float()
    scales = _untile(s["w_s"], e, n, k // BLOCK) if s["layout"] == "tiled" else s["w_s"].reshape(e, n, -1)
    codes = s["w_q"].reshape(e, n, -1)
    if op == "gemv":
        return (x @ _dequantized_mxfp4(codes, scales)[0].t()).to(DTYPE[s["out"]])
    tokens, ids, at = s["tokens"], s["experts"].reshape(-1), s["positions"].long()
    here = (ids >= 0).nonzero()[:, 0] if tokens >= 64 else torch.arange(ids.numel(), device=ids.device)
    ids, at = ids[here], at[here]
    if ids.numel() <= e:  # few rows: each row's weights, instead of all experts'
        c = torch.bmm(_dequantized_mxfp4(codes[ids], scales[ids]), x[here // s["slots"], :, None])[..., 0]
        return torch.zeros_like(s["c"]).index_copy_(0, at, c.to(DTYPE[s["out"]]))
    # each expert's rows at the front of a place for all tokens: a token has an expert once at most
    w = _dequantized_mxfp4(codes, scales)
    begin = torch.nn.functional.pad(s["ends"].long(), (1, 0))
    place = ids * tokens + at - begin[ids]
    given = torch.zeros((e * tokens, k), device=x.device).index_copy_(0, place, x[here // s["slots"]])
    c = torch.bmm(given.reshape(e, tokens, k), w.transpose(1, 2).contiguous()).reshape(e * tokens, n)
    return torch.zeros_like(s["c"]).index_copy_(0, at, c[place].to(DTYPE[s["out"]]))


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    op = case["op"]
    esize = {"bf16": 2, "f32": 4, "i32": 4, "i64": 8}
    if op == "gemv":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": n * k * (1 / 2 + 1 / BLOCK) + m * k * 2 + m * n * esize[case["out"]], "flops": 2 * m * n * k}
    tokens, entries = case["tokens"], case["tokens"] * case["slots"]
    if op == "experts":  # an expert's weights are read where a token has chosen it
        e, n, k = case["e"], case["n"], case["k"]
        chosen = e * (1 - (1 - case["slots"] / e) ** tokens)
        return {"bytes": chosen * n * k * (1 / 2 + 1 / BLOCK) + tokens * k * 2 + entries * n * esize[case["out"]], "flops": 2 * entries * n * k}
    if op == "sort":
        return {"bytes": entries * (esize[case["index"]] + 4) + 4 * _rows(entries, case["e"], case["align"]) + 4 * case["e"], "flops": 0}
    cols = case["cols"]
    if op == "quantize":  # the entries alone, without their padding
        return {"bytes": tokens * cols * esize[case["src"]] + entries * cols * (1 + 1 / BLOCK) * (2 if case["axis"] == "both" else 1) + 8 * entries,
                "flops": entries * cols * (1 if case["weighted"] else 0)}
    other = tokens * cols * esize[case["out"] if op == "combine" else case["dy"]]
    return {"bytes": entries * cols * esize[case["src"]] + other + 8 * entries, "flops": 2 * entries * cols}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------

def _exact_rows(v):
    """E4M3 values and scales of the rows of v, all in 64 bits: 2^n with the smallest n such that no magnitude exceeds 448 * 2^n,
    then the nearest multiple of the spacing 2^-3 of the binade (of 2^-9 below 2^-6), ties to the even one."""
    amax = v.reshape(v.shape[0], -1, BLOCK).abs().amax(-1)
    power = torch.full_like(amax, -127.0)
    for step in (128, 64, 32, 16, 8, 4, 2, 1):  # the largest n that is still too small, plus one
        power = torch.where(amax > 448.0 * torch.exp2(power + step - 1), power + step, power)
    scale = torch.exp2(power.clamp(max=127.0))
    t = v / scale.repeat_interleave(BLOCK, 1)
    spacing = torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(t / spacing) * spacing, scale


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "sort":
        return None
    if op in ("gemv", "experts"):
        e, n, k = case.get("e", 1), case["n"], case["k"]
        codes = s["w_q"].reshape(e, n, k // 2)
        scales = s["w_s"].reshape(e, n, k // BLOCK) if case["layout"] == "rowmajor" else None
        if scales is None:
            r, b = torch.arange(n, device="cuda")[:, None], torch.arange(k // BLOCK, device="cuda")[None, :]
            groups = (k // BLOCK + 3) // 4
            scales = s["w_s"].reshape(e, -1)[:, ((r // 64 * groups + b // 4) * 64 + r % 64) * 4 + b % 4]
        value = torch.tensor(E2M1, dtype=torch.float64, device="cuda")
        out = torch.zeros(s["c"].shape, dtype=torch.float64, device="cuda")
        begin = 0
        for i, end in enumerate([out.shape[0]] if op == "gemv" else s["ends"].tolist()):
            if end > begin:
                w = torch.empty((n, k), dtype=torch.float64, device="cuda")
                w[:, 0::2], w[:, 1::2] = value[(codes[i] & 15).long()], value[(codes[i] >> 4).long()]
                w *= torch.pow(2.0, scales[i].double() - 127).repeat_interleave(BLOCK, 1)
                rows = s["x"] if op == "gemv" else s["x"][s["sources"][begin:end].long() // case["slots"]]
                out[begin:end] = rows.double() @ w.t()
            begin = end
        return out
    if op == "quantize":
        src = s["sources"].long()
        v = torch.zeros((src.numel(), case["cols"]), dtype=torch.float64, device="cuda")
        filled = (src >= 0).nonzero()[:, 0]
        v[filled] = s["x"].double()[src[filled] // case["slots"]]
        if case["weighted"]:
            v[filled] *= s["weights"].double().reshape(-1)[src[filled]][:, None]
        out = {}
        for axis, a in (("row", v), ("colT", v.t())):
            if "q_" + axis in s:
                q, scale = _exact_rows(a.contiguous())
                if case["layout"] == "tiled":
                    r, nb = scale.shape
                    tiled = torch.full(((r + 63) // 64, (nb + 3) // 4, 64, 4), 2.0 ** -127, dtype=torch.float64, device="cuda")
                    i, b = torch.arange(r, device="cuda")[:, None], torch.arange(nb, device="cuda")[None, :]
                    tiled[i // 64, b // 4, i % 64, b % 4] = scale
                    scale = tiled.reshape(-1)
                out.update({"q_" + axis: q, "s_" + axis: scale})
        return out
    at = s["positions"].long()
    total = []
    for j in range(case["slots"]):
        there = (at[:, j] >= 0).nonzero()[:, 0]
        if op == "combine":
            if not total:
                total.append(torch.zeros((case["tokens"], case["cols"]), dtype=torch.float64, device="cuda"))
            w = s["weights"][there, j].double()[:, None] if case["weighted"] else 1.0
            total[0][there] += w * s["y"][at[there, j]].double()
        else:
            dw = torch.zeros(case["tokens"], dtype=torch.float64, device="cuda")
            dw[there] = (s["dy_rows"][there].double() * s["y"][at[there, j]].double()).sum(1)
            total.append(dw)
    return total[0] if op == "combine" else torch.stack(total, 1)
