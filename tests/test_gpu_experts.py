"""GPU parity of the expert rows (include/mxfp8_experts.h): the sort by expert, the quantizer of sorted rows, the weighted sum and
the gradient of its weights against their definitions, and a whole mixture-of-experts layer, forward and backward. Sums are held to
what roundings of their length can amount to: u = 2^-24 an addition or fused multiply-add in FP32, half a step (2^-8 relative) for BF16."""
import numpy as np
import pytest
import torch

import experts_reference as ref
import oracle
import paper_2506_08027_amd as mx
import scale_layout as sl
from mfma_model import hw_tolerance
from paper_2506_08027_amd import synth_inputs as si

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _dev(a):
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16)).cuda().view(torch.bfloat16)
    return torch.from_numpy(a).cuda()


def _host(t):
    t = t.contiguous()
    if t.dtype == torch.bfloat16:
        return si.bf16_bits_to_f32(t.view(torch.int16).cpu().numpy().view(np.uint16))
    return t.cpu().numpy()


def _values(rng, rows, cols, bf16):
    """(device tensor, the same values as float32)"""
    x = (rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal(cols))).astype(np.float32)
    if not bf16:
        return _dev(x), x
    bits = si.to_bf16_bits(x)
    return _dev(bits), si.bf16_bits_to_f32(bits)


def _experts(rng, tokens, slots, groups, dropped=0.1):
    """Uneven choices, some out of range on either side."""
    if not groups:
        return rng.integers(-2, 3, (tokens, slots))
    e = np.minimum((rng.random((tokens, slots)) ** 2 * groups).astype(np.int64), groups - 1)
    drop = rng.random((tokens, slots))
    e[drop < dropped / 2] = -1 - rng.integers(0, 2 ** 20)
    e[drop > 1 - dropped / 2] = groups + rng.integers(0, 2 ** 20)
    return e


def _sort(experts, groups, align, extra_rows=0, index64=False):
    entries = experts.size
    rows = mx.mxfp8_expert_rows(entries, groups, align) + extra_rows
    i32 = dict(dtype=torch.int32, device="cuda")
    out = [torch.full(experts.shape, -7, **i32), torch.full((rows,), -7, **i32), torch.full((groups,), -7, **i32)]
    workspace = torch.full((max(mx.mxfp8_expert_sort_workspace(entries, groups), 1),), 0xA5, dtype=torch.uint8, device="cuda")
    mx.mxfp8_expert_sort(_dev(experts.astype(np.int64 if index64 else np.int32)), align, *out, workspace)
    torch.cuda.synchronize()
    return out


def _check_sort(experts, groups, align, extra_rows=0, index64=False):
    got = _sort(experts, groups, align, extra_rows, index64)
    want = ref.plan(experts, groups, align, got[1].numel())
    for g, w, name in zip(got, want, ("positions", "sources", "group_ends")):
        assert np.array_equal(_host(g), w), name


# ---- sort ------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("index64", [False, True], ids=["i32", "i64"])
@pytest.mark.parametrize("tokens,slots,groups,align", [(1, 1, 1, 1), (1, 8, 64, 1), (5, 3, 7, 32), (37, 2, 5, 128), (64, 4, 64, 64), (255, 1, 200, 1),
                                                       (257, 1, 3, 4), (300, 8, 1000, 2), (1, 5, 4096, 16)])
def test_sort_is_the_definition(tokens, slots, groups, align, index64):
    _check_sort(_experts(np.random.default_rng(tokens + groups), tokens, slots, groups), groups, align, extra_rows=37, index64=index64)


@pytest.mark.parametrize("entries,kind", [(512, "one"), (512, "none"), (300, "each"), (0, "none"), (1024, "last"), (1025, "one")])
def test_sort_of_extreme_choices(entries, kind):
    e = {"one": np.zeros(entries, np.int64), "none": np.full(entries, -1, np.int64), "each": np.arange(entries) % 16,
         "last": np.full(entries, 15, np.int64)}[kind].reshape(-1, 1)
    _check_sort(e, 16, 32)
    _check_sort(e, 16, 1, extra_rows=3)


def test_sort_without_experts_and_of_wide_numbers():
    _check_sort(np.array([[0, -1, 2 ** 31 - 1]]), 0, 1, extra_rows=5)
    e = np.array([[0, 2 ** 32, 2 ** 32 + 1, -2 ** 63, 2 ** 63 - 1, 1]], np.int64)   # their low words would be experts 0 and 1
    _check_sort(e, 2, 4, index64=True)


@pytest.mark.parametrize("index64", [False, True], ids=["i32", "i64"])
@pytest.mark.parametrize("entries,groups,align", [(8192, 64, 1), (8193, 64, 128), (8200, 4096, 2), (300, 256, 128), (32768, 256, 128), (32769, 96, 64), (131072, 128, 128), (40000, 4096, 1), (70001, 1, 32), (524288, 256, 128)])
def test_sort_full_size(entries, groups, align, index64):
    _check_sort(_experts(np.random.default_rng(entries), entries, 1, groups), groups, align, 11, index64)


def test_sort_of_many_entries_without_experts_full_size():
    """Each entry is looked at once, as with an expert, not once by each of the 8192 workgroups (tens of milliseconds)."""
    experts = torch.zeros((1 << 23, 1), dtype=torch.int32, device="cuda")
    took = []
    for groups in (1, 0, 1, 0):
        plan = mx.expert_sort(experts, groups, 1)
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        mx.expert_sort(experts, groups, 1)
        end.record()
        torch.cuda.synchronize()
        took.append(start.elapsed_time(end))
    assert (plan["positions"] == -1).all() and (plan["sources"] == -1).all()
    assert took[3] < 8 * took[2], took


# ---- quantizer of sorted rows -------------------------------------------------------------------------------------------------

def _check_quantize(src, src32, experts, groups, align, slots, weights, axis, tiled, extra_rows=0, rows=None, whole=False):
    tokens, cols = src32.shape
    rows = rows or (ref.rows_needed(experts.size, groups, align) + extra_rows + 31) // 32 * 32
    _, sources, ends = ref.plan(experts, groups, align, rows)
    lay = mx.SCALES_TILED if tiled else mx.SCALES_ROWMAJOR
    shapes = {"row": (rows, cols), "colT": (cols, rows)}
    out = {}
    for name, (r, c) in shapes.items():
        if axis == "both" or axis == {"row": "rowwise", "colT": "colwise"}[name]:
            out["q_" + name] = torch.full((r, c), 0xA5, dtype=torch.uint8, device="cuda")
            out["s_" + name] = torch.full((mx.mxfp8_scale_bytes(r, c, lay),) if tiled else (r, c // 32), 0xA5, dtype=torch.uint8, device="cuda")
    mx.mxfp8_expert_quantize_ex(src, _dev(sources), None if whole else _dev(ends), slots, None if weights is None else _dev(weights), axis, **out,
                                scale_layout=lay)
    torch.cuda.synchronize()
    v = ref.sorted_rows(src32, sources, slots, weights)
    live = rows if whole else min(rows, -(-int(ends[-1]) // 128) * 128)
    for name in ("row", "colT"):
        if "q_" + name not in out:
            continue
        q, s = ref.quantized(v, name)
        got_q, got_s = out["q_" + name].cpu().numpy(), out["s_" + name].cpu().numpy()
        if tiled:
            got_s = sl.untile(got_s, *s.shape)
        if name == "colT":
            q, s, got_q, got_s = q.T, np.repeat(s, 32, 1).T, got_q.T, np.repeat(got_s, 32, 1).T
        assert np.array_equal(got_q[:live], q[:live]) and np.array_equal(got_s[:live], s[:live]), name
        assert (got_q[live:] == 0xA5).all(), "rows behind the last tile were written"
        assert (got_s[live:] == 0xA5).all(), "scales behind the last tile were written"


@pytest.mark.parametrize("tiled", [False, True], ids=["rowmajor", "tiled"])
@pytest.mark.parametrize("bf16", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("weighted", [False, True], ids=["plain", "weighted"])
@pytest.mark.parametrize("axis", ["rowwise", "colwise", "both"])
def test_quantize_of_sorted_rows_is_the_quantizer_of_those_rows(axis, weighted, bf16, tiled):
    rng = np.random.default_rng(3)
    tokens, slots, groups, cols = 45, 3, 6, 160
    src, src32 = _values(rng, tokens, cols, bf16)
    w = rng.random((tokens, slots)).astype(np.float32) if weighted else None
    _check_quantize(src, src32, _experts(rng, tokens, slots, groups), groups, 64 if tiled else 32, slots, w, axis, tiled, extra_rows=256)


@pytest.mark.parametrize("bf16", [False, True], ids=["f32", "bf16"])
def test_quantize_of_special_values(bf16):
    """Every special block of the format, infinities and NaN in rows that are taken and in rows that no entry names, and weights that make
    FP32 subnormals, infinities and zeros."""
    x = si.tiny_with_specials(256, seed=0)
    bits = si.to_bf16_bits(x)
    src, src32 = (_dev(bits), si.bf16_bits_to_f32(bits)) if bf16 else (_dev(x), np.asarray(x, np.float32))
    e = np.zeros((256, 1), np.int64)
    e[5::7] = -1                                     # their rows hold special blocks too
    for weights in (None, np.float32(2.0) ** np.random.default_rng(1).integers(-140, 100, (256, 1)), np.zeros((256, 1))):
        _check_quantize(src, src32, e, 2, 32, 1, None if weights is None else weights.astype(np.float32), "both", False, extra_rows=64)


def test_quantize_padded_source_rows_one_token_and_no_entry():
    rng = np.random.default_rng(9)
    buf = torch.full((40, 128), float("nan"), device="cuda")
    _, src32 = _values(rng, 40, 96, False)
    buf[:, :96] = _dev(src32)
    _check_quantize(buf[:, :96], src32, _experts(rng, 40, 2, 4), 4, 32, 2, None, "both", False)
    _check_quantize(buf[:1, :96], src32[:1], np.array([[1, 3]]), 4, 32, 2, None, "both", True)
    _check_quantize(buf[:, :96], src32, np.full((40, 2), -1), 4, 32, 2, None, "both", False, rows=96)            # nothing is written
    _check_quantize(buf[:, :96], src32, np.full((40, 2), -1), 4, 32, 2, None, "both", False, rows=96, whole=True)  # all rows are zeros
    _check_quantize(buf[:, :96], src32, _experts(rng, 40, 2, 4), 4, 32, 2, None, "both", False, extra_rows=200, whole=True)


def test_quantize_rounds_the_exact_product_once():
    """Products next to a border of the conversion, where FP32's nearest value lies on the other side or on the border itself: the
    result is that of the exact product (taken apart here in whole numbers)."""
    rng = np.random.default_rng(17)
    cols, n = 64, 4096
    near = (1 + (2 * rng.integers(0, 8, n) + 1) / 16) * 2.0 ** rng.integers(-3, 4, n)     # midway between two E4M3 values
    w = (1 + rng.random(n)).astype(np.float32)
    x = np.nextafter((near / w).astype(np.float32), np.float32(100) * rng.choice([-1, 1], n).astype(np.float32))
    src = np.zeros((n, cols), np.float32)
    src[:, 0], src[:, 32] = x, x
    src[:, 1] = np.float32(400) / w                                                        # a block maximum of about 400: scale 1
    src[:, 33] = x * 0.5
    q, s = (torch.empty((n, c), dtype=torch.uint8, device="cuda") for c in (cols, 2))
    mx.mxfp8_expert_quantize_ex(_dev(src), _dev(np.arange(n, dtype=np.int32)), None, 1, _dev(w[:, None]), "rowwise", q, s)
    torch.cuda.synchronize()
    exact = src.astype(np.float64) * w.astype(np.float64)[:, None]                         # 48 bits: exact
    scale = np.repeat(np.exp2(s.cpu().numpy().astype(np.float64) - 127), 32, 1)
    assert (s.cpu().numpy()[:, 0] == 127).all()
    t = exact / scale
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(t), 2.0 ** -6))) - 3)
    want = np.round(t / step) * step                                                       # ties to even; all of it exact in float64
    got = oracle.dequantize(q.cpu().numpy(), s.cpu().numpy(), "f64") / scale
    assert np.array_equal(got, want)
    twice = (src * w[:, None]).astype(np.float64) / scale
    assert (np.round(twice / step) * step != want).sum() > 0, "the inputs do not reach a border"


def test_quantize_of_no_tokens_writes_zeros():
    out = {k: torch.full(s, 0xA5, dtype=torch.uint8, device="cuda") for k, s in (("q_row", (64, 96)), ("s_row", (64, 3)), ("q_colT", (96, 64)), ("s_colT", (96, 2)))}
    for weights in (None, torch.empty((0, 2), device="cuda")):
        mx.mxfp8_expert_quantize_ex(torch.empty((0, 96), device="cuda"), _dev(np.zeros(64, np.int32)), None, 2, weights, "both", **out)
        torch.cuda.synchronize()
        assert all((v.cpu() == 0).all() for v in out.values())


def test_quantize_takes_bad_plans_without_leaving_its_buffers():
    rng = np.random.default_rng(4)
    src, src32 = _values(rng, 10, 64, False)
    sources = np.array([0, 19, 20, 21, 2 ** 31 - 1, -2 ** 31, -5, 7] * 4, np.int32)
    for end in (-3, 0, 32, 1 << 30):
        q = torch.full((32, 64), 0xA5, dtype=torch.uint8, device="cuda")
        s = torch.full((32, 2), 0xA5, dtype=torch.uint8, device="cuda")
        mx.mxfp8_expert_quantize_ex(src, _dev(sources), _dev(np.array([end], np.int32)), 2, None, "rowwise", q, s)
        torch.cuda.synchronize()
        want = oracle.quantize_rowwise(ref.sorted_rows(src32, sources, 2)) if end > 0 else (np.full((32, 64), 0xA5), np.full((32, 2), 0xA5))
        assert np.array_equal(q.cpu().numpy(), want[0]) and np.array_equal(s.cpu().numpy(), want[1])


@pytest.mark.parametrize("tokens,slots,groups,cols,bf16,weighted", [(2048, 2, 8, 2048, True, False), (999, 2, 8, 5632, False, True)])
def test_quantize_full_size(tokens, slots, groups, cols, bf16, weighted):
    rng = np.random.default_rng(tokens)
    src, src32 = _values(rng, tokens, cols, bf16)
    w = rng.random((tokens, slots)).astype(np.float32) if weighted else None
    _check_quantize(src, src32, _experts(rng, tokens, slots, groups, 0.02), groups, 128, slots, w, "both", bf16)


# ---- back to the tokens ----------------------------------------------------------------------------------------------------------

def _positions(rng, tokens, slots, rows):
    p = rng.integers(-1, rows, (tokens, slots)).astype(np.int32)
    if tokens > 2:
        p[1] = -1                                     # a token without any row
        p[2, 0] = rows + 3                            # outside: adds nothing
    return p


def _check_combine(rng, tokens, slots, rows, cols, c_bf16, out_bf16, weighted, pad=0):
    big, big32 = _values(rng, rows, cols + pad, c_bf16)
    c, c32 = big[:, :cols], big32[:, :cols]
    p = _positions(rng, tokens, slots, rows)
    w = rng.standard_normal((tokens, slots)).astype(np.float32) if weighted else None
    if weighted:
        w[p < 0] = np.nan                             # the weight of a dropped entry is not looked at
    out = torch.full((tokens, cols + pad), float("nan"), dtype=torch.bfloat16 if out_bf16 else torch.float32, device="cuda")
    mx.mxfp8_expert_combine(c, _dev(p), None if w is None else _dev(w), out[:, :cols])
    torch.cuda.synchronize()
    want, mag = ref.combine(c32, p, w)
    got = _host(out).astype(np.float64)
    assert np.isnan(got[:, cols:]).all()
    bound = slots * U * 1.01 * mag + (2.0 ** -8 * 1.01 * np.abs(want) if out_bf16 else 0.0) + 1e-37
    assert (np.abs(got[:, :cols] - want) <= bound).all()


@pytest.mark.parametrize("c_bf16", [False, True], ids=["c-f32", "c-bf16"])
@pytest.mark.parametrize("out_bf16", [False, True], ids=["out-f32", "out-bf16"])
@pytest.mark.parametrize("weighted", [False, True], ids=["plain", "weighted"])
@pytest.mark.parametrize("tokens,slots,rows,cols,pad", [(1, 1, 1, 32, 0), (3, 8, 11, 544, 32), (17, 5, 40, 96, 64), (4, 2, 9, 1, 0), (5, 3, 7, 83, 0), (3, 2, 8, 517, 3),
                                                     (4, 3, 5, 1043, 5)])
def test_combine_is_the_weighted_sum(tokens, slots, rows, cols, pad, weighted, out_bf16, c_bf16):
    _check_combine(np.random.default_rng(tokens), tokens, slots, rows, cols, c_bf16, out_bf16, weighted, pad)


def test_combine_without_rows_and_with_infinities():
    out = torch.full((3, 64), 5.0, device="cuda")
    mx.mxfp8_expert_combine(torch.empty((0, 64), device="cuda"), _dev(np.zeros((3, 2), np.int32)), None, out)
    c = torch.full((4, 64), float("inf"), device="cuda")
    c[1] = 2.0
    c[2] = float("nan")
    out2 = torch.empty((3, 64), device="cuda")
    mx.mxfp8_expert_combine(c, _dev(np.array([[1, -1], [0, 1], [1, 1]], np.int32)), _dev(np.array([[3.0, np.inf], [1.0, 1.0], [1.0, 0.5]], np.float32)), out2)
    torch.cuda.synchronize()
    assert (_host(out) == 0.0).all()
    assert (_host(out2)[0] == 6.0).all() and np.isposinf(_host(out2)[1]).all() and (_host(out2)[2] == 3.0).all()


@pytest.mark.parametrize("tokens,slots,cols,c_bf16", [(1500, 4, 4096, True), (2000, 2, 2048, False)])
def test_combine_full_size(tokens, slots, cols, c_bf16):
    _check_combine(np.random.default_rng(tokens), tokens, slots, tokens * slots, cols, c_bf16, True, True)


def _check_weight_grad(rng, tokens, slots, rows, cols, dy_bf16, c_bf16, pad=0):
    big_c, big_c32 = _values(rng, rows, cols + pad, c_bf16)
    big_dy, big_dy32 = _values(rng, tokens, cols + pad, dy_bf16)
    p = _positions(rng, tokens, slots, rows)
    dw = torch.full((tokens, slots), float("nan"), device="cuda")
    mx.mxfp8_expert_weight_grad(big_dy[:, :cols], big_c[:, :cols], _dev(p), dw)
    torch.cuda.synchronize()
    want, mag = ref.weight_grad(big_dy32[:, :cols], big_c32[:, :cols], p)
    adds = 8 * -(-cols // 512) + 16                    # a lane's own products, then the lanes' and wavefronts' sums
    assert (np.abs(_host(dw) - want) <= adds * U * 1.01 * mag + 1e-37).all()


@pytest.mark.parametrize("dy_bf16", [False, True], ids=["dy-f32", "dy-bf16"])
@pytest.mark.parametrize("c_bf16", [False, True], ids=["c-f32", "c-bf16"])
@pytest.mark.parametrize("tokens,slots,rows,cols,pad", [(1, 1, 1, 32, 0), (3, 8, 11, 1056, 32), (17, 5, 40, 96, 64), (4, 2, 9, 1, 0), (5, 3, 7, 83, 0), (3, 2, 8, 517, 3),
                                                     (4, 3, 5, 1043, 5)])
def test_weight_grad_is_the_dot_product(tokens, slots, rows, cols, pad, c_bf16, dy_bf16):
    _check_weight_grad(np.random.default_rng(tokens), tokens, slots, rows, cols, dy_bf16, c_bf16, pad)


def test_weight_grad_of_whole_numbers_is_exact_and_the_difference_quotient():
    """Small whole numbers: every product and sum is exact in FP32. combine is linear in its weights, so the difference of two sums of its
    output, dotted with dy, is the gradient itself."""
    rng = np.random.default_rng(5)
    tokens, slots, rows, cols = 6, 3, 20, 2080
    c, dy = rng.integers(-8, 9, (rows, cols)).astype(np.float32), rng.integers(-8, 9, (tokens, cols)).astype(np.float32)
    p = _positions(rng, tokens, slots, rows)
    w = rng.integers(-4, 5, (tokens, slots)).astype(np.float32)
    dw = _host(mx.expert_weight_grad(_dev(dy), _dev(c), _dev(p)))
    want, _ = ref.weight_grad(dy, c, p)
    assert np.array_equal(dw, want.astype(np.float32))
    base = _host(mx.expert_combine(_dev(c), _dev(p), _dev(w), torch.float32)).astype(np.float64)
    for j in range(slots):
        step = w.copy()
        step[:, j] += 1.0
        moved = _host(mx.expert_combine(_dev(c), _dev(p), _dev(step), torch.float32)).astype(np.float64)
        assert np.array_equal(((moved - base) * dy).sum(1), want[:, j])


@pytest.mark.parametrize("tokens,slots,cols,dy_bf16", [(1003, 6, 2880, False), (1024, 2, 5632, True)])
def test_weight_grad_full_size(tokens, slots, cols, dy_bf16):
    _check_weight_grad(np.random.default_rng(tokens), tokens, slots, tokens * slots, cols, dy_bf16, True)


# ---- a layer, as it is used ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("tiled", [False, True], ids=["rowmajor", "tiled"])
def test_layer_forward_and_backward(tiled):
    """y = sum over a token's experts of w * (x W_e^T) in MXFP8, and its gradients for x, w and every W_e, against the decoded
    operands in float64."""
    rng = np.random.default_rng(12)
    T, k, E, H, O = 60, 2, 4, 256, 256
    lay = mx.SCALES_TILED if tiled else mx.SCALES_ROWMAJOR
    x, x32 = _values(rng, T, H, True)
    dy, dy32 = _values(rng, T, O, False)
    W = [(rng.standard_normal((O, H)) * 0.05).astype(np.float32) for _ in range(E)]
    experts = np.stack([rng.permutation(E)[:k] for _ in range(T)])
    experts[7] = -1
    w = rng.random((T, k)).astype(np.float32)
    plan = mx.expert_sort(_dev(experts), E)
    rows = plan["sources"].numel()
    wq = [mx.quantize(_dev(a), "both", lay) for a in W]
    stack = {n: (torch.stack if n.startswith("q") else torch.cat)([q[n] for q in wq]) for n in wq[0]}
    X = mx.expert_quantize(x, plan["sources"], plan["group_ends"], k, None, "both", lay)
    c = torch.zeros((rows, O), device="cuda")
    mx.mxfp8_gemm_grouped_ex("fprop", X["q_row"], X["s_row"], stack["q_row"], stack["s_row"], plan["group_ends"], c, lay)
    y = mx.expert_combine(c, plan["positions"], _dev(w), torch.float32)
    dw = mx.expert_weight_grad(dy, c, plan["positions"])
    dC = mx.expert_quantize(dy, plan["sources"], plan["group_ends"], k, _dev(w), "both", lay)
    dxs = torch.zeros((rows, H), device="cuda")
    mx.mxfp8_gemm_grouped_ex("dgrad", dC["q_row"], dC["s_row"], stack["q_colT"], stack["s_colT"], plan["group_ends"], dxs, lay)
    dx = mx.expert_combine(dxs, plan["positions"], None, torch.float32)
    dW = torch.full((E, O, H), float("nan"), device="cuda")
    mx.mxfp8_gemm_grouped_ex("wgrad", dC["q_colT"], dC["s_colT"], X["q_colT"], X["s_colT"], plan["group_ends"], dW, lay)
    torch.cuda.synchronize()

    positions, sources, ends = ref.plan(experts, E, 128, rows)
    v, dv = ref.sorted_rows(x32, sources, k), ref.sorted_rows(dy32, sources, k, w)
    vr, vc, dr, dc = oracle.quantize_rowwise(v), oracle.quantize_colwise(v), oracle.quantize_rowwise(dv), oracle.quantize_colwise(dv)
    wr, wc = [oracle.quantize_rowwise(a) for a in W], [oracle.quantize_colwise(a) for a in W]
    got_c, got_dxs = _host(c).astype(np.float64), _host(dxs).astype(np.float64)
    start = 0
    for e, end in enumerate(ends):
        for got, a, b in ((got_c, vr, wr[e]), (got_dxs, dr, wc[e])):
            part = np.arange(start, end)
            want, mag = oracle.gemm_rows(a[0], a[1], b[0], b[1], part)
            assert (np.abs(got[part] - want) <= hw_tolerance(a[0], a[1], b[0], b[1], rows=part) + 2.0 ** -20 * mag).all()
        aq, as_, bq, bs = (np.ascontiguousarray(t) for t in (dc[0][:, start:end], dc[1][:, start // 32:end // 32], vc[0][:, start:end], vc[1][:, start // 32:end // 32]))
        if end > start:
            want, mag = oracle.gemm(aq, as_, bq, bs)
            assert (np.abs(_host(dW)[e] - want) <= hw_tolerance(aq, as_, bq, bs) + 2.0 ** -20 * mag).all()
        start = end
    for got, want, mag, adds in ((_host(y), *ref.combine(got_c, positions, w), k), (_host(dx), *ref.combine(got_dxs, positions), k),
                                 (_host(dw), *ref.weight_grad(dy32, got_c, positions), 8 * -(-O // 512) + 16)):
        assert (np.abs(got - want) <= adds * U * 1.01 * mag + 1e-37).all()
    assert (_host(y)[7] == 0).all() and (_host(dw)[7] == 0).all() and (_host(dx)[7] == 0).all()
