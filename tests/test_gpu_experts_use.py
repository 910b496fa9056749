"""The expert rows and the MXFP4 products of a few rows as programs use them: through the binding's calls in C++ and through its own
checks, on other streams, captured into graphs that are replayed with other inputs, at offsets beyond 32 bits; and what the binding refuses."""
import os

import numpy as np
import pytest
import torch

import experts_reference as ref
import paper_2506_08027_amd as mx
from paper_2506_08027_amd import binding, experts

pytestmark = [pytest.mark.gpu, pytest.mark.skipif("MXFP8_HOSTMODEL_LIB" in os.environ, reason="streams, graphs and GPU memory")]


def _randn(seed, *shape, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _u8(seed, *shape, lo=0, hi=256):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.uint8)


def _experts(seed, tokens, slots, groups):
    e = torch.argsort(_randn(seed, tokens, groups), dim=1)[:, :slots].contiguous()
    e[::7] = -1
    return e


def _calls():
    """(name in the module, call, outputs) of every entry point that both ways take."""
    T, k, E, H, N = 40, 2, 6, 128, 96
    out = []
    for dtype in (torch.int32, torch.int64):
        e = _experts(1, T, k, E).to(dtype)
        rows = mx.mxfp8_expert_rows(T * k, E, 32)
        i32 = dict(dtype=torch.int32, device="cuda")
        o = [torch.zeros((T, k), **i32), torch.zeros(rows, **i32), torch.zeros(E, **i32)]
        out.append(("expert_sort", lambda e=e, o=o: mx.mxfp8_expert_sort(e, 32, *o), o))
    plan = mx.expert_sort(_experts(1, T, k, E), E, 32)
    rows = plan["sources"].numel()
    w = torch.rand((T, k), device="cuda")
    for dtype, weights, lay, axis in ((torch.bfloat16, None, mx.SCALES_TILED, "both"), (torch.float32, w, mx.SCALES_ROWMAJOR, mx.ROWWISE), (torch.bfloat16, w, mx.SCALES_ROWMAJOR, "colwise")):
        x = _randn(2, T, H + 8, dtype=dtype)[:, :H]
        scale = lambda r, c: _u8(0, mx.mxfp8_scale_bytes(r, c, lay)) if lay == mx.SCALES_TILED else _u8(0, r, c // 32)  # noqa: E731
        c = [_u8(0, rows, H), scale(rows, H), _u8(0, H, rows), scale(H, rows)]
        out.append(("expert_quantize", lambda x=x, c=c, weights=weights, lay=lay, axis=axis: mx.mxfp8_expert_quantize_ex(
            x, plan["sources"], plan["group_ends"], k, weights, axis, *c, lay), c))
        out.append(("expert_quantize", lambda x=x, c=c, lay=lay: mx.mxfp8_expert_quantize_ex(x, plan["sources"], None, k, None, "both", *c, lay), c))
    c = _randn(3, rows, H + 8, dtype=torch.bfloat16)[:, :H]
    y, dw = torch.zeros((T, H), device="cuda"), torch.zeros((T, k), device="cuda")
    out.append(("expert_combine", lambda: mx.mxfp8_expert_combine(c, plan["positions"], w, y), [y]))
    out.append(("expert_combine", lambda: mx.mxfp8_expert_combine(c, plan["positions"], None, y), [y]))
    out.append(("expert_weight_grad", lambda: mx.mxfp8_expert_weight_grad(_randn(4, T, H), c, plan["positions"], dw), [dw]))
    x = _randn(5, T, H, dtype=torch.bfloat16)
    for lay in (mx.SCALES_TILED, mx.SCALES_ROWMAJOR):
        q, s = _u8(6, E, N, H // 2), _u8(7, E, mx.mxfp8_scale_bytes(N, H, lay), lo=124, hi=130)
        s1 = s[0] if lay == mx.SCALES_TILED else s[0].view(N, H // 32)
        o, g = torch.zeros((T, N), dtype=torch.bfloat16, device="cuda"), torch.zeros((rows, N), device="cuda")
        out.append(("fp4_gemv", lambda q=q, s1=s1, o=o, lay=lay: mx.mxfp8_fp4_gemv_ex(x, q[0], s1, o, lay), [o]))
        out.append(("fp4_gemv_grouped", lambda q=q, s=s, g=g, lay=lay: mx.mxfp8_fp4_gemv_grouped_ex(x, plan["sources"], k, q, s, plan["group_ends"], g, lay), [g]))
        out.append(("fp4_gemv_grouped", lambda q=q, s=s, g=g, lay=lay: mx.mxfp8_fp4_gemv_grouped_ex(
            _randn(8, rows, H, dtype=torch.bfloat16), None, 1, q, s, plan["group_ends"], g, lay), [g]))
    return out


def _bytes(tensors):
    return [t.contiguous().view(torch.uint8).clone() for t in tensors]


def test_calls_in_cpp_and_through_pythons_checks_do_the_same(monkeypatch):
    mx.load()
    assert binding._fast is not None, "paper_2506_08027_amd/_fastcall.so is not built"
    for name, call, outputs in _calls():
        handled = []
        real = experts._fast
        monkeypatch.setattr(experts, "_fast", lambda *a: handled.append(a[0]) or real(*a))
        got = []
        for fast in (True, False):
            for o in outputs:
                o.view(torch.uint8).fill_(0x5A)
            if fast:
                done = []
                monkeypatch.setattr(experts, "_fast", lambda *a: done.append(real(*a)) or done[-1])
                call()
                assert done == [True], f"{name} was not handled in C++"
            else:
                monkeypatch.setattr(experts, "_fast", lambda *a: False)
                call()
            monkeypatch.setattr(experts, "_fast", real)
            torch.cuda.synchronize()
            got.append(_bytes(outputs))
        assert all(torch.equal(a, b) for a, b in zip(*got)), name


def test_refusals_by_status_come_through_both_ways(monkeypatch):
    x = torch.zeros((4, 72), dtype=torch.bfloat16, device="cuda")[:, 4:68]             # rows 8 bytes off
    q, s, c = _u8(0, 8, 32), _u8(0, 8, 2), torch.zeros((4, 8), device="cuda")
    for fast in (binding._fast, None):
        monkeypatch.setattr(binding, "_fast", fast)
        with pytest.raises(mx.MXFP8Error) as e:
            mx.mxfp8_fp4_gemv_ex(x, q, s, c)
        assert e.value.code == 3
        with pytest.raises(mx.MXFP8Error) as e:
            mx.mxfp8_expert_sort(torch.zeros((4, 2), dtype=torch.int32, device="cuda"), 64, *(torch.zeros(8, dtype=torch.int32, device="cuda") for _ in range(3)))
        assert e.value.code == 2
        with pytest.raises(ValueError, match="GPU memory"):
            mx.mxfp8_fp4_gemv_ex(x.cpu(), q, s, c)


def test_calls_go_to_the_stream_they_are_given():
    """A long kernel holds the stream up; the call behind it must see what it wrote, and the default stream is not waited for."""
    w = _u8(6, 512, 128), _u8(7, 512, 8, lo=124, hi=130)
    want = mx.fp4_gemv(torch.full((2, 256), 3.0, dtype=torch.bfloat16, device="cuda"), *w)
    torch.cuda.synchronize()
    for given in (True, False):
        stream = torch.cuda.Stream()
        x, c = torch.zeros((2, 256), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 512), dtype=torch.bfloat16, device="cuda")
        big = torch.ones((1 << 26,), device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            for _ in range(20):
                big.mul_(1.0)
            x.fill_(3.0)
            if not given:
                mx.mxfp8_fp4_gemv_ex(x, *w, c)
        if given:
            mx.mxfp8_fp4_gemv_ex(x, *w, c, stream=stream)
        stream.synchronize()
        assert torch.equal(c, want)


class _Layer:
    """A mixture-of-experts layer, forward and backward, on buffers that it keeps."""

    def __init__(self, seed, T=96, k=2, E=5, H=256, O=256):
        self.T, self.k, self.E, self.H, self.O = T, k, E, H, O
        self.experts, self.w = _experts(seed, T, k, E), torch.sigmoid(_randn(seed + 40, T, k))
        self.x, self.dy = _randn(seed + 1, T, H, dtype=torch.bfloat16), _randn(seed + 2, T, O)
        wq = [mx.quantize(_randn(seed + 3 + e, O, H) * 0.05, "both", mx.SCALES_TILED) for e in range(E)]
        self.wq = {n: (torch.stack if n.startswith("q") else torch.cat)([q[n] for q in wq]) for n in wq[0]}
        rows = mx.mxfp8_expert_rows(T * k, E, 128)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.positions, self.sources, self.ends = torch.zeros((T, k), **i32), torch.zeros(rows, **i32), torch.zeros(E, **i32)
        self.X, self.dC = self._copies(rows, H), self._copies(rows, O)
        f = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
        self.c, self.dxs, self.y, self.dx, self.dw, self.dW = f(rows, O), f(rows, H), f(T, O), f(T, H), f(T, k), f(E, O, H)

    @staticmethod
    def _copies(r, c):
        n = lambda a, b: torch.zeros(mx.mxfp8_scale_bytes(a, b, mx.SCALES_TILED), dtype=torch.uint8, device="cuda")  # noqa: E731
        return dict(q_row=torch.zeros((r, c), dtype=torch.uint8, device="cuda"), s_row=n(r, c), q_colT=torch.zeros((c, r), dtype=torch.uint8, device="cuda"), s_colT=n(c, r))

    def step(self):
        t, X, dC, wq = mx.SCALES_TILED, self.X, self.dC, self.wq
        mx.mxfp8_expert_sort(self.experts, 128, self.positions, self.sources, self.ends)
        mx.mxfp8_expert_quantize_ex(self.x, self.sources, self.ends, self.k, None, "both", **X, scale_layout=t)
        mx.mxfp8_gemm_grouped_ex("fprop", X["q_row"], X["s_row"], wq["q_row"], wq["s_row"], self.ends, self.c, t)
        mx.mxfp8_expert_combine(self.c, self.positions, self.w, self.y)
        mx.mxfp8_expert_weight_grad(self.dy, self.c, self.positions, self.dw)
        mx.mxfp8_expert_quantize_ex(self.dy, self.sources, self.ends, self.k, self.w, "both", **dC, scale_layout=t)
        mx.mxfp8_gemm_grouped_ex("dgrad", dC["q_row"], dC["s_row"], wq["q_colT"], wq["s_colT"], self.ends, self.dxs, t)
        mx.mxfp8_expert_combine(self.dxs, self.positions, None, self.dx)
        mx.mxfp8_gemm_grouped_ex("wgrad", dC["q_colT"], dC["s_colT"], X["q_colT"], X["s_colT"], self.ends, self.dW, t)

    def results(self):
        return [t.clone() for t in (self.positions, self.sources, self.ends, self.y, self.dw, self.dx, self.dW)]


def _captured(f):
    f()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f()
    return graph


def test_a_captured_layer_replays_with_other_inputs():
    """Two graphs of two layers, replayed in turn with eager work between them; each replay against the eager step on the same inputs."""
    layers, twins = [_Layer(10), _Layer(50, T=61, k=3, E=4)], [_Layer(10), _Layer(50, T=61, k=3, E=4)]
    graphs = [_captured(l.step) for l in layers]
    for turn in range(3):
        for n, (layer, twin) in enumerate(zip(layers, twins)):
            for l in (layer, twin):
                l.experts.copy_(_experts(100 * turn + n, l.T, l.k, l.E))
                l.x.copy_(_randn(200 * turn + n, l.T, l.H))
                l.dy.copy_(_randn(300 * turn + n, l.T, l.O))
            twin.step()
            graphs[n].replay()
            torch.cuda.synchronize()
            torch.ones(1000, device="cuda").sum().item()
            assert all(torch.equal(a, b) for a, b in zip(layer.results(), twin.results()))


def test_captured_sorts_with_a_workspace_each_and_a_captured_decoding_step():
    E, n = 96, 40000
    sorts = []
    for seed in (1, 2):
        e = torch.randint(-1, E, (n, 1), device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))
        i32 = dict(dtype=torch.int32, device="cuda")
        o = [torch.zeros((n, 1), **i32), torch.zeros(mx.mxfp8_expert_rows(n, E, 64), **i32), torch.zeros(E, **i32)]
        ws = torch.zeros(mx.mxfp8_expert_sort_workspace(n, E), dtype=torch.uint8, device="cuda")
        sorts.append((e, o, _captured(lambda e=e, o=o, ws=ws: mx.mxfp8_expert_sort(e, 64, *o, ws))))
    T, k, H, N = 3, 2, 256, 83
    ids, x, w = _experts(3, T, k, E), _randn(4, T, H, dtype=torch.bfloat16), torch.rand((T, k), device="cuda")
    q, s = _u8(5, E, N, H // 2), _u8(6, E, N, H // 32, lo=124, hi=130)
    out = torch.zeros((T, N), device="cuda")

    def decode():
        plan = mx.expert_sort(ids, E, align=1)
        c = mx.fp4_gemv_grouped(x, plan["sources"], k, q, s, plan["group_ends"], torch.float32)
        mx.mxfp8_expert_combine(c, plan["positions"], w, out)
    graph = _captured(decode)
    for turn in range(3):
        for i, (e, o, g) in enumerate(sorts):
            e.copy_(torch.randint(-1, E, (n, 1), device="cuda", generator=torch.Generator(device="cuda").manual_seed(10 * turn + i)))
            g.replay()
        ids.copy_(_experts(20 + turn, T, k, E))
        x.copy_(_randn(30 + turn, T, H))
        graph.replay()
        torch.cuda.synchronize()
        for e, o, g in sorts:
            for a, b in zip(o, ref.plan(e.cpu().numpy(), E, 64, o[1].numel())):
                assert np.array_equal(a.cpu().numpy(), b)
        got = out.clone()
        decode()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and not torch.isnan(out).any()


def test_offsets_beyond_32_bits():
    """The last rows of tensors of more than 4 GiB: sorted rows summed and quantized, rows of x, an expert's weights."""
    rows, cols = 540000, 4096                                                   # 4.4 GB of BF16
    c = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    c[-2:] = _randn(1, 2, cols, dtype=torch.bfloat16)
    c[0] = 1.0
    p = torch.tensor([[rows - 1, 0], [rows - 2, -1]], dtype=torch.int32, device="cuda")
    y, dy = mx.expert_combine(c, p, None, torch.float32), _randn(2, 2, cols)
    dw = mx.expert_weight_grad(dy, c, p)
    last = c[-2:].double()
    assert torch.equal(y[0], (last[1].float() + 1.0)) and torch.equal(y[1], last[0].float())
    want = torch.stack([(dy[0].double() * last[1]).sum(), dy[0].double().sum(), (dy[1].double() * last[0]).sum()])
    assert ((dw.flatten()[[0, 1, 2]].double() - want).abs() <= 80 * 2.0 ** -24 * dy.abs().double().sum() * c[-2:].abs().max().double()).all()
    sources = torch.full((32,), rows - 1, dtype=torch.int32, device="cuda")
    got = mx.expert_quantize(c, sources, None, 1, None, "rowwise")
    one = mx.quantize(c[-1:].expand(32, cols).contiguous(), "rowwise")
    assert torch.equal(got["q_row"], one["q_row"]) and torch.equal(got["s_row"], one["s_row"])
    q1, s1 = _u8(3, 16, cols // 2), _u8(4, 16, cols // 32, lo=124, hi=130)
    ends = torch.tensor([1], dtype=torch.int32, device="cuda")
    g = mx.fp4_gemv_grouped(c, sources[:1].clone(), 1, q1[None], s1[None], ends, torch.float32)
    assert torch.equal(g, mx.fp4_gemv(c[-1:].contiguous(), q1, s1, torch.float32))
    del c
    E, N, K = 530, 4096, 4096
    q, s = torch.empty((E, N, K // 2), dtype=torch.uint8, device="cuda"), torch.full((E, N, K // 32), 127, dtype=torch.uint8, device="cuda")
    q[-1] = _u8(5, N, K // 2)
    x, ends = _randn(6, 1, K, dtype=torch.bfloat16), torch.zeros(E, dtype=torch.int32, device="cuda")
    ends[-1] = 1
    assert torch.equal(mx.fp4_gemv_grouped(x, None, 1, q, s, ends, torch.float32), mx.fp4_gemv(x, q[-1], s[-1], torch.float32))
    torch.cuda.synchronize()


def test_equal_inputs_give_equal_bits():
    layer = _Layer(70)
    layer.step()
    first = layer.results()
    for _ in range(3):
        layer.step()
        assert all(torch.equal(a, b) for a, b in zip(first, layer.results()))
