"""The expert rows and the MXFP4 products of a few rows at the largest sizes that they take: 2^30 entries, and as many tiles of weights as a
launch can have."""
import os

import pytest
import torch

import paper_2506_08027_amd as mx

pytestmark = [pytest.mark.gpu, pytest.mark.skipif("MXFP8_HOSTMODEL_LIB" in os.environ, reason="GPU memory")]
MOST = 1 << 30


def test_sort_of_the_most_entries():
    i = torch.arange(MOST, dtype=torch.int32, device="cuda")
    plan = mx.expert_sort((i & 7).view(-1, 4), 8, 1)
    assert plan["group_ends"].tolist() == [(e + 1) << 27 for e in range(8)]
    assert torch.equal(plan["positions"].view(-1), ((i & 7) << 27) + (i >> 3))
    assert torch.equal(plan["sources"], ((i & ((1 << 27) - 1)) << 3) + (i >> 27))


def test_sums_of_the_most_entries():
    tokens, slots, rows = MOST // 4, 4, 100
    c = torch.arange(rows, device="cuda", dtype=torch.float32).view(rows, 1)
    p = torch.full((tokens, slots), -1, dtype=torch.int32, device="cuda")
    w = torch.full((tokens, slots), float("nan"), device="cuda")
    last = torch.tensor([[1, 2, -1, 99], [7, -1, -1, 3]], dtype=torch.int32, device="cuda")
    p[-2:], w[-2:] = last, torch.tensor([2.0, 0.5, 1.0, 4.0], device="cuda")
    p[0], w[0] = last[1], 1.0
    out = torch.full((tokens, 1), float("nan"), device="cuda")
    mx.mxfp8_expert_combine(c, p, w, out)
    assert out[[0, -2, -1], 0].tolist() == [10.0, 2 + 1 + 396, 14 + 12]
    assert int(torch.count_nonzero(out)) == 3 and not torch.isnan(out).any()
    del out
    dy = torch.full((tokens, 1), 2.0, device="cuda")
    dy[-1] = 3.0
    mx.mxfp8_expert_weight_grad(dy, c, p, w)
    assert w[[0, -2, -1]].tolist() == [[14, 0, 0, 6], [2, 4, 0, 198], [21, 0, 0, 9]]
    assert int(torch.count_nonzero(w)) == 7 and not torch.isnan(w).any()


def test_quantizer_of_the_last_of_the_most_entries():
    """Weights that are powers of two: the products are exact, so the plain quantizer of them is the reference."""
    tokens, slots, cols = MOST // 4, 4, 32
    x, w = torch.empty((tokens, cols), dtype=torch.bfloat16, device="cuda"), torch.empty((tokens, slots), device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    x[-16:] = torch.randn((16, cols), generator=g, device="cuda").bfloat16()
    w[-16:] = torch.exp2(torch.randint(-3, 4, (16, slots), generator=g, device="cuda").float())
    sources = torch.arange(MOST - 64, MOST, dtype=torch.int32, device="cuda")
    sources[5] = -1
    got = mx.expert_quantize(x, sources, None, slots, w, "both")
    v = x[-16:].float().repeat_interleave(slots, 0) * w[-16:].reshape(-1, 1)
    v[5] = 0.0
    want = mx.quantize(v, "both")
    assert all(torch.equal(got[k], want[k]) for k in want)


def test_gemv_of_the_most_columns():
    N, K = (1 << 27) - 16, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.zeros((N, K // 2), dtype=torch.uint8, device="cuda")
    s = torch.full((N, K // 32), 127, dtype=torch.uint8, device="cuda")
    q[-1000:] = torch.randint(0, 256, (1000, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    x = torch.randint(-4, 5, (1, K), generator=g, device="cuda").bfloat16()
    c = mx.fp4_gemv(x, q, s, torch.float32)
    assert torch.equal(c[:, -1000:], mx.fp4_gemv(x, q[-1000:].clone(), s[-1000:].clone(), torch.float32))
    assert int(torch.count_nonzero(c[:, :-1000])) == 0 and not torch.isnan(c).any()
