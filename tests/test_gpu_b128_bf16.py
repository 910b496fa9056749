"""BF16 results of the products with a scale for each block of 128, which the FP8 matrix instructions make: strides, padding, NaN, and offsets beyond
32 bits. (test_gpu_b128.py and test_gpu_b128_use.py ask for FP32 there.)"""
import numpy as np
import pytest
import torch

import b128_reference as ref
import paper_2506_08027_amd as mx
from test_gpu_b128 import _operands, _product

pytestmark = pytest.mark.gpu


def _rounded(want):
    return torch.from_numpy(want.astype(np.float32)).bfloat16().double().numpy()


@pytest.mark.parametrize("which", ["fprop", "dgrad", "wgrad"])
@pytest.mark.parametrize("M,N,K,extra,pad,offset", [(40, 90, 200, 0, 0, 0), (129, 130, 144, 16, 3, 1), (70, 64, 1300, 32, 8, 8), (2, 500, 77, 48, 1, 0), (200, 7, 129, 0, 4, 2),
                                                    (64, 64, 20000, 0, 0, 0)])
def test_whole_numbers_are_rounded_once(M, N, K, extra, pad, offset, which):
    a_q, a_s, b_q, b_s = _operands(np.random.default_rng(K), M, N, K, which == "wgrad", whole=True)
    want = ref.decode(a_q, a_s, False) @ ref.decode(b_q, b_s, which != "wgrad").T
    assert np.array_equal(_product(which, a_q, a_s, b_q, b_s, True, extra, pad, offset), _rounded(want))


@pytest.mark.parametrize("which", ["fprop", "wgrad"])
def test_nan_stays_where_it_belongs(which):
    M, N, K = 40, 150, 300
    a_q, a_s, b_q, b_s = _operands(np.random.default_rng(3), M, N, K, which == "wgrad", whole=True)
    bad = np.zeros((M, N), bool)
    bad[7], bad[:, 9], bad[20] = True, True, True
    want = ref.decode(a_q, a_s, False) @ ref.decode(b_q, b_s, which != "wgrad").T
    a_q[7, 299], b_q[9, 0], a_s[1, 20] = 0x7F, 0xFF, np.nan
    got = _product(which, a_q, a_s, b_q, b_s, True)
    assert np.isnan(got[bad]).all() and np.array_equal(got[~bad], _rounded(want)[~bad])


def test_full_size_offsets_beyond_32_bits():
    """4.4 GB of codes, the last rows of which are whole numbers; a result whose rows lie 2.2 GB apart."""
    N, K = 270000, 16384
    b_q, b_s = torch.zeros((N, K), dtype=torch.uint8, device="cuda"), torch.ones((ref.blocks(N), ref.blocks(K)), device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    codes = torch.tensor([0x00, 0x38, 0x40, 0x44, 0xB8, 0xC0, 0xC4], dtype=torch.uint8, device="cuda")
    b_q[-300:] = codes[torch.randint(0, 7, (300, K), generator=g, device="cuda")]
    a_q, a_s = codes[torch.randint(0, 7, (2, K), generator=g, device="cuda")], torch.ones((ref.blocks(K), 2), device="cuda")
    want = a_q.view(torch.float8_e4m3fn).double() @ b_q[-300:].view(torch.float8_e4m3fn).double().t()
    got = mx.b128_gemm("fprop", a_q, a_s, b_q, b_s, torch.bfloat16)
    assert torch.equal(got[:, -300:], want.bfloat16()) and not got[:, :-300].any()
    flat = torch.empty((2 * 1100000000 + 64,), dtype=torch.bfloat16, device="cuda")
    out = flat.as_strided((3, 64), (1100000000, 1))
    a_q, a_s = codes[torch.randint(0, 7, (3, K), generator=g, device="cuda")], torch.ones((ref.blocks(K), 3), device="cuda")
    need = mx.mxfp8_b128_gemm_workspace("fprop", 3, 64, K)
    small = b_q[-64:].contiguous()
    mx.mxfp8_b128_gemm("fprop", a_q, a_s, small, b_s[-1:].contiguous(), out, torch.empty((need,), dtype=torch.uint8, device="cuda") if need else None)
    assert torch.equal(out, (a_q.view(torch.float8_e4m3fn).double() @ small.view(torch.float8_e4m3fn).double().t()).bfloat16())
