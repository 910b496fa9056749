"""Products of operands with a scale for each block of 128 whose scales take the whole range of FP32: the two scales meet before the block's
sum does, so that one far outside the other's reach leaves the product as it is. The sums are exact here (small whole numbers, powers of two)."""
import numpy as np
import pytest
import torch

import b128_reference as ref
import paper_2506_08027_amd as mx
from test_gpu_b128 import _dev, _host, _product

pytestmark = pytest.mark.gpu


# exponents of A's scales and of B's; the quantizer leaves 2^119.2 where a block holds an infinity
@pytest.mark.parametrize("bf16", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("which", ["fprop", "dgrad", "wgrad"])
@pytest.mark.parametrize("a_exp,b_exp", [(-33, 110), (110, -33), (-120, 120), (120, -120), (-120, 126), (126, -120), (50, 50), (-50, -60)])
def test_scales_meet_before_the_sum(a_exp, b_exp, which, bf16):
    """A second block with other scales of the same product: a_s towards 1 by 2^6, b_s the other way. Blocks' sums are some 300: with a scale of
    2^120 alone they are beyond FP32."""
    M, N, K = 37, 140, 200
    rng = np.random.default_rng(a_exp + 200)
    codes = np.array([0x00, 0x38, 0x40, 0x44], np.uint8)
    a_q, b_q = codes[rng.integers(0, 4, (M, K))], codes[rng.integers(0, 4, (N, K))]
    turn = np.array([0, 6 if a_exp < 0 else -6])
    a_s = np.exp2(a_exp + turn[:, None] + np.zeros((2, M))).astype(np.float32)
    b_s = np.exp2(b_exp - turn[:, None] + np.zeros((2, N))) if which == "wgrad" else np.exp2(b_exp - turn[None, :] + np.zeros((ref.blocks(N), 2)))
    b_s = b_s.astype(np.float32)
    want = ref.decode(a_q, a_s, False) @ ref.decode(b_q, b_s, which != "wgrad").T
    got = _product(which, a_q, a_s, b_q, b_s, bf16)
    assert np.isfinite(want).all() and want.any()
    assert np.array_equal(got, torch.from_numpy(want).bfloat16().double().numpy() if bf16 else want)


@pytest.mark.parametrize("which", ["fprop", "dgrad", "wgrad"])
def test_an_infinity_through_the_quantizer_leaves_finite_products(which):
    """Infinities of both signs count as FLT_MAX and take their blocks with them; a product with small values stays finite, in every pass."""
    T, H, O = 150, 260, 140
    rng = np.random.default_rng(8)
    x, w, dy = (scale * rng.standard_normal(shape).astype(np.float32) for scale, shape in ((1, (T, H)), (0.02, (O, H)), (1e-3, (T, O))))
    wide = dy if which == "dgrad" else x
    wide[3, 5], wide[3, 129], wide[140, 7] = np.inf, -np.inf, -np.inf
    X, W, dY = mx.b128_quantize(_dev(x)), mx.b128_quantize(_dev(w), "both", mx.B128_TILES), mx.b128_quantize(_dev(dy))
    a, b, key = {"fprop": (X, W, "row"), "dgrad": (dY, W, "colT"), "wgrad": (dY, X, "colT")}[which]
    side = "colT" if which == "wgrad" else "row"
    a_q, a_s, b_q, b_s = a["q_" + side], a["s_" + side], b["q_" + key], b["s_" + key]
    got = _host(mx.b128_gemm(which, a_q, a_s, b_q, b_s)).astype(np.float64)
    a_q, a_s, b_q, b_s = _host(a_q), _host(a_s), _host(b_q), _host(b_s)
    av, bv = ref.decode(a_q, a_s, False), ref.decode(b_q, b_s, which != "wgrad")
    want, mag = av @ bv.T, np.abs(av) @ np.abs(bv).T
    assert np.abs(want).max() > 1e30 and np.abs(want).max() < 3e38
    assert (np.abs(got - want) <= ref.gemm_bound(a_q, a_s, b_q, b_s, which != "wgrad", want, mag, False)).all()
