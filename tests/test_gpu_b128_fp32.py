"""FP32 results of the products with a scale for each block of 128: what a caller who asks for FP32 gets is off by FP32 roundings alone. (BF16
results come from the FP8 matrix instructions, which cut every product of a group of eight off at 2^-13 of the largest.)"""
import numpy as np
import pytest

import b128_reference as ref
from test_gpu_b128 import SIZES, _operands, _product

pytestmark = pytest.mark.gpu


def fp32_bound(K, mag):
    """Products of two codes have 8 bits: exact. Each of a block's 128 additions loses 2^-23 of the magnitudes at most (cut off, or 2^-24
    rounded); the two scales' product, the block's sum times it and its addition to the blocks before, and the additions of up to 16 parts 2^-24."""
    return (2 * 128 + 2 + ref.blocks(K) + 16) * 2.0 ** -24 * mag + 1e-37


@pytest.mark.parametrize("which", ["fprop", "dgrad", "wgrad"])
@pytest.mark.parametrize("M,N,K", SIZES + [(64, 64, 16384), (96, 300, 6000), (300, 400, 700)])
def test_fp32_results_lose_fp32_roundings_alone(M, N, K, which):
    a_q, a_s, b_q, b_s = _operands(np.random.default_rng(M * 1000 + K), M, N, K, which == "wgrad")
    a, b = ref.decode(a_q, a_s, False), ref.decode(b_q, b_s, which != "wgrad")
    want, mag = a @ b.T, np.abs(a) @ np.abs(b).T
    assert (np.abs(_product(which, a_q, a_s, b_q, b_s, False) - want) <= fp32_bound(K, mag)).all()


@pytest.mark.parametrize("which", ["fprop", "wgrad"])
@pytest.mark.parametrize("M,N,K", [(20, 70, 256), (130, 140, 1000), (8, 64, 12800)])
def test_small_products_beside_a_large_one_count(M, N, K, which):
    """One code of 448 = 1.75 * 2^8 in each group of eight, the others below 2^-5: seven products that a cut at 2^(8 - 13) leaves nothing of. They
    are 3 * 10^-4 of the result, ten times what FP32 roundings may lose of it."""
    rng = np.random.default_rng(K)
    a_q = rng.integers(0x08, 0x10, (M, K)).astype(np.uint8)  # 2^-6 .. 2^-5
    a_q[:, 3::8] = 0x7E
    a_q[:, 5::8] |= 0x80
    b_q = np.full((N, K), 0x38, np.uint8)
    a_s, b_s = np.ones((ref.blocks(K), M), np.float32), np.ones((ref.blocks(K), N) if which == "wgrad" else (ref.blocks(N), ref.blocks(K)), np.float32)
    want = ref.decode(a_q, a_s, False) @ ref.decode(b_q, b_s, which != "wgrad").T
    small = ref.decode(np.where(a_q == 0x7E, 0, a_q).astype(np.uint8), a_s, False).sum(1)
    assert (small > 2e-4 * want[:, 0]).all()
    got = _product(which, a_q, a_s, b_q, b_s, False)
    assert (np.abs(got - want) <= fp32_bound(K, np.abs(want))).all()
    assert ((got - 448 * len(range(3, K, 8)))[:, 0] > 0.9 * small).all()
