"""Both kinds of results of the products with a scale for each block of 128 on the CPU execution model: the GPU tests of FP32 results' accuracy and of
BF16 results replayed, and BF16 results of the larger tiles, which FP32 results do not take, with AddressSanitizer."""
import numpy as np
import pytest

import b128_reference as ref
from paper_2506_08027_amd import synth_inputs as si
from test_host_model_b128 import _load, _operand_bytes
from test_host_model_experts import ORDERS, Case, driver  # noqa: F401
from test_host_model_replay_b128 import hostmodel_lib, test_gpu_tests_pass_on_the_host_model as _replay  # noqa: F401


@pytest.mark.parametrize("file,at_least", [("test_gpu_b128_fp32.py", 42), ("test_gpu_b128_bf16.py", 20)])
def test_gpu_tests_of_both_results_pass_on_the_host_model(hostmodel_lib, file, at_least):  # noqa: F811
    _replay(hostmodel_lib, file, at_least)


# sizes that take each of the larger tiles; some of their workgroups are run
@pytest.mark.parametrize("which,M,N,K,order", [(0, 4000, 4100, 272, "up"), (2, 4100, 4000, 400, "down"), (0, 2008, 4096, 260, "down"), (2, 2000, 4097, 272, "up"),
                                               (0, 100, 65400, 272, "up"), (0, 1000, 3000, 1000, "down"), (2, 1001, 2999, 1100, "up")])
def test_sampled_workgroups_of_larger_tiles_in_bf16(driver, tmp_path, monkeypatch, which, M, N, K, order):  # noqa: F811
    rng = np.random.default_rng(K)
    codes = np.array([0x00, 0x38, 0x40, 0x44, 0xB8, 0xC0, 0xC4], np.uint8)
    a_q, b_q = codes[rng.integers(0, 7, (M, K))], codes[rng.integers(0, 7, (N, K))]
    a_s = np.exp2(rng.integers(0, 3, (ref.blocks(K), M))).astype(np.float32)
    b_s = np.exp2(rng.integers(0, 3, (ref.blocks(K), N) if which == 2 else (ref.blocks(N), ref.blocks(K)))).astype(np.float32)
    ld = ref.up16(K)
    monkeypatch.setenv("WAVESIM_BLOCKS", "3")
    case = Case(tmp_path, "b128_gemm").number(which).given(_operand_bytes(a_q, ld)).number(ld).given(a_s).given(_operand_bytes(b_q, ld)).number(ld).given(b_s)
    case.number(M, N, K).output("c", M * N * 2).number(1, N).null().run(driver, order)
    got = _load(case, "c", np.uint16, (M, N))
    rows, cols = np.nonzero((got != 0xA5A5).any(1))[0], np.nonzero((got != 0xA5A5).any(0))[0]
    assert rows.size and cols.size
    a, b = ref.decode(a_q[rows], a_s[:, rows], False), ref.decode(b_q, b_s, which != 2)[cols]
    part = got[np.ix_(rows, cols)]
    written = part != 0xA5A5
    assert written.sum() >= 3 * 128 * 64 and np.array_equal(part[written], si.to_bf16_bits((a @ b.T)[written].astype(np.float32)))


# FP32 results whose K is cut into parts, and tiles of both sizes with rows and columns at their ends
@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("which,M,N,K", [(0, 20, 40, 4100), (2, 70, 9, 2100), (0, 129, 40, 200)])
def test_fp32_results_in_parts_of_k(driver, tmp_path, which, M, N, K, order):  # noqa: F811
    import paper_2506_08027_amd as mx
    rng = np.random.default_rng(K)
    (a_q, a_s), (b_q, b_s) = ref.operand(rng.standard_normal((M, K)).astype(np.float32), False), ref.operand(rng.standard_normal((N, K)).astype(np.float32), which != 2)
    ld, need = ref.up16(K), mx.mxfp8_b128_gemm_workspace(which, M, N, K)
    assert (need > 0) == (K > 1000)
    case = Case(tmp_path, "b128_gemm").number(which).given(_operand_bytes(a_q, ld)).number(ld).given(a_s).given(_operand_bytes(b_q, ld)).number(ld).given(b_s)
    case.number(M, N, K).output("c", M * N * 4).number(0, N)
    (case.output("workspace", need) if need else case.null()).run(driver, order)
    a, b = ref.decode(a_q, a_s, False), ref.decode(b_q, b_s, which != 2)
    want, mag = a @ b.T, np.abs(a) @ np.abs(b).T
    assert (np.abs(_load(case, "c", np.float32, (M, N)) - want) <= (2 * 128 + 2 + ref.blocks(K) + 16) * 2.0 ** -24 * mag).all()
