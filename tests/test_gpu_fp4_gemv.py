"""GPU parity of the products of a few BF16 rows with MXFP4 weights (include/mxfp8_experts.h) against the decoded weights in float64.
Every product of a BF16 value and a decoded weight is exact in FP32, so what is allowed is the rounding of the sums: at most
2^-23 of the magnitudes an addition (the matrix instruction may cut off instead of rounding), K additions, and half a step (2^-8) for a
BF16 result. Whole numbers leave no rounding at all: there the result must be exact."""
import numpy as np
import pytest
import torch

import experts_reference as ref
import paper_2506_08027_amd as mx
import scale_layout as sl
from oracle import mxfp4
from paper_2506_08027_amd import synth_inputs as si

pytestmark = pytest.mark.gpu


def _dev(a):
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16)).cuda().view(torch.bfloat16)
    return torch.from_numpy(a).cuda()


def _host(t):
    t = t.contiguous()
    if t.dtype == torch.bfloat16:
        return si.bf16_bits_to_f32(t.view(torch.int16).cpu().numpy().view(np.uint16)).astype(np.float64)
    return t.cpu().numpy().astype(np.float64)


def _x(rng, rows, K):
    bits = si.to_bf16_bits((rng.standard_normal((rows, K)) * np.exp(rng.standard_normal(K))).astype(np.float32))
    return _dev(bits), si.bf16_bits_to_f32(bits)


def _w(rng, n, K, spread=6):
    return rng.integers(0, 256, (n, K // 2), dtype=np.uint8), (120 + rng.integers(-spread, spread + 1, (n, K // 32))).astype(np.uint8)


def _scales(s, tiled):
    """Scale bytes [n x blocks] or [groups x n x blocks] as the call takes them."""
    if not tiled:
        return _dev(s)
    return _dev(np.concatenate([sl.tile(a, filler=0xFF).ravel() for a in (s if s.ndim == 3 else s[None])]))


def _bound(want, mag, K, bf16):
    return K * 2.0 ** -23 * mag + (2.0 ** -8 * 1.01 * np.abs(want) if bf16 else 0.0) + 1e-36


def _run(x, w_q, w_s, N, bf16, tiled, pad=0, offset=0):
    M = x.shape[0]
    flat = torch.full((M * (N + pad) + offset,), float("nan"), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    c = flat[offset:].view(M, N + pad)
    mx.mxfp8_fp4_gemv_ex(x, _dev(w_q), _scales(w_s, tiled), c[:, :N], mx.SCALES_TILED if tiled else mx.SCALES_ROWMAJOR)
    torch.cuda.synchronize()
    got = _host(c)
    assert np.isnan(got[:, N:]).all() and torch.isnan(flat[:offset]).all(), "written outside c"
    return got[:, :N]


@pytest.mark.parametrize("tiled", [False, True], ids=["rowmajor", "tiled"])
@pytest.mark.parametrize("bf16", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(1, 1, 32), (1, 16, 128), (2, 17, 96), (3, 50, 256), (5, 64, 160), (8, 33, 1056), (9, 16, 544), (16, 40, 512), (17, 20, 64),
                                   (31, 16, 288), (33, 18, 128), (64, 16, 96), (70, 31, 192), (1, 100, 2080)])
def test_gemv_is_the_product_with_the_decoded_weights(M, N, K, bf16, tiled):
    rng = np.random.default_rng(M * 1000 + K)
    x, x32 = _x(rng, M, K)
    w_q, w_s = _w(rng, N, K)
    want, mag = ref.gemv(x32, w_q, w_s)
    got = _run(x, w_q, w_s, N, bf16, tiled)
    assert (np.abs(got - want) <= _bound(want, mag, K, bf16)).all()


@pytest.mark.parametrize("tiled", [False, True], ids=["rowmajor", "tiled"])
@pytest.mark.parametrize("M,N,K", [(1, 20, 4096), (4, 16, 8192), (7, 35, 3104), (16, 16, 2048), (40, 16, 1024)])
def test_gemv_of_whole_numbers_is_exact(M, N, K, tiled):
    """Codes are multiples of a half and scales 2 or 4: with x up to 4 no sum of magnitudes reaches 2^24."""
    rng = np.random.default_rng(K + M)
    x = rng.integers(-4, 5, (M, K)).astype(np.float32)
    w_q, w_s = rng.integers(0, 256, (N, K // 2), dtype=np.uint8), rng.integers(128, 130, (N, K // 32)).astype(np.uint8)
    want, mag = ref.gemv(x, w_q, w_s)
    assert mag.max() < 2 ** 24
    assert np.array_equal(_run(_dev(si.to_bf16_bits(x)), w_q, w_s, N, False, tiled), want)


@pytest.mark.parametrize("bf16", [False, True], ids=["f32", "bf16"])
def test_gemv_rows_apart_and_results_off_their_vectors(bf16):
    rng = np.random.default_rng(2)
    big, big32 = _x(rng, 6, 160)
    w_q, w_s = _w(rng, 21, 128)
    want, mag = ref.gemv(big32[:, :128], w_q, w_s)
    for pad, offset in ((3, 0), (0, 1), (7, 3), (11, 0)):
        got = _run(big[:, :128], w_q, w_s, 21, bf16, False, pad, offset)
        assert (np.abs(got - want) <= _bound(want, mag, 128, bf16)).all()


def test_gemv_widens_every_code_and_scale_as_the_decoder_does():
    """One row of x that is 1 at a single k picks weight [n, k]: all 16 codes under all 256 scale bytes, against the decoder's BF16 values."""
    N, K = 256, 32
    w_q = np.tile(np.array([(2 * b) | ((2 * b + 1) << 4) for b in range(8)] * 2, np.uint8), (N, 1))
    w_s = np.arange(256, dtype=np.uint8)[:, None]
    want = _host(mx.fp4_dequantize(_dev(w_q), _dev(w_s), torch.bfloat16))            # [N x 32]
    x = np.zeros((16, K), np.float32)
    x[np.arange(16), np.arange(16)] = 1.0
    got = _run(_dev(si.to_bf16_bits(x)), w_q, w_s, N, False, False).T                 # [N x 16]
    want = want[:, :16]
    ok = np.isfinite(want).all(1)                      # an infinity times the other zeros of x is a NaN, in a scale of 2^126 and more
    assert np.isnan(got[~ok]).all() and np.isnan(got[255]).all() and ok[:253].all()
    assert np.array_equal(got[ok], want[ok])


def test_gemv_nan_and_infinite_activations_stay_in_their_row():
    rng = np.random.default_rng(8)
    _, x32 = _x(rng, 5, 256)
    x32[1, 40], x32[3, 200] = np.nan, np.inf
    w_q, w_s = _w(rng, 30, 256)
    w_q[:, 100] = 0x22                                 # 1.0 at k = 200, 201
    w_s[4, 3] = 0xFF
    got = _run(_dev(si.to_bf16_bits(x32)), w_q, w_s, 30, False, False)
    good = [0, 2, 4]
    cols = [n for n in range(30) if n != 4]
    assert np.isnan(got[1]).all() and np.isposinf(got[3][cols]).all() and np.isnan(got[:, 4]).all()
    want, mag = ref.gemv(x32[good], w_q[cols], w_s[cols])
    assert (np.abs(got[np.ix_(good, cols)] - want) <= _bound(want, mag, 256, False)).all()


def test_gemv_of_nothing():
    c = torch.full((2, 3), 5.0, device="cuda")
    mx.mxfp8_fp4_gemv_ex(torch.empty((2, 0), dtype=torch.bfloat16, device="cuda"), torch.empty((3, 0), dtype=torch.uint8, device="cuda"),
                         torch.empty((3, 0), dtype=torch.uint8, device="cuda"), c)
    torch.cuda.synchronize()
    assert (_host(c) == 0).all()
    assert mx.fp4_gemv(torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((3, 32), dtype=torch.uint8, device="cuda"),
                       torch.zeros((3, 2), dtype=torch.uint8, device="cuda")).shape == (0, 3)


@pytest.mark.parametrize("M,N,K,tiled", [(8, 16400, 160, False), (7, 16384, 2080, True), (16, 16400, 96, True), (13, 17000, 1056, False), (32, 33000, 160, False),
                                         (64, 20000, 640, True), (40, 4100, 544, False), (200, 3000, 320, True), (1, 6144, 4096, False), (12, 4096, 14336, True), (3, 5001, 14304, False), (48, 2048, 4096, True), (16, 4096, 4096, False)])
def test_gemv_full_size(M, N, K, tiled):
    rng = np.random.default_rng(N)
    x, x32 = _x(rng, M, K)
    w_q, w_s = _w(rng, N, K, 2)
    got = _run(x, w_q, w_s, N, True, tiled)
    some = np.unique(np.concatenate([[0, N - 1], rng.integers(0, N, 200)]))
    want, mag = ref.gemv(x32, w_q[some], w_s[some])
    assert (np.abs(got[:, some] - want) <= _bound(want, mag, K, True)).all()
    xi = rng.integers(-2, 3, (M, K)).astype(np.float32)       # exact, so that a missing block cannot hide in the bound
    ones = np.full_like(w_s, 127)
    got = _run(_dev(si.to_bf16_bits(xi)), w_q, ones, N, False, tiled)
    assert np.array_equal(got[:, some], ref.gemv(xi, w_q[some], ones[some])[0])


# ---- each row with its expert's weights ----------------------------------------------------------------------------------------------

def _check_grouped(rng, tokens, slots, groups, N, K, experts, align=1, extra_rows=0, bf16=True, tiled=False, plain=False, whole=False):
    rows = ref.rows_needed(experts.size, groups, align) + extra_rows
    _, sources, ends = ref.plan(experts, groups, align, rows)
    x, x32 = _x(rng, max(rows, tokens) if plain else tokens, K)
    w_q, w_s = (np.stack(a) for a in zip(*(_w(rng, N, K) for _ in range(groups))))
    if whole:
        x32 = rng.integers(-4, 5, x32.shape).astype(np.float32)
        x, w_s = _dev(si.to_bf16_bits(x32)), np.full_like(w_s, 127)
    c = torch.full((rows, N), float("nan"), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    mx.mxfp8_fp4_gemv_grouped_ex(x, None if plain else _dev(sources), slots, _dev(w_q), _scales(w_s, tiled), _dev(ends), c,
                                 mx.SCALES_TILED if tiled else mx.SCALES_ROWMAJOR)
    torch.cuda.synchronize()
    want, mag = ref.gemv_grouped(x32, None if plain else sources, slots, w_q, w_s, ends, rows)
    got = _host(c)
    owned = ~np.isnan(want)
    assert np.array_equal(np.isnan(got), ~owned), "rows of an expert, and only they, are written"
    if whole:
        assert np.array_equal(got[owned], want[owned])
    assert (np.abs(got - want)[owned] <= _bound(want, mag, K, bf16)[owned]).all()


@pytest.mark.parametrize("tiled", [False, True], ids=["rowmajor", "tiled"])
@pytest.mark.parametrize("bf16", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("tokens,slots,groups,align,plain", [(1, 8, 64, 1, False), (5, 2, 3, 1, False), (20, 3, 70, 1, False), (6, 2, 4, 8, True), (40, 1, 2, 1, False)])
def test_grouped_gemv_takes_each_experts_weights(tokens, slots, groups, align, plain, bf16, tiled):
    rng = np.random.default_rng(tokens)
    experts = np.stack([rng.permutation(groups)[:slots] for _ in range(tokens)])
    if tokens > 4:
        experts[3] = -1
    _check_grouped(rng, tokens, slots, groups, 24, 160, experts, align, 5, bf16, tiled, plain)


def test_grouped_gemv_one_expert_for_all_and_more_experts_than_a_wavefront_scans():
    rng = np.random.default_rng(1)
    _check_grouped(rng, 70, 1, 3, 16, 64, np.full((70, 1), 2), bf16=False, whole=True)
    _check_grouped(rng, 9, 2, 200, 16, 64, rng.choice([0, 63, 64, 127, 128, 199], (9, 2)), bf16=False, whole=True)
    _check_grouped(rng, 4, 1, 5, 16, 64, np.full((4, 1), -1), bf16=False)


def test_grouped_gemv_takes_bad_plans_without_leaving_its_buffers():
    rng = np.random.default_rng(6)
    x, x32 = _x(rng, 4, 64)
    w_q, w_s = (np.stack(a) for a in zip(*(_w(rng, 16, 64) for _ in range(3))))
    sources = np.array([0, 7, 8, -9, 2 ** 31 - 1, 3], np.int32)
    for ends, plain in (([2, 4, 1000], [2, 4, 6]), ([-5, 3, 6], [0, 3, 6]), ([2, 2, 5], [2, 2, 5])):
        c = torch.full((6, 16), float("nan"), device="cuda")
        mx.mxfp8_fp4_gemv_grouped_ex(x, _dev(sources), 2, _dev(w_q), _dev(w_s), _dev(np.array(ends, np.int32)), c)
        torch.cuda.synchronize()
        want, mag = ref.gemv_grouped(x32, sources, 2, w_q, w_s, plain, 6)
        owned = ~np.isnan(want)
        assert np.array_equal(np.isnan(_host(c)), ~owned) and (np.abs(_host(c) - want)[owned] <= _bound(want, mag, 64, False)[owned]).all()


@pytest.mark.parametrize("tokens,slots,groups,N,K,tiled", [(1, 8, 64, 704, 2048, False), (48, 4, 32, 512, 1024, True), (200, 8, 16, 256, 512, False),
                                                             (60, 4, 32, 1040, 288, True), (300, 8, 32, 1000, 96, False), (20, 2, 3, 24, 4096, False)])
def test_grouped_gemv_full_size(tokens, slots, groups, N, K, tiled):
    rng = np.random.default_rng(tokens)
    experts = np.stack([rng.permutation(groups)[:slots] for _ in range(tokens)])
    _check_grouped(rng, tokens, slots, groups, N, K, experts, bf16=False, tiled=tiled, whole=True)


def test_a_decoding_step_as_it_is_used():
    """Sort, both products of the experts (a gated activation between them) and the sum back to the tokens."""
    rng = np.random.default_rng(30)
    T, k, E, H, F = 5, 2, 8, 128, 96
    x, x32 = _x(rng, T, H)
    up, down = (tuple(np.stack(a) for a in zip(*(mxfp4.quantize_rowwise((rng.standard_normal(s) * 0.1).astype(np.float32)) for _ in range(E))))
                for s in ((2 * F, H), (H, F)))
    experts = np.stack([rng.permutation(E)[:k] for _ in range(T)])
    w = rng.random((T, k)).astype(np.float32)
    plan = mx.expert_sort(_dev(experts), E, align=1)
    h = mx.fp4_gemv_grouped(x, plan["sources"], k, _dev(up[0]), _dev(up[1]), plan["group_ends"], torch.float32)
    gate, value = h[:, :F], h[:, F:]
    a = (gate * torch.sigmoid(gate) * value).to(torch.bfloat16)
    c = mx.fp4_gemv_grouped(a, None, 1, _dev(down[0]), _dev(down[1]), plan["group_ends"], torch.float32)
    y = _host(mx.expert_combine(c, plan["positions"], _dev(w), torch.float32))
    torch.cuda.synchronize()
    positions, sources, ends = ref.plan(experts, E, 1, T * k)
    want_h, mag_h = ref.gemv_grouped(x32, sources, k, up[0], up[1], ends, T * k)
    assert (np.abs(_host(h) - want_h) <= _bound(want_h, mag_h, H, False)).all()
    want_c, mag_c = ref.gemv_grouped(_host(a).astype(np.float32), None, 1, down[0], down[1], ends, T * k)
    assert (np.abs(_host(c) - want_c) <= _bound(want_c, mag_c, F, False)).all()
    want_y, mag_y = ref.combine(_host(c), positions, w)
    assert (np.abs(y - want_y) <= k * 2.0 ** -24 * 1.01 * mag_y + 1e-37).all()
