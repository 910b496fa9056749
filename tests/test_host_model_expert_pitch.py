"""The weighted sum of an entry's rows and the gradient of its weights where a width of whole 16-byte pieces is not enough for accesses
of 16 bytes: one operand alone starts one element off, or has a pitch of an odd number of elements. On the CPU execution model, where an
access that is not aligned to its size ends the run. Also widths at which the gradient takes four pieces at a time element by element."""
import numpy as np
import pytest

import experts_reference as ref
from paper_2506_08027_amd import synth_inputs as si
from test_host_model_experts import Case, driver  # noqa: F401

WHICH = ["none", "c base", "c pitch", "other base", "other pitch"]


def _operand(rng, rows, cols, ld, off, bf16):
    """(what lies in memory, `off` elements of it in front; values as float32)"""
    x = rng.standard_normal((rows, ld)).astype(np.float32)
    bits = si.to_bf16_bits(x)
    flat = (bits if bf16 else x).ravel()[:(rows - 1) * ld + cols]
    return np.concatenate([np.zeros(off, flat.dtype), flat]), (si.bf16_bits_to_f32(bits) if bf16 else x)[:, :cols]


def _layout(which, what, cols):
    """(pitch, offset) in elements"""
    return cols + (1 if which == what + " pitch" else 8), int(which == what + " base")


@pytest.mark.parametrize("c_bf16", [False, True], ids=["c-f32", "c-bf16"])
@pytest.mark.parametrize("other_bf16", [False, True], ids=["other-f32", "other-bf16"])
@pytest.mark.parametrize("which", WHICH)
def test_one_operand_off_16_bytes(driver, tmp_path, which, other_bf16, c_bf16):  # noqa: F811
    rng = np.random.default_rng(3)
    tokens, slots, rows, cols = 3, 5, 6, 576
    (ldc, c_off), (ld, off) = _layout(which, "c", cols), _layout(which, "other", cols)
    es, c_es = 2 if other_bf16 else 4, 2 if c_bf16 else 4
    flat, c = _operand(rng, rows, cols, ldc, c_off, c_bf16)
    p = rng.integers(-1, rows, (tokens, slots)).astype(np.int32)
    w = rng.standard_normal((tokens, slots)).astype(np.float32)
    n = (tokens - 1) * ld + cols
    out = (Case(tmp_path, "combine").given(flat, c_off * c_es).number(c_bf16, rows, cols, ldc).given(p).given(w).number(tokens, slots)
           .output("out", (off + n) * es, off * es).number(other_bf16, ld).run(driver))
    left = np.uint16(0xA5A5) if other_bf16 else np.uint32(0xA5A5A5A5)      # as the driver fills outputs
    raw = np.full(off + tokens * ld, left)
    raw[:off + n] = np.frombuffer(out["out"], raw.dtype)
    body = raw[off:].reshape(tokens, ld)
    assert (raw[:off] == left).all() and (body[:, cols:] == left).all()
    got = si.bf16_bits_to_f32(body[:, :cols]) if other_bf16 else np.ascontiguousarray(body[:, :cols]).view(np.float32)
    want, mag = ref.combine(c, p, w)
    assert (np.abs(got - want) <= slots * 2.0 ** -24 * 1.01 * mag + (2.0 ** -8 * 1.01 * np.abs(want) if other_bf16 else 0) + 1e-37).all()

    flat_dy, dy = _operand(rng, tokens, cols, ld, off, other_bf16)
    out = (Case(tmp_path, "weight_grad").given(flat_dy, off * es).number(other_bf16, ld).given(flat, c_off * c_es).number(c_bf16, rows, cols, ldc).given(p)
           .number(tokens, slots).output("dw", 4 * tokens * slots).run(driver))
    want, mag = ref.weight_grad(dy, c, p)
    assert (np.abs(np.frombuffer(out["dw"], np.float32).reshape(want.shape) - want) <= (8 * -(-cols // 512) + 16) * 2.0 ** -24 * 1.01 * mag + 1e-37).all()


@pytest.mark.parametrize("c_bf16,dy_bf16", [(False, True), (True, False)])
@pytest.mark.parametrize("cols,ldc,ld", [(2051, 2051, 2053), (4099, 4104, 4100), (2056, 2057, 2056)])
def test_gradient_of_wide_rows_element_by_element(driver, tmp_path, cols, ldc, ld, c_bf16, dy_bf16):  # noqa: F811
    """Whole numbers: exact."""
    rng = np.random.default_rng(cols)
    tokens, slots, rows = 2, 3, 4
    c, dy = rng.integers(-8, 9, (rows, ldc)).astype(np.float32), rng.integers(-8, 9, (tokens, ld)).astype(np.float32)
    p = np.array([[0, 3, -1], [2, 1, 3]], np.int32)
    flat = lambda x, n, bf16: (si.to_bf16_bits(x) if bf16 else x).ravel()[:n]  # noqa: E731
    out = (Case(tmp_path, "weight_grad").given(flat(dy, (tokens - 1) * ld + cols, dy_bf16)).number(dy_bf16, ld).given(flat(c, (rows - 1) * ldc + cols, c_bf16))
           .number(c_bf16, rows, cols, ldc).given(p).number(tokens, slots).output("dw", 4 * tokens * slots).run(driver))
    want, _ = ref.weight_grad(dy[:, :cols], c[:, :cols], p)
    assert np.array_equal(np.frombuffer(out["dw"], np.float32).reshape(want.shape), want.astype(np.float32))
