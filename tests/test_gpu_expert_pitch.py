"""The weighted sum of an entry's rows and the gradient of its weights where a width of whole 16-byte pieces is not enough for accesses of
16 bytes (one operand alone one element off, or with a pitch of an odd number of elements), on wide rows element by element, and where
there is more work than a launch has wavefronts."""
import numpy as np
import pytest
import torch

import experts_reference as ref
import paper_2506_08027_amd as mx
from test_gpu_experts import U, _dev, _host, _positions, _values

pytestmark = pytest.mark.gpu


def _placed(t, ld, off):
    """The matrix t as a view of NaN with that pitch, `off` elements behind an aligned start. Returns (view, all of the memory)."""
    rows, cols = t.shape
    flat = torch.full((off + rows * ld,), float("nan"), dtype=t.dtype, device="cuda")
    view = flat[off:].view(rows, ld)[:, :cols]
    view.copy_(t)
    return view, flat


@pytest.mark.parametrize("c_bf16", [False, True], ids=["c-f32", "c-bf16"])
@pytest.mark.parametrize("other_bf16", [False, True], ids=["other-f32", "other-bf16"])
@pytest.mark.parametrize("which", ["none", "c base", "c pitch", "other base", "other pitch"])
def test_one_operand_off_16_bytes(which, other_bf16, c_bf16):
    rng = np.random.default_rng(3)
    tokens, slots, rows, cols = 9, 5, 14, 576
    layout = lambda what: (cols + (1 if which == what + " pitch" else 8), int(which == what + " base"))  # noqa: E731
    c, c32 = _values(rng, rows, cols, c_bf16)
    other, other32 = _values(rng, tokens, cols, other_bf16)
    c, _ = _placed(c, *layout("c"))
    dy, memory = _placed(other, *layout("other"))
    p, w = _positions(rng, tokens, slots, rows), rng.standard_normal((tokens, slots)).astype(np.float32)
    dw = torch.full((tokens, slots), float("nan"), device="cuda")
    mx.mxfp8_expert_weight_grad(dy, c, _dev(p), dw)
    want, mag = ref.weight_grad(other32, c32, p)
    assert (np.abs(_host(dw) - want) <= (8 * -(-cols // 512) + 16) * U * 1.01 * mag + 1e-37).all()
    memory.fill_(float("nan"))
    mx.mxfp8_expert_combine(c, _dev(p), _dev(w), dy)
    want, mag = ref.combine(c32, p, w)
    got = _host(dy).astype(np.float64)
    assert (np.abs(got - want) <= slots * U * 1.01 * mag + (2.0 ** -8 * 1.01 * np.abs(want) if other_bf16 else 0.0) + 1e-37).all()
    assert int(torch.isnan(memory).sum()) == memory.numel() - tokens * cols, "written outside the rows"


@pytest.mark.parametrize("c_bf16,dy_bf16", [(False, True), (True, False), (True, True)])
@pytest.mark.parametrize("cols,ldc,ld", [(2051, 2051, 2053), (4099, 4104, 4100), (2056, 2057, 2056)])
def test_gradient_of_wide_rows_element_by_element(cols, ldc, ld, c_bf16, dy_bf16):
    """Whole numbers: exact."""
    rng = np.random.default_rng(cols)
    c, dy = rng.integers(-8, 9, (20, cols)).astype(np.float32), rng.integers(-8, 9, (7, cols)).astype(np.float32)
    p = _positions(rng, 7, 3, 20)
    as_type = lambda a, bf16: _dev(a).to(torch.bfloat16 if bf16 else torch.float32)  # noqa: E731
    dw = mx.expert_weight_grad(_placed(as_type(dy, dy_bf16), ld, 0)[0], _placed(as_type(c, c_bf16), ldc, 0)[0], _dev(p))
    assert np.array_equal(_host(dw), ref.weight_grad(dy, c, p)[0].astype(np.float32))


def test_more_work_than_a_launch_has_wavefronts_full_size():
    """More than 2^24 tokens of one column: the first of 4 * 2^22 wavefronts take a second one."""
    tokens, rows = (1 << 24) + 1001, 4099
    g = torch.Generator(device="cuda").manual_seed(1)
    whole = lambda *s: torch.randint(-64, 65, s, generator=g, device="cuda").float()  # noqa: E731
    c, dy, w = whole(rows, 1), whole(tokens, 1), whole(tokens, 1)
    p = torch.randint(-1, rows, (tokens, 1), generator=g, device="cuda", dtype=torch.int32)
    taken = torch.where(p >= 0, c[:, 0][p.clamp(min=0).long()], 0.0)
    out = torch.full((tokens, 1), float("nan"), device="cuda")
    mx.mxfp8_expert_combine(c, p, w, out)
    assert torch.equal(out, taken * w)
    out.fill_(float("nan"))
    mx.mxfp8_expert_weight_grad(dy, c, p, out)
    assert torch.equal(out, taken * dy)
    torch.cuda.synchronize()
