"""The quantizer of sorted rows where its resident grid takes several tiles a workgroup, on the CPU execution model with
AddressSanitizer: a device of one unit has four workgroups (both copies) or eight (one copy) for the 21 or 27 tiles here, with other
rows and weights in each of them, walked across and down. A tile that is left out, taken by two or read with another's rows or
weights shows in the bytes."""
import numpy as np
import pytest

import experts_reference as ref
import scale_layout as sl
from paper_2506_08027_amd import synth_inputs as si
from test_host_model_experts import Case, driver  # noqa: F401


# cols, rows, end of the last expert: 3 x 7 tiles walked across (more rows than columns), 9 x 3 walked down where there is a column copy
@pytest.mark.parametrize("cols,rows,end", [(288, 1056, 800), (1056, 480, 300)], ids=["across", "down"])
@pytest.mark.parametrize("axis", [1, 2, 3])
@pytest.mark.parametrize("bf16,weighted,tiled,order", [(False, False, True, "up"), (True, False, False, "down"), (True, True, True, "down"), (False, True, False, "up")])
def test_quantizer_walks_over_all_tiles(driver, tmp_path, bf16, weighted, tiled, axis, cols, rows, end, order):  # noqa: F811
    rng = np.random.default_rng(cols + axis)
    tokens, slots, ld, workgroups = 300, 3, cols + 8, 4 if axis == 3 else 8
    assert -(-cols // 128) * -(-end // 128) > 2 * workgroups
    x = rng.standard_normal((tokens, ld)).astype(np.float32)
    bits = si.to_bf16_bits(x)
    src, x = (bits, si.bf16_bits_to_f32(bits)) if bf16 else (x, x)
    sources = rng.integers(0, tokens * slots, rows).astype(np.int32)
    sources[rng.random(rows) < 0.1] = -1
    w = rng.standard_normal(tokens * slots).astype(np.float32) if weighted else None
    size = lambda r, c: sl.tiled_bytes(r, c // 32) if tiled else r * (c // 32)  # noqa: E731
    case = Case(tmp_path, "quantize").given(src.ravel()[:(tokens - 1) * ld + cols]).number(bf16, tokens, cols, ld).given(sources).number(slots).given(w)
    case.given(np.array([end // 2, end], np.int32)).number(2, rows, axis)
    for want, name, r, c in ((axis & 1, "row", rows, cols), (axis & 2, "colT", cols, rows)):
        case.output("q_" + name, r * c).output("s_" + name, size(r, c)) if want else case.null().null()
    out = case.number(tiled).run(driver, order, cus=1)
    v = ref.sorted_rows(x[:, :cols], sources, slots, None if w is None else w.reshape(tokens, slots))
    live = -(-end // 128) * 128
    for name in ("row", "colT"):
        if "q_" + name in out:
            q, s = ref.quantized(v, name)
            got_q, got_s = (np.frombuffer(out[k + name], np.uint8) for k in ("q_", "s_"))
            got_q, got_s = got_q.reshape(q.shape), sl.untile(got_s, *s.shape) if tiled else got_s.reshape(s.shape)
            if name == "colT":
                q, s, got_q, got_s = q.T, np.repeat(s, 32, 1).T, got_q.T, np.repeat(got_s, 32, 1).T
            assert np.array_equal(got_q[:live], q[:live]) and np.array_equal(got_s[:live], s[:live]), name
            assert (got_q[live:] == 0xA5).all() and (got_s[live:] == 0xA5).all(), name
