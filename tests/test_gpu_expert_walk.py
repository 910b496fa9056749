"""The quantizer of sorted rows where its resident grid (four workgroups a unit for both copies, eight for one) takes several tiles a
workgroup, against the oracle's bytes: walked across, and down a wide tensor's columns, partial tiles at both edges."""
import numpy as np
import pytest
import torch

import experts_reference as ref
import paper_2506_08027_amd as mx
import scale_layout as sl
from test_gpu_experts import _dev, _experts, _values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,slots,groups,cols,axis,bf16,weighted,tiled", [
    (12000, 2, 8, 1440, "both", True, False, True),          # some 2250 tiles, across
    (16000, 2, 4, 1440, "rowwise", True, True, False),       # some 3000, across
    (500, 2, 3, 20000, "both", False, True, False),          # some 1400, down
    (500, 2, 2, 40000, "colwise", False, False, True),       # some 2800, down
    (10000, 2, 2, 2080, "colwise", True, True, True),        # some 2700, across
])
def test_quantizer_walks_over_all_tiles_full_size(tokens, slots, groups, cols, axis, bf16, weighted, tiled):
    rng = np.random.default_rng(cols)
    src, src32 = _values(rng, tokens, cols, bf16)
    w = rng.standard_normal((tokens, slots)).astype(np.float32) if weighted else None
    experts = _experts(rng, tokens, slots, groups, 0.02)
    rows = ref.rows_needed(experts.size, groups, 128) + 96   # the last tile is a partial one
    _, sources, ends = ref.plan(experts, groups, 128, rows)
    ends[-1] = rows - 32                                     # rows of the padding are converted too: every tile is live
    units = torch.cuda.get_device_properties(0).multi_processor_count
    assert -(-rows // 128) * -(-cols // 128) > units * (4 if axis == "both" else 8), "no workgroup has a second tile"
    lay, out = mx.SCALES_TILED if tiled else mx.SCALES_ROWMAJOR, {}
    for name, wanted, r, c in (("row", axis != "colwise", rows, cols), ("colT", axis != "rowwise", cols, rows)):
        if wanted:
            out["q_" + name] = torch.full((r, c), 0xA5, dtype=torch.uint8, device="cuda")
            out["s_" + name] = torch.full((mx.mxfp8_scale_bytes(r, c, lay),) if tiled else (r, c // 32), 0xA5, dtype=torch.uint8, device="cuda")
    mx.mxfp8_expert_quantize_ex(src, _dev(sources), _dev(ends), slots, None if w is None else _dev(w), axis, **out, scale_layout=lay)
    torch.cuda.synchronize()
    v = ref.sorted_rows(src32, sources, slots, w)
    for name in ("row", "colT"):
        if "q_" + name in out:
            q, s = ref.quantized(v, name)
            got_s = out["s_" + name].cpu().numpy()
            assert np.array_equal(out["q_" + name].cpu().numpy(), q) and np.array_equal(sl.untile(got_s, *s.shape) if tiled else got_s, s), name
