"""The expert rows and the MXFP4 products of a few rows on the CPU execution model, with AddressSanitizer on buffers of their exact
size: no access leaves a buffer for odd sizes, plans whose numbers are wrong included, inputs stay as they are and nothing is written
beside the outputs. Values against the definitions, so that a wrong index shows too."""
import os
import subprocess

import numpy as np
import pytest

import experts_reference as ref
import scale_layout as sl
from paper_2506_08027_amd import synth_inputs as si

HERE = os.path.dirname(os.path.abspath(__file__))
BUILD, BINARY = os.path.join(HERE, "host_model", "build.sh"), os.path.join(HERE, "host_model", "_build", "hostmodel_experts")
ORDERS = ["up", "down"]


@pytest.fixture(scope="session")
def driver():
    mine = f"{BINARY}.{os.getpid()}"   # test processes side by side do not build over each other
    res = subprocess.run([BUILD, "--experts", mine], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    os.replace(mine, BINARY)
    return BINARY


class Case:
    """One call: arguments as the driver wants them, its outputs after run()."""

    def __init__(self, tmp_path, name):
        self.dir, self.words, self.outputs = tmp_path, [name], {}

    def number(self, *values):
        self.words += [str(int(v)) for v in values]
        return self

    def null(self):
        self.words.append("null")
        return self

    def given(self, array, off=0):
        if array is None:
            return self.null()
        path = self.dir / f"in{len(self.words)}.bin"
        np.ascontiguousarray(array).tofile(path)
        self.words.append((f"off:{off}:" if off else "") + f"in:{path}")
        return self

    def output(self, name, nbytes, off=0):
        path = self.dir / f"{name}.bin"
        self.outputs[name] = path
        self.words.append((f"off:{off}:" if off else "") + f"out:{path}:{int(nbytes)}")
        return self

    def run(self, driver, order="up", status=0, cus=3):
        case = self.dir / "case.txt"
        case.write_text(" ".join(self.words) + "\n")
        res = subprocess.run([driver, str(case)], capture_output=True, text=True, timeout=600, env=dict(os.environ, WAVESIM_ORDER=order, WAVESIM_CUS=str(cus)))
        assert res.returncode == 0, (res.stdout + res.stderr)[-4000:]
        assert res.stdout.split()[:2] == ["status", str(status)], res.stdout
        return {name: path.read_bytes() for name, path in self.outputs.items()}


def _i32(b):
    return np.frombuffer(b, np.int32)


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("entries,groups,align,extra,index64", [(1, 1, 1, 0, False), (70, 5, 32, 7, True), (300, 70, 4, 0, False), (1030, 3, 128, 5, False),
                                                                (0, 4, 8, 9, False), (33, 0, 1, 3, True), (260, 1100, 2, 0, False)])
def test_sort(driver, tmp_path, entries, groups, align, extra, index64, order):
    rng = np.random.default_rng(entries)
    experts = rng.integers(-2, groups + 2, entries)
    rows = ref.rows_needed(entries, groups, align) + extra
    out = (Case(tmp_path, "sort").given(experts.astype(np.int64 if index64 else np.int32)).number(index64, entries, groups, align, rows)
           .output("positions", 4 * entries).output("sources", 4 * rows).output("ends", 4 * groups).null().run(driver, order))
    for name, want in zip(("positions", "sources", "ends"), ref.plan(experts, groups, align, rows)):
        assert np.array_equal(_i32(out[name]), want), name


@pytest.mark.parametrize("groups", [7, 1500])
def test_sort_in_two_launches(driver, tmp_path, groups):
    entries, align = 33000, 64
    experts = np.random.default_rng(1).integers(-1, groups, entries)
    rows = ref.rows_needed(entries, groups, align) + 3
    out = (Case(tmp_path, "sort").given(experts.astype(np.int32)).number(0, entries, groups, align, rows).output("positions", 4 * entries)
           .output("sources", 4 * rows).output("ends", 4 * groups).output("workspace", -(-entries // 1024) * groups * 4).run(driver))
    for name, want in zip(("positions", "sources", "ends"), ref.plan(experts, groups, align, rows)):
        assert np.array_equal(_i32(out[name]), want), name


BAD_SOURCES = [-1, -2, 2 ** 31 - 1, -2 ** 31]


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("axis", [1, 2, 3])
@pytest.mark.parametrize("bf16,weighted,tiled,ld", [(False, False, False, 96), (True, False, True, 104), (True, True, False, 96), (False, True, True, 100)])
def test_quantize_of_sorted_rows(driver, tmp_path, bf16, weighted, tiled, ld, axis, order):
    rng = np.random.default_rng(ld)
    tokens, slots, cols, rows = 11, 3, 96, 288
    x = rng.standard_normal((tokens, ld)).astype(np.float32)
    bits = si.to_bf16_bits(x)
    src, x = (bits, si.bf16_bits_to_f32(bits)) if bf16 else (x, x)
    used = src.ravel()[:(tokens - 1) * ld + cols]
    sources = rng.choice(np.array(list(range(tokens * slots)) + [tokens * slots, tokens * slots + 5] + BAD_SOURCES), rows).astype(np.int32)
    w = rng.random(tokens * slots).astype(np.float32) if weighted else None
    lay = int(tiled)
    size = lambda r, c: sl.tiled_bytes(r, c // 32) if tiled else r * (c // 32)  # noqa: E731
    case = Case(tmp_path, "quantize").given(used).number(bf16, tokens, cols, ld).given(sources).number(slots).given(w)
    case.given(np.array([40, 100], np.int32)).number(2, rows, axis)
    for want, name, r, c in ((axis & 1, "row", rows, cols), (axis & 2, "colT", cols, rows)):
        case.output("q_" + name, r * c).output("s_" + name, size(r, c)) if want else case.null().null()
    out = case.number(lay).run(driver, order)
    v = ref.sorted_rows(x[:, :cols], sources, slots, None if w is None else w.reshape(tokens, slots))
    live = 128                                            # the last end, 100, lies in the first tile of 128 rows
    for name in ("row", "colT"):
        if "q_" + name in out:
            q, s = ref.quantized(v, name)
            got_q, got_s = (np.frombuffer(out[k + name], np.uint8) for k in ("q_", "s_"))
            got_q, got_s = got_q.reshape(q.shape), sl.untile(got_s, *s.shape) if tiled else got_s.reshape(s.shape)
            if name == "colT":
                q, s, got_q, got_s = q.T, np.repeat(s, 32, 1).T, got_q.T, np.repeat(got_s, 32, 1).T
            assert np.array_equal(got_q[:live], q[:live]) and np.array_equal(got_s[:live], s[:live])
            assert (got_q[live:] == 0xA5).all() and (got_s[live:] == 0xA5).all()


def _rows(rng, rows, cols, ld, bf16):
    """(what lies in memory, values as float32)"""
    x = rng.standard_normal((rows, ld)).astype(np.float32)
    bits = si.to_bf16_bits(x)
    flat = (bits if bf16 else x).ravel()[:max((rows - 1) * ld + cols, 0)]
    return flat, (si.bf16_bits_to_f32(bits) if bf16 else x)[:, :cols]


@pytest.mark.parametrize("c_bf16,out_bf16,weighted", [(False, False, False), (True, True, True), (False, True, True), (True, False, False)])
@pytest.mark.parametrize("tokens,slots,rows,cols,ld", [(1, 1, 1, 32, 32), (5, 3, 4, 544, 552), (2, 9, 0, 64, 64), (3, 2, 5, 77, 77), (2, 2, 3, 9, 16)])
def test_combine_and_weight_grad(driver, tmp_path, tokens, slots, rows, cols, ld, c_bf16, out_bf16, weighted):
    rng = np.random.default_rng(cols)
    flat, c = _rows(rng, rows, cols, ld, c_bf16)
    p = rng.choice(np.array(list(range(rows)) + [rows, rows + 7] + BAD_SOURCES), (tokens, slots)).astype(np.int32)
    w = rng.standard_normal((tokens, slots)).astype(np.float32) if weighted else None
    es = 2 if out_bf16 else 4
    out = (Case(tmp_path, "combine").given(flat).number(c_bf16, rows, cols, ld).given(p).given(w).number(tokens, slots)
           .output("out", ((tokens - 1) * (cols + 8) + cols) * es).number(out_bf16, cols + 8).run(driver))
    raw = np.full(tokens * (cols + 8) * es, 0xA5, np.uint8)
    raw[:len(out["out"])] = np.frombuffer(out["out"], np.uint8)
    raw = raw.view(np.uint16 if out_bf16 else np.uint32).reshape(tokens, cols + 8)
    assert (raw[:, cols:] == (0xA5A5 if out_bf16 else 0xA5A5A5A5)).all()
    got = (si.bf16_bits_to_f32(raw[:, :cols]) if out_bf16 else raw[:, :cols].view(np.float32)).astype(np.float64)
    want, mag = ref.combine(c, p, w)
    assert (np.abs(got - want) <= slots * 2.0 ** -24 * 1.01 * mag + (2.0 ** -8 * 1.01 * np.abs(want) if out_bf16 else 0) + 1e-37).all()

    flat_dy, dy = _rows(rng, tokens, cols, ld, out_bf16)
    got = (Case(tmp_path, "weight_grad").given(flat_dy).number(out_bf16, ld).given(flat).number(c_bf16, rows, cols, ld).given(p).number(tokens, slots)
           .output("dw", 4 * tokens * slots).run(driver))
    want, mag = ref.weight_grad(dy, c, p)
    assert (np.abs(np.frombuffer(got["dw"], np.float32).reshape(want.shape) - want) <= (8 * -(-cols // 512) + 16) * 2.0 ** -24 * 1.01 * mag + 1e-37).all()


def _gemv_values(rng, rows, K, ldx):
    x = rng.integers(-3, 4, (rows, ldx)).astype(np.float32)
    return si.to_bf16_bits(x).ravel()[:max((rows - 1) * ldx + K, 0)], x[:, :K]


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("tiled,bf16,off", [(False, False, 0), (True, True, 0), (False, True, 2)])
@pytest.mark.parametrize("M,N,K,ldx,ldc", [(1, 1, 32, 32, 1), (3, 21, 160, 168, 24), (16, 16, 1056, 1056, 16), (17, 33, 96, 104, 40), (50, 18, 64, 64, 18), (70, 16, 288, 288, 19)])
def test_gemv(driver, tmp_path, M, N, K, ldx, ldc, tiled, bf16, off, order):
    _check_gemv(driver, tmp_path, M, N, K, ldx, ldc, tiled, bf16, off, order)


# tiles of W by twos and fours: many columns
@pytest.mark.parametrize("M,N,K,tiled", [(6, 16390, 32, True), (11, 16384, 64, False), (20, 8200, 32, False),
                                         pytest.param(40, 16390, 32, True, marks=pytest.mark.slow),
                                         pytest.param(8, 16390, 1120, False, marks=pytest.mark.slow), (33, 4100, 160, True)])
def test_gemv_of_many_columns(driver, tmp_path, M, N, K, tiled):
    _check_gemv(driver, tmp_path, M, N, K, K, N, tiled, False, 0, "down")


def _check_gemv(driver, tmp_path, M, N, K, ldx, ldc, tiled, bf16, off, order):
    rng = np.random.default_rng(K)
    flat, x = _gemv_values(rng, M, K, ldx)
    w_q, w_s = rng.integers(0, 256, (N, K // 2), dtype=np.uint8), rng.integers(126, 129, (N, K // 32)).astype(np.uint8)
    es, n = 2 if bf16 else 4, (M - 1) * ldc + N
    out = (Case(tmp_path, "gemv").given(flat).number(ldx).given(w_q).given(sl.tile(w_s, filler=0xFF) if tiled else w_s).number(M, N, K)
           .output("c", n * es + off, off).number(bf16, ldc, tiled).run(driver, order))
    assert out["c"][:off] == b"\xa5" * off
    raw = np.full(M * ldc, 0xA5A5 if bf16 else 0xA5A5A5A5, np.uint16 if bf16 else np.uint32)
    raw[:n] = np.frombuffer(out["c"][off:], raw.dtype)
    raw = raw.reshape(M, ldc)
    assert (raw[:, N:] == (0xA5A5 if bf16 else 0xA5A5A5A5)).all()
    want, _ = ref.gemv(x, w_q, w_s)                       # whole numbers of quarters: exact in FP32
    if bf16:
        assert np.array_equal(raw[:, :N], si.to_bf16_bits(want.astype(np.float32)))
    else:
        assert np.array_equal(np.ascontiguousarray(raw[:, :N]).view(np.float32), want)


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("tiled", [False, True], ids=["rowmajor", "tiled"])
@pytest.mark.parametrize("ends", [[3, 3, 20, 41], [-4, 9, 1 << 30, 5], [0, 0, 0, 0], [50, 50, 50, 50], [1] * 70 + [44]], ids=["some", "bad", "none", "one", "many"])
def test_gemv_grouped(driver, tmp_path, ends, tiled, order):
    rng = np.random.default_rng(len(ends))
    tokens, slots, rows, N, K = 7, 2, 50, 20, 96
    flat, x = _gemv_values(rng, tokens, K, K)
    groups = len(ends)
    w_q, w_s = rng.integers(0, 256, (groups, N, K // 2), dtype=np.uint8), rng.integers(126, 129, (groups, N, K // 32)).astype(np.uint8)
    sources = rng.choice(np.array(list(range(tokens * slots)) + [tokens * slots] + BAD_SOURCES), rows).astype(np.int32)
    scales = np.concatenate([sl.tile(s, filler=0xFF).ravel() for s in w_s]) if tiled else w_s
    out = (Case(tmp_path, "gemv_grouped").given(flat).number(tokens, K).given(sources).number(slots).given(w_q).given(scales)
           .given(np.array(ends, np.int32)).number(groups, rows, N, K).output("c", rows * N * 4).number(0, N, tiled).run(driver, order))
    got = np.frombuffer(out["c"], np.uint32).reshape(rows, N)
    if ends[:1] == [-4]:
        return                                            # ends that decrease: any values, but inside the buffers
    want, _ = ref.gemv_grouped(x, sources, slots, w_q, w_s, ends, rows)
    owned = ~np.isnan(want)
    assert (got[~owned] == 0xA5A5A5A5).all() and np.array_equal(got.view(np.float32)[owned], want[owned])
