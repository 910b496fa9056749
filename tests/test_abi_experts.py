"""CPU checks of include/mxfp8_experts.h: exports, the binding's names, host arithmetic, and the refusals of every entry point, which come
before any launch."""
import ctypes
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
I64, I32, P, E = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_int
FAKE = P(0x1000)          # aligned and never dereferenced: every call made with it fails validation, or does nothing
OK, NULL, SHAPE, ALIGN, DTYPE, MODE = 0, 1, 2, 3, 4, 5


@pytest.fixture(scope="module")
def lib():
    from paper_2506_08027_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2506_08027_amd.build import build_library
        build_library()
    return ctypes.CDLL(binding.LIB_PATH)


def _declared():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "mxfp8_experts.h")).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(mxfp8_[a-z_0-9]+)\s*\(", text)))


def test_every_declared_function_is_exported_and_bound(lib):
    import paper_2506_08027_amd as mx
    assert _declared() == ["mxfp8_expert_combine", "mxfp8_expert_quantize_ex", "mxfp8_expert_rows", "mxfp8_expert_sort", "mxfp8_expert_sort_workspace",
                           "mxfp8_expert_weight_grad", "mxfp8_fp4_gemv_ex", "mxfp8_fp4_gemv_grouped_ex"]
    for name in _declared():
        assert hasattr(lib, name) and callable(getattr(mx, name)), name
    assert (mx.I32, mx.I64) == (0, 1)


def test_header_compiles_as_c(tmp_path):
    import subprocess
    src = tmp_path / "t.c"
    src.write_text('#include "mxfp8_experts.h"\nint main(void) { return MXFP8_I64 - 1; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), "-c", str(src), "-o", str(tmp_path / "t.o")], check=True)


def test_host_arithmetic(lib):
    rows, ws = lib.mxfp8_expert_rows, lib.mxfp8_expert_sort_workspace
    rows.restype = ws.restype = I64
    rows.argtypes, ws.argtypes = [I64, I32, I32], [I64, I32]
    assert rows(10, 4, 1) == 10 and rows(10, 4, 8) == 32 and rows(2, 64, 128) == 256 and rows(0, 64, 128) == 0 and rows(100, 0, 16) == 96
    for bad in ((-1, 4, 1), (4, -1, 1), (4, 4097, 1), (4, 4, 0), (4, 4, 3), (4, 4, 8192), ((1 << 30) + 1, 1, 1), (1 << 30, 4096, 4096)):
        assert rows(*bad) == -1, bad
    assert ws(100, 64) == 0 and ws(1 << 20, 64) >= 0 and ws(-1, 4) == -1 and ws(4, 4097) == -1
    assert max(rows(n, e, a) for n in (1, 7, 100) for e in (1, 3, 9) for a in (1, 4)) <= 100 + 9 * 3


def test_sort_refuses(lib):
    f = lib.mxfp8_expert_sort
    f.argtypes = [P, E, I64, I32, I32, I64, P, P, P, P, P]
    good = dict(experts=FAKE, t=0, n=10, groups=4, align=8, rows=32, pos=FAKE, src=FAKE, ends=FAKE, ws=None, stream=None)

    def call(**k):
        return f(*{**good, **k}.values())
    assert call(t=2) == DTYPE and call(rows=31) == SHAPE and call(n=-1) == SHAPE and call(groups=4097) == SHAPE and call(align=6) == SHAPE
    assert call(rows=(1 << 30) + 1) == SHAPE
    assert call(experts=None) == NULL and call(pos=None) == NULL and call(src=None) == NULL and call(ends=None) == NULL
    assert call(n=1 << 20, rows=1 << 21) == NULL                                # needs a workspace
    assert call(experts=P(0x1002)) == ALIGN and call(t=1, experts=P(0x1004)) == ALIGN and call(pos=P(0x1001)) == ALIGN and call(ends=P(0x1002)) == ALIGN
    assert call(n=1 << 20, rows=1 << 21, ws=P(0x1002)) == ALIGN
    assert call(n=0, rows=0, groups=0, experts=None, pos=None, src=None, ends=None) == OK


def test_quantize_refuses(lib):
    f = lib.mxfp8_expert_quantize_ex
    f.argtypes = [P, E, I64, I64, I64, P, I32, P, P, I32, I64, E, P, P, P, P, E, P]
    good = dict(src=FAKE, t=0, tokens=8, cols=64, ld=64, sources=FAKE, slots=2, w=FAKE, ends=FAKE, groups=4, rows=32, axis=3, q=FAKE, s=FAKE, qT=FAKE, sT=FAKE,
                lay=0, stream=None)

    def call(**k):
        return f(*{**good, **k}.values())
    assert call(t=2) == DTYPE and call(axis=0) == MODE and call(axis=4) == MODE and call(lay=2) == MODE
    for bad in (dict(tokens=-1), dict(cols=48), dict(cols=-32), dict(ld=32), dict(rows=33), dict(rows=-32), dict(slots=0), dict(slots=4097), dict(groups=-1),
                dict(groups=4097), dict(groups=0), dict(ends=None), dict(tokens=1 << 30, slots=2), dict(rows=(1 << 30) + 32)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(src=None), dict(sources=None), dict(q=None), dict(s=None), dict(qT=None), dict(sT=None)):
        assert call(**bad) == NULL, bad
    for bad in (dict(src=P(0x1008)), dict(ld=66), dict(t=1, ld=68), dict(q=P(0x1004)), dict(qT=P(0x1008)), dict(sources=P(0x1002)), dict(w=P(0x1002)),
                dict(ends=P(0x1002)), dict(lay=1, s=P(0x1004)), dict(lay=1, sT=P(0x1004))):
        assert call(**bad) == ALIGN, bad
    assert call(rows=0, sources=None) == OK and call(cols=0, ld=0, src=None) == OK


@pytest.mark.parametrize("name", ["combine", "weight_grad"])
def test_sums_refuse(lib, name):
    if name == "combine":
        f = lib.mxfp8_expert_combine
        f.argtypes = [P, E, I64, I64, I64, P, P, I64, I32, P, E, I64, P]
        good = dict(c=FAKE, t=0, rows=9, cols=64, ldc=64, pos=FAKE, w=FAKE, tokens=4, slots=2, o=FAKE, ot=0, ldo=64, stream=None)
    else:
        f = lib.mxfp8_expert_weight_grad
        f.argtypes = [P, E, I64, P, E, I64, I64, I64, P, I64, I32, P, P]
        good = dict(o=FAKE, ot=0, ldo=64, c=FAKE, t=0, rows=9, cols=64, ldc=64, pos=FAKE, tokens=4, slots=2, w=FAKE, stream=None)

    def call(**k):
        return f(*{**good, **k}.values())
    assert call(t=2) == DTYPE and call(ot=-1) == DTYPE
    for bad in (dict(rows=-1), dict(cols=-32), dict(ldc=32), dict(ldo=32), dict(tokens=-1), dict(slots=0), dict(slots=4097), dict(tokens=1 << 30),
                dict(rows=(1 << 30) + 1)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(c=None), dict(o=None), dict(pos=None)) + ((dict(w=None),) if name == "weight_grad" else ()):
        assert call(**bad) == NULL, bad
    for bad in (dict(c=P(0x1002)), dict(o=P(0x1006)), dict(t=1, c=P(0x1001)), dict(ot=1, o=P(0x1003)), dict(pos=P(0x1001)), dict(w=P(0x1002))):
        assert call(**bad) == ALIGN, bad
    assert call(tokens=0, c=None, o=None, pos=None, w=None) == OK


def test_gemv_refuses(lib):
    f = lib.mxfp8_fp4_gemv_ex
    f.argtypes = [P, I64, P, P, I64, I64, I64, P, E, I64, E, P]
    good = dict(x=FAKE, ldx=64, q=FAKE, s=FAKE, M=2, N=5, K=64, c=FAKE, t=0, ldc=5, lay=0, stream=None)

    def call(**k):
        return f(*{**good, **k}.values())
    assert call(t=3) == DTYPE and call(lay=-1) == MODE
    for bad in (dict(M=-1), dict(N=-1), dict(K=48), dict(K=-32), dict(ldc=4), dict(ldx=32), dict(M=(1 << 30) + 1), dict(K=(1 << 24) + 32, ldx=1 << 25),
                dict(N=(1 << 30) + 1, ldc=1 << 31), dict(M=1 << 30, N=1 << 30, ldc=1 << 30)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(x=None), dict(q=None), dict(s=None), dict(c=None)):
        assert call(**bad) == NULL, bad
    for bad in (dict(x=P(0x1008)), dict(ldx=68), dict(q=P(0x1008)), dict(lay=1, s=P(0x1004)), dict(c=P(0x1002)), dict(t=1, c=P(0x1001))):
        assert call(**bad) == ALIGN, bad
    assert call(M=0, x=None) == OK and call(N=0, c=None) == OK


def test_grouped_gemv_refuses(lib):
    f = lib.mxfp8_fp4_gemv_grouped_ex
    f.argtypes = [P, I64, I64, P, I32, P, P, P, I32, I64, I64, I64, P, E, I64, E, P]
    good = dict(x=FAKE, tokens=4, ldx=64, src=FAKE, slots=2, q=FAKE, s=FAKE, ends=FAKE, groups=3, M=8, N=5, K=64, c=FAKE, t=0, ldc=5, lay=0, stream=None)

    def call(**k):
        return f(*{**good, **k}.values())
    assert call(t=3) == DTYPE and call(lay=2) == MODE
    for bad in (dict(tokens=-1), dict(slots=0), dict(tokens=1 << 30), dict(groups=-1), dict(groups=4097), dict(M=-1), dict(K=40), dict(ldc=4), dict(ldx=60),
                dict(src=None, tokens=7)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(x=None), dict(q=None), dict(s=None), dict(c=None), dict(ends=None)):
        assert call(**bad) == NULL, bad
    for bad in (dict(x=P(0x1008)), dict(ldx=68), dict(src=P(0x1002)), dict(ends=P(0x1002)), dict(q=P(0x1004)), dict(c=P(0x1003))):
        assert call(**bad) == ALIGN, bad
    assert call(groups=0) == OK and call(M=0) == OK


def test_binding_names_what_is_wrong():
    """Shapes and types that the library cannot see, on host tensors with the check for GPU memory left out."""
    import paper_2506_08027_amd as mx
    from paper_2506_08027_amd import binding, experts
    with pytest.raises(ValueError, match="GPU memory"):
        mx.mxfp8_fp4_gemv_ex(torch.zeros((1, 64), dtype=torch.bfloat16), torch.zeros((4, 32), dtype=torch.uint8), torch.zeros((4, 2), dtype=torch.uint8), torch.zeros((1, 4)))
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)   # noqa: E731
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    f32 = torch.zeros
    calls = [
        (ValueError, "int32 or int64", lambda: mx.mxfp8_expert_sort(f32(4, 2), 1, i32(8), i32(8), i32(4))),
        (ValueError, "int32 or int64", lambda: mx.mxfp8_expert_sort(i32(4, 4)[:, :2], 1, i32(8), i32(8), i32(4))),
        (ValueError, "positions must be", lambda: mx.mxfp8_expert_sort(i32(4, 2), 1, i32(7), i32(8), i32(4))),
        (ValueError, "workspace", lambda: mx.mxfp8_expert_sort(i32(1 << 20), 1, i32(1 << 20), i32(1 << 20), i32(4))),
        (ValueError, "align is", lambda: mx.mxfp8_expert_sort(i32(4, 2), 2 ** 32 + 1, i32(8), i32(8), i32(4))),
        (ValueError, "align is", lambda: mx.mxfp8_expert_rows(8, 4, 2 ** 32 + 1)),
        (ValueError, "groups is", lambda: mx.mxfp8_expert_rows(8, 2 ** 32 + 4, 1)),
        (ValueError, "groups is", lambda: mx.mxfp8_expert_sort_workspace(8, 4 - 2 ** 32)),
        (ValueError, "slots is", lambda: mx.mxfp8_expert_quantize_ex(f32(4, 64), i32(64), i32(2), 2 ** 32 + 2, None, "rowwise", u8(64, 64), u8(64, 2))),
        (ValueError, "slots is", lambda: mx.mxfp8_fp4_gemv_grouped_ex(bf(2, 64), i32(4), 2 ** 32 + 2, u8(3, 4, 32), u8(3, 4, 2), i32(3), f32(4, 4))),
        (mx.MXFP8Error, "bad shape", lambda: mx.mxfp8_expert_sort(i32(4, 2), 4, i32(8), i32(8), i32(4))),
        (ValueError, "multiples of 32", lambda: mx.mxfp8_expert_quantize_ex(f32(4, 64), i32(40), i32(2), 2, None, "rowwise", u8(40, 64), u8(40, 2))),
        (ValueError, "q_row", lambda: mx.mxfp8_expert_quantize_ex(f32(4, 64), i32(64), i32(2), 2, None, "rowwise", u8(32, 64), u8(64, 2))),
        (ValueError, "s_colT", lambda: mx.mxfp8_expert_quantize_ex(f32(4, 64), i32(64), i32(2), 2, None, "colwise", None, None, u8(64, 64), u8(64, 1))),
        (ValueError, "q_colT", lambda: mx.mxfp8_expert_quantize_ex(f32(4, 64), i32(64), i32(2), 2, None, "both", u8(64, 64), u8(64, 2))),
        (ValueError, "weights must be", lambda: mx.mxfp8_expert_quantize_ex(f32(4, 64), i32(64), i32(2), 2, f32(4), "rowwise", u8(64, 64), u8(64, 2))),
        (ValueError, "group_ends is empty", lambda: mx.mxfp8_expert_quantize_ex(f32(4, 64), i32(64), i32(0), 2, None, "rowwise", u8(64, 64), u8(64, 2))),
        (TypeError, "float32 and bfloat16", lambda: mx.mxfp8_expert_quantize_ex(f32(4, 64).half(), i32(64), i32(1), 2, None, "rowwise", u8(64, 64), u8(64, 2))),
        (ValueError, "weights must be", lambda: mx.mxfp8_expert_combine(f32(8, 64), i32(4, 2), f32(4, 2).double(), f32(4, 64))),
        (ValueError, "out must be", lambda: mx.mxfp8_expert_combine(f32(8, 64), i32(4, 2), None, f32(5, 64))),
        (ValueError, "tokens x slots", lambda: mx.mxfp8_expert_combine(f32(8, 64), i32(8), None, f32(4, 64))),
        (ValueError, "c must be", lambda: mx.mxfp8_expert_combine(f32(64, 8).t(), i32(4, 2), None, f32(4, 64))),
        (ValueError, "dy must be", lambda: mx.mxfp8_expert_weight_grad(f32(4, 32), f32(8, 64), i32(4, 2), f32(4, 2))),
        (ValueError, "dweights", lambda: mx.mxfp8_expert_weight_grad(f32(4, 64), f32(8, 64), i32(4, 2), f32(4, 3))),
        (TypeError, "bfloat16", lambda: mx.mxfp8_fp4_gemv_ex(f32(1, 64), u8(4, 32), u8(4, 2), f32(1, 4))),
        (ValueError, "w_q", lambda: mx.mxfp8_fp4_gemv_ex(bf(1, 64), u8(4, 64), u8(4, 2), f32(1, 4))),
        (ValueError, "w_s", lambda: mx.mxfp8_fp4_gemv_ex(bf(1, 64), u8(4, 32), u8(4, 1), f32(1, 4))),
        (ValueError, "c must be", lambda: mx.mxfp8_fp4_gemv_ex(bf(1, 64), u8(4, 32), u8(4, 2), f32(2, 4))),
        (ValueError, "sources must be", lambda: mx.mxfp8_fp4_gemv_grouped_ex(bf(2, 64), i32(3), 2, u8(3, 4, 32), u8(3, 4, 2), i32(3), f32(4, 4))),
        (ValueError, "x has 2 rows", lambda: mx.mxfp8_fp4_gemv_grouped_ex(bf(2, 64), None, 1, u8(3, 4, 32), u8(3, 4, 2), i32(3), f32(4, 4))),
        (ValueError, "w_q must be", lambda: mx.mxfp8_fp4_gemv_grouped_ex(bf(4, 64), None, 1, u8(2, 4, 32), u8(3, 4, 2), i32(3), f32(4, 4))),
        (ValueError, "w_s must be", lambda: mx.mxfp8_fp4_gemv_grouped_ex(bf(4, 64), None, 1, u8(3, 4, 32), u8(2, 4, 2), i32(3), f32(4, 4))),
    ]
    keep = binding._need_cuda, binding._stream
    binding._need_cuda, binding._stream = lambda *t: None, lambda s: None
    try:
        for kind, text, call in calls:
            with pytest.raises(kind, match=text):
                call()
    finally:
        binding._need_cuda, binding._stream = keep
    assert experts.MXFP8Error is mx.MXFP8Error


def test_calls_in_cpp_leave_other_arguments_to_python():
    """-1: not handled; the binding then names what is wrong."""
    from paper_2506_08027_amd import binding
    binding.load()
    if binding._fast is None:
        pytest.skip("the module of the calls in C++ is not built")
    host = torch.zeros((4, 64), dtype=torch.bfloat16)
    for name, n in (("expert_sort", 7), ("expert_quantize", 12), ("expert_combine", 5), ("expert_weight_grad", 5), ("fp4_gemv", 6), ("fp4_gemv_grouped", 9)):
        call = getattr(binding._fast, name)
        for args in ((), (host,) * n, (None,) * n, ("x",) * n, (host,) * (n + 1)):
            assert call(*args) == -1, (name, len(args))
