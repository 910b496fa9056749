// The calls of the binding for the ordinary case: every argument as the entry points want it, tensors in GPU memory. Anything
// else (NOT_HANDLED) goes through binding.py, which checks again, converts what can be converted and names what cannot be.
//
// The last argument of each is the binding's `stream`, passes and axes are what its caller gave.
// Why: a small kernel lasts 3 .. 5 us and HIP takes 2.9 us to launch it, while the checks in Python (a dozen attributes of five
// or six tensors) took 2.3 .. 3 us and the call through ctypes 0.6 us. Here the checks cost 0.1 us and the call 0.2 us.
// The library's entry points are handed over by address, so that this module and the binding call the same library.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <initializer_list>

namespace {

constexpr long NOT_HANDLED = -1;
constexpr int kRowwise = 1, kColwise = 2, kTiled = 1;
// entry points, in the order of the names below
enum { QUANTIZE, GEMM, GEMM_MODE, DEQUANTIZE, GEMM_BF16, GEMM_QUANTIZE, FP4_QUANTIZE, FP4_GEMM, FP6_QUANTIZE, EXPERT_SORT, EXPERT_SORT_WORKSPACE,
       EXPERT_QUANTIZE, EXPERT_COMBINE, EXPERT_WEIGHT_GRAD, FP4_GEMV, FP4_GEMV_GROUPED, B128_QUANTIZE, B128_GEMM_WORKSPACE, B128_GEMM, B128_GEMV,
       EXPERT_LAYER_WORKSPACE, EXPERT_LAYER, ENTRY_POINTS };
const char *const kNames[ENTRY_POINTS] = {"mxfp8_quantize_mode_ex", "mxfp8_gemm_ex", "mxfp8_gemm_mode_ex", "mxfp8_dequantize_mode_ex",
                                          "mxfp8_gemm_bf16", "mxfp8_gemm_quantize_ex", "mxfp8_fp4_quantize_ex",
                                          "mxfp8_fp4_gemm_ex", "mxfp8_fp6_quantize_ex", "mxfp8_expert_sort", "mxfp8_expert_sort_workspace",
                                          "mxfp8_expert_quantize_ex", "mxfp8_expert_combine", "mxfp8_expert_weight_grad", "mxfp8_fp4_gemv_ex",
                                          "mxfp8_fp4_gemv_grouped_ex", "mxfp8_b128_quantize", "mxfp8_b128_gemm_workspace", "mxfp8_b128_gemm",
                                          "mxfp8_b128_gemv", "mxfp8_expert_layer_workspace", "mxfp8_expert_layer"};
void *entry[ENTRY_POINTS];
// The binding's own: names and constants of passes and axes (dicts), and the function that turns its `stream` argument into a handle.
PyObject *passes, *axes, *stream_handle;

// Arguments of a call, taken one after the other; `ok` turns false at the first one that is not what it has to be.
struct Args {
    PyObject *const *args;
    Py_ssize_t left;
    bool ok = true;
    PyObject *next()
    {
        if (left <= 0) {
            ok = false;
            return Py_None;
        }
        --left;
        return *args++;
    }
    int64_t number(int64_t lo, int64_t hi)
    {
        PyObject *o = next();
        if (!PyLong_CheckExact(o)) {
            ok = false;
            return lo;
        }
        int overflow = 0;
        const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
        if (overflow || v < lo || v > hi)
            ok = false;
        return v;
    }
    // what `table` has for the next argument
    int64_t code(PyObject *table, int64_t lo, int64_t hi)
    {
        PyObject *v = table ? PyDict_GetItem(table, next()) : nullptr;  // (nullptr also for what cannot be looked up)
        const long long c = v && PyLong_CheckExact(v) ? PyLong_AsLong(v) : lo - 1;
        if (c < lo || c > hi)
            ok = false;
        return c;
    }
    // a tensor in GPU memory; nullptr for None where that is allowed
    const at::Tensor *tensor(bool none_allowed = false)
    {
        PyObject *o = next();
        if (o == Py_None && none_allowed)
            return nullptr;
        if (THPVariable_CheckTypeExact(Py_TYPE(o))) {  // subclasses may answer for themselves
            const at::Tensor &t = THPVariable_Unpack(o);
            if (t.defined() && t.layout() == at::kStrided && t.is_cuda())
                return &t;
        }
        ok = false;
        return nullptr;
    }
};

uint8_t *ptr(const at::Tensor *t) { return t ? static_cast<uint8_t *>(t->data_ptr()) : nullptr; }
bool dense_bytes(const at::Tensor &t) { return t.scalar_type() == at::kByte && t.is_contiguous(); }
bool dense_matrix(const at::Tensor &t, int64_t rows, int64_t cols) { return t.dim() == 2 && t.size(0) == rows && t.size(1) == cols && dense_bytes(t); }
// scale bytes of an operand [rows x cols]
bool scales(const at::Tensor &s, int64_t rows, int64_t cols, int64_t layout)
{
    if (!dense_bytes(s) || cols % 32)
        return false;
    if (layout == kTiled)
        return s.numel() >= (rows + 63) / 64 * ((cols / 32 + 3) / 4) * 256;
    return s.dim() == 2 && s.size(0) == rows && s.size(1) == cols / 32;
}
// a matrix of FP32 or BF16 values with contiguous rows
struct Values {
    bool ok;
    int dtype;
    int64_t ld;
};
Values values(const at::Tensor &t, int64_t rows, int64_t cols)
{
    const auto type = t.scalar_type();
    const bool ok = t.dim() == 2 && t.size(0) == rows && t.size(1) == cols && rows > 0 && cols > 0 && t.stride(1) == 1 &&
                    (type == at::kFloat || type == at::kBFloat16);
    return {ok, type == at::kBFloat16 ? 1 : 0, ok && rows > 1 ? t.stride(0) : cols};
}

PyObject *not_handled() { return PyLong_FromLong(NOT_HANDLED); }
// The binding asks for the stream after its checks, so that a wrong tensor is reported as one on a machine without a GPU too.
template <class F, class... A> PyObject *call(int which, PyObject *stream, A... args)
{
    if (!entry[which] || !stream_handle)
        return not_handled();
    PyObject *h = PyObject_CallFunctionObjArgs(stream_handle, stream, nullptr);
    if (!h)
        return nullptr;
    void *handle = PyLong_CheckExact(h) ? PyLong_AsVoidPtr(h) : nullptr;
    const bool ok = PyLong_CheckExact(h) && !PyErr_Occurred();
    Py_DECREF(h);
    if (!ok) {
        PyErr_Clear();
        return not_handled();
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = reinterpret_cast<F>(entry[which])(args..., handle);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// The copies of a quantizer: q_row, s_row, q_colT, s_colT; `num` / `den` bytes per element
struct Copies {
    const at::Tensor *q_row, *s_row, *q_colT, *s_colT;
};
bool copies(Args &a, Copies &c, int64_t rows, int64_t cols, int64_t axis, int64_t layout, int num, int den)
{
    const bool row = axis & kRowwise, col = axis & kColwise;
    return a.ok && (!row || (c.q_row && c.s_row && dense_bytes(*c.q_row) && c.q_row->numel() == rows * cols / den * num && scales(*c.s_row, rows, cols, layout))) &&
           (!col || (c.q_colT && c.s_colT && dense_bytes(*c.q_colT) && c.q_colT->numel() == rows * cols / den * num && scales(*c.s_colT, cols, rows, layout)));
}

using I = int64_t;
using P = const uint8_t *;
using Q = uint8_t *;

// src, axis, element, rule, q_row, s_row, q_colT, s_colT, layout, stream; FP4: no element and rule, FP6: no rule
template <int WHICH> PyObject *quantize(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args a{args, n};
    const at::Tensor *src = a.tensor();
    const int64_t axis = a.code(axes, 1, 3), element = WHICH == FP4_QUANTIZE ? 0 : a.number(0, 1), rule = WHICH == QUANTIZE ? a.number(0, 1) : 0;
    Copies c;
    c.q_row = a.tensor(true);
    c.s_row = a.tensor(true);
    c.q_colT = a.tensor(true);
    c.s_colT = a.tensor(true);
    const int64_t layout = a.number(0, 1);
    PyObject *stream = a.next();
    if (!a.ok || a.left || src->dim() != 2)
        return not_handled();
    const int64_t rows = src->size(0), cols = src->size(1);
    const Values v = values(*src, rows, cols);
    if (!v.ok || !copies(a, c, rows, cols, axis, layout, WHICH == FP6_QUANTIZE ? 3 : 1, WHICH == FP6_QUANTIZE ? 4 : WHICH == FP4_QUANTIZE ? 2 : 1))
        return not_handled();
    if constexpr (WHICH == QUANTIZE)
        return call<int (*)(P, int, I, I, I, int, int, int, Q, Q, Q, Q, int, void *)>(
            WHICH, stream, ptr(src), v.dtype, rows, cols, v.ld, (int)axis, (int)element, (int)rule, ptr(c.q_row), ptr(c.s_row), ptr(c.q_colT),
            ptr(c.s_colT), (int)layout);
    else if constexpr (WHICH == FP6_QUANTIZE)
        return call<int (*)(P, int, I, I, I, int, int, Q, Q, Q, Q, int, void *)>(WHICH, stream, ptr(src), v.dtype, rows, cols, v.ld, (int)axis, (int)element,
                                                                                ptr(c.q_row), ptr(c.s_row), ptr(c.q_colT), ptr(c.s_colT), (int)layout);
    else
        return call<int (*)(P, int, I, I, I, int, Q, Q, Q, Q, int, void *)>(WHICH, stream, ptr(src), v.dtype, rows, cols, v.ld, (int)axis, ptr(c.q_row),
                                                                           ptr(c.s_row), ptr(c.q_colT), ptr(c.s_colT), (int)layout);
}

// pass, a_q, a_s, [a_element,] b_q, b_s, [b_element,] c, layout, max_workgroups, stream
template <int WHICH> PyObject *gemm(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args a{args, n};
    const int64_t pass = a.code(passes, 0, 2);
    const at::Tensor *a_q = a.tensor(), *a_s = a.tensor();
    const int64_t a_element = WHICH == GEMM_MODE ? a.number(0, 1) : 0;
    const at::Tensor *b_q = a.tensor(), *b_s = a.tensor();
    const int64_t b_element = WHICH == GEMM_MODE ? a.number(0, 1) : 0;
    const at::Tensor *c = a.tensor();
    const int64_t layout = a.number(0, 1), bound = a.number(0, INT32_MAX);
    PyObject *stream = a.next();
    if (!a.ok || a.left || a_q->dim() != 2 || b_q->dim() != 2)
        return not_handled();
    const int64_t M = a_q->size(0), N = b_q->size(0), bytes = a_q->size(1), K = WHICH == FP4_GEMM ? 2 * bytes : bytes;
    const Values v = values(*c, M, N);
    if (!v.ok || !dense_matrix(*a_q, M, bytes) || !dense_matrix(*b_q, N, bytes) || !scales(*a_s, M, K, layout) || !scales(*b_s, N, K, layout))
        return not_handled();
    if constexpr (WHICH == GEMM_MODE)
        return call<int (*)(int, P, P, int, P, P, int, I, I, I, void *, int, I, int, int32_t, void *)>(
            WHICH, stream, (int)pass, ptr(a_q), ptr(a_s), (int)a_element, ptr(b_q), ptr(b_s), (int)b_element, M, N, K, (void *)ptr(c), v.dtype, v.ld,
            (int)layout, (int32_t)bound);
    else
        return call<int (*)(int, P, P, P, P, I, I, I, void *, int, I, int, int32_t, void *)>(
            WHICH, stream, (int)pass, ptr(a_q), ptr(a_s), ptr(b_q), ptr(b_s), M, N, K, (void *)ptr(c), v.dtype, v.ld, (int)layout, (int32_t)bound);
}

// q, s, element, dst, layout, stream
PyObject *dequantize(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args a{args, n};
    const at::Tensor *q = a.tensor(), *s = a.tensor();
    const int64_t element = a.number(0, 1);
    const at::Tensor *dst = a.tensor();
    const int64_t layout = a.number(0, 1);
    PyObject *stream = a.next();
    if (!a.ok || a.left || q->dim() != 2)
        return not_handled();
    const int64_t rows = q->size(0), cols = q->size(1);
    const Values v = values(*dst, rows, cols);
    if (!v.ok || !dense_bytes(*q) || !scales(*s, rows, cols, layout))
        return not_handled();
    return call<int (*)(P, P, I, I, int, void *, int, I, int, void *)>(DEQUANTIZE, stream, ptr(q), ptr(s), rows, cols, (int)element, (void *)ptr(dst), v.dtype, v.ld,
                                                                      (int)layout);
}

// a, b, c, max_workgroups, stream
PyObject *gemm_bf16(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args a{args, n};
    const at::Tensor *x = a.tensor(), *y = a.tensor(), *c = a.tensor();
    const int64_t bound = a.number(0, INT32_MAX);
    PyObject *stream = a.next();
    if (!a.ok || a.left || x->dim() != 2 || y->dim() != 2)
        return not_handled();
    const int64_t M = x->size(0), N = y->size(0), K = x->size(1);
    const Values v = values(*c, M, N);
    if (!v.ok || y->size(1) != K || x->scalar_type() != at::kBFloat16 || y->scalar_type() != at::kBFloat16 || !x->is_contiguous() || !y->is_contiguous())
        return not_handled();
    return call<int (*)(P, P, I, I, I, void *, int, I, int32_t, void *)>(GEMM_BF16, stream, ptr(x), ptr(y), M, N, K, (void *)ptr(c), v.dtype, v.ld, (int32_t)bound);
}

// pass, a_q, a_s, b_q, b_s, c, axis, cq_row, cs_row, cq_colT, cs_colT, layout, max_workgroups, stream
PyObject *gemm_quantize(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args a{args, n};
    const int64_t pass = a.code(passes, 0, 2);
    const at::Tensor *a_q = a.tensor(), *a_s = a.tensor(), *b_q = a.tensor(), *b_s = a.tensor(), *c = a.tensor();
    const int64_t axis = a.code(axes, 1, 3);
    Copies q;
    q.q_row = a.tensor(true);
    q.s_row = a.tensor(true);
    q.q_colT = a.tensor(true);
    q.s_colT = a.tensor(true);
    const int64_t layout = a.number(0, 1), bound = a.number(0, INT32_MAX);
    PyObject *stream = a.next();
    if (!a.ok || a.left || a_q->dim() != 2 || b_q->dim() != 2)
        return not_handled();
    const int64_t M = a_q->size(0), N = b_q->size(0), K = a_q->size(1);
    const Values v = values(*c, M, N);
    if (!v.ok || v.dtype != 1 || !dense_matrix(*a_q, M, K) || !dense_matrix(*b_q, N, K) || !scales(*a_s, M, K, layout) || !scales(*b_s, N, K, layout) ||
        !copies(a, q, M, N, axis, layout, 1, 1) || ((axis & kRowwise) && !dense_matrix(*q.q_row, M, N)) || ((axis & kColwise) && !dense_matrix(*q.q_colT, N, M)))
        return not_handled();
    return call<int (*)(int, P, P, P, P, I, I, I, void *, I, int, Q, Q, Q, Q, int, int32_t, void *)>(
        GEMM_QUANTIZE, stream, (int)pass, ptr(a_q), ptr(a_s), ptr(b_q), ptr(b_s), M, N, K, (void *)ptr(c), v.ld, (int)axis, ptr(q.q_row), ptr(q.s_row),
        ptr(q.q_colT), ptr(q.s_colT), (int)layout, (int32_t)bound);
}

// ---- expert rows and products of a few rows (experts.py) ----------------------------------------------------------------
// Whether all of them (nullptr: not given) are on the current device.
bool on_current_device(std::initializer_list<const at::Tensor *> tensors)
{
    const auto current = c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice();
    for (const at::Tensor *t : tensors)
        if (t && t->device() != current)
            return false;
    return true;
}
bool numbers(const at::Tensor &t, int64_t n) { return t.scalar_type() == at::kInt && t.is_contiguous() && t.numel() == n; }
bool weights_ok(const at::Tensor *t, int64_t n) { return !t || (t->scalar_type() == at::kFloat && t->is_contiguous() && t->numel() == n); }
constexpr int64_t kMany = int64_t(1) << 30;

// experts, align, positions, sources, group_ends, workspace, stream
PyObject *expert_sort(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args a{args, n};
    const at::Tensor *experts = a.tensor();
    const int64_t align = a.number(1, INT32_MAX);
    const at::Tensor *positions = a.tensor(), *sources = a.tensor(), *ends = a.tensor(), *workspace = a.tensor(true);
    PyObject *stream = a.next();
    if (!a.ok || a.left || !entry[EXPERT_SORT_WORKSPACE])
        return not_handled();
    const int64_t entries = experts->numel(), groups = ends->numel(), rows = sources->numel();
    const bool wide = experts->scalar_type() == at::kLong;
    if ((!wide && experts->scalar_type() != at::kInt) || !experts->is_contiguous() || entries > kMany || groups > INT32_MAX || !numbers(*positions, entries) ||
        !numbers(*sources, rows) || !numbers(*ends, groups) || !on_current_device({experts, positions, sources, ends, workspace}))
        return not_handled();
    const int64_t need = reinterpret_cast<int64_t (*)(int64_t, int32_t)>(entry[EXPERT_SORT_WORKSPACE])(entries, (int32_t)groups);
    if (need < 0 || (need > 0 && (!workspace || !workspace->is_contiguous() || (int64_t)workspace->nbytes() < need)))
        return not_handled();
    return call<int (*)(P, int, I, int32_t, int32_t, I, Q, Q, Q, Q, void *)>(EXPERT_SORT, stream, ptr(experts), wide ? 1 : 0, entries, (int32_t)groups,
                                                                            (int32_t)align, rows, ptr(positions), ptr(sources), ptr(ends), ptr(workspace));
}

// src, sources, group_ends, slots, weights, axis, q_row, s_row, q_colT, s_colT, layout, stream
PyObject *expert_quantize(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args a{args, n};
    const at::Tensor *src = a.tensor(), *sources = a.tensor(), *ends = a.tensor(true);
    const int64_t slots = a.number(1, 4096);
    const at::Tensor *weights = a.tensor(true);
    const int64_t axis = a.code(axes, 1, 3);
    Copies c;
    c.q_row = a.tensor(true);
    c.s_row = a.tensor(true);
    c.q_colT = a.tensor(true);
    c.s_colT = a.tensor(true);
    const int64_t layout = a.number(0, 1);
    PyObject *stream = a.next();
    if (!a.ok || a.left || src->dim() != 2)
        return not_handled();
    const int64_t tokens = src->size(0), cols = src->size(1), rows = sources->numel(), groups = ends ? ends->numel() : 0;
    const Values v = values(*src, tokens, cols);
    if (!v.ok || tokens > kMany || rows > kMany || rows % 32 || cols % 32 || !numbers(*sources, rows) || (ends && (groups == 0 || groups > 4096 || !numbers(*ends, groups))) ||
        !weights_ok(weights, tokens * slots) || !copies(a, c, rows, cols, axis, layout, 1, 1) || ((axis & kRowwise) && !dense_matrix(*c.q_row, rows, cols)) ||
        ((axis & kColwise) && !dense_matrix(*c.q_colT, cols, rows)) || !on_current_device({src, sources, ends, weights, c.q_row, c.s_row, c.q_colT, c.s_colT}))
        return not_handled();
    return call<int (*)(P, int, I, I, I, P, int32_t, P, P, int32_t, I, int, Q, Q, Q, Q, int, void *)>(
        EXPERT_QUANTIZE, stream, ptr(src), v.dtype, tokens, cols, v.ld, ptr(sources), (int32_t)slots, ptr(weights), ptr(ends), (int32_t)groups, rows, (int)axis,
        ptr(c.q_row), ptr(c.s_row), ptr(c.q_colT), ptr(c.s_colT), (int)layout);
}

// c, positions, weights, out, stream
PyObject *expert_combine(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args a{args, n};
    const at::Tensor *c = a.tensor(), *positions = a.tensor(), *weights = a.tensor(true), *out = a.tensor();
    PyObject *stream = a.next();
    if (!a.ok || a.left || c->dim() != 2 || positions->dim() != 2)
        return not_handled();
    const int64_t rows = c->size(0), cols = c->size(1), tokens = positions->size(0), slots = positions->size(1);
    const Values v = values(*c, rows, cols), o = values(*out, tokens, cols);
    if (!v.ok || !o.ok || tokens > kMany || slots > 4096 || !numbers(*positions, tokens * slots) || !weights_ok(weights, tokens * slots) ||
        !on_current_device({c, positions, weights, out}))
        return not_handled();
    return call<int (*)(P, int, I, I, I, P, P, I, int32_t, Q, int, I, void *)>(EXPERT_COMBINE, stream, ptr(c), v.dtype, rows, cols, v.ld, ptr(positions), ptr(weights),
                                                                              tokens, (int32_t)slots, ptr(out), o.dtype, o.ld);
}

// dy, c, positions, dweights, stream
PyObject *expert_weight_grad(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args a{args, n};
    const at::Tensor *dy = a.tensor(), *c = a.tensor(), *positions = a.tensor(), *dw = a.tensor();
    PyObject *stream = a.next();
    if (!a.ok || a.left || c->dim() != 2 || positions->dim() != 2)
        return not_handled();
    const int64_t rows = c->size(0), cols = c->size(1), tokens = positions->size(0), slots = positions->size(1);
    const Values v = values(*c, rows, cols), d = values(*dy, tokens, cols);
    if (!v.ok || !d.ok || tokens > kMany || slots > 4096 || !numbers(*positions, tokens * slots) || !weights_ok(dw, tokens * slots) ||
        !on_current_device({dy, c, positions, dw}))
        return not_handled();
    return call<int (*)(P, int, I, P, int, I, I, I, P, I, int32_t, Q, void *)>(EXPERT_WEIGHT_GRAD, stream, ptr(dy), d.dtype, d.ld, ptr(c), v.dtype, rows, cols, v.ld,
                                                                              ptr(positions), tokens, (int32_t)slots, ptr(dw));
}

// x, w_q, w_s, c, layout, stream
PyObject *fp4_gemv(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args a{args, n};
    const at::Tensor *x = a.tensor(), *w_q = a.tensor(), *w_s = a.tensor(), *c = a.tensor();
    const int64_t layout = a.number(0, 1);
    PyObject *stream = a.next();
    if (!a.ok || a.left || x->dim() != 2 || w_q->dim() != 2)
        return not_handled();
    const int64_t M = x->size(0), K = x->size(1), N = w_q->size(0);
    const Values v = values(*x, M, K), o = values(*c, M, N);
    if (!v.ok || v.dtype != 1 || !o.ok || K % 32 || !dense_matrix(*w_q, N, K / 2) || !scales(*w_s, N, K, layout) || !on_current_device({x, w_q, w_s, c}))
        return not_handled();
    return call<int (*)(P, I, P, P, I, I, I, Q, int, I, int, void *)>(FP4_GEMV, stream, ptr(x), v.ld, ptr(w_q), ptr(w_s), M, N, K, ptr(c), o.dtype, o.ld, (int)layout);
}

// x, sources, slots, w_q, w_s, group_ends, c, layout, stream
PyObject *fp4_gemv_grouped(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args a{args, n};
    const at::Tensor *x = a.tensor(), *sources = a.tensor(true);
    const int64_t slots = a.number(1, 4096);
    const at::Tensor *w_q = a.tensor(), *w_s = a.tensor(), *ends = a.tensor(), *c = a.tensor();
    const int64_t layout = a.number(0, 1);
    PyObject *stream = a.next();
    if (!a.ok || a.left || x->dim() != 2 || w_q->dim() != 3 || c->dim() != 2)
        return not_handled();
    const int64_t tokens = x->size(0), K = x->size(1), groups = w_q->size(0), N = w_q->size(1), M = c->size(0);
    const Values v = values(*x, tokens, K), o = values(*c, M, N);
    if (!v.ok || v.dtype != 1 || !o.ok || K % 32 || N > kMany || groups < 1 || groups > 4096 || w_q->size(2) != K / 2 || !dense_bytes(*w_q) || !dense_bytes(*w_s) ||
        w_s->numel() != groups * (layout == kTiled ? (N + 63) / 64 * ((K / 32 + 3) / 4) * 256 : N * (K / 32)) || !numbers(*ends, groups) ||
        (sources ? !numbers(*sources, M) : tokens < M) || !on_current_device({x, sources, w_q, w_s, ends, c}))
        return not_handled();
    return call<int (*)(P, I, I, P, int32_t, P, P, P, int32_t, I, I, I, Q, int, I, int, void *)>(FP4_GEMV_GROUPED, stream, ptr(x), tokens, v.ld, ptr(sources),
                                                                                                 (int32_t)slots, ptr(w_q), ptr(w_s), ptr(ends), (int32_t)groups, M, N,
                                                                                                 K, ptr(c), o.dtype, o.ld, (int)layout);
}

// ---- operands with a scale for each block of 128 (b128.py), the layer of experts for a few tokens (layer.py) ------------------
int64_t blocks128(int64_t n) { return (n + 127) / 128; }
// leading dimension of an operand [rows x cols], 0 if it is none; its rows are followed by their padding to a multiple of 16 bytes
int64_t operand(const at::Tensor &t, int64_t rows, int64_t cols)
{
    if (t.scalar_type() != at::kByte || t.dim() != 2 || t.size(0) != rows || t.size(1) != cols || rows <= 0 || cols <= 0 || t.stride(1) != 1)
        return 0;
    const int64_t wide = (cols + 15) / 16 * 16, ld = rows > 1 ? t.stride(0) : wide;
    return ld > 0 && t.storage_offset() + (rows - 1) * ld + wide <= (int64_t)t.storage().nbytes() ? ld : 0;
}
bool scales128(const at::Tensor &s, int64_t rows, int64_t cols, bool tiles)
{
    return s.scalar_type() == at::kFloat && s.is_contiguous() && s.dim() == 2 && s.size(0) == blocks128(tiles ? rows : cols) &&
           s.size(1) == (tiles ? blocks128(cols) : rows);
}
bool holds(const at::Tensor *workspace, int64_t need)
{
    return need == 0 || (need > 0 && workspace && workspace->is_contiguous() && (int64_t)workspace->nbytes() >= need);
}

// src, axis, shape, q_row, s_row, q_colT, s_colT, stream
PyObject *b128_quantize(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args a{args, n};
    const at::Tensor *src = a.tensor();
    const int64_t axis = a.code(axes, 1, 3), shape = a.number(0, 1);
    Copies c;
    c.q_row = a.tensor(true);
    c.s_row = a.tensor(true);
    c.q_colT = a.tensor(true);
    c.s_colT = a.tensor(true);
    PyObject *stream = a.next();
    if (!a.ok || a.left || src->dim() != 2)
        return not_handled();
    const int64_t rows = src->size(0), cols = src->size(1);
    const Values v = values(*src, rows, cols);
    if (!v.ok || !on_current_device({src, c.q_row, c.s_row, c.q_colT, c.s_colT}))
        return not_handled();
    int64_t ld_row = 0, ld_col = 0;
    if (axis & kRowwise)
        ld_row = c.q_row && c.s_row && scales128(*c.s_row, rows, cols, shape) ? operand(*c.q_row, rows, cols) : 0;
    if (axis & kColwise)
        ld_col = c.q_colT && c.s_colT && scales128(*c.s_colT, cols, rows, shape) ? operand(*c.q_colT, cols, rows) : 0;
    if (((axis & kRowwise) && !ld_row) || ((axis & kColwise) && !ld_col))
        return not_handled();
    return call<int (*)(P, int, I, I, I, int, int, Q, I, Q, Q, I, Q, void *)>(B128_QUANTIZE, stream, ptr(src), v.dtype, rows, cols, v.ld, (int)axis, (int)shape,
                                                                             ptr(c.q_row), ld_row, ptr(c.s_row), ptr(c.q_colT), ld_col, ptr(c.s_colT));
}

// pass, a_q, a_s, b_q, b_s, c, workspace, stream
PyObject *b128_gemm(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args a{args, n};
    const int64_t pass = a.code(passes, 0, 2);
    const at::Tensor *a_q = a.tensor(), *a_s = a.tensor(), *b_q = a.tensor(), *b_s = a.tensor(), *c = a.tensor(), *workspace = a.tensor(true);
    PyObject *stream = a.next();
    if (!a.ok || a.left || a_q->dim() != 2 || b_q->dim() != 2 || !entry[B128_GEMM_WORKSPACE])
        return not_handled();
    const int64_t M = a_q->size(0), N = b_q->size(0), K = a_q->size(1), lda = operand(*a_q, M, K), ldb = operand(*b_q, N, K);
    const Values v = values(*c, M, N);
    if (!v.ok || !lda || !ldb || !scales128(*a_s, M, K, false) || !scales128(*b_s, N, K, pass != 2) || !on_current_device({a_q, a_s, b_q, b_s, c, workspace}) ||
        !holds(workspace, reinterpret_cast<int64_t (*)(int, I, I, I)>(entry[B128_GEMM_WORKSPACE])((int)pass, M, N, K)))
        return not_handled();
    return call<int (*)(int, P, I, P, P, I, P, I, I, I, Q, int, I, Q, void *)>(B128_GEMM, stream, (int)pass, ptr(a_q), lda, ptr(a_s), ptr(b_q), ldb, ptr(b_s), M, N, K,
                                                                              ptr(c), v.dtype, v.ld, ptr(workspace));
}

// x, w_q, w_s, c, stream
PyObject *b128_gemv(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args a{args, n};
    const at::Tensor *x = a.tensor(), *w_q = a.tensor(), *w_s = a.tensor(), *c = a.tensor();
    PyObject *stream = a.next();
    if (!a.ok || a.left || x->dim() != 2 || w_q->dim() != 2)
        return not_handled();
    const int64_t M = x->size(0), K = x->size(1), N = w_q->size(0), ldw = operand(*w_q, N, K);
    const Values v = values(*x, M, K), o = values(*c, M, N);
    if (!v.ok || v.dtype != 1 || !o.ok || !ldw || !scales128(*w_s, N, K, true) || !on_current_device({x, w_q, w_s, c}))
        return not_handled();
    return call<int (*)(P, I, P, I, P, I, I, I, Q, int, I, void *)>(B128_GEMV, stream, ptr(x), v.ld, ptr(w_q), ldw, ptr(w_s), M, N, K, ptr(c), o.dtype, o.ld);
}

// one matrix [rows x cols] for each expert, format as mxfp8_weights
bool expert_matrices(const at::Tensor &q, const at::Tensor &s, int64_t format, int64_t groups, int64_t rows, int64_t cols, int64_t layout)
{
    if (!dense_bytes(q) || q.dim() != 3 || q.size(0) != groups || q.size(1) != rows || q.size(2) != (format == 0 ? cols / 2 : cols) || !s.is_contiguous())
        return false;
    if (format == 2)
        return s.scalar_type() == at::kFloat && s.dim() == 3 && s.size(0) == groups && s.size(1) == blocks128(rows) && s.size(2) == blocks128(cols);
    return cols % 32 == 0 && s.scalar_type() == at::kByte &&
           s.numel() == groups * (layout == kTiled ? (rows + 63) / 64 * ((cols / 32 + 3) / 4) * 256 : rows * (cols / 32));
}

// x, experts, weights, format, up_q, up_s, down_q, down_s, out, workspace, layout, stream
PyObject *expert_layer(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args a{args, n};
    const at::Tensor *x = a.tensor(), *experts = a.tensor(), *weights = a.tensor();
    const int64_t format = a.number(0, 2);
    const at::Tensor *up_q = a.tensor(), *up_s = a.tensor(), *down_q = a.tensor(), *down_s = a.tensor(), *out = a.tensor(), *workspace = a.tensor();
    const int64_t layout = a.number(0, 1);
    PyObject *stream = a.next();
    if (!a.ok || a.left || x->dim() != 2 || experts->dim() != 2 || down_q->dim() != 3 || !entry[EXPERT_LAYER_WORKSPACE])
        return not_handled();
    const int64_t tokens = x->size(0), hidden = x->size(1), slots = experts->size(1), groups = down_q->size(0), inter = down_q->size(2) * (format == 0 ? 2 : 1);
    const Values v = values(*x, tokens, hidden), o = values(*out, tokens, hidden);
    const bool wide = experts->scalar_type() == at::kLong;
    if (!v.ok || v.dtype != 1 || !o.ok || tokens > kMany || slots < 1 || slots > 4096 || groups < 1 || groups > 4096 || inter > kMany || hidden > kMany ||
        (!wide && experts->scalar_type() != at::kInt) || !experts->is_contiguous() || experts->size(0) != tokens ||
        weights->sizes() != experts->sizes() || !weights_ok(weights, tokens * slots) ||
        !expert_matrices(*up_q, *up_s, format, groups, 2 * inter, hidden, layout) || !expert_matrices(*down_q, *down_s, format, groups, hidden, inter, layout) ||
        !holds(workspace, reinterpret_cast<int64_t (*)(I, int32_t, I)>(entry[EXPERT_LAYER_WORKSPACE])(tokens, (int32_t)slots, inter)) ||
        !on_current_device({x, experts, weights, up_q, up_s, down_q, down_s, out, workspace}))
        return not_handled();
    return call<int (*)(P, I, I, I, P, int, int32_t, P, int, P, P, P, P, int32_t, I, Q, int, I, Q, int, void *)>(
        EXPERT_LAYER, stream, ptr(x), tokens, hidden, v.ld, ptr(experts), wide ? 1 : 0, (int32_t)slots, ptr(weights), (int)format, ptr(up_q), ptr(up_s), ptr(down_q),
        ptr(down_s), (int32_t)groups, inter, ptr(out), o.dtype, o.ld, ptr(workspace), (int)layout);
}

// {name: address} of the entry points, and the binding's "passes", "axes" and "stream"
PyObject *bind(PyObject *, PyObject *table)
{
    if (!PyDict_Check(table)) {
        PyErr_SetString(PyExc_TypeError, "bind() takes a dict of addresses");
        return nullptr;
    }
    const struct {
        const char *name;
        PyObject **to;
        bool dict;
    } own[] = {{"passes", &passes, true}, {"axes", &axes, true}, {"stream", &stream_handle, false}};
    for (const auto &o : own) {
        PyObject *v = PyDict_GetItemString(table, o.name);
        if (v && (o.dict ? !PyDict_Check(v) : !PyCallable_Check(v))) {
            PyErr_Format(PyExc_TypeError, "bind(): bad \"%s\"", o.name);
            return nullptr;
        }
        Py_XINCREF(v);
        Py_XSETREF(*o.to, v);
    }
    for (int i = 0; i < ENTRY_POINTS; ++i) {
        PyObject *v = PyDict_GetItemString(table, kNames[i]);
        entry[i] = v ? PyLong_AsVoidPtr(v) : nullptr;
        if (PyErr_Occurred())
            return nullptr;
    }
    Py_RETURN_NONE;
}

// Tensors without memory of their own (traced, batched) throw when they are asked for it: the binding's checks say so.
template <PyObject *(*FN)(PyObject *, PyObject *const *, Py_ssize_t)> PyObject *guarded(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    try {
        return FN(self, args, n);
    } catch (...) {
        return not_handled();
    }
}

#define FAST(name, ...) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<__VA_ARGS__>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST("quantize", quantize<QUANTIZE>), FAST("fp4_quantize", quantize<FP4_QUANTIZE>), FAST("fp6_quantize", quantize<FP6_QUANTIZE>),
                         FAST("gemm", gemm<GEMM>), FAST("gemm_mode", gemm<GEMM_MODE>), FAST("fp4_gemm", gemm<FP4_GEMM>), FAST("dequantize", dequantize),
                         FAST("gemm_bf16", gemm_bf16), FAST("gemm_quantize", gemm_quantize), FAST("expert_sort", expert_sort),
                         FAST("expert_quantize", expert_quantize), FAST("expert_combine", expert_combine), FAST("expert_weight_grad", expert_weight_grad),
                         FAST("fp4_gemv", fp4_gemv), FAST("fp4_gemv_grouped", fp4_gemv_grouped),
                         FAST("b128_quantize", b128_quantize), FAST("b128_gemm", b128_gemm), FAST("b128_gemv", b128_gemv), FAST("expert_layer", expert_layer), {"bind", bind, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall(void) { return PyModule_Create(&module); }
