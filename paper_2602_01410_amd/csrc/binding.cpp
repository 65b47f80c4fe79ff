// Native half of snip.py: takes torch tensors and QTensor objects apart and calls the C ABI of include/snip.h.  Argument
// marshalling only, like the Python half; the library is called through its exported symbols, looked up once by bind().
//
// A call of the C ABI takes about 3 us of host time, most of it the launch.  Marshalled in Python (attribute reads, one
// ctypes structure per operand, torch.cuda.current_stream()) a call took 8.8-9.5 us, more than the kernels of a small
// training step; the functions below take about 1 us around the launch.
#include <torch/csrc/autograd/python_variable.h>
#include <c10/hip/HIPStream.h>
#include <dlfcn.h>
#include <cstring>
#include <vector>
#include "../../include/snip.h"

namespace {

decltype(&snip_quantize) p_quantize;
decltype(&snip_quantize_both) p_quantize_both;
decltype(&snip_quantize_sr_fp4) p_quantize_sr_fp4;
decltype(&snip_gemm_fwd) p_gemm[3];
decltype(&snip_gemm_fwd_norm) p_gemm_norm[3];
decltype(&snip_quantize_paper) p_quantize_paper;
decltype(&snip_gemm_paper) p_gemm_paper;
decltype(&snip_quant_error_stats) p_stats;
decltype(&snip_quant_error_stats_both) p_stats_both;
decltype(&snip_adamw_sensitivity) p_adamw;
decltype(&snip_rms_norm) p_rms_norm;
decltype(&snip_rms_norm_backward) p_rms_norm_backward;
decltype(&snip_adamw_step) p_adamw_step;
decltype(&snip_gemv) p_gemv;

PyObject *s_codes, *s_scales, *s_scales_g4, *s_rows, *s_cols, *s_fmt;      // interned attribute names
PyObject *s_param, *s_grad, *s_m, *s_v, *s_copy, *s_m_scale, *s_v_scale, *s_weight_decay;

// Every helper returns false (or -1) with a Python exception set when an argument is not what it should be.
bool tensor(PyObject* o, const at::Tensor*& t)
{
    if (!THPVariable_Check(o)) { PyErr_SetString(PyExc_TypeError, "expected a torch.Tensor"); return false; }
    t = &THPVariable_Unpack(o);
    return true;
}
bool pointer(PyObject* o, void*& p)                 // None: null
{
    p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor* t;
    if (!tensor(o, t)) return false;
    p = t->data_ptr();
    return true;
}
bool integer(PyObject* o, int64_t& v) { v = PyLong_AsLongLong(o); return !(v == -1 && PyErr_Occurred()); }

struct Source { void* p; int64_t rows, cols, ld; };
bool source(PyObject* o, Source& s)
{
    const at::Tensor* t;
    if (!tensor(o, t)) return false;
    const at::ScalarType type = t->scalar_type();
    if (t->dim() != 2 || (type != at::kBFloat16 && type != at::kShort && type != at::kUInt16) || !t->is_cuda()) {
        PyErr_SetString(PyExc_ValueError, "expected a 2-D CUDA tensor of bf16 (or its uint16/int16 bit patterns)");
        return false;
    }
    if (t->stride(1) != 1) { PyErr_SetString(PyExc_ValueError, "rows must be contiguous"); return false; }
    s = {t->data_ptr(), t->size(0), t->size(1), t->stride(0)};
    return true;
}
bool attr_int(PyObject* o, PyObject* name, int64_t& v)
{
    PyObject* a = PyObject_GetAttr(o, name);
    if (!a) return false;
    const bool ok = integer(a, v);
    Py_DECREF(a);
    return ok;
}
bool attr_ptr(PyObject* o, PyObject* name, void*& p)
{
    PyObject* a = PyObject_GetAttr(o, name);
    if (!a) return false;
    const bool ok = pointer(a, p);                  // (the object keeps the tensor alive)
    Py_DECREF(a);
    return ok;
}
bool qtensor(PyObject* o, snip_qtensor& q)
{
    void *c, *s, *g;
    int64_t fmt;
    if (!attr_ptr(o, s_codes, c) || !attr_ptr(o, s_scales, s) || !attr_ptr(o, s_scales_g4, g) || !attr_int(o, s_rows, q.rows) ||
        !attr_int(o, s_cols, q.cols) || !attr_int(o, s_fmt, fmt))
        return false;
    q.codes = c; q.scales = (uint8_t*)s; q.scales_g4 = (uint8_t*)g; q.fmt = (int32_t)fmt;
    return true;
}
bool workspace(PyObject* o, void*& p, size_t& n)    // a uint8 tensor or None
{
    p = nullptr; n = 0;
    if (o == Py_None) return true;
    const at::Tensor* t;
    if (!tensor(o, t)) return false;
    p = t->data_ptr(); n = (size_t)t->numel();
    return true;
}
bool stream(PyObject* o, void*& s)                  // None: the current stream of the current device
{
    if (o == Py_None) { s = (void*)c10::hip::getCurrentHIPStream().stream(); return true; }
    s = PyLong_AsVoidPtr(o);
    return !(s == nullptr && PyErr_Occurred());
}
bool plan(PyObject* o, snip_layer_plan& p)          // the ctypes structure of snip.make_plan
{
    Py_buffer b;
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) return false;
    const bool ok = b.len == (Py_ssize_t)sizeof(p);
    if (ok) std::memcpy(&p, b.buf, sizeof(p));
    PyBuffer_Release(&b);
    if (!ok) PyErr_SetString(PyExc_TypeError, "expected a plan");
    return ok;
}
bool count(Py_ssize_t n, Py_ssize_t want)
{
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
    return false;
}

template <class F> PyObject* call(F f)
{
    snip_status st;
    Py_BEGIN_ALLOW_THREADS
    st = f();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)st);
}

// (x, fmt, axis, rule, out, stats, workspace, stream)
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Source x; int64_t fmt, axis, rule; snip_qtensor q; void *st, *ws, *s; size_t wn;
    if (!count(n, 8) || !source(a[0], x) || !integer(a[1], fmt) || !integer(a[2], axis) || !integer(a[3], rule) || !qtensor(a[4], q) ||
        !pointer(a[5], st) || !workspace(a[6], ws, wn) || !stream(a[7], s))
        return nullptr;
    return call([&] { return p_quantize(x.p, x.rows, x.cols, x.ld, (snip_fmt)fmt, (snip_axis)axis, (snip_scale_rule)rule, &q, (snip_stats*)st, ws, wn, s); });
}
// (x, rule, out_row, out_col, stats_row, stats_col, scope, workspace, stream)
PyObject* quantize_both(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Source x; int64_t rule, scope; snip_qtensor qr, qc; void *sr, *sc, *ws, *s; size_t wn;
    if (!count(n, 9) || !source(a[0], x) || !integer(a[1], rule) || !qtensor(a[2], qr) || !qtensor(a[3], qc) || !pointer(a[4], sr) ||
        !pointer(a[5], sc) || !integer(a[6], scope) || !workspace(a[7], ws, wn) || !stream(a[8], s))
        return nullptr;
    return call([&] { return p_quantize_both(x.p, x.rows, x.cols, x.ld, (snip_scale_rule)rule, &qr, &qc, (snip_stats*)sr, (snip_stats*)sc,
                                             (snip_stats_scope)scope, ws, wn, s); });
}
// (x, axis, rule, seed, out, stream)
PyObject* quantize_sr_fp4(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Source x; int64_t axis, rule; snip_qtensor q; void* s;
    if (!count(n, 6) || !source(a[0], x) || !integer(a[1], axis) || !integer(a[2], rule)) return nullptr;
    const unsigned long long seed = PyLong_AsUnsignedLongLong(a[3]);
    if (seed == (unsigned long long)-1 && PyErr_Occurred()) return nullptr;
    if (!qtensor(a[4], q) || !stream(a[5], s)) return nullptr;
    return call([&] { return p_quantize_sr_fp4(x.p, x.rows, x.cols, x.ld, (snip_axis)axis, (snip_scale_rule)rule, seed, &q, s); });
}
struct Output { void* p; int64_t ld; };
bool output(PyObject* o, Output& out)
{
    const at::Tensor* t;
    if (!tensor(o, t)) return false;
    if (t->dim() < 1) { PyErr_SetString(PyExc_ValueError, "expected a matrix as output"); return false; }
    out = {t->data_ptr(), t->stride(0)};
    return true;
}
bool which_gemm(PyObject* o, int64_t& w)
{
    if (!integer(o, w)) return false;
    if (w < 0 || w > 2) { PyErr_SetString(PyExc_ValueError, "no such GEMM"); return false; }
    return true;
}
// (which, plan, a, b, out, out_dtype, stream)
PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    int64_t w, dt; snip_layer_plan p; snip_qtensor qa, qb; Output o; void* s;
    if (!count(n, 7) || !which_gemm(a[0], w) || !plan(a[1], p) || !qtensor(a[2], qa) || !qtensor(a[3], qb) || !output(a[4], o) ||
        !integer(a[5], dt) || !stream(a[6], s))
        return nullptr;
    return call([&] { return p_gemm[w](&p, &qa, &qb, o.p, o.ld, (snip_out_dtype)dt, nullptr, 0, s); });
}
// (which, plan, a, b, out, out_dtype, sum_sq, workspace, stream)
PyObject* gemm_norm(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    int64_t w, dt; snip_layer_plan p; snip_qtensor qa, qb; Output o; void *ss, *ws, *s; size_t wn;
    if (!count(n, 9) || !which_gemm(a[0], w) || !plan(a[1], p) || !qtensor(a[2], qa) || !qtensor(a[3], qb) || !output(a[4], o) ||
        !integer(a[5], dt) || !pointer(a[6], ss) || !workspace(a[7], ws, wn) || !stream(a[8], s))
        return nullptr;
    return call([&] { return p_gemm_norm[w](&p, &qa, &qb, o.p, o.ld, (snip_out_dtype)dt, (double*)ss, ws, wn, s); });
}
// (x, fmt, axis, group, codes, scales, stream)
PyObject* quantize_paper(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Source x; int64_t fmt, axis, group; void *c, *sc, *s;
    if (!count(n, 7) || !source(a[0], x) || !integer(a[1], fmt) || !integer(a[2], axis) || !integer(a[3], group) || !pointer(a[4], c) ||
        !pointer(a[5], sc) || !stream(a[6], s))
        return nullptr;
    return call([&] { return p_quantize_paper(x.p, x.rows, x.cols, x.ld, (snip_fmt)fmt, (snip_axis)axis, (snip_group)group, c, (float*)sc, s); });
}
bool ptensor(PyObject* const* a, snip_ptensor& q)   // codes, scales, fmt, group
{
    const at::Tensor* c;
    int64_t fmt, group;
    void* sc;
    if (!tensor(a[0], c) || !pointer(a[1], sc) || !integer(a[2], fmt) || !integer(a[3], group)) return false;
    if (c->dim() != 2) { PyErr_SetString(PyExc_ValueError, "expected 2-D codes"); return false; }
    q.codes = c->data_ptr(); q.scales = (const float*)sc; q.rows = c->size(0);
    q.cols = fmt == SNIP_FP8_E4M3 ? c->size(1) : 2 * c->size(1); q.fmt = (int32_t)fmt; q.group = (int32_t)group;
    return true;
}
// (a_codes, a_scales, a_fmt, a_group, b_codes, b_scales, b_fmt, b_group, out, out_dtype, stream)
PyObject* gemm_paper(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    snip_ptensor pa, pb; Output o; int64_t dt; void* s;
    if (!count(n, 11) || !ptensor(a, pa) || !ptensor(a + 4, pb) || !output(a[8], o) || !integer(a[9], dt) || !stream(a[10], s)) return nullptr;
    return call([&] { return p_gemm_paper(&pa, &pb, o.p, o.ld, (snip_out_dtype)dt, s); });
}
// (x, axis, rule, out, per_line, workspace, stream)
PyObject* stats(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Source x; int64_t axis, rule; void *o, *pl, *ws, *s; size_t wn;
    if (!count(n, 7) || !source(a[0], x) || !integer(a[1], axis) || !integer(a[2], rule) || !pointer(a[3], o) || !pointer(a[4], pl) ||
        !workspace(a[5], ws, wn) || !stream(a[6], s))
        return nullptr;
    return call([&] { return p_stats(x.p, x.rows, x.cols, x.ld, (snip_axis)axis, (snip_scale_rule)rule, (snip_stats*)o, (float*)pl, ws, wn, s); });
}
// (x, rule, out_row, out_col, workspace, stream)
PyObject* stats_both(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Source x; int64_t rule; void *r, *c, *ws, *s; size_t wn;
    if (!count(n, 6) || !source(a[0], x) || !integer(a[1], rule) || !pointer(a[2], r) || !pointer(a[3], c) || !workspace(a[4], ws, wn) || !stream(a[5], s))
        return nullptr;
    return call([&] { return p_stats_both(x.p, x.rows, x.cols, x.ld, (snip_scale_rule)rule, (snip_stats*)r, (snip_stats*)c, ws, wn, s); });
}
// (m, v, g, g_dtype, n, beta1, beta2, eps, out, workspace, stream)
PyObject* adamw(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    void *m, *v, *g, *o, *ws, *s; int64_t dt, cnt; size_t wn;
    if (!count(n, 11) || !pointer(a[0], m) || !pointer(a[1], v) || !pointer(a[2], g) || !integer(a[3], dt) || !integer(a[4], cnt)) return nullptr;
    const double b1 = PyFloat_AsDouble(a[5]), b2 = PyFloat_AsDouble(a[6]), eps = PyFloat_AsDouble(a[7]);
    if (PyErr_Occurred() || !pointer(a[8], o) || !workspace(a[9], ws, wn) || !stream(a[10], s)) return nullptr;
    return call([&] { return p_adamw((const float*)m, (const float*)v, g, (snip_out_dtype)dt, cnt, (float)b1, (float)b2, (float)eps, (double*)o, ws, wn, s); });
}

// A bf16 matrix of the extents of `like`, or None: null.
bool same_extents(PyObject* o, const Source& like, Source& s)
{
    s = {nullptr, 0, 0, 0};
    if (o == Py_None) return true;
    if (!source(o, s)) return false;
    if (s.rows != like.rows || s.cols != like.cols) { PyErr_SetString(PyExc_ValueError, "expected a matrix with the extents of the input"); return false; }
    return true;
}
// A contiguous vector of n elements on the GPU; `dtype`: which of the two it is (fp32 if only_fp32).  None: null.
bool vector(PyObject* o, int64_t n, bool only_fp32, void*& p, snip_out_dtype& dtype)
{
    p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor* t;
    if (!tensor(o, t)) return false;
    const bool fp32 = t->scalar_type() == at::kFloat;
    if (!t->is_cuda() || !t->is_contiguous() || t->numel() != n || !(fp32 || (!only_fp32 && t->scalar_type() == at::kBFloat16))) {
        PyErr_SetString(PyExc_ValueError, only_fp32 ? "expected a contiguous CUDA tensor of fp32, with as many elements as the call has rows, columns or scalars"
                                                    : "expected a contiguous CUDA tensor of bf16 or fp32, one element for each column");
        return false;
    }
    p = t->data_ptr();
    dtype = fp32 ? SNIP_OUT_FP32 : SNIP_OUT_BF16;
    return true;
}
// (x, weight, eps, residual, rule, sum, rstd, y, out_row, out_col, stream)
PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Source x, r, h, y; int64_t rule; void *w, *rstd, *s; snip_out_dtype dt = SNIP_OUT_BF16, d32; snip_qtensor qr, qc;
    if (!count(n, 11) || !source(a[0], x) || !vector(a[1], x.cols, false, w, dt)) return nullptr;
    const double eps = PyFloat_AsDouble(a[2]);
    if (PyErr_Occurred() || !same_extents(a[3], x, r) || !integer(a[4], rule) || !same_extents(a[5], x, h) || !vector(a[6], x.rows, true, rstd, d32) ||
        !same_extents(a[7], x, y) || (a[8] != Py_None && !qtensor(a[8], qr)) || (a[9] != Py_None && !qtensor(a[9], qc)) || !stream(a[10], s))
        return nullptr;
    return call([&] { return p_rms_norm(x.p, x.rows, x.cols, x.ld, r.p, r.ld, w, dt, (float)eps, (snip_scale_rule)rule, h.p, h.ld, (float*)rstd, y.p, y.ld,
                                        a[8] != Py_None ? &qr : nullptr, a[9] != Py_None ? &qc : nullptr, s); });
}
// (dy, h, weight, rstd, dsum, dx, dweight, workspace, stream)
PyObject* rms_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Source dy, h, ds, dx; void *w, *rstd, *dw, *ws, *s; size_t wn; snip_out_dtype dt = SNIP_OUT_BF16, d32;
    if (!count(n, 9) || !source(a[0], dy) || !same_extents(a[1], dy, h) || !vector(a[2], dy.cols, false, w, dt) || !vector(a[3], dy.rows, true, rstd, d32) ||
        !same_extents(a[4], dy, ds) || !same_extents(a[5], dy, dx) || !vector(a[6], dy.cols, true, dw, d32) || !workspace(a[7], ws, wn) || !stream(a[8], s))
        return nullptr;
    return call([&] { return p_rms_norm_backward(dy.p, dy.rows, dy.cols, dy.ld, h.p, h.ld, w, dt, (const float*)rstd, ds.p, ds.ld, dx.p, dx.ld, (float*)dw, ws, wn, s); });
}

// An attribute of `o`: a contiguous tensor on the GPU of n elements (n < 0: of any number, which n becomes) of one of two types, or None
// where that may be: null.
bool array(PyObject* o, PyObject* name, at::ScalarType type, at::ScalarType or_type, bool optional, int64_t& n, void*& p, at::ScalarType* found = nullptr)
{
    p = nullptr;
    PyObject* v = PyObject_GetAttr(o, name);
    if (!v) return false;
    bool ok = optional && v == Py_None;
    const at::Tensor* t;
    if (!ok && tensor(v, t)) {
        if (n < 0) n = t->numel();
        ok = t->is_cuda() && t->is_contiguous() && t->numel() == n && (t->scalar_type() == type || t->scalar_type() == or_type);
        if (ok) { p = t->data_ptr(); if (found) *found = t->scalar_type(); }
        else PyErr_Format(PyExc_ValueError, "%U: expected a contiguous CUDA tensor of %s%s%s, %lld elements", name, c10::toString(type), type == or_type ? "" : " or ",
                          type == or_type ? "" : c10::toString(or_type), (long long)n);
    }
    Py_DECREF(v);
    return ok;
}
bool adamw_tensor(PyObject* o, snip_adamw_tensor& t)
{
    void *p, *g, *m, *v, *c, *ms, *vs;
    at::ScalarType gt, mt;
    t.n = -1;
    if (!array(o, s_param, at::kFloat, at::kFloat, false, t.n, p) || !array(o, s_grad, at::kFloat, at::kBFloat16, false, t.n, g, &gt) ||
        !array(o, s_m, at::kFloat, at::kByte, false, t.n, m, &mt) || !array(o, s_v, mt, mt, false, t.n, v) ||
        !array(o, s_copy, at::kBFloat16, at::kBFloat16, true, t.n, c))
        return false;
    const bool small = mt == at::kByte;
    int64_t groups = small ? (t.n + 127) / 128 : -1;
    if (!array(o, s_m_scale, at::kFloat, at::kFloat, !small, groups, ms) || !array(o, s_v_scale, at::kFloat, at::kFloat, !small, groups, vs)) return false;
    if (!small && (ms || vs)) { PyErr_SetString(PyExc_ValueError, "scales belong to moments of 8 bits"); return false; }
    PyObject* d = PyObject_GetAttr(o, s_weight_decay);
    if (!d) return false;
    t.weight_decay = (float)PyFloat_AsDouble(d);
    Py_DECREF(d);
    t.param = (float*)p; t.grad = g; t.m = m; t.v = v; t.copy = c; t.m_scale = (float*)ms; t.v_scale = (float*)vs;
    t.grad_dtype = gt == at::kFloat ? SNIP_OUT_FP32 : SNIP_OUT_BF16;
    return !PyErr_Occurred();
}
// The objects of a sequence until the end of the call: an iterable's are held by nobody else, and their memory is the caller's only as long as they are.
struct Items {
    PyObject* seq;
    Items(PyObject* o, const char* message) : seq(PySequence_Fast(o, message)) {}
    ~Items() { Py_XDECREF(seq); }
    Items(const Items&) = delete;
    Items& operator=(const Items&) = delete;
    Py_ssize_t size() const { return PySequence_Fast_GET_SIZE(seq); }
    PyObject* operator[](Py_ssize_t i) const { return PySequence_Fast_GET_ITEM(seq, i); }
};
// (tensors, lr, beta1, beta2, eps, step, grad_scale, seed, stream)
PyObject* adamw_step(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (!count(n, 9)) return nullptr;
    const Items items(a[0], "expected a sequence of tensors with their moments");
    if (!items.seq) return nullptr;
    const Py_ssize_t len = items.size();
    std::vector<snip_adamw_tensor> ts((size_t)len);
    for (Py_ssize_t i = 0; i < len; ++i)
        if (!adamw_tensor(items[i], ts[(size_t)i])) return nullptr;
    const double lr = PyFloat_AsDouble(a[1]), b1 = PyFloat_AsDouble(a[2]), b2 = PyFloat_AsDouble(a[3]), eps = PyFloat_AsDouble(a[4]);
    int64_t step; void *gs, *s; snip_out_dtype d32;
    if (PyErr_Occurred() || !integer(a[5], step) || !vector(a[6], 1, true, gs, d32)) return nullptr;
    const unsigned long long seed = PyLong_AsUnsignedLongLong(a[7]);
    if ((seed == (unsigned long long)-1 && PyErr_Occurred()) || !stream(a[8], s)) return nullptr;
    return call([&] { return p_adamw_step(ts.data(), (int32_t)len, lr, b1, b2, eps, step, (const float*)gs, seed, s); });
}

// (x, weights, outputs, out_dtype, stream): sequences of quantized tensors and of matrices
PyObject* gemv(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Source x; int64_t dt; void* s;
    if (!count(n, 5) || !source(a[0], x) || !integer(a[3], dt) || !stream(a[4], s)) return nullptr;
    const Items ws(a[1], "expected a sequence of quantized weights");
    if (!ws.seq) return nullptr;
    const Items ys(a[2], "expected a sequence of outputs");
    if (!ys.seq) return nullptr;
    const Py_ssize_t len = ws.size();
    std::vector<snip_qtensor> w((size_t)len);
    std::vector<void*> y((size_t)len);
    std::vector<int64_t> ld((size_t)len);
    if (ys.size() != len) { PyErr_SetString(PyExc_ValueError, "expected as many outputs as weights"); return nullptr; }
    for (Py_ssize_t i = 0; i < len; ++i) {
        const at::Tensor* t;
        if (!qtensor(ws[i], w[(size_t)i]) || !tensor(ys[i], t)) return nullptr;
        if (t->dim() != 2 || !t->is_cuda() || t->size(0) != x.rows || t->size(1) != w[(size_t)i].rows || (t->stride(1) != 1 && t->size(1) > 1) ||
            t->scalar_type() != (dt == SNIP_OUT_FP32 ? at::kFloat : at::kBFloat16)) {
            PyErr_SetString(PyExc_ValueError, "expected CUDA matrices of the output type, a row for each token and a column for each row of the weight");
            return nullptr;
        }
        y[(size_t)i] = t->data_ptr();
        ld[(size_t)i] = t->stride(0);
    }
    return call([&] { return p_gemv(x.p, x.rows, x.cols, x.ld, w.data(), y.data(), ld.data(), (int32_t)len, (snip_out_dtype)dt, s); });
}

template <class F> bool find(void* lib, const char* name, F& f)
{
    f = (F)dlsym(lib, name);
    if (!f) PyErr_Format(PyExc_RuntimeError, "the library has no symbol %s", name);
    return f != nullptr;
}
// (path of the library)
PyObject* bind(PyObject*, PyObject* arg)
{
    const char* path = PyUnicode_AsUTF8(arg);
    if (!path) return nullptr;
    void* lib = dlopen(path, RTLD_NOW | RTLD_LOCAL);
    if (!lib) { PyErr_Format(PyExc_RuntimeError, "%s", dlerror()); return nullptr; }
    if (!find(lib, "snip_quantize", p_quantize) || !find(lib, "snip_quantize_both", p_quantize_both) ||
        !find(lib, "snip_quantize_sr_fp4", p_quantize_sr_fp4) || !find(lib, "snip_gemm_fwd", p_gemm[0]) || !find(lib, "snip_gemm_dgrad", p_gemm[1]) ||
        !find(lib, "snip_gemm_wgrad", p_gemm[2]) || !find(lib, "snip_gemm_fwd_norm", p_gemm_norm[0]) ||
        !find(lib, "snip_gemm_dgrad_norm", p_gemm_norm[1]) || !find(lib, "snip_gemm_wgrad_norm", p_gemm_norm[2]) ||
        !find(lib, "snip_quantize_paper", p_quantize_paper) || !find(lib, "snip_gemm_paper", p_gemm_paper) ||
        !find(lib, "snip_quant_error_stats", p_stats) || !find(lib, "snip_quant_error_stats_both", p_stats_both) ||
        !find(lib, "snip_adamw_sensitivity", p_adamw) || !find(lib, "snip_rms_norm", p_rms_norm) ||
        !find(lib, "snip_rms_norm_backward", p_rms_norm_backward) || !find(lib, "snip_adamw_step", p_adamw_step) ||
        !find(lib, "snip_gemv", p_gemv))
        return nullptr;
    Py_RETURN_NONE;
}

// torch reports errors (no device, a tensor without storage) as C++ exceptions
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    try {
        return F(self, a, n);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}
#define SNIP_FAST(name) {#name, (PyCFunction)(void (*)(void))guarded<name>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"bind", bind, METH_O, nullptr}, SNIP_FAST(quantize), SNIP_FAST(quantize_both), SNIP_FAST(quantize_sr_fp4),
                         SNIP_FAST(gemm), SNIP_FAST(gemm_norm), SNIP_FAST(quantize_paper), SNIP_FAST(gemm_paper), SNIP_FAST(stats),
                         SNIP_FAST(stats_both), SNIP_FAST(adamw), SNIP_FAST(rms_norm), SNIP_FAST(rms_norm_backward), SNIP_FAST(adamw_step), SNIP_FAST(gemv), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_snip_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__snip_binding(void)
{
    s_codes = PyUnicode_InternFromString("codes");
    s_scales = PyUnicode_InternFromString("scales");
    s_scales_g4 = PyUnicode_InternFromString("scales_g4");
    s_rows = PyUnicode_InternFromString("rows");
    s_cols = PyUnicode_InternFromString("cols");
    s_fmt = PyUnicode_InternFromString("fmt");
    s_param = PyUnicode_InternFromString("param");
    s_grad = PyUnicode_InternFromString("grad");
    s_m = PyUnicode_InternFromString("m");
    s_v = PyUnicode_InternFromString("v");
    s_copy = PyUnicode_InternFromString("copy");
    s_m_scale = PyUnicode_InternFromString("m_scale");
    s_v_scale = PyUnicode_InternFromString("v_scale");
    s_weight_decay = PyUnicode_InternFromString("weight_decay");
    return PyModule_Create(&module);
}
