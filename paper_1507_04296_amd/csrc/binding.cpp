// Native half of the sequence operators' Python binding: checks tensors, allocates
// outputs and makes the library call.  A single step of one actor costs the GPU 4 us;
// the same checks in Python cost 9 us beside the launch, these under 1.
//
// Functions take (context handle, device index, raw stream, ...) and call the C entry
// points through the addresses that init() is given, so that the library is the one
// that the package loaded.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <array>
#include <string>
#include <vector>

#include "../../include/gorila.h"

namespace {

struct Refused {  // becomes a Python exception
    PyObject* type;
    std::string what;
};

struct Api {
    decltype(&gorila_ctx_set_stream) set_stream;
    decltype(&gorila_add_rmsnorm) add_rmsnorm;
    decltype(&gorila_add_rmsnorm_codes) add_rmsnorm_codes;
    decltype(&gorila_add_rmsnorm_backward) add_rmsnorm_backward;
    decltype(&gorila_causal_conv) causal_conv;
    decltype(&gorila_causal_conv_backward) causal_conv_backward;
    decltype(&gorila_causal_conv_step) causal_conv_step;
    decltype(&gorila_scan) scan;
    decltype(&gorila_scan_backward) scan_backward;
    decltype(&gorila_scan_step) scan_step;
    decltype(&gorila_quantize_weights) quantize_weights;
    decltype(&gorila_qmatvec) qmatvec;
    decltype(&gorila_add_layernorm) add_layernorm;
    decltype(&gorila_add_layernorm_backward) add_layernorm_backward;
    decltype(&gorila_gated_scan) gated_scan;
    decltype(&gorila_gated_scan_backward) gated_scan_backward;
    decltype(&gorila_gated_scan_step) gated_scan_step;
    decltype(&gorila_adamw) adamw;
    decltype(&gorila_adamw_values) adamw_values;
    decltype(&gorila_sample_actions) sample_actions;
};
Api api{};
PyObject* raise_code = nullptr;  // of a return code and a call's name

using at::Tensor;
typedef std::initializer_list<int64_t> Shape;

std::string text(c10::IntArrayRef s) {
    std::string o = "(";
    for (size_t i = 0; i < s.size(); ++i) o += (i ? ", " : "") + std::to_string(s[i]);
    return o + ")";
}
[[noreturn]] void value(const std::string& what) { throw Refused{PyExc_ValueError, what}; }
[[noreturn]] void type(const std::string& what) { throw Refused{PyExc_TypeError, what}; }
void want(bool ok, const char* what) {
    if (!ok) value(what);
}
int32_t size32(int64_t v) {
    want(v <= INT32_MAX, "a dimension does not fit 32 bits");
    return (int32_t)v;
}

// One call's arguments.
struct Call {
    PyObject* const* a;
    gorila_ctx* ctx;
    int index;
    Call(PyObject* const* args, Py_ssize_t n, Py_ssize_t expect) : a(args) {
        if (n != expect) type("wrong number of arguments");
        if (!api.scan) throw Refused{PyExc_RuntimeError, "the library's entry points are not set"};
        ctx = (gorila_ctx*)PyLong_AsVoidPtr(args[0]);
        index = (int)integer(1);
        void* stream = PyLong_AsVoidPtr(args[2]);
        if (PyErr_Occurred()) throw Refused{nullptr, ""};
        check(api.set_stream(ctx, stream), "gorila_ctx_set_stream");
    }
    int64_t integer(int i) const {
        const int64_t v = PyLong_AsLongLong(a[i]);
        if (v == -1 && PyErr_Occurred()) throw Refused{nullptr, ""};
        return v;
    }
    double real(int i) const {
        const double v = PyFloat_AsDouble(a[i]);
        if (v == -1.0 && PyErr_Occurred()) throw Refused{nullptr, ""};
        return v;
    }
    float number(int i) const { return (float)real(i); }
    uint64_t bits(int i) const {
        const uint64_t v = PyLong_AsUnsignedLongLong(a[i]);
        if (PyErr_Occurred()) throw Refused{nullptr, ""};
        return v;
    }
    const Tensor* maybe(int i, const char* name) const {
        if (a[i] == Py_None) return nullptr;
        if (!THPVariable_Check(a[i])) type(std::string(name) + " must be a tensor");
        return &THPVariable_Unpack(a[i]);
    }
    const Tensor& tensor(int i, const char* name) const {
        const Tensor* t = maybe(i, name);
        if (!t) type(std::string(name) + " must be a tensor");
        return *t;
    }
    void check(int rc, const char* what) const {
        if (rc == 0) return;
        PyObject* r = PyObject_CallFunction(raise_code, "is", rc, what);
        Py_XDECREF(r);
        throw Refused{nullptr, ""};
    }
    // Address of an optional tensor of `shape` and `dtype` on the device.  The dimensions
    // from `strided` on are contiguous; the leading ones have strides of their own.
    void* at(const Tensor* t, const char* name, c10::IntArrayRef shape, at::ScalarType dtype, int64_t strided = 0) const {
        if (!t) return nullptr;
        if (t->sizes() != shape) value(std::string(name) + " must have shape " + text(shape) + ", got " + text(t->sizes()));
        if (t->scalar_type() != dtype)
            type(std::string(name) + " must be " + c10::toString(dtype) + ", got " + c10::toString(t->scalar_type()));
        if (!t->is_cuda() || t->get_device() != index) value(std::string(name) + " must be on device " + std::to_string(index));
        if (!t->is_contiguous()) {
            int64_t run = 1;
            for (int64_t d = t->dim() - 1; d >= strided; --d)
                if (t->size(d) > 1) {
                    if (t->stride(d) != run)
                        value(std::string(name) + " must be contiguous from dimension " + std::to_string(strided) + " on");
                    run *= t->size(d);
                }
        }
        return t->data_ptr();
    }
    void* at(const Tensor& t, const char* name, c10::IntArrayRef shape, at::ScalarType dtype, int64_t strided = 0) const {
        return at(&t, name, shape, dtype, strided);
    }
};

constexpr auto F32 = at::kFloat;
int32_t row_type(const Tensor& x) {
    if (x.scalar_type() == at::kFloat) return GORILA_F32;
    if (x.scalar_type() == at::kBFloat16) return GORILA_BF16;
    type(std::string("rows must be float32 or bfloat16, got ") + c10::toString(x.scalar_type()));
}
Tensor make(c10::IntArrayRef shape, const Tensor& like, at::ScalarType dtype) { return at::empty(shape, like.options().dtype(dtype)); }
Tensor same(const Tensor& t) { return at::empty(t.sizes(), t.options()); }
void* ptr(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
// What a call has written in place counts a new version, as after every such update, for
// graphs that still need the old values.
void changed(const Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// A tuple of tensors; an undefined one is None.
PyObject* tuple(std::initializer_list<const Tensor*> ts) {
    PyObject* o = PyTuple_New((Py_ssize_t)ts.size());
    if (!o) throw Refused{nullptr, ""};
    Py_ssize_t i = 0;
    for (const Tensor* t : ts) {
        PyObject* v = t->defined() ? THPVariable_Wrap(*t) : Py_NewRef(Py_None);
        if (!v) {
            Py_DECREF(o);
            throw Refused{nullptr, ""};
        }
        PyTuple_SET_ITEM(o, i++, v);
    }
    return o;
}
PyObject* one(const Tensor& t) {
    PyObject* v = THPVariable_Wrap(t);
    if (!v) throw Refused{nullptr, ""};
    return v;
}

// ---- norm ----

struct Norm {
    const Tensor& x;
    const Tensor* r;
    int64_t rows, width;
    int32_t dtype;
    const void *px, *pr;
    const float* weight;
    Norm(const Call& c) : x(c.tensor(3, "x")), r(c.maybe(5, "residual")) {
        want(x.dim() == 2, "x must be [rows, width]");
        rows = x.size(0), width = x.size(1);
        dtype = row_type(x);
        px = c.at(x, "x", x.sizes(), x.scalar_type(), 1);
        pr = c.at(r, "residual", x.sizes(), x.scalar_type(), 1);
        weight = (const float*)c.at(c.tensor(4, "weight"), "weight", {width}, F32);
    }
    int64_t rs() const { return r ? r->stride(0) : 0; }
    Tensor total() const { return r || !x.is_contiguous() ? same(x) : Tensor(); }
};

// x, weight, residual, eps
PyObject* add_rmsnorm(PyObject* const* args, Py_ssize_t n) {
    const Call c(args, n, 7);
    const Norm m(c);
    const Tensor y = same(m.x), total = m.total(), rstd = make({m.rows}, m.x, F32);
    c.check(api.add_rmsnorm(m.px, m.x.stride(0), m.pr, m.rs(), m.weight, m.rows, size32(m.width), m.dtype, c.number(6), ptr(y),
                            ptr(total), (float*)ptr(rstd), c.ctx), "gorila_add_rmsnorm");
    return tuple({&y, total.defined() ? &total : &m.x, &rstd});
}

PyObject* add_rmsnorm_codes(PyObject* const* args, Py_ssize_t n) {
    const Call c(args, n, 7);
    const Norm m(c);
    const Tensor codes = make(m.x.sizes(), m.x, at::kChar), total = m.total(), scale = make({m.rows}, m.x, F32);
    c.check(api.add_rmsnorm_codes(m.px, m.x.stride(0), m.pr, m.rs(), m.weight, m.rows, size32(m.width), m.dtype, c.number(6),
                                  (int8_t*)ptr(codes), (float*)ptr(scale), ptr(total), c.ctx), "gorila_add_rmsnorm_codes");
    return tuple({&codes, &scale, total.defined() ? &total : &m.x});
}

// dy, total, rstd, weight, dtotal
PyObject* add_rmsnorm_backward(PyObject* const* args, Py_ssize_t n) {
    const Call c(args, n, 8);
    const Tensor &dy = c.tensor(3, "dy"), &total = c.tensor(4, "total");
    const Tensor* dtotal = c.maybe(7, "dtotal");
    want(total.dim() == 2, "total must be [rows, width]");
    const int64_t rows = total.size(0), width = total.size(1);
    const int32_t dtype = row_type(total);
    const auto typ = total.scalar_type();
    const void *pdy = c.at(dy, "dy", total.sizes(), typ, 1), *pdt = c.at(dtotal, "dtotal", total.sizes(), typ, 1);
    const void* pt = c.at(total, "total", total.sizes(), typ);
    const float *rstd = (const float*)c.at(c.tensor(5, "rstd"), "rstd", {rows}, F32),
                *weight = (const float*)c.at(c.tensor(6, "weight"), "weight", {width}, F32);
    const Tensor dx = same(total), dweight = make({width}, total, F32);
    c.check(api.add_rmsnorm_backward(pdy, dy.stride(0), pdt, dtotal ? dtotal->stride(0) : 0, pt, rstd, weight, rows, size32(width),
                                     dtype, ptr(dx), (float*)ptr(dweight), c.ctx), "gorila_add_rmsnorm_backward");
    return tuple({&dx, &dweight});
}

// ---- short causal convolution ----

// x, weight, bias, reset, window (or the pool) from argument `i` on; silu at `silu`.
struct Conv {
    const Tensor &x, &w;
    gorila_causal_conv_args a{};
    Conv(const Call& c, int i, int silu, bool step) : x(c.tensor(i, "x")), w(c.tensor(i + 1, "weight")) {
        want(x.dim() == (step ? 2 : 3), step ? "x must be [rows, channels]" : "x must be [batch, length, channels]");
        a.dtype = row_type(x);
        const int64_t channels = x.size(-1), batch = x.size(0), length = step ? 1 : x.size(1);
        want(w.dim() == 2 && w.size(0) == channels, "weight must be [channels, taps]");
        const auto typ = x.scalar_type();
        a.batch = size32(batch), a.length = size32(length), a.channels = size32(channels), a.taps = size32(w.size(1));
        a.silu = c.integer(silu) != 0;
        a.x = c.at(x, "x", x.sizes(), typ, step ? 1 : 2);
        a.x_batch_stride = x.stride(0), a.x_step_stride = step ? 0 : x.stride(1);
        a.weight = (const float*)c.at(w, "weight", w.sizes(), F32);
        a.bias = (const float*)c.at(c.maybe(i + 2, "bias"), "bias", {channels}, F32);
        const Tensor* reset = c.maybe(i + 3, "reset");
        a.reset = (const uint8_t*)(step ? c.at(reset, "reset", {batch}, at::kByte) : c.at(reset, "reset", {batch, length}, at::kByte));
        if (!step) a.window = c.at(c.maybe(i + 4, "window"), "window", {batch, a.taps - 1, channels}, typ);
    }
};

// x, weight, bias, reset, window, silu
PyObject* causal_conv(PyObject* const* args, Py_ssize_t n) {
    const Call c(args, n, 9);
    const Conv v(c, 3, 8, false);
    const Tensor y = same(v.x), out = make({v.a.batch, v.a.taps > 1 ? v.a.taps - 1 : 0, v.a.channels}, v.x, v.x.scalar_type());
    c.check(api.causal_conv(&v.a, ptr(y), ptr(out), c.ctx), "gorila_causal_conv");
    return tuple({&y, &out});
}

// dy, x, weight, bias, reset, window, silu, dwindow_out
PyObject* causal_conv_backward(PyObject* const* args, Py_ssize_t n) {
    const Call c(args, n, 11);
    const Conv v(c, 4, 9, false);
    const Tensor& dy = c.tensor(3, "dy");
    const auto typ = v.x.scalar_type();
    const void* pdy = c.at(dy, "dy", v.x.sizes(), typ, 2);
    const void* pdw = c.at(c.maybe(10, "dwindow_out"), "dwindow_out", {v.a.batch, v.a.taps - 1, v.a.channels}, typ);
    const Tensor dx = same(v.x), dweight = same(v.w), dbias = v.a.bias ? make({v.a.channels}, v.x, F32) : Tensor();
    const Tensor dwindow = v.a.window ? make({v.a.batch, v.a.taps - 1, v.a.channels}, v.x, typ) : Tensor();
    c.check(api.causal_conv_backward(&v.a, pdy, dy.stride(0), dy.stride(1), pdw, ptr(dx), (float*)ptr(dweight), (float*)ptr(dbias),
                                     ptr(dwindow), c.ctx), "gorila_causal_conv_backward");
    return tuple({&dx, &dweight, &dbias, &dwindow});
}

// x, weight, bias, reset, window_pool, slot, silu
PyObject* causal_conv_step(PyObject* const* args, Py_ssize_t n) {
    const Call c(args, n, 10);
    const Conv v(c, 3, 9, true);
    const Tensor& pool = c.tensor(7, "window_pool");
    want(pool.dim() == 3, "window_pool must be [slots, taps - 1, channels]");
    const int64_t slots = pool.size(0);
    void* p = c.at(pool, "window_pool", {slots, v.a.taps - 1, v.a.channels}, v.x.scalar_type());
    const int32_t* slot = (const int32_t*)c.at(c.maybe(8, "slot"), "slot", {v.a.batch}, at::kInt);
    const Tensor y = same(v.x);
    c.check(api.causal_conv_step(&v.a, p, slots, slot, ptr(y), c.ctx), "gorila_causal_conv_step");
    changed(pool);
    return one(y);
}

// ---- selective scan ----

// x, dt, b, c, a_log, dt_bias, skip, reset, state (or the pool) from argument `i` on.
struct Scan {
    const Tensor &x, &dt, &b, &c;
    gorila_scan_args a{};
    Scan(const Call& k, int i, bool step)
        : x(k.tensor(i, "x")), dt(k.tensor(i + 1, "dt")), b(k.tensor(i + 2, "b")), c(k.tensor(i + 3, "c")) {
        const int64_t lead = step ? 1 : 2;
        want(x.dim() == lead + 2, step ? "x must be [rows, heads, head_dim]" : "x must be [batch, length, heads, head_dim]");
        want(b.dim() == lead + 2, "b must be [..., groups, state_dim]");
        a.dtype = row_type(x);
        const auto typ = x.scalar_type();
        const int64_t batch = x.size(0), length = step ? 1 : x.size(1), heads = x.size(lead), width = x.size(lead + 1);
        const int64_t groups = b.size(lead), n = b.size(lead + 1);
        a.batch = size32(batch), a.length = size32(length), a.heads = size32(heads), a.head_dim = size32(width);
        a.groups = size32(groups), a.state_dim = size32(n);
        a.x = k.at(x, "x", x.sizes(), typ, lead);
        const int64_t step_dt[2] = {batch, heads}, seq_dt[3] = {batch, length, heads};
        const int64_t step_b[3] = {batch, groups, n}, seq_b[4] = {batch, length, groups, n};
        const c10::IntArrayRef sd = step ? c10::IntArrayRef(step_dt, 2) : c10::IntArrayRef(seq_dt, 3);
        const c10::IntArrayRef sb = step ? c10::IntArrayRef(step_b, 3) : c10::IntArrayRef(seq_b, 4);
        a.dt = k.at(dt, "dt", sd, typ, lead);
        a.b = k.at(b, "b", sb, typ, lead);
        a.c = k.at(c, "c", sb, typ, lead);
        a.x_batch_stride = x.stride(0), a.dt_batch_stride = dt.stride(0), a.b_batch_stride = b.stride(0), a.c_batch_stride = c.stride(0);
        if (!step) a.x_step_stride = x.stride(1), a.dt_step_stride = dt.stride(1), a.b_step_stride = b.stride(1), a.c_step_stride = c.stride(1);
        a.a_log = (const float*)k.at(k.tensor(i + 4, "a_log"), "a_log", {heads}, F32);
        a.dt_bias = (const float*)k.at(k.tensor(i + 5, "dt_bias"), "dt_bias", {heads}, F32);
        a.skip = (const float*)k.at(k.tensor(i + 6, "skip"), "skip", {heads}, F32);
        a.reset = (const uint8_t*)k.at(k.maybe(i + 7, "reset"), "reset", sd.slice(0, (size_t)lead), at::kByte);
        if (!step) a.state = (const float*)k.at(k.maybe(i + 8, "state"), "state", {batch, heads, width, n}, F32);
    }
};

PyObject* scan(PyObject* const* args, Py_ssize_t n) {
    const Call c(args, n, 12);
    const Scan v(c, 3, false);
    const Tensor y = same(v.x), out = make({v.a.batch, v.a.heads, v.a.head_dim, v.a.state_dim}, v.x, F32);
    c.check(api.scan(&v.a, ptr(y), (float*)ptr(out), c.ctx), "gorila_scan");
    return tuple({&y, &out});
}

// dy, the inputs, dstate_out
PyObject* scan_backward(PyObject* const* args, Py_ssize_t n) {
    const Call c(args, n, 14);
    const Scan v(c, 4, false);
    const Tensor& dy = c.tensor(3, "dy");
    const void* pdy = c.at(dy, "dy", v.x.sizes(), v.x.scalar_type(), 2);
    const float* pds = (const float*)c.at(c.maybe(13, "dstate_out"), "dstate_out", {v.a.batch, v.a.heads, v.a.head_dim, v.a.state_dim}, F32);
    const Tensor dx = same(v.x), ddt = same(v.dt), db = same(v.b), dc = same(v.c);
    const Tensor da = make({v.a.heads}, v.x, F32), dbias = make({v.a.heads}, v.x, F32), dskip = make({v.a.heads}, v.x, F32);
    const Tensor ds = v.a.state ? make({v.a.batch, v.a.heads, v.a.head_dim, v.a.state_dim}, v.x, F32) : Tensor();
    c.check(api.scan_backward(&v.a, pdy, dy.stride(0), dy.stride(1), pds, ptr(dx), ptr(ddt), ptr(db), ptr(dc), (float*)ptr(da),
                              (float*)ptr(dbias), (float*)ptr(dskip), (float*)ptr(ds), c.ctx), "gorila_scan_backward");
    return tuple({&dx, &ddt, &db, &dc, &da, &dbias, &dskip, &ds});
}

// the inputs with the pool in the state's place, slot
PyObject* scan_step(PyObject* const* args, Py_ssize_t n) {
    const Call c(args, n, 13);
    const Scan v(c, 3, true);
    const Tensor& pool = c.tensor(11, "state_pool");
    want(pool.dim() == 4, "state_pool must be [slots, heads, head_dim, state_dim]");
    const int64_t slots = pool.size(0);
    float* p = (float*)c.at(pool, "state_pool", {slots, v.a.heads, v.a.head_dim, v.a.state_dim}, F32);
    const int32_t* slot = (const int32_t*)c.at(c.maybe(12, "slot"), "slot", {v.a.batch}, at::kInt);
    const Tensor y = same(v.x);
    c.check(api.scan_step(&v.a, p, slots, slot, ptr(y), c.ctx), "gorila_scan_step");
    changed(pool);
    return one(y);
}

// ---- 4-bit weights ----

int32_t group_of(const Call& c, int i) {
    const int64_t g = c.integer(i);
    want(g == 32 || g == 64 || g == 128, "group must be 32, 64 or 128");
    return (int32_t)g;
}

// weights, group
PyObject* quantize_weights(PyObject* const* args, Py_ssize_t n) {
    const Call c(args, n, 5);
    const Tensor& w = c.tensor(3, "weights");
    want(w.dim() == 2, "weights must be [outputs, inputs]");
    const int32_t group = group_of(c, 4), dtype = row_type(w);
    const int64_t outputs = w.size(0), inputs = w.size(1);
    const void* p = c.at(w, "weights", w.sizes(), w.scalar_type(), 1);
    const Tensor codes = make({outputs, 16 * ((inputs + 31) / 32)}, w, at::kByte), scales = make({outputs, (inputs + group - 1) / group}, w, F32);
    c.check(api.quantize_weights(p, w.stride(0), size32(outputs), size32(inputs), dtype, group, (uint8_t*)ptr(codes), (float*)ptr(scales),
                                 c.ctx), "gorila_quantize_weights");
    return tuple({&codes, &scales});
}

// x, codes, scales, group, x_scale
PyObject* qmatvec(PyObject* const* args, Py_ssize_t n) {
    const Call c(args, n, 8);
    const Tensor &x = c.tensor(3, "x"), &codes = c.tensor(4, "codes"), &scales = c.tensor(5, "scales");
    const Tensor* xs = c.maybe(7, "x_scale");
    want(x.dim() == 2 && codes.dim() == 2, "x must be [rows, inputs], codes [outputs, bytes]");
    const int32_t group = group_of(c, 6);
    const int64_t rows = x.size(0), inputs = x.size(1), outputs = codes.size(0);
    const bool whole = x.scalar_type() == at::kChar;
    want(!whole || xs, "int8 rows need x_scale");
    want(whole || !xs, "x_scale goes with int8 rows");
    const int32_t dtype = whole ? (int32_t)GORILA_CODES : row_type(x);
    const void* px = c.at(x, "x", x.sizes(), x.scalar_type(), 1);
    const float* pxs = (const float*)c.at(xs, "x_scale", {rows}, F32);
    const uint8_t* pc = (const uint8_t*)c.at(codes, "codes", {outputs, 16 * ((inputs + 31) / 32)}, at::kByte);
    const float* ps = (const float*)c.at(scales, "scales", {outputs, (inputs + group - 1) / group}, F32);
    const Tensor y = make({rows, outputs}, x, whole ? F32 : x.scalar_type());
    c.check(api.qmatvec(px, x.stride(0), pxs, dtype, rows, pc, ps, size32(outputs), size32(inputs), group, ptr(y), c.ctx), "gorila_qmatvec");
    return one(y);
}

// ---- layer norm ----

// x, weight, bias, residual, eps
PyObject* add_layernorm(PyObject* const* args, Py_ssize_t n) {
    const Call c(args, n, 8);
    const Tensor &x = c.tensor(3, "x"), &w = c.tensor(4, "weight");
    const Tensor *b = c.maybe(5, "bias"), *r = c.maybe(6, "residual");
    want(x.dim() == 2, "x must be [rows, width]");
    const int64_t rows = x.size(0), width = x.size(1);
    const int32_t dtype = row_type(x);
    const void *px = c.at(x, "x", x.sizes(), x.scalar_type(), 1), *pr = c.at(r, "residual", x.sizes(), x.scalar_type(), 1);
    const float *pw = (const float*)c.at(w, "weight", {width}, F32), *pb = (const float*)c.at(b, "bias", {width}, F32);
    const Tensor y = same(x), total = r || !x.is_contiguous() ? same(x) : Tensor(), mean = make({rows}, x, F32), rstd = make({rows}, x, F32);
    c.check(api.add_layernorm(px, x.stride(0), pr, r ? r->stride(0) : 0, pw, pb, rows, size32(width), dtype, c.number(7), ptr(y), ptr(total),
                              (float*)ptr(mean), (float*)ptr(rstd), c.ctx), "gorila_add_layernorm");
    return tuple({&y, total.defined() ? &total : &x, &mean, &rstd});
}

// dy, total, mean, rstd, weight, dtotal
PyObject* add_layernorm_backward(PyObject* const* args, Py_ssize_t n) {
    const Call c(args, n, 9);
    const Tensor &dy = c.tensor(3, "dy"), &total = c.tensor(4, "total");
    const Tensor* dtotal = c.maybe(8, "dtotal");
    want(total.dim() == 2, "total must be [rows, width]");
    const int64_t rows = total.size(0), width = total.size(1);
    const int32_t dtype = row_type(total);
    const auto typ = total.scalar_type();
    const void *pdy = c.at(dy, "dy", total.sizes(), typ, 1), *pdt = c.at(dtotal, "dtotal", total.sizes(), typ, 1);
    const void* pt = c.at(total, "total", total.sizes(), typ);
    const float *mean = (const float*)c.at(c.tensor(5, "mean"), "mean", {rows}, F32),
                *rstd = (const float*)c.at(c.tensor(6, "rstd"), "rstd", {rows}, F32),
                *weight = (const float*)c.at(c.tensor(7, "weight"), "weight", {width}, F32);
    const Tensor dx = same(total), dweight = make({width}, total, F32), dbias = make({width}, total, F32);
    c.check(api.add_layernorm_backward(pdy, dy.stride(0), pdt, dtotal ? dtotal->stride(0) : 0, pt, mean, rstd, weight, rows, size32(width),
                                       dtype, ptr(dx), (float*)ptr(dweight), (float*)ptr(dbias), c.ctx), "gorila_add_layernorm_backward");
    return tuple({&dx, &dweight, &dbias});
}

// ---- gated scan ----

// x, gate_a, gate_x, a_log from argument `i` on, reset at `reset`.
struct Gated {
    const Tensor &x, &ga, &gx;
    gorila_gated_scan_args a{};
    Gated(const Call& k, int i, int reset, bool step) : x(k.tensor(i, "x")), ga(k.tensor(i + 1, "gate_a")), gx(k.tensor(i + 2, "gate_x")) {
        const int64_t lead = step ? 1 : 2;
        want(x.dim() == lead + 1, step ? "x must be [rows, channels]" : "x must be [batch, length, channels]");
        a.dtype = row_type(x);
        const auto typ = x.scalar_type();
        a.batch = size32(x.size(0)), a.length = step ? 1 : size32(x.size(1)), a.channels = size32(x.size(lead));
        a.x = k.at(x, "x", x.sizes(), typ, lead);
        a.gate_a = k.at(ga, "gate_a", x.sizes(), typ, lead);
        a.gate_x = k.at(gx, "gate_x", x.sizes(), typ, lead);
        a.x_batch_stride = x.stride(0), a.gate_a_batch_stride = ga.stride(0), a.gate_x_batch_stride = gx.stride(0);
        if (!step) a.x_step_stride = x.stride(1), a.gate_a_step_stride = ga.stride(1), a.gate_x_step_stride = gx.stride(1);
        a.a_log = (const float*)k.at(k.tensor(i + 3, "a_log"), "a_log", {(int64_t)a.channels}, F32);
        a.reset = (const uint8_t*)k.at(k.maybe(reset, "reset"), "reset", x.sizes().slice(0, (size_t)lead), at::kByte);
    }
    std::array<int64_t, 2> state() const { return {a.batch, a.channels}; }
    std::array<int64_t, 3> marks() const { return {a.batch, ((int64_t)a.length + GORILA_GATED_MARK - 1) / GORILA_GATED_MARK, a.channels}; }
};

// x, gate_a, gate_x, a_log, reset, state, marks
PyObject* gated_scan(PyObject* const* args, Py_ssize_t n) {
    const Call c(args, n, 10);
    Gated v(c, 3, 7, false);
    v.a.state = (const float*)c.at(c.maybe(8, "state"), "state", v.state(), F32);
    const Tensor y = same(v.x), out = make(v.state(), v.x, F32), marks = c.integer(9) ? make(v.marks(), v.x, F32) : Tensor();
    c.check(api.gated_scan(&v.a, ptr(y), (float*)ptr(out), (float*)ptr(marks), c.ctx), "gorila_gated_scan");
    return tuple({&y, &out, &marks});
}

// dy, x, gate_a, gate_x, a_log, marks, reset, dstate_out
PyObject* gated_scan_backward(PyObject* const* args, Py_ssize_t n) {
    const Call c(args, n, 11);
    const Gated v(c, 4, 9, false);
    const Tensor& dy = c.tensor(3, "dy");
    const void* pdy = c.at(dy, "dy", v.x.sizes(), v.x.scalar_type(), 2);
    const float* marks = (const float*)c.at(c.tensor(8, "marks"), "marks", v.marks(), F32);
    const float* pds = (const float*)c.at(c.maybe(10, "dstate_out"), "dstate_out", v.state(), F32);
    const Tensor dx = same(v.x), dga = same(v.x), dgx = same(v.x), da = make({(int64_t)v.a.channels}, v.x, F32), ds = make(v.state(), v.x, F32);
    c.check(api.gated_scan_backward(&v.a, marks, pdy, dy.stride(0), dy.stride(1), pds, ptr(dx), ptr(dga), ptr(dgx), (float*)ptr(da),
                                    (float*)ptr(ds), c.ctx), "gorila_gated_scan_backward");
    return tuple({&dx, &dga, &dgx, &da, &ds});
}

// x, gate_a, gate_x, a_log, state_pool, slot, reset
PyObject* gated_scan_step(PyObject* const* args, Py_ssize_t n) {
    const Call c(args, n, 10);
    const Gated v(c, 3, 9, true);
    const Tensor& pool = c.tensor(7, "state_pool");
    want(pool.dim() == 2, "state_pool must be [slots, channels]");
    const int64_t slots = pool.size(0);
    float* p = (float*)c.at(pool, "state_pool", {slots, (int64_t)v.a.channels}, F32);
    const int32_t* slot = (const int32_t*)c.at(c.maybe(8, "slot"), "slot", {(int64_t)v.a.batch}, at::kInt);
    const Tensor y = same(v.x);
    c.check(api.gated_scan_step(&v.a, p, slots, slot, ptr(y), c.ctx), "gorila_gated_scan_step");
    changed(pool);
    return one(y);
}

// ---- AdamW ----

struct Listed {  // a list or tuple; it must outlive what is taken from it
    PyObject* o;
    Py_ssize_t n;
    Listed(PyObject* from, const char* name) {
        if (!PyList_Check(from) && !PyTuple_Check(from)) type(std::string(name) + " must be a list or a tuple");
        o = from, n = PySequence_Fast_GET_SIZE(from);
    }
    PyObject* operator[](Py_ssize_t i) const { return PySequence_Fast_GET_ITEM(o, i); }
    const Tensor& tensor(Py_ssize_t i, const char* name) const {
        if (!THPVariable_Check((*this)[i])) type(std::string(name) + " must hold tensors");
        return THPVariable_Unpack((*this)[i]);
    }
};
struct Spans {  // bytes that a call writes, and others that it reads
    typedef std::pair<const char*, const char*> Span;
    std::vector<Span> written, read;
    static void add(std::vector<Span>& to, const void* p, int64_t bytes) {
        if (bytes > 0) to.emplace_back((const char*)p, (const char*)p + bytes);
    }
    void write(const void* p, int64_t bytes) { add(written, p, bytes); }
    void check() {
        std::sort(written.begin(), written.end());
        for (size_t i = 1; i < written.size(); ++i) want(written[i].first >= written[i - 1].second, "tensors and states must not overlap");
        for (const Span& r : read) {  // the last written one that starts before its end
            const auto w = std::lower_bound(written.begin(), written.end(), Span(r.second, nullptr));
            if (w != written.begin()) want((w - 1)->second <= r.first, "gradients must not overlap tensors and states");
        }
    }
};
// m and v of a state, and its scales where it has four members (8 bits).
int state_of(const Call& c, PyObject* state, c10::IntArrayRef shape, int64_t n, gorila_adamw_tensor& t, Spans& w) {
    const Listed s(state, "a state");
    want(s.n == 2 || s.n == 4, "a state is (m, v), or (m, v, m_scale, v_scale) in 8 bits");
    const auto typ = s.n == 2 ? F32 : at::kByte;
    const int64_t bytes = s.n == 2 ? 4 : 1, groups = (n + 255) / 256;
    t.m = c.at(s.tensor(0, "a state"), "m", shape, typ);
    t.v = c.at(s.tensor(1, "a state"), "v", shape, typ);
    w.write(t.m, n * bytes), w.write(t.v, n * bytes);
    if (s.n == 4) {
        t.m_scale = (float*)c.at(s.tensor(2, "a state"), "m_scale", {groups}, F32);
        t.v_scale = (float*)c.at(s.tensor(3, "a state"), "v_scale", {groups}, F32);
        w.write(t.m_scale, groups * 4), w.write(t.v_scale, groups * 4);
    }
    return s.n == 2 ? 32 : 8;
}

// thetas, grads, states, clock, lr, beta1, beta2, eps, decay, seed, keep
PyObject* adamw(PyObject* const* args, Py_ssize_t n) {
    const Call c(args, n, 14);
    const Listed thetas(args[3], "thetas"), grads(args[4], "grads"), states(args[5], "states");
    want(grads.n == thetas.n && states.n == thetas.n, "thetas, grads and states must be as many");
    const bool each = PyList_Check(args[11]) || PyTuple_Check(args[11]);
    if (each) want(PySequence_Fast_GET_SIZE(args[11]) == thetas.n, "decay must be a number, or one for each tensor");
    const float all = each ? 0.0f : c.number(11);
    std::vector<gorila_adamw_tensor> ts((size_t)thetas.n);
    Spans w;
    int bits = 32;
    int32_t dtype = GORILA_F32;
    for (Py_ssize_t i = 0; i < thetas.n; ++i) {
        gorila_adamw_tensor& t = ts[(size_t)i];
        const Tensor &theta = thetas.tensor(i, "thetas"), &grad = grads.tensor(i, "grads");
        t = gorila_adamw_tensor{};
        t.n = theta.numel();
        t.theta = (float*)c.at(theta, "theta", theta.sizes(), F32);
        const int32_t d = row_type(grad);
        t.grad = c.at(grad, "grad", theta.sizes(), grad.scalar_type());
        w.write(t.theta, t.n * 4);
        Spans::add(w.read, t.grad, t.n * (d == GORILA_F32 ? 4 : 2));
        const int b = state_of(c, states[i], theta.sizes(), t.n, t, w);
        if (i == 0) bits = b, dtype = d;
        want(b == bits && d == dtype, "all states have the same bits and all gradients the same type");
        t.decay = all;
        if (each) {
            const double v = PyFloat_AsDouble(PySequence_Fast_GET_ITEM(args[11], i));
            if (v == -1.0 && PyErr_Occurred()) throw Refused{nullptr, ""};
            t.decay = (float)v;
        }
    }
    double* clock = (double*)c.at(c.tensor(6, "clock"), "clock", {3}, at::kDouble);
    w.write(clock, 24);
    w.check();
    const Tensor* keep = c.maybe(13, "keep");
    const uint8_t* pk = keep ? (const uint8_t*)c.at(keep, "keep", {1}, at::kByte) : nullptr;
    c.check(api.adamw(ts.data(), size32(thetas.n), dtype, bits, clock, pk, c.number(7), c.real(8), c.real(9), c.number(10), c.bits(12), c.ctx),
            "gorila_adamw");
    changed(c.tensor(6, "clock"));
    for (Py_ssize_t i = 0; i < thetas.n; ++i) {
        changed(thetas.tensor(i, "thetas"));
        const Listed state(states[i], "a state");
        for (Py_ssize_t k = 0; k < state.n; ++k) changed(state.tensor(k, "a state"));
    }
    Py_RETURN_NONE;
}

// states
PyObject* adamw_values(PyObject* const* args, Py_ssize_t n) {
    const Call c(args, n, 4);
    const Listed states(args[3], "states");
    std::vector<gorila_adamw_tensor> ts((size_t)states.n);
    std::vector<Tensor> m, v;
    std::vector<float*> pm, pv;
    Spans w;
    for (Py_ssize_t i = 0; i < states.n; ++i) {
        const Listed state(states[i], "a state");
        want(state.n == 4, "the states must be held in 8 bits");
        const Tensor& first = state.tensor(0, "a state");
        ts[(size_t)i] = gorila_adamw_tensor{};
        ts[(size_t)i].n = first.numel();
        state_of(c, states[i], first.sizes(), ts[(size_t)i].n, ts[(size_t)i], w);
        m.push_back(make(first.sizes(), first, F32)), v.push_back(make(first.sizes(), first, F32));
        pm.push_back((float*)ptr(m.back())), pv.push_back((float*)ptr(v.back()));
    }
    c.check(api.adamw_values(ts.data(), size32(states.n), pm.data(), pv.data(), c.ctx), "gorila_adamw_values");
    PyObject* o = PyList_New(states.n);
    if (!o) throw Refused{nullptr, ""};
    for (Py_ssize_t i = 0; i < states.n; ++i) {
        PyObject* pair = nullptr;
        try {
            pair = tuple({&m[(size_t)i], &v[(size_t)i]});
        } catch (...) {
            Py_DECREF(o);
            throw;
        }
        PyList_SET_ITEM(o, i, pair);
    }
    return o;
}

// ---- sampled actions ----

// values, u, temperature, top_k, top_p, min_p
PyObject* sample_actions(PyObject* const* args, Py_ssize_t n) {
    const Call c(args, n, 9);
    const Tensor& values = c.tensor(3, "values");
    want(values.dim() == 2, "values must be [rows, actions]");
    const int32_t dtype = row_type(values);
    const int64_t rows = values.size(0), actions = values.size(1);
    const void* p = c.at(values, "values", values.sizes(), values.scalar_type(), 1);
    const float* u = (const float*)c.at(c.tensor(4, "u"), "u", {rows}, F32);
    const float* t = (const float*)c.at(c.maybe(5, "temperature"), "temperature", {rows}, F32);
    const int32_t* k = (const int32_t*)c.at(c.maybe(6, "top_k"), "top_k", {rows}, at::kInt);
    const float* tp = (const float*)c.at(c.maybe(7, "top_p"), "top_p", {rows}, F32);
    const float* mp = (const float*)c.at(c.maybe(8, "min_p"), "min_p", {rows}, F32);
    const Tensor action = make({rows}, values, at::kInt), probability = make({rows}, values, F32);
    c.check(api.sample_actions(p, values.stride(0), rows, size32(actions), dtype, u, t, k, tp, mp, (int32_t*)ptr(action), (float*)ptr(probability),
                               c.ctx), "gorila_sample_actions");
    return tuple({&action, &probability});
}

// The Python entry: what is thrown below becomes a Python exception.
template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    try {
        return F(args, n);
    } catch (const Refused& e) {
        if (e.type) PyErr_SetString(e.type, e.what.c_str());
        else if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "the call failed");
    } catch (const c10::Error& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

template <class F>
void take(F& f, PyObject* d, const char* name) {
    PyObject* v = PyDict_GetItemString(d, name);
    if (!v) throw Refused{PyExc_ValueError, std::string("no address of ") + name};
    f = (F)PyLong_AsVoidPtr(v);
}

// {entry point: address}, raise(code, what)
PyObject* init(PyObject* const* args, Py_ssize_t n) {
    if (n != 2 || !PyDict_Check(args[0])) type("init takes the entry points' addresses and a function");
    PyObject* d = args[0];
    Api p{};
    take(p.set_stream, d, "gorila_ctx_set_stream");
    take(p.add_rmsnorm, d, "gorila_add_rmsnorm");
    take(p.add_rmsnorm_codes, d, "gorila_add_rmsnorm_codes");
    take(p.add_rmsnorm_backward, d, "gorila_add_rmsnorm_backward");
    take(p.causal_conv, d, "gorila_causal_conv");
    take(p.causal_conv_backward, d, "gorila_causal_conv_backward");
    take(p.causal_conv_step, d, "gorila_causal_conv_step");
    take(p.scan, d, "gorila_scan");
    take(p.scan_backward, d, "gorila_scan_backward");
    take(p.scan_step, d, "gorila_scan_step");
    take(p.quantize_weights, d, "gorila_quantize_weights");
    take(p.qmatvec, d, "gorila_qmatvec");
    take(p.add_layernorm, d, "gorila_add_layernorm");
    take(p.add_layernorm_backward, d, "gorila_add_layernorm_backward");
    take(p.gated_scan, d, "gorila_gated_scan");
    take(p.gated_scan_backward, d, "gorila_gated_scan_backward");
    take(p.gated_scan_step, d, "gorila_gated_scan_step");
    take(p.adamw, d, "gorila_adamw");
    take(p.adamw_values, d, "gorila_adamw_values");
    take(p.sample_actions, d, "gorila_sample_actions");
    Py_INCREF(args[1]);
    Py_XDECREF(raise_code);
    raise_code = args[1];
    api = p;
    Py_RETURN_NONE;
}

#define ENTRY(name) {#name, (PyCFunction)(void (*)(void))entry<name>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(init), ENTRY(add_rmsnorm), ENTRY(add_rmsnorm_codes), ENTRY(add_rmsnorm_backward), ENTRY(causal_conv),
                         ENTRY(causal_conv_backward), ENTRY(causal_conv_step), ENTRY(scan), ENTRY(scan_backward), ENTRY(scan_step),
                         ENTRY(quantize_weights), ENTRY(qmatvec), ENTRY(add_layernorm), ENTRY(add_layernorm_backward),
                         ENTRY(gated_scan), ENTRY(gated_scan_backward), ENTRY(gated_scan_step), ENTRY(adamw), ENTRY(adamw_values),
                         ENTRY(sample_actions), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", "Native half of the sequence operators' binding.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
