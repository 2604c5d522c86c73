// Calls on rows in 8 bits straight from torch tensors (module _native).  A single token's norm or product takes the GPU 2 to 5 us;
// checking its tensors and marshalling 17 arguments in Python takes two to three times that, so it is done here.  Only argument
// checks and pointers: the calls are those of the C ABI, whose addresses bind() gets from the library that binding.py
// loaded.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/grad_mode.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "dnns.h"

namespace {

struct Calls {
    decltype(&dnns_quantize_rows) quantize_rows;
    decltype(&dnns_rmsnorm_quantize) rmsnorm_quantize;
    decltype(&dnns_rmsnorm_backward) rmsnorm_backward;
    decltype(&dnns_silu_gate_quantize) silu_gate_quantize;
    decltype(&dnns_silu_gate_backward) silu_gate_backward;
    decltype(&dnns_linear_quantized) linear_quantized;
} g_calls = {};

// A tensor that another one was laid out from, as long as somebody else holds it, and its version then.  (Tensors of inference mode
// count none.)
struct Original {
    c10::weak_intrusive_ptr<c10::TensorImpl, c10::UndefinedTensorImpl> t;
    int64_t version;
    static int64_t version_of(c10::TensorImpl* t) { return t->is_inference() ? 0 : (int64_t)t->version_counter().current_version(); }
    explicit Original(const at::Tensor& from) : t(from.getIntrusivePtr()), version(version_of(from.unsafeGetTensorImpl())) {}
};

// Where rows in 8 bits are.
struct Place {
    int8_t* q;
    float* scale;
    uint16_t* values;
    int64_t ldq, ldv;
};
// Rows in 8 bits: a RowsQ8's tensors.  Their addresses are taken at each call, since a tensor may be given other storage in between
// (set_, .data) or lose its own.  Or, without tensors, memory that the caller keeps where it is.
struct Rows {
    PyObject_HEAD
    at::Tensor q, scale, values;  // values: undefined where there are none
    Place place;                  // where q is undefined
    int64_t rows, cols, device;
    Original *of_q, *of_scale;    // null, or the tensors that q and scale were laid out from
};
PyTypeObject RowsType = {PyVarObject_HEAD_INIT(nullptr, 0)};

struct Matrix {
    void* p = nullptr;
    int64_t ld = 0;
    const at::Tensor* t = nullptr;
};

bool refuse(const char* what, const char* wants, PyObject* got) {
    PyErr_Format(PyExc_ValueError, "%s: %s is needed, got %R", what, wants, got);
    return false;
}

const at::Tensor* tensor_of(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }

// The current device, asked for once a call (under the interpreter's lock; guarded() forgets it).
int g_device = -1;
int device() { return g_device < 0 ? g_device = c10::cuda::current_device() : g_device; }

bool on_device(const at::Tensor& t, const char* what) {
    if (t.is_cuda() && t.get_device() == device()) return true;
    PyErr_Format(PyExc_ValueError, "%s: a tensor of the current CUDA device is needed", what);
    return false;
}

// The calls record nothing for autograd, so a result of a tensor that requires a gradient would be cut off from its graph without a
// word: it is refused where torch would record.
bool not_recorded(const at::Tensor& t, const char* what) {
    if (!t.requires_grad() || !at::GradMode::is_enabled()) return true;
    PyErr_Format(PyExc_ValueError, "%s: requires a gradient, which the call would not record: call it under torch.no_grad(), or with a detached tensor", what);
    return false;
}
// A tensor was written: torch's check of what was saved for a gradient sees it.  (Tensors of inference mode count no versions.)
void wrote(const at::Tensor* t) {
    if (t && t->defined() && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}

// dtype of a matrix of fp32 or bf16
bool dtype_of(PyObject* o, const char* what, at::ScalarType* type, int32_t* dtype) {
    const at::Tensor* t = tensor_of(o);
    if (!t || t->dim() != 2 || (t->scalar_type() != at::kFloat && t->scalar_type() != at::kBFloat16))
        return refuse(what, "a float32 or bfloat16 matrix", o);
    *type = t->scalar_type();
    *dtype = *type == at::kFloat ? DNNS_F32 : DNNS_BF16;
    return true;
}

// a rows x cols matrix of unit column stride
bool matrix(PyObject* o, int64_t rows, int64_t cols, at::ScalarType type, const char* what, Matrix* m) {
    const at::Tensor* t = tensor_of(o);
    if (!t || t->dim() != 2 || t->scalar_type() != type || t->size(0) != rows || t->size(1) != cols || (cols > 1 && t->stride(1) != 1)) {
        PyErr_Format(PyExc_ValueError, "%s: a %lld x %lld matrix of the right type with unit column stride is needed", what, (long long)rows, (long long)cols);
        return false;
    }
    if (!on_device(*t, what) || !not_recorded(*t, what)) return false;
    m->t = t;
    m->p = t->data_ptr();
    m->ld = rows > 1 ? t->stride(0) : std::max(cols, t->stride(0));
    return true;
}
bool matrix_or_none(PyObject* o, int64_t rows, int64_t cols, at::ScalarType type, const char* what, Matrix* m) {
    return o == Py_None || matrix(o, rows, cols, type, what, m);
}

bool vector_or_none(PyObject* o, int64_t n, const char* what, float** p, const at::Tensor** which = nullptr) {
    *p = nullptr;
    if (which) *which = nullptr;
    if (o == Py_None) return true;
    const at::Tensor* t = tensor_of(o);
    if (!t || t->scalar_type() != at::kFloat || t->dim() != 1 || t->size(0) != n || !t->is_contiguous()) {
        PyErr_Format(PyExc_ValueError, "%s: a contiguous float32 vector of %lld is needed", what, (long long)n);
        return false;
    }
    if (!on_device(*t, what) || !not_recorded(*t, what)) return false;
    if (which) *which = t;
    *p = static_cast<float*>(t->data_ptr());
    return true;
}

Rows* rows_of(PyObject* o) {
    if (Py_TYPE(o) != &RowsType) return refuse("rows", "rows in 8 bits", o), nullptr;
    return reinterpret_cast<Rows*>(o);
}
// The first rows x cols of a tensor, unit column stride, within its storage (looked at without counting a reference to it).
bool holds(const at::Tensor& t, int64_t rows, int64_t cols) {
    if (rows == 0 || cols == 0) return true;
    return (t.storage_offset() + (rows - 1) * t.stride(0) + cols) * (int64_t)t.itemsize() <= (int64_t)t.unsafeGetTensorImpl()->unsafe_storage().nbytes();
}
// Whether the originals of rows that were laid out anew are both there and have been written since.
bool changed(const Rows* r) {
    if (!r->of_q) return false;
    const auto q = r->of_q->t.lock(), s = r->of_scale->t.lock();
    return q && s && (Original::version_of(q.get()) != r->of_q->version || Original::version_of(s.get()) != r->of_scale->version);
}

// Where the rows are now (after a tensor of the call was found on the current device).
bool rows_here(const Rows* r, Place* p) {
    const at::Tensor &q = r->q, &s = r->scale, &v = r->values;
    if ((q.defined() ? q.get_device() : r->device) != device()) {
        PyErr_SetString(PyExc_ValueError, "rows: rows of the current CUDA device are needed");
        return false;
    }
    if (!q.defined()) return *p = r->place, true;
    if (q.dim() != 2 || q.size(0) != r->rows || q.size(1) < r->cols || (r->cols > 1 && q.stride(1) != 1) || s.dim() != 1 || s.size(0) != r->rows ||
        (r->rows > 1 && s.stride(0) != 1) || !holds(q, r->rows, r->cols) || !holds(s, r->rows, 1) ||
        (v.defined() && (v.dim() != 2 || v.size(0) != r->rows || v.size(1) != r->cols || (r->cols > 1 && v.stride(1) != 1) || !holds(v, r->rows, r->cols)))) {
        PyErr_SetString(PyExc_ValueError, "rows: a tensor of the rows has another shape, or less storage, than when they were made");
        return false;
    }
    if (!not_recorded(s, "scale of rows") || (v.defined() && !not_recorded(v, "values of rows"))) return false;
    p->q = static_cast<int8_t*>(q.data_ptr());
    p->scale = static_cast<float*>(s.data_ptr());
    p->values = v.defined() ? static_cast<uint16_t*>(v.data_ptr()) : nullptr;
    p->ldq = r->rows > 1 ? q.stride(0) : (r->cols + 15) / 16 * 16;
    p->ldv = v.defined() && r->rows > 1 ? v.stride(0) : r->cols;
    return true;
}

void* stream() { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device()).stream(); }

bool count_is(Py_ssize_t n, Py_ssize_t want) {
    if (n != want) PyErr_Format(PyExc_TypeError, "%zd arguments are needed, got %zd", want, n);
    return n == want;
}

PyObject* status(dnns_status s) { return PyLong_FromLong(s); }
// The status of a call that wrote rows, or other tensors.
PyObject* status(dnns_status s, const Rows* r) {
    if (s == DNNS_OK) wrote(&r->q), wrote(&r->scale), wrote(&r->values);
    return status(s);
}
PyObject* status(dnns_status s, std::initializer_list<const at::Tensor*> written) {
    if (s == DNNS_OK)
        for (const at::Tensor* t : written) wrote(t);
    return status(s);
}

// bind(addresses in the order of Calls)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!count_is(n, (Py_ssize_t)(sizeof(Calls) / sizeof(void*)))) return nullptr;
    void* p[sizeof(Calls) / sizeof(void*)];
    for (Py_ssize_t i = 0; i < n; ++i)
        if (!(p[i] = PyLong_AsVoidPtr(a[i]))) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "address %zd is null", i);
    static_assert(sizeof(p) == sizeof(Calls), "one address a call");
    memcpy(&g_calls, p, sizeof(p));
    Py_RETURN_NONE;
}

// rows(q, scale, values or None, cols): tensors that RowsQ8 has checked; or addresses: rows(q, ldq, scale, values, ldv, rows, cols, device)
PyObject* rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 8 && !count_is(n, 4)) return nullptr;
    const at::Tensor *q = nullptr, *scale = nullptr, *values = nullptr;
    long long v[8] = {};
    if (n == 4) {
        q = tensor_of(a[0]), scale = tensor_of(a[1]), values = tensor_of(a[2]);
        if (!q || !scale || (!values && a[2] != Py_None)) return PyErr_Format(PyExc_TypeError, "tensors are needed");
        v[6] = PyLong_AsLongLong(a[3]);
        if (v[6] == -1 && PyErr_Occurred()) return nullptr;
        v[5] = q->size(0);
    } else {
        for (int i = 0; i < 8; ++i) {
            v[i] = PyLong_AsLongLong(a[i]);
            if (v[i] == -1 && PyErr_Occurred()) return nullptr;
        }
    }
    Rows* r = PyObject_New(Rows, &RowsType);
    if (!r) return nullptr;
    new (&r->q) at::Tensor(q ? *q : at::Tensor());
    new (&r->scale) at::Tensor(scale ? *scale : at::Tensor());
    new (&r->values) at::Tensor(values ? *values : at::Tensor());
    r->place = {reinterpret_cast<int8_t*>(v[0]), reinterpret_cast<float*>(v[2]), reinterpret_cast<uint16_t*>(v[3]), v[1], v[4]};
    r->rows = v[5], r->cols = v[6], r->device = v[7];
    r->of_q = r->of_scale = nullptr;
    return reinterpret_cast<PyObject*>(r);
}
void rows_dealloc(PyObject* o) {
    Rows* r = reinterpret_cast<Rows*>(o);
    delete r->of_q;
    delete r->of_scale;
    r->q.~Tensor(), r->scale.~Tensor(), r->values.~Tensor();
    PyObject_Free(o);
}

// laid_out(rows, q, scale): the rows were just laid out from these tensors, and follow them
PyObject* laid_out(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Rows* r;
    if (!count_is(n, 3) || !(r = rows_of(a[0]))) return nullptr;
    const at::Tensor *q = tensor_of(a[1]), *scale = tensor_of(a[2]);
    if (!q || !scale) return PyErr_Format(PyExc_TypeError, "tensors are needed");
    auto of_q = std::make_unique<Original>(*q), of_scale = std::make_unique<Original>(*scale);
    delete r->of_q;
    delete r->of_scale;
    r->of_q = of_q.release(), r->of_scale = of_scale.release();
    Py_RETURN_NONE;
}

// originals(rows): (q, scale) that the rows follow, or None where they follow none, or nobody holds both any more; changed(rows)
PyObject* originals(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Rows* r;
    if (!count_is(n, 1) || !(r = rows_of(a[0]))) return nullptr;
    if (!r->of_q) Py_RETURN_NONE;
    auto q = r->of_q->t.lock(), s = r->of_scale->t.lock();
    if (!q || !s) Py_RETURN_NONE;
    return Py_BuildValue("NN", THPVariable_Wrap(at::Tensor(std::move(q))), THPVariable_Wrap(at::Tensor(std::move(s))));
}
PyObject* changed(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Rows* r;
    if (!count_is(n, 1) || !(r = rows_of(a[0]))) return nullptr;
    return PyBool_FromLong(changed(r));
}

// quantize_rows(x, rows)
PyObject* quantize_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Rows* r;
    at::ScalarType type;
    int32_t dtype;
    Matrix x;
    Place p;
    if (!count_is(n, 2) || !(r = rows_of(a[1])) || !dtype_of(a[0], "x", &type, &dtype) || !matrix(a[0], r->rows, r->cols, type, "x", &x) || !rows_here(r, &p))
        return nullptr;
    return status(g_calls.quantize_rows(x.p, x.ld, dtype, r->rows, r->cols, p.q, p.ldq, p.scale, p.values, p.ldv, stream()), r);
}

// rmsnorm(x, weight, eps, rows, residual, h)
PyObject* rmsnorm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Rows* r;
    at::ScalarType type;
    int32_t dtype;
    Matrix x, res, h;
    Place p;
    float* w;
    if (!count_is(n, 6) || !(r = rows_of(a[3])) || !dtype_of(a[0], "x", &type, &dtype) || !matrix(a[0], r->rows, r->cols, type, "x", &x) ||
        !vector_or_none(a[1], r->cols, "weight", &w) || !matrix_or_none(a[4], r->rows, r->cols, type, "residual", &res) ||
        !matrix_or_none(a[5], r->rows, r->cols, type, "h", &h) || !rows_here(r, &p))
        return nullptr;
    const double eps = PyFloat_AsDouble(a[2]);
    if (eps == -1.0 && PyErr_Occurred()) return nullptr;
    const dnns_status s = g_calls.rmsnorm_quantize(x.p, x.ld, res.p, res.ld, w, (float)eps, dtype, r->rows, r->cols, h.p, h.ld, p.q, p.ldq, p.scale, p.values,
                                                   p.ldv, stream());
    if (s == DNNS_OK) wrote(h.t);
    return status(s, r);
}

// rmsnorm_backward(dy, h, weight, eps, dx, dweight, dh, workspace)
PyObject* rmsnorm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    at::ScalarType type;
    int32_t dtype;
    if (!count_is(n, 8) || !dtype_of(a[1], "h", &type, &dtype)) return nullptr;
    const int64_t rows = tensor_of(a[1])->size(0), cols = tensor_of(a[1])->size(1);
    Matrix dy, h, dx, dh;
    float *w, *dw;
    const at::Tensor* dw_t;
    if (!matrix(a[0], rows, cols, type, "dy", &dy) || !matrix(a[1], rows, cols, type, "h", &h) || !vector_or_none(a[2], cols, "weight", &w) ||
        !matrix(a[4], rows, cols, type, "dx", &dx) || !vector_or_none(a[5], cols, "dweight", &dw, &dw_t) || !matrix_or_none(a[6], rows, cols, type, "dh", &dh))
        return nullptr;
    void* ws = nullptr;
    size_t ws_bytes = 0;
    if (a[7] != Py_None) {
        const at::Tensor* t = tensor_of(a[7]);
        if (!t || !t->is_contiguous()) return refuse("workspace", "a contiguous tensor", a[7]), nullptr;
        if (!on_device(*t, "workspace")) return nullptr;
        ws = t->data_ptr(), ws_bytes = t->nbytes();
    }
    const double eps = PyFloat_AsDouble(a[3]);
    if (eps == -1.0 && PyErr_Occurred()) return nullptr;
    return status(g_calls.rmsnorm_backward(dy.p, dy.ld, h.p, h.ld, w, (float)eps, dh.p, dh.ld, dtype, rows, cols, dx.p, dx.ld, dw, ws, ws_bytes, stream()),
                  {dx.t, dw_t});
}

// silu_gate(gate, up, rows)
PyObject* silu_gate(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Rows* r;
    at::ScalarType type;
    int32_t dtype;
    Matrix g, u;
    Place p;
    if (!count_is(n, 3) || !(r = rows_of(a[2])) || !dtype_of(a[0], "gate", &type, &dtype) || !matrix(a[0], r->rows, r->cols, type, "gate", &g) ||
        !matrix(a[1], r->rows, r->cols, type, "up", &u) || !rows_here(r, &p))
        return nullptr;
    return status(g_calls.silu_gate_quantize(g.p, g.ld, u.p, u.ld, dtype, r->rows, r->cols, p.q, p.ldq, p.scale, p.values, p.ldv, stream()), r);
}

// silu_gate_backward(dy, gate, up, dgate, dup)
PyObject* silu_gate_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    at::ScalarType type;
    int32_t dtype;
    if (!count_is(n, 5) || !dtype_of(a[1], "gate", &type, &dtype)) return nullptr;
    const int64_t rows = tensor_of(a[1])->size(0), cols = tensor_of(a[1])->size(1);
    static const char* const names[] = {"dy", "gate", "up", "dgate", "dup"};
    Matrix m[5];
    for (int i = 0; i < 5; ++i)
        if (!matrix(a[i], rows, cols, type, names[i], &m[i])) return nullptr;
    return status(g_calls.silu_gate_backward(m[0].p, m[0].ld, m[1].p, m[1].ld, m[2].p, m[2].ld, dtype, rows, cols, m[3].p, m[3].ld, m[4].p, m[4].ld, stream()),
                  {m[3].t, m[4].t});
}

// linear(x rows, weight rows, bias or None, y, status address); -1, and nothing done, where the weights' originals were written
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Rows *x, *w;
    at::ScalarType type;
    int32_t dtype;
    Matrix y;
    Place xp, wp;
    float* bias;
    if (!count_is(n, 5) || !(x = rows_of(a[0])) || !(w = rows_of(a[1])) || !vector_or_none(a[2], w->rows, "bias", &bias) ||
        !dtype_of(a[3], "y", &type, &dtype) || !matrix(a[3], x->rows, w->rows, type, "y", &y) || !rows_here(x, &xp) || !rows_here(w, &wp))
        return nullptr;
    if (x->cols != w->cols) return PyErr_Format(PyExc_ValueError, "x has %lld columns, the layer %lld", (long long)x->cols, (long long)w->cols);
    if (changed(w)) return PyLong_FromLong(-1);
    uint32_t* where = static_cast<uint32_t*>(PyLong_AsVoidPtr(a[4]));
    if (!where && PyErr_Occurred()) return nullptr;
    return status(g_calls.linear_quantized(xp.q, xp.ldq, xp.scale, wp.q, wp.ldq, wp.scale, bias, x->rows, x->cols, w->rows, dtype, y.p, y.ld, where, stream()),
                  {y.t});
}

// torch reports by exceptions (no device, a tensor without storage): they end here
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    g_device = -1;
    try {
        return F(self, a, n);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown error");
    }
    return nullptr;
}
#define DNNS_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<name>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {DNNS_METHOD(bind),      DNNS_METHOD(rows),      DNNS_METHOD(laid_out), DNNS_METHOD(originals), DNNS_METHOD(changed), DNNS_METHOD(quantize_rows),      DNNS_METHOD(rmsnorm), DNNS_METHOD(rmsnorm_backward),
                         DNNS_METHOD(silu_gate), DNNS_METHOD(silu_gate_backward), DNNS_METHOD(linear), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", "Calls on rows in 8 bits from torch tensors.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__native() {
    RowsType.tp_name = "_native.Rows";
    RowsType.tp_basicsize = sizeof(Rows);
    RowsType.tp_flags = Py_TPFLAGS_DEFAULT;
    RowsType.tp_dealloc = rows_dealloc;
    if (PyType_Ready(&RowsType) < 0) return nullptr;
    return PyModule_Create(&module);
}
