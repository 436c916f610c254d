// Python's side of the layer norm and checkpoint calls: shapes, types, strides and devices of the tensors are compared here (all lie on the current
// device, whose stream the work goes to) and their addresses handed to the library.  Marshalling only, in C++ because these calls are short: a norm of one 4096-wide row took 8.3 us through
// ctypes, nearly all of it spent on attributes and argument conversions in Python.
//
// Tensors of the wrong shape, type, stride or device raise ValueError; the library's own refusals come back as its status.
#include <Python.h>

#include <c10/core/impl/DeviceGuardImplInterface.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>

#include "../../include/ffint8.h"

namespace {

struct Refused {};   // a Python error is set

[[noreturn]] void refuse(const char* what, const char* expected, int64_t a = -1, int64_t b = -1)
{
    if (b >= 0) PyErr_Format(PyExc_ValueError, "%s: %s [%lld, %lld] expected", what, expected, (long long)a, (long long)b);
    else if (a >= 0) PyErr_Format(PyExc_ValueError, "%s: %s [%lld] expected", what, expected, (long long)a);
    else PyErr_Format(PyExc_ValueError, "%s: %s expected", what, expected);
    throw Refused();
}
const char* name_of(at::ScalarType t)
{
    return t == at::kFloat ? "float32" : t == at::kBFloat16 ? "bfloat16" : t == at::kHalf ? "float16" : t == at::kChar ? "int8" : "uint8";
}

const at::Tensor& tensor(PyObject* o, const char* what)
{
    if (!THPVariable_Check(o)) refuse(what, "a tensor");
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.layout() != at::kStrided) refuse(what, "a dense tensor");   // (others have no address)
    return t;
}
void on_device(const at::Tensor& t, const char* what)
{
    if (!t.is_cuda()) refuse(what, "device tensor");
}
// Of all arguments that are device tensors.  (What else there is among them is refused by its own name.)
void one_device(PyObject* const* a, int n)
{
    int first = -1;
    for (int i = 0; i < n; ++i) {
        if (!THPVariable_Check(a[i])) continue;
        const at::Device d = THPVariable_Unpack(a[i]).device();
        if (!d.is_cuda()) continue;
        if (first >= 0 && d.index() != first) {
            PyErr_Format(PyExc_ValueError, "tensors on one device expected, got cuda:%d and cuda:%d", first, (int)d.index());
            throw Refused();
        }
        first = d.index();
    }
    if (first < 0) return;
    const int current = c10::impl::getDeviceGuardImpl(c10::DeviceType::CUDA)->getDevice().index();
    if (first != current) {
        PyErr_Format(PyExc_ValueError, "tensors on the current device, cuda:%d, expected, got cuda:%d", current, first);
        throw Refused();
    }
}

int32_t kind_of(at::ScalarType t) { return t == at::kFloat ? FF_F32 : t == at::kBFloat16 ? FF_BF16 : t == at::kHalf ? FF_F16 : -1; }

struct Mat {
    void* p = nullptr;
    int64_t ld = 0, rows = 0, cols = 0;
    at::ScalarType type = at::kFloat;
    int32_t kind = 0;
};
// A matrix of float32, bfloat16 or float16 with consecutive columns; any row stride that keeps rows apart.
Mat matrix(PyObject* o, const char* what)
{
    const at::Tensor& t = tensor(o, what);
    Mat m;
    m.type = t.scalar_type();
    m.kind = kind_of(m.type);
    if (t.dim() != 2 || m.kind < 0) refuse(what, "a float32, bfloat16 or float16 matrix");
    m.rows = t.size(0);
    m.cols = t.size(1);
    on_device(t, what);
    m.ld = m.rows <= 1 ? m.cols : t.stride(0);   // (of one row it says nothing)
    if ((t.stride(1) != 1 && m.cols > 1) || m.ld < m.cols) refuse(what, "consecutive columns and rows that do not overlap, as a matrix", m.rows, m.cols);
    m.p = t.data_ptr();
    return m;
}
Mat matrix_like(PyObject* o, const char* what, const Mat& as)
{
    const at::Tensor& t = tensor(o, what);
    if (t.dim() != 2 || t.size(0) != as.rows || t.size(1) != as.cols || t.scalar_type() != as.type) refuse(what, name_of(as.type), as.rows, as.cols);
    return matrix(o, what);
}
Mat maybe_matrix_like(PyObject* o, const char* what, const Mat& as) { return o == Py_None ? Mat() : matrix_like(o, what, as); }

void* vector(PyObject* o, const char* what, int64_t n, at::ScalarType type)
{
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o, what);
    if (t.scalar_type() != type || t.dim() != 1 || t.size(0) != n) refuse(what, name_of(type), n);
    if (n > 1 && t.stride(0) != 1) refuse(what, "contiguous tensor");
    on_device(t, what);
    return t.data_ptr();
}
float* floats(PyObject* o, const char* what, int64_t n) { return (float*)vector(o, what, n, at::kFloat); }

// A pair of parameter vectors, float32 or of the matrix's type, both the same.
struct Params {
    void *a = nullptr, *b = nullptr;
    int32_t kind = FF_F32;
};
Params params(PyObject* a, PyObject* b, const char* what_a, const char* what_b, int64_t n, at::ScalarType type)
{
    Params p;
    PyObject* const first = a != Py_None ? a : b;
    if (first == Py_None) return p;
    const at::ScalarType of = tensor(first, what_a).scalar_type();
    if (of != at::kFloat && of != type) refuse(what_a, name_of(type));
    p.a = vector(a, what_a, n, of);
    p.b = vector(b, what_b, n, of);
    p.kind = kind_of(of);
    return p;
}

struct Ckpt {
    int8_t* q = nullptr;
    uint8_t* e = nullptr;
};
Ckpt checkpoint(PyObject* q, PyObject* e, int64_t rows, int64_t cols)
{
    Ckpt c;
    if (q == Py_None && e == Py_None) return c;
    if (q == Py_None || e == Py_None) refuse("checkpoint", "both codes and exponent bytes");
    const at::Tensor &tq = tensor(q, "codes"), &te = tensor(e, "exponent bytes");
    const int64_t pq = ff_pitch(cols), pe = ff_pitch(ff_ckpt_blocks(cols));
    if (tq.scalar_type() != at::kChar || tq.dim() != 2 || tq.size(0) != rows || tq.size(1) != pq || !tq.is_contiguous()) refuse("codes", "contiguous int8", rows, pq);
    if (te.scalar_type() != at::kByte || te.dim() != 2 || te.size(0) != rows || te.size(1) != pe || !te.is_contiguous()) refuse("exponent bytes", "contiguous uint8", rows, pe);
    on_device(tq, "codes");
    on_device(te, "exponent bytes");
    c.q = (int8_t*)tq.data_ptr();
    c.e = (uint8_t*)te.data_ptr();
    return c;
}

struct Bytes {
    void* p = nullptr;
    size_t n = 0;
};
Bytes workspace(PyObject* o)
{
    if (o == Py_None) return {};
    const at::Tensor& t = tensor(o, "ws");
    if (!t.is_contiguous()) refuse("ws", "contiguous tensor");
    on_device(t, "ws");
    return {t.data_ptr(), (size_t)t.nbytes()};
}

// Numbers.
int64_t whole(PyObject* o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused();
    return v;
}
uint64_t word(PyObject* o)   // modulo 2^64, as seeds and tags are
{
    const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
    if (v == (unsigned long long)-1 && PyErr_Occurred()) throw Refused();
    return v;
}
int32_t small(PyObject* o)
{
    const int64_t v = whole(o);
    return v < INT32_MIN ? INT32_MIN : v > INT32_MAX ? INT32_MAX : (int32_t)v;
}
float real(PyObject* o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused();
    return (float)v;
}
int32_t truth(PyObject* o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Refused();
    return v;
}
void* address(PyObject* o) { return (void*)(uintptr_t)word(o); }

// f(args) as a status, or the Python error that was set; C++ exceptions of the tensor library become errors too.
template <int N, typename F> PyObject* call(PyObject* const* a, Py_ssize_t n, F&& f)
{
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "%d arguments expected, got %zd", N, n);
        return nullptr;
    }
    try {
        one_device(a, N);
        return PyLong_FromLong(f(a));
    } catch (const Refused&) {
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
        return nullptr;
    }
}

PyObject* layer_norm_forward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return call<13>(args, n, [](PyObject* const* a) {
        const Mat x = matrix(a[0], "x"), y = matrix_like(a[4], "y", x);
        const Params p = params(a[1], a[2], "weight", "bias", x.cols, x.type);
        const Ckpt c = checkpoint(a[7], a[8], x.rows, x.cols);
        return ff_layer_norm_forward(x.rows, x.cols, x.kind, p.kind, x.p, x.ld, p.a, p.b, real(a[3]), y.p, y.ld, floats(a[5], "mean", x.rows),
                                     floats(a[6], "rstd", x.rows), c.q, c.e, small(a[9]), word(a[10]), word(a[11]), address(a[12]));
    });
}

PyObject* layer_norm_backward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return call<13>(args, n, [](PyObject* const* a) {
        const Mat dy = matrix(a[0], "dy"), x = maybe_matrix_like(a[1], "x", dy), dx = maybe_matrix_like(a[7], "dx", dy);
        const Ckpt c = checkpoint(a[3], a[4], dy.rows, dy.cols);
        const Params p = params(a[6], Py_None, "weight", "", dy.cols, dy.type);
        const Bytes ws = workspace(a[11]);
        return ff_layer_norm_backward(dy.rows, dy.cols, dy.kind, p.kind, dy.p, dy.ld, x.p, x.ld, floats(a[2], "mean", dy.rows), c.q, c.e,
                                      floats(a[5], "rstd", dy.rows), p.a, dx.p, dx.ld, floats(a[8], "dweight", dy.cols),
                                      floats(a[9], "dbias", dy.cols), truth(a[10]), ws.p, ws.n, address(a[12]));
    });
}

PyObject* ckpt_store(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return call<7>(args, n, [](PyObject* const* a) {
        const Mat x = matrix(a[0], "x");
        const Ckpt c = checkpoint(a[4], a[5], x.rows, x.cols);
        return ff_ckpt_store(x.p, x.kind, x.ld, x.rows, x.cols, small(a[1]), word(a[2]), word(a[3]), c.q, c.e, address(a[6]));
    });
}

PyObject* ckpt_load(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return call<4>(args, n, [](PyObject* const* a) {
        const Mat x = matrix(a[2], "x");
        const Ckpt c = checkpoint(a[0], a[1], x.rows, x.cols);
        return ff_ckpt_load(c.q, c.e, x.rows, x.cols, x.p, x.kind, x.ld, address(a[3]));
    });
}

PyObject* ckpt_act_backward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return call<7>(args, n, [](PyObject* const* a) {
        const Mat dx = matrix(a[5], "dx"), dy = maybe_matrix_like(a[4], "dy", dx);
        const Ckpt c = checkpoint(a[0], a[1], dx.rows, dx.cols);
        return ff_ckpt_act_backward(c.q, c.e, dx.rows, dx.cols, small(a[2]), floats(a[3], "coeff", dx.rows), dy.p, dy.ld, dx.p, dx.ld, dx.kind,
                                    address(a[6]));
    });
}

PyObject* ckpt_weight_grad(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return call<10>(args, n, [](PyObject* const* a) {
        const Mat dy = matrix(a[0], "dy");
        const at::Tensor& dw = tensor(a[5], "dw");
        if (dw.dim() != 2 || dw.size(0) != dy.cols || dw.scalar_type() != at::kFloat || !dw.is_contiguous()) refuse("dw", "contiguous float32", dy.cols, dw.dim() == 2 ? dw.size(1) : -1);
        on_device(dw, "dw");
        const int64_t k = dw.size(1);
        const Ckpt c = checkpoint(a[1], a[2], dy.rows, k);
        const Params p = params(a[3], a[4], "gamma", "beta", k, dy.type);
        const Bytes ws = workspace(a[8]);
        return ff_ckpt_weight_grad(dy.p, dy.kind, dy.ld, c.q, c.e, dy.rows, dy.cols, k, p.a, p.b, p.kind, (float*)dw.data_ptr(),
                                   floats(a[6], "db", dy.cols), truth(a[7]), ws.p, ws.n, address(a[9]));
    });
}

#define METHOD(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(layer_norm_forward), METHOD(layer_norm_backward), METHOD(ckpt_store), METHOD(ckpt_load),
                         METHOD(ckpt_act_backward),  METHOD(ckpt_weight_grad),    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__bind(void) { return PyModule_Create(&module); }
