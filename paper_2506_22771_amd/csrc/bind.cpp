// Python's side of the calls on matrices of floating-point values (norms, checkpoints, gated layers, dropout): shapes, types, strides and devices of the tensors are compared here (all lie on the current
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

// An int8 matrix as the library's quantiser writes it.
const void* codes(PyObject* o, const char* what, int64_t rows, int64_t pitch)
{
    const at::Tensor& t = tensor(o, what);
    if (t.scalar_type() != at::kChar || t.dim() != 2 || t.size(0) != rows || t.size(1) != pitch || !t.is_contiguous()) refuse(what, "contiguous int8", rows, pitch);
    on_device(t, what);
    return t.data_ptr();
}
const float* scalar(PyObject* o, const char* what)
{
    const at::Tensor& t = tensor(o, what);
    if (t.scalar_type() != at::kFloat || t.numel() != 1) refuse(what, "one float32");
    on_device(t, what);
    return (const float*)t.data_ptr();
}
float* table(PyObject* o, const char* what, int64_t rows, int64_t cols)
{
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o, what);
    if (t.scalar_type() != at::kFloat || t.dim() != 2 || t.size(0) != rows || t.size(1) != cols || !t.is_contiguous()) refuse(what, "contiguous float32", rows, cols);
    on_device(t, what);
    return (float*)t.data_ptr();
}
const uint64_t* step(PyObject* o)   // a step number in device memory
{
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o, "step");
    if (t.scalar_type() != at::kLong || t.numel() != 1) refuse("step", "one int64");
    on_device(t, "step");
    return (const uint64_t*)t.data_ptr();
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

PyObject* gated_forward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return call<14>(args, n, [](PyObject* const* a) {
        const Mat y = matrix(a[6], "y");
        const int64_t k = whole(a[4]), pitch = ff_pitch(k);
        const void *aq = codes(a[0], "a_q", y.rows, pitch), *wq = codes(a[1], "w_q", 2 * y.cols, pitch);
        const Ckpt g = checkpoint(a[8], a[9], y.rows, y.cols), u = checkpoint(a[10], a[11], y.rows, y.cols);
        const Bytes ws = workspace(a[12]);
        return ff_gated_forward(y.rows, y.cols, k, (const int8_t*)aq, (const int8_t*)wq, scalar(a[2], "s_a"), scalar(a[3], "s_w"), small(a[5]), y.p, y.kind, y.ld,
                                floats(a[7], "goodness", y.rows), g.q, g.e, u.q, u.e, ws.p, ws.n, address(a[13]));
    });
}

PyObject* gated_backward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return call<10>(args, n, [](PyObject* const* a) {
        const Mat dg = matrix(a[7], "dg"), du = matrix_like(a[8], "du", dg), dy = maybe_matrix_like(a[6], "dy", dg);
        const Ckpt g = checkpoint(a[0], a[1], dg.rows, dg.cols), u = checkpoint(a[2], a[3], dg.rows, dg.cols);
        return ff_gated_backward(g.q, g.e, u.q, u.e, dg.rows, dg.cols, small(a[4]), floats(a[5], "coeff", dg.rows), dy.p, dy.ld, dg.p, dg.ld, du.p, du.ld, dg.kind,
                                 address(a[9]));
    });
}

// Pixels of a sample, of a map of so many rows.
int64_t pixels_of(int64_t rows, int64_t samples, int64_t least = 1)
{
    if (samples < 0 || (samples == 0 ? rows != 0 : rows % samples != 0)) {
        PyErr_Format(PyExc_ValueError, "samples: a number of equal parts of %lld rows expected", (long long)rows);
        throw Refused();
    }
    return samples == 0 ? least : rows / samples;
}

PyObject* group_norm_forward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return call<18>(args, n, [](PyObject* const* a) {
        const Mat x = matrix(a[0], "x"), y = matrix_like(a[7], "y", x);
        const int64_t samples = whole(a[1]), groups = whole(a[2]), pixels = pixels_of(x.rows, samples);
        const Params p = params(a[3], a[4], "weight", "bias", x.cols, x.type);
        const Ckpt c = checkpoint(a[11], a[12], x.rows, x.cols);
        const Bytes ws = workspace(a[16]);
        return ff_group_norm_forward(samples, pixels, x.cols, groups, x.kind, p.kind, x.p, x.ld, p.a, p.b, real(a[5]), small(a[6]), y.p, y.ld,
                                     table(a[8], "mean", samples, groups), table(a[9], "rstd", samples, groups), floats(a[10], "goodness", samples), c.q, c.e,
                                     small(a[13]), word(a[14]), word(a[15]), ws.p, ws.n, address(a[17]));
    });
}

PyObject* group_norm_backward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return call<18>(args, n, [](PyObject* const* a) {
        PyObject* const first = a[0] != Py_None ? a[0] : a[2] != Py_None ? a[2] : a[12];   // dy, x or dx
        if (first == Py_None) refuse("dy, x or dx", "a matrix");
        const Mat like = matrix(first, a[0] != Py_None ? "dy" : a[2] != Py_None ? "x" : "dx");
        const Mat dy = maybe_matrix_like(a[0], "dy", like), x = maybe_matrix_like(a[2], "x", like), dx = maybe_matrix_like(a[12], "dx", like);
        const int64_t samples = whole(a[7]), groups = whole(a[8]), pixels = pixels_of(like.rows, samples);
        const Ckpt c = checkpoint(a[4], a[5], like.rows, like.cols);
        const Params p = params(a[9], a[10], "weight", "bias", like.cols, like.type);
        const Bytes ws = workspace(a[16]);
        return ff_group_norm_backward(samples, pixels, like.cols, groups, like.kind, p.kind, dy.p, dy.ld, floats(a[1], "coeff", samples), x.p, x.ld,
                                      table(a[3], "mean", samples, groups), c.q, c.e, table(a[6], "rstd", samples, groups), p.a, p.b, small(a[11]), dx.p, dx.ld,
                                      floats(a[13], "dweight", like.cols), floats(a[14], "dbias", like.cols), truth(a[15]), ws.p, ws.n, address(a[17]));
    });
}

PyObject* dropout(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return call<8>(args, n, [](PyObject* const* a) {
        const Mat x = matrix(a[0], "x"), r = maybe_matrix_like(a[1], "r", x), y = matrix_like(a[6], "y", x);
        return ff_dropout(x.rows, x.cols, x.kind, x.p, x.ld, r.p, r.ld, real(a[2]), word(a[3]), word(a[4]), step(a[5]), y.p, y.ld, address(a[7]));
    });
}

#define METHOD(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(layer_norm_forward), METHOD(layer_norm_backward), METHOD(ckpt_store), METHOD(ckpt_load),
                         METHOD(ckpt_act_backward),  METHOD(ckpt_weight_grad),    METHOD(gated_forward),
                         METHOD(gated_backward),     METHOD(group_norm_forward),  METHOD(group_norm_backward), METHOD(dropout), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__bind(void) { return PyModule_Create(&module); }
