// CPython front of the calls that a program issues once per operator: turns addresses and handles into the C ABI's arguments
// without a foreign-function layer in between (a call on a mini-batch costs about as much in Python as in the library:
// marshalling through ctypes took 1.1 us of the 4.1 us of a small Apply, here it takes 0.4).
//
// Every function takes plain integers (addresses of the ctypes structures that binding.py owns, table handles, device
// pointers; 0 or None = NULL), contiguous buffers of the stated item size where the ABI takes a host array, and the stream
// last: an integer handle, or None for torch's current stream.  Matrices and activations come as tuples of their structure's
// fields, in its order.  A status other than DOL_OK goes to the error callback set
// with setup(), whose exception leaves the call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cstdint>
#include <initializer_list>
#include <utility>

#include "dolphin_hip.h"

namespace {

PyObject *g_fail = nullptr, *g_device = nullptr, *g_stream = nullptr;

PyObject *done(dol_status st)
{
    if (st == DOL_OK) Py_RETURN_NONE;
    PyObject *code = PyLong_FromLong(st);
    PyObject *r = code ? PyObject_CallOneArg(g_fail, code) : nullptr;
    Py_XDECREF(code);
    return r;                               // (the callback raises)
}

// One call's arguments; `bad` once something did not convert (a Python error is set then).
struct Args {
    PyObject *const *v;
    bool bad = false;

    Args(PyObject *const *args, Py_ssize_t n, Py_ssize_t want) : v(args)
    {
        if (n != want) {
            PyErr_Format(PyExc_TypeError, "%zd arguments, %zd wanted", n, want);
            bad = true;
        }
    }
    template <typename T>
    T *ptr(int k)
    {
        if (bad || v[k] == Py_None) return nullptr;
        void *p = PyLong_AsVoidPtr(v[k]);
        if (!p && PyErr_Occurred()) bad = true;
        return static_cast<T *>(p);
    }
    int64_t num(int k)
    {
        if (bad) return 0;
        const long long x = PyLong_AsLongLong(v[k]);
        if (x == -1 && PyErr_Occurred()) bad = true;
        return x;
    }
    int32_t num32(int k)
    {
        const int64_t x = num(k);
        if (!bad && x != static_cast<int32_t>(x)) {
            PyErr_Format(PyExc_OverflowError, "argument %d: past 32 bits", k);
            bad = true;
        }
        return static_cast<int32_t>(x);
    }
    double real(int k)
    {
        if (bad) return 0.0;
        const double x = PyFloat_AsDouble(v[k]);
        if (x == -1.0 && PyErr_Occurred()) bad = true;
        return x;
    }
    void *stream(int k)
    {
        if (bad) return nullptr;
        if (v[k] != Py_None) return ptr<void>(k);
        PyObject *dev = PyObject_CallNoArgs(g_device);
        PyObject *raw = dev ? PyObject_CallOneArg(g_stream, dev) : nullptr;
        Py_XDECREF(dev);
        void *p = raw ? PyLong_AsVoidPtr(raw) : nullptr;
        if (!raw || (!p && PyErr_Occurred())) bad = true;
        Py_XDECREF(raw);
        return p;
    }
};

// A contiguous host array for the time of a call.
struct Buffer {
    Py_buffer b{};
    bool held = false;

    Buffer(Args &a, int k)
    {
        if (a.bad) return;
        if (PyObject_GetBuffer(a.v[k], &b, PyBUF_SIMPLE) == 0) held = true;
        else a.bad = true;
    }
    ~Buffer()
    {
        if (held) PyBuffer_Release(&b);
    }
    template <typename T>
    const T *data() const { return static_cast<const T *>(b.buf); }
};

#define DOL_CALL(expr)                \
    if (a.bad) return nullptr;        \
    dol_status st;                    \
    Py_BEGIN_ALLOW_THREADS            \
    st = (expr);                      \
    Py_END_ALLOW_THREADS              \
    return done(st)

PyObject *apply2(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 6);
    auto *x = a.ptr<dol_dist>(0), *y = a.ptr<dol_dist>(1);
    auto *f = a.ptr<dol_fn_table>(2);
    auto *p = a.ptr<dol_prov>(3);
    auto *o = a.ptr<dol_dist>(4);
    void *s = a.stream(5);
    DOL_CALL(dol_apply2(x, y, f, p, o, s));
}

PyObject *backward(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 5);
    auto *r = a.ptr<dol_op_record>(0);
    auto *g = a.ptr<float>(1), *ga = a.ptr<float>(2), *gb = a.ptr<float>(3);
    void *s = a.stream(4);
    DOL_CALL(dol_backward(r, g, ga, gb, s));
}

PyObject *filter(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 5);
    auto *d = a.ptr<dol_dist>(0);
    Buffer pred(a, 1);
    auto *p = a.ptr<dol_prov>(2);
    auto *o = a.ptr<dol_dist>(3);
    void *s = a.stream(4);
    DOL_CALL(dol_filter(d, pred.data<uint8_t>(), p, o, s));
}

PyObject *union_(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 5);
    auto *x = a.ptr<dol_dist>(0), *y = a.ptr<dol_dist>(1);
    auto *p = a.ptr<dol_prov>(2);
    auto *o = a.ptr<dol_dist>(3);
    void *s = a.stream(4);
    DOL_CALL(dol_union(x, y, p, o, s));
}

PyObject *nll_grad(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 4);
    auto *d = a.ptr<dol_dist>(0);
    auto *t = a.ptr<int32_t>(1);
    auto *g = a.ptr<float>(2);
    void *s = a.stream(3);
    DOL_CALL(dol_nll_grad(d, t, g, s));
}

PyObject *dtkp_init(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 4);
    auto *d = a.ptr<dol_dist>(0);
    Buffer facts(a, 1);
    auto *p = a.ptr<dol_prov>(2);
    void *s = a.stream(3);
    DOL_CALL(dol_dtkp_init(d, facts.data<int32_t>(), p, s));
}

PyObject *dtkp_apply2_input(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 6);
    auto *x = a.ptr<dol_dist>(0);
    Buffer facts(a, 1);
    auto *f = a.ptr<dol_fn_table>(2);
    auto *p = a.ptr<dol_prov>(3);
    auto *o = a.ptr<dol_dist>(4);
    void *s = a.stream(5);
    DOL_CALL(dol_dtkp_apply2_input(x, facts.data<int32_t>(), f, p, o, s));
}

PyObject *dtkp_backward(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 6);
    auto *d = a.ptr<dol_dist>(0);
    auto *p = a.ptr<dol_prov>(1);
    auto *g = a.ptr<float>(2);
    const int64_t ld = a.num(3);
    auto *gf = a.ptr<float>(4);
    void *s = a.stream(5);
    DOL_CALL(dol_dtkp_backward(d, p, g, ld, gf, s));
}

PyObject *fold_apply2(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 2);
    auto *f = a.ptr<dol_fold>(0);
    void *s = a.stream(1);
    DOL_CALL(dol_fold_apply2(f, s));
}

PyObject *dtkp_fold_apply2(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 3);
    auto *f = a.ptr<dol_dtkp_fold>(0);
    auto *p = a.ptr<dol_prov>(1);
    void *s = a.stream(2);
    DOL_CALL(dol_dtkp_fold_apply2(f, p, s));
}

// A structure of the ABI from the tuple of its n fields, the first `narrow` of them of 32 bits; None = NULL.
bool fields(Args &a, int k, int64_t *to, int n, int narrow)
{
    if (a.bad || a.v[k] == Py_None) return false;
    if (!PyTuple_Check(a.v[k]) || PyTuple_GET_SIZE(a.v[k]) != n) {
        PyErr_Format(PyExc_TypeError, "argument %d: a tuple of %d fields wanted", k, n);
        a.bad = true;
        return false;
    }
    for (int f = 0; f < n && !a.bad; ++f) {
        PyObject *o = PyTuple_GET_ITEM(a.v[k], f);
        to[f] = f == n - 1 ? reinterpret_cast<intptr_t>(PyLong_AsVoidPtr(o)) : PyLong_AsLongLong(o);     // (the address is the last)
        if (f < narrow && to[f] != static_cast<int32_t>(to[f]) && !PyErr_Occurred()) PyErr_Format(PyExc_OverflowError, "argument %d, field %d: past 32 bits", k, f);
        if (PyErr_Occurred()) a.bad = true;
    }
    return !a.bad;
}

struct Matrix {
    dol_matrix m{};
    const bool given;

    Matrix(Args &a, int k) : given(read(a, k)) {}
    const dol_matrix *p() const { return given ? &m : nullptr; }

private:
    bool read(Args &a, int k)
    {
        int64_t f[5];
        if (!fields(a, k, f, 5, 3)) return false;
        m = dol_matrix{static_cast<int32_t>(f[0]), static_cast<int32_t>(f[1]), static_cast<int32_t>(f[2]), f[3], reinterpret_cast<void *>(f[4])};
        return true;
    }
};

struct Activations {
    dol_activations m{};
    const bool given;

    Activations(Args &a, int k) : given(read(a, k)) {}
    const dol_activations *p() const { return given ? &m : nullptr; }

private:
    bool read(Args &a, int k)
    {
        int64_t f[7];
        if (!fields(a, k, f, 7, 4)) return false;
        m = dol_activations{static_cast<int32_t>(f[0]), static_cast<int32_t>(f[1]), static_cast<int32_t>(f[2]), static_cast<int32_t>(f[3]), f[4], f[5],
                            reinterpret_cast<void *>(f[6])};
        return true;
    }
};

PyObject *bytes(dol_status st, int64_t n) { return st == DOL_OK ? PyLong_FromLongLong(n) : done(st); }

PyObject *cross_entropy_workspace(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 3);
    Matrix x(a, 0), w(a, 1);
    const int32_t back = a.num32(2);
    if (a.bad) return nullptr;
    int64_t need = 0;
    const dol_status st = dol_cross_entropy_workspace(x.p(), w.p(), back, &need);
    return bytes(st, need);
}

PyObject *cross_entropy_kernel(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 3);
    Matrix x(a, 0), w(a, 1);
    const int32_t back = a.num32(2);
    return a.bad ? nullptr : PyUnicode_FromString(dol_cross_entropy_kernel(x.p(), w.p(), back));
}

PyObject *cross_entropy(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 9);
    Matrix x(a, 0), w(a, 1);
    auto *b = a.ptr<float>(2);
    auto *t = a.ptr<int32_t>(3);
    auto *loss = a.ptr<float>(4), *lse = a.ptr<float>(5);
    auto *ws = a.ptr<void>(6);
    const int64_t have = a.num(7);
    void *s = a.stream(8);
    DOL_CALL(dol_cross_entropy(x.p(), w.p(), b, t, loss, lse, ws, have, s));
}

PyObject *cross_entropy_backward(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 12);
    Matrix x(a, 0), w(a, 1), gx(a, 6), gw(a, 7);
    auto *b = a.ptr<float>(2);
    auto *t = a.ptr<int32_t>(3);
    auto *lse = a.ptr<float>(4), *g = a.ptr<float>(5), *gb = a.ptr<float>(8);
    auto *ws = a.ptr<void>(9);
    const int64_t have = a.num(10);
    void *s = a.stream(11);
    DOL_CALL(dol_cross_entropy_backward(x.p(), w.p(), b, t, lse, g, gx.p(), gw.p(), gb, ws, have, s));
}

PyObject *group_norm_workspace(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 3);
    Activations x(a, 0);
    const int32_t groups = a.num32(1), back = a.num32(2);
    if (a.bad) return nullptr;
    int64_t need = 0;
    const dol_status st = dol_group_norm_workspace(x.p(), groups, back, &need);
    return bytes(st, need);
}

PyObject *group_norm(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 12);
    Activations x(a, 0), y(a, 6);
    const int32_t groups = a.num32(1), act = a.num32(5);
    auto *gamma = a.ptr<float>(2), *beta = a.ptr<float>(3);
    const float eps = static_cast<float>(a.real(4));
    auto *mean = a.ptr<float>(7), *rstd = a.ptr<float>(8);
    auto *ws = a.ptr<void>(9);
    const int64_t have = a.num(10);
    void *s = a.stream(11);
    DOL_CALL(dol_group_norm(x.p(), groups, gamma, beta, eps, act, y.p(), mean, rstd, ws, have, s));
}

PyObject *group_norm_backward(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 14);
    Activations x(a, 0), gy(a, 7), gx(a, 8);
    const int32_t groups = a.num32(1), act = a.num32(4);
    auto *gamma = a.ptr<float>(2), *beta = a.ptr<float>(3);
    auto *mean = a.ptr<float>(5), *rstd = a.ptr<float>(6);
    auto *gg = a.ptr<float>(9), *gb = a.ptr<float>(10);
    auto *ws = a.ptr<void>(11);
    const int64_t have = a.num(12);
    void *s = a.stream(13);
    DOL_CALL(dol_group_norm_backward(x.p(), groups, gamma, beta, act, mean, rstd, gy.p(), gx.p(), gg, gb, ws, have, s));
}

PyObject *newton_schulz_workspace(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 2);
    Matrix g(a, 0);
    const int32_t batch = a.num32(1);
    if (a.bad) return nullptr;
    int64_t need = 0;
    const dol_status st = dol_newton_schulz_workspace(g.p(), batch, &need);
    return bytes(st, need);
}

PyObject *newton_schulz_kernel(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 2);
    Matrix g(a, 0);
    const int32_t batch = a.num32(1);
    return a.bad ? nullptr : PyUnicode_FromString(dol_newton_schulz_kernel(g.p(), batch));
}

PyObject *newton_schulz(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 13);
    Matrix g(a, 0), o(a, 2);
    const int64_t g_stride = a.num(1), o_stride = a.num(3);
    const int32_t batch = a.num32(4), steps = a.num32(5);
    const float abc[3] = {static_cast<float>(a.real(6)), static_cast<float>(a.real(7)), static_cast<float>(a.real(8))};
    const float eps = static_cast<float>(a.real(9));
    auto *ws = a.ptr<void>(10);
    const int64_t have = a.num(11);
    void *s = a.stream(12);
    DOL_CALL(dol_newton_schulz(g.p(), g_stride, o.p(), o_stride, batch, steps, abc, eps, ws, have, s));
}

PyObject *linear_workspace(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 3);
    Matrix x(a, 0), w(a, 1);
    const int32_t back = a.num32(2);
    if (a.bad) return nullptr;
    int64_t need = 0;
    const dol_status st = dol_linear_workspace(x.p(), w.p(), back, &need);
    return bytes(st, need);
}

PyObject *linear_kernel(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 3);
    Matrix x(a, 0), w(a, 1);
    const int32_t back = a.num32(2);
    return a.bad ? nullptr : PyUnicode_FromString(dol_linear_kernel(x.p(), w.p(), back));
}

PyObject *linear(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 11);
    Matrix x(a, 0), w(a, 1), res(a, 4), y(a, 5), z(a, 6);
    auto *b = a.ptr<float>(2);
    const int32_t act = a.num32(3);
    auto *rest = a.ptr<int16_t>(7);
    auto *ws = a.ptr<void>(8);
    const int64_t have = a.num(9);
    void *s = a.stream(10);
    DOL_CALL(dol_linear(x.p(), w.p(), b, act, res.p(), y.p(), z.p(), rest, ws, have, s));
}

PyObject *linear_backward(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 12);
    Matrix x(a, 0), w(a, 1), z(a, 3), gy(a, 5), gx(a, 6), gw(a, 7);
    const int32_t act = a.num32(2);
    auto *rest = a.ptr<int16_t>(4);
    auto *gb = a.ptr<float>(8);
    auto *ws = a.ptr<void>(9);
    const int64_t have = a.num(10);
    void *s = a.stream(11);
    DOL_CALL(dol_linear_backward(x.p(), w.p(), act, z.p(), rest, gy.p(), gx.p(), gw.p(), gb, ws, have, s));
}

PyObject *residual_norm(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 13);
    Matrix x(a, 0), u(a, 1), gate(a, 4), h(a, 8), y(a, 9);
    const int32_t norm_u = a.num32(2);
    auto *gamma_u = a.ptr<float>(3), *gamma_y = a.ptr<float>(6);
    const float scale = static_cast<float>(a.real(5)), eps = static_cast<float>(a.real(7));
    auto *rstd_u = a.ptr<float>(10), *rstd_h = a.ptr<float>(11);
    void *s = a.stream(12);
    DOL_CALL(dol_residual_norm(x.p(), u.p(), norm_u, gamma_u, gate.p(), scale, gamma_y, eps, h.p(), y.p(), rstd_u, rstd_h, s));
}

PyObject *residual_norm_workspace(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 2);
    Matrix u(a, 0), gate(a, 1);
    if (a.bad) return nullptr;
    int64_t need = 0;
    const dol_status st = dol_residual_norm_workspace(u.p(), gate.p(), &need);
    return bytes(st, need);
}

template <auto CALL>
PyObject *residual_norm_backward(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 19);
    Matrix x(a, 0), u(a, 1), gate(a, 4), gh(a, 9), gy(a, 10), gx(a, 11), gu(a, 12), gg(a, 14);
    const int32_t norm_u = a.num32(2);
    auto *gamma_u = a.ptr<float>(3), *gamma_y = a.ptr<float>(6);
    const float scale = static_cast<float>(a.real(5));
    auto *rstd_u = a.ptr<float>(7), *rstd_h = a.ptr<float>(8), *ggu = a.ptr<float>(13), *ggy = a.ptr<float>(15);
    auto *ws = a.ptr<void>(16);
    const int64_t have = a.num(17);
    void *s = a.stream(18);
    DOL_CALL(CALL(x.p(), u.p(), norm_u, gamma_u, gate.p(), scale, gamma_y, rstd_u, rstd_h, gh.p(), gy.p(), gx.p(), gu.p(), ggu, gg.p(), ggy, ws, have, s));
}

PyObject *grad_norm_workspace(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 1);
    auto *l = a.ptr<dol_tensor_list>(0);
    if (a.bad) return nullptr;
    int64_t need = 0;
    const dol_status st = dol_grad_norm_workspace(l, &need);
    return bytes(st, need);
}

PyObject *grad_norm(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 5);
    auto *l = a.ptr<dol_tensor_list>(0);
    auto *norm = a.ptr<float>(1);
    auto *ws = a.ptr<void>(2);
    const int64_t have = a.num(3);
    void *s = a.stream(4);
    DOL_CALL(dol_grad_norm(l, norm, ws, have, s));
}

PyObject *clip_grads(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 9);
    auto *l = a.ptr<dol_tensor_list>(0), *o = a.ptr<dol_tensor_list>(1);
    const double most = a.real(2), eps = a.real(3);
    auto *norm = a.ptr<float>(4), *coef = a.ptr<float>(5);
    auto *ws = a.ptr<void>(6);
    const int64_t have = a.num(7);
    void *s = a.stream(8);
    DOL_CALL(dol_clip_grads(l, o, most, eps, norm, coef, ws, have, s));
}

// ---- a tensor's description, for the structures above (a Python function of the same checks takes about twice as long); None for None

PyObject *g_float = nullptr, *g_bf16 = nullptr;             // torch.float32, torch.bfloat16
PyObject *s_is_cuda = nullptr, *s_dtype = nullptr, *s_shape = nullptr, *s_stride = nullptr, *s_data_ptr = nullptr;

struct Tensor {
    static constexpr int kMost = 16;
    int dims = 0;
    int64_t size[kMost], stride[kMost];
    PyObject *dtype = nullptr;

    explicit Tensor(PyObject *t) : t_(t) {}
    ~Tensor() { Py_XDECREF(dtype); }

    // False with an error set where it is not a tensor of the device with at most kMost dimensions.
    bool read()
    {
        PyObject *cuda = PyObject_GetAttr(t_, s_is_cuda);
        const bool here = cuda == Py_True;
        Py_XDECREF(cuda);
        if (!cuda || !(here || refuse("not a device tensor"))) return false;
        dtype = PyObject_GetAttr(t_, s_dtype);
        return dtype && numbers(PyObject_GetAttr(t_, s_shape), size) && numbers(PyObject_CallMethodNoArgs(t_, s_stride), stride);
    }
    // dol_dtype, or -1.
    int type() const { return dtype == g_float ? DOL_F32 : dtype == g_bf16 ? DOL_BF16 : -1; }
    bool contiguous() const
    {
        int64_t want = 1;
        for (int k = dims - 1; k >= 0; --k) {
            if (size[k] == 0) return true;
            if (size[k] != 1 && stride[k] != want) return false;
            want *= size[k];
        }
        return true;
    }
    PyObject *address() const { return PyObject_CallMethodNoArgs(t_, s_data_ptr); }
    // Always false, with an AssertionError set.
    static bool refuse(const char *why)
    {
        PyErr_SetString(PyExc_AssertionError, why);
        return false;
    }

private:
    PyObject *t_;
    bool numbers(PyObject *from, int64_t *to)
    {
        if (!from) return false;
        const bool fits = PyTuple_Check(from) && PyTuple_GET_SIZE(from) <= kMost;
        dims = fits ? static_cast<int>(PyTuple_GET_SIZE(from)) : 0;
        for (int k = 0; k < dims; ++k) to[k] = PyLong_AsLongLong(PyTuple_GET_ITEM(from, k));
        Py_DECREF(from);
        return fits ? !PyErr_Occurred() : refuse("too many dimensions");
    }
};

PyObject *described(std::initializer_list<int64_t> numbers, PyObject *address)
{
    PyObject *r = address ? PyTuple_New(static_cast<Py_ssize_t>(numbers.size()) + 1) : nullptr;
    if (!r) {
        Py_XDECREF(address);
        return nullptr;
    }
    Py_ssize_t k = 0;
    for (int64_t n : numbers) PyTuple_SET_ITEM(r, k++, PyLong_FromLongLong(n));
    PyTuple_SET_ITEM(r, k, address);
    return r;
}

// matrix(tensor [rows, cols]): dol_matrix's fields; neighbouring columns next to each other.
PyObject *matrix(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 1);
    if (a.bad) return nullptr;
    if (v[0] == Py_None) Py_RETURN_NONE;
    Tensor t(v[0]);
    if (!t.read()) return nullptr;
    if (t.type() < 0 || t.dims != 2) return Tensor::refuse("a float32 or bfloat16 matrix wanted"), nullptr;
    const int64_t rows = t.size[0], cols = t.size[1];
    if ((cols > 1 && t.stride[1] != 1) || (rows > 1 && t.stride[0] < cols)) return Tensor::refuse("columns of a row next to each other wanted"), nullptr;
    return described({t.type(), rows, cols, rows > 1 ? t.stride[0] : cols > 1 ? cols : 1}, t.address());
}

// activations(tensor [batch, points.., channels]): dol_activations' fields; neighbouring channels next to each other and points at one distance.
PyObject *activations(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 1);
    if (a.bad) return nullptr;
    if (v[0] == Py_None) Py_RETURN_NONE;
    Tensor t(v[0]);
    if (!t.read()) return nullptr;
    if (t.type() < 0 || t.dims < 3) return Tensor::refuse("float32 or bfloat16 activations [batch, points.., channels] wanted"), nullptr;
    const int64_t channels = t.size[t.dims - 1];
    int64_t points = 1, ld = channels;
    bool good = channels <= 1 || t.stride[t.dims - 1] == 1;
    for (int k = t.dims - 2; k > 0; --k) {              // from the innermost: each has to continue the one before
        if (t.size[k] > 1) {
            good = good && (points == 1 || t.stride[k] == ld * points);
            if (points == 1) ld = t.stride[k];
        }
        points *= t.size[k];
    }
    if (!good || (points > 1 && ld < channels)) return Tensor::refuse("channels next to each other and points at one distance wanted"), nullptr;
    return described({t.type(), t.size[0], points, channels, t.stride[0], ld > channels ? ld : channels}, t.address());
}

// values(tensor, dtype, size..): the address of a contiguous tensor of this type and these sizes.
PyObject *values(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (n >= 1 && v[0] == Py_None) Py_RETURN_NONE;
    if (n < 3) return PyErr_Format(PyExc_TypeError, "%zd arguments, at least 3 wanted", n);
    Tensor t(v[0]);
    if (!t.read()) return nullptr;
    bool good = t.dtype == v[1] && t.dims == n - 2 && t.contiguous();
    for (int k = 0; good && k < t.dims; ++k) good = PyLong_AsLongLong(v[k + 2]) == t.size[k];
    if (PyErr_Occurred()) return nullptr;
    if (!good) return Tensor::refuse("a contiguous tensor of another type or size wanted"), nullptr;
    return t.address();
}

// setup(fail, current_device, current_raw_stream, float32, bfloat16)
PyObject *setup(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    Args a(v, n, 5);
    if (a.bad) return nullptr;
    PyObject **to[5] = {&g_fail, &g_device, &g_stream, &g_float, &g_bf16};
    for (int k = 0; k < 5; ++k) {
        Py_INCREF(v[k]);
        Py_XSETREF(*to[k], v[k]);
    }
    const std::pair<PyObject **, const char *> names[] = {{&s_is_cuda, "is_cuda"}, {&s_dtype, "dtype"}, {&s_shape, "shape"}, {&s_stride, "stride"}, {&s_data_ptr, "data_ptr"}};
    for (const auto &name : names) {
        PyObject *s = PyUnicode_InternFromString(name.second);
        if (!s) return nullptr;
        Py_XSETREF(*name.first, s);
    }
    Py_RETURN_NONE;
}

#define DOL_FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr
PyMethodDef g_methods[] = {
    {"setup", DOL_FAST(setup)},
    {"apply2", DOL_FAST(apply2)},
    {"backward", DOL_FAST(backward)},
    {"filter", DOL_FAST(filter)},
    {"union", DOL_FAST(union_)},
    {"nll_grad", DOL_FAST(nll_grad)},
    {"dtkp_init", DOL_FAST(dtkp_init)},
    {"dtkp_apply2_input", DOL_FAST(dtkp_apply2_input)},
    {"dtkp_backward", DOL_FAST(dtkp_backward)},
    {"fold_apply2", DOL_FAST(fold_apply2)},
    {"dtkp_fold_apply2", DOL_FAST(dtkp_fold_apply2)},
    {"cross_entropy_workspace", DOL_FAST(cross_entropy_workspace)},
    {"cross_entropy_kernel", DOL_FAST(cross_entropy_kernel)},
    {"cross_entropy", DOL_FAST(cross_entropy)},
    {"cross_entropy_backward", DOL_FAST(cross_entropy_backward)},
    {"newton_schulz_workspace", DOL_FAST(newton_schulz_workspace)},
    {"newton_schulz_kernel", DOL_FAST(newton_schulz_kernel)},
    {"newton_schulz", DOL_FAST(newton_schulz)},
    {"group_norm_workspace", DOL_FAST(group_norm_workspace)},
    {"group_norm", DOL_FAST(group_norm)},
    {"group_norm_backward", DOL_FAST(group_norm_backward)},
    {"linear_workspace", DOL_FAST(linear_workspace)},
    {"linear_kernel", DOL_FAST(linear_kernel)},
    {"linear", DOL_FAST(linear)},
    {"linear_backward", DOL_FAST(linear_backward)},
    {"residual_norm", DOL_FAST(residual_norm)},
    {"residual_norm_workspace", DOL_FAST(residual_norm_workspace)},
    {"residual_norm_backward", DOL_FAST(residual_norm_backward<dol_residual_norm_backward>)},
    {"residual_norm_backward_from_h", DOL_FAST(residual_norm_backward<dol_residual_norm_backward_from_h>)},
    {"grad_norm_workspace", DOL_FAST(grad_norm_workspace)},
    {"grad_norm", DOL_FAST(grad_norm)},
    {"clip_grads", DOL_FAST(clip_grads)},
    {"matrix", DOL_FAST(matrix)},
    {"activations", DOL_FAST(activations)},
    {"values", DOL_FAST(values)},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&g_module); }
