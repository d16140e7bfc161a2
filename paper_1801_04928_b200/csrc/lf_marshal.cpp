// Marshalling of torch tensors for the layer operators: the checks of the Python binding (type, device, shape,
// layout) and the C argument structs, filled from the tensors directly.  The same work in Python took about as
// long as a kernel launch, which is what the smallest calls consist of.  No arithmetic and no CUDA here;
// the library's entry points arrive as addresses.
//
// Every function takes (entry point, handle, tensors and numbers ...) and returns None, or (status, text) for a
// refusal (text says what was wrong) and for a status of the library (text is None).  No C++ exception leaves them:
// what a tensor throws when it is asked for a size, a stride or an address becomes a refusal.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <limits.h>

#include <exception>
#include <new>
#include <string>
#include <type_traits>

#include "leapfrog.h"

namespace {

constexpr long long ROWS_MOST = 0x7FFFFFFF;

struct call {
    const int device;                // the handle's: the last argument
    std::string problem;
    const at::Tensor* written[6];    // outputs of the call
    int n_written = 0;
    explicit call(PyObject* d) : device((int)PyLong_AsLong(d)) {}

    bool refuse(const char* name, const std::string& what)
    {
        if (problem.empty()) problem = std::string("argument ") + name + ": " + what;
        return false;
    }
    static std::string said(const at::Tensor& t)
    {
        std::string s = c10::toString(t.scalar_type());
        s += " (";
        for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
        s += ") strides (";
        for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.stride(i));
        s += ") on ";
        s += t.device().str();
        return s;
    }
    bool here(const at::Tensor& t) const { return t.is_cuda() && t.device().index() == device; }
    const at::Tensor* tensor(PyObject* o, const char* name)
    {
        if (!THPVariable_Check(o)) { refuse(name, "not a tensor"); return nullptr; }
        const at::Tensor& t = THPVariable_Unpack(o);
        if (t.layout() != at::kStrided || t.is_nested() || !t.has_storage()) { refuse(name, "not a dense tensor with memory of its own"); return nullptr; }
        return &t;
    }
    // enum lf_dtype of a tensor that sets the call's type; -1 after a refusal
    int type(const at::Tensor* t, const char* name)
    {
        if (!t) return -1;
        switch (t->scalar_type()) {
            case at::kFloat: return LF_F32;
            case at::kBFloat16: return LF_BF16;
            case at::kHalf: return LF_F16;
            default: refuse(name, said(*t) + " (float32, bfloat16 or float16 needed)"); return -1;
        }
    }
    // rows and columns of the matrix that sets a call's sizes
    bool shape(const at::Tensor* t, const char* name, int* rows, int* cols)
    {
        *rows = *cols = 0;
        if (!t) return false;
        if (t->dim() != 2) return refuse(name, said(*t) + " (2 dimensions needed)");
        if (t->size(0) > ROWS_MOST || t->size(1) > ROWS_MOST) return refuse(name, said(*t) + " (too large)");
        *rows = (int)t->size(0);
        *cols = (int)t->size(1);
        return true;
    }
    // address and leading dimension of a [rows][cols] matrix with unit stride along its rows; None gives NULL
    bool mat(PyObject* o, const char* name, int rows, int cols, at::ScalarType st, const void** p, long long* ld)
    {
        *p = nullptr;
        *ld = 0;
        if (o == Py_None) return true;
        const at::Tensor* t = tensor(o, name);
        if (!t) return false;
        if (t->scalar_type() != st || !here(*t) || t->dim() != 2 || t->size(0) != rows || t->size(1) != cols)
            return refuse(name, said(*t) + ", " + c10::toString(st) + " (" + std::to_string(rows) + ", " + std::to_string(cols) + ") on cuda:" + std::to_string(device) + " needed");
        if (cols > 1 && t->stride(1) != 1) return refuse(name, said(*t) + " (unit stride along rows needed)");
        if (rows > 1) {
            if (t->stride(0) < cols) return refuse(name, said(*t) + " (rows overlap)");
            *ld = t->stride(0);
        }
        *p = t->const_data_ptr();
        return true;
    }
    // an output: memory that it shares with a lazy copy becomes its own, and its version goes up when the call is accepted
    void* output(PyObject* o)
    {
        if (o == Py_None) return nullptr;
        const at::Tensor& t = THPVariable_Unpack(o);
        written[n_written++] = &t;
        return t.mutable_data_ptr();
    }
    bool mat(PyObject* o, const char* name, int rows, int cols, at::ScalarType st, void** p, long long* ld)
    {
        const void* as_input;
        *p = nullptr;
        if (!mat(o, name, rows, cols, st, &as_input, ld)) return false;
        *p = output(o);
        return true;
    }
    // contiguous tensor of n elements
    bool flat(PyObject* o, const char* name, long long n, at::ScalarType st, const void** p)
    {
        *p = nullptr;
        if (o == Py_None) return true;
        const at::Tensor* t = tensor(o, name);
        if (!t) return false;
        if (t->scalar_type() != st || !here(*t) || t->numel() != n || !t->is_contiguous())
            return refuse(name, said(*t) + ", " + std::to_string(n) + " contiguous elements of " + c10::toString(st) + " on cuda:" + std::to_string(device) + " needed");
        *p = t->const_data_ptr();
        return true;
    }
    template <typename U>
    bool flat(PyObject* o, const char* name, long long n, at::ScalarType st, U** p)
    {
        const void* v;
        *p = nullptr;
        if (!flat(o, name, n, st, &v)) return false;
        if constexpr (std::is_const_v<U>) *p = static_cast<U*>(v);
        else *p = static_cast<U*>(output(o));
        return true;
    }
    template <typename U>
    bool eight(PyObject* q, PyObject* s, int rows, int cols, U** qp, U** sp)
    {
        return flat(q, "q", (long long)rows * cols, at::kByte, qp) & flat(s, "s", (long long)rows * ((cols + 31) / 32), at::kByte, sp);
    }
    // a contiguous float32 [d0][d1] matrix of scales; `or_else`: another shape may fit as well, nothing is refused
    template <typename U>
    bool scales(PyObject* o, const char* name, long long d0, long long d1, U** p, bool or_else = false)
    {
        *p = nullptr;
        if (o == Py_None) return true;
        const at::Tensor* t = tensor(o, name);
        if (!t) return false;
        if (t->scalar_type() != at::kFloat || !here(*t) || t->dim() != 2 || t->size(0) != d0 || t->size(1) != d1 || !t->is_contiguous())
            return or_else ? false : refuse(name, said(*t) + ", contiguous Float (" + std::to_string(d0) + ", " + std::to_string(d1) + ") on cuda:" + std::to_string(device) + " needed");
        if constexpr (std::is_const_v<U>) *p = static_cast<U*>(t->const_data_ptr());
        else *p = static_cast<U*>(output(o));
        return true;
    }
    // an 8-bit matrix of which only its type and shape are looked at here
    template <typename U>
    bool bytes(PyObject* o, const char* name, int rows, int cols, U** p, long long* ld)
    {
        if constexpr (std::is_const_v<U>) {
            const void* v;
            if (!mat(o, name, rows, cols, at::kByte, &v, ld)) return false;
            *p = static_cast<U*>(v);
        } else {
            void* v;
            if (!mat(o, name, rows, cols, at::kByte, &v, ld)) return false;
            *p = static_cast<U*>(v);
        }
        return true;
    }
    // a number for an int of the library: one that is too large is refused, not cut
    int number(PyObject* o, const char* name)
    {
        int beyond = 0;
        const long n = PyLong_AsLongAndOverflow(o, &beyond);
        if (beyond || n < INT_MIN || n > INT_MAX) { refuse(name, "out of range"); return 0; }
        return (int)n;
    }
    PyObject* answer(int rc)
    {
        if (rc == LF_OK) {
            for (int i = 0; i < n_written; ++i)
                if (!written[i]->is_inference()) written[i]->unsafeGetTensorImpl()->bump_version();      // (those have no version)
            Py_RETURN_NONE;
        }
        return Py_BuildValue("(iO)", rc, Py_None);
    }
    PyObject* refused() { return Py_BuildValue("(is)", (int)LF_EINVAL, problem.c_str()); }
};

void* address(PyObject* o) { return PyLong_AsVoidPtr(o); }

#define LF_EXPECT(n)                                                                     \
    if (nargs != (n)) {                                                                  \
        PyErr_Format(PyExc_TypeError, "%zd arguments, %d needed", nargs, (int)(n));      \
        return nullptr;                                                                  \
    }
#define LF_NUMBERS_OK if (PyErr_Occurred()) return nullptr

// linear(f, ops, x, w, y, bias, residual, act, q, s, device)
PyObject* m_linear(PyObject*, PyObject* const* v, Py_ssize_t nargs)
{
    LF_EXPECT(11);
    call c(v[10]);
    lf_linear_args a = {};
    const at::Tensor *x = c.tensor(v[2], "x"), *w = c.tensor(v[3], "w");
    int k = 0, wn = 0;
    a.dtype = c.type(x, "x");
    a.act = c.number(v[7], "act");
    LF_NUMBERS_OK;
    c.shape(x, "x", &a.tokens, &a.n_in);
    c.shape(w, "w", &wn, &k);
    if (!c.problem.empty()) return c.refused();
    a.n_out = wn;
    const at::ScalarType st = x->scalar_type();
    const bool ok = c.mat(v[2], "x", a.tokens, a.n_in, st, &a.x, &a.ld_x) && (k == a.n_in || c.refuse("w", c.said(*w) + ", rows as long as x's needed")) &&
                    c.flat(v[3], "w", (long long)a.n_out * a.n_in, st, &a.w) && c.mat(v[4], "y", a.tokens, a.n_out, st, &a.y, &a.ld_y) &&
                    c.flat(v[5], "bias", a.n_out, at::kFloat, &a.bias) &&
                    c.mat(v[6], "residual", a.tokens, a.n_out, st, &a.residual, &a.ld_residual) && c.eight(v[8], v[9], a.tokens, a.n_out, &a.q, &a.s);
    if (!ok) return c.refused();
    return c.answer(reinterpret_cast<decltype(&lf_linear)>(address(v[0]))(static_cast<lf_ops*>(address(v[1])), &a));
}

// linear_grad_x(f, ops, dz, w, dx, q, s, act, add, device)
PyObject* m_linear_grad_x(PyObject*, PyObject* const* v, Py_ssize_t nargs)
{
    LF_EXPECT(10);
    call c(v[9]);
    lf_linear_grad_x_args a = {};
    const at::Tensor *dz = c.tensor(v[2], "dz"), *w = c.tensor(v[3], "w");
    int wn = 0;
    a.dtype = c.type(dz, "dz");
    a.act = c.number(v[7], "act");
    LF_NUMBERS_OK;
    c.shape(dz, "dz", &a.tokens, &a.n_out);
    c.shape(w, "w", &wn, &a.n_in);
    if (!c.problem.empty()) return c.refused();
    const at::ScalarType st = dz->scalar_type();
    const bool ok = c.mat(v[2], "dz", a.tokens, a.n_out, st, &a.dz, &a.ld_dz) && (wn == a.n_out || c.refuse("w", c.said(*w) + ", as many rows as dz has columns needed")) &&
                    c.flat(v[3], "w", (long long)a.n_out * a.n_in, st, &a.w) && c.mat(v[4], "dx", a.tokens, a.n_in, st, &a.dx, &a.ld_dx) &&
                    c.eight(v[5], v[6], a.tokens, a.n_in, &a.q, &a.s) && c.mat(v[8], "add", a.tokens, a.n_in, st, &a.add, &a.ld_add);
    if (!ok) return c.refused();
    return c.answer(reinterpret_cast<decltype(&lf_linear_grad_x)>(address(v[0]))(static_cast<lf_ops*>(address(v[1])), &a));
}

// linear_grad_w(f, ops, dz, gw, gb, x, q, s, act, device)
PyObject* m_linear_grad_w(PyObject*, PyObject* const* v, Py_ssize_t nargs)
{
    LF_EXPECT(10);
    call c(v[9]);
    lf_linear_grad_w_args a = {};
    const at::Tensor *dz = c.tensor(v[2], "dz"), *gw = c.tensor(v[3], "gw");
    int wn = 0;
    a.dtype = c.type(dz, "dz");
    a.gw_dtype = c.type(gw, "gw");
    a.act = c.number(v[8], "act");
    LF_NUMBERS_OK;
    c.shape(dz, "dz", &a.tokens, &a.n_out);
    c.shape(gw, "gw", &wn, &a.n_in);
    if (!c.problem.empty()) return c.refused();
    const at::ScalarType st = dz->scalar_type();
    const bool ok = c.mat(v[2], "dz", a.tokens, a.n_out, st, &a.dz, &a.ld_dz) && (wn == a.n_out || c.refuse("gw", c.said(*gw) + ", as many rows as dz has columns needed")) &&
                    c.flat(v[3], "gw", (long long)a.n_out * a.n_in, gw->scalar_type(), &a.gw) && c.flat(v[4], "gb", a.n_out, at::kFloat, &a.gb) &&
                    c.mat(v[5], "x", a.tokens, a.n_in, st, &a.x, &a.ld_x) && c.eight(v[6], v[7], a.tokens, a.n_in, &a.q, &a.s);
    if (!ok) return c.refused();
    return c.answer(reinterpret_cast<decltype(&lf_linear_grad_w)>(address(v[0]))(static_cast<lf_ops*>(address(v[1])), &a));
}

// rms_norm(f, ops, x, gain, y, residual, h, q, s, eps, device)
PyObject* m_rms_norm(PyObject*, PyObject* const* v, Py_ssize_t nargs)
{
    LF_EXPECT(11);
    call c(v[10]);
    lf_rms_norm_args a = {};
    const at::Tensor* x = c.tensor(v[2], "x");
    a.dtype = c.type(x, "x");
    a.eps = (float)PyFloat_AsDouble(v[9]);
    LF_NUMBERS_OK;
    c.shape(x, "x", &a.tokens, &a.n);
    if (!c.problem.empty()) return c.refused();
    const at::ScalarType st = x->scalar_type();
    const bool ok = c.mat(v[2], "x", a.tokens, a.n, st, &a.x, &a.ld_x) && c.flat(v[3], "gain", a.n, at::kFloat, &a.gain) &&
                    c.mat(v[4], "y", a.tokens, a.n, st, &a.y, &a.ld_y) && c.mat(v[5], "residual", a.tokens, a.n, st, &a.residual, &a.ld_residual) &&
                    c.mat(v[6], "h", a.tokens, a.n, st, &a.h, &a.ld_h) && c.eight(v[7], v[8], a.tokens, a.n, &a.q, &a.s);
    if (!ok) return c.refused();
    return c.answer(reinterpret_cast<decltype(&lf_rms_norm)>(address(v[0]))(static_cast<lf_ops*>(address(v[1])), &a));
}

// rms_norm_backward(f, ops, dy, h, gain, dh, dgain, dres, eps, device)
PyObject* m_rms_norm_backward(PyObject*, PyObject* const* v, Py_ssize_t nargs)
{
    LF_EXPECT(10);
    call c(v[9]);
    lf_rms_norm_backward_args a = {};
    const at::Tensor* h = c.tensor(v[3], "h");
    a.dtype = c.type(h, "h");
    a.eps = (float)PyFloat_AsDouble(v[8]);
    LF_NUMBERS_OK;
    c.shape(h, "h", &a.tokens, &a.n);
    if (!c.problem.empty()) return c.refused();
    const at::ScalarType st = h->scalar_type();
    const bool ok = c.mat(v[2], "dy", a.tokens, a.n, st, &a.dy, &a.ld_dy) && c.mat(v[3], "h", a.tokens, a.n, st, &a.h, &a.ld_h) &&
                    c.flat(v[4], "gain", a.n, at::kFloat, &a.gain) && c.mat(v[5], "dh", a.tokens, a.n, st, &a.dh, &a.ld_dh) &&
                    c.flat(v[6], "dgain", a.n, at::kFloat, &a.dgain) && c.mat(v[7], "dres", a.tokens, a.n, st, &a.dres, &a.ld_dres);
    if (!ok) return c.refused();
    return c.answer(reinterpret_cast<decltype(&lf_rms_norm_backward)>(address(v[0]))(static_cast<lf_ops*>(address(v[1])), &a));
}

// pack8(f, ops, x, q, s, device)
PyObject* m_pack8(PyObject*, PyObject* const* v, Py_ssize_t nargs)
{
    LF_EXPECT(6);
    call c(v[5]);
    const at::Tensor* x = c.tensor(v[2], "x");
    const int dtype = c.type(x, "x");
    LF_NUMBERS_OK;
    int m, n;
    c.shape(x, "x", &m, &n);
    if (!c.problem.empty()) return c.refused();
    const void* xp;
    unsigned char *q, *s;
    long long ld;
    if (!(c.mat(v[2], "x", m, n, x->scalar_type(), &xp, &ld) && c.eight(v[3], v[4], m, n, &q, &s))) return c.refused();
    return c.answer(reinterpret_cast<decltype(&lf_pack8)>(address(v[0]))(static_cast<lf_ops*>(address(v[1])), dtype, m, n, xp, ld, q, s));
}

// unpack8(f, ops, q, s, x, act, device)
PyObject* m_unpack8(PyObject*, PyObject* const* v, Py_ssize_t nargs)
{
    LF_EXPECT(7);
    call c(v[6]);
    const at::Tensor* x = c.tensor(v[4], "x");
    const int dtype = c.type(x, "x"), act = c.number(v[5], "act");
    LF_NUMBERS_OK;
    int m, n;
    c.shape(x, "x", &m, &n);
    if (!c.problem.empty()) return c.refused();
    void* xp;
    const unsigned char *q, *s;
    long long ld;
    if (!(c.mat(v[4], "x", m, n, x->scalar_type(), &xp, &ld) && c.eight(v[2], v[3], m, n, &q, &s))) return c.refused();
    return c.answer(reinterpret_cast<decltype(&lf_unpack8)>(address(v[0]))(static_cast<lf_ops*>(address(v[1])), dtype, act, m, n, q, s, xp, ld));
}

// act_backward(f, ops, dy, q, s, dz, act, device)
PyObject* m_act_backward(PyObject*, PyObject* const* v, Py_ssize_t nargs)
{
    LF_EXPECT(8);
    call c(v[7]);
    const at::Tensor* dy = c.tensor(v[2], "dy");
    const int dtype = c.type(dy, "dy"), act = c.number(v[6], "act");
    LF_NUMBERS_OK;
    int m, n;
    c.shape(dy, "dy", &m, &n);
    if (!c.problem.empty()) return c.refused();
    const void* yp;
    void* zp;
    const unsigned char *q, *s;
    long long ldy, ldz;
    if (!(c.mat(v[2], "dy", m, n, dy->scalar_type(), &yp, &ldy) && c.mat(v[5], "dz", m, n, dy->scalar_type(), &zp, &ldz) && c.eight(v[3], v[4], m, n, &q, &s)))
        return c.refused();
    return c.answer(reinterpret_cast<decltype(&lf_act_backward)>(address(v[0]))(static_cast<lf_ops*>(address(v[1])), dtype, act, m, n, yp, ldy, q, s, zp, ldz));
}

long long blocks(long long n) { return (n + 127) / 128; }

// layer_norm(f, ops, x, gain, bias, y, residual, h, q, s, mean, rstd, eps, device)
PyObject* m_layer_norm(PyObject*, PyObject* const* v, Py_ssize_t nargs)
{
    LF_EXPECT(14);
    call c(v[13]);
    lf_layer_norm_args a = {};
    const at::Tensor* x = c.tensor(v[2], "x");
    a.dtype = c.type(x, "x");
    a.eps = (float)PyFloat_AsDouble(v[12]);
    LF_NUMBERS_OK;
    c.shape(x, "x", &a.tokens, &a.n);
    if (!c.problem.empty()) return c.refused();
    const at::ScalarType st = x->scalar_type();
    const bool ok = c.mat(v[2], "x", a.tokens, a.n, st, &a.x, &a.ld_x) && c.flat(v[3], "gain", a.n, at::kFloat, &a.gain) &&
                    c.flat(v[4], "bias", a.n, at::kFloat, &a.bias) && c.mat(v[5], "y", a.tokens, a.n, st, &a.y, &a.ld_y) &&
                    c.mat(v[6], "residual", a.tokens, a.n, st, &a.residual, &a.ld_residual) && c.mat(v[7], "h", a.tokens, a.n, st, &a.h, &a.ld_h) &&
                    c.bytes(v[8], "q", a.tokens, a.n, &a.q, &a.ld_q) && c.scales(v[9], "s", blocks(a.n), a.tokens, &a.s) &&
                    c.flat(v[10], "mean", a.tokens, at::kFloat, &a.mean) && c.flat(v[11], "rstd", a.tokens, at::kFloat, &a.rstd);
    if (!ok) return c.refused();
    return c.answer(reinterpret_cast<decltype(&lf_layer_norm)>(address(v[0]))(static_cast<lf_ops*>(address(v[1])), &a));
}

// layer_norm_backward(f, ops, dy, h, gain, mean, rstd, dh, dgain, dbias, dres, device)
PyObject* m_layer_norm_backward(PyObject*, PyObject* const* v, Py_ssize_t nargs)
{
    LF_EXPECT(12);
    call c(v[11]);
    lf_layer_norm_backward_args a = {};
    const at::Tensor* h = c.tensor(v[3], "h");
    a.dtype = c.type(h, "h");
    LF_NUMBERS_OK;
    c.shape(h, "h", &a.tokens, &a.n);
    if (!c.problem.empty()) return c.refused();
    const at::ScalarType st = h->scalar_type();
    const bool ok = c.mat(v[2], "dy", a.tokens, a.n, st, &a.dy, &a.ld_dy) && c.mat(v[3], "h", a.tokens, a.n, st, &a.h, &a.ld_h) &&
                    c.flat(v[4], "gain", a.n, at::kFloat, &a.gain) && c.flat(v[5], "mean", a.tokens, at::kFloat, &a.mean) &&
                    c.flat(v[6], "rstd", a.tokens, at::kFloat, &a.rstd) && c.mat(v[7], "dh", a.tokens, a.n, st, &a.dh, &a.ld_dh) &&
                    c.flat(v[8], "dgain", a.n, at::kFloat, &a.dgain) && c.flat(v[9], "dbias", a.n, at::kFloat, &a.dbias) &&
                    c.mat(v[10], "dres", a.tokens, a.n, st, &a.dres, &a.ld_dres);
    if (!ok) return c.refused();
    return c.answer(reinterpret_cast<decltype(&lf_layer_norm_backward)>(address(v[0]))(static_cast<lf_ops*>(address(v[1])), &a));
}

// pack_blocks(f, ops, x, q, s, qt, st, device), pack_tiles the same
template <bool TILES>
PyObject* pack_any(PyObject* const* v, Py_ssize_t nargs)
{
    LF_EXPECT(8);
    call c(v[7]);
    lf_pack_blocks_args a = {};
    const at::Tensor* x = c.tensor(v[2], "x");
    a.dtype = c.type(x, "x");
    LF_NUMBERS_OK;
    c.shape(x, "x", &a.tokens, &a.n);
    if (!c.problem.empty()) return c.refused();
    const long long tb = blocks(a.tokens), nb = blocks(a.n);
    const bool ok = c.mat(v[2], "x", a.tokens, a.n, x->scalar_type(), &a.x, &a.ld_x) && c.bytes(v[3], "q", a.tokens, a.n, &a.q, &a.ld_q) &&
                    c.scales(v[4], "s", TILES ? tb : nb, TILES ? nb : a.tokens, &a.s) && c.bytes(v[5], "qt", a.n, a.tokens, &a.qt, &a.ld_qt) &&
                    c.scales(v[6], "st", TILES ? nb : tb, TILES ? tb : a.n, &a.st);
    if (!ok) return c.refused();
    return c.answer(reinterpret_cast<decltype(&lf_pack_blocks)>(address(v[0]))(static_cast<lf_ops*>(address(v[1])), &a));
}
PyObject* m_pack_blocks(PyObject*, PyObject* const* v, Py_ssize_t nargs) { return pack_any<false>(v, nargs); }
PyObject* m_pack_tiles(PyObject*, PyObject* const* v, Py_ssize_t nargs) { return pack_any<true>(v, nargs); }

// product_blocks(f, ops, a, sa, b, sb, d, bias, add, device)
PyObject* m_product_blocks(PyObject*, PyObject* const* v, Py_ssize_t nargs)
{
    LF_EXPECT(10);
    call c(v[9]);
    lf_product_blocks_args a = {};
    const at::Tensor *x = c.tensor(v[2], "a"), *w = c.tensor(v[4], "b"), *d = c.tensor(v[6], "d");
    int k = 0;
    a.out_dtype = c.type(d, "d");
    LF_NUMBERS_OK;
    c.shape(x, "a", &a.tokens, &a.n_in);
    c.shape(w, "b", &a.n_out, &k);
    if (!c.problem.empty()) return c.refused();
    const long long kb = blocks(a.n_in);
    bool ok = c.bytes(v[2], "a", a.tokens, a.n_in, &a.a, &a.ld_a) && c.scales(v[3], "sa", kb, a.tokens, &a.sa) &&
              (k == a.n_in || c.refuse("b", c.said(*w) + ", rows as long as a's needed")) && c.bytes(v[4], "b", a.n_out, a.n_in, &a.b, &a.ld_b);
    if (ok && !c.scales(v[5], "sb", kb, a.n_out, &a.sb, true)) {        // (n_out is 8 at least: the two shapes are never the same)
        a.b_tiles = 1;
        ok = c.problem.empty() && c.scales(v[5], "sb (scales of rows or, else, of tiles)", blocks(a.n_out), kb, &a.sb);
    }
    ok = ok && c.mat(v[6], "d", a.tokens, a.n_out, d->scalar_type(), &a.d, &a.ld_d) && c.flat(v[7], "bias", a.n_out, at::kFloat, &a.bias) &&
         c.mat(v[8], "add", a.tokens, a.n_out, d->scalar_type(), &a.add, &a.ld_add);
    if (!ok) return c.refused();
    return c.answer(reinterpret_cast<decltype(&lf_product_blocks)>(address(v[0]))(static_cast<lf_ops*>(address(v[1])), &a));
}

// entries in the order of the indices: their shape, or one dimension (a matrix of as many entries the other way round is in another order)
bool listed_as(const at::Tensor& value, const at::Tensor& index) { return value.dim() == 1 || value.sizes() == index.sizes(); }

// distill(f, ops, z, index, value, loss, lse, weight, dz, temperature, device); distill_backward the same, loss None
template <bool BACKWARD>
PyObject* distill_any(PyObject* const* v, Py_ssize_t nargs)
{
    LF_EXPECT(11);
    call c(v[10]);
    lf_distill_args a = {};
    const at::Tensor *z = c.tensor(v[2], "z"), *index = c.tensor(v[3], "index");
    int rows = 0;
    a.dtype = c.type(z, "z");
    a.temperature = (float)PyFloat_AsDouble(v[9]);
    LF_NUMBERS_OK;
    c.shape(z, "z", &a.tokens, &a.vocab);
    c.shape(index, "index", &rows, &a.top);
    if (!c.problem.empty()) return c.refused();
    const at::ScalarType st = z->scalar_type();
    const long long n = (long long)a.tokens * a.top;
    const float* lse_in = nullptr;
    const bool ok = c.mat(v[2], "z", a.tokens, a.vocab, st, &a.z, &a.ld_z) && (rows == a.tokens || c.refuse("index", c.said(*index) + ", a row for each of z's needed")) &&
                    c.flat(v[3], "index", n, at::kInt, &a.index) && c.flat(v[4], "value", n, at::kFloat, &a.value) &&
                    (v[4] == Py_None || listed_as(THPVariable_Unpack(v[4]), *index) || c.refuse("value", c.said(THPVariable_Unpack(v[4])) + ", the shape of index needed")) &&
                    c.flat(v[5], "loss", a.tokens, at::kFloat, &a.loss) &&
                    (BACKWARD ? c.flat(v[6], "lse", a.tokens, at::kFloat, &lse_in) : c.flat(v[6], "lse", a.tokens, at::kFloat, &a.lse)) &&
                    c.flat(v[7], "weight", a.tokens, at::kFloat, &a.weight) && c.mat(v[8], "dz", a.tokens, a.vocab, st, &a.dz, &a.ld_dz);
    if (!ok) return c.refused();
    if (BACKWARD) a.lse = const_cast<float*>(lse_in);          // (read only)
    return c.answer(reinterpret_cast<decltype(&lf_distill)>(address(v[0]))(static_cast<lf_ops*>(address(v[1])), &a));
}
PyObject* m_distill(PyObject*, PyObject* const* v, Py_ssize_t nargs) { return distill_any<false>(v, nargs); }
PyObject* m_distill_backward(PyObject*, PyObject* const* v, Py_ssize_t nargs) { return distill_any<true>(v, nargs); }

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* entry(PyObject* self, PyObject* const* v, Py_ssize_t nargs) noexcept
{
    try {
        return F(self, v, nargs);
    } catch (const std::bad_alloc&) {
        return PyErr_NoMemory();
    } catch (const c10::Error& e) {
        return PyErr_Occurred() ? nullptr : Py_BuildValue("(is)", (int)LF_EINVAL, e.what_without_backtrace());
    } catch (const std::exception& e) {
        return PyErr_Occurred() ? nullptr : Py_BuildValue("(is)", (int)LF_EINVAL, e.what());
    }
}

#define LF_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(entry<m_##name>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {LF_METHOD(linear),    LF_METHOD(linear_grad_x), LF_METHOD(linear_grad_w), LF_METHOD(rms_norm), LF_METHOD(rms_norm_backward),
                         LF_METHOD(pack8),     LF_METHOD(unpack8),       LF_METHOD(act_backward),  LF_METHOD(layer_norm),    LF_METHOD(layer_norm_backward),
                         LF_METHOD(pack_blocks), LF_METHOD(pack_tiles),  LF_METHOD(product_blocks), LF_METHOD(distill), LF_METHOD(distill_backward),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "tensor marshalling of the layer operators", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
