// The training operators on torch tensors: argument checks, result tensors, torch's
// current stream, and the call of the C entry point (include/novak.h), for ops.py.
// Compiled because a call of a small operator is otherwise spent in the interpreter:
// layer norm of one row of 768 takes 7.1 us a call this way and took 14 marshalled in
// Python over ctypes (its kernel alone 3.9); pack and unpack of 197 x 1000, 11.6 and 19.
// Nothing is linked against libnovak.so: bind() takes the entry points' addresses, so
// the functions are those of the library that binding.py has loaded.
#include <Python.h>

#include <vector>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include "novak.h"

namespace {

using at::Tensor;

struct Refused {};          // a Python exception is set

[[noreturn]] void value_error(const char *fmt, const char *name)
{
    PyErr_Format(PyExc_ValueError, fmt, name);
    throw Refused{};
}

const Tensor &tensor(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s must be a tensor", name);
        throw Refused{};
    }
    return THPVariable_Unpack(o);
}

int type_of(const Tensor &t, const char *name)
{
    if (t.scalar_type() == at::kFloat) return NOVAK_TYPE_F32;
    if (t.scalar_type() == at::kBFloat16) return NOVAK_TYPE_BF16;
    PyErr_Format(PyExc_TypeError, "%s must be float32 or bfloat16, got %s", name, c10::toString(t.scalar_type()));
    throw Refused{};
}

// A tensor seen as rows of its last dimension; the leading dimensions have to fold into
// one.
struct Rows {
    int64_t rows, cols, stride;
};
Rows rows_of(const Tensor &t, const char *name)
{
    if (!t.is_cuda()) value_error("%s must be a CUDA tensor", name);
    const auto shape = t.sizes();
    if (shape.empty() || shape.back() == 0) value_error("%s needs a last dimension of at least one element", name);
    const int64_t cols = shape.back();
    if (t.is_contiguous()) return {t.numel() / cols, cols, cols};
    const auto st = t.strides();
    if (st.back() != 1 && cols > 1) value_error("%s: the last dimension must be contiguous", name);
    int64_t rows = 1, stride = cols;
    for (int64_t i = static_cast<int64_t>(shape.size()) - 2; i >= 0; --i) {
        if (shape[i] == 1) continue;
        if (rows == 1) stride = st[i];
        else if (st[i] != stride * rows) value_error("%s: the leading dimensions must fold into one stride", name);
        rows *= shape[i];
    }
    if (rows > 1 && stride < cols) value_error("%s: rows overlap", name);
    return {rows, cols, stride};
}

void same(const Tensor &t, const char *name, const Tensor &like, at::IntArrayRef shape)
{
    if (t.device() != like.device()) value_error("%s is on another device", name);
    if (t.sizes() != shape) value_error("%s has another shape than the other arguments ask for", name);
}

int vector_type(const Tensor &t, const char *name, const Tensor &like, int64_t n)
{
    same(t, name, like, {n});
    if (!t.is_contiguous()) value_error("%s must be contiguous", name);
    return type_of(t, name);
}

Tensor floats(const Tensor &t, const char *name, const Tensor &like, at::IntArrayRef shape)
{
    same(t, name, like, shape);
    if (t.scalar_type() != at::kFloat) {
        PyErr_Format(PyExc_TypeError, "%s must be float32", name);
        throw Refused{};
    }
    return t.contiguous();
}

// An 8-bit form as ops.Act8 has it: the addresses of its codes and exponents, its size
// and device.
struct Form {
    int8_t *codes = nullptr;
    uint8_t *exps = nullptr;
};
struct Names {
    PyObject *codes_ptr, *exps_ptr, *rows, *cols, *index;
} names;

int64_t attribute(PyObject *o, PyObject *name)
{
    THPObjectPtr v(PyObject_GetAttr(o, name));
    if (!v) throw Refused{};
    const int64_t x = PyLong_AsLongLong(v.get());
    if (x == -1 && PyErr_Occurred()) throw Refused{};
    return x;
}

Form form_of(PyObject *o, int64_t rows, int64_t cols, const Tensor &like, const char *name)
{
    if (attribute(o, names.rows) != rows || (cols > 0 && attribute(o, names.cols) != cols) ||
        attribute(o, names.index) != like.get_device()) {
        PyErr_Format(PyExc_ValueError,
                     "the 8-bit form of %lld x %lld elements on cuda:%lld does not belong to %s of %lld rows",
                     static_cast<long long>(attribute(o, names.rows)), static_cast<long long>(attribute(o, names.cols)),
                     static_cast<long long>(attribute(o, names.index)), name, static_cast<long long>(rows));
        throw Refused{};
    }
    return {reinterpret_cast<int8_t *>(attribute(o, names.codes_ptr)),
            reinterpret_cast<uint8_t *>(attribute(o, names.exps_ptr))};
}

// A new one: one buffer, codes before exponents.
struct NewForm {
    Tensor both;
    Form form;
    NewForm(int64_t rows, int64_t cols, const Tensor &like)
    {
        const int64_t blocks = (cols + 31) / 32;
        both = at::empty({rows * blocks * 33}, like.options().dtype(at::kByte));
        form.codes = static_cast<int8_t *>(both.data_ptr());
        form.exps = static_cast<uint8_t *>(both.data_ptr()) + rows * blocks * 32;
    }
};

Tensor new_like(const Tensor &t) { return at::empty(t.sizes(), t.options()); }

// The C entry points, set by bind().
#define NOVAK_ENTRIES(X)                                                                                               \
    X(novak_act8_pack) X(novak_act8_unpack) X(novak_layer_norm) X(novak_layer_norm_backward_bytes)                     \
    X(novak_layer_norm_backward) X(novak_activation) X(novak_activation_backward) X(novak_linear_weight_grad_bytes)    \
    X(novak_linear_weight_grad) X(novak_rms_norm) X(novak_rms_norm_backward_bytes) X(novak_rms_norm_backward)          \
    X(novak_embedding) X(novak_embedding_grad_bytes) X(novak_embedding_grad) X(novak_orthogonalize_bytes)              \
    X(novak_orthogonalize) X(novak_orthogonal_step) X(novak_orthogonalize_fine_bytes) X(novak_orthogonalize_fine)      \
    X(novak_orthogonal_step_fine) X(novak_ops_error)
struct Api {
#define X(f) decltype(&::f) f = nullptr;
    NOVAK_ENTRIES(X)
#undef X
} api;

void *stream_of(const Tensor &t) { return c10::cuda::getCurrentCUDAStream(t.get_device()).stream(); }

// Calls a C entry point on a tensor's device and torch's current stream there, without
// the interpreter's lock (a launch waits when the queue is full); a status other than
// NOVAK_OK becomes binding.NovakError, which bind() sets.
PyObject *novak_error = nullptr;
template <class F, class... A> void enqueue(F f, const char *where, const Tensor &on, A... a)
{
    const c10::cuda::CUDAGuard guard(on.device());
    PyThreadState *state = PyEval_SaveThread();
    const int status = f(a..., stream_of(on));
    PyEval_RestoreThread(state);
    if (status == NOVAK_OK) return;
    THPObjectPtr e(PyObject_CallFunction(novak_error, "iss", status, where, api.novak_ops_error()));
    if (e) PyErr_SetObject(novak_error, e.get());
    throw Refused{};
}
#define ENQUEUE(f, on, ...) enqueue(api.f, #f, on, __VA_ARGS__)

// A caller's tensor that has been written to: autograd refuses to go back through what was computed from it before, as
// it does after torch's own operations in place.
void changed(const Tensor &t)
{
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

PyObject *wrap(const Tensor &t) { return THPVariable_Wrap(t); }
PyObject *none_or(const Tensor &t)
{
    if (t.defined()) return THPVariable_Wrap(t);
    Py_RETURN_NONE;
}

bool truth(PyObject *o) { return PyObject_IsTrue(o) == 1; }
bool is_none(PyObject *o) { return o == Py_None; }

int64_t integer(PyObject *o)
{
    const int64_t x = PyLong_AsLongLong(o);
    if (x == -1 && PyErr_Occurred()) throw Refused{};
    return x;
}

// Every entry: N arguments, and C++ exceptions become Python's.
template <PyObject *(*F)(PyObject *const *), int N> PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != N) return PyErr_Format(PyExc_TypeError, "%d arguments are needed, got %zd", N, n);
    try {
        return F(args);
    } catch (const Refused &) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// act8_pack(x) -> buffer
PyObject *pack(PyObject *const *args)
{
    const Tensor &x = tensor(args[0], "x");
    const Rows r = rows_of(x, "x");
    const int type = type_of(x, "x");
    const NewForm f(r.rows, r.cols, x);
    ENQUEUE(novak_act8_pack, x, x.data_ptr(), r.stride, type, f.form.codes, f.form.exps, r.rows, r.cols);
    return wrap(f.both);
}

// act8_unpack(kept, out)
PyObject *unpack(PyObject *const *args)
{
    const Tensor &out = tensor(args[1], "out");
    const int64_t cols = attribute(args[0], names.cols), rows = attribute(args[0], names.rows);
    const Form f = form_of(args[0], rows, cols, out, "out");
    if (cols < 1 || !out.is_contiguous() || out.numel() / cols != rows || out.numel() % cols != 0)
        value_error("%s must be contiguous and hold the 8-bit form's elements", "out");
    ENQUEUE(novak_act8_unpack, out, f.codes, f.exps, out.data_ptr(), cols, type_of(out, "dtype"), rows, cols);
    Py_RETURN_NONE;
}

// layer_norm(x, weight, bias, eps, checkpoint) -> (y, mean, rstd, buffer or None)
PyObject *layer_norm(PyObject *const *args)
{
    const Tensor &x = tensor(args[0], "x"), &weight = tensor(args[1], "weight");
    const Rows r = rows_of(x, "x");
    const int type = type_of(x, "x"), param = vector_type(weight, "weight", x, r.cols);
    const void *bias = nullptr;
    if (!is_none(args[2])) {
        const Tensor &b = tensor(args[2], "bias");
        if (vector_type(b, "bias", x, r.cols) != param) {
            PyErr_SetString(PyExc_TypeError, "weight and bias must have one dtype");
            throw Refused{};
        }
        bias = b.data_ptr();
    }
    const double eps = PyFloat_AsDouble(args[3]);
    if (eps == -1.0 && PyErr_Occurred()) throw Refused{};
    const Tensor y = new_like(x);
    c10::DimVector shape{2};                    // both statistics in one buffer
    shape.append(x.sizes().begin(), x.sizes().end() - 1);
    const Tensor stats = at::empty(shape, x.options().dtype(at::kFloat));
    const Tensor mean = stats.select(0, 0), rstd = stats.select(0, 1);
    Form f;
    Tensor both;
    if (truth(args[4])) {
        const NewForm n(r.rows, r.cols, x);
        f = n.form;
        both = n.both;
    }
    ENQUEUE(novak_layer_norm, x, x.data_ptr(), r.stride, y.data_ptr(), r.cols, type, weight.data_ptr(), bias, param,
            eps, static_cast<float *>(mean.data_ptr()), static_cast<float *>(rstd.data_ptr()), f.codes, f.exps,
            r.rows, r.cols);
    return Py_BuildValue("(NNNN)", wrap(y), wrap(mean), wrap(rstd), none_or(both));
}

// layer_norm_backward(dy, kept or None, x or None, mean or None, rstd, weight, gradients' type) -> (dx, dw, db)
PyObject *layer_norm_backward(PyObject *const *args)
{
    const Tensor &dy = tensor(args[0], "dy"), &weight = tensor(args[5], "weight");
    const Rows r = rows_of(dy, "dy");
    const int type = type_of(dy, "dy"), param = vector_type(weight, "weight", dy, r.cols);
    const int grad = static_cast<int>(integer(args[6]));
    const auto stats = dy.sizes().slice(0, dy.dim() - 1);
    const Tensor rstd = floats(tensor(args[4], "rstd"), "rstd", dy, stats);
    Form f;
    Tensor mean;
    const void *x_ptr = nullptr;
    int64_t x_stride = 0;
    if (!is_none(args[1])) {
        f = form_of(args[1], r.rows, r.cols, dy, "dy");
    } else {
        const Tensor &x = tensor(args[2], "x");
        same(x, "x", dy, dy.sizes());
        if (x.scalar_type() != dy.scalar_type()) {
            PyErr_SetString(PyExc_TypeError, "x and dy must have one dtype");
            throw Refused{};
        }
        mean = floats(tensor(args[3], "mean"), "mean", dy, stats);
        x_stride = rows_of(x, "x").stride;
        x_ptr = x.data_ptr();
    }
    const Tensor dx = new_like(dy);
    const auto options = dy.options().dtype(grad == NOVAK_TYPE_BF16 ? at::kBFloat16 : at::kFloat);
    const Tensor dw = at::empty({r.cols}, options), db = at::empty({r.cols}, options);
    const size_t need = api.novak_layer_norm_backward_bytes(r.rows, r.cols);
    const Tensor work = at::empty({static_cast<int64_t>(need)}, dy.options().dtype(at::kByte));
    ENQUEUE(novak_layer_norm_backward, dy, dy.data_ptr(), r.stride, x_ptr, x_stride, type,
            mean.defined() ? static_cast<const float *>(mean.data_ptr()) : nullptr,
            static_cast<const float *>(rstd.data_ptr()), f.codes, f.exps, weight.data_ptr(), param, dx.data_ptr(),
            r.cols, dw.data_ptr(), db.data_ptr(), grad, work.data_ptr(), need, r.rows, r.cols);
    return Py_BuildValue("(NNN)", wrap(dx), wrap(dw), wrap(db));
}

// activation(u, kind, save_input, save_output) -> (a, buffer or None, buffer or None)
PyObject *activation(PyObject *const *args)
{
    const Tensor &u = tensor(args[0], "u");
    const Rows r = rows_of(u, "u");
    const int type = type_of(u, "u"), kind = static_cast<int>(integer(args[1]));
    const Tensor a = new_like(u);
    Form fu, fa;
    Tensor bu, ba;
    if (truth(args[2])) {
        const NewForm n(r.rows, r.cols, u);
        fu = n.form;
        bu = n.both;
    }
    if (truth(args[3])) {
        const NewForm n(r.rows, r.cols, u);
        fa = n.form;
        ba = n.both;
    }
    ENQUEUE(novak_activation, u, u.data_ptr(), r.stride, a.data_ptr(), r.cols, type, kind, fu.codes, fu.exps,
            fa.codes, fa.exps, r.rows, r.cols);
    return Py_BuildValue("(NNN)", wrap(a), none_or(bu), none_or(ba));
}

// activation_backward(da, kept or None, u or None, kind) -> du
PyObject *activation_backward(PyObject *const *args)
{
    const Tensor &da = tensor(args[0], "da");
    const Rows r = rows_of(da, "da");
    const int type = type_of(da, "da"), kind = static_cast<int>(integer(args[3]));
    Form f;
    const void *u_ptr = nullptr;
    int64_t u_stride = 0;
    if (!is_none(args[1])) {
        f = form_of(args[1], r.rows, r.cols, da, "da");
    } else {
        const Tensor &u = tensor(args[2], "u");
        same(u, "u", da, da.sizes());
        if (u.scalar_type() != da.scalar_type()) {
            PyErr_SetString(PyExc_TypeError, "u and da must have one dtype");
            throw Refused{};
        }
        u_stride = rows_of(u, "u").stride;
        u_ptr = u.data_ptr();
    }
    const Tensor du = new_like(da);
    ENQUEUE(novak_activation_backward, da, da.data_ptr(), r.stride, u_ptr, u_stride, type, kind, f.codes, f.exps,
            du.data_ptr(), r.cols, r.rows, r.cols);
    return wrap(du);
}

// linear_weight_grad(dy, kept, weight or None, bias or None, want db, gradients' type) -> (dw, db or None)
PyObject *linear_weight_grad(PyObject *const *args)
{
    const Tensor &dy = tensor(args[0], "dy");
    const Rows r = rows_of(dy, "dy");
    const int type = type_of(dy, "dy"), grad = static_cast<int>(integer(args[5]));
    const int64_t n_in = attribute(args[1], names.cols);
    const Form f = form_of(args[1], r.rows, 0, dy, "dy");
    const void *w = nullptr, *b = nullptr;
    int param = NOVAK_TYPE_F32;
    if (!is_none(args[2])) {
        const Tensor &weight = tensor(args[2], "weight"), &bias = tensor(args[3], "bias");
        param = vector_type(weight, "weight", dy, n_in);
        if (vector_type(bias, "bias", dy, n_in) != param) {
            PyErr_SetString(PyExc_TypeError, "weight and bias must have one dtype");
            throw Refused{};
        }
        w = weight.data_ptr();
        b = bias.data_ptr();
    }
    const auto options = dy.options().dtype(grad == NOVAK_TYPE_BF16 ? at::kBFloat16 : at::kFloat);
    const Tensor dw = at::empty({r.cols, n_in}, options);
    Tensor db, work;
    if (truth(args[4])) db = at::empty({r.cols}, options);
    const size_t need = api.novak_linear_weight_grad_bytes(dy.data_ptr(), r.stride, type, r.rows, r.cols, n_in);
    if (need > 0) work = at::empty({static_cast<int64_t>(need)}, dy.options().dtype(at::kByte));
    ENQUEUE(novak_linear_weight_grad, dy, dy.data_ptr(), r.stride, type, f.codes, f.exps, w, b, param, dw.data_ptr(),
            db.defined() ? db.data_ptr() : nullptr, grad, need > 0 ? work.data_ptr() : nullptr, need, r.rows, r.cols,
            n_in);
    return Py_BuildValue("(NN)", wrap(dw), none_or(db));
}

// A tensor of the other one's type and shape, or none.
const Tensor *beside(PyObject *o, const char *name, const Tensor &like)
{
    if (is_none(o)) return nullptr;
    const Tensor &t = tensor(o, name);
    same(t, name, like, like.sizes());
    if (t.scalar_type() != like.scalar_type()) {
        PyErr_Format(PyExc_TypeError, "%s must be of the same dtype as the other arguments", name);
        throw Refused{};
    }
    return &t;
}

double number(PyObject *o)
{
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) throw Refused{};
    return x;
}

// rms_norm(x, weight, residual or None, eps, checkpoint) -> (y, h, rstd, buffer or None)
PyObject *rms_norm(PyObject *const *args)
{
    const Tensor &x = tensor(args[0], "x"), &weight = tensor(args[1], "weight");
    const Rows r = rows_of(x, "x");
    const int type = type_of(x, "x"), param = vector_type(weight, "weight", x, r.cols);
    const Tensor *residual = beside(args[2], "residual", x);
    const double eps = number(args[3]);
    const int64_t residual_stride = residual ? rows_of(*residual, "residual").stride : 0;
    const Tensor y = at::empty(x.sizes(), x.options()), h = residual ? at::empty(x.sizes(), x.options()) : x;
    const Tensor rstd = at::empty(x.sizes().slice(0, x.dim() - 1), x.options().dtype(at::kFloat));
    Form f;
    Tensor both;
    if (truth(args[4])) {
        const NewForm n(r.rows, r.cols, x);
        f = n.form;
        both = n.both;
    }
    ENQUEUE(novak_rms_norm, x, x.data_ptr(), r.stride, residual ? residual->data_ptr() : nullptr, residual_stride,
            residual ? h.data_ptr() : nullptr, r.cols, y.data_ptr(), r.cols, type, weight.data_ptr(), param, eps,
            static_cast<float *>(rstd.data_ptr()), f.codes, f.exps, r.rows, r.cols);
    return Py_BuildValue("(NNNN)", wrap(y), wrap(h), wrap(rstd), none_or(both));
}

// rms_norm_backward(dy, kept or None, h or None, rstd, weight, dh or None, gradient's type) -> (dx, dw)
PyObject *rms_norm_backward(PyObject *const *args)
{
    const Tensor &dy = tensor(args[0], "dy"), &weight = tensor(args[4], "weight");
    const Rows r = rows_of(dy, "dy");
    const int type = type_of(dy, "dy"), param = vector_type(weight, "weight", dy, r.cols);
    const int grad = static_cast<int>(integer(args[6]));
    const Tensor rstd = floats(tensor(args[3], "rstd"), "rstd", dy, dy.sizes().slice(0, dy.dim() - 1));
    const Tensor *h = beside(args[2], "h", dy), *dh = beside(args[5], "dh", dy);
    Form f;
    if (!h) f = form_of(args[1], r.rows, r.cols, dy, "dy");
    const int64_t h_stride = h ? rows_of(*h, "h").stride : 0, dh_stride = dh ? rows_of(*dh, "dh").stride : 0;
    const Tensor dx = at::empty(dy.sizes(), dy.options());
    const Tensor dw = at::empty({r.cols}, dy.options().dtype(grad == NOVAK_TYPE_BF16 ? at::kBFloat16 : at::kFloat));
    const size_t need = api.novak_rms_norm_backward_bytes(r.rows, r.cols);
    const Tensor work = at::empty({static_cast<int64_t>(need)}, dy.options().dtype(at::kByte));
    ENQUEUE(novak_rms_norm_backward, dy, dy.data_ptr(), r.stride, dh ? dh->data_ptr() : nullptr, dh_stride,
            h ? h->data_ptr() : nullptr, h_stride, type, static_cast<const float *>(rstd.data_ptr()), f.codes, f.exps,
            weight.data_ptr(), param, dx.data_ptr(), r.cols, dw.data_ptr(), grad, work.data_ptr(), need, r.rows, r.cols);
    return Py_BuildValue("(NN)", wrap(dx), wrap(dw));
}

// Token ids as a dense tensor, and their type.
Tensor ids_of(const Tensor &t, const Tensor &like, int &type)
{
    if (t.device() != like.device()) value_error("%s is on another device", "ids");
    if (t.scalar_type() != at::kLong && t.scalar_type() != at::kInt) {
        PyErr_Format(PyExc_TypeError, "ids must be int64 or int32, got %s", c10::toString(t.scalar_type()));
        throw Refused{};
    }
    type = t.scalar_type() == at::kLong ? NOVAK_ID_I64 : NOVAK_ID_I32;
    return t.contiguous();
}

// A matrix as it stands: rows of any stride.
Rows table_of(const Tensor &t, const char *name)
{
    if (t.dim() != 2) value_error("%s must be a matrix", name);
    if (t.size(0) > 0) return rows_of(t, name);
    if (!t.is_cuda()) value_error("%s must be a CUDA tensor", name);
    if (t.size(1) == 0) value_error("%s needs a last dimension of at least one element", name);
    return {0, t.size(1), t.size(1)};
}

at::ScalarType scalar_of(int type) { return type == NOVAK_TYPE_BF16 ? at::kBFloat16 : at::kFloat; }

// embedding(ids, table, scale, type) -> out
PyObject *embedding(PyObject *const *args)
{
    const Tensor &table = tensor(args[1], "table");
    const Rows r = table_of(table, "table");
    const int type = type_of(table, "table"), out_type = static_cast<int>(integer(args[3]));
    int id_type;
    const Tensor ids = ids_of(tensor(args[0], "ids"), table, id_type);
    const double scale = number(args[2]);
    c10::DimVector shape(ids.sizes().begin(), ids.sizes().end());
    shape.push_back(r.cols);
    const Tensor out = at::empty(shape, table.options().dtype(scalar_of(out_type)));
    ENQUEUE(novak_embedding, table, ids.data_ptr(), id_type, table.data_ptr(), r.stride, type, scale, out.data_ptr(),
            r.cols, out_type, ids.numel(), r.rows, r.cols);
    return wrap(out);
}

// embedding_grad(dout, ids, vocab, scale, type, out or None) -> dtable
PyObject *embedding_grad(PyObject *const *args)
{
    const Tensor &dout = tensor(args[0], "dout");
    const Rows r = rows_of(dout, "dout");
    const int type = type_of(dout, "dout");
    int id_type;
    const Tensor ids = ids_of(tensor(args[1], "ids"), dout, id_type);
    if (ids.sizes() != dout.sizes().slice(0, dout.dim() - 1)) value_error("%s has another shape than dout's leading dimensions", "ids");
    const int64_t vocab = integer(args[2]);
    if (vocab < 0) value_error("%s must be >= 0", "vocab");
    const double scale = number(args[3]);
    const bool add = !is_none(args[5]);
    const Tensor out = add ? tensor(args[5], "out") : at::empty({vocab, r.cols}, dout.options().dtype(scalar_of(static_cast<int>(integer(args[4])))));
    same(out, "out", dout, {vocab, r.cols});
    const Rows o = table_of(out, "out");
    const int64_t tokens = ids.numel();
    const size_t need = api.novak_embedding_grad_bytes(tokens, vocab, r.cols);
    const Tensor work = at::empty({static_cast<int64_t>(need)}, dout.options().dtype(at::kByte));
    ENQUEUE(novak_embedding_grad, dout, dout.data_ptr(), r.stride, type, ids.data_ptr(), id_type, scale, out.data_ptr(),
            o.stride, type_of(out, "out"), static_cast<int>(add), work.data_ptr(), need, tokens, vocab, r.cols);
    if (add) changed(out);
    return wrap(out);
}

// Numbers of a sequence, flattened by the caller.
std::vector<double> numbers(PyObject *o, const char *name)
{
    THPObjectPtr fast(PySequence_Fast(o, name));
    if (!fast) throw Refused{};
    std::vector<double> v(PySequence_Fast_GET_SIZE(fast.get()));
    for (size_t i = 0; i < v.size(); ++i) v[i] = number(PySequence_Fast_GET_ITEM(fast.get(), i));
    return v;
}

struct Tensors {
    THPObjectPtr fast;
    Tensors(PyObject *o, const char *name) : fast(PySequence_Fast(o, name))
    {
        if (!fast) throw Refused{};
    }
    int64_t size() const { return PySequence_Fast_GET_SIZE(fast.get()); }
    const Tensor &at(int64_t i, const char *name) const { return tensor(PySequence_Fast_GET_ITEM(fast.get(), i), name); }
};

// The matrices in a list of tensors: a tensor of more than two dimensions is a batch of them.
struct Matrices {
    std::vector<void *> ptr;
    std::vector<int64_t> rows, cols, stride;
    void add(const Tensor &t, const char *name)
    {
        if (!t.is_cuda()) value_error("%s must be CUDA tensors", name);
        if (t.dim() < 2) value_error("%s must have two dimensions or more", name);
        const int64_t r = t.size(-2), c = t.size(-1), bytes = t.element_size();
        if (t.numel() == 0) return;
        if (c > 1 && t.stride(-1) != 1) value_error("%s: the last dimension must be contiguous", name);
        if (r > 1 && t.stride(-2) < c) value_error("%s: rows overlap", name);
        const int64_t batch = t.numel() / (r * c);
        for (int64_t b = 0; b < batch; ++b) {
            int64_t left = b, at = 0;
            for (int64_t d = t.dim() - 3; d >= 0; --d) {
                at += left % t.size(d) * t.stride(d);
                left /= t.size(d);
            }
            ptr.push_back(static_cast<char *>(t.data_ptr()) + at * bytes);
            rows.push_back(r);
            cols.push_back(c);
            stride.push_back(r > 1 ? t.stride(-2) : c);
        }
    }
    int count() const
    {
        if (ptr.size() > (1u << 14)) value_error("%s: 2^14 of them at most", "matrices");
        return static_cast<int>(ptr.size());
    }
};

// orthogonalize(list, coefficients, eps, fine) -> list
PyObject *orthogonalize(PyObject *const *args)
{
    const Tensors list(args[0], "a list of tensors is needed");
    const std::vector<double> abc = numbers(args[1], "coefficients must be numbers");
    const double eps = number(args[2]);
    THPObjectPtr result(PyList_New(list.size()));
    if (!result) throw Refused{};
    Matrices g, out;
    int type = NOVAK_TYPE_F32;
    std::vector<Tensor> outs;
    for (int64_t i = 0; i < list.size(); ++i) {
        const Tensor &t = list.at(i, "a matrix"), &first = list.at(0, "a matrix");
        const int its = type_of(t, "a matrix");
        if (i == 0) type = its;
        if (its != type || t.device() != first.device()) value_error("%s must be of one dtype and on one device", "matrices");
        g.add(t, "matrices");
        outs.push_back(at::empty(t.sizes(), t.options().dtype(at::kBFloat16)));
        out.add(outs.back(), "matrices");
        PyList_SET_ITEM(result.get(), i, wrap(outs.back()));
    }
    const int n = g.count();
    if (n > 0) {
        const Tensor &on = list.at(0, "a matrix");
        const bool fine = truth(args[3]);
        const size_t need = (fine ? api.novak_orthogonalize_fine_bytes : api.novak_orthogonalize_bytes)(g.rows.data(), g.cols.data(), n);
        const Tensor work = at::empty({static_cast<int64_t>(need)}, on.options().dtype(at::kByte));
        enqueue(fine ? api.novak_orthogonalize_fine : api.novak_orthogonalize, fine ? "novak_orthogonalize_fine" : "novak_orthogonalize", on,
                g.ptr.data(), g.stride.data(), type, out.ptr.data(), out.stride.data(), g.rows.data(), g.cols.data(), n, abc.data(),
                static_cast<int>(abc.size() / 3), eps, work.data_ptr(), need);
    }
    return result.release();
}

// orthogonal_step(parameters, gradients, momenta, momentum, nesterov, steps, decay, coefficients, eps, fine)
PyObject *orthogonal_step(PyObject *const *args)
{
    const Tensors params(args[0], "a list of parameters is needed"), grads(args[1], "a list of gradients is needed"),
        momenta(args[2], "a list of momenta is needed");
    const std::vector<double> each = numbers(args[5], "steps must be numbers"), abc = numbers(args[7], "coefficients must be numbers");
    const double momentum = number(args[3]), decay = number(args[6]), eps = number(args[8]);
    const int64_t count = params.size();
    if (grads.size() != count || momenta.size() != count || static_cast<int64_t>(each.size()) != count)
        value_error("%s must be as many as the parameters", "gradients, momenta and steps");
    Matrices theta, g, m;
    std::vector<double> step;
    int type = NOVAK_TYPE_F32;
    for (int64_t i = 0; i < count; ++i) {
        const Tensor &p = params.at(i, "a parameter"), &gr = grads.at(i, "a gradient"), &mo = momenta.at(i, "a momentum");
        if (i == 0) type = type_of(gr, "a gradient");
        if (type_of(gr, "a gradient") != type) value_error("%s must be of one dtype", "gradients");
        same(gr, "a gradient", params.at(0, "a parameter"), p.sizes());
        same(mo, "a momentum", params.at(0, "a parameter"), p.sizes());
        same(p, "a parameter", params.at(0, "a parameter"), p.sizes());
        if (p.scalar_type() != at::kFloat || mo.scalar_type() != at::kFloat) {
            PyErr_SetString(PyExc_TypeError, "parameters and momenta must be float32");
            throw Refused{};
        }
        if (!p.is_contiguous() || !gr.is_contiguous() || !mo.is_contiguous())
            value_error("%s must be contiguous", "parameters, gradients and momenta");
        theta.add(p, "parameters");
        g.add(gr, "gradients");
        m.add(mo, "momenta");
        step.resize(theta.ptr.size(), each[i]);
    }
    const int n = theta.count();
    if (n > 0) {
        const Tensor &on = params.at(0, "a parameter");
        const bool fine = truth(args[9]);
        const size_t need = (fine ? api.novak_orthogonalize_fine_bytes : api.novak_orthogonalize_bytes)(theta.rows.data(), theta.cols.data(), n);
        const Tensor work = at::empty({static_cast<int64_t>(need)}, on.options().dtype(at::kByte));
        enqueue(fine ? api.novak_orthogonal_step_fine : api.novak_orthogonal_step,
                fine ? "novak_orthogonal_step_fine" : "novak_orthogonal_step", on, reinterpret_cast<float *const *>(theta.ptr.data()), g.ptr.data(), type,
                reinterpret_cast<float *const *>(m.ptr.data()), theta.rows.data(), theta.cols.data(), n, momentum,
                static_cast<int>(truth(args[4])), step.data(), decay, abc.data(), static_cast<int>(abc.size() / 3), eps,
                work.data_ptr(), need);
        for (int64_t i = 0; i < count; ++i) {
            changed(params.at(i, "a parameter"));
            changed(momenta.at(i, "a momentum"));
        }
    }
    Py_RETURN_NONE;
}

// bind(error class, address of each of NOVAK_ENTRIES in that order)
PyObject *bind(PyObject *const *args)
{
    int i = 1;
#define X(f) api.f = reinterpret_cast<decltype(api.f)>(PyLong_AsVoidPtr(args[i++]));
    NOVAK_ENTRIES(X)
#undef X
    if (PyErr_Occurred()) throw Refused{};
    Py_INCREF(args[0]);
    Py_XDECREF(novak_error);
    novak_error = args[0];
    Py_RETURN_NONE;
}

template <PyObject *(*F)(PyObject *const *), int N> PyMethodDef def(const char *name)
{
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<F, N>)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {
    def<bind, 23>("bind"),
    def<pack, 1>("pack"),
    def<unpack, 2>("unpack"),
    def<layer_norm, 5>("layer_norm"),
    def<layer_norm_backward, 7>("layer_norm_backward"),
    def<activation, 4>("activation"),
    def<activation_backward, 4>("activation_backward"),
    def<linear_weight_grad, 6>("linear_weight_grad"),
    def<rms_norm, 5>("rms_norm"),
    def<rms_norm_backward, 7>("rms_norm_backward"),
    def<embedding, 4>("embedding"),
    def<embedding_grad, 6>("embedding_grad"),
    def<orthogonalize, 4>("orthogonalize"),
    def<orthogonal_step, 10>("orthogonal_step"),
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_novak_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__novak_torch()
{
    names.codes_ptr = PyUnicode_InternFromString("codes_ptr");
    names.exps_ptr = PyUnicode_InternFromString("exps_ptr");
    names.rows = PyUnicode_InternFromString("rows");
    names.cols = PyUnicode_InternFromString("cols");
    names.index = PyUnicode_InternFromString("index");
    return PyModule_Create(&module);
}
