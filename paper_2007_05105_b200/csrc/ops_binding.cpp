// Python binding of the language-model operators (adascale_ops.h): checks tensors, makes results and
// workspaces in torch's caching allocator, fills in the argument structs and calls the C ABI on the
// current stream.  Argument handling only; ops.py has the signatures and their documentation.
//
// Why not ctypes as for the AdaScale step: that is called once per iteration with arrays of
// addresses that are built once, these are called dozens of times with tensors of their own.  For one
// row of 1024 the Python code of a call took 18 to 23 us around a kernel of 3 us.
#include "../../include/adascale_ops.h"

#include <ATen/ATen.h>
#include <ATen/TensorUtils.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdarg>
#include <cstdio>
#include <optional>
#include <string>

namespace {

// Raised as ValueError (or TypeError) by the entry points.
struct Refused {
    PyObject *kind;
    std::string text;
};
[[noreturn]] void refuse(const char *format, ...)
{
    char text[256];
    va_list args;
    va_start(args, format);
    vsnprintf(text, sizeof text, format, args);
    va_end(args);
    throw Refused{PyExc_ValueError, text};
}

const at::Tensor *tensor(PyObject *o, const char *what)
{
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) throw Refused{PyExc_TypeError, std::string(what) + " is not a tensor"};
    return &THPVariable_Unpack(o);
}
const at::Tensor &wanted(PyObject *o, const char *what)
{
    const at::Tensor *t = tensor(o, what);
    if (!t) throw Refused{PyExc_TypeError, std::string(what) + " is missing"};
    return *t;
}
double number(PyObject *o, const char *what)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Refused{PyExc_TypeError, std::string(what) + " is not a number"};
    }
    return v;
}
int64_t whole(PyObject *o, const char *what)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Refused{PyExc_TypeError, std::string(what) + " is not an integer"};
    }
    return v;
}

bool truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw python_error();  // the error that is pending
    return v;
}

int float_code(at::ScalarType t, const char *what)
{
    if (t == at::kFloat) return ADASCALE_F32;
    if (t == at::kBFloat16) return ADASCALE_BF16;
    refuse("%s: %s is neither float32 nor bfloat16", what, c10::toString(t));
}
int id_code(at::ScalarType t, const char *what)
{
    if (t == at::kInt) return ADASCALE_I32;
    if (t == at::kLong) return ADASCALE_I64;
    refuse("%s: %s is neither int32 nor int64", what, c10::toString(t));
}
at::ScalarType type_of(PyObject *o, at::ScalarType none)
{
    if (o == Py_None) return none;
    if (!THPDtype_Check(o)) throw Refused{PyExc_TypeError, "a dtype is expected"};
    return reinterpret_cast<THPDtype *>(o)->scalar_type;
}

struct Shape {
    int64_t n, d;
};
Shape rows_of(const at::Tensor &t, const char *what)
{
    if (!t.is_cuda()) refuse("%s: the operators take CUDA tensors", what);
    if (t.dim() == 0) refuse("%s: a scalar has no rows", what);
    const int64_t d = t.size(-1);
    return {t.dim() == 2 ? t.size(0) : d ? t.numel() / d : 0, d};
}

// Address and row stride of n rows of d elements (leading dimensions are one).
struct Matrix {
    void *p = nullptr;
    int64_t ld = 0;
};
Matrix matrix(const at::Tensor &t, int64_t n, int64_t d, at::Device device, const char *what)
{
    if (t.device() != device) refuse("%s is on %s, not on %s", what, t.device().str().c_str(), device.str().c_str());
    if (t.dim() != 2) {
        if (t.dim() == 0 || t.size(-1) != d || t.numel() != n * d) refuse("%s: not %lld rows of %lld", what, (long long)n, (long long)d);
        if (!at::detail::computeStride(t.sizes(), t.strides(), c10::IntArrayRef({n, d}))) refuse("%s: its rows have no common stride", what);
        return matrix(t.view({n, d}), n, d, device, what);
    }
    if (t.size(0) != n || t.size(1) != d)
        refuse("%s: shape (%lld, %lld), not %lld rows of %lld", what, (long long)t.size(0), (long long)t.size(1), (long long)n, (long long)d);
    if (d > 1 && t.stride(1) != 1) refuse("%s: the last dimension is not contiguous", what);
    if (n > 1 && t.stride(0) < d) refuse("%s: rows overlap (row stride %lld, %lld elements)", what, (long long)t.stride(0), (long long)d);
    return {t.data_ptr(), n > 1 ? t.stride(0) : d};
}
void *vector(const at::Tensor &t, int64_t n, at::Device device, const char *what)
{
    if (t.device() != device || t.numel() != n || !t.is_contiguous())
        refuse("%s: want %lld contiguous elements on %s", what, (long long)n, device.str().c_str());
    return t.data_ptr();
}
float *f32_vector(const at::Tensor *t, int64_t n, at::Device device, const char *what)
{
    if (!t) return nullptr;
    if (t->scalar_type() != at::kFloat) refuse("%s: %s is not float32", what, c10::toString(t->scalar_type()));
    return static_cast<float *>(vector(*t, n, device, what));
}
void same_type(const at::Tensor &t, at::ScalarType type, const char *what)
{
    if (t.scalar_type() != type) refuse("%s is %s, not %s", what, c10::toString(t.scalar_type()), c10::toString(type));
}

at::Tensor make(at::IntArrayRef shape, at::ScalarType type, at::Device device)
{
    return at::detail::empty_cuda(shape, type, device, std::nullopt);
}
// A workspace: the given one, bytes that lie adjacent on the device, or a new one.
struct Room {
    at::Tensor t;
    void *p;
    int64_t bytes;
    Room(PyObject *given, int64_t need, at::Device device)
    {
        if (const at::Tensor *g = tensor(given, "workspace")) {
            same_type(*g, at::kByte, "workspace");
            t = *g;
        } else {
            t = make({need}, at::kByte, device);
        }
        bytes = t.numel();
        p = vector(t, bytes, device, "workspace");
    }
};
// Vectors that are made together share one allocation: each of its own cost 0.8 us, of the 13.7 us of a
// gradient call of the block boundary.  Starts are 256 bytes apart.
class Together {
  public:
    Together(int count, int64_t n, at::ScalarType type, at::Device device)
        : n_(n), step_((n + 127) / 128 * 128), base_(make({count * step_}, type, device))
    {
    }
    at::Tensor next(bool scalar = false)
    {
        at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(base_.storage()), base_.key_set(), base_.dtype());
        t.unsafeGetTensorImpl()->set_storage_offset(used_++ * step_);
        if (scalar) t.unsafeGetTensorImpl()->set_sizes_contiguous({});
        else t.unsafeGetTensorImpl()->set_sizes_contiguous({n_});
        return t;
    }

  private:
    int64_t n_, step_, used_ = 0;
    at::Tensor base_;
};

// The given tensor, or a new one.
at::Tensor given_or_new(const at::Tensor *t, at::IntArrayRef shape, at::ScalarType type, at::Device device, const char *what)
{
    if (!t) return make(shape, type, device);
    same_type(*t, type, what);
    return *t;
}

// Tells torch that a tensor of the caller's has been written to: what was saved of it for a backward pass is not valid any more.
void written(const at::Tensor *given)
{
    if (given && !given->is_inference()) given->unsafeGetTensorImpl()->bump_version();
}

void *stream_of(at::Device device) { return c10::cuda::getCurrentCUDAStream(device.index()).stream(); }

PyObject *adascale_error = nullptr;  // binding.AdaScaleError

PyObject *status_error(adascale_status s)
{
    if (PyObject *e = PyObject_CallFunction(adascale_error, "is", (int)s, adascale_strerror(s))) {
        PyErr_SetObject(adascale_error, e);
        Py_DECREF(e);
    }
    return nullptr;
}

PyObject *wrap(const at::Tensor &t) { return THPVariable_Wrap(t); }
PyObject *wrap_or_none(const at::Tensor &t)
{
    if (t.defined()) return THPVariable_Wrap(t);
    Py_RETURN_NONE;
}

// Entry points are called by ops.py with all arguments by position.
template <PyObject *(*BODY)(PyObject *const *), int COUNT> PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != COUNT) {
        PyErr_Format(PyExc_TypeError, "%d arguments expected, %zd given", COUNT, n);
        return nullptr;
    }
    try {
        return BODY(args);
    } catch (const Refused &r) {
        PyErr_SetString(r.kind, r.text.c_str());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// tokens, table, scale, out, out_dtype
PyObject *embed(PyObject *const *o)
{
    const at::Tensor &tokens = wanted(o[0], "tokens"), &table = wanted(o[1], "table");
    if (!table.is_cuda() || table.dim() != 2) refuse("table: a [vocab, dim] matrix on a CUDA device is expected");
    const at::Device device = table.device();
    const c10::cuda::CUDAGuard guard(device);
    adascale_embed_args a = {};
    a.vocab = table.size(0);
    a.dim = table.size(1);
    a.n_tokens = tokens.numel();
    const at::Tensor *given = tensor(o[3], "out");
    at::ScalarType type = type_of(o[4], given ? given->scalar_type() : table.scalar_type());
    a.table_dtype = float_code(table.scalar_type(), "table");
    a.out_dtype = float_code(type, "out");
    a.token_type = id_code(tokens.scalar_type(), "tokens");
    a.tokens = vector(tokens, a.n_tokens, device, "tokens");
    c10::DimVector shape(tokens.sizes());
    shape.push_back(a.dim);
    const at::Tensor out = given_or_new(given, shape, type, device, "out");
    Matrix m = matrix(table, a.vocab, a.dim, device, "table");
    a.table = m.p;
    a.ld_table = m.ld;
    m = matrix(out, a.n_tokens, a.dim, device, "out");
    a.out = m.p;
    a.ld_out = m.ld;
    a.scale = (float)number(o[2], "scale");
    const adascale_status s = adascale_embed(&a, stream_of(device));
    if (s != ADASCALE_OK) return status_error(s);
    written(given);
    return wrap(out);
}

// tokens, dout, grad, scale, padding_idx, accumulate, workspace
PyObject *embed_grad(PyObject *const *o)
{
    const at::Tensor &tokens = wanted(o[0], "tokens"), &dout = wanted(o[1], "dout"), &grad = wanted(o[2], "grad");
    if (!grad.is_cuda() || grad.dim() != 2) refuse("grad: a [vocab, dim] matrix on a CUDA device is expected");
    const at::Device device = grad.device();
    const c10::cuda::CUDAGuard guard(device);
    adascale_embed_grad_args a = {};
    a.vocab = grad.size(0);
    a.dim = grad.size(1);
    a.n_tokens = tokens.numel();
    a.dout_dtype = float_code(dout.scalar_type(), "dout");
    a.grad_dtype = float_code(grad.scalar_type(), "grad");
    a.token_type = id_code(tokens.scalar_type(), "tokens");
    a.tokens = vector(tokens, a.n_tokens, device, "tokens");
    Matrix m = matrix(dout, a.n_tokens, a.dim, device, "dout");
    a.dout = m.p;
    a.ld_dout = m.ld;
    m = matrix(grad, a.vocab, a.dim, device, "grad");
    a.grad = m.p;
    a.ld_grad = m.ld;
    a.scale = (float)number(o[3], "scale");
    a.padding_idx = whole(o[4], "padding_idx");
    a.accumulate = truth(o[5]);
    const Room room(o[6], adascale_embed_grad_workspace(a.n_tokens, a.dim), device);
    a.workspace = room.p;
    a.workspace_bytes = room.bytes;
    const adascale_status s = adascale_embed_grad(&a, stream_of(device));
    if (s != ADASCALE_OK) return status_error(s);
    written(&grad);
    Py_INCREF(o[2]);
    return o[2];
}

// logits, teacher_logits, teacher_ids, labels, T, alpha, beta, row_weight, want_grad, dlogits
PyObject *distill(PyObject *const *o)
{
    const at::Tensor &logits = wanted(o[0], "logits");
    const Shape shape = rows_of(logits, "logits");
    const at::Device device = logits.device();
    const c10::cuda::CUDAGuard guard(device);
    const at::Tensor *t = tensor(o[1], "teacher_logits"), *ids = tensor(o[2], "teacher_ids"), *labels = tensor(o[3], "labels"),
                     *weight = tensor(o[7], "row_weight"), *given = tensor(o[9], "dlogits");
    adascale_distill_args a = {};
    a.n_rows = shape.n;
    a.vocab = shape.d;
    a.dtype = float_code(logits.scalar_type(), "logits");
    Matrix m = matrix(logits, shape.n, shape.d, device, "logits");
    a.logits = m.p;
    a.ld_logits = m.ld;
    if (!t != !ids) refuse("teacher_logits and teacher_ids come together");
    if (t) {
        if (ids->dim() == 0) refuse("teacher_ids: a scalar has no rows");
        a.n_top = ids->size(-1);
        m = matrix(*t, shape.n, a.n_top, device, "teacher_logits");
        a.teacher_logits = m.p;
        a.ld_teacher = m.ld;
        m = matrix(*ids, shape.n, a.n_top, device, "teacher_ids");
        a.teacher_ids = m.p;
        a.ld_ids = m.ld;
        a.teacher_dtype = float_code(t->scalar_type(), "teacher_logits");
        a.id_type = id_code(ids->scalar_type(), "teacher_ids");
    }
    if (labels) {
        a.label_type = id_code(labels->scalar_type(), "labels");
        a.labels = vector(*labels, shape.n, device, "labels");
    }
    a.weight = f32_vector(weight, shape.n, device, "row_weight");
    a.temperature = (float)number(o[4], "T");
    a.alpha = (float)number(o[5], "alpha");
    a.beta = (float)number(o[6], "beta");
    at::Tensor dlogits;
    if (given || truth(o[8])) {
        dlogits = given_or_new(given, logits.sizes(), logits.scalar_type(), device, "dlogits");
        m = matrix(dlogits, shape.n, shape.d, device, "dlogits");
        a.dlogits = m.p;
        a.ld_dlogits = m.ld;
    }
    Together room(2, shape.n > 0 ? shape.n : 1, at::kFloat, device);
    const at::Tensor loss = room.next(true), row_loss = shape.n > 0 ? room.next() : make({0}, at::kFloat, device);
    a.row_loss = static_cast<float *>(row_loss.data_ptr());
    a.loss = static_cast<float *>(loss.data_ptr());
    const adascale_status s = adascale_distill(&a, stream_of(device));
    if (s != ADASCALE_OK) return status_error(s);
    written(given);
    return Py_BuildValue("(NNN)", wrap(loss), wrap(row_loss), wrap_or_none(dlogits));
}

// A gate: a float32 vector over the channels, or a matrix of y's type.
int gate_of(const at::Tensor *gate, const Shape &shape, const at::Tensor &y, at::Device device, const void *&p, int64_t &ld)
{
    if (!gate) return ADASCALE_GATE_NONE;
    if (gate->dim() == 1) {
        p = f32_vector(gate, shape.d, device, "gate");
        return ADASCALE_GATE_CHANNEL;
    }
    same_type(*gate, y.scalar_type(), "gate");
    const Matrix m = matrix(*gate, shape.n, shape.d, device, "gate");
    p = m.p;
    ld = m.ld;
    return ADASCALE_GATE_SIGMOID;
}

// x, y, w_pre, b_pre, w_post, b_post, pre, post, gate, res_scale, eps, x_new, h
PyObject *residual_norm(PyObject *const *o)
{
    const at::Tensor &x = wanted(o[0], "x"), &w_pre = wanted(o[2], "w_pre");
    const at::Tensor *y = tensor(o[1], "y"), *b_pre = tensor(o[3], "b_pre"), *w_post = tensor(o[4], "w_post"), *b_post = tensor(o[5], "b_post"),
                     *gate = tensor(o[8], "gate"), *given_x = tensor(o[11], "x_new"), *given_h = tensor(o[12], "h");
    const Shape shape = rows_of(x, "x");
    const at::Device device = x.device();
    const c10::cuda::CUDAGuard guard(device);
    adascale_residual_norm_args a = {};
    a.n_rows = shape.n;
    a.dim = shape.d;
    a.pre = (int32_t)whole(o[6], "pre");
    a.post = (int32_t)whole(o[7], "post");
    a.res_scale = (float)number(o[9], "res_scale");
    a.eps = (float)number(o[10], "eps");
    a.x_dtype = float_code(x.scalar_type(), "x");
    Matrix m = matrix(x, shape.n, shape.d, device, "x");
    a.x = m.p;
    a.ld_x = m.ld;
    at::Tensor x_new, h;
    if (y) {
        x_new = given_or_new(given_x, x.sizes(), x.scalar_type(), device, "x_new");
        h = given_or_new(given_h, x.sizes(), y->scalar_type(), device, "h");
        m = matrix(*y, shape.n, shape.d, device, "y");
        a.y = m.p;
        a.ld_y = m.ld;
        m = matrix(x_new, shape.n, shape.d, device, "x_new");
        a.x_new = m.p;
        a.ld_x_new = m.ld;
        a.gate_kind = gate_of(gate, shape, *y, device, a.gate, a.ld_gate);
    } else {
        h = given_h ? *given_h : make(x.sizes(), x.scalar_type(), device);
    }
    a.y_dtype = float_code(h.scalar_type(), "h");
    m = matrix(h, shape.n, shape.d, device, "h");
    a.h = m.p;
    a.ld_h = m.ld;
    a.w_pre = f32_vector(&w_pre, shape.d, device, "w_pre");
    a.b_pre = f32_vector(b_pre, shape.d, device, "b_pre");
    a.w_post = f32_vector(w_post, shape.d, device, "w_post");
    a.b_post = f32_vector(b_post, shape.d, device, "b_post");
    const adascale_status s = adascale_residual_norm(&a, stream_of(device));
    if (s != ADASCALE_OK) return status_error(s);
    if (y) written(given_x);
    written(given_h);
    PyObject *new_x = y ? wrap(x_new) : (Py_INCREF(o[0]), o[0]);
    return Py_BuildValue("(NN)", new_x, wrap(h));
}

// x_new, y, dx_new, dh, w_pre, w_post, b_post, pre, post, gate, res_scale, eps, wgrad_dtype,
// dx, dy, dgate, dw_post, db_post, dw_pre, db_pre, workspace
PyObject *residual_norm_grad(PyObject *const *o)
{
    const at::Tensor &x = wanted(o[0], "x_new"), &dh = wanted(o[3], "dh"), &w_pre = wanted(o[4], "w_pre");
    const at::Tensor *y = tensor(o[1], "y"), *dx_new = tensor(o[2], "dx_new"), *w_post = tensor(o[5], "w_post"),
                     *b_post = tensor(o[6], "b_post"), *gate = tensor(o[9], "gate");
    const Shape shape = rows_of(x, "x_new");
    const at::Device device = x.device();
    const c10::cuda::CUDAGuard guard(device);
    const at::ScalarType wtype = type_of(o[12], at::kFloat);
    adascale_residual_norm_grad_args a = {};
    a.n_rows = shape.n;
    a.dim = shape.d;
    a.pre = (int32_t)whole(o[7], "pre");
    a.post = y ? (int32_t)whole(o[8], "post") : ADASCALE_NORM_NONE;
    a.res_scale = (float)number(o[10], "res_scale");
    a.eps = (float)number(o[11], "eps");
    a.x_dtype = float_code(x.scalar_type(), "x_new");
    a.y_dtype = float_code(dh.scalar_type(), "dh");
    a.wgrad_dtype = float_code(wtype, "wgrad_dtype");

    auto rows = [&](const at::Tensor &t, at::ScalarType type, const char *what, int64_t &ld) {
        same_type(t, type, what);
        const Matrix m = matrix(t, shape.n, shape.d, device, what);
        ld = m.ld;
        return m.p;
    };
    c10::SmallVector<const at::Tensor *, 8> given_ones;
    auto new_rows = [&](PyObject *given, at::ScalarType type, const char *what, int64_t &ld, void *&p) {
        given_ones.push_back(tensor(given, what));
        const at::Tensor t = given_or_new(given_ones.back(), x.sizes(), type, device, what);
        p = rows(t, type, what, ld);
        return t;
    };
    std::optional<Together> vectors;
    auto new_vector = [&](bool asked, PyObject *given, const char *what, void *&p) {
        if (!asked) return at::Tensor();
        if (given == Py_None) {
            if (!vectors) vectors.emplace(5, shape.d, wtype, device);
            const at::Tensor t = vectors->next();
            p = t.data_ptr();
            return t;
        }
        given_ones.push_back(tensor(given, what));
        const at::Tensor t = given_or_new(given_ones.back(), {shape.d}, wtype, device, what);
        p = vector(t, shape.d, device, what);
        return t;
    };
    a.x_new = rows(x, x.scalar_type(), "x_new", a.ld_x_new);
    a.dh = rows(dh, dh.scalar_type(), "dh", a.ld_dh);
    if (dx_new) a.dx_new = rows(*dx_new, x.scalar_type(), "dx_new", a.ld_dx_new);
    const at::Tensor dx = new_rows(o[13], x.scalar_type(), "dx", a.ld_dx, a.dx);
    at::Tensor dy, dgate;
    if (y) {
        a.y = rows(*y, dh.scalar_type(), "y", a.ld_y);
        dy = new_rows(o[14], dh.scalar_type(), "dy", a.ld_dy, a.dy);
        a.gate_kind = gate_of(gate, shape, *y, device, a.gate, a.ld_gate);
        if (a.gate_kind == ADASCALE_GATE_SIGMOID) dgate = new_rows(o[15], dh.scalar_type(), "dgate", a.ld_dgate, a.dgate);
        else dgate = new_vector(a.gate_kind == ADASCALE_GATE_CHANNEL, o[15], "dgate", a.dgate);
    }
    const at::Tensor dw_post = new_vector(a.post != ADASCALE_NORM_NONE, o[16], "dw_post", a.dw_post);
    const at::Tensor db_post = new_vector(a.post == ADASCALE_NORM_LAYER, o[17], "db_post", a.db_post);
    const at::Tensor dw_pre = new_vector(true, o[18], "dw_pre", a.dw_pre);
    const at::Tensor db_pre = new_vector(a.pre == ADASCALE_NORM_LAYER, o[19], "db_pre", a.db_pre);
    a.w_pre = f32_vector(&w_pre, shape.d, device, "w_pre");
    a.w_post = f32_vector(w_post, shape.d, device, "w_post");
    a.b_post = f32_vector(b_post, shape.d, device, "b_post");
    const Room room(o[20], adascale_residual_norm_grad_workspace(shape.n, shape.d), device);
    a.workspace = room.p;
    a.workspace_bytes = room.bytes;
    const adascale_status s = adascale_residual_norm_grad(&a, stream_of(device));
    if (s != ADASCALE_OK) return status_error(s);
    for (const at::Tensor *t : given_ones) written(t);
    return Py_BuildValue("(NNNNNNN)", wrap(dx), wrap_or_none(dy), wrap_or_none(dgate), wrap_or_none(dw_post), wrap_or_none(db_post),
                         wrap(dw_pre), wrap_or_none(db_pre));
}

#define ENTRY(name, count) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(&entry<name, count>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(embed, 5), ENTRY(embed_grad, 7), ENTRY(distill, 10), ENTRY(residual_norm, 13), ENTRY(residual_norm_grad, 21),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ops_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject *PyInit__ops_binding()
{
    PyObject *binding = PyImport_ImportModule("paper_2007_05105_b200.binding");
    if (!binding) return nullptr;
    adascale_error = PyObject_GetAttrString(binding, "AdaScaleError");
    Py_DECREF(binding);
    return adascale_error ? PyModule_Create(&module) : nullptr;
}
