// The calls of head_binding.py as one native call each: the checks of the tensors, the outputs, the workspace, the current
// stream and the launch.  The smallest calls are a few microseconds of GPU time, and the same steps one by one in Python
// took two to four times that.
//
// A CPython extension on torch's C++ interface.  It is given the addresses of the library's entry points (bind) and knows nothing
// else of the library but head.h.  What it does not take (anything but plain contiguous tensors of the current device that fit
// each other and of which autograd wants no record, active torch function or dispatch modes) it declines with None, and the caller goes the general way, whose
// checks raise the errors; an entry point's error code is returned as an int.
#include <Python.h>

#include <ATen/EmptyTensor.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/grad_mode.h>
#include <ATen/core/Tensor.h>
#include <ATen/hip/impl/HIPCachingAllocatorMasqueradingAsCUDA.h>
#include <ATen/ops/empty.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstdint>
#include <utility>
#include <vector>

#include "../../include/head.h"

namespace {

// The entry points, in the order in which bind() takes them.
struct Entries {
    decltype(&head_embed) embed;
    decltype(&head_embed_grad_bytes) embed_grad_bytes;
    decltype(&head_embed_grad) embed_grad;
    decltype(&head_layer_norm) layer_norm;
    decltype(&head_layer_norm_grad_bytes) layer_norm_grad_bytes;
    decltype(&head_layer_norm_grad) layer_norm_grad;
    decltype(&head_cross_entropy_bytes) cross_entropy_bytes;
    decltype(&head_cross_entropy) cross_entropy;
    decltype(&head_cross_entropy_grad_bytes) cross_entropy_grad_bytes;
    decltype(&head_cross_entropy_grad) cross_entropy_grad;
    decltype(&head_adamw) adamw;
    decltype(&head_adamw_values) adamw_values;
    decltype(&head_linear_bytes) linear_bytes;
    decltype(&head_linear) linear;
    decltype(&head_linear_grad_bytes) linear_grad_bytes;
    decltype(&head_linear_grad) linear_grad;
    decltype(&head_gated_bytes) gated_bytes;
    decltype(&head_gated) gated;
    decltype(&head_gated_grad_bytes) gated_grad_bytes;
    decltype(&head_gated_grad) gated_grad;
    decltype(&head_clip_bytes) clip_bytes;
    decltype(&head_clip) clip;
} entry;
constexpr Py_ssize_t ENTRIES = sizeof(entry) / sizeof(void *);

PyObject *declined() { Py_RETURN_NONE; }

bool modes() { return at::impl::PythonTorchFunctionTLS::stack_len() > 0 || c10::impl::TorchDispatchModeTLS::any_modes_set(); }

// A plain contiguous device tensor; null otherwise.
const at::Tensor *plain(PyObject *o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.is_cuda() && t.layout() == at::kStrided && t.has_storage() && !t.is_conj() && !t.is_neg() && t.is_contiguous() ? &t : nullptr;
}

// One of which autograd wants no record: no gradient, no tangent.
const at::Tensor *tensor(PyObject *o)
{
    const at::Tensor *t = plain(o);
    if (!t || !t->unsafeGetTensorImpl()->autograd_meta()) return t;
    return (t->requires_grad() && at::GradMode::is_enabled()) || t->_fw_grad(0).defined() ? nullptr : t;
}

bool of_current_device(const at::Tensor &t) { return t.get_device() == c10::hip::current_device(); }

// head.h's number of a type; -1: none of them.
int32_t dtype_of(const at::Tensor &t)
{
    return t.scalar_type() == at::kFloat ? HEAD_F32 : t.scalar_type() == at::kBFloat16 ? HEAD_BF16 : -1;
}

bool fits(const at::Tensor *t, const at::Tensor &like, at::ScalarType type, at::IntArrayRef shape)
{
    return t && t->scalar_type() == type && t->device() == like.device() && t->sizes() == shape;
}

void *stream_of(const at::Tensor &like) { return c10::hip::getCurrentHIPStream(like.get_device()).stream(); }

// A new contiguous tensor of the current device, as at::empty makes it, without the dispatcher's half microsecond.
at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType type)
{
    return at::Tensor(at::detail::empty_generic(sizes, c10::hip::HIPCachingAllocatorMasqueradingAsCUDA::get(),
                                                c10::DispatchKeySet(c10::DispatchKey::CUDA), type, c10::nullopt));
}

at::Tensor workspace(int64_t bytes, const at::Tensor &like) { return at::empty({bytes}, like.options().dtype(at::kByte)); }

// A new tuple of tensors; an undefined one is None.
template <class... T>
PyObject *tuple_of(T &&...t)
{
    const at::Tensor all[] = {t...};
    constexpr int N = sizeof...(T);
    PyObject *o = PyTuple_New(N);
    for (int i = 0; o && i < N; ++i) {
        PyObject *one = all[i].defined() ? THPVariable_Wrap(all[i]) : Py_NewRef(Py_None);
        if (!one) {
            Py_DECREF(o);
            return nullptr;
        }
        PyTuple_SET_ITEM(o, i, one);
    }
    return o;
}

template <class Call>
int without_gil(Call call)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return rc;
}

bool ids_of(PyObject *ids_object, PyObject *offsets_object, const at::Tensor &like, int64_t n_vectors, head_ids &out)
{
    const at::Tensor *ids = tensor(ids_object);
    if (!ids || ids->scalar_type() != at::kInt || ids->device() != like.device() || ids->dim() < 1 || ids->dim() > 2) return false;
    const int64_t n_ids = ids->dim() == 2 ? ids->size(1) : 1;
    out = head_ids{ids->size(0), n_ids, n_vectors, static_cast<const int32_t *>(ids->data_ptr()), n_ids, nullptr};
    if (offsets_object == Py_None) return true;
    const at::Tensor *offsets = tensor(offsets_object);
    if (!fits(offsets, like, at::kLong, {n_ids})) return false;
    out.offset = static_cast<const int64_t *>(offsets->data_ptr());
    return true;
}

// embed(table, ids, offsets, scale)
PyObject *embed(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *table = n == 4 ? tensor(args[0]) : nullptr;
    const double scale = n == 4 ? PyFloat_AsDouble(args[3]) : 0;
    if (PyErr_Occurred()) return nullptr;
    head_ids ids;
    if (!table || modes() || table->dim() != 2 || dtype_of(*table) < 0 || !of_current_device(*table) ||
        !ids_of(args[1], args[2], *table, table->size(0), ids))
        return declined();
    const int64_t dim = table->size(1);
    const at::Tensor out = at::empty({ids.n_rows, dim}, table->options());
    const int32_t dtype = dtype_of(*table);
    const void *from = table->data_ptr();
    void *to = out.data_ptr(), *stream = stream_of(*table);
    const int rc = without_gil([&] { return entry.embed(&ids, dtype, dim, from, dim, static_cast<float>(scale), to, stream); });
    return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

// embed_grad(grad, ids, n_vectors, offsets, scale)
PyObject *embed_grad(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *grad = n == 5 ? tensor(args[0]) : nullptr;
    const int64_t n_vectors = n == 5 ? PyLong_AsLongLong(args[2]) : 0;
    const double scale = n == 5 && !PyErr_Occurred() ? PyFloat_AsDouble(args[4]) : 0;
    if (PyErr_Occurred()) return nullptr;
    head_ids ids;
    if (!grad || n_vectors < 0 || modes() || grad->dim() != 2 || dtype_of(*grad) < 0 || !of_current_device(*grad) ||
        !ids_of(args[1], args[3], *grad, n_vectors, ids) || ids.n_rows != grad->size(0))
        return declined();
    const int64_t dim = grad->size(1);
    const int32_t dtype = dtype_of(*grad);
    const int64_t bytes = entry.embed_grad_bytes(&ids, dtype, dim);
    if (bytes < 0) return PyLong_FromLongLong(bytes);
    const at::Tensor out = at::empty({n_vectors, dim}, grad->options()), work = workspace(bytes, *grad);
    const void *from = grad->data_ptr();
    void *to = out.data_ptr(), *space = work.data_ptr(), *stream = stream_of(*grad);
    const int rc = without_gil([&] { return entry.embed_grad(&ids, dtype, dim, from, dim, static_cast<float>(scale), to, space, stream); });
    return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

// layer_norm(x, weight, bias, eps)
PyObject *layer_norm(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *x = n == 4 ? tensor(args[0]) : nullptr;
    const double eps = n == 4 ? PyFloat_AsDouble(args[3]) : 0;
    if (PyErr_Occurred()) return nullptr;
    if (!x || modes() || x->dim() != 2 || dtype_of(*x) < 0 || !of_current_device(*x)) return declined();
    const int64_t rows = x->size(0), dim = x->size(1);
    const at::Tensor *weight = tensor(args[1]), *bias = args[2] == Py_None ? nullptr : tensor(args[2]);
    if (!fits(weight, *x, at::kFloat, {dim}) || (args[2] != Py_None && !fits(bias, *x, at::kFloat, {dim}))) return declined();
    const at::TensorOptions floats = x->options().dtype(at::kFloat);
    const at::Tensor y = at::empty({rows, dim}, x->options()), mean = at::empty({rows}, floats), rstd = at::empty({rows}, floats);
    const int32_t dtype = dtype_of(*x);
    const float *w = static_cast<const float *>(weight->data_ptr()), *b = bias ? static_cast<const float *>(bias->data_ptr()) : nullptr;
    float *m = static_cast<float *>(mean.data_ptr()), *r = static_cast<float *>(rstd.data_ptr());
    const void *from = x->data_ptr();
    void *to = y.data_ptr(), *stream = stream_of(*x);
    const int rc =
        without_gil([&] { return entry.layer_norm(dtype, rows, dim, from, dim, w, b, static_cast<float>(eps), to, m, r, stream); });
    return rc ? PyLong_FromLong(rc) : tuple_of(y, mean, rstd);
    END_HANDLE_TH_ERRORS
}

// layer_norm_grad(grad, x, weight, mean, rstd)
PyObject *layer_norm_grad(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *x = n == 5 ? tensor(args[1]) : nullptr;
    if (!x || modes() || x->dim() != 2 || dtype_of(*x) < 0 || !of_current_device(*x)) return declined();
    const int64_t rows = x->size(0), dim = x->size(1);
    const at::Tensor *grad = tensor(args[0]), *weight = tensor(args[2]), *mean = tensor(args[3]), *rstd = tensor(args[4]);
    if (!fits(grad, *x, x->scalar_type(), {rows, dim}) || !fits(weight, *x, at::kFloat, {dim}) || !fits(mean, *x, at::kFloat, {rows}) ||
        !fits(rstd, *x, at::kFloat, {rows}))
        return declined();
    const int32_t dtype = dtype_of(*x);
    const int64_t bytes = entry.layer_norm_grad_bytes(dtype, rows, dim);
    if (bytes < 0) return PyLong_FromLongLong(bytes);
    const at::TensorOptions floats = x->options().dtype(at::kFloat);
    const at::Tensor gx = at::empty({rows, dim}, x->options()), gw = at::empty({dim}, floats), gb = at::empty({dim}, floats),
                     work = workspace(bytes, *x);
    const float *w = static_cast<const float *>(weight->data_ptr()), *m = static_cast<const float *>(mean->data_ptr()),
                *r = static_cast<const float *>(rstd->data_ptr());
    float *to_w = static_cast<float *>(gw.data_ptr()), *to_b = static_cast<float *>(gb.data_ptr());
    const void *g = grad->data_ptr(), *from = x->data_ptr();
    void *to = gx.data_ptr(), *space = work.data_ptr(), *stream = stream_of(*x);
    const int rc = without_gil(
        [&] { return entry.layer_norm_grad(dtype, rows, dim, g, dim, from, dim, w, m, r, to, to_w, to_b, space, stream); });
    return rc ? PyLong_FromLong(rc) : tuple_of(gx, gw, gb);
    END_HANDLE_TH_ERRORS
}

bool classes_of(PyObject *hidden_object, PyObject *weight_object, PyObject *targets_object, PyObject *bias_object, const at::Tensor *&hidden,
                const at::Tensor *&weight, head_classes &c)
{
    hidden = tensor(hidden_object);
    weight = tensor(weight_object);
    const at::Tensor *targets = tensor(targets_object), *bias = bias_object == Py_None ? nullptr : tensor(bias_object);
    if (!hidden || !weight || modes() || hidden->dim() != 2 || weight->dim() != 2 || dtype_of(*hidden) < 0 || !of_current_device(*hidden))
        return false;
    const int64_t rows = hidden->size(0), dim = hidden->size(1), classes = weight->size(0);
    if (!fits(weight, *hidden, hidden->scalar_type(), {classes, dim}) || !fits(targets, *hidden, at::kInt, {rows}) ||
        (bias_object != Py_None && !fits(bias, *hidden, at::kFloat, {classes})))
        return false;
    c = head_classes{dtype_of(*hidden), rows, dim, classes, hidden->data_ptr(), dim, weight->data_ptr(), dim,
                     bias ? static_cast<const float *>(bias->data_ptr()) : nullptr, static_cast<const int32_t *>(targets->data_ptr())};
    return true;
}

// cross_entropy(hidden, weight, targets, bias)
PyObject *cross_entropy(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *hidden, *weight;
    head_classes c;
    if (n != 4 || !classes_of(args[0], args[1], args[2], args[3], hidden, weight, c)) return declined();
    const int64_t bytes = entry.cross_entropy_bytes(&c);
    if (bytes < 0) return PyLong_FromLongLong(bytes);
    const at::TensorOptions floats = hidden->options().dtype(at::kFloat);
    const at::Tensor loss = at::empty({c.n_rows}, floats), lse = at::empty({c.n_rows}, floats), work = workspace(bytes, *hidden);
    float *to_loss = static_cast<float *>(loss.data_ptr()), *to_lse = static_cast<float *>(lse.data_ptr());
    void *space = work.data_ptr(), *stream = stream_of(*hidden);
    const int rc = without_gil([&] { return entry.cross_entropy(&c, to_loss, to_lse, space, stream); });
    return rc ? PyLong_FromLong(rc) : tuple_of(loss, lse);
    END_HANDLE_TH_ERRORS
}

// cross_entropy_grad(grad_loss, hidden, weight, targets, lse, bias)
PyObject *cross_entropy_grad(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *hidden, *weight;
    head_classes c;
    if (n != 6 || !classes_of(args[1], args[2], args[3], args[5], hidden, weight, c)) return declined();
    const at::Tensor *grad_loss = tensor(args[0]), *lse = tensor(args[4]);
    if (!fits(grad_loss, *hidden, at::kFloat, {c.n_rows}) || !fits(lse, *hidden, at::kFloat, {c.n_rows})) return declined();
    const int64_t bytes = entry.cross_entropy_grad_bytes(&c);
    if (bytes < 0) return PyLong_FromLongLong(bytes);
    const at::Tensor gh = at::empty({c.n_rows, c.dim}, hidden->options()), gw = at::empty({c.n_classes, c.dim}, hidden->options());
    const at::Tensor gb = c.bias ? at::empty({c.n_classes}, hidden->options().dtype(at::kFloat)) : at::Tensor(), work = workspace(bytes, *hidden);
    const float *from_lse = static_cast<const float *>(lse->data_ptr()), *g = static_cast<const float *>(grad_loss->data_ptr());
    float *to_bias = c.bias ? static_cast<float *>(gb.data_ptr()) : nullptr;
    void *to_hidden = gh.data_ptr(), *to_weight = gw.data_ptr(), *space = work.data_ptr(), *stream = stream_of(*hidden);
    const int rc =
        without_gil([&] { return entry.cross_entropy_grad(&c, from_lse, g, to_hidden, to_weight, to_bias, space, stream); });
    return rc ? PyLong_FromLong(rc) : tuple_of(gh, gw, gb);
    END_HANDLE_TH_ERRORS
}

// A layer's x, weight and bias (or None), and the layer they make; `halves`: of z's columns.
bool layer_of(PyObject *x_object, PyObject *weight_object, PyObject *bias_object, PyObject *activation, int halves, const at::Tensor *&x,
              const at::Tensor *&weight, head_layer &l)
{
    x = tensor(x_object);
    weight = tensor(weight_object);
    const at::Tensor *bias = bias_object == Py_None ? nullptr : tensor(bias_object);
    if (!x || !weight || modes() || x->dim() != 2 || weight->dim() != 2 || dtype_of(*x) < 0 || !of_current_device(*x)) return false;
    const int64_t rows = x->size(0), dim = x->size(1), columns = weight->size(0);
    const long act = PyLong_AsLong(activation);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    if (!fits(weight, *x, x->scalar_type(), {columns, dim}) || columns % halves || act < HEAD_IDENTITY || act > HEAD_SILU ||
        (bias_object != Py_None && !fits(bias, *x, at::kFloat, {columns})))
        return false;
    l = head_layer{dtype_of(*x), static_cast<int32_t>(act), rows, dim, columns / halves, x->data_ptr(), dim, weight->data_ptr(), dim,
                   bias ? static_cast<const float *>(bias->data_ptr()) : nullptr};
    return true;
}

void *data_of(const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }

// y, or y and z.
PyObject *results(int rc, const at::Tensor &y, const at::Tensor &z)
{
    if (rc) return PyLong_FromLong(rc);
    return z.defined() ? tuple_of(y, z) : THPVariable_Wrap(y);
}

// linear(x, weight, bias, activation, residual, scale, keep)
PyObject *linear(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *x, *weight;
    head_layer l;
    if (n != 7 || !layer_of(args[0], args[1], args[2], args[3], 1, x, weight, l)) return declined();
    const at::Tensor *residual = args[4] == Py_None ? nullptr : tensor(args[4]);
    if (args[4] != Py_None && !fits(residual, *x, x->scalar_type(), {l.n_rows, l.n_outputs})) return declined();
    const double scale = PyFloat_AsDouble(args[5]);
    if (PyErr_Occurred()) return nullptr;
    const int keep = PyObject_IsTrue(args[6]);
    if (keep < 0) return nullptr;
    const int64_t bytes = entry.linear_bytes(&l);
    if (bytes < 0) return PyLong_FromLongLong(bytes);
    const at::Tensor y = fresh({l.n_rows, l.n_outputs}, x->scalar_type()), z = keep ? fresh({l.n_rows, l.n_outputs}, x->scalar_type()) : at::Tensor(),
                     work = bytes ? fresh({bytes}, at::kByte) : at::Tensor();
    const void *from = residual ? residual->data_ptr() : nullptr;
    void *to = y.data_ptr(), *to_z = data_of(z), *space = data_of(work), *stream = stream_of(*x);
    const int rc =
        without_gil([&] { return entry.linear(&l, from, l.n_outputs, static_cast<float>(scale), to, to_z, space, stream); });
    return results(rc, y, z);
    END_HANDLE_TH_ERRORS
}

// gated(x, weight, bias, activation, keep)
PyObject *gated(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *x, *weight;
    head_layer l;
    if (n != 5 || !layer_of(args[0], args[1], args[2], args[3], 2, x, weight, l)) return declined();
    const int keep = PyObject_IsTrue(args[4]);
    if (keep < 0) return nullptr;
    const int64_t bytes = entry.gated_bytes(&l);
    if (bytes < 0) return PyLong_FromLongLong(bytes);
    const at::Tensor y = fresh({l.n_rows, l.n_outputs}, x->scalar_type()),
                     z = keep ? fresh({l.n_rows, 2 * l.n_outputs}, x->scalar_type()) : at::Tensor(), work = bytes ? fresh({bytes}, at::kByte) : at::Tensor();
    void *to = y.data_ptr(), *to_z = data_of(z), *space = data_of(work), *stream = stream_of(*x);
    const int rc = without_gil([&] { return entry.gated(&l, to, to_z, space, stream); });
    return results(rc, y, z);
    END_HANDLE_TH_ERRORS
}

// grad, z or None, and the results of a layer's gradient; launch(z, grad, to x, to weight, to bias or null, workspace, stream).
template <class Launch>
PyObject *layer_grad(PyObject *grad_object, PyObject *z_object, PyObject *bias_object, const at::Tensor &x, const at::Tensor &weight, const head_layer &l,
                     bool reads_z, int64_t bytes, Launch launch)
{
    const at::Tensor *grad = tensor(grad_object), *z = z_object == Py_None ? nullptr : tensor(z_object);
    const int bias = PyObject_IsTrue(bias_object);
    if (bias < 0) return nullptr;
    if (!fits(grad, x, x.scalar_type(), {l.n_rows, l.n_outputs})) return declined();
    if (z_object != Py_None ? !fits(z, x, x.scalar_type(), {l.n_rows, weight.size(0)}) : reads_z) return declined();
    if (bytes < 0) return PyLong_FromLongLong(bytes);
    const at::Tensor gx = fresh({l.n_rows, l.dim}, x.scalar_type()), gw = fresh({weight.size(0), l.dim}, x.scalar_type()),
                     gb = bias ? fresh({weight.size(0)}, at::kFloat) : at::Tensor(),
                     work = bytes ? fresh({bytes}, at::kByte) : at::Tensor();
    const void *from_z = z ? z->data_ptr() : nullptr, *from = grad->data_ptr();
    void *to_x = gx.data_ptr(), *to_weight = gw.data_ptr(), *space = data_of(work), *stream = stream_of(x);
    float *to_bias = static_cast<float *>(data_of(gb));
    const int rc = without_gil([&] { return launch(from_z, from, to_x, to_weight, to_bias, space, stream); });
    return rc ? PyLong_FromLong(rc) : tuple_of(gx, gw, gb);
}

// linear_grad(grad, x, weight, z, activation, scale, bias)
PyObject *linear_grad(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *x, *weight;
    head_layer l;
    if (n != 7 || !layer_of(args[1], args[2], Py_None, args[4], 1, x, weight, l)) return declined();
    const double scale = PyFloat_AsDouble(args[5]);
    if (PyErr_Occurred()) return nullptr;
    return layer_grad(args[0], args[3], args[6], *x, *weight, l, l.activation != HEAD_IDENTITY, entry.linear_grad_bytes(&l),
                      [&](const void *z, const void *grad, void *to_x, void *to_weight, float *to_bias, void *space, void *stream) {
                          return entry.linear_grad(&l, z, l.n_outputs, grad, l.n_outputs, static_cast<float>(scale), to_x, to_weight, to_bias, space, stream);
                      });
    END_HANDLE_TH_ERRORS
}

// gated_grad(grad, x, weight, z, activation, bias)
PyObject *gated_grad(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *x, *weight;
    head_layer l;
    if (n != 6 || !layer_of(args[1], args[2], Py_None, args[4], 2, x, weight, l)) return declined();
    return layer_grad(args[0], args[3], args[5], *x, *weight, l, true, entry.gated_grad_bytes(&l),
                      [&](const void *z, const void *grad, void *to_x, void *to_weight, float *to_bias, void *space, void *stream) {
                          return entry.gated_grad(&l, z, 2 * l.n_outputs, grad, l.n_outputs, to_x, to_weight, to_bias, space, stream);
                      });
    END_HANDLE_TH_ERRORS
}

// Address of n adjacent values; null: not those.
void *values_at(PyObject *o, const at::Tensor &like, at::ScalarType type, int64_t n)
{
    const at::Tensor *t = plain(o);
    return t && t->scalar_type() == type && t->device() == like.device() && t->numel() == n ? t->data_ptr() : nullptr;
}

// Before values are written: what autograd has kept of a tensor is out of date.
void written(PyObject *o)
{
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// The states of a parameter: (m, v) or (m, m_scale, v, v_scale).
bool state_of(PyObject *o, const at::Tensor &like, Py_ssize_t kind, head_adamw_tensor &t)
{
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != kind) return false;
    if (kind == 2) {
        t.m = values_at(PyTuple_GET_ITEM(o, 0), like, at::kFloat, t.n);
        t.v = values_at(PyTuple_GET_ITEM(o, 1), like, at::kFloat, t.n);
        return t.m && t.v;
    }
    const int64_t blocks = (t.n + HEAD_BLOCK - 1) / HEAD_BLOCK;
    t.m = values_at(PyTuple_GET_ITEM(o, 0), like, at::kByte, t.n);
    t.m_scale = static_cast<uint8_t *>(values_at(PyTuple_GET_ITEM(o, 1), like, at::kByte, blocks));
    t.v = values_at(PyTuple_GET_ITEM(o, 2), like, at::kByte, t.n);
    t.v_scale = static_cast<uint8_t *>(values_at(PyTuple_GET_ITEM(o, 3), like, at::kByte, blocks));
    return t.m && t.m_scale && t.v && t.v_scale;
}

bool is_list(PyObject *o, Py_ssize_t n) { return PyList_CheckExact(o) && PyList_GET_SIZE(o) == n; }

// adamw(params, grads, states, copies, step, rate, beta1, beta2, eps, decay, seed): lists.  Returns True.
PyObject *adamw(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    HANDLE_TH_ERRORS
    if (n_args != 11 || !PyList_CheckExact(args[0]) || modes()) return declined();
    const Py_ssize_t n = PyList_GET_SIZE(args[0]);
    if (n == 0 || n > HEAD_MAX_TENSORS || !is_list(args[1], n) || !is_list(args[2], n) || (args[3] != Py_None && !is_list(args[3], n)))
        return declined();
    head_adamw_rule rule{};
    rule.step = PyLong_AsLongLong(args[4]);
    double numbers[5];
    for (int i = 0; i < 5; ++i) {
        if (PyErr_Occurred()) return nullptr;
        numbers[i] = PyFloat_AsDouble(args[5 + i]);
    }
    if (PyErr_Occurred()) return nullptr;
    rule.rate = numbers[0], rule.beta1 = numbers[1], rule.beta2 = numbers[2], rule.eps = numbers[3], rule.decay = numbers[4];
    rule.seed = static_cast<uint32_t>(PyLong_AsUnsignedLongLongMask(args[10]));
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor *first = plain(PyList_GET_ITEM(args[0], 0)), *grad = plain(PyList_GET_ITEM(args[1], 0));
    PyObject *state = PyList_GET_ITEM(args[2], 0);
    if (!first || !grad || !of_current_device(*first) || !PyTuple_Check(state)) return declined();
    const Py_ssize_t kind = PyTuple_GET_SIZE(state);
    rule.grad_dtype = dtype_of(*grad);
    if (rule.grad_dtype < 0 || (kind != 2 && kind != 4)) return declined();
    rule.bits = kind == 2 ? 32 : 8;
    const at::ScalarType grad_type = grad->scalar_type();
    std::vector<head_adamw_tensor> tensors(n);
    for (Py_ssize_t i = 0; i < n; ++i) {
        head_adamw_tensor &t = tensors[i];
        const at::Tensor *p = plain(PyList_GET_ITEM(args[0], i));
        if (!p || p->numel() == 0) return declined();
        t.n = p->numel();
        t.param = static_cast<float *>(values_at(PyList_GET_ITEM(args[0], i), *first, at::kFloat, t.n));
        t.grad = values_at(PyList_GET_ITEM(args[1], i), *first, grad_type, t.n);
        if (!t.param || !t.grad || !state_of(PyList_GET_ITEM(args[2], i), *first, kind, t)) return declined();
        PyObject *copy = args[3] == Py_None ? Py_None : PyList_GET_ITEM(args[3], i);
        if (copy != Py_None && !(t.copy = values_at(copy, *first, at::kBFloat16, t.n))) return declined();
    }
    for (Py_ssize_t i = 0; i < n; ++i) {
        written(PyList_GET_ITEM(args[0], i));
        PyObject *states = PyList_GET_ITEM(args[2], i);
        for (Py_ssize_t k = 0; k < kind; ++k) written(PyTuple_GET_ITEM(states, k));
        if (args[3] != Py_None && PyList_GET_ITEM(args[3], i) != Py_None) written(PyList_GET_ITEM(args[3], i));
    }
    void *stream = stream_of(*first);
    const int rc = without_gil([&] { return entry.adamw(&rule, tensors.data(), static_cast<int32_t>(n), stream); });
    if (rc) return PyLong_FromLong(rc);
    Py_RETURN_TRUE;
    END_HANDLE_TH_ERRORS
}

// adamw_values(states, params): lists.  Returns a list of (m, v).
PyObject *adamw_values(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    HANDLE_TH_ERRORS
    if (n_args != 2 || !PyList_CheckExact(args[0]) || modes()) return declined();
    const Py_ssize_t n = PyList_GET_SIZE(args[0]);
    if (n == 0 || n > HEAD_MAX_TENSORS || !is_list(args[1], n)) return declined();
    const at::Tensor *first = plain(PyList_GET_ITEM(args[1], 0));
    if (!first || !of_current_device(*first)) return declined();
    std::vector<head_adamw_tensor> tensors(n);
    std::vector<at::Tensor> m(n), v(n);
    std::vector<void *> to_m(n), to_v(n);
    for (Py_ssize_t i = 0; i < n; ++i) {
        const at::Tensor *p = plain(PyList_GET_ITEM(args[1], i));
        if (!p || p->numel() == 0 || p->device() != first->device()) return declined();
        tensors[i].n = p->numel();
        if (!state_of(PyList_GET_ITEM(args[0], i), *first, 4, tensors[i])) return declined();
        m[i] = at::empty(p->sizes(), p->options().dtype(at::kBFloat16));
        v[i] = at::empty(p->sizes(), p->options().dtype(at::kBFloat16));
        to_m[i] = m[i].data_ptr();
        to_v[i] = v[i].data_ptr();
    }
    void *stream = stream_of(*first);
    const int rc =
        without_gil([&] { return entry.adamw_values(tensors.data(), to_m.data(), to_v.data(), static_cast<int32_t>(n), stream); });
    if (rc) return PyLong_FromLong(rc);
    PyObject *list = PyList_New(n);
    for (Py_ssize_t i = 0; list && i < n; ++i) {
        PyObject *pair = tuple_of(m[i], v[i]);
        if (!pair) {
            Py_DECREF(list);
            return nullptr;
        }
        PyList_SET_ITEM(list, i, pair);
    }
    return list;
    END_HANDLE_TH_ERRORS
}

// clip(grads, max_norm, in_place): a list.  Returns (norm, a new list).
PyObject *clip(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    HANDLE_TH_ERRORS
    if (n_args != 3 || !PyList_CheckExact(args[0]) || modes()) return declined();
    const Py_ssize_t n = PyList_GET_SIZE(args[0]);
    if (n == 0 || n > HEAD_MAX_TENSORS) return declined();
    const double max_norm = PyFloat_AsDouble(args[1]);
    if (PyErr_Occurred()) return nullptr;
    const int in_place = PyObject_IsTrue(args[2]);
    if (in_place < 0) return nullptr;
    if (!(max_norm > 0)) return declined();
    const at::Tensor *first = tensor(PyList_GET_ITEM(args[0], 0));
    if (!first || !of_current_device(*first)) return declined();
    std::vector<head_clip_tensor> tensors(n);
    std::vector<at::Tensor> out(n);
    for (Py_ssize_t i = 0; i < n; ++i) {
        const at::Tensor *t = tensor(PyList_GET_ITEM(args[0], i));
        if (!t || dtype_of(*t) < 0 || t->device() != first->device() || t->numel() == 0) return declined();
        tensors[i] = head_clip_tensor{t->data_ptr(), nullptr, t->numel(), dtype_of(*t)};
    }
    if (in_place) {  // the same memory twice is the general way's error
        std::vector<std::pair<uintptr_t, uintptr_t>> ends(n);
        for (Py_ssize_t i = 0; i < n; ++i) {
            const at::Tensor &t = THPVariable_Unpack(PyList_GET_ITEM(args[0], i));
            const uintptr_t at = reinterpret_cast<uintptr_t>(tensors[i].grad);
            ends[i] = {at, at + t.nbytes()};
        }
        std::sort(ends.begin(), ends.end());
        for (Py_ssize_t i = 1; i < n; ++i)
            if (ends[i - 1].second > ends[i].first) return declined();
    }
    const int64_t bytes = entry.clip_bytes(tensors.data(), static_cast<int32_t>(n));
    if (bytes < 0) return PyLong_FromLongLong(bytes);
    const at::Tensor norm = fresh({}, at::kFloat), work = bytes ? fresh({bytes}, at::kByte) : at::Tensor();
    for (Py_ssize_t i = 0; i < n; ++i) {
        const at::Tensor &t = THPVariable_Unpack(PyList_GET_ITEM(args[0], i));
        if (in_place) written(PyList_GET_ITEM(args[0], i));
        out[i] = in_place ? t : fresh(t.sizes(), t.scalar_type());
        tensors[i].out = out[i].data_ptr();
    }
    float *to = static_cast<float *>(norm.data_ptr());
    void *space = data_of(work), *stream = stream_of(*first);
    const int rc = without_gil([&] { return entry.clip(tensors.data(), static_cast<int32_t>(n), max_norm, to, space, stream); });
    if (rc) return PyLong_FromLong(rc);
    PyObject *list = PyList_New(n);
    for (Py_ssize_t i = 0; list && i < n; ++i) {
        PyObject *one = THPVariable_Wrap(out[i]);  // in place: the list's own object, whatever has become of the list meanwhile
        if (!one) {
            Py_DECREF(list);
            return nullptr;
        }
        PyList_SET_ITEM(list, i, one);
    }
    PyObject *first_of_pair = list ? THPVariable_Wrap(norm) : nullptr;
    PyObject *pair = first_of_pair ? PyTuple_Pack(2, first_of_pair, list) : nullptr;
    Py_XDECREF(first_of_pair);
    Py_XDECREF(list);
    return pair;
    END_HANDLE_TH_ERRORS
}

// bind(addresses of the entry points, in Entries' order)
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != ENTRIES) {
        PyErr_Format(PyExc_TypeError, "bind takes %zd addresses", ENTRIES);
        return nullptr;
    }
    void *address[ENTRIES];
    for (Py_ssize_t i = 0; i < n; ++i) {
        address[i] = PyLong_AsVoidPtr(args[i]);
        if (!address[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an entry point has no address");
            return nullptr;
        }
    }
    static_assert(sizeof(address) == sizeof(entry), "pointers and nothing else");
    __builtin_memcpy(&entry, address, sizeof(entry));
    Py_RETURN_NONE;
}

#define HEAD_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef METHODS[] = {HEAD_METHOD(bind),          HEAD_METHOD(embed),         HEAD_METHOD(embed_grad),
                         HEAD_METHOD(layer_norm),    HEAD_METHOD(layer_norm_grad), HEAD_METHOD(cross_entropy),
                         HEAD_METHOD(cross_entropy_grad), HEAD_METHOD(adamw),    HEAD_METHOD(adamw_values),
                         HEAD_METHOD(linear),        HEAD_METHOD(linear_grad),   HEAD_METHOD(gated),
                         HEAD_METHOD(gated_grad),    HEAD_METHOD(clip),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef MODULE = {PyModuleDef_HEAD_INIT, "_head_call", nullptr, -1, METHODS, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__head_call() { return PyModule_Create(&MODULE); }
