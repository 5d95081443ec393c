// The Python binding's check of one tensor argument, natively: type, dtype,
// size, contiguity and device in one call (about 0.1 us; the same checks through
// torch's Python attributes take 0.75 us, and a delivery step makes fifteen of
// them, which kept the GPU waiting on small batches).  It only ever says yes:
// whatever it does not accept, the binding checks again in Python, which raises
// the error or knows better.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include "conduit.h"

namespace {

bool dtype_is(PyObject* want, at::ScalarType have) {
    return THPDtype_Check(want) && reinterpret_cast<THPDtype*>(want)->scalar_type == have;
}

bool dtype_among(PyObject* want, at::ScalarType have) {
    if (!PyTuple_CheckExact(want)) return dtype_is(want, have);
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(want); ++i)
        if (dtype_is(PyTuple_GET_ITEM(want, i), have)) return true;
    return false;
}

// A size in bytes or elements: None (no requirement, 0) or an int; false on anything else
bool read_size(PyObject* o, long long* n) {
    if (o == Py_None) {
        *n = 0;
        return true;
    }
    if (!PyLong_CheckExact(o)) return false;
    *n = PyLong_AsLongLong(o);
    if (*n == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}

// address(t, dtype, nbytes, numel): the device address of a plain contiguous
// tensor on a HIP device, of dtype `dtype` (a dtype, a tuple of them or None)
// and holding at least `nbytes` bytes and `numel` elements (None: any); None if
// it is anything else.
PyObject* address(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 4) {
        PyErr_SetString(PyExc_TypeError, "address takes (tensor, dtype, nbytes, numel)");
        return nullptr;
    }
    long long nbytes = 0, numel = 0;
    if (!THPVariable_CheckExact(args[0]) || !read_size(args[2], &nbytes) || !read_size(args[3], &numel)) Py_RETURN_NONE;
    uintptr_t p = 0;
    try {
        const at::Tensor& t = THPVariable_Unpack(args[0]);
        PyObject* want = args[1];
        if (want != Py_None) {
            if (!dtype_among(want, t.scalar_type())) Py_RETURN_NONE;
        }
        const long long n = t.numel();
        if (!t.is_cuda() || n * (long long)t.element_size() < nbytes || n < numel || !t.is_contiguous()) Py_RETURN_NONE;
        p = reinterpret_cast<uintptr_t>(t.data_ptr());
    } catch (...) {  // a wrapper without storage, a symbolic size: the Python path says so
        Py_RETURN_NONE;
    }
    return PyLong_FromUnsignedLongLong((unsigned long long)p);
}

struct Batch {
    int64_t dim, B, T, stride;
};

// the layout of a per-token tensor: [B, T] or [T] with elements next to each other along T
bool read_batch(const at::Tensor& t, Batch* b) {
    b->dim = t.dim();
    if (b->dim != 1 && b->dim != 2) return false;
    b->B = b->dim == 2 ? t.size(0) : 1;
    b->T = t.size(b->dim - 1);
    if (b->T > 1 && t.stride(b->dim - 1) != 1) return false;
    b->stride = b->dim == 2 && b->B > 1 && b->T > 0 ? t.stride(0) : b->T;
    return true;
}

// token_batch(t0, dtype0, t1, dtype1, ...): (B, T, step between rows, address of
// t0, address of t1, ...) of per-token tensors on a HIP device that all have t0's
// shape and step and their dtype (one or a tuple); a tensor after the first may
// be None (address None).  None if anything is otherwise.
PyObject* token_batch(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (nargs < 2 || nargs % 2 || nargs > 40) {
        PyErr_SetString(PyExc_TypeError, "token_batch takes (tensor, dtype) pairs");
        return nullptr;
    }
    Batch first{};
    uintptr_t at[20] = {0};
    try {
        for (Py_ssize_t i = 0; i < nargs; i += 2) {
            if (args[i] == Py_None && i > 0) continue;
            if (!THPVariable_CheckExact(args[i])) Py_RETURN_NONE;
            const at::Tensor& t = THPVariable_Unpack(args[i]);
            Batch b;
            if (!t.is_cuda() || !dtype_among(args[i + 1], t.scalar_type()) || !read_batch(t, &b)) Py_RETURN_NONE;
            if (i == 0) first = b;
            if (b.dim != first.dim || b.B != first.B || b.T != first.T || b.stride != first.stride) Py_RETURN_NONE;
            at[i / 2] = reinterpret_cast<uintptr_t>(t.data_ptr());
        }
    } catch (...) {
        Py_RETURN_NONE;
    }
    PyObject* out = PyTuple_New(3 + nargs / 2);
    if (!out) return nullptr;
    const int64_t head[3] = {first.B, first.T, first.stride};
    for (int i = 0; i < 3; ++i) PyTuple_SET_ITEM(out, i, PyLong_FromLongLong(head[i]));
    for (Py_ssize_t i = 0; i < nargs / 2; ++i) {
        PyObject* v = Py_None;
        if (args[2 * i] == Py_None) Py_INCREF(v);
        else v = PyLong_FromUnsignedLongLong((unsigned long long)at[i]);
        PyTuple_SET_ITEM(out, 3 + i, v);
    }
    if (PyErr_Occurred()) {
        Py_DECREF(out);
        return nullptr;
    }
    return out;
}

using Rows = conduit_rows;

// rows(address of a Rows, t, tokens, f32, bf16, i32 = -1): fills it in for a
// float32 or bfloat16 tensor on a HIP device of one row for each element of
// `tokens`, and says whether it did.  f32, bf16 and i32 are the library's numbers
// of the dtypes.  With i32 the tensor may be an int32 one too, and `tokens` is
// itself a tensor of rows, one for each of t's.
PyObject* rows(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 5 && nargs != 6) {
        PyErr_SetString(PyExc_TypeError, "rows takes (address, tensor, tokens, f32, bf16[, i32])");
        return nullptr;
    }
    if (!THPVariable_CheckExact(args[1]) || !THPVariable_CheckExact(args[2])) Py_RETURN_FALSE;
    Rows* r = static_cast<Rows*>(PyLong_AsVoidPtr(args[0]));
    const long f32 = PyLong_AsLong(args[3]), bf16 = PyLong_AsLong(args[4]), i32 = nargs == 6 ? PyLong_AsLong(args[5]) : -1;
    if (PyErr_Occurred()) return nullptr;
    try {
        const at::Tensor& t = THPVariable_Unpack(args[1]);
        const at::Tensor& n = THPVariable_Unpack(args[2]);
        const int64_t d = t.dim() - 1;
        if (!t.is_cuda() || (d != 1 && d != 2) || n.dim() != (nargs == 6 ? d + 1 : d)) Py_RETURN_FALSE;
        const bool whole = nargs == 6 && t.scalar_type() == at::kInt;
        if (!whole && t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16) Py_RETURN_FALSE;
        for (int64_t i = 0; i < d; ++i)
            if (t.size(i) != n.size(i)) Py_RETURN_FALSE;
        if (t.size(d) > 1 && t.stride(d) != 1) Py_RETURN_FALSE;
        *r = Rows{t.data_ptr(), (int32_t)(whole ? i32 : t.scalar_type() == at::kFloat ? f32 : bf16), 0, t.size(d),
                  d == 2 ? t.stride(0) : 0, t.stride(d - 1)};
    } catch (...) {
        Py_RETURN_FALSE;
    }
    Py_RETURN_TRUE;
}

// A tensor on a HIP device, exactly of class Tensor; null: not one
const at::Tensor* device_tensor(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.is_cuda() ? &t : nullptr;
}

// conduit_rows of a tensor of rows, one for each row of `ids`
bool rows_like(PyObject* o, const at::Tensor& ids, Rows* r) {
    const at::Tensor* t = device_tensor(o);
    const int64_t d = ids.dim() - 1;
    if (!t || t->dim() != d + 1) return false;
    for (int64_t i = 0; i < d; ++i)
        if (t->size(i) != ids.size(i)) return false;
    if (t->size(d) > 1 && t->stride(d) != 1) return false;
    const at::ScalarType type = t->scalar_type();
    const int32_t dtype = type == at::kFloat ? CONDUIT_F32 : type == at::kBFloat16 ? CONDUIT_BF16 : type == at::kInt ? CONDUIT_I32 : -1;
    if (dtype < 0) return false;
    *r = Rows{t->data_ptr(), dtype, 0, t->size(d), d == 2 ? t->stride(0) : 0, t->stride(d - 1)};
    return true;
}

// listed(which, entry point's address, options' address or None, temperature, stream,
// workspace, stats, logits, ids, values, dlogits, four per-token tensors, mask): a
// call on listed choices (0 alternatives: tokens, logp, lse, entropy; 1
// log-probabilities: rest, lse; 2 their gradient: lse, rest, drest; 3 distillation:
// loss, weight) whose arguments are all plain ones, and its status; None, and no
// call, if anything is otherwise.  (Argument by argument through ctypes a call takes
// 7.4 us on the host, this way 4.8 to 4.9, most of it the launch.)
PyObject* listed(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 16) {
        PyErr_SetString(PyExc_TypeError, "listed takes 16 arguments");
        return nullptr;
    }
    const long which = PyLong_AsLong(args[0]);
    void* const entry = PyLong_AsVoidPtr(args[1]);
    void* const opts = args[2] == Py_None ? nullptr : PyLong_AsVoidPtr(args[2]);
    const double temperature = PyFloat_AsDouble(args[3]);
    void* const stream = PyLong_AsVoidPtr(args[4]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (!entry || which < 0 || which > 3) Py_RETURN_NONE;
    Rows x, ids, values, dx;
    Batch batch{};
    void* at[5] = {nullptr, nullptr, nullptr, nullptr, nullptr};
    void* workspace = nullptr;
    float* stats = nullptr;
    uint64_t bytes = 0;
    try {
        const at::Tensor* i = device_tensor(args[8]);
        if (!i || (i->dim() != 2 && i->dim() != 3) || !rows_like(args[8], *i, &ids) || ids.dtype != CONDUIT_I32) Py_RETURN_NONE;
        if (!rows_like(args[7], *i, &x) || x.dtype == CONDUIT_I32) Py_RETURN_NONE;
        if (!rows_like(args[9], *i, &values) || values.dtype != CONDUIT_F32 || values.width != ids.width) Py_RETURN_NONE;
        if (args[10] != Py_None && (!rows_like(args[10], *i, &dx) || dx.dtype == CONDUIT_I32)) Py_RETURN_NONE;
        batch.dim = i->dim() - 1;
        batch.B = batch.dim == 2 ? i->size(0) : 1;
        batch.T = i->size(batch.dim - 1);
        batch.stride = batch.T;
        bool first = true;
        for (int k = 0; k < 5; ++k) {
            if (args[11 + k] == Py_None) continue;
            const at::Tensor* t = device_tensor(args[11 + k]);
            Batch b;
            if (!t || !read_batch(*t, &b) || b.dim != batch.dim || b.B != batch.B || b.T != batch.T) Py_RETURN_NONE;
            if (!first && b.stride != batch.stride) Py_RETURN_NONE;
            const at::ScalarType type = t->scalar_type();
            if (k == 4 ? type != at::kByte && type != at::kBool : type != (which == 0 && k == 0 ? at::kInt : at::kFloat)) Py_RETURN_NONE;
            batch.stride = b.stride;
            first = false;
            at[k] = t->data_ptr();
        }
        if (args[5] != Py_None) {
            const at::Tensor* t = device_tensor(args[5]);
            if (!t || t->scalar_type() != at::kByte || !t->is_contiguous()) Py_RETURN_NONE;
            workspace = t->data_ptr();
            bytes = (uint64_t)t->numel();
        }
        if (args[6] != Py_None) {
            const at::Tensor* t = device_tensor(args[6]);
            if (!t || t->scalar_type() != at::kFloat || !t->is_contiguous() || t->numel() < 3) Py_RETURN_NONE;
            stats = static_cast<float*>(t->data_ptr());
        }
    } catch (...) {
        Py_RETURN_NONE;
    }
    Rows* const gradient = args[10] == Py_None ? nullptr : &dx;
    float* const f[4] = {static_cast<float*>(at[0]), static_cast<float*>(at[1]), static_cast<float*>(at[2]), static_cast<float*>(at[3])};
    const uint8_t* const mask = static_cast<const uint8_t*>(at[4]);
    const int64_t B = batch.B, T = batch.T, step = batch.stride;
    conduit_status status;
    Py_BEGIN_ALLOW_THREADS;
    switch (which) {
    case 0:
        status = reinterpret_cast<decltype(&conduit_token_alternatives)>(entry)(
            &x, B, T, step, static_cast<const int32_t*>(at[0]), mask, temperature, &ids, &values, f[1], f[2], f[3], workspace, bytes, stream);
        break;
    case 1:
        status = reinterpret_cast<decltype(&conduit_listed_logprobs)>(entry)(&x, B, T, step, &ids, mask, temperature, &values, f[0], f[1],
                                                                             workspace, bytes, stream);
        break;
    case 2:
        status = reinterpret_cast<decltype(&conduit_listed_logprobs_backward)>(entry)(&x, B, T, step, &ids, mask, temperature, f[0], f[1],
                                                                                      &values, f[2], gradient, stream);
        break;
    default:
        status = reinterpret_cast<decltype(&conduit_distill_loss)>(entry)(static_cast<const conduit_distill_opts*>(opts), &x, B, T, step, &ids,
                                                                          &values, f[1], mask, temperature, f[0], stats, gradient, workspace,
                                                                          bytes, stream);
    }
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong((long)status);
}

PyMethodDef methods[] = {
    {"listed", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(listed)), METH_FASTCALL,
     "a call on listed choices with checked tensors: its status, or None"},
    {"token_batch", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(token_batch)), METH_FASTCALL,
     "layout and device addresses of checked per-token tensors, or None"},
    {"rows", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rows)), METH_FASTCALL,
     "fills in a conduit_rows for a checked tensor"},
    {"address", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(address)), METH_FASTCALL,
     "device address of a checked tensor argument, or None"},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensor_check", "checks of the binding's tensor arguments", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensor_check(void) {
    PyObject* m = PyModule_Create(&module);
    // the layouts read above are this torch's: the binding uses no other's
    if (m && PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION_BUILT) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
