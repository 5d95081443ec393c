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

// the members of conduit_rows
struct Rows {
    void* data;
    int32_t dtype, reserved;
    int64_t width, stride_b, stride_t;
};

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

PyMethodDef methods[] = {
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
