// The binding's test of one tensor argument, for lynx.py: a call makes up to 21
// of them, and a short kernel waits for the host.  In Python a test is five
// attribute reads, 0.6 us; here it is one call, 0.1.
//
//   typed(fn, what, t, nbytes, dtype, device) -> the pointer of tensor t
//
// None and ints pass through.  Anything that is not a contiguous tensor of that
// dtype on that device with nbytes bytes at least goes to the Python form of the
// test (set by `otherwise`), which says what is wrong.
#include <Python.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

PyObject *g_otherwise = nullptr;

PyObject *typed(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "typed takes 6 arguments");
        return nullptr;
    }
    PyObject *t = args[2];
    if (t == Py_None || PyLong_CheckExact(t)) {
        Py_INCREF(t);
        return t;
    }
    if (THPVariable_Check(t) && THPDtype_Check(args[4]) && PyLong_Check(args[3]) && PyLong_Check(args[5])) {
        int over = 0, over_dev = 0;
        const long long nbytes = PyLong_AsLongLongAndOverflow(args[3], &over);
        const long dev = PyLong_AsLongAndOverflow(args[5], &over_dev);
        const at::Tensor &x = THPVariable_Unpack(t);
        try {
            if (!over && !over_dev && x.layout() == c10::kStrided && x.is_cuda() && x.get_device() == dev &&
                x.scalar_type() == reinterpret_cast<THPDtype *>(args[4])->scalar_type && x.is_contiguous() &&
                (long long)x.nbytes() >= nbytes)
                return PyLong_FromVoidPtr(x.data_ptr());
        } catch (const std::exception &) {  // (a tensor without storage: the Python form raises)
        }
    }
    if (!g_otherwise) {
        PyErr_SetString(PyExc_RuntimeError, "otherwise() has not been called");
        return nullptr;
    }
    return PyObject_Vectorcall(g_otherwise, args, n, nullptr);
}

PyObject *otherwise(PyObject *, PyObject *f) {
    Py_INCREF(f);
    Py_XSETREF(g_otherwise, f);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"typed", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(typed)), METH_FASTCALL, nullptr},
    {"otherwise", otherwise, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_args", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__args() { return PyModule_Create(&module); }
