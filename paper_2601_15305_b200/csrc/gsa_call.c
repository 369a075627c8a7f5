/* Calls of the C-ABI library from Python without ctypes' conversions, which cost more than a kernel launch does (2 us for twelve arguments
 * against 0.3 here).  call(address, a, b, ...) calls the function at `address`, which returns an int and takes up to sixteen
 * integers or pointers, with the given ints (None: NULL).  In the x86-64 and AArch64 calling conventions a narrower integer argument
 * occupies a whole register or stack slot, so that all of them can be passed as 64 bits. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#define MOST 16
typedef int (*fn_t)(int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t,
                    int64_t, int64_t, int64_t);

static PyObject* call(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    int64_t v[MOST + 1] = {0};
    int rc;
    (void)self;
    if (n < 1 || n > MOST + 1) {
        PyErr_SetString(PyExc_TypeError, "call(address, up to 16 integers)");
        return NULL;
    }
    for (Py_ssize_t i = 0; i < n; ++i) {
        if (args[i] == Py_None) continue;
        if (!PyLong_Check(args[i])) {
            PyErr_SetString(PyExc_TypeError, "arguments are ints or None");
            return NULL;
        }
        /* (addresses and sizes are unsigned, lengths signed: the low 64 bits are right for either) */
        v[i] = (int64_t)PyLong_AsUnsignedLongLongMask(args[i]);
        if (v[i] == -1 && PyErr_Occurred()) return NULL;
    }
    if (!v[0]) {
        PyErr_SetString(PyExc_ValueError, "no function");
        return NULL;
    }
    Py_BEGIN_ALLOW_THREADS
    rc = ((fn_t)(intptr_t)v[0])(v[1], v[2], v[3], v[4], v[5], v[6], v[7], v[8], v[9], v[10], v[11], v[12], v[13], v[14], v[15], v[16]);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyMethodDef methods[] = {{"call", (PyCFunction)(void (*)(void))call, METH_FASTCALL, "call(address, ...): the int it returns"}, {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_gsa_call", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__gsa_call(void) { return PyModule_Create(&module); }
