/* The binding's ttc_execute as a CPython function: four integers unpacked, one call through a pointer, None returned.
   What bounds a small problem is the host: 70 x 33 x 45 fp32 (2,0,1) takes 2.45 us a launch from a C loop, 3.32 us from a Python
   loop through ctypes, whose argument conversions are most of the difference, and 2.99 us through this.  Anything but the plain case (three or four positional arguments that are
   ints, the library loaded) goes to the Python function `slow`, which does what it always did. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

typedef int (*execute_fn)(void*, const void*, void*, void*);
static execute_fn entry = NULL;          /* set once, by bind() */
static PyObject* slow = NULL;            /* (plan, A, B, stream=None), through ctypes */
static PyObject* fail = NULL;            /* (status): raises */

static PyObject* execute(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames)
{
    (void)self;
    int plain = entry != NULL && kwnames == NULL && (nargs == 3 || nargs == 4);
    for (Py_ssize_t i = 0; plain && i < nargs; ++i) plain = PyLong_CheckExact(args[i]) || (i == 3 && args[i] == Py_None);
    if (!plain) {
        if (slow == NULL) {
            PyErr_SetString(PyExc_RuntimeError, "ttc_execute is not bound");
            return NULL;
        }
        return PyObject_Vectorcall(slow, args, (size_t)nargs, kwnames);
    }
    void* p[4] = {NULL, NULL, NULL, NULL};
    for (Py_ssize_t i = 0; i < nargs; ++i)           /* as ctypes takes an int for a pointer: its low 64 bits */
        if (args[i] != Py_None) p[i] = (void*)(uintptr_t)PyLong_AsUnsignedLongLongMask(args[i]);
    if (PyErr_Occurred()) return NULL;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = entry(p[0], p[1], p[2], p[3]);
    Py_END_ALLOW_THREADS
    if (status == 0) Py_RETURN_NONE;
    return PyObject_CallFunction(fail, "i", status);
}

/* bind(slow, fail): the Python side; bind(address): the library's entry point. */
static PyObject* bind(PyObject* self, PyObject* const* args, Py_ssize_t nargs)
{
    (void)self;
    if (nargs == 2) {
        Py_INCREF(args[0]);
        Py_INCREF(args[1]);
        Py_XSETREF(slow, args[0]);
        Py_XSETREF(fail, args[1]);
    } else if (nargs == 1) {
        void* address = PyLong_AsVoidPtr(args[0]);
        if (address == NULL && PyErr_Occurred()) return NULL;
        entry = (execute_fn)address;
    } else {
        PyErr_SetString(PyExc_TypeError, "bind() takes one or two arguments");
        return NULL;
    }
    Py_RETURN_NONE;
}

/* The moves by data (ttc_moves.h): every argument a pointer or a 64-bit integer, the stream last and optional.  Ints are handed on as they
   are, anything else goes to the Python function `slow` of that move.  What ctypes takes for its conversions grows with the arguments: a call
   of eleven that has nothing to move takes 1.4 us through ctypes and 0.2 us here. */
#define MOVE_ARGS 16
typedef uint64_t U;
#define MOVES 7
static struct { void* entry; PyObject *slow, *fail; } moves[MOVES];

static PyObject* move(int which, int count, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames)
{
    int plain = moves[which].entry != NULL && kwnames == NULL && (nargs == count || nargs == count - 1);
    for (Py_ssize_t i = 0; plain && i < nargs; ++i) plain = PyLong_CheckExact(args[i]) || (i == count - 1 && args[i] == Py_None);
    if (!plain) {
        if (moves[which].slow == NULL) {
            PyErr_SetString(PyExc_RuntimeError, "the moves are not bound");
            return NULL;
        }
        return PyObject_Vectorcall(moves[which].slow, args, (size_t)nargs, kwnames);
    }
    U p[MOVE_ARGS] = {0};
    for (Py_ssize_t i = 0; i < nargs; ++i)
        if (args[i] != Py_None) p[i] = (U)PyLong_AsUnsignedLongLongMask(args[i]);
    if (PyErr_Occurred()) return NULL;
    int status = 0;
    void* f = moves[which].entry;
    Py_BEGIN_ALLOW_THREADS
    switch (count) {
    case 9:  status = ((int (*)(U, U, U, U, U, U, U, U, U))f)(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8]); break;
    case 10: status = ((int (*)(U, U, U, U, U, U, U, U, U, U))f)(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], p[9]); break;
    case 11: status = ((int (*)(U, U, U, U, U, U, U, U, U, U, U))f)(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], p[9], p[10]); break;
    case 12: status = ((int (*)(U, U, U, U, U, U, U, U, U, U, U, U))f)(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], p[9], p[10], p[11]); break;
    case 14: status = ((int (*)(U, U, U, U, U, U, U, U, U, U, U, U, U, U))f)(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], p[9], p[10], p[11], p[12], p[13]); break;
    case 16: status = ((int (*)(U, U, U, U, U, U, U, U, U, U, U, U, U, U, U, U))f)(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], p[9], p[10], p[11], p[12], p[13], p[14], p[15]); break;
    }
    Py_END_ALLOW_THREADS
    if (status == 0) Py_RETURN_NONE;
    return PyObject_CallFunction(moves[which].fail, "i", status);
}

#define MOVE(which, name, count)                                                                             \
    static PyObject* name(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames)         \
    {                                                                                                        \
        (void)self;                                                                                          \
        return move(which, count, args, nargs, kwnames);                                                     \
    }
MOVE(0, route_sort, 10)
MOVE(1, route_gather, 11)
MOVE(2, route_combine, 9)
MOVE(3, route_combine_grad, 14)
MOVE(4, pages_map, 16)
MOVE(5, pages_write, 12)
MOVE(6, pages_read, 12)

/* bind_move(which, slow, fail): the Python side of one move; bind_move(which, address): the library's entry point. */
static PyObject* bind_move(PyObject* self, PyObject* const* args, Py_ssize_t nargs)
{
    (void)self;
    const long which = nargs == 2 || nargs == 3 ? PyLong_AsLong(args[0]) : -1;
    if (which == -1 && PyErr_Occurred()) return NULL;
    if (which < 0 || which >= MOVES) {
        PyErr_SetString(PyExc_TypeError, "bind_move() takes the number of a move and its two Python functions or its address");
        return NULL;
    }
    if (nargs == 2) {
        void* address = PyLong_AsVoidPtr(args[1]);
        if (address == NULL && PyErr_Occurred()) return NULL;
        moves[which].entry = address;
    } else {
        Py_INCREF(args[1]);
        Py_INCREF(args[2]);
        Py_XSETREF(moves[which].slow, args[1]);
        Py_XSETREF(moves[which].fail, args[2]);
    }
    Py_RETURN_NONE;
}

#define METHOD(name) {"ttc_" #name, (PyCFunction)(void (*)(void))name, METH_FASTCALL | METH_KEYWORDS, NULL}

static PyMethodDef methods[] = {
    METHOD(route_sort), METHOD(route_gather), METHOD(route_combine), METHOD(route_combine_grad), METHOD(pages_map), METHOD(pages_write), METHOD(pages_read),
    {"bind_move", (PyCFunction)(void (*)(void))bind_move, METH_FASTCALL, NULL},
    {"ttc_execute", (PyCFunction)(void (*)(void))execute, METH_FASTCALL | METH_KEYWORDS,
     "ttc_execute(plan, A, B, stream=None)\n--\n\nA, B: device addresses (tensor.data_ptr()); stream: hipStream_t as an integer or None."},
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__call(void) { return PyModule_Create(&module); }
