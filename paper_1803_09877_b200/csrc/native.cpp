// The calls of a training loop, marshalled natively for CPython: arguments are torch tensors (or anything with data_ptr()), addresses
// or None, as in binding.py, which uses ctypes for everything else.  A call of a library that only launches a kernel is the caller's
// time.  By ctypes / so, us a call: cyclic encode n = 15, s = 2, d = 12,000 3.84 / 3.12, n = 45, s = 5, d = 4096 5.28 / 4.42, repetition encode
// n = 15, d = 100,000 5.65 / 4.71, all on one host (others are faster throughout).
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "dlpack_tensor.h"
#include "draco.h"

namespace {

PyObject* g_check = nullptr;          // binding._check: raises for a negative status
PyObject* g_stream = nullptr;         // binding._stream: any stream argument to a handle
PyObject* g_raw = nullptr;            // handle of a device's current stream, and the current device, once torch's are known
PyObject* g_device = nullptr;
PyObject* g_data_ptr = nullptr;       // "data_ptr"

bool address(PyObject* x, void** out) {
    if (x == Py_None) {
        *out = nullptr;
        return true;
    }
    PyObject* owned = nullptr;
    if (!PyLong_Check(x)) {
        x = owned = PyObject_CallMethodNoArgs(x, g_data_ptr);
        if (!x) return false;
    }
    *out = reinterpret_cast<void*>(static_cast<uintptr_t>(PyLong_AsUnsignedLongLongMask(x)));
    Py_XDECREF(owned);
    return !PyErr_Occurred();
}

bool stream_of(PyObject* x, void** out) {
    PyObject* handle;
    if (x == Py_None && g_raw) {
        PyObject* device = PyObject_CallNoArgs(g_device);
        if (!device) return false;
        handle = PyObject_CallOneArg(g_raw, device);
        Py_DECREF(device);
    } else {
        handle = PyObject_CallOneArg(g_stream, x);
    }
    if (!handle) return false;
    const bool ok = address(handle, out);
    Py_DECREF(handle);
    return ok;
}

// The plan, `count` addresses and, last, the stream.
bool arguments(PyObject* const* args, Py_ssize_t nargs, Py_ssize_t want, int count, void** p, void** stream) {
    if (nargs != want) {
        PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", want, nargs);
        return false;
    }
    for (int k = 0; k < count; ++k)
        if (!address(args[k], &p[k])) return false;
    return stream_of(args[nargs - 1], stream);
}

PyObject* status(int rc) {
    PyObject* value = PyLong_FromLong(rc);
    if (rc >= 0 || !value) return value;
    PyObject* result = PyObject_CallOneArg(g_check, value);
    Py_DECREF(value);
    return result;
}

#define PLAN reinterpret_cast<draco_plan*>(p[0])

PyObject* encode(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    void *p[3], *st;
    if (!arguments(args, nargs, 4, 3, p, &st)) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS rc = draco_encode(PLAN, (const float*)p[1], p[2], st);
    Py_END_ALLOW_THREADS return status(rc);
}

PyObject* locate(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    void *p[4], *st;
    if (!arguments(args, nargs, 5, 4, p, &st)) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS rc = draco_locate(PLAN, p[1], (const float*)p[2], (uint8_t*)p[3], st);
    Py_END_ALLOW_THREADS return status(rc);
}

PyObject* decode(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    void *p[4], *st;
    if (!arguments(args, nargs, 5, 4, p, &st)) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS rc = draco_decode(PLAN, p[1], (const uint8_t*)p[2], (float*)p[3], st);
    Py_END_ALLOW_THREADS return status(rc);
}

PyObject* decode_update(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    void *p[4], *st;
    if (!arguments(args, nargs, 6, 4, p, &st)) return nullptr;
    const float scale = (float)PyFloat_AsDouble(args[4]);
    if (PyErr_Occurred()) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS rc = draco_decode_update(PLAN, p[1], (const uint8_t*)p[2], (float*)p[3], scale, st);
    Py_END_ALLOW_THREADS return status(rc);
}

PyObject* locate_decode(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    void *p[5], *st;
    if (!arguments(args, nargs, 6, 5, p, &st)) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS rc = draco_locate_decode(PLAN, p[1], (const float*)p[2], (uint8_t*)p[3], (float*)p[4], st);
    Py_END_ALLOW_THREADS return status(rc);
}

// ---- lists of tensors ----

// DLPack's C interface, by which a tensor's address, type, sizes and device come in one call: by torch_tensors.cpp where it was built, 11 ns
// a tensor, or else by torch, 120 ns with the question for the negative bit; binding.py itself takes 760.  A list that is not plain tensors of
// the layout's sizes and types on its device is left to binding.py (NotImplemented), which takes what is unusual and names what is wrong.
const DLPackExchangeAPI* g_exchange = nullptr;
const BuiltExchange* g_built = nullptr;                     // the same, if torch_tensors.cpp made it
PyObject* g_is_neg = nullptr;         // "is_neg"
PyObject* g_wrote = nullptr;          // binding._wrote
PyObject *g_tensor = nullptr, *g_parameter = nullptr;       // torch.Tensor and torch.nn.Parameter; their subclasses are left to binding.py

struct Meta {                                               // binding.py's _Meta
    int64_t count, d;
    const int64_t* numels;
    const int32_t* types;
    int32_t device;
};

// Whether the elements fill one piece of memory: in the order of the dimensions, or (ordered false) in any.
bool dense(const DLTensor& t, bool ordered) {
    constexpr int kMost = 8;
    if (t.ndim > kMost) return false;
    int64_t run = 1;
    bool contiguous = true;
    for (int k = t.ndim - 1; k >= 0; --k) {
        if (t.shape[k] == 1) continue;
        if (t.strides && t.strides[k] != run) contiguous = false;
        run *= t.shape[k];
    }
    if (contiguous || run == 0) return true;
    if (ordered) return false;
    bool done[kMost] = {};
    run = 1;
    for (int n = 0; n < t.ndim; ++n) {
        int next = -1;
        for (int k = 0; k < t.ndim; ++k)
            if (!done[k] && t.shape[k] != 1 && t.strides[k] == run) next = k;
        if (next < 0) break;
        done[next] = true;
        run *= t.shape[next];
    }
    for (int k = 0; k < t.ndim; ++k)
        if (!done[k] && t.shape[k] != 1) return false;
    return true;
}

// What the exchange says of a tensor, or false, without an error, where it says nothing or the tensor's memory holds other values than the
// tensor (a negated view; torch's own function does not look at that: the tensor itself is asked).  written: the memory is the tensor's alone;
// one that shares it until either is written (a lazy clone) gets its own here, from torch's own function in any case.
bool tensor_of(PyObject* x, bool written, DLTensor* t) {
    bool plain = (g_built && written ? g_built->written_from_object : g_exchange->tensor_from_object)(x, t) == 0;
    if (plain && !g_built) {
        PyObject* negated = PyObject_CallMethodNoArgs(x, g_is_neg);
        plain = negated == Py_False;
        Py_XDECREF(negated);
    }
    if (!plain) PyErr_Clear();
    return plain;
}

bool is_plain(PyObject* x) { return (PyObject*)Py_TYPE(x) == g_tensor || (PyObject*)Py_TYPE(x) == g_parameter; }

// The tensor as the layout has it, or false, without an error.
bool as_told(PyObject* x, int64_t numel, int type, int device, bool ordered, bool written, DLTensor* t) {
    if (!g_exchange || !is_plain(x)) return false;
    if (!tensor_of(x, written, t)) return false;
    static const DLDataType types[] = {{2, 32, 1}, {4, 16, 1}, {2, 16, 1}};       // DRACO_F32, DRACO_BF16, DRACO_F16
    constexpr int kCuda = 2;
    if (type < 0 || type > 2 || t->device.type != kCuda || t->device.id != device || t->dtype.code != types[type].code ||
        t->dtype.bits != types[type].bits || t->dtype.lanes != 1)
        return false;
    int64_t n = 1;
    for (int k = 0; k < t->ndim; ++k) n *= t->shape[k];
    return n == numel && (t->data || !n) && dense(*t, ordered);
}

// Address of an fp32 vector of n elements, an int or None.
bool vector_address(PyObject* x, const Meta* m, int64_t n, bool written, void** out) {
    if (x == Py_None || PyLong_Check(x)) return address(x, out);
    DLTensor t;
    if (!as_told(x, n, DRACO_F32, m->device, true, written, &t)) return false;
    *out = static_cast<char*>(t.data) + t.byte_offset;
    return true;
}

struct Addresses {
    void* few[512];
    void** p = few;
    ~Addresses() {
        if (p != few) PyMem_Free(p);
    }
    // beside: a list whose tensors have the same sizes and strides
    bool take(PyObject* list, const Meta* m, bool ordered, bool written, PyObject* beside = nullptr) {
        if (!PyList_Check(list) && !PyTuple_Check(list)) return false;
        if (PySequence_Fast_GET_SIZE(list) != m->count) return false;
        if (m->count > (int64_t)(sizeof(few) / sizeof(few[0]))) {
            p = static_cast<void**>(PyMem_Malloc(sizeof(void*) * m->count));
            if (!p) {
                p = few;
                return false;
            }
        }
        PyObject** items = PySequence_Fast_ITEMS(list);
        for (int64_t i = 0; i < m->count; ++i) {
            PyObject* x = items[i];
            p[i] = nullptr;
            if (x == Py_None) continue;
            DLTensor t, b;
            if (!as_told(x, m->numels[i], m->types[i], m->device, ordered, written, &t)) return false;
            if (beside) {
                PyObject* y = PySequence_Fast_ITEMS(beside)[i];
                if (y == Py_None || g_exchange->tensor_from_object(y, &b) != 0) {
                    PyErr_Clear();
                    return false;
                }
                if (t.ndim != b.ndim) return false;
                for (int k = 0; k < t.ndim; ++k)
                    if (t.shape[k] != b.shape[k] || (t.shape[k] != 1 && t.strides[k] != b.strides[k])) return false;
            }
            p[i] = static_cast<char*>(t.data) + t.byte_offset;
        }
        return true;
    }
};

#define LAYOUT reinterpret_cast<draco_layout*>(layout)
#define META const Meta* m = static_cast<const Meta*>(meta)

bool layout_of(PyObject* const* args, Py_ssize_t nargs, Py_ssize_t want, void** layout, void** meta) {
    if (nargs != want) {
        PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", want, nargs);
        return false;
    }
    return address(args[0], layout) && address(args[1], meta);
}

bool number(PyObject* x, float* out) {
    *out = (float)PyFloat_AsDouble(x);
    return !PyErr_Occurred();
}

bool whole(PyObject* x, int* out) {
    const long v = PyLong_AsLong(x);
    *out = v < INT32_MIN || v > INT32_MAX ? -1 : (int)v;
    return !PyErr_Occurred();
}

// The status of a call that has written these tensors and lists of tensors, of which autograd is told.
PyObject* written(int rc, PyObject* list, PyObject* a, PyObject* b) {
    if (rc < 0) return status(rc);
    if (!g_built) {
        PyObject* done = PyObject_CallFunctionObjArgs(g_wrote, list, a, b, nullptr);
        if (!done) return nullptr;
        Py_DECREF(done);
        return status(rc);
    }
    if (list != Py_None)
        for (Py_ssize_t i = 0; i < PySequence_Fast_GET_SIZE(list); ++i) {
            PyObject* x = PySequence_Fast_GET_ITEM(list, i);
            if (is_plain(x)) g_built->increment_version(x);
        }
    if (is_plain(a)) g_built->increment_version(a);
    if (is_plain(b)) g_built->increment_version(b);
    return status(rc);
}

PyObject* left_to_python() {
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NOTIMPLEMENTED;
}

// (layout, meta, tensors, norm, each, kind, stream)
PyObject* norm(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    void *layout, *meta, *norm, *each, *st;
    int kind;
    if (!layout_of(args, nargs, 7, &layout, &meta)) return nullptr;
    META;
    Addresses a;
    if (!a.take(args[2], m, false, false) || !vector_address(args[3], m, 1, true, &norm) || !vector_address(args[4], m, m->count, true, &each))
        return left_to_python();
    if (!whole(args[5], &kind) || !stream_of(args[6], &st)) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS rc = draco_norm(LAYOUT, a.p, kind, (float*)norm, (float*)each, st);
    Py_END_ALLOW_THREADS return written(rc, Py_None, args[3], args[4]);
}

// (layout, meta, tensors, max_norm, out, norm, each, separately, kind, stream)
PyObject* clip(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    void *layout, *meta, *norm, *each, *st;
    int kind;
    float max_norm;
    if (!layout_of(args, nargs, 10, &layout, &meta)) return nullptr;
    META;
    Addresses a, b;
    const bool out = args[4] != Py_None;
    if (!a.take(args[2], m, false, !out) || (out && !b.take(args[4], m, false, true, args[2])) || !vector_address(args[5], m, 1, true, &norm) ||
        !vector_address(args[6], m, m->count, true, &each))
        return left_to_python();
    const int separately = PyObject_IsTrue(args[7]);
    if (separately < 0 || !number(args[3], &max_norm) || !whole(args[8], &kind) || !stream_of(args[9], &st)) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS rc = draco_clip(LAYOUT, a.p, out ? b.p : nullptr, kind, max_norm, separately, (float*)norm, (float*)each, st);
    Py_END_ALLOW_THREADS return written(rc, out ? args[4] : args[2], args[5], args[6]);
}

// (layout, meta, tensors, row, max_norm, norm, kind, stream)
PyObject* pack(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    void *layout, *meta, *row, *norm, *st;
    int kind;
    float max_norm;
    if (!layout_of(args, nargs, 8, &layout, &meta)) return nullptr;
    META;
    Addresses a;
    if (!a.take(args[2], m, true, false) || !vector_address(args[3], m, m->d, true, &row) || !vector_address(args[5], m, 1, true, &norm))
        return left_to_python();
    if (!number(args[4], &max_norm) || !whole(args[6], &kind) || !stream_of(args[7], &st)) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS rc = draco_pack(LAYOUT, a.p, kind, max_norm, (float*)row, (float*)norm, st);
    Py_END_ALLOW_THREADS return written(rc, Py_None, args[3], args[5]);
}

// (layout, meta, params, u, scale, max_norm, master, norm, kind, stream)
PyObject* update(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    void *layout, *meta, *u, *master, *norm, *st;
    int kind;
    float scale, max_norm;
    if (!layout_of(args, nargs, 10, &layout, &meta)) return nullptr;
    META;
    Addresses a;
    if (!a.take(args[2], m, true, true) || !vector_address(args[3], m, m->d, false, &u) || !vector_address(args[6], m, m->d, true, &master) ||
        !vector_address(args[7], m, 1, true, &norm))
        return left_to_python();
    if (!number(args[4], &scale) || !number(args[5], &max_norm) || !whole(args[8], &kind) || !stream_of(args[9], &st)) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS rc = draco_update(LAYOUT, a.p, (const float*)u, (float*)master, kind, max_norm, scale, (float*)norm, st);
    Py_END_ALLOW_THREADS return written(rc, args[2], args[6], args[7]);
}

void keep(PyObject*& slot, PyObject* value) {
    Py_INCREF(value);
    Py_XSETREF(slot, value);
}

PyObject* set_functions(PyObject*, PyObject* args) {          // (check, stream, wrote)
    PyObject *check, *stream, *wrote;
    if (!PyArg_ParseTuple(args, "OOO", &check, &stream, &wrote)) return nullptr;
    keep(g_check, check);
    keep(g_stream, stream);
    keep(g_wrote, wrote);
    Py_RETURN_NONE;
}

PyObject* set_current_stream(PyObject*, PyObject* args) {     // (raw, device)
    PyObject *raw, *device;
    if (!PyArg_ParseTuple(args, "OO", &raw, &device)) return nullptr;
    keep(g_device, device);
    keep(g_raw, raw);
    Py_RETURN_NONE;
}

PyObject* set_exchange(PyObject*, PyObject* args) {           // (torch.Tensor, torch.nn.Parameter, its DLPack exchange capsule)
    PyObject *tensor, *parameter, *capsule;
    if (!PyArg_ParseTuple(args, "OOO", &tensor, &parameter, &capsule)) return nullptr;
    const BuiltExchange* built = nullptr;
    if (PyCapsule_IsValid(capsule, kBuiltExchange)) built = static_cast<const BuiltExchange*>(PyCapsule_GetPointer(capsule, kBuiltExchange));
    const auto* api = built ? &built->read : static_cast<const DLPackExchangeAPI*>(PyCapsule_GetPointer(capsule, "dlpack_exchange_api"));
    if (!api) return nullptr;
    if (api->major == 1 && api->tensor_from_object) {
        g_built = built;
        keep(g_tensor, tensor);
        keep(g_parameter, parameter);
        g_exchange = api;
    }
    Py_RETURN_NONE;
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(encode), FAST(locate), FAST(decode), FAST(decode_update), FAST(locate_decode),
                         FAST(norm), FAST(clip), FAST(pack), FAST(update), {"set_exchange", set_exchange, METH_VARARGS, nullptr},
                         {"set_functions", set_functions, METH_VARARGS, nullptr},
                         {"set_current_stream", set_current_stream, METH_VARARGS, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) {
    g_data_ptr = PyUnicode_InternFromString("data_ptr");
    g_is_neg = PyUnicode_InternFromString("is_neg");
    return g_data_ptr && g_is_neg ? PyModule_Create(&module) : nullptr;
}
