// seqmix_py.cpp -- the checks and the call of the token-mixing helpers as one C++ step.
//
// A call on a few tokens takes 5 us on the GPU.  Checking its 6 to 10 tensors one attribute at a time and
// marshalling their addresses takes Python as long; here it takes a tenth of that.  Python builds a Call
// once per descriptor (the C function, the descriptor, what each tensor has to be) and runs it with the tensors.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <vector>

namespace {

constexpr int kMost = 10;  // tensors of a call

struct Want {
    int64_t element;  // bytes and kind: at::ScalarType
    bool out;         // is written
    std::vector<int64_t> sizes, strides;
};
struct Call {
    void* fn;
    void* desc;
    std::vector<Want> wants;
};
const char* const kName = "seqmix.Call";

void free_call(PyObject* o) { delete static_cast<Call*>(PyCapsule_GetPointer(o, kName)); }

bool numbers(PyObject* seq, std::vector<int64_t>* out) {
    const Py_ssize_t n = PySequence_Size(seq);
    for (Py_ssize_t i = 0; i < n; ++i) {
        PyObject* v = PySequence_GetItem(seq, i);
        if (!v) return false;
        out->push_back(PyLong_AsLongLong(v));
        Py_DECREF(v);
    }
    return n >= 0 && !PyErr_Occurred();
}

PyObject* make_call(PyObject* args) {
    unsigned long long fn = 0, desc = 0;
    PyObject* list = nullptr;
    if (!PyArg_ParseTuple(args, "KKO!", &fn, &desc, &PyList_Type, &list)) return nullptr;
    Call* c = new Call{reinterpret_cast<void*>(fn), reinterpret_cast<void*>(desc), {}};
    PyObject* capsule = PyCapsule_New(c, kName, free_call);
    if (!capsule) {
        delete c;
        return nullptr;
    }
    const Py_ssize_t n = PyList_GET_SIZE(list);
    bool ok = n <= kMost;
    for (Py_ssize_t i = 0; ok && i < n; ++i) {
        PyObject *like = nullptr, *sizes = nullptr, *strides = nullptr;
        int written = 0;
        ok = PyArg_ParseTuple(PyList_GET_ITEM(list, i), "OOOp", &like, &sizes, &strides, &written) && THPVariable_Check(like);
        if (!ok) break;
        Want w{static_cast<int64_t>(THPVariable_Unpack(like).scalar_type()), written != 0, {}, {}};
        ok = numbers(sizes, &w.sizes) && numbers(strides, &w.strides) && w.sizes.size() == w.strides.size();
        c->wants.push_back(std::move(w));
    }
    if (!ok) {
        Py_DECREF(capsule);
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "seqmix: a call takes up to 10 tensors");
        return nullptr;
    }
    return capsule;
}

// make(fn address, descriptor, [(example tensor of the type, sizes, strides, is written), ...])
PyObject* make(PyObject*, PyObject* args) {
    try {
        return make_call(args);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// The address of t where it is what the call needs.  What stands for a tensor without having memory of its own (in
// a transform, or a fake one) throws when asked for its strides or address, or has the address zero.
bool address(const at::Tensor& t, const Want& w, int64_t device, void** out) {
    if (t.layout() != at::kStrided || t.is_neg()) return false;
    if (t.requires_grad() && c10::GradMode::is_enabled()) return false;  // there is no backward pass
    if (static_cast<int64_t>(t.scalar_type()) != w.element || !t.is_cuda() || t.get_device() != device) return false;
    const auto sizes = t.sizes();
    if (sizes.size() != w.sizes.size()) return false;
    const auto strides = t.strides();
    bool same = true, empty = false;
    for (size_t i = 0; i < sizes.size(); ++i) {
        if (sizes[i] != w.sizes[i]) return false;
        empty |= sizes[i] == 0;
        same &= sizes[i] <= 1 || strides[i] == w.strides[i];
    }
    if (!same && !empty) return false;  // the strides of extents of one and of empty tensors are open
    *out = const_cast<void*>(t.const_data_ptr());
    return *out || empty;
}

// run(call, device, stream, tensor or None, ...): the C function's status, or 1 + the place of the first tensor that does
// not fit.
PyObject* run(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n < 3) {
        PyErr_SetString(PyExc_TypeError, "seqmix: run(call, device, stream, tensors...)");
        return nullptr;
    }
    const Call* c = static_cast<const Call*>(PyCapsule_GetPointer(args[0], kName));
    if (!c) return nullptr;
    const int64_t device = PyLong_AsLongLong(args[1]);
    void* const stream = PyLong_AsVoidPtr(args[2]);
    if (PyErr_Occurred()) return nullptr;
    args += 3;
    const Py_ssize_t tensors = n - 3;
    if (tensors != static_cast<Py_ssize_t>(c->wants.size())) {
        PyErr_SetString(PyExc_TypeError, "seqmix: another number of tensors");
        return nullptr;
    }
    void* p[kMost] = {};
    for (Py_ssize_t i = 0; i < tensors; ++i) {
        if (args[i] == Py_None) continue;
        if (!THPVariable_Check(args[i])) return PyLong_FromSsize_t(1 + i);
        bool fits = false;
        try {
            fits = address(THPVariable_Unpack(args[i]), c->wants[i], device, &p[i]);
        } catch (const std::exception&) {
        }
        if (!fits) return PyLong_FromSsize_t(1 + i);
    }
    for (Py_ssize_t i = 0; i < tensors; ++i)  // graphs that hold an output's former values are to notice
        if (args[i] != Py_None && c->wants[i].out) {
            const at::Tensor& t = THPVariable_Unpack(args[i]);
            if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
        }
    int st = 0;
    using V = void*;
    Py_BEGIN_ALLOW_THREADS;
    switch (tensors) {
        case 8:
            st = reinterpret_cast<int (*)(V, V, V, V, V, V, V, V, V, V)>(c->fn)(c->desc, p[0], p[1], p[2], p[3], p[4], p[5],
                                                                              p[6], p[7], stream);
            break;
        case 9:
            st = reinterpret_cast<int (*)(V, V, V, V, V, V, V, V, V, V, V)>(c->fn)(c->desc, p[0], p[1], p[2], p[3], p[4],
                                                                                 p[5], p[6], p[7], p[8], stream);
            break;
        default:
            st = reinterpret_cast<int (*)(V, V, V, V, V, V, V, V, V, V, V, V)>(c->fn)(
                c->desc, p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], p[9], stream);
    }
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(st);
}

PyMethodDef methods[] = {{"make", make, METH_VARARGS, nullptr},
                         {"run", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(run)), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_seqmix", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__seqmix() { return PyModule_Create(&module); }
