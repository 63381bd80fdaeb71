// One call of a device entry point of the C ABI from Python: checks the tensors, takes their addresses and sizes and the
// current stream, and calls.  The same marshalling in Python and ctypes cost 4 to 8 us a call, of the 6 to 10 us a small call
// took altogether (a training step of 384 units of 49 tokens was bound by its four calls: 29 us for 21 us of kernels).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

using P = const void*;
using W = void*;   // (pointers are passed alike whatever they point to)
constexpr int kMaxTensors = 11;

// call(address, stream or None, v, same_dtype, tau or None, tensor, ...): status of the entry point.  Sizes come from the
// four dimensions of the first tensor and, with v >= 0, the last of tensor v; a None among the tensors is a null pointer.
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    const Py_ssize_t nt = nargs - 5;
    if (nt < 1 || nt > kMaxTensors) {
        PyErr_SetString(PyExc_TypeError, "call(address, stream, v, same_dtype, tau, tensor, ...)");
        return nullptr;
    }
    void* fn = PyLong_AsVoidPtr(args[0]);
    if (!fn) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null entry point");
        return nullptr;
    }
    const long vi = PyLong_AsLong(args[2]);
    const int same = PyObject_IsTrue(args[3]);
    const bool has_tau = args[4] != Py_None;
    const float tau = has_tau ? (float)PyFloat_AsDouble(args[4]) : 0.f;
    if (PyErr_Occurred()) return nullptr;
    W p[kMaxTensors];
    int d[5] = {0, 0, 0, 0, 0};
    at::ScalarType type = at::ScalarType::Undefined;
    for (Py_ssize_t i = 0; i < nt; ++i) {
        PyObject* o = args[5 + i];
        if (o == Py_None && i > 0) {
            p[i] = nullptr;
            continue;
        }
        if (!THPVariable_Check(o)) {
            PyErr_SetString(PyExc_TypeError, "device entry points take torch tensors");
            return nullptr;
        }
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda() || !t.is_contiguous()) {
            PyErr_SetString(PyExc_ValueError, "device entry points take contiguous CUDA tensors");
            return nullptr;
        }
        if (i == 0 || i == vi) {
            if (t.dim() != 4) {
                PyErr_SetString(PyExc_ValueError, "tensors of four dimensions expected");
                return nullptr;
            }
            if (i == 0)
                for (int x = 0; x < 4; ++x) d[x] = (int)t.size(x);
            if (i == vi) d[4] = (int)t.size(3);
        }
        if (i == 0) type = t.scalar_type();
        else if (same && t.scalar_type() != type) {
            PyErr_SetString(PyExc_ValueError, "all tensors of one call share a dtype");
            return nullptr;
        }
        p[i] = t.data_ptr();
    }
    W stream = nullptr;
    if (args[1] == Py_None) {
        stream = c10::cuda::getCurrentCUDAStream().stream();
    } else {
        stream = PyLong_AsVoidPtr(args[1]);
        if (PyErr_Occurred()) return nullptr;
    }
    int status = 0;
    bool known = true;
    const int kind = (int)nt * 4 + (vi >= 0 ? 2 : 0) + (has_tau ? 1 : 0);
    Py_BEGIN_ALLOW_THREADS
    switch (kind) {
        case 4 * 4 + 0:
            status = reinterpret_cast<int (*)(P, P, P, W, int, int, int, int, W)>(fn)(p[0], p[1], p[2], p[3], d[0], d[1], d[2], d[3], stream);
            break;
        case 4 * 4 + 1:
            status = reinterpret_cast<int (*)(P, P, W, W, int, int, int, int, float, W)>(fn)(p[0], p[1], p[2], p[3], d[0], d[1], d[2], d[3], tau, stream);
            break;
        case 6 * 4 + 1:
            status = reinterpret_cast<int (*)(P, P, P, P, W, W, int, int, int, int, float, W)>(fn)(p[0], p[1], p[2], p[3], p[4], p[5], d[0], d[1], d[2],
                                                                                                   d[3], tau, stream);
            break;
        case 6 * 4 + 2:
            status = reinterpret_cast<int (*)(P, P, P, P, P, W, int, int, int, int, int, W)>(fn)(p[0], p[1], p[2], p[3], p[4], p[5], d[0], d[1], d[2],
                                                                                                 d[3], d[4], stream);
            break;
        case 6 * 4 + 3:
            status = reinterpret_cast<int (*)(P, P, P, P, P, W, int, int, int, int, int, float, W)>(fn)(p[0], p[1], p[2], p[3], p[4], p[5], d[0], d[1],
                                                                                                        d[2], d[3], d[4], tau, stream);
            break;
        case 8 * 4 + 3:
            status = reinterpret_cast<int (*)(P, P, P, P, P, P, P, W, int, int, int, int, int, float, W)>(fn)(
                p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], d[0], d[1], d[2], d[3], d[4], tau, stream);
            break;
        case 11 * 4 + 2:
            status = reinterpret_cast<int (*)(P, P, P, P, P, P, W, W, W, W, W, int, int, int, int, int, W)>(fn)(
                p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], p[9], p[10], d[0], d[1], d[2], d[3], d[4], stream);
            break;
        default: known = false;
    }
    Py_END_ALLOW_THREADS
    if (!known) {
        PyErr_SetString(PyExc_TypeError, "no entry point takes these arguments");
        return nullptr;
    }
    return PyLong_FromLong(status);
    END_HANDLE_TH_ERRORS
}

// ---- gated delta rule, group norm: sizes from the tensors, and every tensor checked against them -----------------------------
struct Shape {
    int n;
    int64_t d[4];
};

// The address of a contiguous CUDA tensor of the current device, of this type and shape; None where that is allowed: null.
bool take(PyObject* o, const char* name, at::ScalarType type, const Shape& shape, bool optional, W* p) {
    *p = nullptr;
    if (o == Py_None && optional) return true;
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s: a torch tensor expected", name);
        return false;
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous()) {
        PyErr_Format(PyExc_ValueError, "%s: device entry points take contiguous CUDA tensors", name);
        return false;
    }
    if (t.device().index() != c10::cuda::current_device()) {
        PyErr_Format(PyExc_ValueError, "%s: on device %d, the current one is %d", name, (int)t.device().index(), (int)c10::cuda::current_device());
        return false;
    }
    if (t.scalar_type() != type) {
        PyErr_Format(PyExc_ValueError, "%s: dtype %s expected, got %s", name, c10::toString(type), c10::toString(t.scalar_type()));
        return false;
    }
    bool same = t.dim() == shape.n;
    for (int i = 0; same && i < shape.n; ++i) same = t.size(i) == shape.d[i];
    if (!same) {
        PyErr_Format(PyExc_ValueError, "%s: its shape does not fit the other tensors'", name);
        return false;
    }
    *p = t.data_ptr();
    return true;
}

// The tensor that the sizes come from: of n dimensions, bf16 or fp32.
bool lead(PyObject* o, const char* name, int n, at::ScalarType* type, Shape* shape) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s: a torch tensor expected", name);
        return false;
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.dim() != n) {
        PyErr_Format(PyExc_ValueError, "%s: %d dimensions expected", name, n);
        return false;
    }
    *type = t.scalar_type();
    if (*type != at::kBFloat16 && *type != at::kFloat) {
        PyErr_Format(PyExc_ValueError, "%s: bf16 or fp32 tensors only", name);
        return false;
    }
    shape->n = n;
    for (int i = 0; i < n; ++i) {
        shape->d[i] = t.size(i);
        if (shape->d[i] > 0x7fffffff) {
            PyErr_Format(PyExc_ValueError, "%s: a dimension beyond 32 bits", name);
            return false;
        }
    }
    return true;
}

bool stream_of(PyObject* o, W* stream) {
    *stream = o == Py_None ? (W)c10::cuda::getCurrentCUDAStream().stream() : PyLong_AsVoidPtr(o);
    return !PyErr_Occurred();
}

// The entry point of the type: addresses come as (bf16, fp32).
void* entry(PyObject* const* args, at::ScalarType type) { return PyLong_AsVoidPtr(args[type == at::kFloat ? 1 : 0]); }

bool count(const char* usage, Py_ssize_t nargs, Py_ssize_t want) {
    if (nargs == want) return true;
    PyErr_SetString(PyExc_TypeError, usage);
    return false;
}

template <typename F>
PyObject* without_gil(F f) {
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = f();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

// gdr_fwd(bf16, fp32, stream, reverse, q, k, v, log_alpha, beta, state_in, out, state_out)
PyObject* gdr_fwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (!count("gdr_fwd takes twelve arguments", nargs, 12)) return nullptr;
    at::ScalarType T, Tv;
    Shape q, v;
    W stream, p[8];
    const int reverse = PyObject_IsTrue(args[3]);
    if (reverse < 0 || !lead(args[4], "q", 4, &T, &q) || !lead(args[6], "v", 4, &Tv, &v)) return nullptr;
    const Shape vs = {4, {q.d[0], q.d[1], q.d[2], v.d[3]}}, gate = {3, {q.d[0], q.d[1], q.d[2]}}, state = {4, {q.d[0], q.d[1], q.d[3], v.d[3]}};
    PyObject* const* t = args + 4;
    if (!take(t[0], "q", T, q, false, p) || !take(t[1], "k", T, q, false, p + 1) || !take(t[2], "v", T, vs, false, p + 2) ||
        !take(t[3], "log_alpha", T, gate, false, p + 3) || !take(t[4], "beta", T, gate, false, p + 4) ||
        !take(t[5], "state_in", at::kFloat, state, true, p + 5) || !take(t[6], "out", T, vs, false, p + 6) ||
        !take(t[7], "state_out", at::kFloat, state, true, p + 7))
        return nullptr;
    void* fn = entry(args, T);
    if (!fn || !stream_of(args[2], &stream)) return nullptr;
    return without_gil([&] {
        return reinterpret_cast<int (*)(P, P, P, P, P, P, W, W, int, int, int, int, int, int, W)>(fn)(
            p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], (int)q.d[0], (int)q.d[1], (int)q.d[2], (int)q.d[3], (int)v.d[3], reverse, stream);
    });
    END_HANDLE_TH_ERRORS
}

// gdr_bwd(bf16, fp32, stream, reverse, q, k, v, log_alpha, beta, state_in, d_out, d_state_out, dq, dk, dv, dlog_alpha, dbeta, d_state_in)
PyObject* gdr_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (!count("gdr_bwd takes eighteen arguments", nargs, 18)) return nullptr;
    at::ScalarType T, Tv;
    Shape q, v;
    W stream, p[14];
    const int reverse = PyObject_IsTrue(args[3]);
    if (reverse < 0 || !lead(args[4], "q", 4, &T, &q) || !lead(args[6], "v", 4, &Tv, &v)) return nullptr;
    const Shape vs = {4, {q.d[0], q.d[1], q.d[2], v.d[3]}}, gate = {3, {q.d[0], q.d[1], q.d[2]}}, state = {4, {q.d[0], q.d[1], q.d[3], v.d[3]}};
    const struct {
        const char* name;
        at::ScalarType type;
        const Shape* shape;
        bool optional;
    } want[14] = {{"q", T, &q, false},          {"k", T, &q, false},   {"v", T, &vs, false},   {"log_alpha", T, &gate, false},
                  {"beta", T, &gate, false},    {"state_in", at::kFloat, &state, true},        {"d_out", T, &vs, false},
                  {"d_state_out", at::kFloat, &state, true},           {"dq", T, &q, false},   {"dk", T, &q, false},
                  {"dv", T, &vs, false},        {"dlog_alpha", T, &gate, false},               {"dbeta", T, &gate, false},
                  {"d_state_in", at::kFloat, &state, true}};
    for (int i = 0; i < 14; ++i)
        if (!take(args[4 + i], want[i].name, want[i].type, *want[i].shape, want[i].optional, p + i)) return nullptr;
    void* fn = entry(args, T);
    if (!fn || !stream_of(args[2], &stream)) return nullptr;
    return without_gil([&] {
        return reinterpret_cast<int (*)(P, P, P, P, P, P, P, P, W, W, W, W, W, W, int, int, int, int, int, int, W)>(fn)(
            p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], p[9], p[10], p[11], p[12], p[13], (int)q.d[0], (int)q.d[1], (int)q.d[2], (int)q.d[3],
            (int)v.d[3], reverse, stream);
    });
    END_HANDLE_TH_ERRORS
}

// gdr_step(bf16, fp32, stream, q, k, v, log_alpha, beta, state, out)
PyObject* gdr_step(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (!count("gdr_step takes ten arguments", nargs, 10)) return nullptr;
    at::ScalarType T, Tv;
    Shape q, v;
    W stream, p[7];
    if (!lead(args[3], "q", 3, &T, &q) || !lead(args[5], "v", 3, &Tv, &v)) return nullptr;
    const Shape vs = {3, {q.d[0], q.d[1], v.d[2]}}, gate = {2, {q.d[0], q.d[1]}}, state = {4, {q.d[0], q.d[1], q.d[2], v.d[2]}};
    PyObject* const* t = args + 3;
    if (!take(t[0], "q", T, q, false, p) || !take(t[1], "k", T, q, false, p + 1) || !take(t[2], "v", T, vs, false, p + 2) ||
        !take(t[3], "log_alpha", T, gate, false, p + 3) || !take(t[4], "beta", T, gate, false, p + 4) ||
        !take(t[5], "state", at::kFloat, state, false, p + 5) || !take(t[6], "out", T, vs, false, p + 6))
        return nullptr;
    void* fn = entry(args, T);
    if (!fn || !stream_of(args[2], &stream)) return nullptr;
    return without_gil([&] {
        return reinterpret_cast<int (*)(P, P, P, P, P, W, W, int, int, int, int, W)>(fn)(p[0], p[1], p[2], p[3], p[4], p[5], p[6], (int)q.d[0],
                                                                                         (int)q.d[1], (int)q.d[2], (int)v.d[2], stream);
    });
    END_HANDLE_TH_ERRORS
}

int small_int(PyObject* o) {
    const long x = PyLong_AsLong(o);
    if (!PyErr_Occurred() && (x > 0x7fffffffL || x < -0x7fffffffL)) PyErr_SetString(PyExc_ValueError, "a size beyond 32 bits");
    return (int)x;
}

// group_norm(bf16, fp32, stream, groups, eps, act, x, weight, bias, out, mean, rstd)
PyObject* group_norm(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (!count("group_norm takes twelve arguments", nargs, 12)) return nullptr;
    at::ScalarType T;
    Shape x;
    W stream, p[6];
    const int groups = small_int(args[3]);
    const double eps = PyFloat_AsDouble(args[4]);
    const int act = small_int(args[5]);
    if (PyErr_Occurred() || !lead(args[6], "x", 4, &T, &x)) return nullptr;
    const Shape ch = {1, {x.d[3]}}, stats = {2, {x.d[0], groups}};
    PyObject* const* t = args + 6;
    if (!take(t[0], "x", T, x, false, p) || !take(t[1], "weight", T, ch, true, p + 1) || !take(t[2], "bias", T, ch, true, p + 2) ||
        !take(t[3], "out", T, x, false, p + 3) || !take(t[4], "mean", at::kFloat, stats, true, p + 4) || !take(t[5], "rstd", at::kFloat, stats, true, p + 5))
        return nullptr;
    void* fn = entry(args, T);
    if (!fn || !stream_of(args[2], &stream)) return nullptr;
    return without_gil([&] {
        return reinterpret_cast<int (*)(P, P, P, W, W, W, int, int, int, int, int, float, int, W)>(fn)(
            p[0], p[1], p[2], p[3], p[4], p[5], (int)x.d[0], (int)x.d[1], (int)x.d[2], (int)x.d[3], groups, (float)eps, act, stream);
    });
    END_HANDLE_TH_ERRORS
}

// group_norm_bwd(bf16, fp32, stream, groups, act, x, weight, bias, mean, rstd, d_out, dx, dweight, dbias)
PyObject* group_norm_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (!count("group_norm_bwd takes fourteen arguments", nargs, 14)) return nullptr;
    at::ScalarType T;
    Shape x;
    W stream, p[9];
    const int groups = small_int(args[3]);
    const int act = small_int(args[4]);
    if (PyErr_Occurred() || !lead(args[5], "x", 4, &T, &x)) return nullptr;
    const Shape ch = {1, {x.d[3]}}, stats = {2, {x.d[0], groups}};
    PyObject* const* t = args + 5;
    if (!take(t[0], "x", T, x, false, p) || !take(t[1], "weight", T, ch, true, p + 1) || !take(t[2], "bias", T, ch, true, p + 2) ||
        !take(t[3], "mean", at::kFloat, stats, false, p + 3) || !take(t[4], "rstd", at::kFloat, stats, false, p + 4) ||
        !take(t[5], "d_out", T, x, false, p + 5) || !take(t[6], "dx", T, x, false, p + 6) || !take(t[7], "dweight", T, ch, true, p + 7) ||
        !take(t[8], "dbias", T, ch, true, p + 8))
        return nullptr;
    void* fn = entry(args, T);
    if (!fn || !stream_of(args[2], &stream)) return nullptr;
    return without_gil([&] {
        return reinterpret_cast<int (*)(P, P, P, P, P, P, W, W, W, int, int, int, int, int, int, W)>(fn)(
            p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], (int)x.d[0], (int)x.d[1], (int)x.d[2], (int)x.d[3], groups, act, stream);
    });
    END_HANDLE_TH_ERRORS
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name, const char* doc) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, doc};
}

PyMethodDef kMethods[] = {method<call>("call", "calls a device entry point"),
                          method<gdr_fwd>("gdr_fwd", "calls vig_gdr_fwd_*"),
                          method<gdr_bwd>("gdr_bwd", "calls vig_gdr_bwd_*"),
                          method<gdr_step>("gdr_step", "calls vig_gdr_step_*"),
                          method<group_norm>("group_norm", "calls vig_group_norm_*"),
                          method<group_norm_bwd>("group_norm_bwd", "calls vig_group_norm_bwd_*"),
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_binding_call", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding_call() { return PyModule_Create(&kModule); }
