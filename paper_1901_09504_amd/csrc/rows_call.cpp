// The Python side of the calls with a grid per row and of token scoring: marshalling only, as binding.py does for the other calls through
// ctypes.  These four are made once or twice per generated token, on work of 2 to 6 us, and a ctypes call of 20 arguments costs the host
// 1.9 to 2.7 us beside the 3.2 of a launch; this takes the tensors as they are and costs 0.6 to 1.0.
//
// bind(float32, bfloat16, float16, current_device, current_raw_stream) comes first.  A tensor argument may be None (NULL), or False as
// a layer without a bias says it; an element type is its tensor's own, -1 for any other; stream is None (the current one) or has a
// `cuda_stream`.  Every call returns the OCS_E_* code.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/ocs.h"

static PyObject *s_data_ptr, *s_dtype, *s_nbytes, *s_cuda_stream;
static PyObject *types[3], *current_device, *current_stream;

// Reads the arguments in turn; after the first that does not fit, `ok` is false, a Python error is set and the rest read as zero.
struct Args {
    PyObject* const* at;
    bool ok;
    explicit Args(PyObject* const* args, Py_ssize_t given, Py_ssize_t want) : at(args), ok(given == want) {
        if (!ok) PyErr_Format(PyExc_TypeError, "%zd arguments given, %zd wanted", given, want);
        else if (current_stream == nullptr) {
            ok = false;
            PyErr_SetString(PyExc_RuntimeError, "bind() comes first");
        }
    }
    long long int64() {
        if (!ok) return 0;
        const long long v = PyLong_AsLongLong(*at++);
        if (v == -1 && PyErr_Occurred()) ok = false;
        return v;
    }
    int int32() {
        const long long v = int64();
        if (ok && v != (int)v) {
            ok = false;
            PyErr_SetString(PyExc_OverflowError, "an argument does not fit 32 bits");
        }
        return (int)v;
    }
    float number() {
        if (!ok) return 0.0f;
        const double v = PyFloat_AsDouble(*at++);
        if (v == -1.0 && PyErr_Occurred()) ok = false;
        return (float)v;
    }
    // the value of a Python integer, which this takes over
    void* address(PyObject* value) {
        if (value == nullptr) {
            ok = false;
            return nullptr;
        }
        void* p = PyLong_AsVoidPtr(value);
        Py_DECREF(value);
        if (p == nullptr && PyErr_Occurred()) ok = false;
        return p;
    }
    void* tensor() {
        if (!ok) return nullptr;
        PyObject* t = *at++;
        return t == Py_None || t == Py_False ? nullptr : address(PyObject_CallMethodNoArgs(t, s_data_ptr));
    }
    template <typename T>
    T* tensor_of() {
        return static_cast<T*>(tensor());
    }
    // the element type of the next argument, which tensor() then reads
    int type() {
        if (!ok || *at == Py_None) return -1;
        PyObject* d = PyObject_GetAttr(*at, s_dtype);
        if (d == nullptr) {
            ok = false;
            return -1;
        }
        Py_DECREF(d);                                              // torch keeps its types
        for (int i = 0; i < 3; ++i)
            if (d == types[i]) return i;
        return -1;
    }
    size_t nbytes() {                                              // of the next argument, as type()
        if (!ok || *at == Py_None) return 0;
        PyObject* n = PyObject_GetAttr(*at, s_nbytes);
        const size_t v = n == nullptr ? 0 : PyLong_AsSize_t(n);
        Py_XDECREF(n);
        if (PyErr_Occurred()) ok = false;
        return v;
    }
    void* stream() {
        if (!ok) return nullptr;
        PyObject* s = *at++;
        if (s != Py_None) return address(PyObject_GetAttr(s, s_cuda_stream));
        PyObject* device = PyObject_CallNoArgs(current_device);
        if (device == nullptr) {
            ok = false;
            return nullptr;
        }
        PyObject* raw = PyObject_CallOneArg(current_stream, device);
        Py_DECREF(device);
        return address(raw);
    }
};

// The call itself, with the interpreter free for other threads: a full queue makes a launch wait.
template <typename F>
static PyObject* answer(const Args& a, F call) {
    if (!a.ok) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject* split_quantize_rows(PyObject*, PyObject* const* args, Py_ssize_t given) {
    Args a(args, given, 14);
    const int type = a.type();
    const void* X = a.tensor();
    const int64_t M = a.int64();
    const int C = a.int32(), g = a.int32();
    const int64_t ldx = a.int64();
    const int32_t* src = a.tensor_of<int32_t>();
    const int32_t* depth = a.tensor_of<int32_t>();
    const int s = a.int32(), bits = a.int32();
    const float clip = a.number();
    int8_t* Xq = a.tensor_of<int8_t>();
    const int64_t ldq = a.int64();
    float* step = a.tensor_of<float>();
    void* stream = a.stream();
    return answer(a, [&] { return ocs_split_quantize_rows(X, type, M, C, g, ldx, src, depth, s, bits, clip, Xq, ldq, step, stream); });
}

static PyObject* qgemm_rows(PyObject*, PyObject* const* args, Py_ssize_t given) {
    Args a(args, given, 15);
    const int8_t* Xq = a.tensor_of<int8_t>();
    const int64_t ldx = a.int64();
    const int8_t* Wq = a.tensor_of<int8_t>();
    const int64_t ldw = a.int64(), M = a.int64(), N = a.int64(), K = a.int64();
    const int bx = a.int32(), bw = a.int32();
    const float* sx = a.tensor_of<float>();
    const float* sw = a.tensor_of<float>();
    const float* bias = a.tensor_of<float>();
    const int type = a.type();
    void* Y = a.tensor();
    const int64_t ldy = a.int64();
    void* stream = a.stream();
    return answer(a, [&] { return ocs_qgemm_rows(Xq, ldx, Wq, ldw, M, N, K, bx, bw, sx, sw, bias, Y, type, ldy, stream); });
}

static PyObject* forward_rows(PyObject*, PyObject* const* args, Py_ssize_t given) {
    Args a(args, given, 21);
    const int type = a.type();
    const void* X = a.tensor();
    const int64_t M = a.int64();
    const int C = a.int32(), g = a.int32();
    const int64_t ldx = a.int64();
    const int32_t* src = a.tensor_of<int32_t>();
    const int s = a.int32(), bx = a.int32();
    const float clip = a.number();
    int8_t* Xq = a.tensor_of<int8_t>();
    const int64_t ldq = a.int64();
    float* step = a.tensor_of<float>();
    const int8_t* Wq = a.tensor_of<int8_t>();
    const int64_t ldw = a.int64(), N = a.int64();
    const int bw = a.int32();
    const float* sw = a.tensor_of<float>();
    const float* bias = a.tensor_of<float>();
    const int out = a.type();
    void* Y = a.tensor();
    const int64_t ldy = a.int64();
    void* stream = a.stream();
    return answer(a, [&] {
        return ocs_forward_rows(X, type, M, C, g, ldx, src, s, bx, clip, Xq, ldq, step, Wq, ldw, N, bw, sw, bias, Y, out, ldy, stream);
    });
}

static PyObject* token_logprobs(PyObject*, PyObject* const* args, Py_ssize_t given) {
    Args a(args, given, 12);
    const int type = a.type();
    const void* logits = a.tensor();
    const int64_t M = a.int64(), V = a.int64(), ld = a.int64();
    const int32_t* tokens = a.tensor_of<int32_t>();
    const int k = a.int32();
    float* logprob = a.tensor_of<float>();
    float* entropy = a.tensor_of<float>();
    int32_t* ids = a.tensor_of<int32_t>();
    float* top = a.tensor_of<float>();
    const size_t bytes = a.nbytes();
    void* workspace = a.tensor();
    void* stream = a.stream();
    return answer(a, [&] { return ocs_token_logprobs(logits, type, M, V, ld, tokens, k, logprob, entropy, ids, top, workspace, bytes, stream); });
}

static PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t given) {
    if (given != 5) {
        PyErr_SetString(PyExc_TypeError, "three element types, the current device's and the current stream's function");
        return nullptr;
    }
    PyObject** to[5] = {&types[0], &types[1], &types[2], &current_device, &current_stream};
    for (int i = 0; i < 5; ++i) {
        Py_INCREF(args[i]);
        PyObject* old = *to[i];
        *to[i] = args[i];
        Py_XDECREF(old);
    }
    Py_RETURN_NONE;
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
static PyMethodDef methods[] = {METHOD(bind),         METHOD(split_quantize_rows), METHOD(qgemm_rows),
                                METHOD(forward_rows), METHOD(token_logprobs),      {nullptr, nullptr, 0, nullptr}};
static PyModuleDef module = {PyModuleDef_HEAD_INIT, "_rows_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

PyMODINIT_FUNC PyInit__rows_call(void) {
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_nbytes = PyUnicode_InternFromString("nbytes");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    if (!s_data_ptr || !s_dtype || !s_nbytes || !s_cuda_stream) return nullptr;
    return PyModule_Create(&module);
}
