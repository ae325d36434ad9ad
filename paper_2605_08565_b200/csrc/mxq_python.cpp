// The calls of binding.py that sit in a caller's inner loop, with their arguments unpacked in C++ instead of ctypes: a ctypes call of
// fifteen arguments and the tensors' attributes cost 2.5 to 3.5 us, which is what the kernels of a small tensor take on the GPU.  Every function takes what its Python counterpart takes and
// returns the library's status, or -1 for arguments it does not know (anything but None or a contiguous CUDA tensor of
// type Tensor or Parameter for a pointer, an int, a float): the caller then goes through ctypes, which converts or refuses them.  us a call on
// the host's side of a pass, ctypes -> here: abs-max and quantization of 4 x 4096 activations 10.1 -> 5.2, quantize + MSE of 37 K
// elements 8.6 -> 5.1, the seven calls that score a recipe on 130 K elements 32 -> 24.
// The library is not linked: bind() receives the addresses of its functions.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/mxq.h"

namespace {

// The library's functions, by name as bind() finds them.
struct Library {
    decltype(&mxq_quantize_ex) quantize_ex;
    decltype(&mxq_quantize_mse) quantize_mse;
    decltype(&mxq_quantize_batch) quantize_batch;
    decltype(&mxq_fake_quantize) fake_quantize;
    decltype(&mxq_tensor_amax) tensor_amax;
    decltype(&mxq_tensor_mse) tensor_mse;
    decltype(&mxq_dequantize_ex) dequantize_ex;
    decltype(&mxq_block_clip_sse) block_clip_sse;
    decltype(&mxq_histograms) histograms;
    decltype(&mxq_segment_mse) segment_mse;
    decltype(&mxq_quantize8) quantize8;
    decltype(&mxq_dequantize8) dequantize8;
    decltype(&mxq_add_rmsnorm8) add_rmsnorm8;
    decltype(&mxq_add_rmsnorm8_backward) add_rmsnorm8_backward;
    decltype(&mxq_swiglu8) swiglu8;
    decltype(&mxq_swiglu8_backward) swiglu8_backward;
    decltype(&mxq_set_option) set_option;
} lib;
bool bound = false;

// Arguments of one call, read in order; `ok` falls with the first one that is not of the expected kind.
struct Args {
    PyObject* const* a;
    bool ok;
    Args(PyObject* const* args, Py_ssize_t n, Py_ssize_t expected) : a(args), ok(n == expected) {}

    const at::Tensor* tensor(int i) {
        if (!ok || !THPVariable_CheckExact(a[i])) {
            ok = false;
            return nullptr;
        }
        const at::Tensor& t = THPVariable_Unpack(a[i]);
        if (!t.is_cuda() || !t.is_contiguous()) ok = false;
        return &t;
    }
    void* ptr(int i) {
        if (!ok || a[i] == Py_None) return nullptr;
        const at::Tensor* t = tensor(i);
        return ok ? t->data_ptr() : nullptr;
    }
    int dtype(int i) {   // after ptr(i)
        if (!ok || a[i] == Py_None) {
            ok = false;
            return 0;
        }
        const auto d = THPVariable_Unpack(a[i]).scalar_type();
        if (d != at::kFloat && d != at::kBFloat16) ok = false;
        return d == at::kFloat ? MXQ_F32 : MXQ_BF16;
    }
    size_t bytes(int i) {
        if (!ok || a[i] == Py_None) return 0;
        return THPVariable_Unpack(a[i]).nbytes();
    }
    size_t size(int i) {
        if (!ok || !PyLong_Check(a[i])) {
            ok = false;
            return 0;
        }
        const size_t v = PyLong_AsSize_t(a[i]);
        if (v == (size_t)-1 && PyErr_Occurred()) {
            PyErr_Clear();
            ok = false;
        }
        return v;
    }
    int integer(int i) {
        if (!ok || !PyLong_Check(a[i])) {
            ok = false;
            return 0;
        }
        const long v = PyLong_AsLong(a[i]);
        if ((v == -1 && PyErr_Occurred()) || v != (int)v) {
            PyErr_Clear();
            ok = false;
        }
        return (int)v;
    }
    float number(int i) {
        if (!ok || !PyFloat_Check(a[i])) {   // an int among others
            ok = false;
            return 0.0f;
        }
        return (float)PyFloat_AS_DOUBLE(a[i]);
    }
    // None: the current stream of the device that the tensor a[like] lies on; else an object with a cuda_stream
    void* stream(int i, int like) {
        if (!ok) return nullptr;
        if (a[i] == Py_None) {
            const at::Tensor* t = tensor(like);
            return ok ? (void*)c10::cuda::getCurrentCUDAStream(t->get_device()).stream() : nullptr;
        }
        PyObject* s = PyObject_GetAttrString(a[i], "cuda_stream");
        void* p = s != nullptr && PyLong_Check(s) ? PyLong_AsVoidPtr(s) : nullptr;
        if (s == nullptr || !PyLong_Check(s) || (p == nullptr && PyErr_Occurred())) {
            PyErr_Clear();
            ok = false;
        }
        Py_XDECREF(s);
        return p;
    }
};

// Tensors of the operators on 8-bit activations, checked against the first wide one of the call (rows x cols of one type, on the current
// device).  What binding.py would refuse, or views differently, is left to it.
struct Args8 : Args {
    int64_t rows = -1, cols = 0, blocks = 0;
    int type = 0, device = -1, block_size = 0, elem = 0;

    Args8(PyObject* const* args, Py_ssize_t n, Py_ssize_t expected, int i_block, int i_elem) : Args(args, n, expected) {
        block_size = integer(i_block);
        elem = integer(i_elem);
        if (block_size != 16 && block_size != 32 && block_size != 64 && block_size != 128) ok = false;
    }
    const at::Tensor* any(int i) {
        if (!ok || !THPVariable_CheckExact(a[i])) {
            ok = false;
            return nullptr;
        }
        const at::Tensor& t = THPVariable_Unpack(a[i]);
        if (!t.is_cuda() || t.get_device() != device) ok = false;
        return ok ? &t : nullptr;
    }
    // The call's first wide tensor.
    void first(int i) {
        device = (int)c10::cuda::current_device();
        const at::Tensor* t = any(i);
        if (t == nullptr) return;
        type = dtype(i);
        if (t->dim() == 0 || t->numel() == 0) ok = false;
        if (!ok) return;
        cols = t->size(-1);
        rows = t->numel() / cols;
        blocks = (cols + block_size - 1) / block_size;
    }
    void* wide(int i, size_t& stride, bool optional = false) {
        stride = 0;
        if (optional && ok && a[i] == Py_None) return nullptr;
        const at::Tensor* t = any(i);
        if (t == nullptr) return nullptr;
        const int64_t d = t->dim();
        if (dtype(i) != type || d == 0 || t->size(-1) != cols || t->numel() != rows * cols || (d > 2 && !t->is_contiguous()) || (cols > 1 && t->stride(-1) != 1)) ok = false;
        if (!ok) return nullptr;
        const int64_t s = d == 2 && rows > 1 ? t->stride(0) : cols;
        if (s < 0) ok = false;
        stride = (size_t)s;
        return t->data_ptr();
    }
    uint8_t* bytes_of(int i, int64_t count, at::ScalarType other, bool optional) {
        if (optional && ok && a[i] == Py_None) return nullptr;
        const at::Tensor* t = any(i);
        if (t == nullptr) return nullptr;
        if ((t->scalar_type() != at::kByte && t->scalar_type() != other) || !t->is_contiguous() || t->numel() != count) ok = false;
        return ok ? (uint8_t*)t->data_ptr() : nullptr;
    }
    uint8_t* codes(int i, bool optional = false) { return bytes_of(i, rows * cols, elem == MXQ_E4M3 ? at::kFloat8_e4m3fn : at::kFloat8_e5m2, optional); }
    uint8_t* scales(int i, bool optional = false) { return bytes_of(i, rows * blocks, at::kFloat8_e8m0fnu, optional); }
    float* floats(int i, int64_t count, bool optional = false) {
        if (optional && ok && a[i] == Py_None) return nullptr;
        const at::Tensor* t = any(i);
        if (t == nullptr) return nullptr;
        if (t->scalar_type() != at::kFloat || !t->is_contiguous() || t->numel() != count) ok = false;
        return ok ? (float*)t->data_ptr() : nullptr;
    }
    void* weight(int i, int& wtype) {
        wtype = 0;
        const at::Tensor* t = any(i);
        if (t == nullptr) return nullptr;
        wtype = dtype(i);
        if (!t->is_contiguous() || t->numel() != cols) ok = false;
        return ok ? t->data_ptr() : nullptr;
    }
    // As Args::stream, for a tensor whose device is the current one and that need not be contiguous.
    void* stream8(int i) {
        if (!ok) return nullptr;
        if (a[i] == Py_None) return (void*)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
        return stream(i, 0);
    }
};

// Calls f() without the interpreter's lock, as ctypes does.
template <typename F>
PyObject* status_of(const Args& a, F f) {
    if (!a.ok) return PyLong_FromLong(-1);
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = f();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

// A tensor without storage and the like throws where its address is asked for: left to the caller's other path.
template <PyObject* (*BODY)(PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (!bound) return PyLong_FromLong(-1);
    try {
        return BODY(args, n);
    } catch (...) {
        PyErr_Clear();
        return PyLong_FromLong(-1);
    }
}

// The arguments are read into locals first: the lambda runs without the lock and touches no Python object.
PyObject* quantize_ex(PyObject* const* p, Py_ssize_t np) {
    Args a(p, np, 11);
    const void* x = a.ptr(0);
    const int dt = a.dtype(0);
    const size_t n = a.size(1);
    const int B = a.integer(2), fmt = a.integer(3), recipe = a.integer(4);
    const float g = a.number(5);
    const float* dg = (const float*)a.ptr(6);
    uint8_t *codes = (uint8_t*)a.ptr(7), *scales = (uint8_t*)a.ptr(8);
    float* sse = (float*)a.ptr(9);
    void* s = a.stream(10, 0);
    return status_of(a, [&] { return lib.quantize_ex(x, dt, n, B, fmt, recipe, g, dg, codes, scales, sse, s); });
}

PyObject* quantize_mse(PyObject* const* p, Py_ssize_t np) {
    Args a(p, np, 13);
    const void* x = a.ptr(0);
    const int dt = a.dtype(0);
    const size_t n = a.size(1);
    const int B = a.integer(2), fmt = a.integer(3), recipe = a.integer(4);
    const float g = a.number(5);
    const float* dg = (const float*)a.ptr(6);
    uint8_t *codes = (uint8_t*)a.ptr(7), *scales = (uint8_t*)a.ptr(8);
    float* sse = (float*)a.ptr(9);
    double* mse = (double*)a.ptr(10);
    void* ws = a.ptr(11);
    const size_t ws_bytes = a.bytes(11);
    void* s = a.stream(12, 0);
    return status_of(a, [&] { return lib.quantize_mse(x, dt, n, B, fmt, recipe, g, dg, codes, scales, sse, mse, ws, ws_bytes, s); });
}

PyObject* quantize_batch(PyObject* const* p, Py_ssize_t np) {   // h_descs: its address
    Args a(p, np, 10);
    const size_t h = a.size(0);
    const mxq_tensor_desc* d = (const mxq_tensor_desc*)a.ptr(1);
    const size_t nt = a.size(2);
    const int dt = a.integer(3), B = a.integer(4), fmt = a.integer(5), recipe = a.integer(6);
    const float g = a.number(7);
    const float* dg = (const float*)a.ptr(8);
    void* s = a.stream(9, 1);
    return status_of(a, [&] { return lib.quantize_batch((const mxq_tensor_desc*)h, d, nt, dt, B, fmt, recipe, g, dg, s); });
}

PyObject* fake_quantize(PyObject* const* p, Py_ssize_t np) {
    Args a(p, np, 9);
    const void* x = a.ptr(0);
    const int dt = a.dtype(0);
    const size_t n = a.size(1);
    const int B = a.integer(2), fmt = a.integer(3), recipe = a.integer(4);
    const float g = a.number(5);
    const float* dg = (const float*)a.ptr(6);
    void* out = a.ptr(7);
    const int odt = a.dtype(7);
    void* s = a.stream(8, 0);
    return status_of(a, [&] { return lib.fake_quantize(x, dt, n, B, fmt, recipe, g, dg, out, odt, s); });
}

PyObject* tensor_amax(PyObject* const* p, Py_ssize_t np) {
    Args a(p, np, 5);
    const void* x = a.ptr(0);
    const int dt = a.dtype(0);
    const size_t n = a.size(1);
    float *amax = (float*)a.ptr(2), *g = (float*)a.ptr(3);
    void* s = a.stream(4, 0);
    return status_of(a, [&] { return lib.tensor_amax(x, dt, n, amax, g, s); });
}

PyObject* tensor_mse(PyObject* const* p, Py_ssize_t np) {
    Args a(p, np, 6);
    const float* sse = (const float*)a.ptr(0);
    const size_t nb = a.size(1), n = a.size(2);
    double* out = (double*)a.ptr(3);
    void* ws = a.ptr(4);
    const size_t ws_bytes = a.bytes(4);
    void* s = a.stream(5, 0);
    return status_of(a, [&] { return lib.tensor_mse(sse, nb, n, out, ws, ws_bytes, s); });
}

PyObject* dequantize_ex(PyObject* const* p, Py_ssize_t np) {
    Args a(p, np, 9);
    const uint8_t *codes = (const uint8_t*)a.ptr(0), *scales = (const uint8_t*)a.ptr(1);
    const size_t n = a.size(2);
    const int B = a.integer(3), fmt = a.integer(4);
    const float g = a.number(5);
    const float* dg = (const float*)a.ptr(6);
    void* out = a.ptr(7);
    const int odt = a.dtype(7);
    void* s = a.stream(8, 7);
    return status_of(a, [&] { return lib.dequantize_ex(codes, scales, n, B, fmt, g, dg, out, odt, s); });
}

PyObject* block_clip_sse(PyObject* const* p, Py_ssize_t np) {
    Args a(p, np, 9);
    const void* x = a.ptr(0);
    const int dt = a.dtype(0);
    const size_t n = a.size(1);
    const int B = a.integer(2), fmt = a.integer(3);
    const float g = a.number(4);
    const float* dg = (const float*)a.ptr(5);
    const uint8_t* scales = (const uint8_t*)a.ptr(6);
    float* out = (float*)a.ptr(7);
    void* s = a.stream(8, 0);
    return status_of(a, [&] { return lib.block_clip_sse(x, dt, n, B, fmt, g, dg, scales, out, s); });
}

PyObject* histograms(PyObject* const* p, Py_ssize_t np) {
    Args a(p, np, 7);
    const uint8_t *codes = (const uint8_t*)a.ptr(0), *scales = (const uint8_t*)a.ptr(1);
    const size_t n = a.size(2);
    const int B = a.integer(3);
    auto *ch = (unsigned long long*)a.ptr(4), *sh = (unsigned long long*)a.ptr(5);
    void* s = a.stream(6, 0);
    return status_of(a, [&] { return lib.histograms(codes, scales, n, B, ch, sh, s); });
}

PyObject* segment_mse(PyObject* const* p, Py_ssize_t np) {
    Args a(p, np, 6);
    const float* sse = (const float*)a.ptr(0);
    const size_t nb = a.size(1), per = a.size(2), elems = a.size(3);
    double* out = (double*)a.ptr(4);
    void* s = a.stream(5, 0);
    return status_of(a, [&] { return lib.segment_mse(sse, nb, per, elems, out, s); });
}

PyObject* quantize8(PyObject* const* p, Py_ssize_t np) {
    Args8 a(p, np, 6, 1, 2);
    size_t sx;
    a.first(0);
    const void* x = a.wide(0, sx);
    uint8_t *codes = a.codes(3), *scales = a.scales(4);
    void* s = a.stream8(5);
    return status_of(a, [&] { return lib.quantize8(x, a.type, a.rows, a.cols, sx, a.block_size, a.elem, codes, scales, s); });
}

PyObject* dequantize8(PyObject* const* p, Py_ssize_t np) {
    Args8 a(p, np, 6, 2, 3);
    size_t so;
    a.first(4);
    void* out = a.wide(4, so);
    const uint8_t *codes = a.codes(0), *scales = a.scales(1);
    void* s = a.stream8(5);
    return status_of(a, [&] { return lib.dequantize8(codes, scales, a.rows, a.cols, a.block_size, a.elem, out, a.type, so, s); });
}

PyObject* add_rmsnorm8(PyObject* const* p, Py_ssize_t np) {
    Args8 a(p, np, 13, 4, 5);
    size_t sx, sr, ss;
    int wt;
    a.first(0);
    const void *x = a.wide(0, sx), *r = a.wide(1, sr, true), *w = a.weight(2, wt);
    const float eps = a.number(3);
    void* sum = a.wide(6, ss, true);
    uint8_t *codes = a.codes(7), *scales = a.scales(8), *kc = a.codes(9, true), *ks = a.scales(10, true);
    float* rstd = a.floats(11, a.rows, true);
    void* s = a.stream8(12);
    return status_of(a, [&] {
        return lib.add_rmsnorm8(x, r, w, a.type, wt, a.rows, a.cols, sx, sr, eps, a.block_size, a.elem, sum, ss, codes, scales, kc, ks, rstd, s);
    });
}

PyObject* add_rmsnorm8_backward(PyObject* const* p, Py_ssize_t np) {
    Args8 a(p, np, 12, 6, 7);
    size_t sy, ss, sx;
    int wt;
    a.first(0);
    const void *dy = a.wide(0, sy), *ds = a.wide(1, ss, true), *w = a.weight(2, wt);
    const uint8_t *kc = a.codes(3), *ks = a.scales(4);
    const float* rstd = a.floats(5, a.rows);
    void* dx = a.wide(8, sx);
    float* dw = a.floats(9, a.cols, true);
    void* ws = a.ptr(10);
    if (a.ok && ws) a.any(10);
    const size_t ws_bytes = a.bytes(10);
    void* s = a.stream8(11);
    return status_of(a, [&] {
        return lib.add_rmsnorm8_backward(dy, ds, w, a.type, wt, a.rows, a.cols, sy, ss, kc, ks, rstd, a.block_size, a.elem, dx, sx, dw, ws, ws_bytes, s);
    });
}

PyObject* swiglu8(PyObject* const* p, Py_ssize_t np) {
    Args8 a(p, np, 11, 2, 3);
    size_t sg, su;
    a.first(0);
    const void *g = a.wide(0, sg), *u = a.wide(1, su);
    uint8_t *codes = a.codes(4), *scales = a.scales(5), *gc = a.codes(6, true), *gs = a.scales(7, true), *uc = a.codes(8, true), *us = a.scales(9, true);
    void* s = a.stream8(10);
    return status_of(a, [&] { return lib.swiglu8(g, u, a.type, a.rows, a.cols, sg, su, a.block_size, a.elem, codes, scales, gc, gs, uc, us, s); });
}

PyObject* swiglu8_backward(PyObject* const* p, Py_ssize_t np) {
    Args8 a(p, np, 10, 5, 6);
    size_t sy, sg, su;
    a.first(0);
    const void* dy = a.wide(0, sy);
    const uint8_t *gc = a.codes(1), *gs = a.scales(2), *uc = a.codes(3), *us = a.scales(4);
    void *dg = a.wide(7, sg), *du = a.wide(8, su);
    void* s = a.stream8(9);
    return status_of(a, [&] { return lib.swiglu8_backward(dy, a.type, a.rows, a.cols, sy, gc, gs, uc, us, a.block_size, a.elem, dg, sg, du, su, s); });
}

PyObject* set_option(PyObject* const* p, Py_ssize_t np) {   // two ints, taken modulo 2^32 as ctypes takes them
    if (np != 2 || !PyLong_Check(p[0]) || !PyLong_Check(p[1])) return PyLong_FromLong(MXQ_ERR_BAD_ENUM);
    return PyLong_FromLong(lib.set_option((int)PyLong_AsUnsignedLongMask(p[0]), (int)PyLong_AsUnsignedLongMask(p[1])));
}

// bind({"mxq_quantize_ex": address, ...})
PyObject* bind(PyObject*, PyObject* addresses) {
    if (!PyDict_Check(addresses)) {
        PyErr_SetString(PyExc_TypeError, "a dict of addresses is expected");
        return nullptr;
    }
    Library l;
    bool ok = true;
    auto get = [&](const char* name) -> void* {
        PyObject* v = PyDict_GetItemString(addresses, name);
        void* p = v != nullptr && PyLong_Check(v) ? PyLong_AsVoidPtr(v) : nullptr;
        if (p == nullptr) ok = false;
        return p;
    };
    l.quantize_ex = (decltype(l.quantize_ex))get("mxq_quantize_ex");
    l.quantize_mse = (decltype(l.quantize_mse))get("mxq_quantize_mse");
    l.quantize_batch = (decltype(l.quantize_batch))get("mxq_quantize_batch");
    l.fake_quantize = (decltype(l.fake_quantize))get("mxq_fake_quantize");
    l.tensor_amax = (decltype(l.tensor_amax))get("mxq_tensor_amax");
    l.tensor_mse = (decltype(l.tensor_mse))get("mxq_tensor_mse");
    l.dequantize_ex = (decltype(l.dequantize_ex))get("mxq_dequantize_ex");
    l.block_clip_sse = (decltype(l.block_clip_sse))get("mxq_block_clip_sse");
    l.histograms = (decltype(l.histograms))get("mxq_histograms");
    l.segment_mse = (decltype(l.segment_mse))get("mxq_segment_mse");
    l.quantize8 = (decltype(l.quantize8))get("mxq_quantize8");
    l.dequantize8 = (decltype(l.dequantize8))get("mxq_dequantize8");
    l.add_rmsnorm8 = (decltype(l.add_rmsnorm8))get("mxq_add_rmsnorm8");
    l.add_rmsnorm8_backward = (decltype(l.add_rmsnorm8_backward))get("mxq_add_rmsnorm8_backward");
    l.swiglu8 = (decltype(l.swiglu8))get("mxq_swiglu8");
    l.swiglu8_backward = (decltype(l.swiglu8_backward))get("mxq_swiglu8_backward");
    l.set_option = (decltype(l.set_option))get("mxq_set_option");
    if (!ok) {
        PyErr_Clear();
        PyErr_SetString(PyExc_ValueError, "an address is missing");
        return nullptr;
    }
    lib = l;
    bound = true;
    Py_RETURN_NONE;
}

#define MXQ_METHOD(f) {#f, (PyCFunction)(void (*)(void))guarded<f>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"bind", bind, METH_O, nullptr},
    MXQ_METHOD(quantize_ex), MXQ_METHOD(quantize_mse), MXQ_METHOD(quantize_batch), MXQ_METHOD(fake_quantize), MXQ_METHOD(tensor_amax),
    MXQ_METHOD(tensor_mse), MXQ_METHOD(dequantize_ex), MXQ_METHOD(block_clip_sse), MXQ_METHOD(histograms), MXQ_METHOD(segment_mse),
    MXQ_METHOD(quantize8), MXQ_METHOD(dequantize8), MXQ_METHOD(add_rmsnorm8), MXQ_METHOD(add_rmsnorm8_backward), MXQ_METHOD(swiglu8),
    MXQ_METHOD(swiglu8_backward), MXQ_METHOD(set_option),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", "libmxq's inner-loop calls without ctypes", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&module); }
