// CPython entry to the device calls: takes the torch tensors as they are and calls the C ABI.
//
// What bounds a short call is the host: with thirteen arguments marshalled through ctypes, and a method call or two on every
// tensor, calls on a 4096 x 4096 layer followed each other every 10.8 us although the kernel runs 5; here a tensor
// costs a type check and a pointer read, and they follow every 5.1 us.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "fq.h"

namespace {

// What a call of the tensor library threw (a tensor without storage, or of a kind that has no strides) as a Python error: nothing
// may leave a C entry.
template <class F>
bool guarded(F&& f) {
    try {
        return f();
    } catch (const c10::Error& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return false;
}

// Device pointer of a contiguous CUDA tensor; None is the null pointer.  `written`: the call writes to it, so that a
// tensor that shares its storage until it is written gets one of its own.  `bytes` (if given): its size.
bool device_pointer(PyObject* o, void** out, bool written = false, size_t* bytes = nullptr) {
    if (bytes) *bytes = 0;
    if (o == Py_None) {
        *out = nullptr;
        return true;
    }
    if (!THPVariable_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "expected a torch tensor");
        return false;
    }
    return guarded([&] {
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda() || !t.is_contiguous()) {
            PyErr_SetString(PyExc_ValueError, "expected a contiguous CUDA tensor");
            return false;
        }
        *out = written ? t.mutable_data_ptr() : const_cast<void*>(t.const_data_ptr());
        if (bytes) *bytes = t.nbytes();
        return true;
    });
}

// The stream's handle: the given stream object's, or the current stream of the current device.
bool stream_handle(PyObject* o, void** out) {
    if (o == Py_None)                                      // (throws where there is no usable device)
        return guarded([&] {
            *out = c10::cuda::getCurrentCUDAStream().stream();
            return true;
        });
    PyObject* h = PyObject_GetAttrString(o, "cuda_stream");
    if (!h) return false;
    *out = PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    return !PyErr_Occurred();
}

bool host_pointer(PyObject* o, void** out) {
    *out = PyLong_AsVoidPtr(o);
    return !PyErr_Occurred();
}

struct LayoutView {
    Py_buffer b{};
    bool held = false;
    ~LayoutView() { if (held) PyBuffer_Release(&b); }
    const fq_layout_t* get(PyObject* o) {
        if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) return nullptr;
        held = true;
        if ((size_t)b.len != sizeof(fq_layout_t)) {
            PyErr_SetString(PyExc_TypeError, "expected a Layout");
            return nullptr;
        }
        return (const fq_layout_t*)b.buf;
    }
};

bool take(PyObject* const* args, Py_ssize_t n, Py_ssize_t want) {
    if (n != want) PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
    return n == want;
}

// L, X, M, wq, scale, zero, tile_indptr, bucket_info, packed, Y, workspace, stream -> status
PyObject* fused(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!take(a, n, 12)) return nullptr;
    LayoutView lv;
    const fq_layout_t* L = lv.get(a[0]);
    if (!L) return nullptr;
    const unsigned long M = PyLong_AsUnsignedLongMask(a[2]);
    if (PyErr_Occurred()) return nullptr;
    void *X, *w[6], *Y, *ws, *stream;
    if (!device_pointer(a[1], &X)) return nullptr;
    for (int i = 0; i < 6; ++i)
        if (!device_pointer(a[3 + i], &w[i])) return nullptr;
    size_t ws_bytes;
    if (!device_pointer(a[9], &Y, true) || !device_pointer(a[10], &ws, true, &ws_bytes) || !stream_handle(a[11], &stream)) return nullptr;
    fq_status_t st;
    Py_BEGIN_ALLOW_THREADS
    st = fq_fused_w4a16_outlier_gemm(L, X, (uint32_t)M, w[0], w[1], w[2], w[3], w[4], w[5], Y, ws, ws_bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

// L, X_host, M, x_dev, wq, scale, zero, tile_indptr, bucket_info, packed, y_dev, Y_host, workspace, stream, wait -> status
PyObject* host_io(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!take(a, n, 15)) return nullptr;
    LayoutView lv;
    const fq_layout_t* L = lv.get(a[0]);
    if (!L) return nullptr;
    const unsigned long M = PyLong_AsUnsignedLongMask(a[2]);
    if (PyErr_Occurred()) return nullptr;
    void *xh, *yh, *x, *w[6], *y, *ws, *stream;
    if (!host_pointer(a[1], &xh) || !host_pointer(a[11], &yh) || !device_pointer(a[3], &x, true)) return nullptr;
    for (int i = 0; i < 6; ++i)
        if (!device_pointer(a[4 + i], &w[i])) return nullptr;
    size_t ws_bytes;
    if (!device_pointer(a[10], &y, true) || !device_pointer(a[12], &ws, true, &ws_bytes) || !stream_handle(a[13], &stream)) return nullptr;
    const auto call = a[14] == Py_True ? fq_fused_host_io : fq_fused_host_io_async;
    fq_status_t st;
    Py_BEGIN_ALLOW_THREADS
    st = call(L, xh, (uint32_t)M, x, w[0], w[1], w[2], w[3], w[4], w[5], y, yh, ws, ws_bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

// ---- microscaled FP4 operators: shapes, types and strides are the tensors', and all are on one device, which the call is made on

struct MxArgs {
    int device = -1;
    bool no(const char* name, const char* what) {
        PyErr_Format(PyExc_ValueError, "%s: %s", name, what);
        return false;
    }
    // A strided CUDA tensor, on the device of the others.
    bool tensor(const at::Tensor& t, const char* name) {
        if (!t.is_cuda() || t.layout() != at::kStrided) return no(name, "expected a strided CUDA tensor");
        if (device >= 0 && t.get_device() != device) return no(name, "is on another device than the tensors before it");
        device = t.get_device();
        return true;
    }
    static void* pointer(const at::Tensor& t, bool written) { return written ? t.mutable_data_ptr() : const_cast<void*>(t.const_data_ptr()); }
    bool type_of(const at::Tensor& t, const char* name, uint32_t* type) {
        switch (t.scalar_type()) {
            case at::kBFloat16: *type = FQ_TYPE_BF16; return true;
            case at::kHalf: *type = FQ_TYPE_FP16; return true;
            case at::kFloat: *type = FQ_TYPE_FP32; return true;
            default: return no(name, "expected bfloat16, float16 or float32");
        }
    }
    // rows x cols values with adjacent columns.  `type`: what it has to be, or ~0 to be told.  `one_row`: a single row for all, or a row
    // stride of 0, gives *ld = 0.
    bool matrix(PyObject* o, const char* name, uint64_t rows, uint64_t cols, bool written, uint32_t* type, void** p, uint64_t* ld, bool one_row = false) {
        if (!THPVariable_Check(o)) return no(name, "expected a torch tensor");
        return guarded([&] {
            const at::Tensor& t = THPVariable_Unpack(o);
            uint32_t ty;
            if (!tensor(t, name) || !type_of(t, name, &ty)) return false;
            if (*type != ~0u && ty != *type) return no(name, "has another type than the tensors before it");
            *type = ty;
            const bool single = one_row && t.dim() == 2 && (t.size(0) == 1 || t.stride(0) == 0);
            if (t.dim() != 2 || (uint64_t)t.size(1) != cols || ((uint64_t)t.size(0) != rows && !(one_row && t.size(0) == 1))) {
                PyErr_Format(PyExc_ValueError, "%s: expected %llu x %llu values", name, (unsigned long long)rows, (unsigned long long)cols);
                return false;
            }
            if (cols > 1 && t.stride(1) != 1) return no(name, "expected adjacent columns");
            *ld = single ? 0 : t.size(0) == 1 ? cols : (uint64_t)t.stride(0);
            *p = pointer(t, written);
            return true;
        });
    }
    bool vector(PyObject* o, const char* name, uint64_t n, uint32_t type, void** p) {
        *p = nullptr;
        if (o == Py_None) return true;
        if (!THPVariable_Check(o)) return no(name, "expected a torch tensor");
        return guarded([&] {
            const at::Tensor& t = THPVariable_Unpack(o);
            uint32_t ty;
            if (!tensor(t, name) || !type_of(t, name, &ty)) return false;
            if (ty != type) return no(name, "has another type than the tensors before it");
            if (!t.is_contiguous() || (uint64_t)t.numel() != n) return no(name, "expected a contiguous vector, one value for each column");
            *p = pointer(t, false);
            return true;
        });
    }
    // at least `need` contiguous bytes
    bool bytes(PyObject* o, const char* name, size_t need, bool written, void** p, size_t* have = nullptr) {
        if (!THPVariable_Check(o)) return no(name, "expected a torch tensor");
        return guarded([&] {
            const at::Tensor& t = THPVariable_Unpack(o);
            if (!tensor(t, name)) return false;
            if (!t.is_contiguous()) return no(name, "expected a contiguous tensor");
            if (t.nbytes() < need) {
                PyErr_Format(PyExc_ValueError, "%s: holds %zu bytes, %zu needed", name, (size_t)t.nbytes(), need);
                return false;
            }
            if (have) *have = t.nbytes();
            *p = pointer(t, written);
            return true;
        });
    }
    bool scale(PyObject* o, const char* name, const float** p) {
        *p = nullptr;
        if (o == Py_None) return true;
        if (!THPVariable_Check(o)) return no(name, "expected a torch tensor");
        return guarded([&] {
            const at::Tensor& t = THPVariable_Unpack(o);
            if (!tensor(t, name)) return false;
            if (t.scalar_type() != at::kFloat || t.numel() != 1) return no(name, "expected one float32 value");
            *p = (const float*)pointer(t, false);
            return true;
        });
    }
    // Runs f(stream) with the tensors' device current: on the given stream, or on that device's current one.
    template <class F>
    PyObject* run(PyObject* stream, F&& f) {
        fq_status_t st = FQ_OK;
        void* given = nullptr;
        if (stream != Py_None) {
            if (!stream_handle(stream, &given)) return nullptr;
            PyObject* d = PyObject_GetAttrString(stream, "device_index");
            if (!d) return nullptr;
            const long at = PyLong_AsLong(d);
            Py_DECREF(d);
            if (PyErr_Occurred()) return nullptr;
            if (at != device) return no("stream", "is on another device than the tensors"), nullptr;
        }
        const bool ok = guarded([&] {
            const c10::cuda::CUDAGuard guard((c10::DeviceIndex)device);
            void* s = stream == Py_None ? (void*)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream() : given;
            Py_BEGIN_ALLOW_THREADS
            st = f(s);
            Py_END_ALLOW_THREADS
            return true;
        });
        return ok ? PyLong_FromLong(st) : nullptr;
    }
};

struct MxLayoutView {
    fq_mx_layout_t L{};
    size_t codes = 0, scales = 0;
    // a layout that the library refuses has sizes 0 here, and is refused by the call itself
    bool get(PyObject* o) {
        Py_buffer b{};
        if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) return false;
        const bool fits = (size_t)b.len == sizeof(L);
        if (fits) memcpy(&L, b.buf, sizeof(L));
        PyBuffer_Release(&b);
        if (!fits) PyErr_SetString(PyExc_TypeError, "expected an MxLayout");
        else if (fq_mx_sizes(&L, &codes, &scales) != FQ_OK) codes = scales = 0;
        return fits;
    }
};

// L, X, codes, scales, tensor_scale, stream -> status
PyObject* mx_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    MxLayoutView v;
    if (!take(a, n, 6) || !v.get(a[0])) return nullptr;
    MxArgs m;
    void *x, *c, *s;
    const float* ts;
    uint32_t type = ~0u;
    uint64_t ld;
    if (!m.bytes(a[2], "codes", v.codes, true, &c) || !m.bytes(a[3], "scales", v.scales, true, &s) ||
        !m.matrix(a[1], "X", v.L.rows, v.L.K, false, &type, &x, &ld) || !m.scale(a[4], "tensor_scale", &ts))
        return nullptr;
    return m.run(a[5], [&](void* st) { return fq_mx_quantize(&v.L, x, type, ld, ts, c, s, st); });
}

// L, gate, up, codes, scales, tensor_scale, stream -> status
PyObject* mx_quantize_swiglu(PyObject*, PyObject* const* a, Py_ssize_t n) {
    MxLayoutView v;
    if (!take(a, n, 7) || !v.get(a[0])) return nullptr;
    MxArgs m;
    void *g, *u, *c, *s;
    const float* ts;
    uint32_t type = ~0u;
    uint64_t lg, lu;
    if (!m.bytes(a[3], "codes", v.codes, true, &c) || !m.bytes(a[4], "scales", v.scales, true, &s) ||
        !m.matrix(a[1], "gate", v.L.rows, v.L.K, false, &type, &g, &lg) || !m.matrix(a[2], "up", v.L.rows, v.L.K, false, &type, &u, &lu) ||
        !m.scale(a[5], "tensor_scale", &ts))
        return nullptr;
    return m.run(a[6], [&](void* st) { return fq_mx_quantize_swiglu(&v.L, g, lg, u, lu, type, ts, c, s, st); });
}

// L, codes, scales, Y, tensor_scale, stream -> status
PyObject* mx_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    MxLayoutView v;
    if (!take(a, n, 6) || !v.get(a[0])) return nullptr;
    MxArgs m;
    void *y, *c, *s;
    const float* ts;
    uint32_t type = ~0u;
    uint64_t ld;
    if (!m.matrix(a[3], "Y", v.L.rows, v.L.K, true, &type, &y, &ld) || !m.bytes(a[1], "codes", v.codes, false, &c) ||
        !m.bytes(a[2], "scales", v.scales, false, &s) || !m.scale(a[4], "tensor_scale", &ts))
        return nullptr;
    return m.run(a[5], [&](void* st) { return fq_mx_dequantize(&v.L, c, s, ts, y, type, ld, st); });
}

// LX, x_codes, x_scales, x_tensor_scale, LW, w_codes, w_scales, w_tensor_scale, Y, workspace, stream -> status
PyObject* mx_gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    MxLayoutView x, w;
    if (!take(a, n, 11) || !x.get(a[0]) || !w.get(a[4])) return nullptr;
    MxArgs m;
    void *y, *ws, *xc, *xs, *wc, *wsc;
    const float *xt, *wt;
    uint32_t type = ~0u;
    uint64_t ld;
    size_t ws_bytes;
    if (!m.matrix(a[8], "Y", x.L.rows, w.L.rows, true, &type, &y, &ld) || !m.bytes(a[9], "workspace", 0, true, &ws, &ws_bytes) ||
        !m.bytes(a[1], "x_codes", x.codes, false, &xc) || !m.bytes(a[2], "x_scales", x.scales, false, &xs) || !m.scale(a[3], "x_tensor_scale", &xt) ||
        !m.bytes(a[5], "w_codes", w.codes, false, &wc) || !m.bytes(a[6], "w_scales", w.scales, false, &wsc) || !m.scale(a[7], "w_tensor_scale", &wt))
        return nullptr;
    return m.run(a[10], [&](void* st) { return fq_mx_gemm(&x.L, xc, xs, xt, &w.L, wc, wsc, wt, y, type, ld, ws, ws_bytes, st); });
}

// X, eps, block, block_weight, gate, residual_scale, R, weight, H, layout, codes, scales, tensor_scale, stream -> status
PyObject* norm_block(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!take(a, n, 14)) return nullptr;
    fq_norm_args_t p{};
    MxArgs m;
    MxLayoutView v;
    p.eps = (float)PyFloat_AsDouble(a[1]);
    p.residual_scale = (float)PyFloat_AsDouble(a[5]);
    if (PyErr_Occurred()) return nullptr;
    if (!THPVariable_Check(a[0])) return m.no("X", "expected a torch tensor"), nullptr;
    uint64_t rows = 0, D = 0;
    if (!guarded([&] {
            const at::Tensor& t = THPVariable_Unpack(a[0]);
            if (t.layout() != at::kStrided || t.dim() != 2 || t.size(0) > 0xffffffffll || t.size(1) > 0xffffffffll) return m.no("X", "expected a matrix");
            rows = (uint64_t)t.size(0), D = (uint64_t)t.size(1);
            return true;
        }))
        return nullptr;
    p.rows = (uint32_t)rows, p.D = (uint32_t)D;
    uint32_t type = ~0u;
    void* q;
    auto optional = [&](int i, const char* name, bool written, void** to, uint64_t* ld, bool one_row = false) {
        *to = nullptr;
        return a[i] == Py_None || m.matrix(a[i], name, rows, D, written, &type, to, ld, one_row);
    };
    // what is written first: a tensor that shares its storage until it is written then has its own when an input's address is taken
    if (!optional(6, "R", true, &p.R, &p.ld_r) || !optional(8, "H", true, &p.H, &p.ld_h)) return nullptr;
    if (a[9] != Py_None) {
        if (!v.get(a[9]) || !m.bytes(a[10], "codes", v.codes, true, &p.codes) || !m.bytes(a[11], "scales", v.scales, true, &p.scales)) return nullptr;
        p.layout = &v.L;
    } else if (a[10] != Py_None || a[11] != Py_None) {
        return m.no("layout", "codes and scales need one"), nullptr;
    }
    if (!m.matrix(a[0], "X", rows, D, false, &type, &q, &p.ld_x)) return nullptr;
    p.X = q;
    if (!optional(2, "block", false, &q, &p.ld_block)) return nullptr;
    p.block = q;
    if (!optional(4, "gate", false, &q, &p.ld_gate, true)) return nullptr;
    p.gate = q;
    if (!m.vector(a[3], "block_weight", D, type, &q)) return nullptr;
    p.block_weight = q;
    if (!m.vector(a[7], "weight", D, type, &q)) return nullptr;
    p.weight = q;
    if (!m.scale(a[12], "tensor_scale", &p.tensor_scale)) return nullptr;
    p.type = type;
    return m.run(a[13], [&](void* st) { return fq_norm_block(&p, st); });
}

PyMethodDef methods[] = {
    {"fused", (PyCFunction)(void (*)(void))fused, METH_FASTCALL, nullptr},
    {"host_io", (PyCFunction)(void (*)(void))host_io, METH_FASTCALL, nullptr},
    {"mx_quantize", (PyCFunction)(void (*)(void))mx_quantize, METH_FASTCALL, nullptr},
    {"mx_quantize_swiglu", (PyCFunction)(void (*)(void))mx_quantize_swiglu, METH_FASTCALL, nullptr},
    {"mx_dequantize", (PyCFunction)(void (*)(void))mx_dequantize, METH_FASTCALL, nullptr},
    {"mx_gemm", (PyCFunction)(void (*)(void))mx_gemm, METH_FASTCALL, nullptr},
    {"norm_block", (PyCFunction)(void (*)(void))norm_block, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fqcall", nullptr, -1, methods};

}  // namespace

// `built_for`: the torch whose C++ interface this file was compiled against.
PyMODINIT_FUNC PyInit__fqcall(void) {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", FQ_TORCH_TAG) != 0) Py_CLEAR(m);
    return m;
}
