// The per-layer calls of the binding without ctypes: a serving loop calls w4a8_quantize_act and w4a8_linear
// once per layer each, and at a few microseconds of device time the call itself is what it waits for.
// Through ctypes a call cost about 7 us (five to eight pointer objects, a conversion per argument, attribute
// look-ups on the tensors); here the tensors' addresses and strides are read directly, which leaves the
// launch.  Marshalling only: every check and decision is the C-ABI library's.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>

#include "../../include/w4a8.h"

namespace {

// Thrown after a Python error has been set.
struct Raised {};

const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "expected a tensor, got %s", Py_TYPE(o)->tp_name);
        throw Raised{};
    }
    return THPVariable_Unpack(o);
}
void* address(PyObject* o) { return o == Py_None ? nullptr : tensor(o).data_ptr(); }
int64_t integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return v;
}
void check(bool ok, const char* what) {
    if (!ok) {
        PyErr_SetString(PyExc_AssertionError, what);
        throw Raised{};
    }
}

template <class F>
PyObject* guarded(Py_ssize_t nargs, Py_ssize_t want, F f) {
    if (nargs != want) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, nargs);
        return nullptr;
    }
    try {
        return PyLong_FromLong(f());
    } catch (const Raised&) {
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}

// (x, x8, s_x, scale_mode, static_scale or None) -> status
PyObject* quantize_act(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 5, [&]() -> int {
        const at::Tensor &x = tensor(a[0]), &x8 = tensor(a[1]);
        check(x.is_cuda() && x.scalar_type() == at::kBFloat16 && x.dim() == 2 && x.stride(1) == 1,
              "x: BF16 [M, K] on the device, contiguous along K");
        const void* xp = x.data_ptr();
        const int64_t M = x.size(0), K = x.size(1), ldx = x.stride(0), ldx8 = x8.stride(0);
        uint8_t* x8p = static_cast<uint8_t*>(x8.data_ptr());
        float* sp = static_cast<float*>(address(a[2]));
        const int mode = static_cast<int>(integer(a[3]));
        const float* ss = static_cast<const float*>(address(a[4]));
        void* stream = c10::cuda::getCurrentCUDAStream().stream();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = w4a8_quantize_act(xp, M, K, ldx, x8p, ldx8, sp, mode, ss, stream);
        Py_END_ALLOW_THREADS
        return rc;
    });
}

// (x8, s_x, weights, gscale or None, gzero or None, format, s_w, N, K, group, out, out_dtype, workspace or None) -> status
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 13, [&]() -> int {
        const at::Tensor &x8 = tensor(a[0]), &s_w = tensor(a[6]), &out = tensor(a[10]);
        check(x8.dim() == 2, "x8: [M, K]");
        const int64_t M = x8.size(0), N = integer(a[7]), K = integer(a[8]);
        check(x8.size(1) == K, "x8 and the weights differ in K");
        const uint8_t* xp = static_cast<const uint8_t*>(x8.data_ptr());
        const float* sp = static_cast<const float*>(address(a[1]));
        const uint8_t* wp = static_cast<const uint8_t*>(address(a[2]));
        const void* gs = address(a[3]);
        const uint8_t* gz = static_cast<const uint8_t*>(address(a[4]));
        const float* sw = static_cast<const float*>(s_w.data_ptr());
        const int64_t ldx8 = x8.stride(0), ldy = out.stride(0);
        void* yp = out.data_ptr();
        void* ws = address(a[12]);
        const size_t wsn = ws ? tensor(a[12]).nbytes() : 0;
        const int fmt = static_cast<int>(integer(a[5])), group = static_cast<int>(integer(a[9])),
                  od = static_cast<int>(integer(a[11])), sw_stride = s_w.numel() == 1 ? 0 : 1;
        void* stream = c10::cuda::getCurrentCUDAStream().stream();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = w4a8_linear(xp, ldx8, sp, M, wp, gs, gz, fmt, sw, sw_stride, N, K, group, yp, ldy, od, ws, wsn, stream);
        Py_END_ALLOW_THREADS
        return rc;
    });
}

// (M, N, K, format) -> bytes
PyObject* linear_workspace_bytes(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 4, [&]() -> long {
        return static_cast<long>(w4a8_linear_workspace_bytes(integer(a[0]), integer(a[1]), integer(a[2]),
                                                             static_cast<int>(integer(a[3]))));
    });
}

// ---- FP8 layers with block scales, mixture of experts -----------------------------------------------------------
// Tensors may live on another device than the current one: the call runs there, on that device's current stream.
const at::Tensor& on_device(PyObject* o, const char* what, at::ScalarType type, int64_t dim) {
    const at::Tensor& t = tensor(o);
    if (!t.is_cuda() || t.scalar_type() != type || t.dim() != dim || (dim > 0 && t.size(dim - 1) > 1 && t.stride(dim - 1) != 1)) {
        PyErr_Format(PyExc_AssertionError, "%s: expected a %s tensor of %d dimensions on the device, contiguous along the last", what,
                     c10::toString(type), static_cast<int>(dim));
        throw Raised{};
    }
    return t;
}
const at::Tensor& e4m3(PyObject* o, const char* what, int64_t dim) {
    return on_device(o, what, tensor(o).scalar_type() == at::kFloat8_e4m3fn ? at::kFloat8_e4m3fn : at::kByte, dim);
}
// W4A8_OUT_*; also checks what on_device checks
int dtype_of(PyObject* o, const char* what, int64_t dim) {
    const bool fp32 = tensor(o).scalar_type() == at::kFloat;
    on_device(o, what, fp32 ? at::kFloat : at::kBFloat16, dim);
    return fp32 ? W4A8_OUT_FP32 : W4A8_OUT_BF16;
}
void same_device(const at::Tensor& a, const at::Tensor& b) { check(a.device() == b.device(), "tensors on different devices"); }

template <class F>
int run_on(const at::Tensor& t, F f) {
    const c10::cuda::CUDAGuard guard(t.device());
    void* stream = c10::cuda::getCurrentCUDAStream().stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f(stream);
    Py_END_ALLOW_THREADS
    return rc;
}

// From row to row; of a single one (whose stride PyTorch leaves open) its width.
int64_t row_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }

int64_t blocks_of(int64_t n) { return (n + 127) / 128; }

// (x, input_kind, slots or None, x8, s_x) -> status
PyObject* quantize_act_blocks(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 5, [&]() -> int {
        const at::Tensor &x = on_device(a[0], "x", at::kBFloat16, 2), &x8 = e4m3(a[3], "x8", 2), &s_x = on_device(a[4], "s_x", at::kFloat, 2);
        const int kind = static_cast<int>(integer(a[1]));
        const int64_t K = kind == W4A8_CHAIN_INPUT_SILU_MUL ? x.size(1) / 2 : x.size(1);
        check(kind != W4A8_CHAIN_INPUT_SILU_MUL || x.size(1) % 2 == 0, "x: gate and up of equal width");
        check(x8.size(1) == K && s_x.size(1) == blocks_of(K) && s_x.size(0) == x8.size(0), "x8 [rows, K] and s_x [rows, ceil(K / 128)]");
        same_device(x, x8);
        same_device(x, s_x);
        const int32_t* slots = nullptr;
        int top_k = 0;
        if (a[2] != Py_None) {
            const at::Tensor& t = on_device(a[2], "slots", at::kInt, 2);
            check(t.is_contiguous() && t.size(0) == x.size(0), "slots: [M, top_k], contiguous");
            same_device(x, t);
            slots = static_cast<const int32_t*>(t.data_ptr());
            top_k = static_cast<int>(t.size(1));
        }
        return run_on(x, [&](void* stream) {
            return w4a8_quantize_act_blocks(x.data_ptr(), x.size(0), K, row_stride(x), kind, slots, top_k, static_cast<uint8_t*>(x8.data_ptr()),
                                            x8.size(0), row_stride(x8), static_cast<float*>(s_x.data_ptr()), row_stride(s_x), stream);
        });
    });
}

// (x8, s_x, offsets or None, w8, s_w, out, out_dtype) -> status; with offsets the experts' products
PyObject* linear_fp8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 7, [&]() -> int {
        const bool experts = a[2] != Py_None;
        const int64_t d = experts ? 3 : 2;
        const at::Tensor &x8 = e4m3(a[0], "x8", 2), &s_x = on_device(a[1], "s_x", at::kFloat, 2), &w8 = e4m3(a[3], "w8", d),
                         &s_w = on_device(a[4], "s_w", at::kFloat, d), &out = tensor(a[5]);
        const int od = static_cast<int>(integer(a[6]));
        check(dtype_of(a[5], "out", 2) == od, "out and out_dtype differ");
        const int64_t M = x8.size(0), K = x8.size(1), N = w8.size(d - 2), E = experts ? w8.size(0) : 1;
        check(w8.size(d - 1) == K, "x8 and w8 differ in K");
        check(s_x.size(0) == M && s_x.size(1) == blocks_of(K), "s_x: [M, ceil(K / 128)]");
        check(s_w.is_contiguous() && s_w.size(d - 2) == blocks_of(N) && s_w.size(d - 1) == blocks_of(K) && (!experts || s_w.size(0) == E),
              "s_w: a scale per 128 x 128 weights, contiguous");
        check(out.size(0) == M && out.size(1) == N, "out: [M, N]");
        same_device(x8, s_x);
        same_device(x8, w8);
        same_device(x8, s_w);
        same_device(x8, out);
        const uint8_t *xp = static_cast<const uint8_t*>(x8.data_ptr()), *wp = static_cast<const uint8_t*>(w8.data_ptr());
        const float *sx = static_cast<const float*>(s_x.data_ptr()), *sw = static_cast<const float*>(s_w.data_ptr());
        if (!experts)
            return run_on(x8, [&](void* stream) {
                return w4a8_linear_fp8_blocks(xp, row_stride(x8), sx, row_stride(s_x), M, wp, row_stride(w8), sw, N, K, out.data_ptr(),
                                              row_stride(out), od, stream);
            });
        const at::Tensor& offsets = on_device(a[2], "offsets", at::kInt, 1);
        check(offsets.size(0) == E + 1, "offsets: [experts + 1]");
        same_device(x8, offsets);
        const int64_t ldw = w8.stride(1), w_stride = E > 1 ? w8.stride(0) : N * ldw;
        return run_on(x8, [&](void* stream) {
            return w4a8_linear_fp8_experts(xp, row_stride(x8), sx, row_stride(s_x), M, static_cast<const int32_t*>(offsets.data_ptr()), E, wp,
                                           ldw, w_stride, sw, N, K, out.data_ptr(), row_stride(out), od, stream);
        });
    });
}

// (logits, score, bias or None, groups, top_groups, group_best, renormalize, scale, ids, weights, offsets, slots, workspace or None) -> status
PyObject* route_experts(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 13, [&]() -> int {
        const int dtype = dtype_of(a[0], "logits", 2);
        const at::Tensor &logits = tensor(a[0]), &ids = on_device(a[8], "ids", at::kInt, 2), &weights = on_device(a[9], "weights", at::kFloat, 2),
                         &offsets = on_device(a[10], "offsets", at::kInt, 1), &slots = on_device(a[11], "slots", at::kInt, 2);
        const int64_t M = logits.size(0), E = logits.size(1), k = ids.size(1);
        check(ids.is_contiguous() && weights.is_contiguous() && slots.is_contiguous() && ids.size(0) == M && weights.sizes() == ids.sizes() &&
                  slots.sizes() == ids.sizes() && offsets.size(0) == E + 1,
              "ids, weights and slots: [M, top_k], contiguous; offsets: [E + 1]");
        const float* bias = nullptr;
        if (a[2] != Py_None) {
            const at::Tensor& b = on_device(a[2], "bias", at::kFloat, 1);
            check(b.size(0) == E, "bias: [E]");
            same_device(logits, b);
            bias = static_cast<const float*>(b.data_ptr());
        }
        void* ws = nullptr;
        size_t wsn = 0;
        if (a[12] != Py_None) {
            const at::Tensor& w = tensor(a[12]);
            check(w.is_cuda() && w.is_contiguous(), "workspace: contiguous, on the device");
            same_device(logits, w);
            ws = w.data_ptr();
            wsn = w.nbytes();
        }
        same_device(logits, ids);
        same_device(logits, weights);
        same_device(logits, offsets);
        same_device(logits, slots);
        const int score = static_cast<int>(integer(a[1])), groups = static_cast<int>(integer(a[3])), top_groups = static_cast<int>(integer(a[4])),
                  best = static_cast<int>(integer(a[5])), renormalize = static_cast<int>(integer(a[6]));
        const double scale = PyFloat_AsDouble(a[7]);
        if (scale == -1.0 && PyErr_Occurred()) throw Raised{};
        return run_on(logits, [&](void* stream) {
            return w4a8_route_experts(logits.data_ptr(), dtype, M, row_stride(logits), E, static_cast<int>(k), score, bias, groups, top_groups, best,
                                      renormalize, static_cast<float>(scale), static_cast<int32_t*>(ids.data_ptr()),
                                      static_cast<float*>(weights.data_ptr()), static_cast<int32_t*>(offsets.data_ptr()),
                                      static_cast<int32_t*>(slots.data_ptr()), ws, wsn, stream);
        });
    });
}

// (y, slots, weights, add or None, out) -> status
PyObject* combine_experts(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 5, [&]() -> int {
        const int yd = dtype_of(a[0], "y", 2), od = dtype_of(a[4], "out", 2);
        const at::Tensor &y = tensor(a[0]), &out = tensor(a[4]), &slots = on_device(a[1], "slots", at::kInt, 2),
                         &weights = on_device(a[2], "weights", at::kFloat, 2);
        const int64_t M = slots.size(0), N = y.size(1);
        check(slots.is_contiguous() && weights.is_contiguous() && weights.sizes() == slots.sizes(), "slots and weights: [M, top_k], contiguous");
        check(out.size(0) == M && out.size(1) == N, "out: [M, N]");
        const void* add = nullptr;
        int64_t ldadd = 0;
        if (a[3] != Py_None) {
            const at::Tensor& t = tensor(a[3]);
            check(dtype_of(a[3], "add", 2) == od && t.sizes() == out.sizes(), "add: of the shape and type of the result");
            same_device(y, t);
            add = t.data_ptr();
            ldadd = row_stride(t);
        }
        same_device(y, slots);
        same_device(y, weights);
        same_device(y, out);
        return run_on(y, [&](void* stream) {
            return w4a8_combine_experts(y.data_ptr(), yd, y.size(0), row_stride(y), static_cast<const int32_t*>(slots.data_ptr()),
                                        static_cast<const float*>(weights.data_ptr()), M, static_cast<int>(slots.size(1)), N, add, ldadd,
                                        out.data_ptr(), row_stride(out), od, stream);
        });
    });
}

PyMethodDef methods[] = {
    {"quantize_act_blocks", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(quantize_act_blocks)), METH_FASTCALL, nullptr},
    {"linear_fp8", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear_fp8)), METH_FASTCALL, nullptr},
    {"route_experts", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(route_experts)), METH_FASTCALL, nullptr},
    {"combine_experts", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(combine_experts)), METH_FASTCALL, nullptr},
    {"quantize_act", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(quantize_act)), METH_FASTCALL, nullptr},
    {"linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear)), METH_FASTCALL, nullptr},
    {"linear_workspace_bytes", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear_workspace_bytes)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
// (the versions that it was compiled against: the build looks for them and compiles again for others)
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_w4a8_host", W4A8_HOST_VERSIONS, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__w4a8_host(void) { return PyModule_Create(&module); }
