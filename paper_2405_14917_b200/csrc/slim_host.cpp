// The per-call half of the Python binding, as a CPython extension: what binding.py does between a caller's tensors and
// the C ABI for the calls that a decode loop makes per layer (one linear layer, in low bits or in 8-bit floats, one layer set) and
// a training loop per step (the distillation loss).
//
// One token through a 4096 x 4096 layer takes 5.7 us on the device.  Checked and marshalled in Python (six tensors, a
// numpy bit map, the stream, an output, a ctypes call of thirteen arguments) the call took 15 us of the host, so the
// device waited for it; here the tensors are read without the interpreter, and the calls of a loop follow each other every
// 6.0 us (10.2 instead of 16.4 at a group size of 64).  A layer's very first call: 37 -> 24 us.
//
// Nothing is decided here.  A call that is not the plain one (another dtype or layout, a tensor subclass, a bit map that
// is not a one-dimensional uint8 buffer, ...) returns None before anything has been enqueued and binding.py takes its
// general path, which converts or raises.  The entry points of the C ABI arrive as addresses, so this file links
// against nothing of the CUDA library and keeps no state.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

using LinearFn = int (*)(const void*, const void*, const uint8_t*, const void*, const void*, void*, int, int, int, int, void*, size_t, void*);
using SetFn = int (*)(const void*, const void*, void*, size_t, void*);

const at::Tensor* plain(PyObject* o, c10::ScalarType dtype) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.is_cuda() && t.layout() == c10::kStrided && t.scalar_type() == dtype && t.is_contiguous() ? &t : nullptr;
}

bool as_int(PyObject* o, int* out) {
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
    if (overflow != 0 || v < INT_MIN || v > INT_MAX) return false;
    *out = static_cast<int>(v);
    return true;
}

void* stream_of(const at::Tensor& t) { return c10::cuda::getCurrentCUDAStream(t.get_device()).stream(); }

// The bit map of a layer: a one-dimensional uint8 array that numpy can be asked for without a copy.
struct Bits {
    Py_buffer b;
    bool held = false;
    bool open(PyObject* o) {
        if (PyBytes_Check(o) || PyByteArray_Check(o) || PyMemoryView_Check(o)) return false;      // the general path says what they are
        if (PyObject_GetBuffer(o, &b, PyBUF_FORMAT | PyBUF_ND | PyBUF_C_CONTIGUOUS) != 0) { PyErr_Clear(); return false; }
        held = true;
        return b.ndim == 1 && b.itemsize == 1 && b.format != nullptr && b.format[0] == 'B' && b.format[1] == 0;
    }
    ~Bits() { if (held) PyBuffer_Release(&b); }
};

// What torch throws (a tensor without storage or of a layout that has no strides, no memory left) leaves as the Python
// exception that the same call in Python raises.
// linear(address, x, packed, bits, scales, zeros, N, workspace, out or None, g) -> y, or the status of a call that failed, or None (see above)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 10) { PyErr_SetString(PyExc_TypeError, "linear: 10 arguments"); return nullptr; }
    LinearFn fn = reinterpret_cast<LinearFn>(PyLong_AsVoidPtr(a[0]));
    if (fn == nullptr) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "linear: no entry point"); return nullptr; }
    int N = 0, g = 0;
    const at::Tensor *x = plain(a[1], at::kHalf), *packed = plain(a[2], at::kByte), *scales = plain(a[4], at::kHalf),
                     *zeros = plain(a[5], at::kHalf), *ws = plain(a[7], at::kByte);
    if (x == nullptr || packed == nullptr || scales == nullptr || zeros == nullptr || ws == nullptr || x->dim() != 2 ||
        !as_int(a[6], &N) || N < 0 || !as_int(a[9], &g) || x->size(0) > INT_MAX || x->size(1) > INT_MAX)
        Py_RETURN_NONE;
    const at::Tensor* given = nullptr;
    if (a[8] != Py_None && (given = plain(a[8], at::kHalf)) == nullptr) Py_RETURN_NONE;
    Bits bits;
    if (!bits.open(a[3])) Py_RETURN_NONE;
    const int M = static_cast<int>(x->size(0)), K = static_cast<int>(x->size(1));
    at::Tensor fresh;
    if (given == nullptr) fresh = at::empty({M, N}, x->options());
    const at::Tensor& y = given != nullptr ? *given : fresh;
    void *xp = x->data_ptr(), *wp = packed->data_ptr(), *sp = scales->data_ptr(), *zp = zeros->data_ptr(), *yp = y.data_ptr();
    void *wsp = ws->data_ptr(), *stream = stream_of(*x);
    const size_t wsb = static_cast<size_t>(ws->numel());
    int status = 0;
    Py_BEGIN_ALLOW_THREADS                      // the tensors and the bit map are held by the caller's arguments
    status = fn(xp, wp, static_cast<const uint8_t*>(bits.b.buf), sp, zp, yp, M, N, K, g, wsp, wsb, stream);
    Py_END_ALLOW_THREADS
    if (status != 0) return PyLong_FromLong(status);
    return given != nullptr ? Py_NewRef(a[8]) : THPVariable_Wrap(fresh);
    END_HANDLE_TH_ERRORS
}

// run_set(address, launch record, plan, workspace) -> status, or None
PyObject* run_set(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 4) { PyErr_SetString(PyExc_TypeError, "run_set: 4 arguments"); return nullptr; }
    SetFn fn = reinterpret_cast<SetFn>(PyLong_AsVoidPtr(a[0]));
    const void* info = fn != nullptr ? PyLong_AsVoidPtr(a[1]) : nullptr;
    if (fn == nullptr || info == nullptr) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "run_set: no entry point"); return nullptr; }
    const at::Tensor *plan = plain(a[2], at::kByte), *ws = plain(a[3], at::kByte);
    if (plan == nullptr || ws == nullptr) Py_RETURN_NONE;
    void *pp = plan->data_ptr(), *wp = ws->data_ptr(), *stream = stream_of(*plan);
    const size_t wsb = static_cast<size_t>(ws->numel());
    int status = 0;
    Py_BEGIN_ALLOW_THREADS
    status = fn(info, pp, wp, wsb, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
    END_HANDLE_TH_ERRORS
}

using Fp8Fn = int (*)(const void*, int, long long, const void*, const float*, void*, int, long long, int, int, int, void*, size_t, void*);
using DistillLossFn = int (*)(const void*, int, long long, const void*, int, const void*, int, const float*, double, int, int, int, float*, float*, void*);
using DistillGradFn = int (*)(const void*, int, long long, const void*, int, const void*, int, const float*, double, int, int, int, const float*,
                              const float*, void*, long long, void*);
using DistillStepFn = int (*)(const void*, int, long long, const void*, int, const void*, int, const float*, double, int, int, int, const float*, float*,
                              void*, long long, void*);

// SLIM_F32, SLIM_F16, SLIM_BF16, or -1
int element_type(c10::ScalarType t) { return t == at::kFloat ? 0 : t == at::kHalf ? 1 : t == at::kBFloat16 ? 2 : -1; }

// A matrix on the current device whose rows are contiguous and do not overlap; its row stride.
const at::Tensor* rows(PyObject* o, long long* ld) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.layout() != c10::kStrided || t.dim() != 2 || t.size(0) > INT_MAX || t.size(1) > INT_MAX || t.size(1) < 1) return nullptr;
    if ((t.size(1) > 1 && t.stride(1) != 1) || (t.size(0) > 1 && t.stride(0) < t.size(1))) return nullptr;
    *ld = t.size(0) > 1 ? t.stride(0) : t.size(1);
    return &t;
}
bool here(const at::Tensor& t, c10::DeviceIndex d) { return t.get_device() == d; }

// fp8_linear(address, x, codes, scales, workspace, out or None, type of y or -1) -> y, or the status of a call that failed, or None (see above)
PyObject* fp8_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 7) { PyErr_SetString(PyExc_TypeError, "fp8_linear: 7 arguments"); return nullptr; }
    Fp8Fn fn = reinterpret_cast<Fp8Fn>(PyLong_AsVoidPtr(a[0]));
    if (fn == nullptr) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "fp8_linear: no entry point"); return nullptr; }
    long long ldx = 0, ldy = 0;
    int want = -1;
    const at::Tensor *x = rows(a[1], &ldx), *codes = plain(a[2], at::kFloat8_e4m3fn), *scales = plain(a[3], at::kFloat), *ws = plain(a[4], at::kByte);
    if (x == nullptr || codes == nullptr || scales == nullptr || ws == nullptr || codes->dim() != 2 || scales->dim() != 2 || !as_int(a[6], &want)) Py_RETURN_NONE;
    const int xt = element_type(x->scalar_type());
    const long long M = x->size(0), K = x->size(1), N = codes->size(0);
    const c10::DeviceIndex d = c10::cuda::current_device();
    if ((xt != 1 && xt != 2) || codes->size(1) != K || N < 1 || N > INT_MAX || scales->size(0) != (N + 127) / 128 || scales->size(1) != (K + 127) / 128 ||
        !here(*x, d) || !here(*codes, d) || !here(*scales, d) || !here(*ws, d))
        Py_RETURN_NONE;
    const at::Tensor* given = nullptr;
    if (a[5] != Py_None && ((given = rows(a[5], &ldy)) == nullptr || given->size(0) != M || given->size(1) != N || !here(*given, d))) Py_RETURN_NONE;
    const int yt = given != nullptr ? element_type(given->scalar_type()) : want < 0 ? xt : want;
    if ((yt != xt && yt != 0) || (want >= 0 && want != yt)) Py_RETURN_NONE;
    at::Tensor fresh;
    if (given == nullptr) {
        fresh = at::empty({M, N}, yt == 0 ? x->options().dtype(at::kFloat) : x->options());
        ldy = N;
    }
    void *xp = x->data_ptr(), *cp = codes->data_ptr(), *yp = (given != nullptr ? *given : fresh).data_ptr(), *wsp = ws->data_ptr(), *stream = stream_of(*x);
    const float* sp = static_cast<const float*>(scales->data_ptr());
    const size_t wsb = static_cast<size_t>(ws->numel());
    int status = 0;
    Py_BEGIN_ALLOW_THREADS                      // the tensors are held by the caller's arguments
    status = fn(xp, xt, ldx, cp, sp, yp, yt, ldy, static_cast<int>(M), static_cast<int>(N), static_cast<int>(K), wsp, wsb, stream);
    Py_END_ALLOW_THREADS
    if (status != 0) return PyLong_FromLong(status);
    return given != nullptr ? Py_NewRef(a[5]) : THPVariable_Wrap(fresh);
    END_HANDLE_TH_ERRORS
}

// distill(address, 0 loss / 1 gradient / 2 both, logits, index, value, lse or None, temperature, saved or None, dloss or None, out or None)
//   -> (loss, saved), gradient, (loss, gradient), or the status of a call that failed, or None (see above)
PyObject* distill(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 10) { PyErr_SetString(PyExc_TypeError, "distill: 10 arguments"); return nullptr; }
    void* fn = PyLong_AsVoidPtr(a[0]);
    if (fn == nullptr) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "distill: no entry point"); return nullptr; }
    int mode = 0;
    long long ld = 0, ldg = 0;
    const at::Tensor* s = rows(a[2], &ld);
    if (!as_int(a[1], &mode) || s == nullptr || !PyFloat_CheckExact(a[6]) || !THPVariable_CheckExact(a[3]) || !THPVariable_CheckExact(a[4])) Py_RETURN_NONE;
    const int type = element_type(s->scalar_type());
    const at::Tensor &index = THPVariable_Unpack(a[3]), &value = THPVariable_Unpack(a[4]);
    const bool wide = index.scalar_type() == at::kLong;
    const int value_type = element_type(value.scalar_type());
    const long long M = s->size(0), V = s->size(1);
    const c10::DeviceIndex d = c10::cuda::current_device();
    if (type < 0 || value_type < 0 || (!wide && index.scalar_type() != at::kInt) || plain(a[3], index.scalar_type()) == nullptr ||
        plain(a[4], value.scalar_type()) == nullptr || index.dim() != 2 || value.dim() != 2 || index.size(0) != M || value.size(0) != M ||
        index.size(1) != value.size(1) || index.size(1) > INT_MAX || !here(*s, d) || !here(index, d) || !here(value, d))
        Py_RETURN_NONE;
    auto vector = [&](PyObject* o, long long count) -> const at::Tensor* {
        const at::Tensor* t = plain(o, at::kFloat);
        return t != nullptr && t->numel() == count && here(*t, d) ? t : nullptr;
    };
    const at::Tensor *lse = nullptr, *saved = nullptr, *dloss = nullptr, *given = nullptr;
    if (a[5] != Py_None && (lse = vector(a[5], M)) == nullptr) Py_RETURN_NONE;
    if (mode == 1 && (saved = vector(a[7], 4 * M)) == nullptr) Py_RETURN_NONE;
    if (mode != 0 && (dloss = vector(a[8], M)) == nullptr) Py_RETURN_NONE;
    if (mode != 0 && a[9] != Py_None &&
        ((given = rows(a[9], &ldg)) == nullptr || given->scalar_type() != s->scalar_type() || given->size(0) != M || given->size(1) != V || !here(*given, d)))
        Py_RETURN_NONE;
    at::Tensor loss, keep, grad;
    if (mode != 1) loss = at::empty({M}, s->options().dtype(at::kFloat));
    if (mode == 0) keep = at::empty({M, 4}, s->options().dtype(at::kFloat));
    if (mode != 0 && given == nullptr) { grad = at::empty({M, V}, s->options()); ldg = V; }
    auto floats = [](const at::Tensor* t) { return t != nullptr ? static_cast<float*>(t->data_ptr()) : nullptr; };
    const void *sp = s->data_ptr(), *ip = index.data_ptr(), *vp = value.data_ptr();
    const float *zp = floats(lse), *kp = floats(saved), *dp = floats(dloss);
    float *lp = loss.defined() ? floats(&loss) : nullptr, *op = keep.defined() ? floats(&keep) : nullptr;
    void *gp = mode == 0 ? nullptr : (given != nullptr ? *given : grad).data_ptr(), *stream = stream_of(*s);
    const double T = PyFloat_AS_DOUBLE(a[6]);
    const int m = static_cast<int>(M), v = static_cast<int>(V), k = static_cast<int>(index.size(1)), ib = wide ? 8 : 4;
    int status = 0;
    Py_BEGIN_ALLOW_THREADS
    if (mode == 0) status = reinterpret_cast<DistillLossFn>(fn)(sp, type, ld, ip, ib, vp, value_type, zp, T, m, v, k, lp, op, stream);
    else if (mode == 1) status = reinterpret_cast<DistillGradFn>(fn)(sp, type, ld, ip, ib, vp, value_type, zp, T, m, v, k, kp, dp, gp, ldg, stream);
    else status = reinterpret_cast<DistillStepFn>(fn)(sp, type, ld, ip, ib, vp, value_type, zp, T, m, v, k, dp, lp, gp, ldg, stream);
    Py_END_ALLOW_THREADS
    if (status != 0) return PyLong_FromLong(status);
    PyObject* g = mode == 0 ? THPVariable_Wrap(keep) : given != nullptr ? Py_NewRef(a[9]) : THPVariable_Wrap(grad);
    if (mode == 1 || g == nullptr) return g;
    PyObject* l = THPVariable_Wrap(loss);
    PyObject* both = l != nullptr ? PyTuple_New(2) : nullptr;
    if (both == nullptr) { Py_XDECREF(l); Py_DECREF(g); return nullptr; }
    PyTuple_SET_ITEM(both, 0, l);
    PyTuple_SET_ITEM(both, 1, g);
    return both;
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"fp8_linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fp8_linear)), METH_FASTCALL, nullptr},
    {"distill", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(distill)), METH_FASTCALL, nullptr},
    {"linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear)), METH_FASTCALL, nullptr},
    {"run_set", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(run_set)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "slim_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_slim_host(void) { return PyModule_Create(&module_def); }
