// The common calls of binding.py in native code: checks, output tensors and the library call without a Python object for
// each step.  Every function here takes what its namesake in binding.py takes, outputs as None where they are to be
// allocated, and returns
//   a tuple   the outputs, as the Python code returns them;
//   an int    the status of a call that the library refused;
//   None      where anything is out of the ordinary -- another type than a plain tensor, number or bool, a layout or
//             dtype that the Python code refuses or treats apart, a torch function or dispatch mode, an allocation that
//             failed: binding.py then takes its own way, and reports what it finds.
// An exception raised in Python code that runs inside (a Python allocator, say) is passed on as it is.
// The library's functions come in as addresses (bind), so there is one copy of it in the process.  The GIL is released
// around the library call, as ctypes does.
// Host time of a call, us, ctypes and torch.empty / so: fa_fwd 8.9 / 5.9, fa_bwd 12.1 / 7.6,
// fa_fp8_quant_hadamard 8.4 / 5.6, fa_fwd_fp8 9.2 / 6.1 (the launch itself is 2.4 to 3 of it); the calls on a cache check more:
// fa_rope 13.2 / 6.2, fa_cache_write 12.8 / 5.4, fa_cache_read 10.4 / 4.4, fa_fwd_cache in one launch 16.0 / 6.6.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/DeviceGuardImplInterface.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/fa_mi355.h"

namespace {

struct {
    decltype(&fa_fwd_gqa) fwd;
    decltype(&fa_fwd_fp8_gqa) fwd_fp8;
    decltype(&fa_fp8_quant_hadamard) quant;
    decltype(&fa_bwd_workspace_bytes) workspace_bytes;
    decltype(&fa_bwd_gqa) bwd;
    decltype(&fa_rope) rope, rope_bwd;
    decltype(&fa_cache_write) cache_write;
    decltype(&fa_cache_read) cache_read;
    decltype(&fa_fwd_cache_workspace_bytes) cache_workspace_bytes;
    decltype(&fa_fwd_cache) fwd_cache;
} lib;

// The arguments of a call; `ok` turns false at the first that is not as the native way takes it.
struct Arguments {
    PyObject* const* args;
    Py_ssize_t n;
    bool ok = true;

    Arguments(PyObject* const* a, Py_ssize_t count, Py_ssize_t expected) : args(a), n(count), ok(count == expected) {
        if (lib.fwd == nullptr || at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set())
            ok = false;
    }
    bool given(Py_ssize_t i) const { return ok && args[i] != Py_None; }
    // a plain contiguous device tensor
    const at::Tensor* tensor(Py_ssize_t i) {
        if (!ok || !THPVariable_CheckExact(args[i])) return fail();
        const at::Tensor& t = THPVariable_Unpack(args[i]);
        if (!t.defined() || !t.is_cuda() || !t.is_contiguous()) return fail();
        return &t;
    }
    double number(Py_ssize_t i) {
        if (ok && PyFloat_CheckExact(args[i])) return PyFloat_AS_DOUBLE(args[i]);
        ok = false;
        return 0.0;
    }
    int flag(Py_ssize_t i) {
        if (ok && PyLong_Check(args[i])) return PyObject_IsTrue(args[i]);  // a bool or an int
        ok = false;
        return 0;
    }
    // What the function args[i] says is the current stream, asked when everything else is in order.  Its failure is a case for
    // the Python code, which asks again; what is no Exception (an interrupt from the keyboard comes only once) stays set.
    void* stream(Py_ssize_t i) {
        if (!ok) return nullptr;
        PyObject* handle = PyObject_CallNoArgs(args[i]);
        void* p = handle ? PyLong_AsVoidPtr(handle) : nullptr;
        Py_XDECREF(handle);
        if (PyErr_Occurred()) {
            if (PyErr_ExceptionMatches(PyExc_Exception)) PyErr_Clear();
            ok = false;
        }
        return p;
    }

private:
    std::nullptr_t fail() {
        ok = false;
        return nullptr;
    }
};

struct Shape {
    int B, H, N, d;
};
// [B, H, N, d] of a 4-dimensional tensor
bool shape_of(const at::Tensor& t, Shape& s) {
    if (t.dim() != 4) return false;
    const auto sizes = t.sizes();
    for (int64_t x : sizes)
        if (x > 0x7fffffff) return false;
    s = {(int)sizes[0], (int)sizes[1], (int)sizes[2], (int)sizes[3]};
    return true;
}
bool dtype_code(const at::Tensor& t, int& code) {
    switch (t.scalar_type()) {
        case at::kFloat: code = FA_F32; return true;
        case at::kBFloat16: code = FA_BF16; return true;
        case at::kHalf: code = FA_F16; return true;
        default: return false;
    }
}

// The given output tensor, or a new one of these sizes on the device of `like`
at::Tensor output(Arguments& a, Py_ssize_t i, at::IntArrayRef sizes, const at::Tensor& like, at::ScalarType type) {
    if (a.given(i)) {
        const at::Tensor* t = a.tensor(i);
        return t ? *t : at::Tensor();
    }
    return a.ok ? at::empty(sizes, like.options().dtype(type)) : at::Tensor();
}
// ... with the strides of `like`
at::Tensor gradient(Arguments& a, Py_ssize_t i, const at::Tensor& like) {
    if (a.given(i)) {
        const at::Tensor* t = a.tensor(i);
        return t ? *t : at::Tensor();
    }
    return a.ok ? at::empty_strided(like.sizes(), like.strides(), like.options()) : at::Tensor();
}

template <typename Call>
int without_gil(Call&& call) {
    PyThreadState* state = PyEval_SaveThread();
    const int status = call();
    PyEval_RestoreThread(state);
    return status;
}

// A tuple of the tensors, given ones as the objects they came as, or the status
template <size_t K>
PyObject* result(int status, const Arguments& a, const Py_ssize_t (&index)[K], const at::Tensor (&tensors)[K]) {
    if (status != FA_OK) return PyLong_FromLong(status);
    PyObject* out = PyTuple_New(K);
    if (!out) return nullptr;
    for (size_t i = 0; i < K; ++i) {
        PyObject* t = a.given(index[i]) ? Py_NewRef(a.args[index[i]]) : THPVariable_Wrap(tensors[i]);
        if (!t) {
            Py_DECREF(out);
            return nullptr;
        }
        PyTuple_SET_ITEM(out, i, t);
    }
    return out;
}

// Runs `body`; an exception is a case for the Python code, but for one that Python has set already
template <typename Body>
PyObject* native(Body&& body) {
    try {
        PyObject* r = body();
        if (r) return r;
    } catch (...) {
    }
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

// (q, k, v, scale, causal, o, lse, shared, stream)
PyObject* fwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return native([&]() -> PyObject* {
        Arguments a(args, n, 9);
        const at::Tensor *q = a.tensor(0), *k = a.tensor(1), *v = a.tensor(2);
        const double scale = a.number(3);
        const int causal = a.flag(4), shared = a.flag(7);
        void* stream = a.stream(8);
        Shape s;
        int code;
        if (!a.ok || !shape_of(*q, s) || !dtype_code(*q, code) || (shared && k->dim() < 2)) return nullptr;
        const int64_t kv_heads = shared ? k->size(1) : s.H;
        if (kv_heads > 0x7fffffff) return nullptr;
        const at::Tensor o = output(a, 5, q->sizes(), *q, q->scalar_type());
        const at::Tensor lse = output(a, 6, {s.B, s.H, s.N}, *q, at::kFloat);
        if (!a.ok) return nullptr;
        const void *qp = q->data_ptr(), *kp = k->data_ptr(), *vp = v->data_ptr();
        void* op = o.data_ptr();
        float* lp = static_cast<float*>(lse.data_ptr());
        const int st = without_gil([&] {
            return lib.fwd(qp, kp, vp, op, lp, s.B, s.H, (int)kv_heads, s.N, s.d, (float)scale, causal, code, stream);
        });
        return result(st, a, {5, 6}, {o, lse});
    });
}

// (q8, k8, v8, q_scale, k_scale, v_scale, scale, causal, o, lse, shared, stream), blocks of 128 rows
PyObject* fwd_fp8(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return native([&]() -> PyObject* {
        Arguments a(args, n, 12);
        const at::Tensor *q = a.tensor(0), *k = a.tensor(1), *v = a.tensor(2);
        const at::Tensor *qs = a.tensor(3), *ks = a.tensor(4), *vs = a.tensor(5);
        const double scale = a.number(6);
        const int causal = a.flag(7), shared = a.flag(10);
        void* stream = a.stream(11);
        Shape s;
        if (!a.ok || !shape_of(*q, s) || (shared && k->dim() < 2)) return nullptr;
        const int64_t kv_heads = shared ? k->size(1) : s.H;
        if (kv_heads > 0x7fffffff) return nullptr;
        const at::Tensor o = output(a, 8, q->sizes(), *q, at::kBFloat16);
        const at::Tensor lse = output(a, 9, {s.B, s.H, s.N}, *q, at::kFloat);
        if (!a.ok) return nullptr;
        const void *qp = q->data_ptr(), *kp = k->data_ptr(), *vp = v->data_ptr();
        const float *qsp = static_cast<const float*>(qs->data_ptr()), *ksp = static_cast<const float*>(ks->data_ptr()),
                    *vsp = static_cast<const float*>(vs->data_ptr());
        void* op = o.data_ptr();
        float* lp = static_cast<float*>(lse.data_ptr());
        const int st = without_gil([&] {
            return lib.fwd_fp8(qp, kp, vp, qsp, ksp, vsp, op, lp, s.B, s.H, (int)kv_heads, s.N, s.d, 128, (float)scale, causal,
                               stream);
        });
        return result(st, a, {8, 9}, {o, lse});
    });
}

// (x, signs, per_tensor, x8, scales, stream), blocks of 128 rows
PyObject* quant(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return native([&]() -> PyObject* {
        Arguments a(args, n, 6);
        const at::Tensor* x = a.tensor(0);
        const at::Tensor* signs = a.given(1) ? a.tensor(1) : nullptr;
        const int per_tensor = a.flag(2);
        void* stream = a.stream(5);
        Shape s;
        int code;
        if (!a.ok || !shape_of(*x, s) || !dtype_code(*x, code)) return nullptr;
        const at::Tensor x8 = output(a, 3, x->sizes(), *x, at::kByte);
        const at::Tensor scales = output(a, 4, {s.B, s.H, (s.N + 127L) / 128}, *x, at::kFloat);
        if (!a.ok) return nullptr;
        const void* xp = x->data_ptr();
        const signed char* sp = signs ? static_cast<const signed char*>(signs->data_ptr()) : nullptr;
        void* cp = x8.data_ptr();
        float* scp = static_cast<float*>(scales.data_ptr());
        const int st =
            without_gil([&] { return lib.quant(xp, code, cp, scp, s.B, s.H, s.N, s.d, 128, sp, per_tensor, stream); });
        return result(st, a, {3, 4}, {x8, scales});
    });
}

// (q, k, v, o, lse, dout, scale, causal, dq, dk, dv, workspace, shared, stream)
PyObject* bwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return native([&]() -> PyObject* {
        Arguments a(args, n, 14);
        const at::Tensor *q = a.tensor(0), *k = a.tensor(1), *v = a.tensor(2), *o = a.tensor(3), *lse = a.tensor(4);
        const at::Tensor* dout = a.tensor(5);
        const double scale = a.number(6);
        const int causal = a.flag(7), shared = a.flag(12);
        void* stream = a.stream(13);
        Shape s;
        int code;
        if (!a.ok || !shape_of(*q, s) || !dtype_code(*q, code) || (shared && k->dim() < 2)) return nullptr;
        const int64_t kv_heads = shared ? k->size(1) : s.H;
        if (kv_heads > 0x7fffffff) return nullptr;
        at::Tensor workspace;
        if (a.given(11)) {
            const at::Tensor* t = a.tensor(11);
            if (!t) return nullptr;
            workspace = *t;
        } else {
            const int64_t need = (int64_t)lib.workspace_bytes(s.B, s.H, s.N, s.d, code);
            workspace = at::empty({need > 16 ? need : 16}, q->options().dtype(at::kByte));
        }
        const at::Tensor dq = gradient(a, 8, *q), dk = gradient(a, 9, *k), dv = gradient(a, 10, *v);
        if (!a.ok) return nullptr;
        const void *qp = q->data_ptr(), *kp = k->data_ptr(), *vp = v->data_ptr(), *op = o->data_ptr(), *dop = dout->data_ptr();
        const float* lp = static_cast<const float*>(lse->data_ptr());
        void *dqp = dq.data_ptr(), *dkp = dk.data_ptr(), *dvp = dv.data_ptr(), *wp = workspace.data_ptr();
        const size_t bytes = (size_t)workspace.numel();
        const int st = without_gil([&] {
            return lib.bwd(qp, kp, vp, op, lp, dop, dqp, dkp, dvp, wp, bytes, s.B, s.H, (int)kv_heads, s.N, s.d, (float)scale, causal,
                           code, stream);
        });
        return result(st, a, {8, 9, 10}, {dq, dk, dv});
    });
}

// ---- Rotary positions, the cache and attention over it.  These calls also see to shapes, types and the current device, as their
// Python code does; where one is not as it should be, that says so.

int current_device() { return c10::impl::getDeviceGuardImpl(c10::DeviceType::CUDA)->getDevice().index(); }

// A tensor on the device `device`, of these sizes and this type, contiguous, or with contiguous rows where `strides` can say how:
// then *strides points to three numbers in `room`, otherwise to nothing.
struct Strides {
    long long room[3];
    const long long* p = nullptr;
};
const at::Tensor* fitting(Arguments& a, Py_ssize_t i, int device, at::IntArrayRef sizes, at::ScalarType type, Strides* strides = nullptr) {
    if (!a.ok) return nullptr;
    a.ok = false;
    if (!THPVariable_CheckExact(a.args[i])) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(a.args[i]);
    if (!t.defined() || !t.is_cuda() || t.device().index() != device || t.scalar_type() != type || t.sizes() != sizes) return nullptr;
    if (!t.is_contiguous()) {
        if (!strides || t.dim() != 4 || t.stride(3) != 1) return nullptr;
        for (int k = 0; k < 3; ++k) strides->room[k] = t.stride(k);
        strides->p = strides->room;
    }
    a.ok = true;
    return &t;
}
// A plain 4-dimensional device tensor (its shape says what the others have to be)
const at::Tensor* four(Arguments& a, Py_ssize_t i, Shape& s) {
    if (!a.ok || !THPVariable_CheckExact(a.args[i])) {
        a.ok = false;
        return nullptr;
    }
    const at::Tensor& t = THPVariable_Unpack(a.args[i]);
    a.ok = t.defined() && t.is_cuda() && shape_of(t, s);
    return a.ok ? &t : nullptr;
}
// The given output, or a new contiguous one
at::Tensor fitting_output(Arguments& a, Py_ssize_t i, int device, at::IntArrayRef sizes, at::ScalarType type, const at::Tensor& like,
                          Strides* strides = nullptr) {
    if (a.given(i)) {
        const at::Tensor* t = fitting(a, i, device, sizes, type, strides);
        return t ? *t : at::Tensor();
    }
    return a.ok ? at::empty(sizes, like.options().dtype(type).memory_format(at::MemoryFormat::Contiguous)) : at::Tensor();
}
template <typename T = void>
T* pointer(const at::Tensor* t) {
    return t ? static_cast<T*>(t->data_ptr()) : nullptr;
}

// (backward, q, inv_freq, k, positions, rot_dim, interleaved, amplitude, q_out, k_out, stream)
PyObject* rope(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return native([&]() -> PyObject* {
        Arguments a(args, n, 11);
        const int backward = a.flag(0), interleaved = a.flag(6);
        const double amplitude = a.number(7);
        Shape s, sk = {};
        int code;
        const at::Tensor* q = four(a, 1, s);
        if (!a.ok || !dtype_code(*q, code)) return nullptr;
        const int device = current_device();
        const at::ScalarType type = q->scalar_type();
        long rot_dim = s.d;
        if (a.given(5)) {
            if (!PyLong_CheckExact(args[5])) return nullptr;
            rot_dim = PyLong_AsLong(args[5]);
            if (rot_dim < 0 || rot_dim > 0x7fffffff) return nullptr;  // (and an overflow's -1)
        }
        Strides qs, ks, qos, kos;
        fitting(a, 1, device, q->sizes(), type, &qs);
        const at::Tensor* f = fitting(a, 2, device, {rot_dim / 2}, at::kDouble);
        const at::Tensor* k = a.given(3) ? four(a, 3, sk) : nullptr;
        if (k) fitting(a, 3, device, {s.B, sk.H, s.N, s.d}, type, &ks);
        const at::Tensor* positions = a.given(4) ? fitting(a, 4, device, {s.B, s.N}, at::kInt) : nullptr;
        if (!a.ok || (!k && args[9] != Py_None)) return nullptr;
        void* stream = a.stream(10);
        const at::Tensor q_out = fitting_output(a, 8, device, q->sizes(), type, *q, &qos);
        const at::Tensor k_out = k ? fitting_output(a, 9, device, k->sizes(), type, *k, &kos) : at::Tensor();
        if (!a.ok) return nullptr;
        const void *qp = q->data_ptr(), *kp = pointer(k);
        void *qop = q_out.data_ptr(), *kop = k ? k_out.data_ptr() : nullptr;
        const double* fp = pointer<double>(f);
        const int* pp = pointer<int>(positions);
        const auto call = backward ? lib.rope_bwd : lib.rope;
        const int st = without_gil([&] {
            return call(qp, qs.p, kp, ks.p, qop, qos.p, kop, kos.p, fp, pp, s.B, s.H, sk.H, s.N, s.d, (int)rot_dim, (float)amplitude,
                        interleaved, code, stream);
        });
        return result(st, a, {8, 9}, {q_out, k_out});  // (an undefined tensor becomes None)
    });
}

// The tensors of a cache, from argument `at` on: k_pages, v_pages, block_table, lens; scales and counts where they stand
struct CacheArguments {
    const at::Tensor *k, *v, *table, *lens, *k_scales, *v_scales, *counts;
    Shape s;  // n_pages, H_kv, page_size, d
    int code, max_pages;
};
bool cache_arguments(Arguments& a, CacheArguments& c, int device, Py_ssize_t at, int B, Py_ssize_t k_scales, Py_ssize_t v_scales, Py_ssize_t counts) {
    c.k = four(a, at, c.s);
    if (!a.ok) return false;
    const at::ScalarType type = c.k->scalar_type();
    switch (type) {
        case at::kBFloat16: c.code = FA_BF16; break;
        case at::kHalf: c.code = FA_F16; break;
        case at::kByte:
        case at::kFloat8_e4m3fn: c.code = FA_FP8_E4M3; break;
        default: return a.ok = false;
    }
    fitting(a, at, device, c.k->sizes(), type);
    c.v = fitting(a, at + 1, device, c.k->sizes(), type);
    if (!a.ok || !THPVariable_CheckExact(a.args[at + 2]) || THPVariable_Unpack(a.args[at + 2]).dim() != 2) return a.ok = false;
    const int64_t wide = THPVariable_Unpack(a.args[at + 2]).size(1);
    if (wide > 0x7fffffff) return a.ok = false;
    c.max_pages = (int)wide;
    c.table = fitting(a, at + 2, device, {B, wide}, at::kInt);
    c.lens = fitting(a, at + 3, device, {B}, at::kInt);
    c.k_scales = c.v_scales = c.counts = nullptr;
    if (a.given(k_scales) != (c.code == FA_FP8_E4M3) || a.given(v_scales) != (c.code == FA_FP8_E4M3)) return a.ok = false;
    if (c.code == FA_FP8_E4M3) {
        c.k_scales = fitting(a, k_scales, device, {c.s.B, c.s.H, c.s.N}, at::kFloat);
        c.v_scales = fitting(a, v_scales, device, {c.s.B, c.s.H, c.s.N}, at::kFloat);
    }
    if (counts >= 0 && a.given(counts)) c.counts = fitting(a, counts, device, {B}, at::kInt);
    return a.ok;
}

// (k, v, k_pages, v_pages, block_table, lens, counts, k_scales, v_scales, stream)
PyObject* cache_write(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return native([&]() -> PyObject* {
        Arguments a(args, n, 10);
        Shape s;
        int code;
        const at::Tensor* k = four(a, 0, s);
        if (!a.ok || !dtype_code(*k, code)) return nullptr;
        const int device = current_device();
        Strides ks, vs;
        CacheArguments c;
        fitting(a, 0, device, k->sizes(), k->scalar_type(), &ks);
        const at::Tensor* v = fitting(a, 1, device, k->sizes(), k->scalar_type(), &vs);
        if (!a.ok || !cache_arguments(a, c, device, 2, s.B, 7, 8, 6) || c.s.H != s.H || c.s.d != s.d) return nullptr;
        void* stream = a.stream(9);
        if (!a.ok) return nullptr;
        const void *kp = k->data_ptr(), *vp = v->data_ptr();
        void *kpp = c.k->data_ptr(), *vpp = c.v->data_ptr();
        float *ksp = pointer<float>(c.k_scales), *vsp = pointer<float>(c.v_scales);
        const int *tp = pointer<int>(c.table), *lp = pointer<int>(c.lens), *cp = pointer<int>(c.counts);
        const int st = without_gil([&] {
            return lib.cache_write(kp, ks.p, vp, vs.p, kpp, vpp, ksp, vsp, tp, lp, cp, s.B, s.H, s.N, s.d, c.s.N, c.s.B, c.max_pages, code,
                                   c.code, stream);
        });
        return result(st, a, {2, 3}, {*c.k, *c.v});
    });
}

// (k_pages, v_pages, block_table, lens, N, dtype, k_scales, v_scales, k, v, stream)
PyObject* cache_read(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return native([&]() -> PyObject* {
        Arguments a(args, n, 11);
        if (!a.ok || !THPVariable_CheckExact(args[2]) || THPVariable_Unpack(args[2]).dim() != 2) return nullptr;
        const int64_t B = THPVariable_Unpack(args[2]).size(0);
        if (B > 0x7fffffff) return nullptr;
        const int device = current_device();
        CacheArguments c;
        if (!cache_arguments(a, c, device, 0, (int)B, 6, 7, -1)) return nullptr;
        const Py_ssize_t given = a.given(8) ? 8 : 9;
        Shape s = {(int)B, c.s.H, 0, c.s.d};
        at::ScalarType type = c.code == FA_FP8_E4M3 ? at::kBFloat16 : c.k->scalar_type();
        if (a.given(given)) {
            const at::Tensor* t = four(a, given, s);
            if (!a.ok) return nullptr;
            type = t->scalar_type();
        }
        if (a.given(5)) {
            if (!THPDtype_Check(args[5])) return nullptr;
            type = reinterpret_cast<THPDtype*>(args[5])->scalar_type;
        }
        long N = s.N;
        if (a.given(4)) {
            if (!PyLong_CheckExact(args[4])) return nullptr;
            N = PyLong_AsLong(args[4]);
        } else if (!a.given(given)) {
            return nullptr;
        }
        int code;
        if (N < 0 || N > 0x7fffffff) return nullptr;
        switch (type) {
            case at::kFloat: code = FA_F32; break;
            case at::kBFloat16: code = FA_BF16; break;
            case at::kHalf: code = FA_F16; break;
            default: return nullptr;
        }
        void* stream = a.stream(10);
        const at::Tensor k = fitting_output(a, 8, device, {B, c.s.H, N, c.s.d}, type, *c.k);
        const at::Tensor v = fitting_output(a, 9, device, {B, c.s.H, N, c.s.d}, type, *c.k);
        if (!a.ok) return nullptr;
        const void *kpp = c.k->data_ptr(), *vpp = c.v->data_ptr();
        const float *ksp = pointer<float>(c.k_scales), *vsp = pointer<float>(c.v_scales);
        const int *tp = pointer<int>(c.table), *lp = pointer<int>(c.lens);
        void *kp = k.data_ptr(), *vp = v.data_ptr();
        const int st = without_gil([&] {
            return lib.cache_read(kpp, vpp, ksp, vsp, tp, lp, kp, vp, (int)B, c.s.H, (int)N, c.s.d, c.s.N, c.s.B, c.max_pages, c.code, code, stream);
        });
        return result(st, a, {8, 9}, {k, v});
    });
}

// (q, k_pages, v_pages, block_table, lens, scale, tree, counts, k_scales, v_scales, max_len, o, lse, workspace, stream)
PyObject* fwd_cache(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return native([&]() -> PyObject* {
        Arguments a(args, n, 15);
        const double scale = a.number(5);
        Shape s;
        int code;
        const at::Tensor* q = four(a, 0, s);
        if (!a.ok || !dtype_code(*q, code) || code == FA_F32 || !PyLong_CheckExact(args[10])) return nullptr;
        const long max_len = PyLong_AsLong(args[10]);
        if (max_len < 0 || max_len > 0x7fffffff) return nullptr;
        const int device = current_device();
        Strides qs, os;
        CacheArguments c;
        fitting(a, 0, device, q->sizes(), q->scalar_type(), &qs);
        if (!a.ok || !cache_arguments(a, c, device, 1, s.B, 8, 9, 7) || c.s.d != s.d) return nullptr;
        const at::Tensor* tree = nullptr;
        int batches = 0;
        if (a.given(6)) {
            if (!THPVariable_CheckExact(args[6])) return nullptr;
            const at::Tensor& t = THPVariable_Unpack(args[6]);
            batches = t.dim() == 3 && t.size(0) == s.B ? s.B : 1;
            tree = fitting(a, 6, device, {batches, s.N, (s.N + 31L) / 32}, at::kInt);
        }
        void* stream = a.stream(14);
        const at::Tensor o = fitting_output(a, 11, device, q->sizes(), q->scalar_type(), *q, &os);
        const at::Tensor lse = fitting_output(a, 12, device, {s.B, s.H, s.N}, at::kFloat, *q);
        if (!a.ok) return nullptr;
        const long places = max_len ? max_len : (long)c.max_pages * c.s.N;
        const int64_t need = places > 0x7fffffff ? 0 : (int64_t)lib.cache_workspace_bytes(s.B, s.H, c.s.H, s.N, s.d, (int)places, c.code);
        at::Tensor workspace;
        if (a.given(13)) {
            const at::Tensor* t = a.tensor(13);
            if (!t || t->device().index() != device || t->scalar_type() != at::kByte || t->dim() != 1) return nullptr;
            workspace = *t;
        } else if (need > 0) {
            workspace = at::empty({need}, q->options().dtype(at::kByte));
        }
        const void *qp = q->data_ptr(), *kpp = c.k->data_ptr(), *vpp = c.v->data_ptr();
        const float *ksp = pointer<float>(c.k_scales), *vsp = pointer<float>(c.v_scales);
        const int *tp = pointer<int>(c.table), *lp = pointer<int>(c.lens), *cp = pointer<int>(c.counts), *wp = pointer<int>(tree);
        void *op = o.data_ptr(), *space = workspace.defined() ? workspace.data_ptr() : nullptr;
        float* lsep = static_cast<float*>(lse.data_ptr());
        const size_t bytes = workspace.defined() ? (size_t)workspace.numel() : 0;
        const int st = without_gil([&] {
            return lib.fwd_cache(qp, qs.p, kpp, vpp, ksp, vsp, tp, lp, cp, wp, batches, op, os.p, lsep, space, bytes, s.B, s.H, c.s.H, s.N, s.d,
                                 c.s.N, c.s.B, c.max_pages, (int)max_len, (float)scale, code, c.code, stream);
        });
        return result(st, a, {11, 12}, {o, lse});
    });
}

// bind(address of fa_fwd_gqa, fa_fwd_fp8_gqa, fa_fp8_quant_hadamard, fa_bwd_workspace_bytes, fa_bwd_gqa, fa_rope, fa_rope_bwd, fa_cache_write,
// fa_cache_read, fa_fwd_cache_workspace_bytes, fa_fwd_cache)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
    constexpr int kAddresses = 11;
    void* p[kAddresses];
    if (n != kAddresses) {
        PyErr_SetString(PyExc_TypeError, "bind takes eleven addresses");
        return nullptr;
    }
    for (int i = 0; i < kAddresses; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    lib.fwd = reinterpret_cast<decltype(lib.fwd)>(p[0]);
    lib.fwd_fp8 = reinterpret_cast<decltype(lib.fwd_fp8)>(p[1]);
    lib.quant = reinterpret_cast<decltype(lib.quant)>(p[2]);
    lib.workspace_bytes = reinterpret_cast<decltype(lib.workspace_bytes)>(p[3]);
    lib.bwd = reinterpret_cast<decltype(lib.bwd)>(p[4]);
    lib.rope = reinterpret_cast<decltype(lib.rope)>(p[5]);
    lib.rope_bwd = reinterpret_cast<decltype(lib.rope_bwd)>(p[6]);
    lib.cache_write = reinterpret_cast<decltype(lib.cache_write)>(p[7]);
    lib.cache_read = reinterpret_cast<decltype(lib.cache_read)>(p[8]);
    lib.cache_workspace_bytes = reinterpret_cast<decltype(lib.cache_workspace_bytes)>(p[9]);
    lib.fwd_cache = reinterpret_cast<decltype(lib.fwd_cache)>(p[10]);
    Py_RETURN_NONE;
}

#define FA_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FA_METHOD(bind), FA_METHOD(fwd), FA_METHOD(fwd_fp8), FA_METHOD(quant), FA_METHOD(bwd), FA_METHOD(rope), FA_METHOD(cache_write),
                         FA_METHOD(cache_read), FA_METHOD(fwd_cache), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fa_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

// Whether the torch of this process is the one that this file was compiled against; if not, ImportError is set
bool same_torch() {
    PyObject* torch = PyImport_ImportModule("torch");
    PyObject* version = torch ? PyObject_GetAttrString(torch, "__version__") : nullptr;
    PyObject* text = version ? PyObject_Str(version) : nullptr;
    const bool same = text && PyUnicode_CompareWithASCIIString(text, FA_TORCH_VERSION) == 0;
    if (text && !same) PyErr_Format(PyExc_ImportError, "built for torch " FA_TORCH_VERSION ", not for %U", text);
    Py_XDECREF(text);
    Py_XDECREF(version);
    Py_XDECREF(torch);
    return same;
}

}  // namespace

PyMODINIT_FUNC PyInit__fa_binding() { return same_torch() ? PyModule_Create(&module) : nullptr; }
