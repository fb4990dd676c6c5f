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
// fa_rope 13.2 / 6.2, fa_cache_write 12.8 / 5.4, fa_cache_read 10.4 / 4.4, fa_fwd_cache in one launch 16.0 / 6.6,
// fa_rope_axes 13.5 / 5.5, fa_cache_fork 16.6 / 5.8, fa_cache_extend 9.0 / 5.0, fa_cache_compact 14.4 / 5.8, fa_cache_copy 8.4 / 3.9.
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
    decltype(&fa_rope_axes) rope_axes, rope_axes_bwd;
    decltype(&fa_cache_pages_workspace_bytes) pages_workspace_bytes;
    decltype(&fa_cache_fork) cache_fork;
    decltype(&fa_cache_extend) cache_extend;
    decltype(&fa_cache_compact) cache_compact;
    decltype(&fa_cache_copy) cache_copy;
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

// (backward, q, inv_freq, k, positions, rot_dim, interleaved, amplitude, q_out, k_out, stream); with several axes, their numbers too
template <bool AXES>
PyObject* rope_any(PyObject* const* args, Py_ssize_t n) {
    return native([&]() -> PyObject* {
        Arguments a(args, n, AXES ? 12 : 11);
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
        const at::Tensor *positions = nullptr, *axis = nullptr;
        int axes = 0;
        if constexpr (AXES) {
            if (!a.ok || !THPVariable_CheckExact(args[4])) return nullptr;
            const at::Tensor& t = THPVariable_Unpack(args[4]);
            if (!t.defined() || t.dim() != 3 || t.size(0) > 0x7fffffff) return nullptr;
            axes = (int)t.size(0);
            positions = fitting(a, 4, device, {axes, s.B, s.N}, at::kInt);
            axis = fitting(a, 11, device, {rot_dim / 2}, at::kInt);
        } else if (a.given(4)) {
            positions = fitting(a, 4, device, {s.B, s.N}, at::kInt);
        }
        if (!a.ok || (!k && args[9] != Py_None)) return nullptr;
        void* stream = a.stream(10);
        const at::Tensor q_out = fitting_output(a, 8, device, q->sizes(), type, *q, &qos);
        const at::Tensor k_out = k ? fitting_output(a, 9, device, k->sizes(), type, *k, &kos) : at::Tensor();
        if (!a.ok) return nullptr;
        const void *qp = q->data_ptr(), *kp = pointer(k);
        void *qop = q_out.data_ptr(), *kop = k ? k_out.data_ptr() : nullptr;
        const double* fp = pointer<double>(f);
        const int *pp = pointer<int>(positions), *ap = pointer<int>(axis);
        const int st = without_gil([&] {
            if constexpr (AXES) {
                const auto call = backward ? lib.rope_axes_bwd : lib.rope_axes;
                return call(qp, qs.p, kp, ks.p, qop, qos.p, kop, kos.p, fp, ap, pp, axes, s.B, s.H, sk.H, s.N, s.d, (int)rot_dim, (float)amplitude,
                            interleaved, code, stream);
            }
            const auto call = backward ? lib.rope_bwd : lib.rope;
            return call(qp, qs.p, kp, ks.p, qop, qos.p, kop, kos.p, fp, pp, s.B, s.H, sk.H, s.N, s.d, (int)rot_dim, (float)amplitude,
                        interleaved, code, stream);
        });
        return result(st, a, {8, 9}, {q_out, k_out});  // (an undefined tensor becomes None)
    });
}

PyObject* rope(PyObject*, PyObject* const* args, Py_ssize_t n) { return rope_any<false>(args, n); }
PyObject* rope_axes(PyObject*, PyObject* const* args, Py_ssize_t n) { return rope_any<true>(args, n); }

// Pages and scales from argument `at`, `k_scales` and `v_scales` on: whether they belong together, what they hold, and of 4-bit ones
// the whole d
struct PagesArguments {
    const at::Tensor *k, *v, *k_scales, *v_scales;
    Shape s;  // n_pages, H_kv, page_size, d
    int code;
};
bool pages_arguments(Arguments& a, PagesArguments& c, int device, Py_ssize_t at, Py_ssize_t k_scales, Py_ssize_t v_scales) {
    auto of_powers = [&](Py_ssize_t i, at::ScalarType& type) {
        if (!a.given(i) || !THPVariable_CheckExact(a.args[i])) return false;
        type = THPVariable_Unpack(a.args[i]).scalar_type();
        return type == at::kByte || type == at::kFloat8_e8m0fnu;
    };
    c.k = four(a, at, c.s);
    if (!a.ok) return false;
    const at::ScalarType type = c.k->scalar_type();
    at::ScalarType powers;
    switch (type) {
        case at::kBFloat16: c.code = FA_BF16; break;
        case at::kHalf: c.code = FA_F16; break;
        case at::kByte: c.code = of_powers(k_scales, powers) ? FA_FP4_E2M1 : FA_FP8_E4M3; break;
        case at::kFloat4_e2m1fn_x2: c.code = FA_FP4_E2M1; break;
        case at::kFloat8_e4m3fn: c.code = FA_FP8_E4M3; break;
        default: return a.ok = false;
    }
    fitting(a, at, device, c.k->sizes(), type);
    c.v = fitting(a, at + 1, device, c.k->sizes(), type);
    if (!a.ok) return false;
    c.k_scales = c.v_scales = nullptr;
    const bool scaled = c.code == FA_FP8_E4M3 || c.code == FA_FP4_E2M1;
    if (a.given(k_scales) != scaled || a.given(v_scales) != scaled) return a.ok = false;
    if (c.code == FA_FP8_E4M3) {
        c.k_scales = fitting(a, k_scales, device, {c.s.B, c.s.H, c.s.N}, at::kFloat);
        c.v_scales = fitting(a, v_scales, device, {c.s.B, c.s.H, c.s.N}, at::kFloat);
    }
    if (c.code == FA_FP4_E2M1) {
        if (c.s.d > 0x3fffffff) return a.ok = false;
        c.s.d *= 2;
        if (!of_powers(k_scales, powers)) return a.ok = false;
        c.k_scales = fitting(a, k_scales, device, {c.s.B, c.s.H, c.s.N, c.s.d / 32}, powers);
        if (!of_powers(v_scales, powers)) return a.ok = false;
        c.v_scales = fitting(a, v_scales, device, {c.s.B, c.s.H, c.s.N, c.s.d / 32}, powers);
    }
    return a.ok;
}

// The tensors of a cache, from argument `at` on: k_pages, v_pages, block_table, lens; scales and counts where they stand
struct CacheArguments : PagesArguments {
    const at::Tensor *table, *lens, *counts;
    int max_pages;
};
bool cache_arguments(Arguments& a, CacheArguments& c, int device, Py_ssize_t at, int B, Py_ssize_t k_scales, Py_ssize_t v_scales, Py_ssize_t counts) {
    if (!pages_arguments(a, c, device, at, k_scales, v_scales) || !THPVariable_CheckExact(a.args[at + 2]) || THPVariable_Unpack(a.args[at + 2]).dim() != 2) return a.ok = false;
    const int64_t wide = THPVariable_Unpack(a.args[at + 2]).size(1);
    if (wide > 0x7fffffff) return a.ok = false;
    c.max_pages = (int)wide;
    c.table = fitting(a, at + 2, device, {B, wide}, at::kInt);
    c.lens = fitting(a, at + 3, device, {B}, at::kInt);
    c.counts = nullptr;
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
        void *ksp = pointer(c.k_scales), *vsp = pointer(c.v_scales);
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
        at::ScalarType type = c.code == FA_FP8_E4M3 || c.code == FA_FP4_E2M1 ? at::kBFloat16 : c.k->scalar_type();
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
        const void *ksp = pointer(c.k_scales), *vsp = pointer(c.v_scales);
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
        const void *ksp = pointer(c.k_scales), *vsp = pointer(c.v_scales);
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

// ---- Pages of a pool

// Argument i as a whole number of int's range
int whole(Arguments& a, Py_ssize_t i) {
    if (!a.ok || !PyLong_CheckExact(a.args[i])) return a.ok = false;
    const long x = PyLong_AsLong(a.args[i]);
    if (x < 0 || x > 0x7fffffff) a.ok = false;  // (and an overflow's -1; Python's ints go through the Python way)
    return (int)x;
}
// [B, max_pages]
const at::Tensor* table_of(Arguments& a, Py_ssize_t i, int device, int& B, int& max_pages) {
    if (!a.ok || !THPVariable_CheckExact(a.args[i])) {
        a.ok = false;
        return nullptr;
    }
    const at::Tensor& t = THPVariable_Unpack(a.args[i]);
    if (!t.defined() || t.dim() != 2 || t.size(0) > 0x7fffffff || t.size(1) > 0x7fffffff) {
        a.ok = false;
        return nullptr;
    }
    B = (int)t.size(0);
    max_pages = (int)t.size(1);
    return fitting(a, i, device, {B, max_pages}, at::kInt);
}
const at::Tensor* ints_or_none(Arguments& a, Py_ssize_t i, int device, int64_t size) { return a.given(i) ? fitting(a, i, device, {size}, at::kInt) : nullptr; }
// The given tensors of ints, and new ones of these sizes for those that are not, in one allocation
template <size_t K>
void together(Arguments& a, const Py_ssize_t (&index)[K], int device, const int64_t (&sizes)[K], const at::Tensor& like, at::Tensor (&out)[K]) {
    int64_t total = 0, at = 0;
    for (size_t i = 0; i < K; ++i) {
        if (a.given(index[i])) {
            const at::Tensor* t = fitting(a, index[i], device, {sizes[i]}, at::kInt);
            if (t) out[i] = *t;
        } else {
            total += sizes[i];
        }
    }
    if (!a.ok || total == 0) return;
    const at::Tensor all = at::empty({total}, like.options());
    for (size_t i = 0; i < K; ++i)
        if (!a.given(index[i])) {
            // (what a view does, without the dispatcher's microsecond)
            auto impl = c10::make_intrusive<c10::TensorImpl>(c10::Storage(all.storage()), all.key_set(), all.dtype());
            impl->set_storage_offset(at);
            impl->set_sizes_contiguous({sizes[i]});
            out[i] = at::Tensor(std::move(impl));
            at += sizes[i];
        }
}
// (undefined where none is given and none is needed)
at::Tensor pages_workspace(Arguments& a, Py_ssize_t i, int device, int B, int n_pages, const at::Tensor& like) {
    if (!a.given(i)) {
        const int64_t need = a.ok ? (int64_t)lib.pages_workspace_bytes(B, n_pages) : 0;
        return need > 0 ? at::empty({need}, like.options().dtype(at::kByte)) : at::Tensor();
    }
    const at::Tensor* t = a.tensor(i);
    if (!t || t->device().index() != device || t->scalar_type() != at::kByte || t->dim() != 1) {
        a.ok = false;
        return at::Tensor();
    }
    return *t;
}

// (block_table, lens, parents, page_size, n_pages, held, new_table, new_lens, src, dst, missing, workspace, stream)
PyObject* cache_fork(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return native([&]() -> PyObject* {
        Arguments a(args, n, 13);
        if (!a.ok) return nullptr;
        const int device = current_device();
        int B = 0, max_pages = 0;
        const at::Tensor* table = table_of(a, 0, device, B, max_pages);
        const at::Tensor* lens = fitting(a, 1, device, {B}, at::kInt);
        if (!a.ok || !THPVariable_CheckExact(args[2]) || THPVariable_Unpack(args[2]).dim() != 1) return nullptr;
        const int64_t rows = THPVariable_Unpack(args[2]).size(0);
        if (rows > 0x7fffffff) return nullptr;
        const at::Tensor* parents = fitting(a, 2, device, {rows}, at::kInt);
        const int page_size = whole(a, 3), n_pages = whole(a, 4), B_new = (int)rows;
        const at::Tensor* held = ints_or_none(a, 5, device, n_pages);
        void* stream = a.stream(12);
        if (!a.ok) return nullptr;
        const at::Tensor new_table = fitting_output(a, 6, device, {B_new, max_pages}, at::kInt, *table);
        at::Tensor rest[4];
        together(a, {7, 8, 9, 10}, device, {B_new, B_new, B_new, 1}, *table, rest);
        if (!a.ok) return nullptr;
        const at::Tensor &new_lens = rest[0], &src = rest[1], &dst = rest[2], &missing = rest[3];
        const at::Tensor workspace = pages_workspace(a, 11, device, B_new, n_pages, *table);
        if (!a.ok) return nullptr;
        const int *tp = pointer<int>(table), *lp = pointer<int>(lens), *pp = pointer<int>(parents), *hp = pointer<int>(held);
        int *ntp = pointer<int>(&new_table), *nlp = pointer<int>(&new_lens), *sp = pointer<int>(&src), *dp = pointer<int>(&dst), *mp = pointer<int>(&missing);
        void* wp = workspace.defined() ? workspace.data_ptr() : nullptr;
        const size_t bytes = workspace.defined() ? (size_t)workspace.numel() : 0;
        const int st = without_gil([&] {
            return lib.cache_fork(tp, lp, pp, hp, ntp, nlp, sp, dp, mp, wp, bytes, B, B_new, page_size, n_pages, max_pages, stream);
        });
        return result(st, a, {6, 7, 8, 9, 10}, {new_table, new_lens, src, dst, missing});
    });
}

// (block_table, lens, T, page_size, n_pages, counts, held, missing, workspace, stream)
PyObject* cache_extend(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return native([&]() -> PyObject* {
        Arguments a(args, n, 10);
        if (!a.ok) return nullptr;
        const int device = current_device();
        int B = 0, max_pages = 0;
        const at::Tensor* table = table_of(a, 0, device, B, max_pages);
        const at::Tensor* lens = fitting(a, 1, device, {B}, at::kInt);
        const int T = whole(a, 2), page_size = whole(a, 3), n_pages = whole(a, 4);
        const at::Tensor *counts = ints_or_none(a, 5, device, B), *held = ints_or_none(a, 6, device, n_pages);
        void* stream = a.stream(9);
        if (!a.ok) return nullptr;
        const at::Tensor missing = fitting_output(a, 7, device, {1}, at::kInt, *table);
        const at::Tensor workspace = pages_workspace(a, 8, device, B, n_pages, *table);
        if (!a.ok) return nullptr;
        int *tp = pointer<int>(table), *mp = pointer<int>(&missing);
        const int *lp = pointer<int>(lens), *cp = pointer<int>(counts), *hp = pointer<int>(held);
        void* wp = workspace.defined() ? workspace.data_ptr() : nullptr;
        const size_t bytes = workspace.defined() ? (size_t)workspace.numel() : 0;
        const int st = without_gil([&] { return lib.cache_extend(tp, lp, cp, hp, mp, wp, bytes, B, T, page_size, n_pages, max_pages, stream); });
        return result(st, a, {0, 7}, {*table, missing});
    });
}

// (block_table, n_pages, moves, held, new_table, src, dst, top, workspace, stream)
PyObject* cache_compact(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return native([&]() -> PyObject* {
        Arguments a(args, n, 10);
        if (!a.ok) return nullptr;
        const int device = current_device();
        int B = 0, max_pages = 0;
        const at::Tensor* table = table_of(a, 0, device, B, max_pages);
        const int n_pages = whole(a, 1), moves = a.given(2) ? whole(a, 2) : n_pages > 1 ? n_pages / 2 : 1;
        const at::Tensor* held = ints_or_none(a, 3, device, n_pages);
        void* stream = a.stream(9);
        if (!a.ok) return nullptr;
        const at::Tensor new_table = fitting_output(a, 4, device, {B, max_pages}, at::kInt, *table);
        at::Tensor rest[3];
        together(a, {5, 6, 7}, device, {moves, moves, 1}, *table, rest);
        if (!a.ok) return nullptr;
        const at::Tensor &src = rest[0], &dst = rest[1], &top = rest[2];
        const at::Tensor workspace = pages_workspace(a, 8, device, B, n_pages, *table);
        if (!a.ok) return nullptr;
        const int *tp = pointer<int>(table), *hp = pointer<int>(held);
        int *ntp = pointer<int>(&new_table), *sp = pointer<int>(&src), *dp = pointer<int>(&dst), *top_p = pointer<int>(&top);
        void* wp = workspace.defined() ? workspace.data_ptr() : nullptr;
        const size_t bytes = workspace.defined() ? (size_t)workspace.numel() : 0;
        const int st = without_gil([&] { return lib.cache_compact(tp, hp, ntp, sp, dp, top_p, wp, bytes, B, moves, n_pages, max_pages, stream); });
        return result(st, a, {4, 5, 6, 7}, {new_table, src, dst, top});
    });
}

// (k_pages, v_pages, src, dst, k_scales, v_scales, stream)
PyObject* cache_copy(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return native([&]() -> PyObject* {
        Arguments a(args, n, 7);
        if (!a.ok) return nullptr;
        const int device = current_device();
        PagesArguments c;
        if (!pages_arguments(a, c, device, 0, 4, 5) || !THPVariable_CheckExact(args[2]) || THPVariable_Unpack(args[2]).dim() != 1) return nullptr;
        const int64_t pairs = THPVariable_Unpack(args[2]).size(0);
        if (pairs > 0x7fffffff) return nullptr;
        const at::Tensor *src = fitting(a, 2, device, {pairs}, at::kInt), *dst = fitting(a, 3, device, {pairs}, at::kInt);
        void* stream = a.stream(6);
        if (!a.ok) return nullptr;
        void *kp = c.k->data_ptr(), *vp = c.v->data_ptr(), *ksp = pointer(c.k_scales), *vsp = pointer(c.v_scales);
        const int *sp = pointer<int>(src), *dp = pointer<int>(dst);
        const int st = without_gil([&] { return lib.cache_copy(kp, vp, ksp, vsp, sp, dp, (int)pairs, c.s.H, c.s.d, c.s.N, c.s.B, c.code, stream); });
        return result(st, a, {0, 1}, {*c.k, *c.v});
    });
}

// bind(address of fa_fwd_gqa, fa_fwd_fp8_gqa, fa_fp8_quant_hadamard, fa_bwd_workspace_bytes, fa_bwd_gqa, fa_rope, fa_rope_bwd, fa_cache_write,
// fa_cache_read, fa_fwd_cache_workspace_bytes, fa_fwd_cache, fa_rope_axes, fa_rope_axes_bwd, fa_cache_pages_workspace_bytes, fa_cache_fork,
// fa_cache_extend, fa_cache_compact, fa_cache_copy)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
    constexpr int kAddresses = 18;
    void* p[kAddresses];
    if (n != kAddresses) {
        PyErr_SetString(PyExc_TypeError, "bind takes eighteen addresses");
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
    lib.rope_axes = reinterpret_cast<decltype(lib.rope_axes)>(p[11]);
    lib.rope_axes_bwd = reinterpret_cast<decltype(lib.rope_axes_bwd)>(p[12]);
    lib.pages_workspace_bytes = reinterpret_cast<decltype(lib.pages_workspace_bytes)>(p[13]);
    lib.cache_fork = reinterpret_cast<decltype(lib.cache_fork)>(p[14]);
    lib.cache_extend = reinterpret_cast<decltype(lib.cache_extend)>(p[15]);
    lib.cache_compact = reinterpret_cast<decltype(lib.cache_compact)>(p[16]);
    lib.cache_copy = reinterpret_cast<decltype(lib.cache_copy)>(p[17]);
    Py_RETURN_NONE;
}

#define FA_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FA_METHOD(bind), FA_METHOD(fwd), FA_METHOD(fwd_fp8), FA_METHOD(quant), FA_METHOD(bwd), FA_METHOD(rope), FA_METHOD(cache_write),
                         FA_METHOD(cache_read), FA_METHOD(fwd_cache), FA_METHOD(rope_axes), FA_METHOD(cache_fork), FA_METHOD(cache_extend),
                         FA_METHOD(cache_compact), FA_METHOD(cache_copy), {nullptr, nullptr, 0, nullptr}};
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
