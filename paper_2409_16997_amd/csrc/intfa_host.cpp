// The Python binding's plain calls, natively: take the tensors apart, allocate the outputs, call the C ABI on torch's current stream.
// What such a call costs the host bounds every small shape (quantize Q, K, V of one 128 x 64 head and attend: 26.1 us a pass with the
// arguments taken apart and the seven outputs allocated in Python, 11.1 like this, of which the two kernels take 6.6; a first pass on new inputs 38 and 24).
//
// Every function returns None for anything but the plain case -- a tensor subclass, an active torch function or dispatch mode, a tensor
// that is not contiguous, not on the current device or of another type, shapes that do not agree, a call that the C ABI refuses -- and
// the binding then takes its general path, which handles or refuses it.  An error of the HIP runtime is raised from here.  The C ABI is
// reached through the addresses that init() is given, those of the library the binding has loaded.  The GIL is released around a call, as ctypes does.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>

#include <climits>
#include <cstring>

#include "intfa.h"

namespace {

struct Abi {
    decltype(&::quantize_tokenwise_ex) tokenwise;
    decltype(&::quantize_headwise_ex) headwise;
    decltype(&::quantize_blockwise) blockwise;
    decltype(&::quantize_qkv) qkv;
    decltype(&::quantize_qk) qk;
    decltype(&::int_flash_attn_fwd_rect) fwd;
    decltype(&::int_flash_attn_fwd_vblock_rect) vblock;
    decltype(&::int_flash_attn_fwd_half_rect) half;
    decltype(&::int_flash_attn_fwd_splitk) splitk;
    decltype(&::int_flash_attn_fwd_splitk_static) splitk_static;
    decltype(&::ifa_window_workspace_bytes) window_bytes;
    decltype(&::int_flash_attn_fwd_window) window;
    decltype(&::ifa_prefix_workspace_bytes) prefix_bytes;
    decltype(&::int_flash_attn_fwd_prefix) prefix;
    decltype(&::ifa_key_weights_workspace_bytes) weights_bytes;
    decltype(&::key_weights) weights;
    decltype(&::evict_keys) evict;
    decltype(&::append_keys) append;
    decltype(&::read_keys) read;
    decltype(&::ifa_int4_workspace_bytes) int4_bytes;
    decltype(&::int_flash_attn_fwd_int4) int4;
    decltype(&::ifa_block_cols) block_cols;
} abi;
constexpr int ABI_FUNCTIONS = sizeof(Abi) / sizeof(void *);
PyObject *check = nullptr;                                       // the binding's: check(status, name of the call) raises what such a status raises

// init(check, address of every function of Abi)
PyObject *init(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 1 + ABI_FUNCTIONS) { PyErr_SetString(PyExc_TypeError, "init: check() and one address per function of the C ABI"); return nullptr; }
    void *p[ABI_FUNCTIONS];
    for (int i = 0; i < ABI_FUNCTIONS; ++i) {
        p[i] = PyLong_AsVoidPtr(args[1 + i]);
        if (!p[i]) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "init: null address"); return nullptr; }
    }
    memcpy(&abi, p, sizeof p);
    Py_INCREF(args[0]);
    Py_XSETREF(check, args[0]);
    Py_RETURN_NONE;
}

// A plain tensor: contiguous, with storage of its own kind on the current device
const at::Tensor *plain(PyObject *o, c10::DeviceIndex device) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.defined() && t.is_cuda() && t.layout() == at::kStrided && t.has_storage() && !t.is_neg() && !t.is_conj() && t.numel() > 0 &&
           t.device().index() == device && t.is_contiguous() ? &t : nullptr;
}
bool modes() { return at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set(); }
int dtype_enum(at::ScalarType t) { return t == at::kFloat ? IFA_F32 : t == at::kHalf ? IFA_F16 : t == at::kBFloat16 ? IFA_BF16 : -1; }
signed char *i8(const at::Tensor &t) { return static_cast<signed char *>(t.data_ptr()); }
float *f32(const at::Tensor &t) { return static_cast<float *>(t.data_ptr()); }
// Outputs, straight from the caching allocator: nothing between here and there (autograd of integers, a mode, a subclass) has anything to do for a
// plain call, and every output is written whole.  The six outputs of quantize_qkv: 2.9 us of host, 4.9 through the dispatcher.
at::Tensor like(const at::Tensor &x, at::ScalarType dtype) { return at::detail::empty_strided_cuda(x.sizes(), x.strides(), dtype, x.device()); }
at::Tensor codes(const at::Tensor &x) { return like(x, at::kChar); }
at::Tensor scales(const at::Tensor &x, at::IntArrayRef shape) { return at::detail::empty_cuda(shape, at::kFloat, x.device(), std::nullopt); }
// One call of the C ABI (which does not throw) without the GIL.  The arguments, data_ptr() among them, which can throw, are evaluated before it is released.
template <typename... P, typename... A> int unlocked(int (*fn)(P...), A... a) {
    PyThreadState *const state = PyEval_SaveThread();
    const int rc = fn(a...);
    PyEval_RestoreThread(state);
    return rc;
}
// False for a refusal, which comes before anything is enqueued and which the general path repeats and reports; a HIP error is raised at once:
// the runtime has forgotten it by the time of a second call, which would enqueue again what the first one has.
bool succeeded(int rc, const char *what) {
    if (rc == IFA_ERR_HIP) Py_XDECREF(PyObject_CallFunction(check, "is", rc, what));
    return rc == IFA_OK;
}
// C++ exceptions end here: the general path meets the same condition and says so
template <typename F> PyObject *guarded(F f) {
    try {
        if (modes()) Py_RETURN_NONE;
        PyObject *r = f(c10::hip::current_device());
        if (r || PyErr_Occurred()) return r;
    } catch (const std::exception &) {
    }
    Py_RETURN_NONE;
}
PyObject *tuple(std::initializer_list<at::Tensor> ts) {
    PyObject *t = PyTuple_New(static_cast<Py_ssize_t>(ts.size()));
    if (!t) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor &x : ts) {
        PyObject *o = THPVariable_Wrap(x);
        if (!o) { Py_DECREF(t); return nullptr; }
        PyTuple_SET_ITEM(t, i++, o);
    }
    return t;
}
bool number(PyObject *o, double &v) {                            // a plain Python float or int; anything else goes the general way
    if (PyFloat_CheckExact(o)) { v = PyFloat_AS_DOUBLE(o); return true; }
    if (!PyLong_CheckExact(o)) return false;
    v = PyLong_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); return false; }
    return true;
}
hipStream_t stream(c10::DeviceIndex device) { return c10::hip::getCurrentHIPStream(device).stream(); }

// quantize_tokenwise(X, scale_mul)
PyObject *tokenwise(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&](c10::DeviceIndex dev) -> PyObject * {
        double mul;
        const at::Tensor *x = n == 2 ? plain(a[0], dev) : nullptr;
        if (!x || x->dim() < 1 || !number(a[1], mul) || dtype_enum(x->scalar_type()) < 0) return nullptr;
        const auto shape = x->sizes();
        const long d = shape.back();
        at::Tensor q = codes(*x), s = scales(*x, shape.slice(0, shape.size() - 1));
        const hipStream_t st = stream(dev);
        const int rc = unlocked(abi.tokenwise, x->data_ptr(), dtype_enum(x->scalar_type()), x->numel() / d, static_cast<int>(d), i8(q), f32(s), static_cast<float>(mul), st);
        return succeeded(rc, "quantize_tokenwise") ? tuple({q, s}) : nullptr;
    });
}

// quantize_headwise(X)
PyObject *headwise(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&](c10::DeviceIndex dev) -> PyObject * {
        const at::Tensor *x = n == 1 ? plain(a[0], dev) : nullptr;
        if (!x || x->dim() < 2 || dtype_enum(x->scalar_type()) < 0) return nullptr;
        const auto shape = x->sizes();
        const long d = shape.back(), N = shape[shape.size() - 2];
        at::Tensor q = codes(*x), s = scales(*x, shape.slice(0, shape.size() - 2));
        const hipStream_t st = stream(dev);
        const int rc = unlocked(abi.headwise, x->data_ptr(), dtype_enum(x->scalar_type()), x->numel() / (N * d), N, d, i8(q), f32(s), 0, st);
        return succeeded(rc, "quantize_headwise_ex") ? tuple({q, s}) : nullptr;
    });
}

// quantize_blockwise(X, block_keys)
PyObject *blockwise(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&](c10::DeviceIndex dev) -> PyObject * {
        const at::Tensor *x = n == 2 ? plain(a[0], dev) : nullptr;
        if (!x || x->dim() < 2 || dtype_enum(x->scalar_type()) < 0 || !PyLong_CheckExact(a[1])) return nullptr;
        int overflow = 0;
        const long block = PyLong_AsLongAndOverflow(a[1], &overflow);
        if (overflow || block <= 0 || block > INT_MAX) return nullptr;
        const auto shape = x->sizes();
        const long d = shape.back(), N = shape[shape.size() - 2];
        if (d > INT_MAX) return nullptr;
        c10::SmallVector<int64_t, 5> sshape(shape.begin(), shape.end() - 1);
        sshape.back() = (N + block - 1) / block;
        at::Tensor q = codes(*x), s = scales(*x, sshape);
        const hipStream_t st = stream(dev);
        const int rc = unlocked(abi.blockwise, x->data_ptr(), dtype_enum(x->scalar_type()), x->numel() / (N * d), N, static_cast<int>(d), static_cast<int>(block), i8(q), f32(s), st);
        return succeeded(rc, "quantize_blockwise") ? tuple({q, s}) : nullptr;
    });
}

// quantize_qkv(Q, K, V, s_Q_mul)
PyObject *qkv(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&](c10::DeviceIndex dev) -> PyObject * {
        double mul;
        const at::Tensor *q = n == 4 ? plain(a[0], dev) : nullptr, *k = q ? plain(a[1], dev) : nullptr, *v = k ? plain(a[2], dev) : nullptr;
        if (!v || q->dim() < 2 || !number(a[3], mul)) return nullptr;
        const int dt = dtype_enum(q->scalar_type());
        if (dt < 0 || k->scalar_type() != q->scalar_type() || v->scalar_type() != q->scalar_type() || k->sizes() != q->sizes() || v->sizes() != q->sizes()) return nullptr;
        const auto shape = q->sizes();
        const long d = shape.back(), N = shape[shape.size() - 2];
        at::Tensor q8 = codes(*q), k8 = codes(*q), v8 = codes(*q);
        at::Tensor sq = scales(*q, shape.slice(0, shape.size() - 1)), sk = scales(*q, shape.slice(0, shape.size() - 1)), sv = scales(*q, shape.slice(0, shape.size() - 2));
        const hipStream_t st = stream(dev);
        const int rc = unlocked(abi.qkv, q->data_ptr(), k->data_ptr(), v->data_ptr(), dt, q->numel() / (N * d), N, static_cast<int>(d), i8(q8), i8(k8), i8(v8), f32(sq), f32(sk), f32(sv), static_cast<float>(mul), st);
        return succeeded(rc, "quantize_qkv") ? tuple({q8, k8, v8, sq, sk, sv}) : nullptr;
    });
}

// quantize_qk(Q, K, s_Q_mul, hadamard)
PyObject *qk(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&](c10::DeviceIndex dev) -> PyObject * {
        double mul;
        const at::Tensor *q = n == 4 ? plain(a[0], dev) : nullptr, *k = q ? plain(a[1], dev) : nullptr;
        if (!k || q->dim() < 1 || !number(a[2], mul) || !PyBool_Check(a[3])) return nullptr;
        const int dt = dtype_enum(q->scalar_type()), had = a[3] == Py_True;
        if (dt < 0 || k->scalar_type() != q->scalar_type() || k->sizes() != q->sizes()) return nullptr;
        const auto shape = q->sizes();
        const long d = shape.back();
        at::Tensor q8 = codes(*q), k8 = codes(*q), sq = scales(*q, shape.slice(0, shape.size() - 1)), sk = scales(*q, shape.slice(0, shape.size() - 1));
        const hipStream_t st = stream(dev);
        const int rc = unlocked(abi.qk, q->data_ptr(), k->data_ptr(), dt, q->numel() / d, static_cast<int>(d), i8(q8), i8(k8), f32(sq), f32(sk), static_cast<float>(mul), had, st);
        return succeeded(rc, "quantize_qk") ? tuple({q8, k8, sq, sk}) : nullptr;
    });
}

// The operands of an attention call: int8 Q [B, H, Nq, d], K, V [B, H, Nk, d] (V of `vtype`), s_Q, s_K, and the output type
struct Call {
    const at::Tensor *q, *k, *v, *sq, *sk, *sv = nullptr;
    int B, H, Nq, Nk, d, causal, o_dtype;
    at::Tensor out;
    bool take(PyObject *const *a, c10::DeviceIndex dev, at::ScalarType vtype, PyObject *s_v, PyObject *causal_, PyObject *out_dtype) {
        if (!(q = plain(a[0], dev)) || !(k = plain(a[1], dev)) || !(v = plain(a[2], dev)) || !(sq = plain(a[3], dev)) || !(sk = plain(a[4], dev))) return false;
        if (s_v && (!(sv = plain(s_v, dev)) || sv->scalar_type() != at::kFloat)) return false;
        if (q->scalar_type() != at::kChar || k->scalar_type() != at::kChar || v->scalar_type() != vtype || sq->scalar_type() != at::kFloat || sk->scalar_type() != at::kFloat) return false;
        if (q->dim() != 4 || k->dim() != 4 || v->sizes() != k->sizes() || sq->sizes() != q->sizes().slice(0, 3) || sk->sizes() != k->sizes().slice(0, 3)) return false;
        if (k->size(0) != q->size(0) || k->size(1) != q->size(1) || k->size(3) != q->size(3)) return false;
        for (const at::Tensor *t : {q, k})
            for (const auto s : t->sizes()) if (s > INT_MAX) return false;
        B = static_cast<int>(q->size(0)), H = static_cast<int>(q->size(1)), Nq = static_cast<int>(q->size(2)), Nk = static_cast<int>(k->size(2)), d = static_cast<int>(q->size(3));
        if (!PyBool_Check(causal_)) return false;
        causal = causal_ == Py_True;
        const at::ScalarType ot = out_dtype == Py_None ? at::kHalf : THPDtype_Check(out_dtype) ? reinterpret_cast<THPDtype *>(out_dtype)->scalar_type : at::kChar;
        if ((o_dtype = dtype_enum(ot)) < 0) return false;
        out = like(*q, ot);
        return true;
    }
};

// fwd(Q, K, V, s_Q, s_K, s_V, causal, out_dtype)
PyObject *fwd(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&](c10::DeviceIndex dev) -> PyObject * {
        Call c;
        if (n != 8 || !c.take(a, dev, at::kChar, a[5], a[6], a[7])) return nullptr;
        const bool vb = c.sv->dim() == 3;
        if (vb) {
            const int bc = abi.block_cols(c.d, c.causal);
            if (bc <= 0 || c.sv->size(0) != c.B || c.sv->size(1) != c.H || c.sv->size(2) != (c.Nk + bc - 1) / bc) return nullptr;
        } else if (c.sv->numel() < static_cast<int64_t>(c.B) * c.H) return nullptr;              // a scale of every head is read
        const hipStream_t st = stream(dev);
        const int rc = unlocked(vb ? abi.vblock : abi.fwd, i8(*c.q), i8(*c.k), i8(*c.v), f32(*c.sq), f32(*c.sk), f32(*c.sv), c.B, c.H, c.Nq, c.Nk, c.d, c.causal, c.out.data_ptr(), c.o_dtype, st);
        return succeeded(rc, "int_flash_attn_fwd") ? THPVariable_Wrap(c.out) : nullptr;
    });
}

// half(Q, K, V, s_Q, s_K, causal, out_dtype)
PyObject *half(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&](c10::DeviceIndex dev) -> PyObject * {
        Call c;
        if (n != 7 || !c.take(a, dev, at::kHalf, nullptr, a[5], a[6])) return nullptr;
        const hipStream_t st = stream(dev);
        const int rc = unlocked(abi.half, i8(*c.q), i8(*c.k), c.v->data_ptr(), f32(*c.sq), f32(*c.sk), c.B, c.H, c.Nq, c.Nk, c.d, c.causal, c.out.data_ptr(), c.o_dtype, st);
        return succeeded(rc, "int_flash_attn_fwd_half") ? THPVariable_Wrap(c.out) : nullptr;
    });
}

// splitk(Q, K, V, s_Q, s_K, s_V, causal, out_dtype, workspace or None for the built-in one)
PyObject *splitk(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&](c10::DeviceIndex dev) -> PyObject * {
        Call c;
        const at::Tensor *ws = nullptr;
        if (n != 9 || (a[8] != Py_None && (!(ws = plain(a[8], dev)) || ws->scalar_type() != at::kByte))) return nullptr;
        if (!c.take(a, dev, at::kChar, a[5], a[6], a[7]) || c.sv->dim() != 2 || c.sv->size(0) != c.B || c.sv->size(1) != c.H) return nullptr;
        const hipStream_t st = stream(dev);
        const int rc = ws ? unlocked(abi.splitk, i8(*c.q), i8(*c.k), i8(*c.v), f32(*c.sq), f32(*c.sk), f32(*c.sv), c.B, c.H, c.Nq, c.Nk, c.d, c.causal, c.out.data_ptr(), c.o_dtype, ws->data_ptr(), ws->numel(), st)
                          : unlocked(abi.splitk_static, i8(*c.q), i8(*c.k), i8(*c.v), f32(*c.sq), f32(*c.sk), f32(*c.sv), c.B, c.H, c.Nq, c.Nk, c.d, c.causal, c.out.data_ptr(), c.o_dtype, st);
        return succeeded(rc, ws ? "int_flash_attn_fwd_splitk" : "int_flash_attn_fwd_splitk_static") ? THPVariable_Wrap(c.out) : nullptr;
    });
}

// ---- a quantized cache in long use: 17 to 27 us of host a call through Python, 5 to 9 like this
bool optional(PyObject *o, c10::DeviceIndex dev, const at::Tensor *&t) { return o == Py_None || (t = plain(o, dev)); }
bool integer(PyObject *o, int &v) {                              // a plain int; what lies above INT_MAX means "all of them" everywhere here
    int overflow = 0;
    if (!PyLong_CheckExact(o)) return false;
    const long x = PyLong_AsLongAndOverflow(o, &overflow);
    if (overflow < 0 || x < 0) return false;
    v = overflow || x > INT_MAX ? INT_MAX : static_cast<int>(x);
    return true;
}
bool is(const at::Tensor *t, at::ScalarType type, at::IntArrayRef shape) { return t->scalar_type() == type && t->sizes() == shape; }

// Q [B, H, Nq, d] and s_Q against a cache K [B, Hkv, Nk, d], s_K, optional lens [B]
struct Cached {
    const at::Tensor *q, *k, *sq, *sk, *lens = nullptr;
    int B, H, Hkv, Nq, Nk, d;
    bool take(c10::DeviceIndex dev, PyObject *q_, PyObject *k_, PyObject *sq_, PyObject *sk_, PyObject *lens_) {
        if (!(q = plain(q_, dev)) || !(k = plain(k_, dev)) || !(sq = plain(sq_, dev)) || !(sk = plain(sk_, dev)) || !optional(lens_, dev, lens)) return false;
        if (q->dim() != 4 || k->dim() != 4 || q->scalar_type() != at::kChar || k->scalar_type() != at::kChar) return false;
        for (const at::Tensor *t : {q, k})
            for (const auto s : t->sizes()) if (s > INT_MAX) return false;
        B = static_cast<int>(q->size(0)), H = static_cast<int>(q->size(1)), Nq = static_cast<int>(q->size(2)), d = static_cast<int>(q->size(3));
        Hkv = static_cast<int>(k->size(1)), Nk = static_cast<int>(k->size(2));
        return k->size(0) == B && k->size(3) == d && H % Hkv == 0 && is(sq, at::kFloat, {B, H, Nq}) && is(sk, at::kFloat, {B, Hkv, Nk}) && (!lens || is(lens, at::kInt, {B}));
    }
    const int *lengths() const { return lens ? static_cast<const int *>(lens->data_ptr()) : nullptr; }
};
// V [..., d] and its scale: fp16 and none, or INT8 and one of that shape
bool values(const at::Tensor *v, const at::Tensor *sv, at::IntArrayRef shape, at::IntArrayRef scale_shape) {
    return is(v, sv ? at::kChar : at::kHalf, shape) && (!sv || is(sv, at::kFloat, scale_shape));
}
bool output(const at::Tensor &q, PyObject *out_dtype, at::Tensor &out, int &o_dtype) {
    const at::ScalarType ot = out_dtype == Py_None ? at::kHalf : THPDtype_Check(out_dtype) ? reinterpret_cast<THPDtype *>(out_dtype)->scalar_type : at::kChar;
    if ((o_dtype = dtype_enum(ot)) < 0) return false;
    out = like(q, ot);
    return true;
}
// The caller's workspace, or one from the caching allocator, which keeps it for this stream
struct Workspace {
    at::Tensor own;
    void *p = nullptr;
    long bytes = 0;
    bool take(const at::Tensor *given, long need, const at::Device &device) {
        if (need < 0 || (given && given->scalar_type() != at::kByte)) return false;
        if (!given && need > 0) own = at::detail::empty_cuda({need}, at::kByte, device, std::nullopt);
        const at::Tensor *t = given ? given : own.defined() ? &own : nullptr;
        if (t) p = t->data_ptr(), bytes = t->numel();
        return true;
    }
};

// window(Q, K, V, s_Q, s_K, window, sinks, s_V, lens, out_dtype, workspace)
PyObject *window(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&](c10::DeviceIndex dev) -> PyObject * {
        Cached c;
        const at::Tensor *v, *sv = nullptr, *given = nullptr;
        int w, sinks, o_dtype;
        at::Tensor out;
        Workspace ws;
        if (n != 11 || !c.take(dev, a[0], a[1], a[3], a[4], a[8]) || !(v = plain(a[2], dev)) || !integer(a[5], w) || !integer(a[6], sinks) || !optional(a[7], dev, sv) || !optional(a[10], dev, given) ||
            !values(v, sv, c.k->sizes(), {c.B, c.Hkv}) || !output(*c.q, a[9], out, o_dtype) || !ws.take(given, abi.window_bytes(c.B, c.H, c.Hkv, c.Nq, c.Nk, c.d, w, sinks), c.q->device())) return nullptr;
        const hipStream_t st = stream(dev);
        const int rc = unlocked(abi.window, i8(*c.q), i8(*c.k), v->data_ptr(), f32(*c.sq), f32(*c.sk), sv ? f32(*sv) : nullptr, c.lengths(), c.B, c.H, c.Hkv, c.Nq, c.Nk, c.d, w, sinks, out.data_ptr(), o_dtype,
                                ws.p, ws.bytes, st);
        return succeeded(rc, "int_flash_attn_fwd_window") ? THPVariable_Wrap(out) : nullptr;
    });
}

// prefix(Q, Kp, Vp, K, V, s_Q, s_Kp, s_K, s_Vp, s_V, lens, out_dtype, workspace)
PyObject *prefix(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&](c10::DeviceIndex dev) -> PyObject * {
        Cached c;
        const at::Tensor *kp, *vp, *v, *skp, *svp = nullptr, *sv = nullptr, *given = nullptr;
        int o_dtype;
        at::Tensor out;
        Workspace ws;
        if (n != 13 || !c.take(dev, a[0], a[3], a[5], a[7], a[10]) || !(kp = plain(a[1], dev)) || !(vp = plain(a[2], dev)) || !(v = plain(a[4], dev)) || !(skp = plain(a[6], dev)) ||
            !optional(a[8], dev, svp) || !optional(a[9], dev, sv) || !optional(a[12], dev, given) || !svp != !sv || kp->dim() != 3 || kp->size(1) > INT_MAX) return nullptr;
        const int Np = static_cast<int>(kp->size(1));
        if (!is(kp, at::kChar, {c.Hkv, Np, c.d}) || !is(skp, at::kFloat, {c.Hkv, Np}) || !values(vp, svp, kp->sizes(), {c.Hkv}) || !values(v, sv, c.k->sizes(), {c.B, c.Hkv}) ||
            !output(*c.q, a[11], out, o_dtype) || !ws.take(given, abi.prefix_bytes(c.B, c.H, c.Hkv, c.Nq, Np, c.Nk, c.d), c.q->device())) return nullptr;
        const hipStream_t st = stream(dev);
        const int rc = unlocked(abi.prefix, i8(*c.q), i8(*kp), vp->data_ptr(), i8(*c.k), v->data_ptr(), f32(*c.sq), f32(*skp), f32(*c.sk), svp ? f32(*svp) : nullptr, sv ? f32(*sv) : nullptr, c.lengths(),
                                c.B, c.H, c.Hkv, c.Nq, Np, c.Nk, c.d, out.data_ptr(), o_dtype, ws.p, ws.bytes, st);
        return succeeded(rc, "int_flash_attn_fwd_prefix") ? THPVariable_Wrap(out) : nullptr;
    });
}

// weights(Q, K, s_Q, s_K, W, lens, out, workspace)
PyObject *weights(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&](c10::DeviceIndex dev) -> PyObject * {
        Cached c;
        const at::Tensor *w = nullptr, *to = nullptr, *given = nullptr;
        Workspace ws;
        if (n != 8 || !c.take(dev, a[0], a[1], a[2], a[3], a[5]) || !optional(a[4], dev, w) || !optional(a[6], dev, to) || !optional(a[7], dev, given)) return nullptr;
        if ((w && !is(w, at::kFloat, c.sk->sizes())) || (to && !is(to, at::kFloat, c.sk->sizes()))) return nullptr;
        if (!ws.take(given, abi.weights_bytes(c.B, c.H, c.Hkv, c.Nq, c.Nk, c.d), c.q->device())) return nullptr;
        const at::Tensor out = to ? *to : like(*c.sk, at::kFloat);
        const hipStream_t st = stream(dev);
        const int rc = unlocked(abi.weights, i8(*c.q), i8(*c.k), f32(*c.sq), f32(*c.sk), c.lengths(), w ? f32(*w) : nullptr, c.B, c.H, c.Hkv, c.Nq, c.Nk, c.d, f32(out), ws.p, ws.bytes, st);
        return succeeded(rc, "key_weights") ? THPVariable_Wrap(out) : nullptr;
    });
}

// evict(K, s_K, V, W, keep, recent, sinks, lens)
PyObject *evict(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&](c10::DeviceIndex dev) -> PyObject * {
        const at::Tensor *k, *sk, *v, *w, *lens = nullptr;
        int keep, recent, sinks;
        if (n != 8 || !(k = plain(a[0], dev)) || !(sk = plain(a[1], dev)) || !(v = plain(a[2], dev)) || !(w = plain(a[3], dev)) || !integer(a[4], keep) || !integer(a[5], recent) || !integer(a[6], sinks) ||
            !optional(a[7], dev, lens) || k->dim() != 4 || k->scalar_type() != at::kChar) return nullptr;
        for (const auto s : k->sizes()) if (s > INT_MAX) return nullptr;
        const int B = static_cast<int>(k->size(0)), Hkv = static_cast<int>(k->size(1)), Nk = static_cast<int>(k->size(2)), d = static_cast<int>(k->size(3));
        const at::ScalarType vt = v->scalar_type();
        if (!is(sk, at::kFloat, {B, Hkv, Nk}) || !is(w, at::kFloat, {B, Hkv, Nk}) || (vt != at::kChar && vt != at::kHalf) || v->sizes() != k->sizes() || (lens && !is(lens, at::kInt, {B}))) return nullptr;
        if (keep < 1 || keep > Nk || static_cast<long>(recent) + sinks > keep) return nullptr;
        const at::Device device = k->device();
        auto rows = [&](at::ScalarType type) { return at::detail::empty_cuda({B, Hkv, keep}, type, device, std::nullopt); };
        auto wide = [&](at::ScalarType type) { return at::detail::empty_cuda({B, Hkv, keep, d}, type, device, std::nullopt); };
        const at::Tensor k2 = wide(at::kChar), sk2 = rows(at::kFloat), v2 = wide(vt), w2 = rows(at::kFloat), index = rows(at::kInt), left = at::detail::empty_cuda({B}, at::kInt, device, std::nullopt);
        const hipStream_t st = stream(dev);
        const int rc = unlocked(abi.evict, i8(*k), f32(*sk), v->data_ptr(), static_cast<int>(v->element_size()), f32(*w), lens ? static_cast<const int *>(lens->data_ptr()) : nullptr, B, Hkv, Nk, d, keep, recent, sinks,
                                i8(k2), f32(sk2), v2.data_ptr(), f32(w2), static_cast<int *>(index.data_ptr()), static_cast<int *>(left.data_ptr()), st);
        return succeeded(rc, "evict_keys") ? tuple({k2, sk2, v2, w2, index, left}) : nullptr;
    });
}

// ---- writing the cache, and a cache in 4 bits
// The cache's arrays K, s_K, V, s_V (None for fp16 V) and lens, from a[0] on
struct Held {
    const at::Tensor *k, *sk, *v, *sv = nullptr, *lens = nullptr;
    int held, B, Hkv, Nk, d;
    bool take(c10::DeviceIndex dev, PyObject *const *a, PyObject *lens_) {
        if (!(k = plain(a[0], dev)) || !(sk = plain(a[1], dev)) || !(v = plain(a[2], dev)) || !optional(a[3], dev, sv) || !optional(lens_, dev, lens) || k->dim() != 4) return false;
        for (const auto s : k->sizes()) if (s > INT_MAX / 2) return false;
        B = static_cast<int>(k->size(0)), Hkv = static_cast<int>(k->size(1)), Nk = static_cast<int>(k->size(2)), d = static_cast<int>(k->size(3));
        const bool four = k->scalar_type() == at::kByte;
        if (!four && k->scalar_type() != at::kChar) return false;
        held = four ? IFA_CACHE_I4 : sv ? IFA_CACHE_I8 : IFA_CACHE_I8_F16;
        if (four) d *= 2;
        if (!is(v, four ? at::kByte : sv ? at::kChar : at::kHalf, k->sizes()) || !is(sk, at::kFloat, {B, Hkv, Nk}) || (lens && !is(lens, at::kInt, {B}))) return false;
        return four ? sv && is(sv, at::kFloat, {B, Hkv, Nk}) : !sv || is(sv, at::kFloat, {B, Hkv});
    }
    float *scale() const { return sv ? f32(*sv) : nullptr; }
    const int *lengths() const { return lens ? static_cast<const int *>(lens->data_ptr()) : nullptr; }
};
// Activations [B, Hkv, Nn, d] whose rows are contiguous, of any strides otherwise
const at::Tensor *tokens(PyObject *o, c10::DeviceIndex device, const Held &c) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.defined() && t.is_cuda() && t.layout() == at::kStrided && t.has_storage() && !t.is_neg() && !t.is_conj() && t.numel() > 0 && t.device().index() == device && t.dim() == 4 &&
           t.stride(3) == 1 && t.size(0) == c.B && t.size(1) == c.Hkv && t.size(2) <= INT_MAX && t.size(3) == c.d ? &t : nullptr;
}

// append(K, V, K_c, s_K, V_c, s_V, lens, hadamard): True when it is done
PyObject *append(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&](c10::DeviceIndex dev) -> PyObject * {
        Held c;
        const at::Tensor *k, *v;
        if (n != 8 || !c.take(dev, a + 2, a[6]) || !(k = tokens(a[0], dev, c)) || !(v = tokens(a[1], dev, c)) || !PyBool_Check(a[7])) return nullptr;
        const int dt = dtype_enum(k->scalar_type());
        if (dt < 0 || v->scalar_type() != k->scalar_type() || v->sizes() != k->sizes()) return nullptr;
        const hipStream_t st = stream(dev);
        const int rc = unlocked(abi.append, k->data_ptr(), v->data_ptr(), dt, k->stride(0), k->stride(1), k->stride(2), v->stride(0), v->stride(1), v->stride(2), c.lengths(), c.B, c.Hkv,
                                static_cast<int>(k->size(2)), c.Nk, c.d, c.held, static_cast<int>(a[7] == Py_True), c.k->data_ptr(), f32(*c.sk), c.v->data_ptr(), c.scale(), st);
        if (!succeeded(rc, "append_keys")) return nullptr;
        Py_RETURN_TRUE;
    });
}

// read(K_c, s_K, V_c, s_V, lens, first (-1: the last), count, hadamard, out_dtype)
PyObject *read(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&](c10::DeviceIndex dev) -> PyObject * {
        Held c;
        int count, overflow = 0;
        if (n != 9 || !c.take(dev, a, a[4]) || !PyLong_CheckExact(a[5]) || !integer(a[6], count) || count < 1 || !PyBool_Check(a[7])) return nullptr;
        const long first = PyLong_AsLongAndOverflow(a[5], &overflow);
        const at::ScalarType ot = a[8] == Py_None ? at::kHalf : THPDtype_Check(a[8]) ? reinterpret_cast<THPDtype *>(a[8])->scalar_type : at::kChar;
        const int dt = dtype_enum(ot);
        if (overflow || first < -1 || first > c.Nk || dt < 0 || static_cast<long>(c.B) * c.Hkv * count > 1L << 28 || (c.d != 64 && c.d != 128)) return nullptr;      // (sizes that are refused allocate nothing)
        const at::Tensor k = at::detail::empty_cuda({c.B, c.Hkv, count, c.d}, ot, c.k->device(), std::nullopt), v = at::detail::empty_cuda({c.B, c.Hkv, count, c.d}, ot, c.k->device(), std::nullopt);
        const hipStream_t st = stream(dev);
        const int rc = unlocked(abi.read, c.k->data_ptr(), f32(*c.sk), c.v->data_ptr(), c.scale(), c.lengths(), c.B, c.Hkv, c.Nk, c.d, c.held, static_cast<int>(a[7] == Py_True), first, count, k.data_ptr(),
                                v.data_ptr(), dt, st);
        return succeeded(rc, "read_keys") ? tuple({k, v}) : nullptr;
    });
}

// int4(Q, K, V, s_Q, s_K, s_V, window or None, sinks, lens, out_dtype, workspace)
PyObject *int4(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&](c10::DeviceIndex dev) -> PyObject * {
        Held c;
        const at::Tensor *q, *sq, *given = nullptr;
        int w = INT_MAX, sinks, o_dtype;
        at::Tensor out;
        Workspace ws;
        if (n != 11) return nullptr;
        PyObject *const cache[4] = {a[1], a[4], a[2], a[5]};
        if (!c.take(dev, cache, a[8]) || c.held != IFA_CACHE_I4 || !(q = plain(a[0], dev)) || !(sq = plain(a[3], dev)) || (a[6] != Py_None && !integer(a[6], w)) || !integer(a[7], sinks) || !optional(a[10], dev, given) ||
            q->dim() != 4 || q->scalar_type() != at::kChar || q->size(0) != c.B || q->size(1) > INT_MAX || q->size(1) % c.Hkv || q->size(2) > INT_MAX || q->size(3) != c.d) return nullptr;
        const int H = static_cast<int>(q->size(1)), Nq = static_cast<int>(q->size(2));
        if (!is(sq, at::kFloat, {c.B, H, Nq}) || !output(*q, a[9], out, o_dtype) || !ws.take(given, abi.int4_bytes(c.B, H, c.Hkv, Nq, c.Nk, c.d, w, sinks), q->device())) return nullptr;
        const hipStream_t st = stream(dev);
        const int rc = unlocked(abi.int4, i8(*q), c.k->data_ptr(), c.v->data_ptr(), f32(*sq), f32(*c.sk), f32(*c.sv), c.lengths(), c.B, H, c.Hkv, Nq, c.Nk, c.d, w, sinks, out.data_ptr(), o_dtype, ws.p, ws.bytes, st);
        return succeeded(rc, "int_flash_attn_fwd_int4") ? THPVariable_Wrap(out) : nullptr;
    });
}

#define FASTCALL(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FASTCALL(init), FASTCALL(tokenwise), FASTCALL(headwise), FASTCALL(blockwise), FASTCALL(qkv), FASTCALL(qk), FASTCALL(fwd), FASTCALL(half), FASTCALL(splitk), FASTCALL(window), FASTCALL(prefix), FASTCALL(weights), FASTCALL(evict), FASTCALL(append), FASTCALL(read), FASTCALL(int4), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_intfa_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__intfa_host() {
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", INTFA_TORCH_VERSION) < 0) Py_CLEAR(m);      // the one whose internals it was built for
    return m;
}
