// fastcall.cpp -- the binding's entry points for well-formed calls, in native code.
//
// A one-byte step takes the GPU a few microseconds, and marshalling its call in Python
// (argument checks, an output allocation and a ctypes call with 15 arguments) took about
// 10: decoding was bound by the host.  Each function here takes the arguments of the
// Python function of the same name, all positional.  If every tensor is a plain dense
// GPU tensor of the expected shape, type and layout on the current device, it allocates
// the outputs, calls the C ABI on the current stream and returns what the Python function
// returns.  Anything else returns None with nothing done, and the Python function goes on
// to its own checks, which raise the errors; a call that the library refuses returns its
// status (an int).  Per decoded byte (conv1d_step and scan_step, 3584 channels, batch 1):
// 21.3 us before, 10.0 now.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <optional>
#include <utility>
#include <vector>

#include "mbscan.h"

namespace {

decltype(&mb_scan_fwd) scan_fwd_fn;
decltype(&mb_scan_fwd_states) scan_fwd_states_fn;
decltype(&mb_scan_fwd_ckpt) scan_fwd_ckpt_fn;
decltype(&mb_scan_step) scan_step_fn;
decltype(&mb_conv1d_fwd) conv1d_fwd_fn;
decltype(&mb_conv1d_step) conv1d_step_fn;
decltype(&mb_verify_rank) verify_rank_fn;
decltype(&mb_embedding_fwd) embedding_fwd_fn;
decltype(&mb_embedding_bwd) embedding_bwd_fn;
decltype(&mb_embedding_bwd_workspace) embedding_bwd_workspace_fn;
decltype(&mb_conv1d_bwd) conv1d_bwd_fn;
decltype(&mb_conv1d_bwd_workspace) conv1d_bwd_workspace_fn;
decltype(&mb_grad_norm) grad_norm_fn;
decltype(&mb_grad_norm_workspace) grad_norm_workspace_fn;
decltype(&mb_clip_grad_norm) clip_grad_norm_fn;
decltype(&mb_verify_sample) verify_sample_fn;
decltype(&mb_verify_sample_workspace) verify_sample_workspace_fn;
decltype(&mb_rms_norm_fwd) rms_norm_fwd_fn;
decltype(&mb_rms_norm_bwd) rms_norm_bwd_fn;
decltype(&mb_rms_norm_bwd_workspace) rms_norm_bwd_workspace_fn;
decltype(&mb_quantize_fp8) quantize_fp8_fn;
decltype(&mb_matmul_fp8) matmul_fp8_fn;
decltype(&mb_sample) sample_fn;
PyObject *current_device, *raw_stream, *parameter_type;   // torch's accessors and nn.Parameter

// A plain dense tensor on the GPU (no subclass, no transform's wrapper), or null.
const at::Tensor *plain(PyObject *o) {
    if (!THPVariable_CheckExact(o) && reinterpret_cast<PyObject *>(Py_TYPE(o)) != parameter_type) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    const auto ks = t.unsafeGetTensorImpl()->key_set();
    if (!t.defined() || !ks.has(c10::DispatchKey::CUDA) || ks.has(c10::DispatchKey::Python) || !t.has_storage())
        return nullptr;
    return &t;
}

// The checks of one call: ok stays true while every argument is as the library wants it.
struct Call {
    bool ok = true;
    c10::Device dev{c10::DeviceType::CPU};
    void *stream = nullptr;

    // The tensor that fixes the device: dims dimensions, on the current device.
    const at::Tensor *first(PyObject *o, int64_t dims) {
        const at::Tensor *t = plain(o);
        if (!t || t->dim() != dims || c10::impl::TorchDispatchModeTLS::any_modes_set()) { ok = false; return nullptr; }
        dev = t->device();
        PyObject *cur = PyObject_CallNoArgs(current_device);
        if (!cur) { PyErr_Clear(); ok = false; return nullptr; }
        const long index = PyLong_AsLong(cur);
        Py_DECREF(cur);
        if (index != dev.index()) { ok = false; return nullptr; }
        PyObject *at = PyLong_FromLong(index);
        PyObject *s = PyObject_CallOneArg(raw_stream, at);
        Py_DECREF(at);
        if (!s) { PyErr_Clear(); ok = false; return nullptr; }
        stream = PyLong_AsVoidPtr(s);
        Py_DECREF(s);
        return t;
    }
    // A required tensor of this shape and type; its data.
    void *need(PyObject *o, at::IntArrayRef shape, at::ScalarType type) {
        const at::Tensor *t = ok ? plain(o) : nullptr;
        if (!t || t->scalar_type() != type || t->device() != dev || t->sizes() != shape ||
            !t->is_contiguous()) {
            ok = false;
            return nullptr;
        }
        return t->data_ptr();
    }
    // The same, or None: null.
    void *maybe(PyObject *o, at::IntArrayRef shape, at::ScalarType type) {
        return o == Py_None ? nullptr : need(o, shape, type);
    }
    static bool act(at::ScalarType t) { return t == at::kFloat || t == at::kBFloat16; }
    // An output given by the caller (any activation type), or its type when it is None.
    void *given(PyObject *o, at::IntArrayRef shape, at::ScalarType &type) {
        if (o == Py_None) return nullptr;
        const at::Tensor *t = ok ? plain(o) : nullptr;
        if (!t || !act(t->scalar_type())) { ok = false; return nullptr; }
        type = t->scalar_type();
        return need(o, shape, type);
    }
    void dtype(PyObject *o, at::ScalarType &type) {
        if (!THPDtype_Check(o) || !act(reinterpret_cast<THPDtype *>(o)->scalar_type)) ok = false;
        else type = reinterpret_cast<THPDtype *>(o)->scalar_type;
    }
    at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type) const {
        return at::empty(shape, at::TensorOptions().dtype(type).device(dev));
    }
    // A call's workspace of this size (a negative status: the call itself will refuse, and needs none).
    at::Tensor workspace(int64_t size) const { return size > 0 ? fresh({size}, at::kByte) : at::Tensor(); }
};

int32_t code(at::ScalarType t) { return t == at::kBFloat16 ? MB_BF16 : MB_F32; }
const float *f(void *p) { return static_cast<const float *>(p); }
PyObject *wrap(at::Tensor t) { return THPVariable_Wrap(std::move(t)); }
PyObject *same(PyObject *o) { Py_INCREF(o); return o; }

// Runs the library call without the interpreter lock.
template <class F> int unlocked(F call) {
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = call();
    Py_END_ALLOW_THREADS
    return st;
}

// No C++ exception leaves an entry: torch's errors become the Python errors they are for
// torch's own functions (OutOfMemoryError among them).
template <class F> PyObject *guarded(F body) {
    HANDLE_TH_ERRORS
    return body();
    END_HANDLE_TH_ERRORS
}

#define ARGS(n) if (nargs != (n)) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); return nullptr; }
#define PLAIN_OR_NONE(c) if (!(c).ok) Py_RETURN_NONE

// h, u_t, delta_t, A, B_t, C_t, D, dt_bias, z_t, delta_softplus, out_dtype, out
PyObject *scan_step(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    ARGS(12)
    return guarded([&]() -> PyObject * {
        Call c;
        const at::Tensor *h = c.first(a[0], 3);
        const at::Tensor *u = c.ok ? plain(a[1]) : nullptr;
        if (!u || !Call::act(u->scalar_type())) Py_RETURN_NONE;
        const int64_t nb = h->size(0), dim = h->size(1), N = h->size(2);
        const auto act = u->scalar_type();
        void *hp = c.need(a[0], {nb, dim, N}, at::kFloat), *up = c.need(a[1], {nb, dim}, act);
        void *dp = c.need(a[2], {nb, dim}, act), *Ap = c.need(a[3], {dim, N}, at::kFloat);
        void *Bp = c.need(a[4], {nb, N}, act), *Cp = c.need(a[5], {nb, N}, act);
        void *Dp = c.maybe(a[6], {dim}, at::kFloat), *bp = c.maybe(a[7], {dim}, at::kFloat);
        void *zp = c.maybe(a[8], {nb, dim}, act);
        const int sp = PyObject_IsTrue(a[9]);
        at::ScalarType ot = at::kFloat;
        if (a[11] == Py_None) c.dtype(a[10], ot);
        void *op = c.given(a[11], {nb, dim}, ot);
        if (sp < 0) { PyErr_Clear(); c.ok = false; }
        PLAIN_OR_NONE(c);
        at::Tensor out;
        if (a[11] == Py_None) {
            out = c.fresh({nb, dim}, ot);
            op = out.data_ptr();
        }
        const int st = unlocked([&] {
            return scan_step_fn(nb, dim, N, code(act), code(ot), sp, up, dp, f(Ap), Bp, Cp, f(Dp), f(bp), zp,
                                static_cast<float *>(hp), op, c.stream);
        });
        if (st != MB_OK) return PyLong_FromLong(st);
        return a[11] == Py_None ? wrap(std::move(out)) : same(a[11]);
    });
}

// u, delta, A, B, C, D, dt_bias, z, h0, delta_softplus, out_dtype, return_last_state, out, h_last, positions, h_at,
// return_ckpt, ck
PyObject *scan_fwd(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    ARGS(18)
    return guarded([&]() -> PyObject * {
        Call c;
        const at::Tensor *u = c.first(a[0], 3);
        const at::Tensor *A = c.ok ? plain(a[2]) : nullptr;
        if (!A || A->dim() != 2 || !Call::act(u->scalar_type())) Py_RETURN_NONE;
        const int64_t nb = u->size(0), dim = u->size(1), L = u->size(2), N = A->size(1);
        const auto act = u->scalar_type();
        void *up = c.need(a[0], {nb, dim, L}, act), *dp = c.need(a[1], {nb, dim, L}, act);
        void *Ap = c.need(a[2], {dim, N}, at::kFloat);
        void *Bp = c.need(a[3], {nb, N, L}, act), *Cp = c.need(a[4], {nb, N, L}, act);
        void *Dp = c.maybe(a[5], {dim}, at::kFloat), *bp = c.maybe(a[6], {dim}, at::kFloat);
        void *zp = c.maybe(a[7], {nb, dim, L}, act), *h0 = c.maybe(a[8], {nb, dim, N}, at::kFloat);
        const int sp = PyObject_IsTrue(a[9]), want_last = PyObject_IsTrue(a[11]), want_ck = PyObject_IsTrue(a[16]);
        at::ScalarType ot = at::kFloat;
        if (a[12] == Py_None) c.dtype(a[10], ot);
        void *op = c.given(a[12], {nb, dim, L}, ot), *lp = c.maybe(a[13], {nb, dim, N}, at::kFloat);
        const bool has_pos = a[14] != Py_None, has_ck = want_ck > 0 || a[17] != Py_None;
        int64_t npos = 0;
        void *pp = nullptr, *hp = nullptr, *kp = nullptr;
        if (has_pos) {
            const at::Tensor *pos = c.ok ? plain(a[14]) : nullptr;
            if (!pos || pos->dim() != 2) Py_RETURN_NONE;
            npos = pos->size(0);
            pp = c.need(a[14], {npos, nb}, at::kInt);
            hp = c.maybe(a[15], {npos, nb, dim, N}, at::kFloat);
        } else if (a[15] != Py_None) {
            c.ok = false;
        }
        if (has_ck) kp = c.maybe(a[17], {L / 16, nb, dim, N}, at::kFloat);
        if (sp < 0 || want_last < 0 || want_ck < 0 || (has_ck && has_pos)) { PyErr_Clear(); c.ok = false; }
        PLAIN_OR_NONE(c);
        at::Tensor out, last, at_pos, ck;
        if (a[12] == Py_None) op = (out = c.fresh({nb, dim, L}, ot)).data_ptr();
        if (want_last && a[13] == Py_None) lp = (last = c.fresh({nb, dim, N}, at::kFloat)).data_ptr();
        if (has_pos && a[15] == Py_None) hp = (at_pos = c.fresh({npos, nb, dim, N}, at::kFloat)).data_ptr();
        if (has_ck && a[17] == Py_None) kp = (ck = c.fresh({L / 16, nb, dim, N}, at::kFloat)).data_ptr();
        const mb_scan_desc desc{nb, dim, L, N, code(act), code(ot), sp, 0};
        const int st = unlocked([&] {
            if (has_ck)
                return scan_fwd_ckpt_fn(&desc, up, dp, f(Ap), Bp, Cp, f(Dp), f(bp), zp, f(h0), op,
                                        static_cast<float *>(lp), static_cast<float *>(kp), c.stream);
            if (has_pos)
                return scan_fwd_states_fn(&desc, up, dp, f(Ap), Bp, Cp, f(Dp), f(bp), zp, f(h0), op,
                                          static_cast<float *>(lp), static_cast<const int32_t *>(pp), npos,
                                          static_cast<float *>(hp), c.stream);
            return scan_fwd_fn(&desc, up, dp, f(Ap), Bp, Cp, f(Dp), f(bp), zp, f(h0), op, static_cast<float *>(lp),
                               c.stream);
        });
        if (st != MB_OK) return PyLong_FromLong(st);
        PyObject *res[4];
        int n = 0;
        res[n++] = a[12] == Py_None ? wrap(std::move(out)) : same(a[12]);
        if (want_last || a[13] != Py_None) res[n++] = a[13] == Py_None ? wrap(std::move(last)) : same(a[13]);
        if (has_pos) res[n++] = a[15] == Py_None ? wrap(std::move(at_pos)) : same(a[15]);
        if (has_ck) res[n++] = a[17] == Py_None ? wrap(std::move(ck)) : same(a[17]);
        if (n == 1) return res[0];
        PyObject *t = PyTuple_New(n);
        for (int i = 0; i < n; ++i) PyTuple_SET_ITEM(t, i, res[i]);
        return t;
    });
}

// x, w, bias, state, apply_silu, out_dtype, return_state, out, state_out
PyObject *conv1d(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    ARGS(9)
    return guarded([&]() -> PyObject * {
        Call c;
        const at::Tensor *x = c.first(a[0], 3);
        const at::Tensor *w = c.ok ? plain(a[1]) : nullptr;
        if (!w || w->dim() != 2 || w->size(1) < 2 || !Call::act(x->scalar_type())) Py_RETURN_NONE;
        const int64_t nb = x->size(0), dim = x->size(1), L = x->size(2), K = w->size(1);
        const auto in = x->scalar_type();
        void *xp = c.need(a[0], {nb, dim, L}, in), *wp = c.need(a[1], {dim, K}, at::kFloat);
        void *bp = c.maybe(a[2], {dim}, at::kFloat), *sp = c.maybe(a[3], {nb, dim, K - 1}, at::kFloat);
        const int silu = PyObject_IsTrue(a[4]), want = PyObject_IsTrue(a[6]);
        at::ScalarType ot = in;
        if (a[7] == Py_None && a[5] != Py_None) c.dtype(a[5], ot);
        void *op = c.given(a[7], {nb, dim, L}, ot), *np = c.maybe(a[8], {nb, dim, K - 1}, at::kFloat);
        if (silu < 0 || want < 0 || K > INT32_MAX) { PyErr_Clear(); c.ok = false; }
        PLAIN_OR_NONE(c);
        at::Tensor out, next;
        if (a[7] == Py_None) op = (out = c.fresh({nb, dim, L}, ot)).data_ptr();
        if (want && a[8] == Py_None) np = (next = c.fresh({nb, dim, K - 1}, at::kFloat)).data_ptr();
        const mb_conv_desc desc{nb, dim, L, (int32_t)K, code(in), code(ot), silu, 0, 0};
        const int st = unlocked([&] {
            return conv1d_fwd_fn(&desc, xp, f(wp), f(bp), f(sp), op, static_cast<float *>(np), c.stream);
        });
        if (st != MB_OK) return PyLong_FromLong(st);
        PyObject *y = a[7] == Py_None ? wrap(std::move(out)) : same(a[7]);
        if (!want && a[8] == Py_None) return y;
        PyObject *t = PyTuple_New(2);
        PyTuple_SET_ITEM(t, 0, y);
        PyTuple_SET_ITEM(t, 1, a[8] == Py_None ? wrap(std::move(next)) : same(a[8]));
        return t;
    });
}

// state, x_t, w, bias, apply_silu, out_dtype, out
PyObject *conv1d_step(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    ARGS(7)
    return guarded([&]() -> PyObject * {
        Call c;
        const at::Tensor *x = c.first(a[1], 2);
        const at::Tensor *w = c.ok ? plain(a[2]) : nullptr;
        if (!w || w->dim() != 2 || w->size(1) < 2 || !Call::act(x->scalar_type())) Py_RETURN_NONE;
        const int64_t nb = x->size(0), dim = x->size(1), K = w->size(1);
        const auto in = x->scalar_type();
        void *xp = c.need(a[1], {nb, dim}, in), *wp = c.need(a[2], {dim, K}, at::kFloat);
        void *bp = c.maybe(a[3], {dim}, at::kFloat), *sp = c.need(a[0], {nb, dim, K - 1}, at::kFloat);
        const int silu = PyObject_IsTrue(a[4]);
        at::ScalarType ot = in;
        if (a[6] == Py_None && a[5] != Py_None) c.dtype(a[5], ot);
        void *op = c.given(a[6], {nb, dim}, ot);
        if (silu < 0 || K > INT32_MAX) { PyErr_Clear(); c.ok = false; }
        PLAIN_OR_NONE(c);
        at::Tensor out;
        if (a[6] == Py_None) op = (out = c.fresh({nb, dim}, ot)).data_ptr();
        const int st = unlocked([&] {
            return conv1d_step_fn(nb, dim, (int32_t)K, code(in), code(ot), silu, xp, f(wp), f(bp),
                                  static_cast<float *>(sp), op, c.stream);
        });
        if (st != MB_OK) return PyLong_FromLong(st);
        return a[6] == Py_None ? wrap(std::move(out)) : same(a[6]);
    });
}

// logits, draft, beta, return_ranks
PyObject *verify_rank(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    ARGS(4)
    return guarded([&]() -> PyObject * {
        if (!PyLong_CheckExact(a[2])) Py_RETURN_NONE;
        int over = 0;
        const long long beta = PyLong_AsLongLongAndOverflow(a[2], &over);
        if (over || beta < INT32_MIN || beta > INT32_MAX) Py_RETURN_NONE;
        Call c;
        const at::Tensor *lg = c.first(a[0], 3);
        if (!c.ok || !Call::act(lg->scalar_type())) Py_RETURN_NONE;
        const int64_t nb = lg->size(0), n = lg->size(1), V = lg->size(2);
        void *lp = c.need(a[0], {nb, n, V}, lg->scalar_type()), *dp = c.need(a[1], {nb, n}, at::kInt);
        const int want = PyObject_IsTrue(a[3]);
        if (want < 0) { PyErr_Clear(); c.ok = false; }
        PLAIN_OR_NONE(c);
        at::Tensor acc = c.fresh({nb}, at::kInt), pos = c.fresh({nb}, at::kInt), ranks;
        if (want) ranks = c.fresh({nb, n}, at::kInt);
        const int st = unlocked([&] {
            return verify_rank_fn(nb, n, V, code(lg->scalar_type()), (int32_t)beta, lp,
                                  static_cast<const int32_t *>(dp),
                                  want ? static_cast<int32_t *>(ranks.data_ptr()) : nullptr,
                                  static_cast<int32_t *>(acc.data_ptr()), static_cast<int32_t *>(pos.data_ptr()),
                                  c.stream);
        });
        if (st != MB_OK) return PyLong_FromLong(st);
        PyObject *t = PyTuple_New(want ? 3 : 2);
        PyTuple_SET_ITEM(t, 0, wrap(std::move(acc)));
        PyTuple_SET_ITEM(t, 1, wrap(std::move(pos)));
        if (want) PyTuple_SET_ITEM(t, 2, wrap(std::move(ranks)));
        return t;
    });
}

void *data(const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }

// A caller's tensor was written through its address: counted, so that autograd refuses a gradient for which it had saved it.
void was_written(PyObject *o) {
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// A real number as a float; ok becomes false where it is none.
float real(PyObject *o, bool &ok) {
    const double v = PyFloat_CheckExact(o) ? PyFloat_AS_DOUBLE(o) : PyLong_CheckExact(o) ? PyLong_AsDouble(o) : (ok = false, 0.0);
    if (PyErr_Occurred()) { PyErr_Clear(); ok = false; }
    return (float)v;
}

int token_code(at::ScalarType t) {
    return t == at::kByte ? MB_TOKEN_U8 : t == at::kInt ? MB_TOKEN_I32 : t == at::kLong ? MB_TOKEN_I64 : -1;
}

// tokens, weight, scale, out_dtype, out
PyObject *embedding_fwd(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    ARGS(5)
    return guarded([&]() -> PyObject * {
        Call c;
        const at::Tensor *w = c.first(a[1], 2);
        const at::Tensor *t = c.ok ? plain(a[0]) : nullptr;
        if (!t || !Call::act(w->scalar_type()) || token_code(t->scalar_type()) < 0) Py_RETURN_NONE;
        const int64_t V = w->size(0), d = w->size(1);
        c10::SmallVector<int64_t, 5> shape(t->sizes().begin(), t->sizes().end());
        void *tp = c.need(a[0], shape, t->scalar_type()), *wp = c.need(a[1], {V, d}, w->scalar_type());
        shape.push_back(d);
        const float scale = real(a[2], c.ok);
        at::ScalarType ot = w->scalar_type();
        if (a[4] == Py_None && a[3] != Py_None) c.dtype(a[3], ot);
        void *op = c.given(a[4], shape, ot);
        PLAIN_OR_NONE(c);
        at::Tensor out;
        if (a[4] == Py_None) op = (out = c.fresh(shape, ot)).data_ptr();
        const int st = unlocked([&] {
            return embedding_fwd_fn(t->numel(), V, d, token_code(t->scalar_type()), code(w->scalar_type()), code(ot), scale, tp,
                                    wp, op, c.stream);
        });
        if (st != MB_OK) return PyLong_FromLong(st);
        if (a[4] != Py_None) was_written(a[4]);
        return a[4] == Py_None ? wrap(std::move(out)) : same(a[4]);
    });
}

// tokens, dy, vocab, scale, out_dtype, out
PyObject *embedding_bwd(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    ARGS(6)
    return guarded([&]() -> PyObject * {
        if (!PyLong_CheckExact(a[2])) Py_RETURN_NONE;
        int over = 0;
        const long long V = PyLong_AsLongLongAndOverflow(a[2], &over);
        if (over || V < 0) Py_RETURN_NONE;
        Call c;
        const at::Tensor *t = plain(a[0]);
        if (!t || token_code(t->scalar_type()) < 0) Py_RETURN_NONE;
        const at::Tensor *dy = c.first(a[1], t->dim() + 1);
        if (!c.ok || !Call::act(dy->scalar_type())) Py_RETURN_NONE;
        const int64_t d = dy->size(-1);
        c10::SmallVector<int64_t, 5> shape(t->sizes().begin(), t->sizes().end());
        void *tp = c.need(a[0], shape, t->scalar_type());
        shape.push_back(d);
        void *yp = c.need(a[1], shape, dy->scalar_type());
        const float scale = real(a[3], c.ok);
        at::ScalarType ot = at::kFloat;
        if (a[5] == Py_None) c.dtype(a[4], ot);
        void *op = c.given(a[5], {V, d}, ot);
        PLAIN_OR_NONE(c);
        at::Tensor out, ws = c.workspace(embedding_bwd_workspace_fn(t->numel(), V, d));
        if (a[5] == Py_None) op = (out = c.fresh({V, d}, ot)).data_ptr();
        const int st = unlocked([&] {
            return embedding_bwd_fn(t->numel(), V, d, token_code(t->scalar_type()), code(dy->scalar_type()), code(ot), scale, tp,
                                    yp, op, data(ws), c.stream);
        });
        if (st != MB_OK) return PyLong_FromLong(st);
        if (a[5] != Py_None) was_written(a[5]);
        return a[5] == Py_None ? wrap(std::move(out)) : same(a[5]);
    });
}

// x, w, dy, bias, state, dstate_out, apply_silu: dx, dw, dbias, dstate
PyObject *conv1d_bwd(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    ARGS(7)
    return guarded([&]() -> PyObject * {
        Call c;
        const at::Tensor *x = c.first(a[0], 3);
        const at::Tensor *w = c.ok ? plain(a[1]) : nullptr, *dy = c.ok ? plain(a[2]) : nullptr;
        if (!w || !dy || w->dim() != 2 || w->size(1) < 2 || !Call::act(x->scalar_type()) || !Call::act(dy->scalar_type()))
            Py_RETURN_NONE;
        const int64_t nb = x->size(0), dim = x->size(1), L = x->size(2), K = w->size(1);
        const auto in = x->scalar_type(), ot = dy->scalar_type();
        void *xp = c.need(a[0], {nb, dim, L}, in), *wp = c.need(a[1], {dim, K}, at::kFloat);
        void *yp = c.need(a[2], {nb, dim, L}, ot), *bp = c.maybe(a[3], {dim}, at::kFloat);
        void *sp = c.maybe(a[4], {nb, dim, K - 1}, at::kFloat), *dp = c.maybe(a[5], {nb, dim, K - 1}, at::kFloat);
        const int silu = PyObject_IsTrue(a[6]);
        if (silu < 0 || K > INT32_MAX) { PyErr_Clear(); c.ok = false; }
        PLAIN_OR_NONE(c);
        const mb_conv_desc desc{nb, dim, L, (int32_t)K, code(in), code(ot), silu, 0, 0};
        at::Tensor dx = c.fresh({nb, dim, L}, ot), dw = c.fresh({dim, K}, at::kFloat), db;
        at::Tensor ds = c.fresh({nb, dim, K - 1}, at::kFloat), ws = c.workspace(conv1d_bwd_workspace_fn(&desc));
        if (bp) db = c.fresh({dim}, at::kFloat);
        const int st = unlocked([&] {
            return conv1d_bwd_fn(&desc, xp, f(wp), f(bp), f(sp), yp, f(dp), dx.data_ptr(), static_cast<float *>(dw.data_ptr()),
                                 static_cast<float *>(data(db)), static_cast<float *>(ds.data_ptr()), data(ws), c.stream);
        });
        if (st != MB_OK) return PyLong_FromLong(st);
        PyObject *t = PyTuple_New(4);
        PyTuple_SET_ITEM(t, 0, wrap(std::move(dx)));
        PyTuple_SET_ITEM(t, 1, wrap(std::move(dw)));
        PyTuple_SET_ITEM(t, 2, bp ? wrap(std::move(db)) : same(Py_None));
        PyTuple_SET_ITEM(t, 3, wrap(std::move(ds)));
        return t;
    });
}

// A list or tuple of dense fp32 and bf16 tensors on one device, as the library takes it.  It holds them: another thread may
// change the list while the library is called without the interpreter lock.
struct TensorList {
    std::vector<PyObject *> held;
    std::vector<const void *> at;
    std::vector<int64_t> sizes;
    std::vector<int32_t> types;
    static bool is_list(PyObject *o) { return PyList_CheckExact(o) || PyTuple_CheckExact(o); }
    // `like`: the tensors' shapes and types have to be that list's
    TensorList(Call &c, PyObject *o, PyObject *like = nullptr) {
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(o);
        PyObject **item = PySequence_Fast_ITEMS(o), **other = like ? PySequence_Fast_ITEMS(like) : nullptr;
        if (like && PySequence_Fast_GET_SIZE(like) != n) c.ok = false;
        held.reserve(n);
        at.reserve(n);
        if (!like) { sizes.reserve(n); types.reserve(n); }
        for (Py_ssize_t i = 0; c.ok && i < n; ++i) {
            const at::Tensor *t = plain(item[i]);
            if (t && i == 0 && !like) t = c.first(item[i], t->dim());
            if (!t || !c.ok || !Call::act(t->scalar_type()) || t->device() != c.dev || !t->is_contiguous()) { c.ok = false; return; }
            if (like) {
                const at::Tensor &g = THPVariable_Unpack(other[i]);
                if (t->scalar_type() != g.scalar_type() || t->sizes() != g.sizes()) { c.ok = false; return; }
            } else {
                sizes.push_back(t->numel());
                types.push_back(code(t->scalar_type()));
            }
            held.push_back(same(item[i]));
            at.push_back(t->data_ptr());
        }
    }
    TensorList(const TensorList &) = delete;
    ~TensorList() {
        for (PyObject *o : held) Py_DECREF(o);
    }
};

// grads
PyObject *grad_norm(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    ARGS(1)
    return guarded([&]() -> PyObject * {
        if (!TensorList::is_list(a[0]) || PySequence_Fast_GET_SIZE(a[0]) == 0) Py_RETURN_NONE;
        Call c;
        const TensorList g(c, a[0]);
        PLAIN_OR_NONE(c);
        const int64_t n = (int64_t)g.at.size();
        at::Tensor norm = c.fresh({}, at::kFloat), ws = c.workspace(grad_norm_workspace_fn(n));
        const int st = unlocked([&] {
            return grad_norm_fn(n, g.at.data(), g.sizes.data(), g.types.data(), static_cast<float *>(norm.data_ptr()), data(ws),
                                c.stream);
        });
        return st != MB_OK ? PyLong_FromLong(st) : wrap(std::move(norm));
    });
}

// grads, max_norm, eps, out
PyObject *clip_grad_norm(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    ARGS(4)
    return guarded([&]() -> PyObject * {
        if (!TensorList::is_list(a[0]) || PySequence_Fast_GET_SIZE(a[0]) == 0) Py_RETURN_NONE;
        if (a[3] != Py_None && !TensorList::is_list(a[3])) Py_RETURN_NONE;
        Call c;
        const TensorList g(c, a[0]);
        const float max_norm = real(a[1], c.ok), eps = real(a[2], c.ok);
        PLAIN_OR_NONE(c);
        // what is written are gradients, not the parameters that torch's function of this name takes
        std::optional<TensorList> given;
        if (a[3] != Py_None) given.emplace(c, a[3], a[0]);
        PLAIN_OR_NONE(c);
        const TensorList &written = given ? *given : g;
        std::vector<void *> out;
        for (PyObject *o : written.held)
            if (THPVariable_Unpack(o).requires_grad()) Py_RETURN_NONE;
        for (size_t i = 0; given && i < written.at.size(); ++i) out.push_back(const_cast<void *>(written.at[i]));
        const int64_t n = (int64_t)g.at.size();
        at::Tensor norm = c.fresh({}, at::kFloat), ws = c.workspace(grad_norm_workspace_fn(n));
        const int st = unlocked([&] {
            return clip_grad_norm_fn(n, g.at.data(), given ? out.data() : nullptr, g.sizes.data(), g.types.data(),
                                     max_norm, eps, static_cast<float *>(norm.data_ptr()), data(ws), c.stream);
        });
        if (st != MB_OK) return PyLong_FromLong(st);
        for (PyObject *o : written.held) was_written(o);
        return wrap(std::move(norm));
    });
}

// logits, draft, uniform, noise, draft_logits, lengths, temperature, return_probs
PyObject *verify_sample(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    ARGS(8)
    return guarded([&]() -> PyObject * {
        Call c;
        const at::Tensor *lg = c.first(a[0], 3);
        if (!c.ok || !Call::act(lg->scalar_type()) || lg->size(1) < 1) Py_RETURN_NONE;
        const int64_t nb = lg->size(0), n = lg->size(1) - 1, V = lg->size(2);
        const auto act = lg->scalar_type();
        void *lp = c.need(a[0], {nb, n + 1, V}, act), *dp = c.need(a[1], {nb, n}, at::kInt);
        void *up = c.need(a[2], {nb, n}, at::kFloat), *np = c.need(a[3], {nb, V}, at::kFloat);
        void *qp = c.maybe(a[4], {nb, n, V}, act), *sp = c.maybe(a[5], {nb}, at::kInt);
        const float temperature = real(a[6], c.ok);
        const int want = PyObject_IsTrue(a[7]);
        if (want < 0) { PyErr_Clear(); c.ok = false; }
        PLAIN_OR_NONE(c);
        at::Tensor acc = c.fresh({nb}, at::kInt), pos = c.fresh({nb}, at::kInt), next = c.fresh({nb}, at::kInt), probs;
        if (want) probs = c.fresh({nb, n}, at::kFloat);
        at::Tensor ws = c.workspace(verify_sample_workspace_fn(nb, n, V));
        const int st = unlocked([&] {
            return verify_sample_fn(nb, n, V, code(act), temperature, lp, qp, static_cast<const int32_t *>(dp),
                                    static_cast<const int32_t *>(sp), f(up), f(np), static_cast<int32_t *>(acc.data_ptr()),
                                    static_cast<int32_t *>(pos.data_ptr()), static_cast<int32_t *>(next.data_ptr()),
                                    static_cast<float *>(data(probs)), data(ws), c.stream);
        });
        if (st != MB_OK) return PyLong_FromLong(st);
        PyObject *t = PyTuple_New(want ? 4 : 3);
        PyTuple_SET_ITEM(t, 0, wrap(std::move(acc)));
        PyTuple_SET_ITEM(t, 1, wrap(std::move(pos)));
        PyTuple_SET_ITEM(t, 2, wrap(std::move(next)));
        if (want) PyTuple_SET_ITEM(t, 3, wrap(std::move(probs)));
        return t;
    });
}

constexpr auto kFp8 = at::kFloat8_e4m3fn;
int64_t blocks(int64_t n) { return (n + 127) / 128; }
using Shape = c10::SmallVector<int64_t, 5>;

PyObject *tuple(std::initializer_list<PyObject *> items) {
    PyObject *t = PyTuple_New((Py_ssize_t)items.size());
    Py_ssize_t i = 0;
    for (PyObject *o : items) PyTuple_SET_ITEM(t, i++, o);
    return t;
}

// x, weight, residual, eps, out_dtype, return_rstd, out, residual_out
PyObject *rms_norm_fwd(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    ARGS(8)
    return guarded([&]() -> PyObject * {
        Call c;
        const at::Tensor *x = plain(a[0]);
        if (!x || x->dim() < 1) Py_RETURN_NONE;
        x = c.first(a[0], x->dim());
        const at::Tensor *res = c.ok && a[2] != Py_None ? plain(a[2]) : nullptr;
        if (!c.ok || !Call::act(x->scalar_type()) || (a[2] != Py_None && (!res || !Call::act(res->scalar_type())))) Py_RETURN_NONE;
        const Shape shape(x->sizes().begin(), x->sizes().end());
        const int64_t d = shape.back();
        if (d == 0) Py_RETURN_NONE;
        const auto rt = res ? res->scalar_type() : at::kFloat;
        void *xp = c.need(a[0], shape, x->scalar_type()), *wp = c.maybe(a[1], {d}, at::kFloat), *rp = c.maybe(a[2], shape, rt);
        const float eps = real(a[3], c.ok);
        at::ScalarType ot = x->scalar_type();
        if (a[6] == Py_None && a[4] != Py_None) c.dtype(a[4], ot);
        void *op = c.given(a[6], shape, ot), *hp = c.maybe(a[7], shape, rt);
        const int want = PyObject_IsTrue(a[5]);
        if (want < 0 || (!res && hp)) { PyErr_Clear(); c.ok = false; }
        PLAIN_OR_NONE(c);
        at::Tensor out, h, rstd;
        if (a[6] == Py_None) op = (out = c.fresh(shape, ot)).data_ptr();
        if (res && a[7] == Py_None) hp = (h = c.fresh(shape, rt)).data_ptr();
        if (want) rstd = c.fresh(at::IntArrayRef(shape.data(), shape.size() - 1), at::kFloat);
        const int st = unlocked([&] {
            return rms_norm_fwd_fn(x->numel() / d, d, code(x->scalar_type()), code(rt), code(ot), eps, xp, f(wp), rp, op, nullptr, hp,
                                   static_cast<float *>(data(rstd)), c.stream);
        });
        if (st != MB_OK) return PyLong_FromLong(st);
        if (a[6] != Py_None) was_written(a[6]);
        if (a[7] != Py_None) was_written(a[7]);
        PyObject *y = a[6] == Py_None ? wrap(std::move(out)) : same(a[6]);
        if (!res) return want ? tuple({y, wrap(std::move(rstd))}) : y;
        PyObject *k = a[7] == Py_None ? wrap(std::move(h)) : same(a[7]);
        return want ? tuple({y, k, wrap(std::move(rstd))}) : tuple({y, k});
    });
}

// x, weight, residual, eps, residual_out
PyObject *rms_norm_fp8(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    ARGS(5)
    return guarded([&]() -> PyObject * {
        Call c;
        const at::Tensor *x = plain(a[0]);
        if (!x || x->dim() < 1) Py_RETURN_NONE;
        x = c.first(a[0], x->dim());
        const at::Tensor *res = c.ok && a[2] != Py_None ? plain(a[2]) : nullptr;
        if (!c.ok || !Call::act(x->scalar_type()) || (a[2] != Py_None && (!res || !Call::act(res->scalar_type())))) Py_RETURN_NONE;
        Shape shape(x->sizes().begin(), x->sizes().end());
        const int64_t d = shape.back();
        if (d == 0) Py_RETURN_NONE;
        const auto rt = res ? res->scalar_type() : at::kFloat;
        void *xp = c.need(a[0], shape, x->scalar_type()), *wp = c.maybe(a[1], {d}, at::kFloat), *rp = c.maybe(a[2], shape, rt);
        const float eps = real(a[3], c.ok);
        void *hp = c.maybe(a[4], shape, rt);
        if (!res && hp) c.ok = false;
        PLAIN_OR_NONE(c);
        at::Tensor q = c.fresh(shape, kFp8), h;
        if (res && a[4] == Py_None) hp = (h = c.fresh(shape, rt)).data_ptr();
        shape.back() = blocks(d);
        at::Tensor scale = c.fresh(shape, at::kFloat);
        const int st = unlocked([&] {
            return rms_norm_fwd_fn(x->numel() / d, d, code(x->scalar_type()), code(rt), MB_FP8, eps, xp, f(wp), rp, q.data_ptr(),
                                   static_cast<float *>(scale.data_ptr()), hp, nullptr, c.stream);
        });
        if (st != MB_OK) return PyLong_FromLong(st);
        if (a[4] != Py_None) was_written(a[4]);
        PyObject *qo = wrap(std::move(q)), *so = wrap(std::move(scale));
        return res ? tuple({qo, so, a[4] == Py_None ? wrap(std::move(h)) : same(a[4])}) : tuple({qo, so});
    });
}

// dy, h, rstd, weight, dh, dx_dtype: dx, dweight, dresidual
PyObject *rms_norm_bwd(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    ARGS(6)
    return guarded([&]() -> PyObject * {
        Call c;
        const at::Tensor *h = plain(a[1]), *dy = plain(a[0]);
        if (!h || !dy || h->dim() < 1) Py_RETURN_NONE;
        h = c.first(a[1], h->dim());
        if (!c.ok || !Call::act(h->scalar_type()) || !Call::act(dy->scalar_type())) Py_RETURN_NONE;
        const Shape shape(h->sizes().begin(), h->sizes().end());
        const int64_t d = shape.back();
        if (d == 0) Py_RETURN_NONE;
        const auto ht = h->scalar_type();
        void *hp = c.need(a[1], shape, ht), *yp = c.need(a[0], shape, dy->scalar_type());
        void *sp = c.need(a[2], at::IntArrayRef(shape.data(), shape.size() - 1), at::kFloat);
        void *wp = c.maybe(a[3], {d}, at::kFloat), *dp = c.maybe(a[4], shape, ht);
        at::ScalarType xt = dy->scalar_type();
        if (a[5] != Py_None) c.dtype(a[5], xt);
        PLAIN_OR_NONE(c);
        const int64_t rows = h->numel() / d;
        at::Tensor dx = c.fresh(shape, xt), dw, dres, ws;
        if (wp) {
            dw = c.fresh({d}, at::kFloat);
            ws = c.workspace(rms_norm_bwd_workspace_fn(rows, d));
        }
        const bool apart = dp && ht != xt;
        if (apart) dres = c.fresh(shape, ht);
        const int st = unlocked([&] {
            return rms_norm_bwd_fn(rows, d, code(dy->scalar_type()), code(ht), code(xt), yp, hp, f(sp), f(wp), dp, dx.data_ptr(),
                                   data(dres), static_cast<float *>(data(dw)), data(ws), c.stream);
        });
        if (st != MB_OK) return PyLong_FromLong(st);
        PyObject *x = wrap(std::move(dx)), *w = wp ? wrap(std::move(dw)) : same(Py_None);
        return tuple({x, w, !dp ? same(Py_None) : apart ? wrap(std::move(dres)) : same(x)});
    });
}

// x, tile, transpose
PyObject *quantize_fp8(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    ARGS(3)
    return guarded([&]() -> PyObject * {
        Call c;
        const at::Tensor *x = plain(a[0]);
        if (!x || x->dim() < 2) Py_RETURN_NONE;
        x = c.first(a[0], x->dim());
        if (!c.ok || !Call::act(x->scalar_type())) Py_RETURN_NONE;
        Shape shape(x->sizes().begin(), x->sizes().end());
        void *xp = c.need(a[0], shape, x->scalar_type());
        const int tile = PyObject_IsTrue(a[1]), transpose = PyObject_IsTrue(a[2]);
        if (tile < 0 || transpose < 0) { PyErr_Clear(); c.ok = false; }
        PLAIN_OR_NONE(c);
        const size_t n = shape.size();
        const int64_t rows = shape[n - 2], cols = shape[n - 1];
        int64_t batch = 1;
        for (size_t i = 0; i + 2 < n; ++i) batch *= shape[i];
        if (transpose) std::swap(shape[n - 2], shape[n - 1]);
        at::Tensor q = c.fresh(shape, kFp8);
        if (tile) shape[n - 2] = blocks(shape[n - 2]);
        shape[n - 1] = blocks(shape[n - 1]);
        at::Tensor scale = c.fresh(shape, at::kFloat);
        const int st = unlocked([&] {
            return quantize_fp8_fn(batch, rows, cols, code(x->scalar_type()), tile, transpose, xp, q.data_ptr(),
                                   static_cast<float *>(scale.data_ptr()), c.stream);
        });
        if (st != MB_OK) return PyLong_FromLong(st);
        PyObject *qo = wrap(std::move(q));
        return tuple({qo, wrap(std::move(scale))});
    });
}

// a, a_scale, b, b_scale, out_dtype, out
PyObject *matmul_fp8(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    ARGS(6)
    return guarded([&]() -> PyObject * {
        Call c;
        const at::Tensor *t[2] = {plain(a[0]), plain(a[2])};
        if (!t[0] || !t[1] || !c.first(a[0], t[0]->dim())) Py_RETURN_NONE;
        void *at[2], *scales[2];
        bool tile[2];
        int64_t batch = -1;
        for (int i = 0; i < 2; ++i) {
            const int64_t n = t[i]->dim();
            if (n != 2 && n != 3) Py_RETURN_NONE;
            if (n == 3) {
                if (batch >= 0 && batch != t[i]->size(0)) Py_RETURN_NONE;
                batch = t[i]->size(0);
            }
            const at::Tensor *s = plain(a[2 * i + 1]);
            if (!s || s->dim() != n) Py_RETURN_NONE;
            Shape shape(t[i]->sizes().begin(), t[i]->sizes().end());
            at[i] = c.need(a[2 * i], shape, kFp8);
            const int64_t rows = shape[n - 2];
            shape[n - 1] = blocks(shape[n - 1]);
            tile[i] = s->size(n - 2) != rows;
            if (tile[i]) shape[n - 2] = blocks(rows);
            scales[i] = c.need(a[2 * i + 1], shape, at::kFloat);
        }
        const int64_t m = t[0]->size(-2), n = t[1]->size(-2), k = t[0]->size(-1);
        if (t[1]->size(-1) != k) Py_RETURN_NONE;
        Shape shape;
        if (batch >= 0) shape.push_back(batch);
        shape.push_back(m);
        shape.push_back(n);
        at::ScalarType ot = at::kBFloat16;
        if (a[5] == Py_None) c.dtype(a[4], ot);
        void *op = c.given(a[5], shape, ot);
        PLAIN_OR_NONE(c);
        at::Tensor out;
        if (a[5] == Py_None) op = (out = c.fresh(shape, ot)).data_ptr();
        const mb_matmul_desc desc{batch < 0 ? 1 : batch, m, n, k, t[0]->dim() == 3, t[1]->dim() == 3, tile[0], tile[1], code(ot), 0};
        const int st = unlocked([&] { return matmul_fp8_fn(&desc, at[0], f(scales[0]), at[1], f(scales[1]), op, c.stream); });
        if (st != MB_OK) return PyLong_FromLong(st);
        if (a[5] != Py_None) was_written(a[5]);
        return a[5] == Py_None ? wrap(std::move(out)) : same(a[5]);
    });
}

// logits, noise, temperature, top_k, top_p, min_p, return_prob
PyObject *sample(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    ARGS(7)
    return guarded([&]() -> PyObject * {
        Call c;
        const at::Tensor *lg = c.first(a[0], 2);
        if (!c.ok || !Call::act(lg->scalar_type())) Py_RETURN_NONE;
        const int64_t nb = lg->size(0), V = lg->size(1);
        void *lp = c.need(a[0], {nb, V}, lg->scalar_type()), *np = c.need(a[1], {nb, V}, at::kFloat);
        // each setting a number for all, or a tensor of one for each
        float one[4] = {1.0f, 0.0f, 1.0f, 0.0f};
        void *each[4] = {};
        int32_t top_k = 0;
        for (int i = 0; i < 4; ++i) {
            PyObject *o = a[2 + i];
            if (THPVariable_Check(o)) {
                each[i] = c.need(o, {nb}, i == 1 ? at::kInt : at::kFloat);
            } else if (i == 1) {
                int over = 0;
                if (!PyLong_CheckExact(o)) Py_RETURN_NONE;
                const long long k = PyLong_AsLongLongAndOverflow(o, &over);
                if (over || k < 0 || k > INT32_MAX) Py_RETURN_NONE;
                top_k = (int32_t)k;
            } else {
                one[i] = real(o, c.ok);
            }
        }
        const int want = PyObject_IsTrue(a[6]);
        if (want < 0) { PyErr_Clear(); c.ok = false; }
        PLAIN_OR_NONE(c);
        at::Tensor token = c.fresh({nb}, at::kInt), prob;
        if (want) prob = c.fresh({nb}, at::kFloat);
        const int st = unlocked([&] {
            return sample_fn(nb, V, code(lg->scalar_type()), one[0], top_k, one[2], one[3], f(each[0]), static_cast<const int32_t *>(each[1]),
                             f(each[2]), f(each[3]), lp, f(np), static_cast<int32_t *>(token.data_ptr()),
                             static_cast<float *>(data(prob)), c.stream);
        });
        if (st != MB_OK) return PyLong_FromLong(st);
        PyObject *t = wrap(std::move(token));
        return want ? tuple({t, wrap(std::move(prob))}) : t;
    });
}

// setup(function addresses in the order below, current_device, raw_stream, Parameter)
PyObject *setup(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    constexpr int kFunctions = 23;
    ARGS(kFunctions + 3)
    void *at[kFunctions];
    for (int i = 0; i < kFunctions; ++i) {
        at[i] = PyLong_AsVoidPtr(a[i]);
        if (!at[i]) return PyErr_Occurred() ? nullptr : (PyErr_SetString(PyExc_ValueError, "null address"), nullptr);
    }
    int k = 0;
    auto take = [&](auto &fn) { fn = reinterpret_cast<std::decay_t<decltype(fn)>>(at[k++]); };
    take(scan_fwd_fn);
    take(scan_fwd_states_fn);
    take(scan_fwd_ckpt_fn);
    take(scan_step_fn);
    take(conv1d_fwd_fn);
    take(conv1d_step_fn);
    take(verify_rank_fn);
    take(embedding_fwd_fn);
    take(embedding_bwd_fn);
    take(embedding_bwd_workspace_fn);
    take(conv1d_bwd_fn);
    take(conv1d_bwd_workspace_fn);
    take(grad_norm_fn);
    take(grad_norm_workspace_fn);
    take(clip_grad_norm_fn);
    take(verify_sample_fn);
    take(verify_sample_workspace_fn);
    take(rms_norm_fwd_fn);
    take(rms_norm_bwd_fn);
    take(rms_norm_bwd_workspace_fn);
    take(quantize_fp8_fn);
    take(matmul_fp8_fn);
    take(sample_fn);
    current_device = same(a[k]);
    raw_stream = same(a[k + 1]);
    parameter_type = same(a[k + 2]);
    Py_RETURN_NONE;
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(setup),  METHOD(scan_step),   METHOD(scan_fwd),
                         METHOD(conv1d), METHOD(conv1d_step), METHOD(verify_rank),
                         METHOD(embedding_fwd), METHOD(embedding_bwd), METHOD(conv1d_bwd),
                         METHOD(grad_norm), METHOD(clip_grad_norm), METHOD(verify_sample),
                         METHOD(rms_norm_fwd), METHOD(rms_norm_fp8), METHOD(rms_norm_bwd),
                         METHOD(quantize_fp8), METHOD(matmul_fp8), METHOD(sample),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall() {
    PyObject *m = PyModule_Create(&module);
    // the torch whose object layouts this was compiled against: the binding uses no other
    if (m && PyModule_AddStringConstant(m, "torch_version", MB_TORCH_VERSION) != 0) Py_CLEAR(m);
    return m;
}
