// The Python calls of a layer's step - forward, input gradient, weight gradient, both gradients, and the block operators - without the interpreter:
// the checks of binding.py, the output allocation and the C call in one native function.  A call through binding.py is some
// thirty Python-level calls, about half of what a small call took from the host (B1 C256 L4096 K64 fp32 forward 7.0 us a call,
// 4.5-5.1 here, its kernel 4.7; B4 C64 L1024 K16, three calls 22.0 us, 12.7-14.8 here, its kernels 3.2 each).
//
// A function here does the call or returns None: anything but plain strided device tensors of a supported type, laid out as the
// library takes them, on the current device (subclasses, wrappers of transforms, active torch function or dispatch modes, traces,
// arguments that are not exact ints, mismatched shapes) is left to binding.py, whose checks and messages are the only ones.
// A status other than 0 is raised by binding.py's own exception.
//
// Built for one PyTorch and one Python (DWCONV_BUILT_FOR names them): it reads their objects by its headers' layouts.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>

#include <climits>
#include <cmath>
#include <vector>

#include "../../include/dwconv_block.h"

namespace {

typedef int (*CorrFn)(const void *, const void *, void *, int, int, int, int, int, int, void *);
typedef int (*WeightFn)(const void *, const void *, void *, void *, size_t, int, int, int, int, int, int, void *);
typedef int (*BothFn)(const void *, const void *, const void *, void *, void *, void *, size_t, int, int, int, int, int, int, void *);

CorrFn fn_fwd, fn_bwd_input;
WeightFn fn_bwd_weight;
BothFn fn_bwd;
PyObject *current_device, *raw_stream, *check;       // binding.py's queries and its check of a status

// A tensor the library can take as it is, or nullptr.
const at::Tensor *plain(PyObject *o, int64_t dim, long device)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || t.layout() != at::kStrided || !t.is_cuda() || t.get_device() != device) return nullptr;
    // (nothing but a device tensor under autograd and autocast: no wrapper of a transform, no lazy conjugate or negative)
    if ((t.key_set() - c10::autograd_dispatch_keyset_with_ADInplaceOrView - c10::autocast_dispatch_keyset).highestPriorityTypeId() !=
        c10::DispatchKey::CUDA)
        return nullptr;
    if ((dim >= 0 && t.dim() != dim) || !t.is_contiguous()) return nullptr;
    return &t;
}

int dtype_code(const at::Tensor &t)
{
    return t.scalar_type() == at::kFloat ? 0 : t.scalar_type() == at::kBFloat16 ? 1 : -1;
}

bool exact_int(PyObject *o, int &v)
{
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    const long l = PyLong_AsLongAndOverflow(o, &overflow);
    if (overflow || l < INT_MIN || l > INT_MAX) return false;
    v = (int)l;
    return true;
}

struct Call {
    long device = -1;
    void *stream = nullptr;
    // False (no error set): binding.py's turn; with an error set: the error.
    bool begin(PyObject *first)
    {
        // (the queries are there to be asked once a device tensor is)
        if (!THPVariable_CheckExact(first) || !THPVariable_Unpack(first).is_cuda()) return false;
        if (at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set() || torch::jit::tracer::isTracing())
            return false;
        PyObject *d = PyObject_CallNoArgs(current_device);
        if (!d) return false;
        device = PyLong_AsLong(d);
        PyObject *s = PyErr_Occurred() ? nullptr : PyObject_CallOneArg(raw_stream, d);
        Py_DECREF(d);
        if (!s) return false;
        stream = PyLong_AsVoidPtr(s);
        Py_DECREF(s);
        return !PyErr_Occurred();
    }
    bool bad() const { return PyErr_Occurred() != nullptr; }
};

// Without the interpreter's lock while it lives: around allocation and launch, either of which may wait (for memory, for a place in the
// queue, for code to be loaded) while other threads, or a host function the queue waits for, want the lock.
struct Unlocked {
    PyThreadState *state = PyEval_SaveThread();
    Unlocked() = default;
    Unlocked(const Unlocked &) = delete;
    Unlocked &operator=(const Unlocked &) = delete;
    ~Unlocked() { PyEval_RestoreThread(state); }
};

PyObject *decline() { Py_RETURN_NONE; }
bool raised(int status)
{
    if (status == 0) return false;
    PyObject *s = PyLong_FromLong(status), *r = s ? PyObject_CallOneArg(check, s) : nullptr;
    Py_XDECREF(s);
    Py_XDECREF(r);
    return true;
}

struct Dims {
    int B, C, L, K;
};
bool dims_of(const at::Tensor &x, int64_t K, Dims &d)
{
    if (x.size(0) > INT_MAX || x.size(1) > INT_MAX || x.size(2) > INT_MAX || K > INT_MAX) return false;
    d = Dims{(int)x.size(0), (int)x.size(1), (int)x.size(2), (int)K};
    return true;
}

// (in, filter, pad_left, out or None) -> out
PyObject *corr(CorrFn fn, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Call call;
    int pad;
    Dims d;
    if (n != 4 || !exact_int(a[2], pad)) return decline();
    if (!call.begin(a[0])) return call.bad() ? nullptr : decline();
    const at::Tensor *x = plain(a[0], 3, call.device), *w = plain(a[1], 2, call.device);
    if (!x || !w || w->scalar_type() != x->scalar_type() || w->size(0) != x->size(1) || !dims_of(*x, w->size(1), d)) return decline();
    const int code = dtype_code(*x);
    if (code < 0) return decline();
    const at::Tensor *out = nullptr;
    if (a[3] != Py_None) {
        out = plain(a[3], 3, call.device);
        if (!out || out->sizes() != x->sizes() || out->scalar_type() != x->scalar_type()) return decline();
    }
    const void *px = x->const_data_ptr(), *pw = w->const_data_ptr();
    void *py = out ? out->mutable_data_ptr() : nullptr;
    at::Tensor made;
    int status;
    {
        Unlocked unlocked;
        if (!out) {
            made = at::empty_like(*x);
            py = made.mutable_data_ptr();
        }
        status = fn(px, pw, py, d.B, d.C, d.L, d.K, pad, code, call.stream);
    }
    if (raised(status)) return nullptr;
    if (a[3] == Py_None) return THPVariable_Wrap(std::move(made));
    Py_INCREF(a[3]);
    return a[3];
    END_HANDLE_TH_ERRORS
}
PyObject *fwd(PyObject *, PyObject *const *a, Py_ssize_t n) { return corr(fn_fwd, a, n); }
PyObject *bwd_input(PyObject *, PyObject *const *a, Py_ssize_t n) { return corr(fn_bwd_input, a, n); }

// A [C, K] output of the caller's.
const at::Tensor *weight_out(PyObject *o, const at::Tensor &x, const Dims &d, long device)
{
    const at::Tensor *dw = plain(o, 2, device);
    return dw && dw->size(0) == d.C && dw->size(1) == d.K && dw->scalar_type() == x.scalar_type() ? dw : nullptr;
}

// (x, dy, K, pad_left, workspace, out or None) -> out
PyObject *bwd_weight(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Call call;
    int K, pad;
    Dims d;
    if (n != 6 || a[4] == Py_None || !exact_int(a[2], K) || K < 1 || !exact_int(a[3], pad)) return decline();
    if (!call.begin(a[0])) return call.bad() ? nullptr : decline();
    const at::Tensor *x = plain(a[0], 3, call.device), *dy = plain(a[1], 3, call.device), *ws = plain(a[4], -1, call.device);
    if (!x || !dy || !ws || dy->sizes() != x->sizes() || dy->scalar_type() != x->scalar_type() || !dims_of(*x, K, d)) return decline();
    const int code = dtype_code(*x);
    if (code < 0) return decline();
    const at::Tensor *out = nullptr;
    if (a[5] != Py_None && !(out = weight_out(a[5], *x, d, call.device))) return decline();
    const void *px = x->const_data_ptr(), *pdy = dy->const_data_ptr();
    void *pdw = out ? out->mutable_data_ptr() : nullptr, *pws = ws->mutable_data_ptr();
    const size_t bytes = ws->nbytes();
    at::Tensor made;
    int status;
    {
        Unlocked unlocked;
        if (!out) {
            made = at::empty({d.C, d.K}, x->options());
            pdw = made.mutable_data_ptr();
        }
        status = fn_bwd_weight(px, pdy, pdw, pws, bytes, d.B, d.C, d.L, d.K, pad, code, call.stream);
    }
    if (raised(status)) return nullptr;
    if (a[5] == Py_None) return THPVariable_Wrap(std::move(made));
    Py_INCREF(a[5]);
    return a[5];
    END_HANDLE_TH_ERRORS
}

// (dy, x, w, pad_left, workspace, out_dx or None, out_dw or None) -> (dx, dw)
PyObject *bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Call call;
    int pad;
    Dims d;
    if (n != 7 || a[4] == Py_None || !exact_int(a[3], pad)) return decline();
    if (!call.begin(a[0])) return call.bad() ? nullptr : decline();
    const at::Tensor *dy = plain(a[0], 3, call.device), *x = plain(a[1], 3, call.device), *w = plain(a[2], 2, call.device),
                     *ws = plain(a[4], -1, call.device);
    if (!dy || !x || !w || !ws || dy->sizes() != x->sizes() || dy->scalar_type() != x->scalar_type() || w->scalar_type() != x->scalar_type() ||
        w->size(0) != x->size(1) || !dims_of(*x, w->size(1), d))
        return decline();
    const int code = dtype_code(*x);
    if (code < 0) return decline();
    const at::Tensor *dx = nullptr, *dw = nullptr;
    if (a[5] != Py_None) {
        dx = plain(a[5], 3, call.device);
        if (!dx || dx->sizes() != dy->sizes() || dx->scalar_type() != dy->scalar_type()) return decline();
    }
    if (a[6] != Py_None && !(dw = weight_out(a[6], *x, d, call.device))) return decline();
    const void *pdy = dy->const_data_ptr(), *px = x->const_data_ptr(), *pw = w->const_data_ptr();
    void *pdx = dx ? dx->mutable_data_ptr() : nullptr, *pdw = dw ? dw->mutable_data_ptr() : nullptr, *pws = ws->mutable_data_ptr();
    const size_t bytes = ws->nbytes();
    at::Tensor made_dx, made_dw;
    int status;
    {
        Unlocked unlocked;
        if (!dx) {
            made_dx = at::empty_like(*dy);
            pdx = made_dx.mutable_data_ptr();
        }
        if (!dw) {
            made_dw = at::empty({d.C, d.K}, x->options());
            pdw = made_dw.mutable_data_ptr();
        }
        status = fn_bwd(pdy, px, pw, pdx, pdw, pws, bytes, d.B, d.C, d.L, d.K, pad, code, call.stream);
    }
    if (raised(status)) return nullptr;
    PyObject *out_dx = a[5], *out_dw = a[6];
    if (out_dx == Py_None) out_dx = THPVariable_Wrap(std::move(made_dx));
    else Py_INCREF(out_dx);
    if (out_dw == Py_None) out_dw = THPVariable_Wrap(std::move(made_dw));
    else Py_INCREF(out_dw);
    PyObject *pair = out_dx && out_dw ? PyTuple_Pack(2, out_dx, out_dw) : nullptr;
    Py_XDECREF(out_dx);
    Py_XDECREF(out_dw);
    return pair;
    END_HANDLE_TH_ERRORS
}

// setup(address of dwconv_fwd, dwconv_bwd_input, dwconv_bwd_weight, dwconv_bwd, current_device, raw_stream, check)
PyObject *setup(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 7) {
        PyErr_SetString(PyExc_TypeError, "setup takes seven arguments");
        return nullptr;
    }
    void *p[4];
    for (int i = 0; i < 4; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i]) return PyErr_Occurred() ? nullptr : decline();
    }
    fn_fwd = (CorrFn)p[0];
    fn_bwd_input = (CorrFn)p[1];
    fn_bwd_weight = (WeightFn)p[2];
    fn_bwd = (BothFn)p[3];
    PyObject **to[3] = {&current_device, &raw_stream, &check};
    for (int i = 0; i < 3; ++i) {
        Py_INCREF(a[4 + i]);
        Py_XSETREF(*to[i], a[4 + i]);
    }
    Py_RETURN_NONE;
}

// ---- the block operators (block.py) ----

struct BlockFns {
    decltype(&dwconv_scan_fwd) scan_fwd;
    decltype(&dwconv_scan_bwd) scan_bwd;
    decltype(&dwconv_scan_states) scan_states;
    decltype(&dwconv_scan_workspace_bytes) scan_workspace;
    decltype(&dwconv_scan_step) scan_step;
    decltype(&dwconv_norm_fwd) norm_fwd;
    decltype(&dwconv_norm_bwd) norm_bwd;
    decltype(&dwconv_norm_workspace_bytes) norm_workspace;
    decltype(&dwconv_clip_grad_norm) clip;
    decltype(&dwconv_clip_workspace_bytes) clip_workspace;
    decltype(&dwconv_conv_step) conv_step;
} blk;
struct DeltaFns {
    decltype(&dwconv_delta_fwd) fwd;
    decltype(&dwconv_delta_bwd) bwd;
    decltype(&dwconv_delta_states) states;
    decltype(&dwconv_delta_workspace_bytes) workspace;
    decltype(&dwconv_delta_step) step;
    decltype(&dwconv_dropout) dropout;
} dlt;

// A device tensor of any strides, or nullptr.
const at::Tensor *on_device(PyObject *o, long device)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || t.layout() != at::kStrided || !t.is_cuda() || t.get_device() != device) return nullptr;
    if ((t.key_set() - c10::autograd_dispatch_keyset_with_ADInplaceOrView - c10::autocast_dispatch_keyset).highestPriorityTypeId() !=
        c10::DispatchKey::CUDA)
        return nullptr;
    return &t;
}

// The arguments of a call, taken in turn; `ok` turns false at the first that is not plainly what the call takes.
struct Args {
    Call call;
    bool ok = true;
    int B = 0, C = 0, L = 0;
    at::ScalarType type = at::kFloat;

    // The tensor that gives the call its sizes and type: [B, C, L], or [B, C] (dims = 2, L = 1).
    const at::Tensor *first(PyObject *o, int dims)
    {
        const at::Tensor *t = on_device(o, call.device);
        ok = t && t->dim() == dims && dtype_code(*t) >= 0;
        if (!ok) return nullptr;
        for (int k = 0; k < dims; ++k) ok = ok && t->size(k) <= INT_MAX;
        if (!ok) return nullptr;
        B = (int)t->size(0), C = (int)t->size(1), L = dims == 3 ? (int)t->size(2) : 1;
        type = t->scalar_type();
        return t;
    }
    // Sizes, type and strides of a sequence.
    bool fits(const at::Tensor &t, int dims, bool written, long long &batch_stride)
    {
        if (t.dim() != dims || t.scalar_type() != type || t.size(0) != B || t.size(1) != C || (dims == 3 && t.size(2) != L)) return false;
        if ((dims == 3 && L > 1 && t.stride(2) != 1) || (C > 1 && t.stride(1) != L)) return false;
        batch_stride = B > 1 ? t.stride(0) : (long long)C * L;
        return !written || B == 1 || batch_stride >= (long long)C * L;
    }
    dwconv_seq seq(PyObject *o, int dims)
    {
        dwconv_seq s{nullptr, 0};
        const at::Tensor *t = ok ? on_device(o, call.device) : nullptr;
        ok = t && fits(*t, dims, false, s.batch_stride);
        if (ok) s.data = t->const_data_ptr();
        return s;
    }
    // An output of the caller's; None: made later by make().
    dwconv_seq_out out(PyObject *o, int dims)
    {
        dwconv_seq_out s{nullptr, (long long)C * L};
        if (!ok || o == Py_None) return s;
        const at::Tensor *t = on_device(o, call.device);
        ok = t && fits(*t, dims, true, s.batch_stride);
        if (ok) s.data = t->mutable_data_ptr();
        return s;
    }
    // A sequence of `channels` channels and of a type of its own, of the call's B and L.
    template <typename S> S seq_of(PyObject *o, int dims, int64_t channels, at::ScalarType dt, bool written)
    {
        S s{nullptr, (long long)channels * L};
        if (!ok || (written && o == Py_None)) return s;
        const at::Tensor *t = on_device(o, call.device);
        ok = t && t->dim() == dims && t->scalar_type() == dt && t->size(0) == B && t->size(1) == channels && (dims < 3 || t->size(2) == L) &&
             (dims < 3 || L == 1 || t->stride(2) == 1) && (channels == 1 || t->stride(1) == L);
        if (!ok) return s;
        if (B > 1) s.batch_stride = t->stride(0);
        ok = !written || s.batch_stride >= (long long)channels * L;
        if (ok) s.data = const_cast<void *>(written ? t->mutable_data_ptr() : t->const_data_ptr());
        return s;
    }
    // A contiguous tensor of that type and those sizes (of fewer dimensions: -1 behind).
    const at::Tensor *dense(PyObject *o, at::ScalarType dt, int64_t a, int64_t b = -1, int64_t c = -1)
    {
        const at::Tensor *t = ok ? on_device(o, call.device) : nullptr;
        const int dims = c >= 0 ? 3 : b >= 0 ? 2 : 1;
        ok = t && t->scalar_type() == dt && t->dim() == dims && t->is_contiguous() && t->size(0) == a && (dims < 2 || t->size(1) == b) &&
             (dims < 3 || t->size(2) == c);
        return ok ? t : nullptr;
    }
    float *dense_f32(PyObject *o, at::IntArrayRef sizes)
    {
        const at::Tensor *t = ok ? on_device(o, call.device) : nullptr;
        ok = t && t->scalar_type() == at::kFloat && t->sizes() == sizes && t->is_contiguous();
        return ok ? static_cast<float *>(const_cast<void *>(t->const_data_ptr())) : nullptr;
    }
    float *f32(PyObject *o, int64_t a, int64_t b = -1, int64_t c = -1)
    {
        const at::Tensor *t = dense(o, at::kFloat, a, b, c);
        return t ? static_cast<float *>(const_cast<void *>(t->const_data_ptr())) : nullptr;
    }
    float *f32_or_none(PyObject *o, int64_t a, int64_t b = -1) { return o == Py_None ? nullptr : f32(o, a, b); }
    const int *index(PyObject *o)
    {
        if (o == Py_None) return nullptr;
        const at::Tensor *t = dense(o, at::kInt, B);
        return t ? static_cast<const int *>(t->const_data_ptr()) : nullptr;
    }
    float number(PyObject *o)
    {
        if (ok && PyFloat_CheckExact(o)) return (float)PyFloat_AS_DOUBLE(o);
        ok = false;
        return 0.0f;
    }
    bool flag(PyObject *o)
    {
        ok = ok && (o == Py_True || o == Py_False);
        return o == Py_True;
    }
    // A workspace of the caller's; None: of `need` bytes, made later.  (An empty one is no request for another: block.py's turn.)
    void *workspace(PyObject *o, size_t &bytes)
    {
        bytes = 0;
        if (!ok || o == Py_None) return nullptr;
        const at::Tensor *t = plain(o, -1, call.device);
        ok = t && t->nbytes() > 0;
        if (!ok) return nullptr;
        bytes = t->nbytes();
        return t->mutable_data_ptr();
    }
};

at::Tensor like(const at::Tensor &t, at::ScalarType type, at::IntArrayRef sizes) { return at::empty(sizes, t.options().dtype(type)); }
template <typename S> void make(S &s, at::Tensor &made, const at::Tensor &t)
{
    if (s.data) return;
    made = at::empty(t.sizes(), t.options());
    s.data = made.mutable_data_ptr();
}
float *make_f32(at::Tensor &made, const at::Tensor &t, at::IntArrayRef sizes)
{
    made = like(t, at::kFloat, sizes);
    return static_cast<float *>(made.mutable_data_ptr());
}
void make_workspace(void *&p, size_t &bytes, size_t need, at::Tensor &made, const at::Tensor &t)
{
    if (p || !need) return;
    made = like(t, at::kByte, {(int64_t)need});
    p = made.mutable_data_ptr();
    bytes = need;
}
// The caller's object, or the tensor made in its place; None for neither.
PyObject *result(PyObject *given, at::Tensor &made)
{
    if (made.defined()) return THPVariable_Wrap(std::move(made));
    Py_INCREF(given);
    return given;
}
template <int N> PyObject *results(PyObject *(&&o)[N])
{
    PyObject *all = PyTuple_New(N);
    for (int k = 0; k < N; ++k) {
        if (!o[k]) Py_CLEAR(all);
    }
    for (int k = 0; k < N; ++k) {
        if (all) PyTuple_SET_ITEM(all, k, o[k]);
        else Py_XDECREF(o[k]);
    }
    return all;
}

// (x, r, i, lam, h0, lengths, rate, save, out, workspace) -> (y, h_last, states)
PyObject *scan_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args g;
    if (n != 10 || !blk.scan_fwd) return decline();
    if (!g.call.begin(a[0])) return g.call.bad() ? nullptr : decline();
    const at::Tensor *x = g.first(a[0], 3);
    dwconv_seq xs = g.seq(a[0], 3), rs = g.seq(a[1], 3), is = g.seq(a[2], 3);
    const float *lam = g.f32(a[3], g.C), *h0 = g.f32_or_none(a[4], g.B, g.C);
    const int *lengths = g.index(a[5]);
    const float rate = g.number(a[6]);
    const bool save = g.flag(a[7]);
    dwconv_seq_out ys = g.out(a[8], 3);
    size_t bytes;
    void *ws = g.workspace(a[9], bytes);
    if (!g.ok) return decline();
    at::Tensor y, h_last, states, space;
    int status;
    {
        Unlocked unlocked;
        make(ys, y, *x);
        float *hp = make_f32(h_last, *x, {g.B, g.C}), *sp = save ? make_f32(states, *x, {g.B, g.C, blk.scan_states(g.L)}) : nullptr;
        make_workspace(ws, bytes, blk.scan_workspace(g.B, g.C, g.L, 0), space, *x);
        status = blk.scan_fwd(xs, rs, is, lam, h0, lengths, ys, hp, sp, ws, bytes, g.B, g.C, g.L, rate, dtype_code(*x), g.call.stream);
    }
    if (raised(status)) return nullptr;
    return results<3>({result(a[8], y), result(Py_None, h_last), result(Py_None, states)});
    END_HANDLE_TH_ERRORS
}

// (dy, x, r, i, lam, states, dh_last, lengths, rate, dx, dr, di (outputs or None), workspace) -> (dx, dr, di, dlam, dh0)
PyObject *scan_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args g;
    if (n != 13 || !blk.scan_bwd) return decline();
    if (!g.call.begin(a[1])) return g.call.bad() ? nullptr : decline();
    const at::Tensor *x = g.first(a[1], 3);
    dwconv_seq dys = g.seq(a[0], 3), xs = g.seq(a[1], 3), rs = g.seq(a[2], 3), is = g.seq(a[3], 3);
    const float *lam = g.f32(a[4], g.C);
    const float *states = g.ok ? g.f32(a[5], g.B, g.C, blk.scan_states(g.L)) : nullptr, *dh = g.f32_or_none(a[6], g.B, g.C);
    const int *lengths = g.index(a[7]);
    const float rate = g.number(a[8]);
    dwconv_seq_out dxs = g.out(a[9], 3), drs = g.out(a[10], 3), dis = g.out(a[11], 3);
    size_t bytes;
    void *ws = g.workspace(a[12], bytes);
    if (!g.ok) return decline();
    at::Tensor dx, dr, di, dlam, dh0, space;
    int status;
    {
        Unlocked unlocked;
        make(dxs, dx, *x), make(drs, dr, *x), make(dis, di, *x);
        float *lp = make_f32(dlam, *x, {g.C}), *hp = make_f32(dh0, *x, {g.B, g.C});
        make_workspace(ws, bytes, blk.scan_workspace(g.B, g.C, g.L, 1), space, *x);
        status = blk.scan_bwd(dys, xs, rs, is, lam, states, dh, lengths, dxs, drs, dis, lp, hp, ws, bytes, g.B, g.C, g.L, rate, dtype_code(*x),
                              g.call.stream);
    }
    if (raised(status)) return nullptr;
    return results<5>({result(a[9], dx), result(a[10], dr), result(a[11], di), result(Py_None, dlam), result(Py_None, dh0)});
    END_HANDLE_TH_ERRORS
}

// (x, r, i, lam, h, slots, rate, out) -> y
PyObject *scan_step(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args g;
    if (n != 8 || !blk.scan_step) return decline();
    if (!g.call.begin(a[0])) return g.call.bad() ? nullptr : decline();
    const at::Tensor *x = g.first(a[0], 2);
    dwconv_seq xs = g.seq(a[0], 2), rs = g.seq(a[1], 2), is = g.seq(a[2], 2);
    const float *lam = g.f32(a[3], g.C);
    const at::Tensor *pool = g.ok ? plain(a[4], 2, g.call.device) : nullptr;
    g.ok = pool && pool->size(0) <= INT_MAX;
    float *h = g.ok ? g.f32(a[4], pool->size(0), g.C) : nullptr;
    const int *slots = g.index(a[5]);
    const float rate = g.number(a[6]);
    dwconv_seq_out ys = g.out(a[7], 2);
    if (!g.ok) return decline();
    at::Tensor y;
    int status;
    {
        Unlocked unlocked;
        make(ys, y, *x);
        status = blk.scan_step(xs, rs, is, lam, h, slots, (int)pool->size(0), ys, g.B, g.C, rate, dtype_code(*x), g.call.stream);
    }
    if (raised(status)) return nullptr;
    return result(a[7], y);
    END_HANDLE_TH_ERRORS
}

// (y, z, res, w, w_next, eps, scale, save, out, out_n) -> (out, n, stats)
PyObject *norm_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args g;
    if (n != 10 || !blk.norm_fwd) return decline();
    const bool block = a[0] != Py_None;
    if (!block && (a[1] != Py_None || a[3] != Py_None || a[8] != Py_None)) return decline();
    if (!g.call.begin(a[2])) return g.call.bad() ? nullptr : decline();
    const at::Tensor *res = g.first(a[2], 3);
    dwconv_seq ys{nullptr, 0}, zs{nullptr, 0}, rs = g.seq(a[2], 3);
    dwconv_seq_out os{nullptr, 0}, ns = g.out(a[9], 3);
    const float *w = nullptr, *w_next = g.f32(a[4], g.C);
    if (block) ys = g.seq(a[0], 3), zs = g.seq(a[1], 3), w = g.f32(a[3], g.C), os = g.out(a[8], 3);
    const float eps = g.number(a[5]), scale = g.number(a[6]);
    const bool save = g.flag(a[7]);
    if (!g.ok) return decline();
    at::Tensor out, next, stats;
    int status;
    {
        Unlocked unlocked;
        if (block) make(os, out, *res);
        make(ns, next, *res);
        float *sp = save ? make_f32(stats, *res, {g.B, 2, g.L}) : nullptr;
        status = blk.norm_fwd(ys, zs, rs, w, w_next, os, ns, sp, g.B, g.C, g.L, eps, scale, dtype_code(*res), g.call.stream);
    }
    if (raised(status)) return nullptr;
    return results<3>({result(a[8], out), result(a[9], next), result(Py_None, stats)});
    END_HANDLE_TH_ERRORS
}

// (dout, dn, y, z, res, w, w_next, stats, scale, dy, dz, dres, workspace) -> (dy, dz, dres, dw, dw_next)
PyObject *norm_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args g;
    if (n != 13 || !blk.norm_bwd) return decline();
    const bool block = a[2] != Py_None;
    if (!block && (a[3] != Py_None || a[5] != Py_None || a[9] != Py_None || a[10] != Py_None)) return decline();
    if (!g.call.begin(a[4])) return g.call.bad() ? nullptr : decline();
    const at::Tensor *res = g.first(a[4], 3);
    dwconv_seq ds{nullptr, 0}, ns = g.seq(a[1], 3), ys{nullptr, 0}, zs{nullptr, 0}, rs = g.seq(a[4], 3);
    if (a[0] != Py_None) ds = g.seq(a[0], 3);
    dwconv_seq_out dys{nullptr, 0}, dzs{nullptr, 0}, drs = g.out(a[11], 3);
    const float *w = nullptr, *w_next = g.f32(a[6], g.C), *stats = g.f32(a[7], g.B, 2, g.L);
    if (block) ys = g.seq(a[2], 3), zs = g.seq(a[3], 3), w = g.f32(a[5], g.C), dys = g.out(a[9], 3), dzs = g.out(a[10], 3);
    const float scale = g.number(a[8]);
    size_t bytes;
    void *ws = g.workspace(a[12], bytes);
    if (!g.ok) return decline();
    at::Tensor dy, dz, dres, dw, dw_next, space;
    int status;
    {
        Unlocked unlocked;
        float *wp = nullptr;
        if (block) make(dys, dy, *res), make(dzs, dz, *res), wp = make_f32(dw, *res, {g.C});
        make(drs, dres, *res);
        float *np = make_f32(dw_next, *res, {g.C});
        make_workspace(ws, bytes, blk.norm_workspace(g.B, g.C, g.L, dtype_code(*res)), space, *res);
        status = blk.norm_bwd(ds, ns, ys, zs, rs, w, w_next, stats, dys, dzs, drs, wp, np, ws, bytes, g.B, g.C, g.L, scale, dtype_code(*res),
                              g.call.stream);
    }
    if (raised(status)) return nullptr;
    return results<5>({result(a[9], dy), result(a[10], dz), result(a[11], dres), result(Py_None, dw), result(Py_None, dw_next)});
    END_HANDLE_TH_ERRORS
}

// (x, w, ring, pos, slots, out) -> y
PyObject *conv_step(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args g;
    if (n != 6 || !blk.conv_step) return decline();
    if (!g.call.begin(a[0])) return g.call.bad() ? nullptr : decline();
    const at::Tensor *x = g.first(a[0], 2);
    dwconv_seq xs = g.seq(a[0], 2);
    const at::Tensor *ring = g.ok ? plain(a[2], 3, g.call.device) : nullptr;
    g.ok = ring && ring->scalar_type() == g.type && ring->size(0) <= INT_MAX && ring->size(1) == g.C && ring->size(2) <= INT_MAX;
    const at::Tensor *w = g.ok ? g.dense(a[1], g.type, g.C, ring->size(2)) : nullptr;
    const int *pos = a[3] == Py_None ? nullptr : g.index(a[3]), *slots = g.index(a[4]);
    dwconv_seq_out ys = g.out(a[5], 2);
    if (!g.ok || !pos) return decline();
    void *rp = ring->mutable_data_ptr();
    at::Tensor y;
    int status;
    {
        Unlocked unlocked;
        make(ys, y, *x);
        status = blk.conv_step(xs, w->const_data_ptr(), rp, pos, slots, (int)ring->size(0), ys, g.B, g.C, (int)ring->size(2), dtype_code(*x),
                               g.call.stream);
    }
    if (raised(status)) return nullptr;
    return result(a[5], y);
    END_HANDLE_TH_ERRORS
}

// (grads, max_norm, out or None, workspace) -> norm; grads and out lists or tuples of tensors
PyObject *clip_grad_norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args g;
    const auto listed = [](PyObject *o) { return PyList_CheckExact(o) || PyTuple_CheckExact(o); };
    if (n != 4 || !blk.clip || !listed(a[0]) || (a[2] != Py_None && !listed(a[2]))) return decline();
    // (the lists' own items for the whole call: the caller holds the lists only, which other threads may change while the lock is away)
    struct Held {
        PyObject *items;
        ~Held() { Py_XDECREF(items); }
    } grads{PySequence_Tuple(a[0])}, outs{a[2] == Py_None || !grads.items ? nullptr : PySequence_Tuple(a[2])};
    if (!grads.items || (a[2] != Py_None && !outs.items)) return nullptr;
    const Py_ssize_t count = PyTuple_GET_SIZE(grads.items);
    if (count < 1 || count > INT_MAX || (outs.items && PyTuple_GET_SIZE(outs.items) != count)) return decline();
    PyObject **in = PySequence_Fast_ITEMS(grads.items), **out = outs.items ? PySequence_Fast_ITEMS(outs.items) : in;
    if (!g.call.begin(in[0])) return g.call.bad() ? nullptr : decline();
    std::vector<const void *> from(count);
    std::vector<void *> to(count);
    std::vector<long long> sizes(count);
    std::vector<int> types(count);
    const at::Tensor *first = nullptr;
    for (Py_ssize_t k = 0; k < count; ++k) {
        const at::Tensor *t = on_device(in[k], g.call.device), *o = out[k] == in[k] ? t : on_device(out[k], g.call.device);
        if (!t || !o || dtype_code(*t) < 0 || !t->is_non_overlapping_and_dense()) return decline();
        if (o != t && (o->scalar_type() != t->scalar_type() || o->sizes() != t->sizes() || o->strides() != t->strides())) return decline();
        from[k] = t->const_data_ptr(), to[k] = o->mutable_data_ptr(), sizes[k] = t->numel(), types[k] = dtype_code(*t);
        if (!first) first = t;
    }
    const float max_norm = g.number(a[1]);
    size_t bytes;
    void *ws = g.workspace(a[3], bytes);
    if (!g.ok) return decline();
    at::Tensor norm, space;
    int status;
    {
        Unlocked unlocked;
        float *np = make_f32(norm, *first, {});
        make_workspace(ws, bytes, blk.clip_workspace(), space, *first);
        status = blk.clip(from.data(), to.data(), sizes.data(), types.data(), (int)count, max_norm, np, ws, bytes, g.call.stream);
    }
    if (raised(status)) return nullptr;
    return result(Py_None, norm);
    END_HANDLE_TH_ERRORS
}

// The heads of a call of the delta rule, from q, v, g and key_heads.
struct Heads {
    int H = 0, Hk = 0, DK = 0, DV = 0;
    float scale = 1.0f;
    Heads(Args &g, PyObject *q, PyObject *v, PyObject *gate, PyObject *key_heads, PyObject *scaled, int dims)
    {
        const at::Tensor *qt = g.first(q, dims), *vt = g.ok ? on_device(v, g.call.device) : nullptr, *gt = g.ok ? on_device(gate, g.call.device) : nullptr;
        g.ok = qt && vt && gt && vt->dim() == dims && gt->dim() == dims && gt->size(1) >= 1 && gt->size(1) <= INT_MAX && vt->size(1) <= INT_MAX;
        if (!g.ok) return;
        H = Hk = (int)gt->size(1);
        if (key_heads != Py_None) g.ok = exact_int(key_heads, Hk);
        g.ok = g.ok && Hk >= 1 && H % Hk == 0 && g.C % Hk == 0 && vt->size(1) % H == 0 && g.C >= Hk;
        if (!g.ok) return;
        DK = g.C / Hk, DV = (int)(vt->size(1) / H);
        scale = scaled == Py_None ? (float)std::pow((double)DK, -0.5) : g.number(scaled);
    }
};
template <typename S> S made_out(S s, at::Tensor &made, const at::Tensor &t, at::IntArrayRef sizes)
{
    if (s.data) return s;
    made = at::empty(sizes, t.options());
    s.data = made.mutable_data_ptr();
    return s;
}

// (q, k, v, g, beta, s0, lengths, key_heads, scale, eps, save, out, workspace) -> (o, s_last, states)
PyObject *delta_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args g;
    if (n != 13 || !dlt.fwd) return decline();
    if (!g.call.begin(a[0])) return g.call.bad() ? nullptr : decline();
    const Heads hd(g, a[0], a[2], a[3], a[7], a[8], 3);
    if (!g.ok) return decline();
    const int keys = g.C, values = hd.H * hd.DV;
    dwconv_seq q = g.seq_of<dwconv_seq>(a[0], 3, keys, g.type, false), k = g.seq_of<dwconv_seq>(a[1], 3, keys, g.type, false),
               v = g.seq_of<dwconv_seq>(a[2], 3, values, g.type, false), gt = g.seq_of<dwconv_seq>(a[3], 3, hd.H, at::kFloat, false),
               bt = g.seq_of<dwconv_seq>(a[4], 3, hd.H, at::kFloat, false);
    const int64_t state[] = {g.B, hd.H, hd.DK, hd.DV};
    const float *s0 = a[5] == Py_None ? nullptr : g.dense_f32(a[5], state);
    const int *lengths = g.index(a[6]);
    const float eps = g.number(a[9]);
    const bool save = g.flag(a[10]);
    dwconv_seq_out os = g.seq_of<dwconv_seq_out>(a[11], 3, values, g.type, true);
    size_t bytes;
    void *ws = g.workspace(a[12], bytes);
    if (!g.ok) return decline();
    const at::Tensor &like_q = THPVariable_Unpack(a[0]);
    at::Tensor o, s_last, states, space;
    int status;
    {
        Unlocked unlocked;
        os = made_out(os, o, like_q, {g.B, values, g.L});
        float *lp = make_f32(s_last, like_q, state), *sp = save ? make_f32(states, like_q, {g.B, hd.H, dlt.states(g.L), hd.DK, hd.DV}) : nullptr;
        make_workspace(ws, bytes, dlt.workspace(g.B, hd.H, hd.Hk, hd.DK, hd.DV, g.L, 0), space, like_q);
        status = dlt.fwd(q, k, v, gt, bt, s0, lengths, os, lp, sp, ws, bytes, g.B, hd.H, hd.Hk, hd.DK, hd.DV, g.L, hd.scale, eps, dtype_code(like_q),
                         g.call.stream);
    }
    if (raised(status)) return nullptr;
    return results<3>({result(a[11], o), result(Py_None, s_last), result(Py_None, states)});
    END_HANDLE_TH_ERRORS
}

// (do, q, k, v, g, beta, states, ds_last, lengths, key_heads, scale, eps, dq, dk, dv (outputs or None), workspace) -> (dq, dk, dv, dg, dbeta, ds0)
PyObject *delta_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args g;
    if (n != 16 || !dlt.bwd) return decline();
    if (!g.call.begin(a[1])) return g.call.bad() ? nullptr : decline();
    const Heads hd(g, a[1], a[3], a[4], a[9], a[10], 3);
    if (!g.ok) return decline();
    const int keys = g.C, values = hd.H * hd.DV;
    dwconv_seq d = g.seq_of<dwconv_seq>(a[0], 3, values, g.type, false), q = g.seq_of<dwconv_seq>(a[1], 3, keys, g.type, false),
               k = g.seq_of<dwconv_seq>(a[2], 3, keys, g.type, false), v = g.seq_of<dwconv_seq>(a[3], 3, values, g.type, false),
               gt = g.seq_of<dwconv_seq>(a[4], 3, hd.H, at::kFloat, false), bt = g.seq_of<dwconv_seq>(a[5], 3, hd.H, at::kFloat, false);
    const int64_t state[] = {g.B, hd.H, hd.DK, hd.DV}, kept[] = {g.B, hd.H, dlt.states(g.L), hd.DK, hd.DV};
    const float *states = g.dense_f32(a[6], kept), *ds = a[7] == Py_None ? nullptr : g.dense_f32(a[7], state);
    const int *lengths = g.index(a[8]);
    const float eps = g.number(a[11]);
    dwconv_seq_out dqs = g.seq_of<dwconv_seq_out>(a[12], 3, keys, g.type, true), dks = g.seq_of<dwconv_seq_out>(a[13], 3, keys, g.type, true),
                   dvs = g.seq_of<dwconv_seq_out>(a[14], 3, values, g.type, true);
    size_t bytes;
    void *ws = g.workspace(a[15], bytes);
    if (!g.ok) return decline();
    const at::Tensor &like_q = THPVariable_Unpack(a[1]);
    at::Tensor dq, dk, dv, dg, dbeta, ds0, space;
    int status;
    {
        Unlocked unlocked;
        dqs = made_out(dqs, dq, like_q, {g.B, keys, g.L}), dks = made_out(dks, dk, like_q, {g.B, keys, g.L}), dvs = made_out(dvs, dv, like_q, {g.B, values, g.L});
        float *gp = make_f32(dg, like_q, {g.B, hd.H, g.L}), *bp = make_f32(dbeta, like_q, {g.B, hd.H, g.L}), *sp = make_f32(ds0, like_q, state);
        make_workspace(ws, bytes, dlt.workspace(g.B, hd.H, hd.Hk, hd.DK, hd.DV, g.L, 1), space, like_q);
        status = dlt.bwd(d, q, k, v, gt, bt, states, ds, lengths, dqs, dks, dvs, gp, bp, sp, ws, bytes, g.B, hd.H, hd.Hk, hd.DK, hd.DV, g.L, hd.scale, eps,
                         dtype_code(like_q), g.call.stream);
    }
    if (raised(status)) return nullptr;
    return results<6>({result(a[12], dq), result(a[13], dk), result(a[14], dv), result(Py_None, dg), result(Py_None, dbeta), result(Py_None, ds0)});
    END_HANDLE_TH_ERRORS
}

// (q, k, v, g, beta, s, slots, key_heads, scale, eps, out) -> o
PyObject *delta_step(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args g;
    if (n != 11 || !dlt.step) return decline();
    if (!g.call.begin(a[0])) return g.call.bad() ? nullptr : decline();
    const Heads hd(g, a[0], a[2], a[3], a[7], a[8], 2);
    if (!g.ok) return decline();
    const int keys = g.C, values = hd.H * hd.DV;
    dwconv_seq q = g.seq_of<dwconv_seq>(a[0], 2, keys, g.type, false), k = g.seq_of<dwconv_seq>(a[1], 2, keys, g.type, false),
               v = g.seq_of<dwconv_seq>(a[2], 2, values, g.type, false), gt = g.seq_of<dwconv_seq>(a[3], 2, hd.H, at::kFloat, false),
               bt = g.seq_of<dwconv_seq>(a[4], 2, hd.H, at::kFloat, false);
    const at::Tensor *pool = g.ok ? plain(a[5], 4, g.call.device) : nullptr;
    g.ok = pool && pool->size(0) <= INT_MAX;
    float *s = g.ok ? g.dense_f32(a[5], {pool->size(0), hd.H, hd.DK, hd.DV}) : nullptr;
    const int *slots = g.index(a[6]);
    const float eps = g.number(a[9]);
    dwconv_seq_out os = g.seq_of<dwconv_seq_out>(a[10], 2, values, g.type, true);
    if (!g.ok) return decline();
    const at::Tensor &like_q = THPVariable_Unpack(a[0]);
    at::Tensor o;
    int status;
    {
        Unlocked unlocked;
        os = made_out(os, o, like_q, {g.B, values});
        status = dlt.step(q, k, v, gt, bt, s, slots, (int)pool->size(0), os, g.B, hd.H, hd.Hk, hd.DK, hd.DV, hd.scale, eps, dtype_code(like_q), g.call.stream);
    }
    if (raised(status)) return nullptr;
    return result(a[10], o);
    END_HANDLE_TH_ERRORS
}

// (x, p, rng, layer, res, scale, tied, out) -> out
PyObject *dropout(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args g;
    if (n != 8 || !dlt.dropout) return decline();
    if (!g.call.begin(a[0])) return g.call.bad() ? nullptr : decline();
    const at::Tensor *x = g.first(a[0], 3);
    dwconv_seq xs = g.seq(a[0], 3), rs{nullptr, 0};
    const float p = g.number(a[1]);
    const at::Tensor *rng = g.dense(a[2], at::kLong, 2);
    int layer = 0;
    g.ok = g.ok && exact_int(a[3], layer);
    if (a[4] != Py_None) rs = g.seq(a[4], 3);
    const float scale = g.number(a[5]);
    const bool tied = g.flag(a[6]);
    dwconv_seq_out os = g.out(a[7], 3);
    if (!g.ok) return decline();
    at::Tensor o;
    int status;
    {
        Unlocked unlocked;
        make(os, o, *x);
        status = dlt.dropout(xs, rs, os, static_cast<const long long *>(rng->const_data_ptr()), layer, g.B, g.C, g.L, p, scale, tied, dtype_code(*x), g.call.stream);
    }
    if (raised(status)) return nullptr;
    return result(a[7], o);
    END_HANDLE_TH_ERRORS
}

// setup_delta(the addresses of DeltaFns in its order)
PyObject *setup_delta(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    void *p[6];
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "setup_delta takes six addresses");
        return nullptr;
    }
    for (int k = 0; k < 6; ++k) {
        p[k] = PyLong_AsVoidPtr(a[k]);
        if (!p[k]) return PyErr_Occurred() ? nullptr : decline();
    }
    dlt = DeltaFns{(decltype(dlt.fwd))p[0], (decltype(dlt.bwd))p[1], (decltype(dlt.states))p[2], (decltype(dlt.workspace))p[3], (decltype(dlt.step))p[4],
                   (decltype(dlt.dropout))p[5]};
    Py_RETURN_NONE;
}

// setup_block(the addresses of BlockFns in its order)
PyObject *setup_block(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    void *p[11];
    if (n != 11) {
        PyErr_SetString(PyExc_TypeError, "setup_block takes eleven addresses");
        return nullptr;
    }
    for (int k = 0; k < 11; ++k) {
        p[k] = PyLong_AsVoidPtr(a[k]);
        if (!p[k]) return PyErr_Occurred() ? nullptr : decline();
    }
    blk = BlockFns{(decltype(blk.scan_fwd))p[0], (decltype(blk.scan_bwd))p[1], (decltype(blk.scan_states))p[2], (decltype(blk.scan_workspace))p[3],
                   (decltype(blk.scan_step))p[4], (decltype(blk.norm_fwd))p[5], (decltype(blk.norm_bwd))p[6], (decltype(blk.norm_workspace))p[7],
                   (decltype(blk.clip))p[8], (decltype(blk.clip_workspace))p[9], (decltype(blk.conv_step))p[10]};
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"setup", (PyCFunction)(void (*)())setup, METH_FASTCALL, nullptr},
    {"fwd", (PyCFunction)(void (*)())fwd, METH_FASTCALL, nullptr},
    {"bwd_input", (PyCFunction)(void (*)())bwd_input, METH_FASTCALL, nullptr},
    {"bwd_weight", (PyCFunction)(void (*)())bwd_weight, METH_FASTCALL, nullptr},
    {"bwd", (PyCFunction)(void (*)())bwd, METH_FASTCALL, nullptr},
    {"setup_block", (PyCFunction)(void (*)())setup_block, METH_FASTCALL, nullptr},
    {"scan_fwd", (PyCFunction)(void (*)())scan_fwd, METH_FASTCALL, nullptr},
    {"scan_bwd", (PyCFunction)(void (*)())scan_bwd, METH_FASTCALL, nullptr},
    {"scan_step", (PyCFunction)(void (*)())scan_step, METH_FASTCALL, nullptr},
    {"norm_fwd", (PyCFunction)(void (*)())norm_fwd, METH_FASTCALL, nullptr},
    {"norm_bwd", (PyCFunction)(void (*)())norm_bwd, METH_FASTCALL, nullptr},
    {"conv_step", (PyCFunction)(void (*)())conv_step, METH_FASTCALL, nullptr},
    {"clip_grad_norm", (PyCFunction)(void (*)())clip_grad_norm, METH_FASTCALL, nullptr},
    {"setup_delta", (PyCFunction)(void (*)())setup_delta, METH_FASTCALL, nullptr},
    {"delta_fwd", (PyCFunction)(void (*)())delta_fwd, METH_FASTCALL, nullptr},
    {"delta_bwd", (PyCFunction)(void (*)())delta_bwd, METH_FASTCALL, nullptr},
    {"delta_step", (PyCFunction)(void (*)())delta_step, METH_FASTCALL, nullptr},
    {"dropout", (PyCFunction)(void (*)())dropout, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// (binding.py compares `built_for` with the PyTorch and the Python that are there before it calls anything)
PyMODINIT_FUNC PyInit__fastcall()
{
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", DWCONV_BUILT_FOR) < 0) Py_CLEAR(m);
    return m;
}
