// The binding's hot calls without ctypes: tensors in, parameter struct filled, library called.  A call marshals ten to
// twenty tensors, and in Python the checks, the struct's fields and the foreign call were most of the time of a short one.
// us per call among others, through ctypes / here: one token of a layer, D 4096, batch 1 13.8 / 8.9, of the scan, batch 64 9.6 / 7.6 (its kernel
// 7.1); forward + backward of 1 x 64 x 256 float32 through autograd 199 / 144.
//
// Only the plain case is served: exact torch.Tensors (or Parameters) with memory of their own, on the GPU, contiguous, of the expected
// type and shape.  Everything else returns None before anything has been allocated or enqueued, and binding.py takes it
// through its own marshalling, which raises what is to be raised.  Results: the call's tensors, or the library's error code as an int.
#include <Python.h>

#include <initializer_list>
#include <optional>

#include <ATen/ATen.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <vector>

#include "ss_adamw.h"
#include "ss_embed.h"
#include "ss_gate.h"
#include "ss_layer.h"
#include "ss_logprob.h"
#include "ss_norm.h"
#include "ss_quant.h"
#include "ss_scan.h"

namespace {

typedef std::initializer_list<int64_t> Shape;
constexpr int64_t CHANNEL_SKEW_BYTES = 66560;   // as binding.empty_channel_skewed

// Arguments of one call; `ok` falls when one of them is not the plain case.
struct Args {
    PyObject* const* a;
    bool ok = true;
    const at::Tensor* tensor(int i)
    {
        if (!THPVariable_CheckExact(a[i])) { ok = false; return nullptr; }
        const at::Tensor& t = THPVariable_Unpack(a[i]);
        if (!t.is_cuda() || !t.has_storage() || !t.is_contiguous()) { ok = false; return nullptr; }
        return &t;
    }
    // device pointer of argument i; None gives a null pointer where `optional`
    void* ptr(int i, at::ScalarType type, Shape shape, bool optional = false)
    {
        if (optional && a[i] == Py_None) return nullptr;
        const at::Tensor* t = ok ? tensor(i) : nullptr;
        if (!t) return nullptr;
        if (t->scalar_type() != type || !t->sizes().equals(at::IntArrayRef(shape))) { ok = false; return nullptr; }
        return t->data_ptr();
    }
    bool none(int i) const { return a[i] == Py_None; }
    long number(int i)
    {
        const long v = PyLong_AsLong(a[i]);
        if (v == -1 && PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        return v;
    }
    void* stream(int i)
    {
        void* v = PyLong_AsVoidPtr(a[i]);
        if (!v && PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        return v;
    }
};

bool io_type(const at::Tensor& t, int32_t& code)
{
    if (t.scalar_type() == at::kFloat) code = SS_F32;
    else if (t.scalar_type() == at::kBFloat16) code = SS_BF16;
    else return false;
    return true;
}
inline bool fits(int64_t v) { return v >= 0 && v <= 0x7fffffff; }

template <typename P, typename F>
int call(F f, const P& p, void* stream)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f(&p, stream);
    Py_END_ALLOW_THREADS
    return rc;
}
PyObject* wrapped(const at::Tensor& t) { return THPVariable_Wrap(t); }
at::Tensor empty_f32(at::IntArrayRef shape, const at::Tensor& like) { return at::empty(shape, like.options().dtype(at::kFloat).requires_grad(false)); }

// step(h, u_t, delta_t, A, B_t, C_t, Dskip, z_t, delta_bias, out_t, flags, stream) -> out_t
PyObject* py_step(PyObject*, PyObject* const* argv, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 12) Py_RETURN_NONE;
    Args a{argv};
    const at::Tensor *h = a.tensor(0), *u = a.ok ? a.tensor(1) : nullptr;
    if (!a.ok || h->dim() != 3) Py_RETURN_NONE;
    const int64_t nb = h->size(0), nd = h->size(1), nn = h->size(2);
    ss_step_params p{};
    if (!io_type(*u, p.io_dtype) || !fits(nb) || !fits(nd) || !fits(nn)) Py_RETURN_NONE;
    const at::ScalarType io = u->scalar_type(), f32 = at::kFloat;
    p.batch = (int32_t)nb; p.dim = (int32_t)nd; p.dstate = (int32_t)nn;
    p.flags = (uint32_t)a.number(10);
    const bool bfix = p.flags & SS_B_FIXED, cfix = p.flags & SS_C_FIXED;
    p.h = static_cast<float*>(a.ptr(0, f32, {nb, nd, nn}));
    p.u_t = a.ptr(1, io, {nb, nd});
    p.delta_t = a.ptr(2, io, {nb, nd});
    p.A = static_cast<const float*>(a.ptr(3, f32, {nd, nn}));
    p.B_t = bfix ? a.ptr(4, f32, {nd, nn}) : a.ptr(4, io, {nb, nn});
    p.C_t = cfix ? a.ptr(5, f32, {nd, nn}) : a.ptr(5, io, {nb, nn});
    p.Dskip = static_cast<const float*>(a.ptr(6, f32, {nd}, true));
    p.z_t = a.ptr(7, io, {nb, nd}, true);
    p.delta_bias = static_cast<const float*>(a.ptr(8, f32, {nd}, true));
    void* out = a.ptr(9, io, {nb, nd}, true);
    void* stream = a.stream(11);
    if (!a.ok) Py_RETURN_NONE;
    if (!a.none(6)) p.flags |= SS_HAS_D;
    if (!a.none(7)) p.flags |= SS_HAS_Z;
    if (!a.none(8)) p.flags |= SS_HAS_DELTA_BIAS;
    at::Tensor fresh;
    if (a.none(9)) {
        fresh = at::empty_like(*u);
        out = fresh.data_ptr();
    }
    p.out_t = out;
    const int rc = call(ss_step, p, stream);
    if (rc != SS_OK) return PyLong_FromLong(rc);
    if (a.none(9)) return wrapped(fresh);
    Py_INCREF(argv[9]);
    return argv[9];
    END_HANDLE_TH_ERRORS
}

// layer_step(h, conv_state, x_t, z_t, conv_w, conv_b, W_x, W_dt, dt_bias, A, Dskip, scratch, out_t, stream) -> out_t
PyObject* py_layer_step(PyObject*, PyObject* const* argv, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 14) Py_RETURN_NONE;
    Args a{argv};
    const at::Tensor* h = a.tensor(0);
    const at::Tensor* x = a.ok ? a.tensor(2) : nullptr;
    const at::Tensor* cw = a.ok ? a.tensor(4) : nullptr;
    const at::Tensor* wdt = a.ok ? a.tensor(7) : nullptr;
    const at::Tensor* scratch = a.ok ? a.tensor(11) : nullptr;
    if (!a.ok || h->dim() != 3 || cw->dim() != 2 || wdt->dim() != 2 || scratch->scalar_type() != at::kByte) Py_RETURN_NONE;
    const int64_t nb = h->size(0), nd = h->size(1), nn = h->size(2), width = cw->size(1), rank = wdt->size(1);
    ss_layer_step_params p{};
    if (!io_type(*x, p.io_dtype) || !fits(nb) || !fits(nd) || !fits(nn) || !fits(rank) || width < 1 || !fits(width)) Py_RETURN_NONE;
    const at::ScalarType io = x->scalar_type(), f32 = at::kFloat;
    p.batch = (int32_t)nb; p.dim = (int32_t)nd; p.dstate = (int32_t)nn; p.dt_rank = (int32_t)rank; p.conv_width = (int32_t)width;
    p.h = static_cast<float*>(a.ptr(0, f32, {nb, nd, nn}));
    p.conv_state = a.ptr(1, io, {nb, nd, width - 1});
    p.x_t = a.ptr(2, io, {nb, nd});
    p.z_t = a.ptr(3, io, {nb, nd});
    p.conv_w = static_cast<const float*>(a.ptr(4, f32, {nd, width}));
    p.conv_b = static_cast<const float*>(a.ptr(5, f32, {nd}));
    p.W_x = a.ptr(6, io, {rank + 2 * nn, nd});
    p.W_dt = a.ptr(7, io, {nd, rank});
    p.dt_bias = static_cast<const float*>(a.ptr(8, f32, {nd}));
    p.A = static_cast<const float*>(a.ptr(9, f32, {nd, nn}));
    p.Dskip = static_cast<const float*>(a.ptr(10, f32, {nd}));
    void* out = a.ptr(12, io, {nb, nd}, true);
    void* stream = a.stream(13);
    if (!a.ok) Py_RETURN_NONE;
    p.scratch = scratch->data_ptr();
    p.scratch_bytes = (size_t)scratch->numel();
    at::Tensor fresh;
    if (a.none(12)) {
        fresh = at::empty_like(*x);
        out = fresh.data_ptr();
    }
    p.out_t = out;
    const int rc = call(ss_layer_step, p, stream);
    if (rc != SS_OK) return PyLong_FromLong(rc);
    if (a.none(12)) return wrapped(fresh);
    Py_INCREF(argv[12]);
    return argv[12];
    END_HANDLE_TH_ERRORS
}

// The scan's inputs: u, delta, A, B, C, Dskip, z, delta_bias, h0 from argument `at` on; real state.
bool scan_inputs(Args& a, int at, uint32_t flags, ss_fwd_params& p)
{
    const at::Tensor *u = a.tensor(at), *A = a.ok ? a.tensor(at + 2) : nullptr;
    const at::Tensor *B = a.ok ? a.tensor(at + 3) : nullptr, *C = a.ok ? a.tensor(at + 4) : nullptr;
    if (!a.ok || u->dim() != 3 || A->dim() != 2 || !io_type(*u, p.io_dtype)) return false;
    const int64_t nb = u->size(0), nd = u->size(1), nl = u->size(2), nn = A->size(1);
    if (!fits(nb) || !fits(nd) || !fits(nl) || !fits(nn)) return false;
    const at::ScalarType io = u->scalar_type(), f32 = at::kFloat;
    p.batch = (int32_t)nb; p.dim = (int32_t)nd; p.seqlen = (int32_t)nl; p.dstate = (int32_t)nn;
    p.flags = flags;
    p.u = a.ptr(at, io, {nb, nd, nl});
    p.delta = a.ptr(at + 1, io, {nb, nd, nl});
    p.A = static_cast<const float*>(a.ptr(at + 2, f32, {nd, nn}));
    if (B->dim() == 2) p.flags |= SS_B_FIXED;   // (D,N): the time-invariant form
    if (C->dim() == 2) p.flags |= SS_C_FIXED;
    p.Bmat = B->dim() == 2 ? a.ptr(at + 3, f32, {nd, nn}) : a.ptr(at + 3, io, {nb, nn, nl});
    p.Cmat = C->dim() == 2 ? a.ptr(at + 4, f32, {nd, nn}) : a.ptr(at + 4, io, {nb, nn, nl});
    p.Dskip = static_cast<const float*>(a.ptr(at + 5, f32, {nd}, true));
    p.z = a.ptr(at + 6, io, {nb, nd, nl}, true);
    p.delta_bias = static_cast<const float*>(a.ptr(at + 7, f32, {nd}, true));
    p.h0 = static_cast<const float*>(a.ptr(at + 8, f32, {nb, nd, nn}, true));
    if (!a.none(at + 5)) p.flags |= SS_HAS_D;
    if (!a.none(at + 6)) p.flags |= SS_HAS_Z;
    if (!a.none(at + 7)) p.flags |= SS_HAS_DELTA_BIAS;
    if (!a.none(at + 8)) p.flags |= SS_HAS_H0;
    return a.ok;
}
bool workspace_of(Args& a, int i, ss_fwd_params& p)
{
    const at::Tensor* ws = a.tensor(i);
    if (!ws || ws->scalar_type() != at::kByte) return false;
    p.workspace = ws->data_ptr();
    p.workspace_bytes = (size_t)ws->numel();
    return true;
}

// scan_fwd(u, delta, A, B, C, Dskip, z, delta_bias, h0, workspace, flags, want_last, stream) -> (out, h_last or None)
PyObject* py_scan_fwd(PyObject*, PyObject* const* argv, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 13) Py_RETURN_NONE;
    Args a{argv};
    ss_fwd_params p{};
    const uint32_t flags = (uint32_t)a.number(10);
    const bool last = argv[11] == Py_True;
    void* stream = a.stream(12);
    if (!a.ok || !scan_inputs(a, 0, flags, p)) Py_RETURN_NONE;
    if (a.none(9)) p.flags &= ~(uint32_t)SS_SAVE_FOR_BWD;
    else if (!workspace_of(a, 9, p)) Py_RETURN_NONE;
    const at::Tensor& u = *a.tensor(0);
    at::Tensor out = at::empty_like(u), h_last;
    p.out = out.data_ptr();
    if (last) {
        h_last = empty_f32({p.batch, p.dim, p.dstate}, u);
        p.h_last = static_cast<float*>(h_last.data_ptr());
        p.flags |= SS_WRITE_H_LAST;
    }
    const int rc = call(ss_scan_fwd, p, stream);
    if (rc != SS_OK) return PyLong_FromLong(rc);
    PyObject* res = PyTuple_New(2);
    if (!res) return nullptr;
    PyTuple_SET_ITEM(res, 0, wrapped(out));
    if (last) PyTuple_SET_ITEM(res, 1, wrapped(h_last));
    else { Py_INCREF(Py_None); PyTuple_SET_ITEM(res, 1, Py_None); }
    return res;
    END_HANDLE_TH_ERRORS
}

// scan_bwd(u, delta, A, B, C, Dskip, z, delta_bias, h0, workspace, dout, dh_last, flags, want_dh0, stream) -> dict of gradients
PyObject* py_scan_bwd(PyObject*, PyObject* const* argv, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 15) Py_RETURN_NONE;
    Args a{argv};
    ss_bwd_params q{};
    const uint32_t flags = (uint32_t)a.number(12);
    const bool want_dh0 = argv[13] == Py_True;
    void* stream = a.stream(14);
    if (!a.ok || !scan_inputs(a, 0, flags, q.fwd) || !workspace_of(a, 9, q.fwd)) Py_RETURN_NONE;
    const at::Tensor &u = *a.tensor(0), &A = *a.tensor(2), &B = *a.tensor(3), &C = *a.tensor(4);
    const int64_t nb = u.size(0), nd = u.size(1), nl = u.size(2), nn = A.size(1);
    q.dout = a.ptr(10, u.scalar_type(), {nb, nd, nl});
    q.dh_last = static_cast<const float*>(a.ptr(11, at::kFloat, {nb, nd, nn}, true));
    if (!a.ok) Py_RETURN_NONE;
    // du, ddelta and dz in one allocation, 65 KiB further apart than their size (binding.empty_channel_skewed)
    const bool has_z = !a.none(6);
    const int64_t esz = (int64_t)u.element_size(), pitch = ((u.numel() * esz + 255) / 256 * 256 + CHANNEL_SKEW_BYTES) / esz;
    const at::Tensor pool = at::empty({(has_z ? 3 : 2) * pitch}, u.options().requires_grad(false));
    const int64_t row = nl > 1 ? nl : 1, entry = row * (nd > 1 ? nd : 1);
    auto carve = [&](int64_t i) { return at::as_strided(pool, u.sizes(), {entry, row, 1}, i * pitch); };
    at::Tensor du = carve(0), ddelta = carve(1), dz, dD, dbias, dh0;
    at::Tensor dB = empty_f32(B.sizes(), u), dC = empty_f32(C.sizes(), u), dA = empty_f32(A.sizes(), u);
    if (has_z) dz = carve(2);
    if (!a.none(5)) dD = empty_f32({nd}, u);
    if (!a.none(7)) dbias = empty_f32({nd}, u);
    if (want_dh0) dh0 = empty_f32({nb, nd, nn}, u);
    auto f = [](const at::Tensor& t) { return t.defined() ? static_cast<float*>(t.data_ptr()) : nullptr; };
    q.du = du.data_ptr(); q.ddelta = ddelta.data_ptr(); q.dz = has_z ? dz.data_ptr() : nullptr;
    q.dB = f(dB); q.dC = f(dC); q.dA = f(dA); q.dD = f(dD); q.ddelta_bias = f(dbias); q.dh0 = f(dh0);
    const int rc = call(ss_scan_bwd, q, stream);
    if (rc != SS_OK) return PyLong_FromLong(rc);
    PyObject* res = PyDict_New();
    if (!res) return nullptr;
    auto put = [&](const char* name, const at::Tensor& t) {
        PyObject* o = t.defined() ? wrapped(t) : (Py_INCREF(Py_None), Py_None);
        const bool good = o && PyDict_SetItemString(res, name, o) == 0;
        Py_XDECREF(o);
        return good;
    };
    if (!(put("du", du) && put("ddelta", ddelta) && put("dz", dz) && put("dB", dB) && put("dC", dC) && put("dA", dA) && put("dD", dD) &&
          put("ddelta_bias", dbias) && put("dh0", dh0))) {
        Py_DECREF(res);
        return nullptr;
    }
    return res;
    END_HANDLE_TH_ERRORS
}

// The layer's inputs from argument `at` on: x, z, conv_w, conv_b, W_x, W_dt, dt_bias, A, Dskip, scratch, saved (or None).
bool layer_inputs(Args& a, int at, ss_layer_params& p)
{
    const at::Tensor* x = a.tensor(at);
    const at::Tensor* cw = a.ok ? a.tensor(at + 2) : nullptr;
    const at::Tensor* wdt = a.ok ? a.tensor(at + 5) : nullptr;
    const at::Tensor* A = a.ok ? a.tensor(at + 7) : nullptr;
    const at::Tensor* scratch = a.ok ? a.tensor(at + 9) : nullptr;
    if (!a.ok || x->dim() != 3 || cw->dim() != 2 || wdt->dim() != 2 || A->dim() != 2 || scratch->scalar_type() != at::kByte) return false;
    const int64_t nb = x->size(0), nd = x->size(1), nl = x->size(2), nn = A->size(1), width = cw->size(1), rank = wdt->size(1);
    if (!io_type(*x, p.io_dtype) || !fits(nb) || !fits(nd) || !fits(nl) || !fits(nn) || !fits(rank) || width < 1 || !fits(width)) return false;
    const at::ScalarType io = x->scalar_type(), f32 = at::kFloat;
    p.batch = (int32_t)nb; p.dim = (int32_t)nd; p.seqlen = (int32_t)nl; p.dstate = (int32_t)nn; p.dt_rank = (int32_t)rank; p.conv_width = (int32_t)width;
    p.x = a.ptr(at, io, {nb, nd, nl});
    p.z = a.ptr(at + 1, io, {nb, nd, nl});
    p.conv_w = static_cast<const float*>(a.ptr(at + 2, f32, {nd, width}));
    p.conv_b = static_cast<const float*>(a.ptr(at + 3, f32, {nd}));
    p.W_x = a.ptr(at + 4, io, {rank + 2 * nn, nd});
    p.W_dt = a.ptr(at + 5, io, {nd, rank});
    p.dt_bias = static_cast<const float*>(a.ptr(at + 6, f32, {nd}));
    p.A = static_cast<const float*>(a.ptr(at + 7, f32, {nd, nn}));
    p.Dskip = static_cast<const float*>(a.ptr(at + 8, f32, {nd}));
    p.scratch = scratch->data_ptr();
    p.scratch_bytes = (size_t)scratch->numel();
    if (a.ok && !a.none(at + 10)) {
        const at::Tensor* saved = a.tensor(at + 10);
        if (!saved || saved->scalar_type() != at::kByte) return false;
        p.saved = saved->data_ptr();
        p.saved_bytes = (size_t)saved->numel();
    }
    return a.ok;
}

// layer_fwd(x .. saved, return_states, stream) -> out, or (out, h_last, conv_state)
PyObject* py_layer_fwd(PyObject*, PyObject* const* argv, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 13) Py_RETURN_NONE;
    Args a{argv};
    ss_layer_params p{};
    const bool states = argv[11] == Py_True;
    void* stream = a.stream(12);
    if (!a.ok || !layer_inputs(a, 0, p)) Py_RETURN_NONE;
    const at::Tensor& x = *a.tensor(0);
    at::Tensor out = at::empty_like(x), h_last, conv_state;
    p.out = out.data_ptr();
    if (states) {
        h_last = empty_f32({p.batch, p.dim, p.dstate}, x);
        conv_state = at::empty({p.batch, p.dim, p.conv_width - 1}, x.options().requires_grad(false));
        p.h_last = static_cast<float*>(h_last.data_ptr());
        p.conv_state = conv_state.data_ptr();
    }
    const int rc = call(ss_layer_fwd, p, stream);
    if (rc != SS_OK) return PyLong_FromLong(rc);
    if (!states) return wrapped(out);
    PyObject* res = PyTuple_New(3);
    if (!res) return nullptr;
    PyTuple_SET_ITEM(res, 0, wrapped(out));
    PyTuple_SET_ITEM(res, 1, wrapped(h_last));
    PyTuple_SET_ITEM(res, 2, wrapped(conv_state));
    return res;
    END_HANDLE_TH_ERRORS
}

// layer_bwd(x .. saved, dout, stream) -> dict of gradients
PyObject* py_layer_bwd(PyObject*, PyObject* const* argv, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 13) Py_RETURN_NONE;
    Args a{argv};
    ss_layer_bwd_params q{};
    void* stream = a.stream(12);
    if (!a.ok || !layer_inputs(a, 0, q.fwd)) Py_RETURN_NONE;
    const at::Tensor &x = *a.tensor(0), &cw = *a.tensor(2), &cb = *a.tensor(3), &wx = *a.tensor(4), &wdt = *a.tensor(5), &bias = *a.tensor(6),
                     &A = *a.tensor(7), &D = *a.tensor(8);
    q.dout = a.ptr(11, x.scalar_type(), {q.fwd.batch, q.fwd.dim, q.fwd.seqlen});
    if (!a.ok) Py_RETURN_NONE;
    const char* const names[] = {"dx", "dz", "dconv_w", "dconv_b", "dW_x", "dW_dt", "ddt_bias", "dA", "dD"};
    const at::Tensor g[] = {at::empty_like(x), at::empty_like(x), at::empty_like(cw), at::empty_like(cb), empty_f32(wx.sizes(), x),
                            empty_f32(wdt.sizes(), x), at::empty_like(bias), at::empty_like(A), at::empty_like(D)};
    auto f = [&](int i) { return static_cast<float*>(g[i].data_ptr()); };
    q.dx = g[0].data_ptr(); q.dz = g[1].data_ptr();
    q.dconv_w = f(2); q.dconv_b = f(3); q.dW_x = f(4); q.dW_dt = f(5); q.ddt_bias = f(6); q.dA = f(7); q.dD = f(8);
    const int rc = call(ss_layer_bwd, q, stream);
    if (rc != SS_OK) return PyLong_FromLong(rc);
    PyObject* res = PyDict_New();
    if (!res) return nullptr;
    for (int i = 0; i < 9; ++i) {
        PyObject* o = wrapped(g[i]);
        const bool good = o && PyDict_SetItemString(res, names[i], o) == 0;
        Py_XDECREF(o);
        if (!good) {
            Py_DECREF(res);
            return nullptr;
        }
    }
    return res;
    END_HANDLE_TH_ERRORS
}

// ---- layer norm, gated recurrence, 8-bit products --------------------------------------------------
PyObject* wrapped_or_none(const at::Tensor& t)
{
    if (t.defined()) return wrapped(t);
    Py_RETURN_NONE;
}
PyObject* tuple_of(std::initializer_list<at::Tensor> ts)
{
    PyObject* res = PyTuple_New((Py_ssize_t)ts.size());
    if (!res) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor& t : ts) {
        PyObject* o = wrapped_or_none(t);
        if (!o) {
            Py_DECREF(res);
            return nullptr;
        }
        PyTuple_SET_ITEM(res, i++, o);
    }
    return res;
}
struct Named {
    const char* name;
    const at::Tensor& t;
};
PyObject* dict_of(std::initializer_list<Named> ts)
{
    PyObject* res = PyDict_New();
    if (!res) return nullptr;
    for (const Named& n : ts) {
        PyObject* o = wrapped_or_none(n.t);
        const bool good = o && PyDict_SetItemString(res, n.name, o) == 0;
        Py_XDECREF(o);
        if (!good) {
            Py_DECREF(res);
            return nullptr;
        }
    }
    return res;
}
template <typename T = void>
T* data(const at::Tensor& t) { return t.defined() ? static_cast<T*>(t.data_ptr()) : nullptr; }
at::Tensor empty_bytes(size_t n, const at::Tensor& like)
{
    return at::empty({(int64_t)(n < 256 ? 256 : n)}, like.options().dtype(at::kByte).requires_grad(false));
}
at::Tensor empty_io(const at::Tensor& like) { return at::empty(like.sizes(), like.options().requires_grad(false)); }

// rows and width of a tensor whose last axis is normalised
bool norm_sizes(const at::Tensor& x, ss_norm_params& p)
{
    if (x.dim() < 1 || !io_type(x, p.io_dtype)) return false;
    const int64_t width = x.size(-1), rows = width ? x.numel() / width : 0;
    if (!fits(width) || !fits(rows)) return false;
    p.rows = (int32_t)rows;
    p.width = (int32_t)width;
    return true;
}
// a tensor of x's shape held in float32 or in x's type
const at::Tensor* held(Args& a, int i, const at::Tensor& x)
{
    const at::Tensor* t = a.tensor(i);
    if (!t) return nullptr;
    if (!t->sizes().equals(x.sizes()) || (t->scalar_type() != at::kFloat && t->scalar_type() != x.scalar_type())) {
        a.ok = false;
        return nullptr;
    }
    return t;
}

// The calls themselves, on tensors that have been looked at.  They hold no lock and are also what the gradient functions call.
struct Norm {
    at::Tensor out, summed, stats;
    int fwd(const at::Tensor& x, const at::Tensor& weight, const at::Tensor& bias, const at::Tensor& residual, double eps, bool rms, bool save, void* stream)
    {
        ss_norm_params p{};
        if (!norm_sizes(x, p)) return SS_ERR_SHAPE;
        p.eps = (float)eps;
        p.x = x.data_ptr();
        p.weight = data<const float>(weight);
        p.bias = data<const float>(bias);
        p.flags = (weight.defined() ? SS_NORM_HAS_WEIGHT : 0u) | (bias.defined() ? SS_NORM_HAS_BIAS : 0u) | (rms ? SS_NORM_RMS : 0u);
        out = empty_io(x);
        p.out = out.data_ptr();
        if (residual.defined()) {
            p.flags |= SS_NORM_HAS_RESIDUAL | (residual.scalar_type() == at::kFloat ? SS_NORM_RESIDUAL_F32 : 0u);
            p.residual = residual.data_ptr();
            summed = empty_io(residual);
            p.summed = summed.data_ptr();
        }
        if (save) {
            p.flags |= SS_NORM_SAVE_STATS;
            stats = rms ? empty_f32({p.rows}, x) : empty_f32({2, p.rows}, x);
            p.stats = data<float>(stats);
        }
        return ss_norm_fwd(&p, stream);
    }
};
struct NormGrads {
    at::Tensor dx, dresidual, dweight, dbias;
    int bwd(const at::Tensor& dout, const at::Tensor& s, const at::Tensor& stats, const at::Tensor& weight, bool has_bias, bool res, const at::Tensor& more,
            double eps, bool rms, void* stream)
    {
        ss_norm_bwd_params q{};
        ss_norm_params& p = q.fwd;
        if (!norm_sizes(dout, p)) return SS_ERR_SHAPE;
        p.eps = (float)eps;
        p.flags = rms ? SS_NORM_RMS : 0u;
        p.stats = data<float>(stats);
        p.weight = data<const float>(weight);
        dx = empty_io(dout);
        const bool two = res && s.scalar_type() != dout.scalar_type();
        if (res) {
            p.flags |= SS_NORM_HAS_RESIDUAL | (s.scalar_type() == at::kFloat ? SS_NORM_RESIDUAL_F32 : 0u);
            p.summed = s.data_ptr();
            dresidual = two ? empty_io(s) : dx;
        } else {
            p.x = s.data_ptr();
        }
        if (weight.defined()) {
            p.flags |= SS_NORM_HAS_WEIGHT;
            dweight = empty_f32({p.width}, dout);
        }
        if (has_bias) {
            p.flags |= SS_NORM_HAS_BIAS;
            dbias = empty_f32({p.width}, dout);
        }
        q.dout = dout.data_ptr();
        q.dsummed = data<const void>(more);
        q.dx = dx.data_ptr();
        q.dresidual = two ? dresidual.data_ptr() : nullptr;
        q.dweight = data<float>(dweight);
        q.dbias = data<float>(dbias);
        const at::Tensor ws = empty_bytes(ss_norm_workspace_bytes(&p), dout);
        q.workspace = ws.data_ptr();
        q.workspace_bytes = (size_t)ws.numel();
        return ss_norm_bwd(&q, stream);
    }
};
// Whether the forward call's tensors are the plain case; they are left in `t` (x, weight, bias, residual).
bool norm_tensors(Args& a, int at, at::Tensor (&t)[4])
{
    const at::Tensor* x = a.tensor(at);
    ss_norm_params p{};
    if (!x || !norm_sizes(*x, p)) return false;
    a.ptr(at + 1, at::kFloat, {p.width}, true);
    a.ptr(at + 2, at::kFloat, {p.width}, true);
    if (a.ok && !a.none(at + 3)) held(a, at + 3, *x);
    if (!a.ok) return false;
    for (int i = 0; i < 4; ++i)
        if (!a.none(at + i)) t[i] = THPVariable_Unpack(a.a[at + i]);
    return true;
}
// Whether a tensor lies on the device whose stream the call takes.
bool on_device(const at::Tensor& t, long device) { return t.is_cuda() && t.device().index() == device; }
bool all_on_device(const at::Tensor (&t)[4], long device)
{
    for (const at::Tensor& v : t)
        if (v.defined() && !on_device(v, device)) return false;
    return true;
}
bool real_number(PyObject* o, double& v)
{
    if (!PyFloat_CheckExact(o)) return false;
    v = PyFloat_AS_DOUBLE(o);
    return true;
}
struct Unlocked {   // without the interpreter's lock, also where an exception passes
    PyThreadState* state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};
struct Refused {    // the library's code on its way out of a gradient function's forward call
    int rc;
};
typedef std::optional<at::Tensor> Optional;   // what an input of a gradient function is that may be missing
at::Tensor given(const Optional& t) { return t.has_value() ? *t : at::Tensor(); }
Optional optional(const at::Tensor& t) { return t.defined() ? Optional(t) : Optional(); }
void backward_check(int rc) { TORCH_CHECK(rc == SS_OK, "ss_scan error ", rc, ": ", ss_strerror(rc)); }

// norm_fwd(x, weight, bias, residual, eps, rms, save, stream, device) -> (out, summed or None, stats or None)
PyObject* py_norm_fwd(PyObject*, PyObject* const* argv, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 9) Py_RETURN_NONE;
    Args a{argv};
    at::Tensor t[4];
    double eps;
    if (!norm_tensors(a, 0, t) || !real_number(argv[4], eps)) Py_RETURN_NONE;
    void* stream = a.stream(7);
    if (!all_on_device(t, a.number(8)) || !a.ok) Py_RETURN_NONE;
    Norm c;
    int rc;
    {
        Unlocked u;
        rc = c.fwd(t[0], t[1], t[2], t[3], eps, argv[5] == Py_True, argv[6] == Py_True, stream);
    }
    if (rc != SS_OK) return PyLong_FromLong(rc);
    return tuple_of({c.out, c.summed, c.stats});
    END_HANDLE_TH_ERRORS
}

// norm_quant(x, weight, bias, residual, eps, rms, stream, device) -> (q, scale, summed or None)
PyObject* py_norm_quant(PyObject*, PyObject* const* argv, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 8) Py_RETURN_NONE;
    Args a{argv};
    at::Tensor t[4];
    double eps;
    if (!norm_tensors(a, 0, t) || !real_number(argv[4], eps)) Py_RETURN_NONE;
    void* stream = a.stream(6);
    ss_norm_quant_params p{};
    if (!all_on_device(t, a.number(7)) || !a.ok || !norm_sizes(t[0], p.fwd) || !p.fwd.width) Py_RETURN_NONE;
    p.fwd.eps = (float)eps;
    p.fwd.flags = argv[5] == Py_True ? SS_NORM_RMS : 0u;
    p.fwd.x = t[0].data_ptr();
    p.fwd.weight = data<const float>(t[1]);
    p.fwd.bias = data<const float>(t[2]);
    if (t[1].defined()) p.fwd.flags |= SS_NORM_HAS_WEIGHT;
    if (t[2].defined()) p.fwd.flags |= SS_NORM_HAS_BIAS;
    at::Tensor summed;
    if (t[3].defined()) {
        p.fwd.flags |= SS_NORM_HAS_RESIDUAL | (t[3].scalar_type() == at::kFloat ? SS_NORM_RESIDUAL_F32 : 0u);
        p.fwd.residual = t[3].data_ptr();
        summed = empty_io(t[3]);
        p.fwd.summed = summed.data_ptr();
    }
    const at::Tensor q = at::empty({p.fwd.rows, (int64_t)ss_quant_pitch(p.fwd.width)}, t[0].options().dtype(at::kChar).requires_grad(false));
    const at::Tensor scale = empty_f32({p.fwd.rows}, t[0]);
    p.q = static_cast<int8_t*>(q.data_ptr());
    p.scale = data<float>(scale);
    const int rc = call(ss_norm_quant, p, stream);
    if (rc != SS_OK) return PyLong_FromLong(rc);
    return tuple_of({q, scale, summed});
    END_HANDLE_TH_ERRORS
}

// norm_bwd(dout, s, stats, weight, has_bias, has_residual, dsummed, eps, rms, stream, device) -> dict of gradients
PyObject* py_norm_bwd(PyObject*, PyObject* const* argv, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 11) Py_RETURN_NONE;
    Args a{argv};
    ss_norm_params p{};
    const at::Tensor* dout = a.tensor(0);
    double eps;
    if (!dout || !norm_sizes(*dout, p) || !real_number(argv[7], eps)) Py_RETURN_NONE;
    const bool res = argv[5] == Py_True;
    const at::Tensor* s = held(a, 1, *dout);
    if (!s || (!res && (s->scalar_type() != dout->scalar_type() || !a.none(6)))) Py_RETURN_NONE;
    const bool rms = argv[8] == Py_True;
    if (rms) a.ptr(2, at::kFloat, {p.rows});
    else a.ptr(2, at::kFloat, {2, p.rows});
    a.ptr(3, at::kFloat, {p.width}, true);
    const at::Tensor* more = a.ok && !a.none(6) ? held(a, 6, *dout) : nullptr;
    void* stream = a.stream(9);
    const long device = a.number(10);
    if (!a.ok || (more && more->scalar_type() != s->scalar_type())) Py_RETURN_NONE;
    const at::Tensor& stats = THPVariable_Unpack(argv[2]);
    const at::Tensor weight = a.none(3) ? at::Tensor() : THPVariable_Unpack(argv[3]), dsummed = more ? *more : at::Tensor();
    if (!on_device(*dout, device) || !all_on_device({*s, stats, weight, dsummed}, device)) Py_RETURN_NONE;
    NormGrads g;
    int rc;
    {
        Unlocked u;
        rc = g.bwd(*dout, *s, stats, weight, argv[4] == Py_True, res, dsummed, eps, rms, stream);
    }
    if (rc != SS_OK) return PyLong_FromLong(rc);
    return dict_of({{"dx", g.dx}, {"dresidual", g.dresidual}, {"dweight", g.dweight}, {"dbias", g.dbias}});
    END_HANDLE_TH_ERRORS
}

// Layer norm and RMS norm as a node of torch's graph (what autograd._LayerNorm is in Python): the backward pass runs on the stream of the forward pass,
// which is also the one that torch makes current for it.
// A backward pass's gradients have no graph of their own: where one is being built, they are connected to what they depend on through
// an error, so that going through them again is refused whichever way it is asked for.
torch::autograd::variable_list differentiable_once(torch::autograd::variable_list grads, std::initializer_list<const torch::autograd::variable_list*> from)
{
    if (!at::GradMode::is_enabled()) return grads;
    torch::autograd::variable_list sources;
    for (const auto* list : from)
        for (const at::Tensor& t : *list)
            if (t.defined() && t.requires_grad()) sources.push_back(t);
    if (sources.empty()) return grads;
    const std::shared_ptr<torch::autograd::Node> error(
        new torch::autograd::Error("the gradients of this operator cannot be differentiated again", torch::autograd::collect_next_edges(sources)),
        torch::autograd::deleteNode);
    for (at::Tensor& g : grads)
        if (g.defined()) {
            g = g.detach();
            torch::autograd::create_gradient_edge(g, error);
        }
    return grads;
}
struct NormFunction : torch::autograd::Function<NormFunction> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, const Optional& weight_, const Optional& bias_,
                                                  const Optional& residual_, double eps, bool rms, int64_t stream)
    {
        const at::Tensor weight = given(weight_), bias = given(bias_), residual = given(residual_);
        Norm c;
        const int rc = c.fwd(x, weight, bias, residual, eps, rms, true, reinterpret_cast<void*>(stream));
        if (rc != SS_OK) throw Refused{rc};
        ctx->set_materialize_grads(false);
        ctx->save_for_backward({residual.defined() ? c.summed : x, weight, c.stats});
        ctx->saved_data["bias"] = bias.defined();
        ctx->saved_data["residual"] = residual.defined();
        ctx->saved_data["eps"] = eps;
        ctx->saved_data["rms"] = rms;
        ctx->saved_data["stream"] = stream;
        ctx->saved_data["io"] = (int64_t)x.scalar_type();
        if (residual.defined()) return {c.out, c.summed};
        return {c.out};
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        const bool res = ctx->saved_data["residual"].toBool();
        const at::Tensor more = res && grads[1].defined() ? grads[1].contiguous() : at::Tensor();
        if (!grads[0].defined()) {   // only the sum was used
            const auto io = (at::ScalarType)ctx->saved_data["io"].toInt();
            return differentiable_once({more.defined() ? more.to(io) : at::Tensor(), at::Tensor(), at::Tensor(), more, at::Tensor(), at::Tensor(), at::Tensor()}, {&grads});
        }
        const auto saved = ctx->get_saved_variables();
        NormGrads g;
        backward_check(g.bwd(grads[0].contiguous(), saved[0], saved[2], saved[1], ctx->saved_data["bias"].toBool(), res, more,
                             ctx->saved_data["eps"].toDouble(), ctx->saved_data["rms"].toBool(), reinterpret_cast<void*>(ctx->saved_data["stream"].toInt())));
        return differentiable_once({g.dx, g.dweight, g.dbias, g.dresidual, at::Tensor(), at::Tensor(), at::Tensor()}, {&saved, &grads});
    }
};
// layer_norm(x, weight, bias, residual, eps, rms, stream, device) -> (out,) or (out, summed), with gradients
PyObject* py_layer_norm(PyObject*, PyObject* const* argv, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 8) Py_RETURN_NONE;
    Args a{argv};
    at::Tensor t[4];
    double eps;
    if (!norm_tensors(a, 0, t) || !real_number(argv[4], eps)) Py_RETURN_NONE;
    const bool rms = argv[5] == Py_True;
    void* stream = a.stream(6);
    if (!all_on_device(t, a.number(7)) || !a.ok) Py_RETURN_NONE;
    torch::autograd::variable_list r;
    try {
        Unlocked u;
        r = NormFunction::apply(t[0], optional(t[1]), optional(t[2]), optional(t[3]), eps, rms, reinterpret_cast<int64_t>(stream));
    } catch (const Refused& e) {
        return PyLong_FromLong(e.rc);
    }
    return r.size() == 2 ? tuple_of({r[0], r[1]}) : tuple_of({r[0]});
    END_HANDLE_TH_ERRORS
}

// A (B,D,L) or (B,D) tensor whose batch entries are dense.
void* rows_of(Args& a, int i, at::ScalarType io, at::IntArrayRef shape, int64_t& batch)
{
    if (a.none(i) || !a.ok) return nullptr;
    if (!THPVariable_CheckExact(a.a[i])) { a.ok = false; return nullptr; }
    const at::Tensor& t = THPVariable_Unpack(a.a[i]);
    if (!t.is_cuda() || !t.has_storage() || t.scalar_type() != io || !t.sizes().equals(shape)) { a.ok = false; return nullptr; }
    int64_t dense = 1;
    for (size_t k = shape.size(); k-- > 1;) {
        if (shape[k] != 1 && t.stride((int64_t)k) != dense) { a.ok = false; return nullptr; }
        dense *= shape[k];
    }
    batch = shape[0] == 1 ? dense : t.stride(0);
    if (batch < dense) { a.ok = false; return nullptr; }
    return t.data_ptr();
}
// x, f, i, z, rate, f_bias, i_bias from argument `at` on
template <typename P>
bool gate_inputs(Args& a, int at, const at::Tensor& x, P& p, const void*& px, const void*& pf, const void*& pi, const void*& pz)
{
    if (!io_type(x, p.io_dtype) || !fits(x.size(0)) || !fits(x.size(1))) return false;
    const at::ScalarType io = x.scalar_type();
    const int64_t nd = x.size(1);
    p.batch = (int32_t)x.size(0);
    p.dim = (int32_t)nd;
    px = rows_of(a, at, io, x.sizes(), p.x_batch);
    pf = rows_of(a, at + 1, io, x.sizes(), p.f_batch);
    pi = rows_of(a, at + 2, io, x.sizes(), p.i_batch);
    pz = rows_of(a, at + 3, io, x.sizes(), p.z_batch);
    p.rate = static_cast<const float*>(a.ptr(at + 4, at::kFloat, {nd}));
    p.f_bias = static_cast<const float*>(a.ptr(at + 5, at::kFloat, {nd}, true));
    p.i_bias = static_cast<const float*>(a.ptr(at + 6, at::kFloat, {nd}, true));
    if (!a.ok || a.none(at + 1) || (a.none(at + 2) && !a.none(at + 6))) return false;
    p.flags |= (a.none(at + 2) ? 0u : SS_GATE_HAS_I) | (a.none(at + 3) ? 0u : SS_GATE_HAS_Z) | (a.none(at + 5) ? 0u : SS_GATE_HAS_F_BIAS) |
               (a.none(at + 6) ? 0u : SS_GATE_HAS_I_BIAS);
    return true;
}
const uint8_t* marks_of(Args& a, int i, Shape shape)
{
    if (a.none(i) || !a.ok) return nullptr;
    const at::Tensor* t = a.tensor(i);
    if (!t) return nullptr;
    if ((t->scalar_type() != at::kBool && t->scalar_type() != at::kByte) || !t->sizes().equals(at::IntArrayRef(shape))) {
        a.ok = false;
        return nullptr;
    }
    return static_cast<const uint8_t*>(t->data_ptr());
}
const at::Tensor* gate_x(Args& a, int i, int64_t dim)
{
    if (!THPVariable_CheckExact(a.a[i])) return nullptr;
    const at::Tensor& x = THPVariable_Unpack(a.a[i]);
    return x.is_cuda() && x.dim() == dim ? &x : nullptr;
}
// x, f, i, z, rate, f_bias, i_bias, reset, h0
bool gate_all(Args& a, int at, const at::Tensor& x, ss_gate_params& p)
{
    if (!fits(x.size(2)) || !gate_inputs(a, at, x, p, p.x, p.f, p.i, p.z)) return false;
    p.seqlen = (int32_t)x.size(2);
    p.reset = marks_of(a, at + 7, {x.size(0), x.size(2)});
    p.h0 = static_cast<const float*>(a.ptr(at + 8, at::kFloat, {x.size(0), x.size(1)}, true));
    p.flags |= (a.none(at + 7) ? 0u : SS_GATE_HAS_RESET) | (a.none(at + 8) ? 0u : SS_GATE_HAS_H0);
    return a.ok;
}

// The recurrence's calls, with the struct filled by gate_all or by gate_refill.
struct Gate {
    at::Tensor out, h_last;
    int fwd(const at::Tensor& x, ss_gate_params p, const at::Tensor& ws, bool save, bool want_last, void* stream)
    {
        if (ws.defined()) {
            p.workspace = ws.data_ptr();
            p.workspace_bytes = (size_t)ws.numel();
        }
        if (save) p.flags |= SS_GATE_SAVE_FOR_BWD;
        out = at::empty(x.sizes(), x.options().requires_grad(false));
        p.out = out.data_ptr();
        if (want_last) {
            h_last = empty_f32({p.batch, p.dim}, x);
            p.h_last = data<float>(h_last);
            p.flags |= SS_GATE_WRITE_H_LAST;
        }
        return ss_gate_fwd(&p, stream);
    }
};
struct GateGrads {
    at::Tensor dx, df, di, dz, drate, df_bias, di_bias, dh0;
    int bwd(const at::Tensor& x, const ss_gate_params& p, const at::Tensor& ws, const at::Tensor& dout, const at::Tensor& dh_last, bool want_dh0, void* stream)
    {
        ss_gate_bwd_params q{};
        q.fwd = p;
        q.fwd.workspace = ws.data_ptr();
        q.fwd.workspace_bytes = (size_t)ws.numel();
        q.dout = dout.data_ptr();
        q.dh_last = data<const float>(dh_last);
        const int64_t nd = p.dim;
        dx = empty_io(x);
        df = empty_io(x);
        drate = empty_f32({nd}, x);
        if (p.flags & SS_GATE_HAS_I) di = empty_io(x);
        if (p.flags & SS_GATE_HAS_Z) dz = empty_io(x);
        if (p.flags & SS_GATE_HAS_F_BIAS) df_bias = empty_f32({nd}, x);
        if (p.flags & SS_GATE_HAS_I_BIAS) di_bias = empty_f32({nd}, x);
        if (want_dh0) dh0 = empty_f32({p.batch, nd}, x);
        q.dx = dx.data_ptr(); q.df = df.data_ptr(); q.di = data(di); q.dz = data(dz);
        q.dx_batch = q.df_batch = q.di_batch = q.dz_batch = nd * p.seqlen;
        q.drate = data<float>(drate); q.df_bias = data<float>(df_bias); q.di_bias = data<float>(di_bias); q.dh0 = data<float>(dh0);
        return ss_gate_bwd(&q, stream);
    }
};

// gate_fwd(x, f, i, z, rate, f_bias, i_bias, reset, h0, workspace, save, want_last, stream) -> (out, h_last or None)
PyObject* py_gate_fwd(PyObject*, PyObject* const* argv, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 13) Py_RETURN_NONE;
    Args a{argv};
    ss_gate_params p{};
    const at::Tensor* x = gate_x(a, 0, 3);
    void* stream = a.stream(12);
    if (!x || !a.ok || !gate_all(a, 0, *x, p)) Py_RETURN_NONE;
    at::Tensor ws;
    const bool save = argv[10] == Py_True;
    if (!a.none(9)) {
        const at::Tensor* t = a.tensor(9);
        if (!t || t->scalar_type() != at::kByte) Py_RETURN_NONE;
        ws = *t;
    } else if (save) {
        Py_RETURN_NONE;
    } else {
        const size_t need = ss_gate_workspace_bytes(&p, 0);
        if (need) ws = empty_bytes(need, *x);
    }
    Gate g;
    int rc;
    {
        Unlocked u;
        rc = g.fwd(*x, p, ws, save, argv[11] == Py_True, stream);
    }
    if (rc != SS_OK) return PyLong_FromLong(rc);
    return tuple_of({g.out, g.h_last});
    END_HANDLE_TH_ERRORS
}

// gate_bwd(x, f, i, z, rate, f_bias, i_bias, reset, h0, workspace, dout, dh_last, want_dh0, stream) -> dict of gradients
PyObject* py_gate_bwd(PyObject*, PyObject* const* argv, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 14) Py_RETURN_NONE;
    Args a{argv};
    ss_gate_params p{};
    const at::Tensor* x = gate_x(a, 0, 3);
    void* stream = a.stream(13);
    if (!x || !a.ok || !gate_all(a, 0, *x, p)) Py_RETURN_NONE;
    const at::Tensor* ws = a.tensor(9);
    if (!ws || ws->scalar_type() != at::kByte) Py_RETURN_NONE;
    a.ptr(10, x->scalar_type(), {p.batch, p.dim, p.seqlen});
    a.ptr(11, at::kFloat, {p.batch, p.dim}, true);
    if (!a.ok) Py_RETURN_NONE;
    const at::Tensor dh_last = a.none(11) ? at::Tensor() : THPVariable_Unpack(argv[11]);
    GateGrads g;
    int rc;
    {
        Unlocked u;
        rc = g.bwd(*x, p, *ws, THPVariable_Unpack(argv[10]), dh_last, argv[12] == Py_True, stream);
    }
    if (rc != SS_OK) return PyLong_FromLong(rc);
    return dict_of({{"dx", g.dx}, {"df", g.df}, {"di", g.di}, {"dz", g.dz}, {"drate", g.drate}, {"df_bias", g.df_bias}, {"di_bias", g.di_bias}, {"dh0", g.dh0}});
    END_HANDLE_TH_ERRORS
}

// The recurrence as a node of torch's graph (what autograd._GatedRecurrence is in Python).
struct GateFunction : torch::autograd::Function<GateFunction> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, const at::Tensor& f, const Optional& i,
                                                  const Optional& z, const at::Tensor& rate, const Optional& f_bias, const Optional& i_bias,
                                                  const Optional& reset, const Optional& h0, bool want_last, const ss_gate_params* p, int64_t stream)
    {
        const at::Tensor ws = empty_bytes(ss_gate_workspace_bytes(p, 1), x);
        Gate g;
        const int rc = g.fwd(x, *p, ws, true, want_last, reinterpret_cast<void*>(stream));
        if (rc != SS_OK) throw Refused{rc};
        ctx->save_for_backward({x, f, given(i), given(z), rate, given(f_bias), given(i_bias), given(reset), given(h0), ws});
        ctx->saved_data["flags"] = (int64_t)p->flags;
        ctx->saved_data["stream"] = stream;
        if (want_last) return {g.out, g.h_last};
        return {g.out};
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        const auto t = ctx->get_saved_variables();
        const at::Tensor& x = t[0];
        ss_gate_params p{};
        io_type(x, p.io_dtype);
        p.batch = (int32_t)x.size(0); p.dim = (int32_t)x.size(1); p.seqlen = (int32_t)x.size(2);
        p.flags = (uint32_t)ctx->saved_data["flags"].toInt();
        const int64_t dense = x.size(1) * x.size(2);
        auto rows = [&](const at::Tensor& v, int64_t& batch) {
            batch = v.defined() && x.size(0) > 1 ? v.stride(0) : dense;
            return data<const void>(v);
        };
        p.x = rows(t[0], p.x_batch); p.f = rows(t[1], p.f_batch); p.i = rows(t[2], p.i_batch); p.z = rows(t[3], p.z_batch);
        p.rate = data<const float>(t[4]); p.f_bias = data<const float>(t[5]); p.i_bias = data<const float>(t[6]);
        p.reset = data<const uint8_t>(t[7]); p.h0 = data<const float>(t[8]);
        GateGrads g;
        backward_check(g.bwd(x, p, t[9], grads[0].contiguous(), grads.size() > 1 ? grads[1].contiguous() : at::Tensor(), t[8].defined(),
                             reinterpret_cast<void*>(ctx->saved_data["stream"].toInt())));
        return differentiable_once({g.dx, g.df, g.di, g.dz, g.drate, g.df_bias, g.di_bias, at::Tensor(), g.dh0, at::Tensor(), at::Tensor(), at::Tensor()}, {&t, &grads});
    }
};
// gated_recurrence(x, f, i, z, rate, f_bias, i_bias, reset, h0, want_last, stream) -> (out,) or (out, h_last), with gradients
PyObject* py_gated_recurrence(PyObject*, PyObject* const* argv, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 11) Py_RETURN_NONE;
    Args a{argv};
    ss_gate_params p{};
    const at::Tensor* x = gate_x(a, 0, 3);
    void* stream = a.stream(10);
    if (!x || !a.ok || !gate_all(a, 0, *x, p)) Py_RETURN_NONE;
    at::Tensor t[9];
    for (int i = 0; i < 9; ++i)
        if (!a.none(i)) t[i] = THPVariable_Unpack(argv[i]);
    torch::autograd::variable_list r;
    try {
        Unlocked u;
        r = GateFunction::apply(t[0], t[1], optional(t[2]), optional(t[3]), t[4], optional(t[5]), optional(t[6]), optional(t[7]), optional(t[8]), argv[9] == Py_True, &p, reinterpret_cast<int64_t>(stream));
    } catch (const Refused& e) {
        return PyLong_FromLong(e.rc);
    }
    return r.size() == 2 ? tuple_of({r[0], r[1]}) : tuple_of({r[0]});
    END_HANDLE_TH_ERRORS
}

// gate_step(x_t, f_t, i_t, z_t, rate, f_bias, i_bias, reset_t, h, out_t, stream) -> out_t
PyObject* py_gate_step(PyObject*, PyObject* const* argv, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 11) Py_RETURN_NONE;
    Args a{argv};
    ss_gate_step_params p{};
    const at::Tensor* x = gate_x(a, 0, 2);
    void* stream = a.stream(10);
    if (!x || !a.ok || !gate_inputs(a, 0, *x, p, p.x_t, p.f_t, p.i_t, p.z_t)) Py_RETURN_NONE;
    p.reset_t = marks_of(a, 7, {p.batch});
    if (!a.none(7)) p.flags |= SS_GATE_HAS_RESET;
    p.h = static_cast<float*>(a.ptr(8, at::kFloat, {p.batch, p.dim}));
    void* out = a.ptr(9, x->scalar_type(), {p.batch, p.dim}, true);
    if (!a.ok) Py_RETURN_NONE;
    at::Tensor fresh;
    if (a.none(9)) {
        fresh = empty_io(*x);
        out = fresh.data_ptr();
    }
    p.out_t = out;
    const int rc = call(ss_gate_step, p, stream);
    if (rc != SS_OK) return PyLong_FromLong(rc);
    if (a.none(9)) return wrapped(fresh);
    Py_INCREF(argv[9]);
    return argv[9];
    END_HANDLE_TH_ERRORS
}

// The type of a code of io types; `ok` falls if it is none.
at::ScalarType type_of_code(long code, bool& ok)
{
    if (code == SS_F32) return at::kFloat;
    if (code != SS_BF16) ok = false;
    return at::kBFloat16;
}
// qlinear(x, weight, scale, bias, flags, x_scale or None, dim, type of the result, stream) -> out, scratch of the call's own; dim and the type are looked at where
// there is x_scale: the tokens are quantised (else x's)
PyObject* py_qlinear(PyObject*, PyObject* const* argv, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 9) Py_RETURN_NONE;
    Args a{argv};
    ss_qlinear_params p{};
    const at::Tensor *x = a.tensor(0), *w = a.ok ? a.tensor(1) : nullptr;
    p.flags = (uint32_t)a.number(4);
    void* stream = a.stream(8);
    const bool quantised = !a.none(5);
    if (!a.ok || w->dim() != 2 || x->dim() < 1) Py_RETURN_NONE;
    const at::ScalarType io = quantised ? (a.none(7) ? at::kBFloat16 : type_of_code(a.number(7), a.ok)) : x->scalar_type();
    if (!a.ok || (!quantised && !io_type(*x, p.io_dtype))) Py_RETURN_NONE;
    const bool x_last = p.flags & SS_Q_X_SEQ_LAST, out_last = p.flags & SS_Q_OUT_SEQ_LAST;
    if ((x_last || out_last) && x->dim() != 3) Py_RETURN_NONE;
    if (quantised && (x_last || x->scalar_type() != at::kChar)) Py_RETURN_NONE;
    const int64_t dim = quantised ? a.number(6) : (x_last ? x->size(1) : x->size(-1)), features = w->size(0);
    if (!a.ok || dim < 1 || !fits(dim) || !fits(features)) Py_RETURN_NONE;
    const int64_t batch = x_last || out_last ? x->size(0) : 1, seqlen = x_last ? x->size(2) : (out_last ? x->size(1) : x->numel() / std::max<int64_t>(x->size(-1), 1));
    if (!fits(batch) || !fits(seqlen)) Py_RETURN_NONE;
    p.batch = (int32_t)batch; p.seqlen = (int32_t)seqlen; p.dim = (int32_t)dim; p.features = (int32_t)features;
    p.x = x->data_ptr();
    p.weight = a.ptr(1, at::kChar, {features, (int64_t)ss_quant_pitch((int32_t)dim)});
    p.scale = static_cast<const float*>(a.ptr(2, at::kFloat, {features}));
    p.bias = static_cast<const float*>(a.ptr(3, at::kFloat, {features}, true));
    if (quantised) {
        p.flags |= SS_Q_X_QUANTISED;
        p.io_dtype = io == at::kFloat ? SS_F32 : SS_BF16;
        p.x_scale = static_cast<const float*>(a.ptr(5, at::kFloat, {batch * seqlen}));
        if (x->size(-1) != (int64_t)ss_quant_pitch((int32_t)dim)) Py_RETURN_NONE;
    }
    if (!a.ok) Py_RETURN_NONE;
    if (p.bias) p.flags |= SS_Q_HAS_BIAS;
    at::Tensor out;
    const at::TensorOptions options = x->options().dtype(io).requires_grad(false);
    if (out_last) out = at::empty({batch, features, seqlen}, options);
    else if (x_last) out = at::empty({batch, seqlen, features}, options);
    else {
        c10::SmallVector<int64_t, 6> shape(x->sizes().begin(), x->sizes().end());
        shape.back() = features;
        out = at::empty(shape, options);
    }
    p.out = out.data_ptr();
    const at::Tensor ws = empty_bytes(ss_qlinear_scratch_bytes(&p), *x);
    p.scratch = ws.data_ptr();
    p.scratch_bytes = (size_t)ws.numel();
    const int rc = call(ss_qlinear, p, stream);
    if (rc != SS_OK) return PyLong_FromLong(rc);
    return wrapped(out);
    END_HANDLE_TH_ERRORS
}

// ---- embedding, log probabilities, AdamW -----------------------------------------------------------
// whole numbers in 64 or 32 bits
bool whole_type(const at::Tensor& t, uint32_t flag_of_32, uint32_t& flags)
{
    if (t.scalar_type() == at::kInt) flags |= flag_of_32;
    else if (t.scalar_type() != at::kLong) return false;
    return true;
}
struct Embed {
    at::Tensor out;
    int fwd(const at::Tensor& ids, const at::Tensor& table, double scale, at::ScalarType type, void* stream)
    {
        ss_embed_params p{};
        if (!sizes(p, ids, table.size(0), table.size(1), scale) || !io_type(table, p.table_dtype)) return SS_ERR_UNSUPPORTED;
        c10::SmallVector<int64_t, 6> shape(ids.sizes().begin(), ids.sizes().end());
        shape.push_back(table.size(1));
        out = at::empty(shape, table.options().dtype(type).requires_grad(false));
        io_type(out, p.io_dtype);
        p.table = table.data_ptr();
        p.out = out.data_ptr();
        return ss_embed_fwd(&p, stream);
    }
    int bwd(const at::Tensor& dout, const at::Tensor& ids, int64_t vocab, double scale, at::ScalarType type, void* stream)
    {
        ss_embed_bwd_params q{};
        ss_embed_params& p = q.fwd;
        if (!sizes(p, ids, vocab, dout.size(-1), scale) || !io_type(dout, p.io_dtype)) return SS_ERR_UNSUPPORTED;
        out = at::empty({vocab, dout.size(-1)}, dout.options().dtype(type).requires_grad(false));
        io_type(out, p.table_dtype);
        q.dout = dout.data_ptr();
        q.dtable = out.data_ptr();
        const at::Tensor ws = empty_bytes(ss_embed_workspace_bytes(&p), dout);
        q.workspace = ws.data_ptr();
        q.workspace_bytes = (size_t)ws.numel();
        return ss_embed_bwd(&q, stream);
    }
    static bool sizes(ss_embed_params& p, const at::Tensor& ids, int64_t vocab, int64_t dim, double scale)
    {
        if (!fits(ids.numel()) || !fits(vocab) || !fits(dim) || !whole_type(ids, SS_EMBED_IDS_32, p.flags)) return false;
        p.tokens = (int32_t)ids.numel(); p.vocab = (int32_t)vocab; p.dim = (int32_t)dim;
        p.scale = (float)scale;
        p.ids = ids.data_ptr();
        return true;
    }
};
// ids, table, scale, type of the result, stream, device
bool embed_inputs(Args& a, double& scale, at::ScalarType& type, void*& stream)
{
    const at::Tensor *ids = a.tensor(0), *table = a.ok ? a.tensor(1) : nullptr;
    if (!a.ok || table->dim() != 2 || !real_number(a.a[2], scale)) return false;
    int32_t code;
    uint32_t flags = 0;
    if (!io_type(*table, code) || !whole_type(*ids, SS_EMBED_IDS_32, flags)) return false;
    type = a.none(3) ? table->scalar_type() : type_of_code(a.number(3), a.ok);
    stream = a.stream(4);
    const long device = a.number(5);
    return a.ok && on_device(*ids, device) && on_device(*table, device) && fits(ids->numel()) && fits(table->size(0)) && fits(table->size(1));
}
// embed_fwd(ids, table, scale, type or None, stream, device) -> out
PyObject* py_embed_fwd(PyObject*, PyObject* const* argv, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 6) Py_RETURN_NONE;
    Args a{argv};
    double scale;
    at::ScalarType type;
    void* stream;
    if (!embed_inputs(a, scale, type, stream)) Py_RETURN_NONE;
    Embed e;
    int rc;
    {
        Unlocked u;
        rc = e.fwd(THPVariable_Unpack(argv[0]), THPVariable_Unpack(argv[1]), scale, type, stream);
    }
    if (rc != SS_OK) return PyLong_FromLong(rc);
    return wrapped(e.out);
    END_HANDLE_TH_ERRORS
}
// The embedding as a node of torch's graph (what autograd._Embedding is in Python).
struct EmbedFunction : torch::autograd::Function<EmbedFunction> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const at::Tensor& ids, const at::Tensor& table, double scale, int64_t type, int64_t stream)
    {
        Embed e;
        const int rc = e.fwd(ids, table, scale, (at::ScalarType)type, reinterpret_cast<void*>(stream));
        if (rc != SS_OK) throw Refused{rc};
        ctx->save_for_backward({ids});
        ctx->saved_data["vocab"] = table.size(0);
        ctx->saved_data["scale"] = scale;
        ctx->saved_data["type"] = (int64_t)table.scalar_type();
        ctx->saved_data["stream"] = stream;
        return {e.out};
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        const auto saved = ctx->get_saved_variables();
        Embed e;
        backward_check(e.bwd(grads[0].contiguous(), saved[0], ctx->saved_data["vocab"].toInt(), ctx->saved_data["scale"].toDouble(),
                             (at::ScalarType)ctx->saved_data["type"].toInt(), reinterpret_cast<void*>(ctx->saved_data["stream"].toInt())));
        return differentiable_once({at::Tensor(), e.out, at::Tensor(), at::Tensor(), at::Tensor()}, {&grads});
    }
};
// embedding(ids, table, scale, type or None, stream, device) -> out, with a gradient
PyObject* py_embedding(PyObject*, PyObject* const* argv, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 6) Py_RETURN_NONE;
    Args a{argv};
    double scale;
    at::ScalarType type;
    void* stream;
    if (!embed_inputs(a, scale, type, stream)) Py_RETURN_NONE;
    torch::autograd::variable_list r;
    try {
        Unlocked u;
        r = EmbedFunction::apply(THPVariable_Unpack(argv[0]), THPVariable_Unpack(argv[1]), scale, (int64_t)type, reinterpret_cast<int64_t>(stream));
    } catch (const Refused& e) {
        return PyLong_FromLong(e.rc);
    }
    return wrapped(r[0]);
    END_HANDLE_TH_ERRORS
}

// Rows of logits, which may lie in wider ones: elements from one to the next; 0 where they are not equally far from each other, or overlap.
int64_t row_stride(const at::Tensor& t)
{
    const int64_t width = t.size(-1);
    if (t.is_contiguous()) return width;
    if (t.stride(-1) != 1 && width != 1) return 0;
    int64_t stride = width, at = 0;
    bool first = true;
    for (int64_t k = t.dim() - 1; k-- > 0;) {
        if (t.size(k) == 1) continue;
        if (first) stride = t.stride(k);
        else if (t.stride(k) != at) return 0;
        first = false;
        at = t.stride(k) * t.size(k);
    }
    return stride < width ? 0 : stride;
}
struct Logprob {
    at::Tensor logp, entropy, stats, top_logp, top_ids;
    static bool sizes(ss_logprob_params& p, const at::Tensor& x, const at::Tensor& targets)
    {
        if (x.dim() < 1 || x.size(-1) < 1 || !io_type(x, p.io_dtype)) return false;
        const int64_t rows = x.numel() / x.size(-1);
        p.row_stride = row_stride(x);
        if (!p.row_stride || !fits(rows) || !fits(x.size(-1))) return false;
        p.rows = (int32_t)rows; p.vocab = (int32_t)x.size(-1);
        p.logits = x.data_ptr();
        if (targets.defined()) {
            if (!whole_type(targets, SS_LOGPROB_TARGETS_32, p.flags) || !targets.sizes().equals(x.sizes().slice(0, x.dim() - 1))) return false;
            p.targets = targets.data_ptr();
        }
        return true;
    }
    int fwd(const at::Tensor& x, const at::Tensor& targets, int64_t top, void* stream)
    {
        ss_logprob_params p{};
        if (!sizes(p, x, targets)) return SS_ERR_SHAPE;
        p.top = (int32_t)top;
        const at::IntArrayRef shape = x.sizes().slice(0, x.dim() - 1);
        if (targets.defined()) logp = empty_f32(shape, x);
        entropy = empty_f32(shape, x);
        stats = empty_f32({2, p.rows}, x);
        p.logp = data<float>(logp); p.entropy = data<float>(entropy); p.stats = data<float>(stats);
        if (top) {
            c10::SmallVector<int64_t, 6> wide(shape.begin(), shape.end());
            wide.push_back(top);
            top_logp = empty_f32(wide, x);
            top_ids = at::empty(wide, x.options().dtype(at::kLong).requires_grad(false));
            p.top_logp = data<float>(top_logp); p.top_ids = data<int64_t>(top_ids);
        }
        at::Tensor ws;
        if (const size_t need = ss_logprob_workspace_bytes(&p)) {
            ws = empty_bytes(need, x);
            p.workspace = ws.data_ptr();
            p.workspace_bytes = (size_t)ws.numel();
        }
        return ss_logprob_fwd(&p, stream);
    }
};
int logprob_bwd(const at::Tensor& x, const at::Tensor& targets, const at::Tensor& entropy, const at::Tensor& stats, const at::Tensor& dlogp, const at::Tensor& dentropy,
                at::Tensor& out, void* stream)
{
    ss_logprob_bwd_params q{};
    if (!Logprob::sizes(q.fwd, x, targets)) return SS_ERR_SHAPE;
    q.fwd.stats = data<float>(stats);
    q.fwd.entropy = data<float>(entropy);
    q.dlogp = data<const float>(dlogp);
    q.dentropy = data<const float>(dentropy);
    out = at::empty(x.sizes(), x.options().requires_grad(false));
    q.dlogits = out.data_ptr();
    return ss_logprob_bwd(&q, stream);
}
// logits, targets or None, top, stream, device
bool logprob_inputs(Args& a, at::Tensor& x, at::Tensor& targets, int64_t& top, void*& stream)
{
    if (!THPVariable_CheckExact(a.a[0])) return false;
    x = THPVariable_Unpack(a.a[0]);
    const long device = a.number(4);
    if (!x.has_storage() || !on_device(x, device)) return false;
    if (!a.none(1)) {
        const at::Tensor* t = a.tensor(1);
        if (!t || !on_device(*t, device)) return false;
        targets = *t;
    }
    top = a.number(2);
    stream = a.stream(3);
    ss_logprob_params p{};
    return a.ok && Logprob::sizes(p, x, targets) && top >= 0 && top <= SS_LOGPROB_MAX_TOP && top <= p.vocab;
}
// logprob_fwd(logits, targets or None, top, stream, device) -> (logp or None, entropy, stats, top_logp or None, top_ids or None)
PyObject* py_logprob_fwd(PyObject*, PyObject* const* argv, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 5) Py_RETURN_NONE;
    Args a{argv};
    at::Tensor x, targets;
    int64_t top;
    void* stream;
    if (!logprob_inputs(a, x, targets, top, stream)) Py_RETURN_NONE;
    Logprob l;
    int rc;
    {
        Unlocked u;
        rc = l.fwd(x, targets, top, stream);
    }
    if (rc != SS_OK) return PyLong_FromLong(rc);
    return tuple_of({l.logp, l.entropy, l.stats, l.top_logp, l.top_ids});
    END_HANDLE_TH_ERRORS
}
// Log probabilities as a node of torch's graph (what autograd._TokenLogprobs is in Python).
struct LogprobFunction : torch::autograd::Function<LogprobFunction> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, const at::Tensor& targets, int64_t top, int64_t stream)
    {
        Logprob l;
        const int rc = l.fwd(x, targets, top, reinterpret_cast<void*>(stream));
        if (rc != SS_OK) throw Refused{rc};
        ctx->set_materialize_grads(false);
        ctx->save_for_backward({x, targets, l.entropy, l.stats});
        ctx->saved_data["stream"] = stream;
        if (!top) return {l.logp, l.entropy};
        ctx->mark_non_differentiable({l.top_logp, l.top_ids});
        return {l.logp, l.entropy, l.top_logp, l.top_ids};
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        if (!grads[0].defined() && !grads[1].defined()) return {at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor()};
        const auto t = ctx->get_saved_variables();
        at::Tensor dx;
        auto dense = [](const at::Tensor& v) { return v.defined() ? v.contiguous() : v; };
        const at::Tensor dlogp = dense(grads[0]), dentropy = dense(grads[1]);
        backward_check(logprob_bwd(t[0], t[1], t[2], t[3], dlogp, dentropy, dx, reinterpret_cast<void*>(ctx->saved_data["stream"].toInt())));
        return differentiable_once({dx, at::Tensor(), at::Tensor(), at::Tensor()}, {&t, &grads});
    }
};
// token_logprobs(logits, targets, top, stream, device) -> (logp, entropy) or (logp, entropy, top_logp, top_ids), with gradients
PyObject* py_token_logprobs(PyObject*, PyObject* const* argv, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 5) Py_RETURN_NONE;
    Args a{argv};
    at::Tensor x, targets;
    int64_t top;
    void* stream;
    if (!logprob_inputs(a, x, targets, top, stream) || !targets.defined()) Py_RETURN_NONE;
    torch::autograd::variable_list r;
    try {
        Unlocked u;
        r = LogprobFunction::apply(x, targets, top, reinterpret_cast<int64_t>(stream));
    } catch (const Refused& e) {
        return PyLong_FromLong(e.rc);
    }
    return r.size() == 2 ? tuple_of({r[0], r[1]}) : tuple_of({r[0], r[1], r[2], r[3]});
    END_HANDLE_TH_ERRORS
}

// Plain tensors of a list, all on one device; `ok` falls when one of them is not.
struct Listed {
    PyObject* list;
    Py_ssize_t n = 0;
    bool ok = true;
    Listed(PyObject* o, bool optional) : list(o)
    {
        if (optional && o == Py_None) list = nullptr;
        else if (!PyList_CheckExact(o)) ok = false;
        else n = PyList_GET_SIZE(o);
    }
    const at::Tensor* at(Py_ssize_t k, const at::Tensor* like, bool optional = false)
    {
        PyObject* o = PyList_GET_ITEM(list, k);
        if (optional && o == Py_None) return nullptr;
        if (!THPVariable_CheckExact(o)) { ok = false; return nullptr; }
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda() || !t.has_storage() || !t.is_contiguous() || (like && t.device() != like->device())) { ok = false; return nullptr; }
        return &t;
    }
};
const float* one_float(PyObject* o, const at::Tensor& like, bool& ok)
{
    if (o == Py_None) return nullptr;
    if (!THPVariable_CheckExact(o)) { ok = false; return nullptr; }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.has_storage() || t.device() != like.device() || t.scalar_type() != at::kFloat || t.numel() != 1) { ok = false; return nullptr; }
    return static_cast<const float*>(t.data_ptr());
}
// adamw_step(params, grads, m, v, masters or None, m_scales or None, v_scales or None, count, lr, lr tensor or None, beta1, beta2, eps, weight_decay,
//            grad_scale or None, stream) -> True
PyObject* py_adamw_step(PyObject*, PyObject* const* argv, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 16) Py_RETURN_NONE;
    Args a{argv};
    const at::Tensor* count = a.tensor(7);
    if (!a.ok || count->scalar_type() != at::kInt || count->numel() != 2) Py_RETURN_NONE;
    Listed params(argv[0], false), grads(argv[1], false), m(argv[2], false), v(argv[3], false), masters(argv[4], true), ms(argv[5], true), vs(argv[6], true);
    if (!params.ok || !grads.ok || !m.ok || !v.ok || !masters.ok || !ms.ok || !vs.ok) Py_RETURN_NONE;
    const bool eight = ms.list && vs.list;
    const Py_ssize_t all = params.n;
    if (grads.n != all || m.n != all || v.n != all || (masters.list && masters.n != all) || (eight && (ms.n != all || vs.n != all)) ||
        (!ms.list != !vs.list) || !fits(all))
        Py_RETURN_NONE;
    ss_adamw_params p{};
    if (!real_number(argv[8], p.lr) || !real_number(argv[10], p.beta1) || !real_number(argv[11], p.beta2) || !real_number(argv[12], p.eps) ||
        !real_number(argv[13], p.weight_decay))
        Py_RETURN_NONE;
    bool ok = true;
    p.lr_device = one_float(argv[9], *count, ok);
    p.grad_scale = one_float(argv[14], *count, ok);
    void* stream = a.stream(15);
    if (!ok || !a.ok) Py_RETURN_NONE;
    std::vector<ss_adamw_tensor> list((size_t)all);
    std::vector<void*> seen;
    seen.reserve((size_t)all);
    const at::ScalarType m_type = eight ? at::kChar : at::kFloat, v_type = eight ? at::kByte : at::kFloat;
    for (Py_ssize_t k = 0; k < all; ++k) {
        ss_adamw_tensor& e = list[(size_t)k];
        const at::Tensor *t = params.at(k, count), *g = grads.at(k, count), *tm = m.at(k, count), *tv = v.at(k, count);
        const at::Tensor* master = masters.list ? masters.at(k, count, true) : nullptr;
        if (!params.ok || !grads.ok || !m.ok || !v.ok || !masters.ok) Py_RETURN_NONE;
        e.n = t->numel();
        if (!io_type(*t, e.param_dtype) || !io_type(*g, e.grad_dtype) || tm->scalar_type() != m_type || tv->scalar_type() != v_type) Py_RETURN_NONE;
        if (!g->sizes().equals(t->sizes()) || !tm->sizes().equals(t->sizes()) || !tv->sizes().equals(t->sizes())) Py_RETURN_NONE;
        if (master && (master->scalar_type() != at::kFloat || e.param_dtype != SS_BF16 || !master->sizes().equals(t->sizes()))) Py_RETURN_NONE;
        if (eight) {
            const at::Tensor *a1 = ms.at(k, count), *a2 = vs.at(k, count);
            const int64_t blocks = (e.n + SS_ADAMW_BLOCK - 1) / SS_ADAMW_BLOCK;
            if (!ms.ok || !vs.ok || a1->scalar_type() != at::kFloat || a2->scalar_type() != at::kFloat || a1->dim() != 1 || a2->dim() != 1 ||
                a1->numel() != blocks || a2->numel() != blocks)
                Py_RETURN_NONE;
            e.m_scale = data<float>(*a1);
            e.v_scale = data<float>(*a2);
        }
        e.param = t->data_ptr();
        e.grad = g->data_ptr();
        e.master = master ? data<float>(*master) : nullptr;
        e.m = tm->data_ptr();
        e.v = tv->data_ptr();
        if (e.n) seen.push_back(e.param);
    }
    std::sort(seen.begin(), seen.end());
    if (std::adjacent_find(seen.begin(), seen.end()) != seen.end()) Py_RETURN_NONE;
    p.tensors = (int32_t)all;
    p.state_bits = eight ? 8 : 32;
    p.list = list.data();
    p.count = static_cast<int32_t*>(count->data_ptr());
    const int rc = call(ss_adamw_step, p, stream);
    if (rc != SS_OK) return PyLong_FromLong(rc);
    Py_RETURN_TRUE;
    END_HANDLE_TH_ERRORS
}

#define SS_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(py_##name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {SS_METHOD(step), SS_METHOD(layer_step), SS_METHOD(scan_fwd), SS_METHOD(scan_bwd),
                         SS_METHOD(layer_fwd), SS_METHOD(layer_bwd), SS_METHOD(norm_fwd), SS_METHOD(norm_quant), SS_METHOD(norm_bwd), SS_METHOD(gate_fwd),
                         SS_METHOD(gate_bwd), SS_METHOD(gate_step), SS_METHOD(qlinear), SS_METHOD(layer_norm), SS_METHOD(gated_recurrence), SS_METHOD(adamw_step),
                         SS_METHOD(embed_fwd), SS_METHOD(embedding), SS_METHOD(logprob_fwd), SS_METHOD(token_logprobs), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
