// The well-formed calls of the Python binding, marshalled natively: a small call's time is its marshalling (per call, 60 in a row: forward
// and backward of 2 heads x 128 tokens 25 us for 15 us of kernels, a decode step of 8 x 16 heads against 273 keys 11.8 for 6.9; what an
// argument costs is its attributes read from Python and its ctypes conversion).  Every function here does what its namesake in
// __init__.py does for plain torch tensors that pass all of that function's checks, and returns None for anything else, without having
// done anything: the Python text then runs and raises what there is to raise.  An int is the library's error code.
#include <Python.h>
#include <ATen/ATen.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "../../include/attn.h"

namespace {

// entry points of libattn.so, which the package loads: addresses given once (bind)
decltype(&attn_fwd_dtype) p_fwd = nullptr;
decltype(&attn_bwd_phases) p_bwd_phases = nullptr;
decltype(&attn_bwd_dtype) p_bwd_dtype = nullptr;
decltype(&attn_bwd_workspace_bytes) p_bwd_bytes = nullptr;
decltype(&attn_varlen_fwd_dtype) p_varlen_fwd = nullptr;
decltype(&attn_varlen_bwd_dtype) p_varlen_bwd = nullptr;
decltype(&attn_varlen_workspace_bytes) p_varlen_bytes = nullptr;
decltype(&attn_fwd_strided) p_fwd_strided = nullptr;
decltype(&attn_bwd_strided) p_bwd_strided = nullptr;
decltype(&attn_strided_workspace_bytes) p_strided_bytes = nullptr;
decltype(&attn_rope_fwd) p_rope_fwd = nullptr;
decltype(&attn_rope_bwd) p_rope_bwd = nullptr;
decltype(&attn_rope_workspace_bytes) p_rope_bytes = nullptr;
decltype(&attn_cache_write) p_cache_write = nullptr;
decltype(&attn_cache_read) p_cache_read = nullptr;
decltype(&attn_cache_fwd) p_cache_fwd = nullptr;
decltype(&attn_cache_workspace_bytes) p_cache_bytes = nullptr;
PyObject *get_device = nullptr, *get_stream = nullptr;      // torch._C._cuda_getDevice, _cuda_getCurrentRawStream
PyTypeObject* parameter = nullptr;                          // torch.nn.Parameter

using Sizes = std::initializer_list<int64_t>;

// A plain tensor (no subclass that may have a say in what happens to it), or null.
const at::Tensor* plain(PyObject* x)
{
    if (Py_TYPE(x) != (PyTypeObject*)THPVariableClass && Py_TYPE(x) != parameter) return nullptr;
    return &THPVariable_Unpack(x);
}

// Arguments of one call.  `ok` falls with the first that is not as the Python text wants it.
struct Call {
    bool ok = true;
    at::ScalarType type = at::kBFloat16;
    int dtype = ATTN_BF16;
    attn_strides_t strides[8];
    int nstrides = 0;

    bool fits(int64_t x)
    {
        if (x < 0 || x > 0x7fffffff) ok = false;
        return ok;
    }
    // the first tensor gives the element type
    const at::Tensor* first(PyObject* x, int64_t dims)
    {
        const at::Tensor* t = plain(x);
        if (!t || t->dim() != dims || !t->is_cuda()) { ok = false; return nullptr; }
        type = t->scalar_type();
        if (type != at::kBFloat16 && type != at::kHalf) ok = false;
        dtype = type == at::kHalf ? ATTN_F16 : ATTN_BF16;
        for (int64_t n : t->sizes()) fits(n);
        return ok ? t : nullptr;
    }
    const at::Tensor* other(PyObject* x, int64_t dims)
    {
        const at::Tensor* t = ok ? plain(x) : nullptr;
        if (!t || t->dim() != dims) { ok = false; return nullptr; }
        for (int64_t n : t->sizes()) fits(n);
        return ok ? t : nullptr;
    }
    void* dense(const at::Tensor& t, Sizes shape, at::ScalarType as)
    {
        if (!ok || !t.is_cuda() || t.scalar_type() != as || !t.is_contiguous() || t.sizes() != at::IntArrayRef(shape)) { ok = false; return nullptr; }
        return t.data_ptr();
    }
    void* view(const at::Tensor& t, Sizes shape)
    {
        if (!ok || !t.is_cuda() || t.scalar_type() != type || t.sizes() != at::IntArrayRef(shape) || (t.stride(3) != 1 && t.size(3) != 1)) { ok = false; return nullptr; }
        strides[nstrides++] = {t.stride(0), t.stride(1), t.stride(2)};
        return t.data_ptr();
    }
    // an optional output: the caller's, or (made by `make`, once every check has passed) a new one
    at::Tensor given(PyObject* x)
    {
        if (x == Py_None || !ok) return at::Tensor();
        const at::Tensor* t = plain(x);
        if (!t) ok = false;
        return t ? *t : at::Tensor();
    }
    double number(PyObject* x)
    {
        if (PyFloat_CheckExact(x)) return PyFloat_AS_DOUBLE(x);
        ok = false;
        return 0;
    }
    int truth(PyObject* x)
    {
        if (x == Py_True || x == Py_False) return x == Py_True;
        ok = false;
        return 0;
    }
    // the stream's handle, or the current one of the current device; called after every other check
    void* stream(PyObject* x)
    {
        PyObject* h = nullptr;
        if (x != Py_None) {
            h = PyObject_GetAttrString(x, "cuda_stream");
        } else if (PyObject* d = PyObject_CallNoArgs(get_device)) {
            h = PyObject_CallOneArg(get_stream, d);
            Py_DECREF(d);
        }
        void* s = h && PyLong_Check(h) ? PyLong_AsVoidPtr(h) : nullptr;
        if (!h || !PyLong_Check(h) || PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        Py_XDECREF(h);
        return s;
    }
};

int size(const at::Tensor* t, int dim) { return (int)t->size(dim); }       // (Call::fits)

at::Tensor make(const at::Tensor& like, Sizes shape) { return at::empty(shape, like.options().requires_grad(false)); }
at::Tensor make_f32(const at::Tensor& like, Sizes shape) { return at::empty(shape, like.options().requires_grad(false).dtype(at::kFloat)); }
at::Tensor make_bytes(const at::Tensor& like, size_t n)
{
    return at::empty({(int64_t)(n < 256 ? 256 : n)}, like.options().requires_grad(false).dtype(at::kByte));
}

// What goes back: the caller's own objects, or new tensors.
PyObject* out(PyObject* mine, const at::Tensor& t)
{
    if (mine != Py_None) { Py_INCREF(mine); return mine; }
    return THPVariable_Wrap(t);
}
PyObject* outs(int rc, std::initializer_list<std::pair<PyObject*, const at::Tensor*>> list)
{
    if (rc != ATTN_OK) return PyLong_FromLong(rc);
    PyObject* r = PyTuple_New((Py_ssize_t)list.size());
    Py_ssize_t i = 0;
    for (const auto& x : list) PyTuple_SET_ITEM(r, i++, out(x.first, *x.second));
    return r;
}

// Other Python threads run while this lives: allocations, which may wait for memory, and the library's call, as with torch.empty and ctypes.
struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    Unlocked() = default;
    Unlocked(const Unlocked&) = delete;
    ~Unlocked() { PyEval_RestoreThread(state); }
};

#define NOT_HERE Py_RETURN_NONE

// q, k, v, scale, causal, o, lse, stream
PyObject* fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Call c;
    if (n != 8) NOT_HERE;
    const at::Tensor *q = c.first(a[0], 4), *k = c.other(a[1], 4), *v = c.other(a[2], 4);
    if (!c.ok) NOT_HERE;
    const int B = size(q, 0), N = size(q, 1), H = size(q, 2), dqk = size(q, 3), Hkv = size(k, 2), dv = size(v, 3);
    const double scale = c.number(a[3]);
    const int causal = c.truth(a[4]);
    at::Tensor o = c.given(a[5]), lse = c.given(a[6]);
    void *qp = c.dense(*q, {B, N, H, dqk}, c.type), *kp = c.dense(*k, {B, N, Hkv, dqk}, c.type), *vp = c.dense(*v, {B, N, Hkv, dv}, c.type);
    if (o.defined()) c.dense(o, {B, N, H, dv}, c.type);
    if (lse.defined()) c.dense(lse, {B, H, N}, at::kFloat);
    if (!c.ok) NOT_HERE;
    void* s = c.stream(a[7]);
    if (!c.ok) NOT_HERE;
    int rc;
    {
        Unlocked threads;
        if (!o.defined()) o = make(*q, {B, N, H, dv});
        if (!lse.defined()) lse = make_f32(*q, {B, H, N});
        rc = p_fwd(c.dtype, qp, kp, vp, o.data_ptr(), (float*)lse.data_ptr(), B, H, Hkv, N, dqk, dv, (float)scale, causal, s);
    }
    return outs(rc, {{a[5], &o}, {a[6], &lse}});
    END_HANDLE_TH_ERRORS
}

// q, k, v, o, do, lse, scale, causal, dq, dk, dv, workspace, stream, phases
PyObject* bwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Call c;
    if (n != 14 || !PyLong_CheckExact(a[13])) NOT_HERE;
    const at::Tensor *q = c.first(a[0], 4), *k = c.other(a[1], 4), *v = c.other(a[2], 4), *o = c.other(a[3], 4), *g = c.other(a[4], 4), *lse = c.other(a[5], 3);
    if (!c.ok) NOT_HERE;
    const long phases = PyLong_AsLong(a[13]);
    if (PyErr_Occurred()) { PyErr_Clear(); NOT_HERE; }
    const int B = size(q, 0), N = size(q, 1), H = size(q, 2), dqk = size(q, 3), Hkv = size(k, 2), dvd = size(v, 3);
    const double scale = c.number(a[6]);
    const int causal = c.truth(a[7]);
    at::Tensor dq = c.given(a[8]), dk = c.given(a[9]), dv = c.given(a[10]), ws = c.given(a[11]);
    void *qp = c.dense(*q, {B, N, H, dqk}, c.type), *kp = c.dense(*k, {B, N, Hkv, dqk}, c.type), *vp = c.dense(*v, {B, N, Hkv, dvd}, c.type),
         *op = c.dense(*o, {B, N, H, dvd}, c.type), *gp = c.dense(*g, {B, N, H, dvd}, c.type), *lp = c.dense(*lse, {B, H, N}, at::kFloat);
    if (dq.defined()) c.dense(dq, {B, N, H, dqk}, c.type);
    if (dk.defined()) c.dense(dk, {B, N, Hkv, dqk}, c.type);
    if (dv.defined()) c.dense(dv, {B, N, Hkv, dvd}, c.type);
    if (!c.ok || (phases != ATTN_BWD_ALL && (c.type == at::kHalf || phases < 0 || phases > ATTN_BWD_ALL))) NOT_HERE;
    const size_t need = p_bwd_bytes(B, H, Hkv, N, dqk, dvd);
    if (need == 0 || (ws.defined() && !ws.is_cuda())) NOT_HERE;
    void* s = c.stream(a[12]);
    if (!c.ok) NOT_HERE;
    int rc;
    {
        Unlocked threads;
        if (!dq.defined()) dq = make(*q, {B, N, H, dqk});
        if (!dk.defined()) dk = make(*q, {B, N, Hkv, dqk});
        if (!dv.defined()) dv = make(*q, {B, N, Hkv, dvd});
        if (!ws.defined()) ws = make_bytes(*q, need);
        const size_t bytes = (size_t)ws.numel() * ws.element_size();
        rc = c.type == at::kHalf
            ? p_bwd_dtype(c.dtype, qp, kp, vp, op, gp, (float*)lp, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), B, H, Hkv, N, dqk, dvd, (float)scale, causal,
                          ws.data_ptr(), bytes, s)
            : p_bwd_phases(qp, kp, vp, op, gp, (float*)lp, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), B, H, Hkv, N, dqk, dvd, (float)scale, causal,
                           ws.data_ptr(), bytes, s, (int)phases);
    }
    return outs(rc, {{a[8], &dq}, {a[9], &dk}, {a[10], &dv}});
    END_HANDLE_TH_ERRORS
}

// Boundaries [B + 1] on the device; both given here (tables kept in a workspace: the Python text).
const int* boundaries(Call& c, PyObject* x, int B)
{
    const at::Tensor* t = c.ok ? plain(x) : nullptr;
    if (!t) { c.ok = false; return nullptr; }
    return (const int*)c.dense(*t, {(int64_t)B + 1}, at::kInt);
}

// q, k, v, cu_seqlens, scale, causal, o, lse, workspace, stream, cu_seqlens_k
PyObject* varlen_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Call c;
    if (n != 11) NOT_HERE;
    const at::Tensor *q = c.first(a[0], 3), *k = c.other(a[1], 3), *v = c.other(a[2], 3), *cu = c.other(a[3], 1);
    if (!c.ok) NOT_HERE;
    const int T = size(q, 0), H = size(q, 1), dqk = size(q, 2), Tk = size(k, 0), Hkv = size(k, 1), dv = size(v, 2), B = size(cu, 0) - 1;
    const double scale = c.number(a[4]);
    const int causal = c.truth(a[5]);
    const int *cq = boundaries(c, a[3], B), *ck = a[10] == Py_None ? cq : boundaries(c, a[10], B);
    at::Tensor o = c.given(a[6]), lse = c.given(a[7]), ws = c.given(a[8]);
    void *qp = c.dense(*q, {T, H, dqk}, c.type), *kp = c.dense(*k, {Tk, Hkv, dqk}, c.type), *vp = c.dense(*v, {Tk, Hkv, dv}, c.type);
    if (o.defined()) c.dense(o, {T, H, dv}, c.type);
    if (lse.defined()) c.dense(lse, {H, T}, at::kFloat);
    if (!c.ok || B < 1) NOT_HERE;
    const size_t need = ws.defined() ? 0 : p_varlen_bytes(B, T, Tk, H, Hkv, dqk, dv, 0);
    void* s = c.stream(a[9]);
    if (!c.ok) NOT_HERE;
    int rc;
    {
        Unlocked threads;
        if (!o.defined()) o = make(*q, {T, H, dv});
        if (!lse.defined()) lse = make_f32(*q, {H, T});
        if (!ws.defined()) ws = make_bytes(*q, need);
        rc = p_varlen_fwd(c.dtype, qp, kp, vp, o.data_ptr(), (float*)lse.data_ptr(), cq, ck, B, T, Tk, H, Hkv, dqk, dv, (float)scale, causal,
                          ws.data_ptr(), (size_t)ws.numel(), s);
    }
    return outs(rc, {{a[6], &o}, {a[7], &lse}});
    END_HANDLE_TH_ERRORS
}

// q, k, v, o, d_o, lse, cu_seqlens, scale, causal, dq, dk, dv, workspace, stream, cu_seqlens_k
PyObject* varlen_bwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Call c;
    if (n != 15) NOT_HERE;
    const at::Tensor *q = c.first(a[0], 3), *k = c.other(a[1], 3), *v = c.other(a[2], 3), *o = c.other(a[3], 3), *g = c.other(a[4], 3), *lse = c.other(a[5], 2),
                     *cu = c.other(a[6], 1);
    if (!c.ok) NOT_HERE;
    const int T = size(q, 0), H = size(q, 1), dqk = size(q, 2), Tk = size(k, 0), Hkv = size(k, 1), dvd = size(v, 2), B = size(cu, 0) - 1;
    const double scale = c.number(a[7]);
    const int causal = c.truth(a[8]);
    const int *cq = boundaries(c, a[6], B), *ck = a[14] == Py_None ? cq : boundaries(c, a[14], B);
    at::Tensor dq = c.given(a[9]), dk = c.given(a[10]), dv = c.given(a[11]), ws = c.given(a[12]);
    void *qp = c.dense(*q, {T, H, dqk}, c.type), *kp = c.dense(*k, {Tk, Hkv, dqk}, c.type), *vp = c.dense(*v, {Tk, Hkv, dvd}, c.type),
         *op = c.dense(*o, {T, H, dvd}, c.type), *gp = c.dense(*g, {T, H, dvd}, c.type), *lp = c.dense(*lse, {H, T}, at::kFloat);
    if (dq.defined()) c.dense(dq, {T, H, dqk}, c.type);
    if (dk.defined()) c.dense(dk, {Tk, Hkv, dqk}, c.type);
    if (dv.defined()) c.dense(dv, {Tk, Hkv, dvd}, c.type);
    if (!c.ok || B < 1) NOT_HERE;
    const size_t need = ws.defined() ? 0 : p_varlen_bytes(B, T, Tk, H, Hkv, dqk, dvd, 1);
    void* s = c.stream(a[13]);
    if (!c.ok) NOT_HERE;
    int rc;
    {
        Unlocked threads;
        if (!dq.defined()) dq = make(*q, {T, H, dqk});
        if (!dk.defined()) dk = make(*q, {Tk, Hkv, dqk});
        if (!dv.defined()) dv = make(*q, {Tk, Hkv, dvd});
        if (!ws.defined()) ws = make_bytes(*q, need);
        rc = p_varlen_bwd(c.dtype, qp, kp, vp, op, gp, (float*)lp, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), cq, ck, B, T, Tk, H, Hkv, dqk, dvd,
                          (float)scale, causal, ws.data_ptr(), (size_t)ws.numel(), s);
    }
    return outs(rc, {{a[9], &dq}, {a[10], &dk}, {a[11], &dv}});
    END_HANDLE_TH_ERRORS
}

// q, k, v, scale, causal, o, lse, workspace, stream
PyObject* fwd_strided(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Call c;
    if (n != 9) NOT_HERE;
    const at::Tensor *q = c.first(a[0], 4), *k = c.other(a[1], 4), *v = c.other(a[2], 4);
    if (!c.ok) NOT_HERE;
    const int B = size(q, 0), N = size(q, 1), H = size(q, 2), dqk = size(q, 3), Nk = size(k, 1), Hkv = size(k, 2), dv = size(v, 3);
    const double scale = c.number(a[3]);
    const int causal = c.truth(a[4]);
    at::Tensor o = c.given(a[5]), lse = c.given(a[6]), ws = c.given(a[7]);
    if (o.defined() && o.dim() != 4) NOT_HERE;
    void *qp = c.view(*q, {B, N, H, dqk}), *kp = c.view(*k, {B, Nk, Hkv, dqk}), *vp = c.view(*v, {B, Nk, Hkv, dv});
    if (o.defined()) c.view(o, {B, N, H, dv});
    if (lse.defined()) c.dense(lse, {B, H, N}, at::kFloat);
    if (!c.ok) NOT_HERE;
    const size_t need = ws.defined() ? 0 : p_strided_bytes(B, H, Hkv, N, Nk, dqk, dv, 0);
    void* s = c.stream(a[8]);
    if (!c.ok) NOT_HERE;
    int rc;
    {
        Unlocked threads;
        if (!o.defined()) { o = make(*q, {B, N, H, dv}); c.view(o, {B, N, H, dv}); }
        if (!lse.defined()) lse = make_f32(*q, {B, H, N});
        if (!ws.defined()) ws = make_bytes(*q, need);
        const attn_strides_t* st = c.strides;
        rc = p_fwd_strided(c.dtype, qp, st, kp, st + 1, vp, st + 2, o.data_ptr(), st + 3, (float*)lse.data_ptr(), B, H, Hkv, N, Nk, dqk, dv, (float)scale,
                           causal, ws.data_ptr(), (size_t)ws.numel(), s);
    }
    return outs(rc, {{a[5], &o}, {a[6], &lse}});
    END_HANDLE_TH_ERRORS
}

// q, k, v, o, d_o, lse, scale, causal, dq, dk, dv, workspace, stream
PyObject* bwd_strided(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Call c;
    if (n != 13) NOT_HERE;
    const at::Tensor *q = c.first(a[0], 4), *k = c.other(a[1], 4), *v = c.other(a[2], 4), *o = c.other(a[3], 4), *g = c.other(a[4], 4), *lse = c.other(a[5], 3);
    if (!c.ok) NOT_HERE;
    const int B = size(q, 0), N = size(q, 1), H = size(q, 2), dqk = size(q, 3), Nk = size(k, 1), Hkv = size(k, 2), dvd = size(v, 3);
    const double scale = c.number(a[6]);
    const int causal = c.truth(a[7]);
    at::Tensor dq = c.given(a[8]), dk = c.given(a[9]), dv = c.given(a[10]), ws = c.given(a[11]);
    for (const at::Tensor* t : {&dq, &dk, &dv}) if (t->defined() && t->dim() != 4) NOT_HERE;
    void *qp = c.view(*q, {B, N, H, dqk}), *kp = c.view(*k, {B, Nk, Hkv, dqk}), *vp = c.view(*v, {B, Nk, Hkv, dvd}), *op = c.view(*o, {B, N, H, dvd}),
         *gp = c.view(*g, {B, N, H, dvd}), *lp = c.dense(*lse, {B, H, N}, at::kFloat);
    // (checked here; their strides are taken below, in the order of the call, once the missing ones exist)
    const int inputs = c.nstrides;
    if (dq.defined()) c.view(dq, {B, N, H, dqk});
    if (dk.defined()) c.view(dk, {B, Nk, Hkv, dqk});
    if (dv.defined()) c.view(dv, {B, Nk, Hkv, dvd});
    if (!c.ok) NOT_HERE;
    const size_t need = ws.defined() ? 0 : p_strided_bytes(B, H, Hkv, N, Nk, dqk, dvd, 1);
    void* s = c.stream(a[12]);
    if (!c.ok) NOT_HERE;
    int rc;
    {
        Unlocked threads;
        if (!dq.defined()) dq = make(*q, {B, N, H, dqk});
        if (!dk.defined()) dk = make(*q, {B, Nk, Hkv, dqk});
        if (!dv.defined()) dv = make(*q, {B, Nk, Hkv, dvd});
        if (!ws.defined()) ws = make_bytes(*q, need);
        c.nstrides = inputs;
        c.view(dq, {B, N, H, dqk});
        c.view(dk, {B, Nk, Hkv, dqk});
        c.view(dv, {B, Nk, Hkv, dvd});
        const attn_strides_t* st = c.strides;
        rc = p_bwd_strided(c.dtype, qp, st, kp, st + 1, vp, st + 2, op, st + 3, gp, st + 4, (float*)lp, dq.data_ptr(), st + 5, dk.data_ptr(), st + 6,
                           dv.data_ptr(), st + 7, B, H, Hkv, N, Nk, dqk, dvd, (float)scale, causal, ws.data_ptr(), (size_t)ws.numel(), s);
    }
    return outs(rc, {{a[8], &dq}, {a[9], &dk}, {a[10], &dv}});
    END_HANDLE_TH_ERRORS
}

// ---- rotary positions and the quantised cache: calls on the current device's current stream (others are left to the Python text)

// A call whose tensors all have to be on one device, the current one.
struct CallHere : Call {
    int64_t device = -1;
    const at::Tensor* tensor(PyObject* x)
    {
        const at::Tensor* t = ok ? plain(x) : nullptr;
        if (!t || !t->is_cuda() || (device >= 0 && t->device().index() != device)) { ok = false; return nullptr; }
        device = t->device().index();
        for (int64_t n : t->sizes()) fits(n);
        return ok ? t : nullptr;
    }
    // [B, N, heads, d] or [T, heads, d] with a contiguous last axis; its strides are noted (0 along axes of one)
    void* rows(const at::Tensor* t, at::ScalarType as, at::IntArrayRef shape = {})
    {
        const int64_t n = t ? t->dim() : 0;
        if (!ok || (n != 3 && n != 4) || t->scalar_type() != as || (t->stride(n - 1) != 1 && t->size(n - 1) != 1) || (!shape.empty() && t->sizes() != shape)) {
            ok = false;
            return nullptr;
        }
        auto step = [&](int64_t i) -> long long { return i >= 0 && t->size(i) > 1 ? t->stride(i) : 0; };
        strides[nstrides++] = {step(n - 4), step(n - 3), step(n - 2)};
        return t->data_ptr();
    }
    void* none() { strides[nstrides++] = {0, 0, 0}; return nullptr; }
    // contiguous, of this type and shape
    void* flat(const at::Tensor* t, at::ScalarType as, at::IntArrayRef shape)
    {
        if (!ok || !t || t->scalar_type() != as || !t->is_contiguous() || t->sizes() != shape) { ok = false; return nullptr; }
        return t->data_ptr();
    }
    int integer(PyObject* x)
    {
        const long n = PyLong_CheckExact(x) ? PyLong_AsLong(x) : -1;
        if (PyErr_Occurred()) PyErr_Clear();
        if (n < 0 || n > 0x7fffffff) ok = false;
        return ok ? (int)n : 0;
    }
    void* stream_here(PyObject* x)
    {
        void* s = nullptr;
        PyObject* d = x == Py_None && ok ? PyObject_CallNoArgs(get_device) : nullptr;
        PyObject* h = d && PyLong_Check(d) && PyLong_AsLong(d) == device ? PyObject_CallOneArg(get_stream, d) : nullptr;
        if (h && PyLong_Check(h)) s = PyLong_AsVoidPtr(h);
        else ok = false;
        if (PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        Py_XDECREF(h);
        Py_XDECREF(d);
        return s;
    }
    void element(const at::Tensor* t)
    {
        if (!t) return;
        type = t->scalar_type();
        if (type != at::kBFloat16 && type != at::kHalf) ok = false;
        dtype = type == at::kHalf ? ATTN_F16 : ATTN_BF16;
    }
};

// B, N, H, Hkv, d of rows q (and k, null: none), whose shapes have to agree
struct RopeSizes {
    int B, N, H, Hkv, d;
    RopeSizes(CallHere& c, const at::Tensor* q, const at::Tensor* k)
    {
        const int64_t n = q ? q->dim() : 0;
        if (!c.ok || (n != 3 && n != 4) || (k && k->dim() != n)) { c.ok = false; B = N = H = Hkv = d = 0; return; }
        B = n == 4 ? size(q, 0) : 1;
        N = size(q, (int)n - 3);
        H = size(q, (int)n - 2);
        d = size(q, (int)n - 1);
        Hkv = k ? size(k, (int)n - 2) : 0;
        for (int64_t i = 0; k && i < n; ++i)
            if (i != n - 2 && k->size(i) != q->size(i)) c.ok = false;
    }
};

// freqs, positions, interleaved, offset, amplitude, eps, q_weight, k_weight at a[0] ... a[7]
attn_rope_t rope_of(CallHere& c, PyObject* const* a, const RopeSizes& z, bool k)
{
    attn_rope_t r = {};
    const at::Tensor* f = c.tensor(a[0]);
    r.freqs = f && f->dim() == 1 ? (const float*)c.flat(f, at::kFloat, f->sizes()) : nullptr;
    if (!r.freqs || f->size(0) > 4096) { c.ok = false; return r; }
    r.rot = 2 * size(f, 0);
    if (a[1] != Py_None) {
        const at::Tensor* p = c.tensor(a[1]);
        const bool each = p && p->dim() == 2;
        const int64_t both[] = {z.B, z.N};
        r.positions = (const int*)c.flat(p, at::kInt, each ? at::IntArrayRef(both, 2) : at::IntArrayRef(both + 1, 1));
        r.positions_batch = each ? z.N : 0;
    }
    r.interleaved = c.truth(a[2]);
    r.offset = c.integer(a[3]);
    r.amplitude = (float)c.number(a[4]);
    r.norm = a[5] != Py_None;
    r.eps = r.norm ? (float)c.number(a[5]) : 0.f;
    if (!r.norm && (a[6] != Py_None || a[7] != Py_None)) c.ok = false;
    if (!k && a[7] != Py_None) c.ok = false;
    const int64_t d = z.d;
    if (a[6] != Py_None) r.q_weight = c.flat(c.tensor(a[6]), c.type, at::IntArrayRef(&d, 1));
    if (a[7] != Py_None) r.k_weight = c.flat(c.tensor(a[7]), c.type, at::IntArrayRef(&d, 1));
    return r;
}

// q, k, freqs, positions, interleaved, offset, amplitude, eps, q_weight, k_weight, q_out, k_out, stream
PyObject* rope_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    CallHere c;
    if (n != 13) NOT_HERE;
    const bool both = a[1] != Py_None;
    const at::Tensor *q = c.tensor(a[0]), *k = both ? c.tensor(a[1]) : nullptr;
    c.element(q);
    const RopeSizes z(c, q, k);
    if (!c.ok || (!both && a[11] != Py_None)) NOT_HERE;
    const attn_rope_t r = rope_of(c, a + 2, z, both);
    void *qp = c.rows(q, c.type), *kp = both ? c.rows(k, c.type) : c.none();
    at::Tensor qo, ko;
    if (a[10] != Py_None) { const at::Tensor* t = c.tensor(a[10]); if (t) qo = *t; }
    if (a[11] != Py_None) { const at::Tensor* t = c.tensor(a[11]); if (t) ko = *t; }
    if (!c.ok) NOT_HERE;
    if (qo.defined() && qo.sizes() != q->sizes()) NOT_HERE;
    if (ko.defined() && ko.sizes() != k->sizes()) NOT_HERE;
    void* s = c.stream_here(a[12]);
    if (!c.ok) NOT_HERE;
    if (qo.defined() && (qo.scalar_type() != c.type || qo.stride(qo.dim() - 1) != 1)) NOT_HERE;
    if (ko.defined() && (ko.scalar_type() != c.type || ko.stride(ko.dim() - 1) != 1)) NOT_HERE;
    int rc;
    {
        Unlocked threads;
        if (!qo.defined()) qo = at::empty(q->sizes(), q->options().requires_grad(false));
        if (both && !ko.defined()) ko = at::empty(k->sizes(), k->options().requires_grad(false));
        void *qop = c.rows(&qo, c.type), *kop = both ? c.rows(&ko, c.type) : c.none();
        const attn_strides_t* st = c.strides;
        rc = p_rope_fwd(c.dtype, &r, qp, st, kp, st + 1, qop, st + 2, kop, st + 3, z.B, z.N, z.H, z.Hkv, z.d, s);
    }
    if (rc != ATTN_OK) return PyLong_FromLong(rc);
    if (!both) return Py_BuildValue("(NO)", out(a[10], qo), Py_None);
    return outs(rc, {{a[10], &qo}, {a[11], &ko}});
    END_HANDLE_TH_ERRORS
}

// dq, dk, freqs, positions, interleaved, offset, amplitude, eps, q_weight, k_weight, q, k, dq_in, dk_in, workspace, stream
PyObject* rope_bwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    CallHere c;
    if (n != 16) NOT_HERE;
    const bool both = a[1] != Py_None, norm = a[7] != Py_None;
    const at::Tensor *g = c.tensor(a[0]), *h = both ? c.tensor(a[1]) : nullptr;
    c.element(g);
    const RopeSizes z(c, g, h);
    if (!c.ok || (norm && (a[10] == Py_None || (a[11] != Py_None) != both)) || (!both && a[13] != Py_None)) NOT_HERE;
    const attn_rope_t r = rope_of(c, a + 2, z, both);
    const at::Tensor *q = norm ? c.tensor(a[10]) : nullptr, *k = norm && both ? c.tensor(a[11]) : nullptr;
    const at::IntArrayRef gs = g->sizes(), hs = both ? h->sizes() : at::IntArrayRef();
    void *gp = c.rows(g, c.type), *hp = both ? c.rows(h, c.type) : c.none();
    void *qp = norm ? c.rows(q, c.type, gs) : c.none(), *kp = norm && both ? c.rows(k, c.type, hs) : c.none();
    at::Tensor gi, hi, wq, wk, ws;
    if (a[12] != Py_None) { const at::Tensor* t = c.tensor(a[12]); if (t) { gi = *t; c.rows(t, c.type, gs); --c.nstrides; } }
    if (a[13] != Py_None) { const at::Tensor* t = c.tensor(a[13]); if (t) { hi = *t; c.rows(t, c.type, hs); --c.nstrides; } }
    if (a[14] != Py_None) { const at::Tensor* t = c.tensor(a[14]); if (t) { ws = *t; if (t->scalar_type() != at::kByte || !t->is_contiguous()) c.ok = false; } }
    if (!c.ok) NOT_HERE;
    const bool sums = r.q_weight || r.k_weight;
    const size_t need = sums && !ws.defined() ? p_rope_bytes(z.B, z.N, z.H, z.Hkv, z.d) : 0;
    void* s = c.stream_here(a[15]);
    if (!c.ok) NOT_HERE;
    int rc;
    {
        Unlocked threads;
        const auto options = g->options().requires_grad(false);
        if (!gi.defined()) gi = at::empty(gs, options);
        if (both && !hi.defined()) hi = at::empty(hs, options);
        if (r.q_weight) wq = make_f32(*g, {z.d});
        if (r.k_weight) wk = make_f32(*g, {z.d});
        if (sums && !ws.defined()) ws = make_bytes(*g, need);
        void *gip = c.rows(&gi, c.type), *hip = both ? c.rows(&hi, c.type) : c.none();
        const attn_strides_t* st = c.strides;
        rc = p_rope_bwd(c.dtype, &r, gp, st, hp, st + 1, qp, st + 2, kp, st + 3, gip, st + 4, hip, st + 5, r.q_weight ? (float*)wq.data_ptr() : nullptr,
                        r.k_weight ? (float*)wk.data_ptr() : nullptr, z.B, z.N, z.H, z.Hkv, z.d, ws.defined() ? ws.data_ptr() : nullptr,
                        ws.defined() ? (size_t)ws.numel() : 0, s);
    }
    if (rc != ATTN_OK) return PyLong_FromLong(rc);
    PyObject* t = PyTuple_New(4);
    PyObject* const mine[] = {a[12], a[13], Py_None, Py_None};
    const at::Tensor* const made[] = {&gi, &hi, &wq, &wk};
    for (Py_ssize_t i = 0; i < 4; ++i) {
        PyObject* x = made[i]->defined() ? out(mine[i], *made[i]) : Py_None;
        if (x == Py_None) Py_INCREF(x);
        PyTuple_SET_ITEM(t, i, x);
    }
    return t;
    END_HANDLE_TH_ERRORS
}

attn_cache_t cache_of(CallHere& c, PyObject* x)
{
    attn_cache_t r = {};
    if (!PyTuple_Check(x) || PyTuple_GET_SIZE(x) != 4) { c.ok = false; return r; }
    const at::Tensor* t[4];
    void* p[4];
    for (int i = 0; i < 4; ++i) {
        t[i] = c.tensor(PyTuple_GET_ITEM(x, i));
        if (!t[i] || t[i]->dim() != 4 || t[i]->scalar_type() != at::kByte || !t[i]->is_contiguous() || t[i]->sizes().slice(0, 3) != t[0]->sizes().slice(0, 3)) {
            c.ok = false;
            return r;
        }
        p[i] = t[i]->data_ptr();
    }
    const int64_t dk = 32 * t[1]->size(3), dv = 32 * t[3]->size(3), bits = t[0]->size(3) == dk ? 8 : 4;
    if (dk > 4096 || dv > 4096 || t[0]->size(3) != dk * bits / 8 || t[2]->size(3) != dv * bits / 8) { c.ok = false; return r; }
    return {p[0], p[1], p[2], p[3], size(t[0], 0), size(t[0], 2), size(t[0], 1), (int)dk, (int)dv, (int)bits};
}

// k, v, slots, cache, stream
PyObject* cache_write(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    CallHere c;
    if (n != 5) NOT_HERE;
    const at::Tensor *k = c.tensor(a[0]), *v = c.tensor(a[1]), *slots = c.tensor(a[2]);
    c.element(k);
    const attn_cache_t cache = cache_of(c, a[3]);
    if (!c.ok || k->dim() != 3) NOT_HERE;
    const int64_t T = k->size(0);
    const int64_t ks[] = {T, cache.Hkv, cache.d_qk}, vs[] = {T, cache.Hkv, cache.d_v};
    void *kp = c.rows(k, c.type, ks), *vp = c.rows(v, c.type, vs), *sp = c.flat(slots, at::kInt, at::IntArrayRef(&T, 1));
    void* s = c.stream_here(a[4]);
    if (!c.ok) NOT_HERE;
    int rc;
    {
        Unlocked threads;
        rc = p_cache_write(c.dtype, &cache, kp, c.strides, vp, c.strides + 1, (const int*)sp, (int)T, s);
    }
    return PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// slots, cache, whether fp16 (bf16 otherwise), k, v, stream
PyObject* cache_read(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    CallHere c;
    if (n != 6) NOT_HERE;
    const at::Tensor* slots = c.tensor(a[0]);
    const attn_cache_t cache = cache_of(c, a[1]);
    const int f16 = c.truth(a[2]);
    if (!c.ok || slots->dim() != 1) NOT_HERE;
    const int64_t T = slots->size(0);
    void* sp = c.flat(slots, at::kInt, at::IntArrayRef(&T, 1));
    const auto as = f16 ? at::kHalf : at::kBFloat16;
    const int64_t ks[] = {T, cache.Hkv, cache.d_qk}, vs[] = {T, cache.Hkv, cache.d_v};
    at::Tensor k, v;
    if (a[3] != Py_None) { const at::Tensor* t = c.tensor(a[3]); c.flat(t, as, ks); if (t) k = *t; }
    if (a[4] != Py_None) { const at::Tensor* t = c.tensor(a[4]); c.flat(t, as, vs); if (t) v = *t; }
    void* s = c.stream_here(a[5]);
    if (!c.ok) NOT_HERE;
    int rc;
    {
        Unlocked threads;
        const auto options = slots->options().requires_grad(false).dtype(as);
        if (!k.defined()) k = at::empty(ks, options);
        if (!v.defined()) v = at::empty(vs, options);
        rc = p_cache_read(f16 ? ATTN_F16 : ATTN_BF16, &cache, (const int*)sp, (int)T, k.data_ptr(), v.data_ptr(), s);
    }
    return outs(rc, {{a[3], &k}, {a[4], &v}});
    END_HANDLE_TH_ERRORS
}

// q, cache, block_table, lens, scale, causal, o, lse, workspace, stream
PyObject* cache_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    CallHere c;
    if (n != 10) NOT_HERE;
    const at::Tensor *q = c.tensor(a[0]), *table = c.tensor(a[2]), *lens = c.tensor(a[3]);
    c.element(q);
    const attn_cache_t cache = cache_of(c, a[1]);
    if (!c.ok || q->dim() != 4 || table->dim() != 2) NOT_HERE;
    const int B = size(q, 0), Nq = size(q, 1), H = size(q, 2), width = size(table, 1);
    const double scale = c.number(a[4]);
    const int causal = c.truth(a[5]);
    const int64_t qs[] = {B, Nq, H, cache.d_qk}, os[] = {B, Nq, H, cache.d_v}, ts[] = {B, width}, ls[] = {B, H, Nq};
    void *qp = c.rows(q, c.type, qs), *tp = c.flat(table, at::kInt, ts), *np = c.flat(lens, at::kInt, at::IntArrayRef(ts, 1));
    at::Tensor o, lse, ws;
    if (a[6] != Py_None) { const at::Tensor* t = c.tensor(a[6]); if (t) o = *t; }
    if (a[7] != Py_None) { const at::Tensor* t = c.tensor(a[7]); c.flat(t, at::kFloat, ls); if (t) lse = *t; }
    if (a[8] != Py_None) { const at::Tensor* t = c.tensor(a[8]); if (t) { ws = *t; if (t->scalar_type() != at::kByte || !t->is_contiguous()) c.ok = false; } }
    if (o.defined()) { c.rows(&o, c.type, os); --c.nstrides; }
    if (!c.ok) NOT_HERE;
    const size_t need = ws.defined() ? 0 : p_cache_bytes(&cache, B, Nq, H, width);
    void* s = c.stream_here(a[9]);
    if (!c.ok) NOT_HERE;
    int rc;
    {
        Unlocked threads;
        if (!o.defined()) o = make(*q, {B, Nq, H, cache.d_v});
        if (!lse.defined()) lse = make_f32(*q, {B, H, Nq});
        if (!ws.defined()) ws = make_bytes(*q, need);
        void* op = c.rows(&o, c.type, os);
        rc = p_cache_fwd(c.dtype, &cache, qp, c.strides, op, c.strides + 1, (float*)lse.data_ptr(), (const int*)tp, width, (const int*)np, B, Nq, H, (float)scale,
                         causal, ws.data_ptr(), (size_t)ws.numel(), s);
    }
    return outs(rc, {{a[6], &o}, {a[7], &lse}});
    END_HANDLE_TH_ERRORS
}

// bind(the addresses, in the order below; _cuda_getDevice, _cuda_getCurrentRawStream, Parameter)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    void** const to[] = {(void**)&p_fwd, (void**)&p_bwd_phases, (void**)&p_bwd_dtype, (void**)&p_bwd_bytes, (void**)&p_varlen_fwd, (void**)&p_varlen_bwd,
                         (void**)&p_varlen_bytes, (void**)&p_fwd_strided, (void**)&p_bwd_strided, (void**)&p_strided_bytes, (void**)&p_rope_fwd, (void**)&p_rope_bwd,
                         (void**)&p_rope_bytes, (void**)&p_cache_write, (void**)&p_cache_read, (void**)&p_cache_fwd, (void**)&p_cache_bytes};
    constexpr int N = sizeof(to) / sizeof(to[0]);
    if (n != N + 3 || !PyType_Check(a[N + 2])) { PyErr_SetString(PyExc_TypeError, "bind: the addresses, two functions, a type"); return nullptr; }
    for (int i = 0; i < N; ++i) {
        *to[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    for (int i = N; i < N + 3; ++i) Py_INCREF(a[i]);
    get_device = a[N];
    get_stream = a[N + 1];
    parameter = (PyTypeObject*)a[N + 2];
    Py_RETURN_NONE;
}

#define METHOD(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(bind), METHOD(fwd), METHOD(bwd), METHOD(varlen_fwd), METHOD(varlen_bwd), METHOD(fwd_strided), METHOD(bwd_strided),
                         METHOD(rope_fwd), METHOD(rope_bwd), METHOD(cache_write), METHOD(cache_read), METHOD(cache_fwd),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit__binding() { return PyModule_Create(&module); }
