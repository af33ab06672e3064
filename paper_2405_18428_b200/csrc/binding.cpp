// CPython module over the C ABI (include/dig_gla.h) for torch CUDA tensors: checks, allocation of results and
// workspace, the current stream and the call, without a line of Python in between.  Through ctypes a call of one
// launch took 14 to 19 us of host time (3.4 us of it to ask for the current stream, 2.6 us per allocation, 0.6 us
// per checked tensor), more than the small problems take on the GPU; here it takes 4 to 5 us, the launch
// included.  dig.py holds the documented functions, which hand their arguments over by position.
// The interpreter lock is released around every library call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <string>
#include <vector>

#include "dig_gla.h"
#include "row_sets.h"

namespace {

using at::Tensor;
using at::ScalarType;

PyObject *g_error = nullptr;        // dig.DigError(status, where)

struct Raised {};                    // a Python exception is set

[[noreturn]] void raise(PyObject *type, const std::string &msg)
{
    PyErr_SetString(type, msg.c_str());
    throw Raised{};
}
void check(int status, const char *where)
{
    if (status == DIG_OK) return;
    PyObject *e = PyObject_CallFunction(g_error, "is", status, where);
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    throw Raised{};
}

// ---- arguments -------------------------------------------------------------------------------------
bool none(PyObject *o) { return o == Py_None; }
const Tensor &tensor(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o)) raise(PyExc_TypeError, std::string(name) + ": need a torch tensor, got " + Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
}
int integer(PyObject *o)
{
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    if (v < INT_MIN || v > INT_MAX) raise(PyExc_OverflowError, "integer argument out of range");
    return (int)v;
}
// A set of scan orders, one bit each, of which the library takes the lowest four and refuses the others up to 32.
unsigned order_mask(PyObject *o)
{
    const unsigned long v = PyLong_AsUnsignedLongMask(o);
    if (v == (unsigned long)-1 && PyErr_Occurred()) throw Raised{};
    return (unsigned)v;
}
bool truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Raised{};
    return v != 0;
}
float real(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised{};
    return (float)v;
}

std::string text(at::IntArrayRef s)
{
    std::string t = "(";
    for (size_t i = 0; i < s.size(); ++i) t += (i ? ", " : "") + std::to_string(s[i]);
    return t + (s.size() == 1 ? ",)" : ")");
}
// The library takes sizes of 31 bits; larger ones would be cut to them.
int size31(int64_t n, const char *name)
{
    if (n > INT_MAX) raise(PyExc_ValueError, std::string(name) + ": a dimension of " + std::to_string(n) + " is too large");
    return (int)n;
}
// Device pointer of a checked tensor.
void *dev(const Tensor &t, ScalarType st, const char *name)
{
    if (!t.is_cuda() || !t.is_contiguous() || t.scalar_type() != st)
        raise(PyExc_ValueError, std::string(name) + ": need a contiguous CUDA tensor of " + c10::toString(st) + ", got " +
                                    c10::toString(t.scalar_type()) + " on " + t.device().str());
    return t.data_ptr();
}
// ... of the given shape, on the device of `like`.
void *dev(const Tensor &t, ScalarType st, at::IntArrayRef shape, const char *name, const Tensor &like)
{
    void *p = dev(t, st, name);
    if (t.sizes() != shape) raise(PyExc_ValueError, std::string(name) + ": shape " + text(t.sizes()) + " != " + text(shape));
    if (t.device() != like.device()) raise(PyExc_ValueError, std::string(name) + ": on " + t.device().str() + ", the other tensors on " + like.device().str());
    return p;
}
void *dev(PyObject *o, ScalarType st, at::IntArrayRef shape, const char *name, const Tensor &like) { return dev(tensor(o, name), st, shape, name, like); }
void *dev_opt(PyObject *o, ScalarType st, at::IntArrayRef shape, const char *name, const Tensor &like)
{
    return none(o) ? nullptr : dev(o, st, shape, name, like);
}

Tensor empty(at::IntArrayRef shape, ScalarType st, const Tensor &like)
{
    return at::detail::empty_cuda(shape, st, like.device(), std::nullopt);
}
// The caller's tensor where there is one, else a new one.
Tensor given(PyObject *o, at::IntArrayRef shape, ScalarType st, const Tensor &like, const char *name)
{
    if (none(o)) return empty(shape, st, like);
    return tensor(o, name);
}
PyObject *wrap(Tensor t) { return THPVariable_Wrap(std::move(t)); }
PyObject *wrap_opt(const Tensor &t) { return t.defined() ? wrap(t) : Py_NewRef(Py_None); }
PyObject *pack(std::initializer_list<Tensor> ts)
{
    PyObject *r = PyTuple_New((Py_ssize_t)ts.size());
    Py_ssize_t i = 0;
    for (const Tensor &t : ts) PyTuple_SET_ITEM(r, i++, wrap_opt(t));
    return r;
}

void *stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

constexpr ScalarType kF32 = ScalarType::Float, kBf16 = ScalarType::BFloat16, kByte = ScalarType::Byte;
int dtype_of(const Tensor &t, bool f32_out)
{
    if (t.scalar_type() == kF32) return DIG_F32;
    if (t.scalar_type() == kBf16) return f32_out ? DIG_BF16_F32OUT : DIG_BF16;
    raise(PyExc_TypeError, std::string("unsupported storage type ") + c10::toString(t.scalar_type()));
}
ScalarType storage(int dtype) { return dtype == DIG_F32 ? kF32 : kBf16; }
ScalarType out_storage(int dtype) { return dtype == DIG_BF16 ? kBf16 : kF32; }

struct Ws {
    Tensor t;
    void *p = nullptr;
    size_t n = 0;
};
Ws workspace(PyObject *o, size_t need, const Tensor &like)
{
    Ws w;
    if (none(o)) {
        w.t = empty({(int64_t)(need > 16 ? need : 16)}, kByte, like);
    } else {                             // any type and shape: it is scratch
        w.t = tensor(o, "workspace");
        if (!w.t.is_cuda() || !w.t.is_non_overlapping_and_dense() || w.t.device() != like.device())
            raise(PyExc_ValueError, "workspace: need a dense tensor on " + like.device().str() + ", got one on " + w.t.device().str());
    }
    w.p = w.t.data_ptr();
    w.n = (size_t)w.t.numel() * w.t.element_size();
    return w;
}

// Shapes and types shared by the GLA entry points; q, k, v and the gate checked.
struct Gla {
    const Tensor &q_t;
    int B, L, H, dk, dv, gh, gw, chunk, dtype;
    std::vector<int64_t> ks, vs;
    ScalarType st, ost;
    void *q, *k, *v;
    float *gate;
    Gla(PyObject *const *a, PyObject *gh_, PyObject *gw_, PyObject *chunk_, bool f32_out) : q_t(tensor(a[0], "q"))
    {
        const Tensor &v_t = tensor(a[2], "v");
        if (q_t.dim() != 4) raise(PyExc_ValueError, "q: need 4 dimensions [B, L, H, d_k], got shape " + text(q_t.sizes()));
        if (v_t.dim() < 1) raise(PyExc_ValueError, "v: need 4 dimensions [B, L, H, d_v], got shape " + text(v_t.sizes()));
        ks = q_t.sizes().vec();
        vs = ks;
        vs[3] = v_t.size(-1);
        B = (int)ks[0]; L = (int)ks[1]; H = (int)ks[2]; dk = (int)ks[3]; dv = (int)vs[3];
        gh = integer(gh_); gw = integer(gw_); chunk = integer(chunk_);
        dtype = dtype_of(q_t, f32_out);
        st = storage(dtype);
        ost = out_storage(dtype);
        q = dev(q_t, st, "q");
        k = dev(a[1], st, ks, "k", q_t);
        v = dev(v_t, st, vs, "v", q_t);
        gate = (float *)dev(a[3], kF32, ks, "gate", q_t);
    }
    std::vector<int64_t> state() const { return {B, H, dk, dv}; }
};

#define CALL(expr, where)            \
    do {                             \
        int st_;                     \
        Py_BEGIN_ALLOW_THREADS       \
        st_ = (int)(expr);           \
        Py_END_ALLOW_THREADS         \
        check(st_, where);           \
    } while (0)

// ---- entry points (arguments by position, in the order dig.py passes them) ----------------------------
PyObject *gate_logsigmoid(PyObject *const *a)
{
    const Tensor &g = tensor(a[0], "g");
    if (g.dim() != 4) raise(PyExc_ValueError, "g: need 4 dimensions [B, L, H, d_k], got shape " + text(g.sizes()));
    const int B = (int)g.size(0), L = (int)g.size(1), H = (int)g.size(2), dk = (int)g.size(3), dtype = dtype_of(g, false);
    PyObject *seq = PySequence_Fast(a[1], "tau_per_head: need a sequence of numbers");
    if (!seq) throw Raised{};
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
    std::vector<float> tau(H, 0.f);
    bool bad = n > H;
    if (bad) PyErr_SetString(PyExc_IndexError, "tau_per_head: more values than heads");
    for (Py_ssize_t i = 0; i < n && !bad; ++i) {
        const double v = PyFloat_AsDouble(PySequence_Fast_GET_ITEM(seq, i));
        bad = v == -1.0 && PyErr_Occurred();
        tau[i] = (float)v;
    }
    Py_DECREF(seq);
    if (bad) throw Raised{};
    void *gp = dev(g, storage(dtype), "g");
    Tensor gate = given(a[2], g.sizes(), kF32, g, "gate");
    float *op = (float *)dev(gate, kF32, g.sizes(), "gate", g);
    void *s = stream();
    CALL(dig_gate_logsigmoid(gp, tau.data(), op, B, L, H, dk, dtype, s), "dig_gate_logsigmoid");
    return wrap(gate);
}

// q k v gate grid_h grid_w chunk direction f32_out out workspace
PyObject *gla_fwd(PyObject *const *a)
{
    const Gla g(a, a[4], a[5], a[6], truth(a[8]));
    const int dir = integer(a[7]);
    Tensor out = given(a[9], g.vs, g.ost, g.q_t, "out");
    void *op = dev(out, g.ost, g.vs, "out", g.q_t);
    const Ws w = workspace(a[10], none(a[10]) ? dig_gla_workspace_bytes(g.B, g.H, g.gh, g.gw, g.dk, g.dv, g.chunk, g.dtype, 0) : 0, g.q_t);
    void *s = stream();
    CALL(dig_gla_fwd(g.q, g.k, g.v, g.gate, op, g.B, g.H, g.gh, g.gw, g.dk, g.dv, g.chunk, dir, g.dtype, w.p, w.n, s), "dig_gla_fwd");
    return wrap(out);
}

// The four gradients: the caller's or new ones.
struct Grads {
    Tensor dq, dk, dv, dg;
    void *pq, *pk, *pv;
    float *pg;
    Grads(PyObject *o, const Gla &g)
    {
        if (none(o)) {
            dq = empty(g.ks, g.ost, g.q_t);
            dk = empty(g.ks, g.ost, g.q_t);
            dv = empty(g.vs, g.ost, g.q_t);
            dg = empty(g.ks, kF32, g.q_t);
        } else {
            PyObject *seq = PySequence_Fast(o, "grads: need (dq, dk, dv, dgate)");
            if (!seq) throw Raised{};
            const bool four = PySequence_Fast_GET_SIZE(seq) == 4;
            PyObject **it = PySequence_Fast_ITEMS(seq);
            bool tensors = four;
            for (int i = 0; i < 4 && tensors; ++i) tensors = THPVariable_Check(it[i]);
            if (tensors) {
                dq = THPVariable_Unpack(it[0]);
                dk = THPVariable_Unpack(it[1]);
                dv = THPVariable_Unpack(it[2]);
                dg = THPVariable_Unpack(it[3]);
            }
            Py_DECREF(seq);
            if (!tensors) raise(PyExc_ValueError, "grads: need four tensors (dq, dk, dv, dgate)");
        }
        pq = dev(dq, g.ost, g.ks, "dq", g.q_t);
        pk = dev(dk, g.ost, g.ks, "dk", g.q_t);
        pv = dev(dv, g.ost, g.vs, "dv", g.q_t);
        pg = (float *)dev(dg, kF32, g.ks, "dgate", g.q_t);
    }
};

// q k v gate d_out grid_h grid_w chunk direction f32_out grads workspace
PyObject *gla_bwd(PyObject *const *a)
{
    const Gla g(a, a[5], a[6], a[7], truth(a[9]));
    const int dir = integer(a[8]);
    void *dop = dev(a[4], g.st, g.vs, "d_out", g.q_t);
    const Grads r(a[10], g);
    const Ws w = workspace(a[11], none(a[11]) ? dig_gla_workspace_bytes(g.B, g.H, g.gh, g.gw, g.dk, g.dv, g.chunk, g.dtype, 1) : 0, g.q_t);
    void *s = stream();
    CALL(dig_gla_bwd(g.q, g.k, g.v, g.gate, dop, r.pq, r.pk, r.pv, r.pg, g.B, g.H, g.gh, g.gw, g.dk, g.dv, g.chunk, dir, g.dtype, w.p, w.n, s),
         "dig_gla_bwd");
    return pack({r.dq, r.dk, r.dv, r.dg});
}

// q k v gate s_in grid_h grid_w chunk direction f32_out want_s_out workspace
PyObject *gla_fwd_state(PyObject *const *a)
{
    const Gla g(a, a[5], a[6], a[7], truth(a[9]));
    const int dir = integer(a[8]);
    const float *si = (const float *)dev_opt(a[4], kF32, g.state(), "s_in", g.q_t);
    Tensor out = empty(g.vs, g.ost, g.q_t), so;
    if (truth(a[10])) so = empty(g.state(), kF32, g.q_t);
    const Ws w = workspace(a[11], none(a[11]) ? dig_gla_workspace_bytes(g.B, g.H, g.gh, g.gw, g.dk, g.dv, g.chunk, g.dtype, 0) : 0, g.q_t);
    void *op = out.data_ptr();
    float *sop = so.defined() ? (float *)so.data_ptr() : nullptr;
    void *s = stream();
    CALL(dig_gla_fwd_state(g.q, g.k, g.v, g.gate, si, op, sop, g.B, g.H, g.gh, g.gw, g.dk, g.dv, g.chunk, dir, g.dtype, w.p, w.n, s),
         "dig_gla_fwd_state");
    return pack({out, so});
}

// q k v gate d_out s_in ds_out grid_h grid_w chunk direction f32_out workspace
PyObject *gla_bwd_state(PyObject *const *a)
{
    const Gla g(a, a[7], a[8], a[9], truth(a[11]));
    const int dir = integer(a[10]);
    void *dop = dev(a[4], g.st, g.vs, "d_out", g.q_t);
    const float *si = (const float *)dev_opt(a[5], kF32, g.state(), "s_in", g.q_t), *dso = (const float *)dev_opt(a[6], kF32, g.state(), "ds_out", g.q_t);
    const Grads r(Py_None, g);
    Tensor dsi = empty(g.state(), kF32, g.q_t);
    float *dsip = (float *)dsi.data_ptr();
    const Ws w = workspace(a[12], none(a[12]) ? dig_gla_workspace_bytes(g.B, g.H, g.gh, g.gw, g.dk, g.dv, g.chunk, g.dtype, 1) : 0, g.q_t);
    void *s = stream();
    CALL(dig_gla_bwd_state(g.q, g.k, g.v, g.gate, dop, si, dso, r.pq, r.pk, r.pv, r.pg, dsip, g.B, g.H, g.gh, g.gw, g.dk, g.dv, g.chunk, dir,
                           g.dtype, w.p, w.n, s), "dig_gla_bwd_state");
    return pack({r.dq, r.dk, r.dv, r.dg, dsi});
}

// q k v gate grid_h grid_w mask chunk f32_out out workspace
PyObject *gla_fwd_multi(PyObject *const *a)
{
    const Gla g(a, a[4], a[5], a[7], truth(a[8]));
    const unsigned mask = order_mask(a[6]);
    Tensor out = given(a[9], g.vs, g.ost, g.q_t, "out");
    void *op = dev(out, g.ost, g.vs, "out", g.q_t);
    const Ws w = workspace(a[10], none(a[10]) ? dig_gla_multi_workspace_bytes(g.B, g.H, g.gh, g.gw, g.dk, g.dv, g.chunk, g.dtype, 0) : 0, g.q_t);
    void *s = stream();
    CALL(dig_gla_fwd_multi(g.q, g.k, g.v, g.gate, op, g.B, g.H, g.gh, g.gw, g.dk, g.dv, g.chunk, mask, g.dtype, w.p, w.n, s), "dig_gla_fwd_multi");
    return wrap(out);
}

// q k v gate d_out grid_h grid_w mask chunk f32_out grads workspace
PyObject *gla_bwd_multi(PyObject *const *a)
{
    const Gla g(a, a[5], a[6], a[8], truth(a[9]));
    const unsigned mask = order_mask(a[7]);
    void *dop = dev(a[4], g.st, g.vs, "d_out", g.q_t);
    const Grads r(a[10], g);
    const Ws w = workspace(a[11], none(a[11]) ? dig_gla_multi_workspace_bytes(g.B, g.H, g.gh, g.gw, g.dk, g.dv, g.chunk, g.dtype, 1) : 0, g.q_t);
    void *s = stream();
    CALL(dig_gla_bwd_multi(g.q, g.k, g.v, g.gate, dop, r.pq, r.pk, r.pv, r.pg, g.B, g.H, g.gh, g.gw, g.dk, g.dv, g.chunk, mask, g.dtype, w.p, w.n, s),
         "dig_gla_bwd_multi");
    return pack({r.dq, r.dk, r.dv, r.dg});
}

size_t beta_need(const Gla &g, int backward)
{
    const size_t need = dig_gla_beta_workspace_bytes(g.B, g.H, g.gh, g.gw, g.dk, g.dv, g.chunk, g.dtype, backward);
    if (need == 0) check(DIG_ERR_UNSUPPORTED, "dig_gla_beta_workspace_bytes");
    return need;
}
// q k v gate bgate grid_h grid_w chunk direction f32_out workspace
PyObject *gla_fwd_beta(PyObject *const *a)
{
    const Gla g(a, a[5], a[6], a[7], truth(a[9]));
    const int dir = integer(a[8]);
    const float *bg = (const float *)dev(a[4], kF32, g.vs, "bgate", g.q_t);
    const Ws w = workspace(a[10], beta_need(g, 0), g.q_t);
    Tensor out = empty(g.vs, g.ost, g.q_t);
    void *op = out.data_ptr(), *s = stream();
    CALL(dig_gla_fwd_beta(g.q, g.k, g.v, g.gate, bg, op, g.B, g.H, g.gh, g.gw, g.dk, g.dv, g.chunk, dir, g.dtype, w.p, w.n, s), "dig_gla_fwd_beta");
    return wrap(out);
}
// q k v gate bgate d_out grid_h grid_w chunk direction f32_out workspace
PyObject *gla_bwd_beta(PyObject *const *a)
{
    const Gla g(a, a[6], a[7], a[8], truth(a[10]));
    const int dir = integer(a[9]);
    const float *bg = (const float *)dev(a[4], kF32, g.vs, "bgate", g.q_t);
    void *dop = dev(a[5], g.st, g.vs, "d_out", g.q_t);
    const Ws w = workspace(a[11], beta_need(g, 1), g.q_t);
    const Grads r(Py_None, g);
    Tensor db = empty(g.vs, kF32, g.q_t);
    float *dbp = (float *)db.data_ptr();
    void *s = stream();
    CALL(dig_gla_bwd_beta(g.q, g.k, g.v, g.gate, bg, dop, r.pq, r.pk, r.pv, r.pg, dbp, g.B, g.H, g.gh, g.gw, g.dk, g.dv, g.chunk, dir, g.dtype, w.p,
                          w.n, s), "dig_gla_bwd_beta");
    return pack({r.dq, r.dk, r.dv, r.dg, db});
}

// q k v gate r grid_h grid_w chunk direction ln_w ln_b eps f32_out want_out workspace
PyObject *gla_fwd_outgate(PyObject *const *a)
{
    const Gla g(a, a[5], a[6], a[7], truth(a[12]));
    const int dir = integer(a[8]);
    const void *rp = dev(a[4], g.st, g.vs, "r", g.q_t);
    const float *lw = (const float *)dev_opt(a[9], kF32, {g.dv}, "ln_w", g.q_t), *lb = (const float *)dev_opt(a[10], kF32, {g.dv}, "ln_b", g.q_t);
    const float eps = real(a[11]);
    Tensor out, z = empty(g.vs, g.ost, g.q_t);
    if (truth(a[13])) out = empty(g.vs, g.ost, g.q_t);
    const Ws w = workspace(a[14], none(a[14]) ? dig_gla_workspace_bytes(g.B, g.H, g.gh, g.gw, g.dk, g.dv, g.chunk, g.dtype, 0) : 0, g.q_t);
    void *op = out.defined() ? out.data_ptr() : nullptr, *zp = z.data_ptr(), *s = stream();
    CALL(dig_gla_fwd_outgate(g.q, g.k, g.v, g.gate, rp, lw, lb, eps, op, zp, g.B, g.H, g.gh, g.gw, g.dk, g.dv, g.chunk, dir, g.dtype, w.p, w.n, s),
         "dig_gla_fwd_outgate");
    return pack({out, z});
}

// The rows of a tensor [..., d].
void rows_of(const Tensor &o, int &d, long long &rows, const char *name)
{
    if (o.dim() < 1 || o.size(-1) < 1) raise(PyExc_ValueError, std::string(name) + ": need rows of at least one value, got shape " + text(o.sizes()));
    d = size31(o.size(-1), name);
    rows = o.numel() / d;
}
// o r ln_w ln_b eps f32_out
PyObject *outgate_fwd(PyObject *const *a)
{
    const Tensor &o = tensor(a[0], "o");
    int d;
    long long rows;
    rows_of(o, d, rows, "o");
    const int dtype = dtype_of(o, truth(a[5]));
    const ScalarType st = storage(dtype);
    const void *op = dev(o, st, "o"), *rp = dev(a[1], st, o.sizes(), "r", o);
    const float *lw = (const float *)dev_opt(a[2], kF32, {d}, "ln_w", o), *lb = (const float *)dev_opt(a[3], kF32, {d}, "ln_b", o);
    const float eps = real(a[4]);
    Tensor z = empty(o.sizes(), out_storage(dtype), o);
    void *zp = z.data_ptr(), *s = stream();
    CALL(dig_gla_outgate_fwd(op, rp, lw, lb, zp, rows, d, eps, dtype, s), "dig_gla_outgate_fwd");
    return wrap(z);
}
// o r dz ln_w ln_b eps affine_grads f32_out workspace
PyObject *outgate_bwd(PyObject *const *a)
{
    const Tensor &o = tensor(a[0], "o");
    int d;
    long long rows;
    rows_of(o, d, rows, "o");
    const int dtype = dtype_of(o, truth(a[7]));
    const ScalarType st = storage(dtype);
    const void *op = dev(o, st, "o"), *rp = dev(a[1], st, o.sizes(), "r", o), *zp = dev(a[2], st, o.sizes(), "dz", o);
    const float *lw = (const float *)dev_opt(a[3], kF32, {d}, "ln_w", o), *lb = (const float *)dev_opt(a[4], kF32, {d}, "ln_b", o);
    const float eps = real(a[5]);
    Tensor d_o = empty(o.sizes(), out_storage(dtype), o), d_r = empty(o.sizes(), out_storage(dtype), o), dw, db;
    Ws w;
    if (truth(a[6])) {
        dw = empty({d}, kF32, o);
        db = empty({d}, kF32, o);
        if (!none(a[8])) dev(tensor(a[8], "workspace"), kByte, "workspace");
        w = workspace(a[8], none(a[8]) ? dig_gla_outgate_bwd_workspace_bytes(rows, d) : 0, o);
    }
    void *dop = d_o.data_ptr(), *drp = d_r.data_ptr(), *s = stream();
    float *dwp = dw.defined() ? (float *)dw.data_ptr() : nullptr, *dbp = db.defined() ? (float *)db.data_ptr() : nullptr;
    CALL(dig_gla_outgate_bwd(op, rp, lw, lb, zp, dop, drp, dwp, dbp, rows, d, eps, dtype, w.p, w.n, s), "dig_gla_outgate_bwd");
    return pack({d_o, d_r, dw, db});
}

// x w bias grid_h grid_w direction f32_out y
PyObject *dwconv(PyObject *const *a)
{
    const Tensor &x = tensor(a[0], "x");
    if (x.dim() != 3) raise(PyExc_ValueError, "x: need 3 dimensions [B, L, D], got shape " + text(x.sizes()));
    const int64_t D = x.size(2);
    const int gh = integer(a[3]), gw = integer(a[4]), dir = integer(a[5]);
    if (x.size(1) != (int64_t)gh * gw) raise(PyExc_ValueError, "x: L != grid_h*grid_w");
    const int dtype = dtype_of(x, truth(a[6]));
    const ScalarType st = storage(dtype), ost = out_storage(dtype);
    const void *xp = dev(x, st, "x"), *wp = dev(a[1], st, {3, 3, D}, "w", x), *bp = dev_opt(a[2], st, {D}, "bias", x);
    Tensor y = given(a[7], x.sizes(), ost, x, "y");
    void *yp = dev(y, ost, x.sizes(), "y", x), *s = stream();
    const int B = (int)x.size(0);
    CALL(dig_srem_dwconv(xp, wp, bp, yp, B, gh, gw, (int)D, dir, dtype, s), "dig_srem_dwconv");
    return wrap(y);
}
// x w dy grid_h grid_w direction with_bias f32_out workspace
PyObject *dwconv_bwd(PyObject *const *a)
{
    const Tensor &x = tensor(a[0], "x");
    if (x.dim() != 3) raise(PyExc_ValueError, "x: need 3 dimensions [B, L, D], got shape " + text(x.sizes()));
    const int64_t D = x.size(2);
    const int gh = integer(a[3]), gw = integer(a[4]), dir = integer(a[5]), B = (int)x.size(0);
    if (x.size(1) != (int64_t)gh * gw) raise(PyExc_ValueError, "x.shape[1] must equal grid_h * grid_w");
    const int dtype = dtype_of(x, truth(a[7]));
    const ScalarType st = storage(dtype);
    const size_t need = dig_srem_dwconv_bwd_workspace_bytes(B, gh, gw, (int)D);
    if (need == 0) raise(PyExc_ValueError, "dig_srem_dwconv_bwd: unsupported sizes");
    const void *xp = dev(x, st, "x"), *wp = dev(a[1], st, {3, 3, D}, "w", x), *gp = dev(a[2], st, x.sizes(), "dy", x);
    if (!none(a[8])) dev(tensor(a[8], "workspace"), kByte, "workspace");
    const Ws w = workspace(a[8], need, x);
    Tensor dx = empty(x.sizes(), out_storage(dtype), x), dw = empty({3, 3, D}, kF32, x), db;
    if (truth(a[6])) db = empty({D}, kF32, x);
    void *dxp = dx.data_ptr(), *s = stream();
    float *dwp = (float *)dw.data_ptr(), *dbp = db.defined() ? (float *)db.data_ptr() : nullptr;
    CALL(dig_srem_dwconv_bwd(xp, wp, gp, dxp, dwp, dbp, B, gh, gw, (int)D, dir, dtype, w.p, w.n, s), "dig_srem_dwconv_bwd");
    return pack({dx, dw, db});
}

// ---- linear attention with a decay for each head, rotary positions, layer norm -------------------------------------
// These run on their tensors' device and its current stream, whatever the current device is.
void on_cuda(const Tensor &t, const char *name)
{
    if (!t.is_cuda()) raise(PyExc_ValueError, std::string(name) + ": need a CUDA tensor, got one on " + t.device().str());
}
struct On {
    c10::cuda::CUDAGuard guard;
    explicit On(const Tensor &t) : guard(t.device()) {}
    void *stream() const { return c10::cuda::getCurrentCUDAStream().stream(); }
};
// H numbers.
std::vector<float> numbers(PyObject *o, int64_t H, const char *name)
{
    PyObject *seq = PySequence_Fast(o, "need a sequence of numbers");
    if (!seq) throw Raised{};
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
    std::vector<float> v(n);
    bool bad = false;
    for (Py_ssize_t i = 0; i < n && !bad; ++i) {
        const double x = PyFloat_AsDouble(PySequence_Fast_GET_ITEM(seq, i));
        bad = x == -1.0 && PyErr_Occurred();
        v[i] = (float)x;
    }
    Py_DECREF(seq);
    if (bad) throw Raised{};
    if (n != H) raise(PyExc_ValueError, std::string(name) + ": " + std::to_string(n) + " values for " + std::to_string(H) + " heads");
    return v;
}
// A tensor [B, L, H, d] whose heads stand side by side: its pointer, and the batch and token strides.  Strides of dimensions of one
// element say nothing.
void *rows(const Tensor &t, ScalarType st, const char *name, const Tensor &like, long long *strides)
{
    on_cuda(t, name);
    if (t.dim() != 4) raise(PyExc_ValueError, std::string(name) + ": need 4 dimensions [B, L, H, d], got shape " + text(t.sizes()));
    if (t.scalar_type() != st) raise(PyExc_ValueError, std::string(name) + ": need a tensor of " + c10::toString(st) + ", got " + c10::toString(t.scalar_type()));
    if (t.device() != like.device()) raise(PyExc_ValueError, std::string(name) + ": on " + t.device().str() + ", the other tensors on " + like.device().str());
    const int64_t H = t.size(2), d = t.size(3);
    if (t.numel() == 0) raise(PyExc_ValueError, std::string(name) + ": empty, shape " + text(t.sizes()));
    for (const int64_t n : t.sizes()) size31(n, name);
    if ((d > 1 && t.stride(3) != 1) || (H > 1 && t.stride(2) != d))
        raise(PyExc_ValueError, std::string(name) + ": the last two dimensions have to be dense, got strides " + text(t.strides()));
    strides[1] = t.size(1) > 1 ? t.stride(1) : H * d;
    strides[0] = t.size(0) > 1 ? t.stride(0) : t.size(1) * strides[1];
    const int64_t unit = st == kF32 ? 4 : 8;
    if (strides[0] % unit || strides[1] % unit || (reinterpret_cast<uintptr_t>(t.data_ptr()) & 15))
        raise(PyExc_ValueError, std::string(name) + ": rows have to start on 16-byte boundaries, got strides " + text(t.strides()));
    return t.data_ptr();
}

// Dense tensors that a result must not overlap.
void apart(std::initializer_list<const Tensor *> reads, const Tensor &t, const char *name)
{
    const char *p = (const char *)t.data_ptr(), *end = p + t.numel() * t.element_size();
    for (const Tensor *r : reads) {
        const char *o = (const char *)r->data_ptr();
        if (p < o + r->numel() * r->element_size() && o < end) raise(PyExc_ValueError, std::string(name) + ": overlaps another tensor of the call");
    }
}
// What a result must not overlap: rows of the inputs, and dense tensors.
struct Reads {
    struct One {
        const char *name, *p;
        dig::RowSet rows;                // in bytes
    };
    std::vector<One> all;
    void add(const Tensor &t, const char *name, const long long *strides)
    {
        const long long e = t.element_size();
        all.push_back({name, (const char *)t.data_ptr(), {(int)t.size(0), (int)t.size(1), strides[0] * e, strides[1] * e, t.size(2) * t.size(3) * e}});
    }
    void add(const Tensor &t, const char *name)
    {
        all.push_back({name, (const char *)t.data_ptr(), {1, 1, 0, 0, (long long)t.numel() * (long long)t.element_size()}});
    }
    void add(PyObject *o, const char *name)
    {
        if (!none(o)) add(tensor(o, name), name);
    }
    // A result, or scratch, that the caller gave; the ones after it must not overlap it either.
    void write(const Tensor &t, const char *name)
    {
        const long long n = (long long)t.numel() * (long long)t.element_size();
        const char *p = (const char *)t.data_ptr();
        for (const One &r : all)
            if (dig::rows_meet_block(r.rows, (long long)(uintptr_t)p - (long long)(uintptr_t)r.p, n))
                raise(PyExc_ValueError, std::string(name) + ": overlaps " + r.name);
        add(t, name);
    }
    void write(PyObject *o, const char *name)
    {
        if (!none(o)) write(tensor(o, name), name);
    }
};

struct Decay {
    const Tensor &q_t;
    int B, L, H, Hk, dk, dv, gh, gw, dtype;
    ScalarType st;
    long long strides[6];
    void *q, *k, *v;
    std::vector<float> decay;
    Decay(PyObject *const *a, PyObject *gh_, PyObject *gw_) : q_t(tensor(a[0], "q"))
    {
        const Tensor &k_t = tensor(a[1], "k"), &v_t = tensor(a[2], "v");
        dtype = dtype_of(q_t, false);
        st = storage(dtype);
        q = rows(q_t, st, "q", q_t, strides);
        k = rows(k_t, st, "k", q_t, strides + 2);
        v = rows(v_t, st, "v", q_t, strides + 4);
        const auto n = q_t.sizes();
        if (k_t.size(0) != n[0] || k_t.size(1) != n[1] || k_t.size(3) != n[3] || n[2] % k_t.size(2) != 0)
            raise(PyExc_ValueError, "k: shape " + text(k_t.sizes()) + " does not go with q of " + text(n));
        if (v_t.size(0) != n[0] || v_t.size(1) != n[1] || v_t.size(2) != k_t.size(2))
            raise(PyExc_ValueError, "v: shape " + text(v_t.sizes()) + " does not go with k of " + text(k_t.sizes()));
        gh = integer(gh_); gw = integer(gw_);
        if (n[1] != (int64_t)gh * gw) raise(PyExc_ValueError, "q: L != grid_h*grid_w");
        B = (int)n[0]; L = (int)n[1]; H = (int)n[2]; Hk = (int)k_t.size(2); dk = (int)n[3]; dv = (int)v_t.size(3);
        decay = numbers(a[3], H, "log_decay");
    }
    Reads reads(PyObject *const *a) const
    {
        Reads r;
        r.add(q_t, "q", strides);
        r.add(tensor(a[1], "k"), "k", strides + 2);
        r.add(tensor(a[2], "v"), "v", strides + 4);
        return r;
    }
    std::vector<int64_t> state() const { return {B, H, dk, dv}; }
    const int *lengths(PyObject *o) const { return (const int *)dev_opt(o, ScalarType::Int, {B}, "lengths", q_t); }
    Ws space(PyObject *o, int backward) const
    {
        return workspace(o, none(o) ? dig_decay_workspace_bytes(B, H, Hk, gh, gw, dk, dv, dtype, backward) : 0, q_t);
    }
};

// q k v log_decay grid_h grid_w direction s_in lengths want_s_out out workspace
PyObject *decay_fwd(PyObject *const *a)
{
    const Decay g(a, a[4], a[5]);
    const On on(g.q_t);
    const int dir = integer(a[6]);
    const float *si = (const float *)dev_opt(a[7], kF32, g.state(), "s_in", g.q_t);
    const int *len = g.lengths(a[8]);
    const std::vector<int64_t> shape = {g.B, g.L, g.H, g.dv};
    Tensor out = given(a[10], shape, g.st, g.q_t, "out"), so;
    void *op = dev(out, g.st, shape, "out", g.q_t);
    if (truth(a[9])) so = empty(g.state(), kF32, g.q_t);
    const Ws w = g.space(a[11], 0);
    if (!none(a[10]) || !none(a[11])) {
        Reads r = g.reads(a);
        r.add(a[7], "s_in");
        r.add(a[8], "lengths");
        r.write(a[10], "out");
        r.write(a[11], "workspace");
    }
    float *sop = so.defined() ? (float *)so.data_ptr() : nullptr;
    void *s = on.stream();
    CALL(dig_decay_fwd(g.q, g.k, g.v, g.strides, g.decay.data(), len, si, op, sop, g.B, g.H, g.Hk, g.gh, g.gw, g.dk, g.dv, dir, g.dtype, w.p, w.n, s), "dig_decay_fwd");
    return pack({out, so});
}

// q k v log_decay d_out grid_h grid_w direction s_in ds_out lengths want_ds_in grads workspace
PyObject *decay_bwd(PyObject *const *a)
{
    const Decay g(a, a[5], a[6]);
    const On on(g.q_t);
    const int dir = integer(a[7]);
    const std::vector<int64_t> ks = {g.B, g.L, g.Hk, g.dk}, vs = {g.B, g.L, g.Hk, g.dv};
    const void *gp = dev(a[4], g.st, {g.B, g.L, g.H, g.dv}, "d_out", g.q_t);
    const float *si = (const float *)dev_opt(a[8], kF32, g.state(), "s_in", g.q_t), *dso = (const float *)dev_opt(a[9], kF32, g.state(), "ds_out", g.q_t);
    const int *len = g.lengths(a[10]);
    Tensor dq, dk, dv, dsi;
    if (none(a[12])) {
        dq = empty(g.q_t.sizes(), g.st, g.q_t);
        dk = empty(ks, g.st, g.q_t);
        dv = empty(vs, g.st, g.q_t);
    } else {
        PyObject *seq = PySequence_Fast(a[12], "grads: need (dq, dk, dv)");
        if (!seq) throw Raised{};
        PyObject **it = PySequence_Fast_ITEMS(seq);
        const bool three = PySequence_Fast_GET_SIZE(seq) == 3 && THPVariable_Check(it[0]) && THPVariable_Check(it[1]) && THPVariable_Check(it[2]);
        if (three) {
            dq = THPVariable_Unpack(it[0]);
            dk = THPVariable_Unpack(it[1]);
            dv = THPVariable_Unpack(it[2]);
        }
        Py_DECREF(seq);
        if (!three) raise(PyExc_ValueError, "grads: need three tensors (dq, dk, dv)");
    }
    void *qp = dev(dq, g.st, g.q_t.sizes(), "dq", g.q_t), *kp = dev(dk, g.st, ks, "dk", g.q_t), *vp = dev(dv, g.st, vs, "dv", g.q_t);
    if (truth(a[11])) dsi = empty(g.state(), kF32, g.q_t);
    const Ws w = g.space(a[13], 1);
    if (!none(a[12]) || !none(a[13])) {
        Reads r = g.reads(a);
        r.add(a[4], "d_out");
        r.add(a[8], "s_in");
        r.add(a[9], "ds_out");
        r.add(a[10], "lengths");
        r.write(dq, "dq");
        r.write(dk, "dk");
        r.write(dv, "dv");
        r.write(a[13], "workspace");
    }
    float *dsip = dsi.defined() ? (float *)dsi.data_ptr() : nullptr;
    void *s = on.stream();
    CALL(dig_decay_bwd(g.q, g.k, g.v, g.strides, g.decay.data(), len, gp, si, dso, qp, kp, vp, dsip, g.B, g.H, g.Hk, g.gh, g.gw, g.dk, g.dv, dir, g.dtype, w.p, w.n, s),
         "dig_decay_bwd");
    return pack({dq, dk, dv, dsi});
}

// q k v log_decay state out
PyObject *decay_step(PyObject *const *a)
{
    const Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &v = tensor(a[2], "v");
    if (q.dim() != 3) raise(PyExc_ValueError, "q: need 3 dimensions [B, H, d_k], got shape " + text(q.sizes()));
    if (k.dim() != 3 || k.size(1) < 1 || q.size(1) % k.size(1) != 0) raise(PyExc_ValueError, "k: shape " + text(k.sizes()) + " does not go with q of " + text(q.sizes()));
    if (v.dim() != 3) raise(PyExc_ValueError, "v: need 3 dimensions [B, H_kv, d_v], got shape " + text(v.sizes()));
    const int64_t B = q.size(0), H = q.size(1), Hk = k.size(1), dk = q.size(2), dv = v.size(2);
    for (const int64_t n : {B, H, Hk, dk, dv}) size31(n, "q, k, v");
    const int dtype = dtype_of(q, false);
    const ScalarType st = storage(dtype);
    const void *qp = dev(q, st, "q"), *kp = dev(k, st, {B, Hk, dk}, "k", q), *vp = dev(v, st, {B, Hk, dv}, "v", q);
    const On on(q);
    const std::vector<float> decay = numbers(a[3], H, "log_decay");
    float *sp = (float *)dev(a[4], kF32, {B, H, dk, dv}, "state", q);
    const std::vector<int64_t> shape = {B, H, dv};
    Tensor out = given(a[5], shape, st, q, "out");
    void *op = dev(out, st, shape, "out", q), *s = on.stream();
    apart({&q, &k, &v}, tensor(a[4], "state"), "state");
    if (!none(a[5])) apart({&q, &k, &v, &tensor(a[4], "state")}, out, "out");
    CALL(dig_decay_step(qp, kp, vp, decay.data(), sp, op, sp, (int)B, (int)H, (int)Hk, (int)dk, (int)dv, dtype, s), "dig_decay_step");
    return wrap(out);
}

// q k positions freqs axes interleaved inverse inplace
PyObject *rope(PyObject *const *a)
{
    const Tensor &q = tensor(a[0], "q"), &pos = tensor(a[2], "positions");
    const int dtype = dtype_of(q, false);
    const ScalarType st = storage(dtype);
    long long strides[4] = {0, 0, 0, 0};
    const void *qp = rows(q, st, "q", q, strides), *kp = nullptr;
    const int64_t B = q.size(0), L = q.size(1), d = q.size(3);
    const On on(q);
    int Hk = 0;
    if (!none(a[1])) {
        const Tensor &k = tensor(a[1], "k");
        kp = rows(k, st, "k", q, strides + 2);
        if (k.size(0) != B || k.size(1) != L || k.size(3) != d) raise(PyExc_ValueError, "k: shape " + text(k.sizes()) + " does not go with q of " + text(q.sizes()));
        Hk = (int)k.size(2);
    }
    const bool batched = pos.dim() == 3;
    if (!(pos.dim() == 2 || (batched && pos.size(0) == B)) || pos.size(-2) != L) raise(PyExc_ValueError, "positions: need [L, axes] or [B, L, axes], got shape " + text(pos.sizes()));
    const int *pp = (const int *)dev(pos, ScalarType::Int, pos.sizes(), "positions", q);
    const int n_axes = size31(pos.size(-1), "positions");
    std::vector<double> freqs;
    std::vector<int> axes;
    for (int which = 0; which < 2; ++which) {
        PyObject *seq = PySequence_Fast(a[3 + which], which ? "axes: need a sequence of integers" : "freqs: need a sequence of numbers");
        if (!seq) throw Raised{};
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
        bool bad = false;
        for (Py_ssize_t i = 0; i < n && !bad; ++i) {
            PyObject *o = PySequence_Fast_GET_ITEM(seq, i);
            if (which) {
                const long v = PyLong_AsLong(o);
                bad = v == -1 && PyErr_Occurred();
                axes.push_back(v < 0 || v > 255 ? -1 : (int)v);
            } else {
                freqs.push_back(PyFloat_AsDouble(o));
                bad = freqs.back() == -1.0 && PyErr_Occurred();
            }
        }
        Py_DECREF(seq);
        if (bad) throw Raised{};
    }
    if (freqs.size() != axes.size()) raise(PyExc_ValueError, "freqs and axes: " + std::to_string(freqs.size()) + " and " + std::to_string(axes.size()) + " values");
    const bool in_place = truth(a[7]);
    Tensor qo = in_place ? q : empty(q.sizes(), st, q), ko;
    if (kp) ko = in_place ? tensor(a[1], "k") : empty(tensor(a[1], "k").sizes(), st, q);
    const int inter = truth(a[5]), inv = truth(a[6]);
    void *qop = qo.data_ptr(), *kop = kp ? ko.data_ptr() : nullptr, *s = on.stream();
    if (in_place)           // rows that coincide cannot all be written
        for (int i = 0; i < (kp ? 2 : 1); ++i)
            if (!dig::distinct({(int)B, (int)L, strides[2 * i], strides[2 * i + 1], (i ? Hk : q.size(2)) * d}))
                raise(PyExc_ValueError, std::string(i ? "k" : "q") + ": rows overlap, they cannot be turned in place");
    CALL(dig_rope(qp, kp, strides, pp, batched ? (int)B : 1, n_axes, freqs.data(), axes.data(), (int)freqs.size(), qop, kop, (int)B, (int)L, (int)q.size(2), Hk,
                  (int)d, inter, inv, dtype, s), "dig_rope");
    return pack({qo, ko});
}

// Groups of an affine parameter [D] or [groups, D].
int groups_of(const Tensor &t, int D, const char *name)
{
    if ((t.dim() != 1 && t.dim() != 2) || t.size(-1) != D || t.numel() == 0)
        raise(PyExc_ValueError, std::string(name) + ": need [" + std::to_string(D) + "] or [groups, " + std::to_string(D) + "], got shape " + text(t.sizes()));
    return t.dim() == 1 ? 1 : size31(t.size(0), name);
}
// x w b eps
PyObject *layernorm_fwd(PyObject *const *a)
{
    const Tensor &x = tensor(a[0], "x");
    int D, groups = 1;
    long long rows;
    if (x.dim() < 1 || x.numel() == 0) raise(PyExc_ValueError, "x: need rows of at least one value, got shape " + text(x.sizes()));
    rows_of(x, D, rows, "x");
    const int dtype = dtype_of(x, false);
    const ScalarType st = storage(dtype);
    const void *xp = dev(x, st, "x");
    const On on(x);
    const float *wp = nullptr, *bp = nullptr;
    if (!none(a[1])) {
        const Tensor &w = tensor(a[1], "w");
        groups = groups_of(w, D, "w");
        wp = (const float *)dev(w, kF32, w.sizes(), "w", x);
    }
    if (!none(a[2])) {
        const Tensor &b = tensor(a[2], "b");
        const int g = groups_of(b, D, "b");
        if (wp && g != groups) raise(PyExc_ValueError, "b: shape " + text(b.sizes()) + " does not go with w of " + text(tensor(a[1], "w").sizes()));
        groups = g;
        bp = (const float *)dev(b, kF32, b.sizes(), "b", x);
    }
    if (rows % groups) raise(PyExc_ValueError, "x: " + std::to_string(rows) + " rows in " + std::to_string(groups) + " groups");
    const float eps = real(a[3]);
    Tensor y = empty(x.sizes(), st, x);
    void *yp = y.data_ptr(), *s = on.stream();
    CALL(dig_layernorm_fwd(xp, wp, bp, yp, rows, groups, D, eps, dtype, s), "dig_layernorm_fwd");
    return wrap(y);
}
// x dy w eps affine_grads workspace
PyObject *layernorm_bwd(PyObject *const *a)
{
    const Tensor &x = tensor(a[0], "x");
    int D, groups = 1;
    long long rows;
    if (x.dim() < 1 || x.numel() == 0) raise(PyExc_ValueError, "x: need rows of at least one value, got shape " + text(x.sizes()));
    rows_of(x, D, rows, "x");
    const int dtype = dtype_of(x, false);
    const ScalarType st = storage(dtype);
    const void *xp = dev(x, st, "x"), *gp = dev(a[1], st, x.sizes(), "dy", x);
    const On on(x);
    const float *wp = nullptr;
    std::vector<int64_t> shape = {D};
    if (!none(a[2])) {
        const Tensor &w = tensor(a[2], "w");
        groups = groups_of(w, D, "w");
        shape = w.sizes().vec();
        wp = (const float *)dev(w, kF32, shape, "w", x);
    }
    if (rows % groups) raise(PyExc_ValueError, "x: " + std::to_string(rows) + " rows in " + std::to_string(groups) + " groups");
    const float eps = real(a[3]);
    Tensor dx = empty(x.sizes(), st, x), dw, db;
    Ws w;
    if (truth(a[4])) {
        dw = empty(shape, kF32, x);
        db = empty(shape, kF32, x);
        w = workspace(a[5], none(a[5]) ? dig_layernorm_bwd_workspace_bytes(rows, groups, D) : 0, x);
    }
    void *dxp = dx.data_ptr(), *s = on.stream();
    float *dwp = dw.defined() ? (float *)dw.data_ptr() : nullptr, *dbp = db.defined() ? (float *)db.data_ptr() : nullptr;
    CALL(dig_layernorm_bwd(xp, gp, wp, dxp, dwp, dbp, rows, groups, D, eps, dtype, w.p, w.n, s), "dig_layernorm_bwd");
    return pack({dx, dw, db});
}

template <PyObject *(*F)(PyObject *const *), int N>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "need %d arguments, got %zd", N, n);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const Raised &) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

PyObject *set_error(PyObject *, PyObject *cls)
{
    Py_XSETREF(g_error, Py_NewRef(cls));
    Py_RETURN_NONE;
}

#define FAST(name, n) {#name, (PyCFunction)(void (*)(void))entry<name, n>, METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {
    {"set_error", set_error, METH_O, nullptr},
    FAST(gate_logsigmoid, 3), FAST(gla_fwd, 11), FAST(gla_bwd, 12), FAST(gla_fwd_state, 12), FAST(gla_bwd_state, 13),
    FAST(gla_fwd_multi, 11), FAST(gla_bwd_multi, 12), FAST(gla_fwd_beta, 11), FAST(gla_bwd_beta, 12), FAST(gla_fwd_outgate, 15),
    FAST(outgate_fwd, 6), FAST(outgate_bwd, 9), FAST(dwconv, 8), FAST(dwconv_bwd, 9),
    FAST(decay_fwd, 12), FAST(decay_bwd, 14), FAST(decay_step, 6), FAST(rope, 8), FAST(layernorm_fwd, 4), FAST(layernorm_bwd, 6),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&kModule); }
